"""Selective scan on the GPU against its definition, position by position in 64 bits."""
import numpy as np
import pytest

from paper_1907_03329_amd import state_space
from tests.state_space_common import Given, close, ragged, scan

pytestmark = pytest.mark.gpu

# fp32 arithmetic before the rounding of a result, relative to the largest value of the array.  A step size is off by some 2^-22 of itself, the exponent
# d A of a decay by 2^-23 of itself more, so a state that remembers m positions, d A m about 1, by some 2^-21 of its size from its decays and by
# sqrt(m) 2^-24 from its additions; an output adds N such states.  The reverse pass adds as much again, sums over channels and states as many
# roundings as terms at most, 2^-24 each: 3e-5 has room for all of it, and a dropped or doubled term is off by 1e-3 or more.
ARITHMETIC = 3e-5
NAMES = ("out", "last", "grad_x", "grad_delta", "grad_A", "grad_b", "grad_c", "grad_D", "grad_bias", "grad_initial")
ELEMENTS = {"out", "grad_x", "grad_delta", "grad_b", "grad_c"}


def check(B, T, C, N=16, groups=1, dtype="float32", kind="softplus", time_major=False, lengths=None, initial=False, layout="plain", D=True, bias=True,
          own_places=False, seed=0):
    import torch
    rng = np.random.default_rng(seed)
    n = ragged(rng, B, T) if isinstance(lengths, str) else np.full(B, T) if lengths is None else np.asarray(lengths)
    g = Given(rng, B, T, dtype, time_major, None if lengths is None else n, layout)
    x, x64 = g.rows(C)
    delta, delta64 = g.rows(C, loc=-2.0) if kind == "softplus" else g.rows(C, loc=0.2, sd=0.05)
    b, b64 = g.rows(groups, N)
    c, c64 = g.rows(groups, N)
    d, d64 = g.rows(C)
    A = -(rng.uniform(0.2, 1.0, size=(C, N)) * np.arange(1, N + 1))
    A, A64 = torch.from_numpy(A).float().cuda(), torch.from_numpy(A).float().double().numpy()
    Dt, D64 = g.floats(C) if D else (None, np.zeros(C))
    bt, bias64 = g.floats(C, sd=0.3 if kind == "softplus" else 0.01) if bias else (None, np.zeros(C))
    h0, h64 = g.floats(B, C, N) if initial else (None, np.zeros((B, C, N)))
    dl, dl64 = g.floats(B, C, N) if initial else (None, np.zeros((B, C, N)))
    layer = state_space.SelectiveScan(B, T, C, N, groups=groups, delta_kind=kind, dtype=g.dt, time_major=time_major)
    for t in (layer.out, layer.last, layer.saved, layer.grad_x, layer.grad_delta, layer.grad_A, layer.grad_b, layer.grad_c, layer.grad_D, layer.grad_bias,
              layer.grad_initial):
        t.fill_(float("nan"))
    layer.workspace.fill_(255)
    lens = None if lengths is None else torch.from_numpy(n.astype(np.int32)).cuda()
    operands, given = (x, delta, A, b, c), dict(D=Dt, bias=bt, lengths=lens)
    out, last = layer.forward(*operands, initial=h0, **given)
    places = [g.places(C), g.places(C), g.places(groups, N), g.places(groups, N)] if own_places else []
    into = dict(zip(("grad_x", "grad_delta", "grad_b", "grad_c"), (p for p, _ in places)))
    grads = layer.backward(*operands, d, grad_last=dl, **given, **into)
    want = scan(x64, delta64, A64, b64, c64, D64, bias64, h64, n, kind, d64, dl64)
    what = (B, T, C, N, groups, dtype, kind, time_major, layout)
    for name, got, expected in zip(NAMES, (out, last, *grads), want):
        element = name in ELEMENTS
        close(g.turn(got) if element else got, expected, dtype if element else "float32", ARITHMETIC, (name,) + what)
        if element and lengths is not None:
            for i in range(B):
                assert not g.turn(got)[i, n[i]:].any(), (name,) + what
    assert all(untouched() for _, untouched in places), what
    return layer, (operands, d, given, h0, dl), (out, last, *grads)


@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 15, 16, 17, 23, 24, 25, 31, 33, 64, 65, 129, 257, 515])
def test_lengths_around_every_piece(T):
    check(2, T, 68, initial=True, seed=T)


@pytest.mark.parametrize("N", [1, 2, 3, 4, 5, 7, 8, 9, 12, 15, 16, 17, 24, 31, 32, 33, 47, 64])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_states(N, dtype):
    check(2, 37, 66, N, dtype=dtype, initial=True, lengths="ragged", seed=N)


@pytest.mark.parametrize("C,groups", [(1, 1), (2, 2), (5, 1), (63, 1), (64, 1), (65, 1), (66, 2), (128, 2), (129, 3), (200, 1), (260, 4), (130, 130)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_channels_and_groups(C, groups, dtype):
    check(2, 21, C, 16, groups, dtype=dtype, initial=True, seed=C)
    check(2, 21, C, 5, groups, dtype=dtype, seed=C + 1)


@pytest.mark.parametrize("layout", ["plain", "gaps", "slices"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("time_major", [False, True])
def test_strides_lengths_and_places(layout, dtype, time_major):
    check(7, 43, 50, 8, 2, dtype=dtype, time_major=time_major, lengths="ragged", initial=True, layout=layout, own_places=True, seed=5)
    check(3, 43, 50, 16, 1, dtype=dtype, time_major=time_major, lengths="ragged", initial=True, layout=layout, seed=6)


@pytest.mark.parametrize("lengths", [[0, 0, 0], [1, 0, 2], [0, 40, 8], [16, 17, 24]])
@pytest.mark.parametrize("N", [16, 20])
def test_short_and_empty_sequences(lengths, N):
    check(3, 40, 66, N, lengths=lengths, initial=True, seed=1)


@pytest.mark.parametrize("N,C,groups", [(6, 140, 1), (33, 140, 1), (40, 300, 2), (64, 66, 1)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_gradients_of_several_tiles_at_odd_places(N, C, groups, dtype):
    """States that are no whole fours or slices, gradients with gaps between their rows, and positions past the lengths."""
    check(3, 29, C, N, groups, dtype=dtype, lengths=[29, 0, 18], initial=True, layout="gaps", own_places=True, seed=9)


@pytest.mark.parametrize("kind", ["softplus", "given"])
@pytest.mark.parametrize("D,bias", [(True, False), (False, True), (False, False)])
def test_operands_that_are_left_out(kind, D, bias):
    check(3, 30, 70, kind=kind, D=D, bias=bias, seed=2)


def test_many_lines_and_segments():
    """From one segment for each sequence to as many as there are, ragged across their ends."""
    check(600, 19, 50, 4, lengths="ragged", initial=True, seed=3)
    check(1, 3000, 64, 4, dtype="bfloat16", initial=True, seed=4)
    check(2, 1100, 20, 16, lengths=[1100, 497], initial=True, seed=5)
    check(1, 1000, 30, 40, lengths=[777], initial=True, seed=6)


@pytest.mark.parametrize("T,C,N,groups,lengths", [(2000, 64, 16, 1, None), (3000, 140, 8, 2, None), (2600, 9, 20, 1, [1500, 2600]), (12000, 20, 4, 1, None),
                                                  (12000, 70, 16, 1, [11003])])
def test_segments_by_the_hundred(T, C, N, groups, lengths):
    """Maps of many segments are put together by a launch of their own, in runs of neighbours, ends of sequences among them."""
    check(len(lengths or [0]), T, C, N, groups, lengths=lengths, initial=True, seed=7)


def test_step_sizes_from_nothing_to_large():
    """softplus from where it is e^v to where it is v, element by element, as the output of one position that begins at zero: d b c x."""
    import torch
    v = torch.cat([torch.linspace(-85, -10, 300), torch.linspace(-10, 10, 801), torch.linspace(10, 85, 200)])
    C = v.numel()
    one = torch.ones(1, 1, 1, 1, device="cuda")
    layer = state_space.SelectiveScan(1, 1, C, 1)
    x = torch.ones(1, 1, C, device="cuda")
    out, _ = layer.forward(x, v.view(1, 1, C).cuda(), -torch.ones(C, 1, device="cuda"), one, one)
    want = np.logaddexp(v.double().numpy(), 0.0)
    # exp(-|v|): the exponent |v| log2 e is one rounded product, |v| 2^-24 of it, and the power a unit in the last place; the series, a reciprocal and the
    # last sums some units more
    room = (np.abs(v.double().numpy()) * 2.0 ** -24 + 8 * 2.0 ** -24) * want
    assert (np.abs(out.double().cpu().numpy()[0, 0] - want) <= room).all()


def test_gradients_by_differences():
    """The sum of out times its gradient changes with every operand as the gradients say."""
    import torch
    layer, (operands, d, given, h0, dl), results = check(2, 21, 24, 6, 2, initial=True, seed=8)
    grads = dict(zip(("x", "delta", "A", "b", "c", "D", "bias", "h0"), (t.clone() for t in results[2:])))
    args = dict(zip(("x", "delta", "A", "b", "c"), operands)) | {"D": given["D"], "bias": given["bias"], "h0": h0}

    def value(x, delta, A, b, c, D, bias, h0):
        out, last = layer.forward(x, delta, A, b, c, D=D, bias=bias, initial=h0)
        return float((out.double() * d.double()).sum() + (last.double() * dl.double()).sum())

    eps = 1e-2
    torch.manual_seed(0)
    for which, grad in grads.items():
        dirs = torch.randn_like(grad)
        up, down = ({**args, which: args[which] + s * eps * dirs} for s in (1, -1))
        got, want = (value(**up) - value(**down)) / (2 * eps), float((grad.double() * dirs.double()).sum())
        # (third order: eps^2 times third derivatives of values of one size; fp32 sums 2^-20 / eps)
        assert abs(got - want) <= 5e-3 * float((grad.double() * dirs.double()).abs().sum()), which


def test_sequences_in_pieces_and_position_by_position():
    """A sequence cut in two with the state handed over, by the layer's own `last` too, and position by position."""
    import torch
    torch.manual_seed(1)
    B, T, C, N, G = 5, 24, 48, 16, 2
    dt = torch.bfloat16
    x, delta, b, c = (torch.randn(*s, device="cuda").to(dt) for s in ((B, T, C), (B, T, C), (B, T, G, N), (B, T, G, N)))
    A, D, bias = -torch.rand(C, N, device="cuda"), torch.randn(C, device="cuda"), torch.randn(C, device="cuda") - 2.0
    whole = state_space.SelectiveScan(B, T, C, N, G, dtype=dt, training=False)
    out, last = (t.clone() for t in whole.forward(x, delta, A, b, c, D, bias))
    half = state_space.SelectiveScan(B, T // 2, C, N, G, dtype=dt, training=False)
    cut = lambda i: [t[:, i * T // 2:(i + 1) * T // 2] for t in (x, delta)] + [A] + [t[:, i * T // 2:(i + 1) * T // 2] for t in (b, c)]  # noqa: E731
    first, carried = half.forward(*cut(0), D, bias)
    first = first.clone()
    second, end = half.forward(*cut(1), D, bias, initial=carried)
    scale = float(last.abs().max())
    close(torch.cat([first, second], 1), out.double().cpu().numpy(), "bfloat16", 2.0 ** -8)
    assert float((end - last).abs().max()) <= ARITHMETIC * scale
    pool = torch.full((9, C, N), 3.0, device="cuda")
    slots = torch.tensor([4, 0, 8, 2, 5], dtype=torch.int32, device="cuda")
    pool[slots.long()] = 0.0
    one = torch.empty(B, C, dtype=dt, device="cuda")
    for t in range(T):
        state_space.selective_step(x[:, t], delta[:, t], A, b[:, t], c[:, t], pool, one, D, bias, slots)
        close(one, out[:, t].double().cpu().numpy(), "bfloat16", 2.0 ** -8, t)
    assert float((pool[slots.long()] - last).abs().max()) <= ARITHMETIC * scale
    rest = [i for i in range(9) if i not in slots.tolist()]
    assert bool((pool[rest] == 3.0).all())


@pytest.mark.parametrize("N", [1, 3, 4, 7, 8, 13, 16, 20, 32, 50, 64])
@pytest.mark.parametrize("dtype,C,groups", [("float32", 50, 1), ("bfloat16", 130, 2), ("float16", 7, 7), ("bfloat16", 1, 1)])
@pytest.mark.parametrize("kind", ["softplus", "given"])
def test_single_positions(N, dtype, C, groups, kind):
    import torch
    rng = np.random.default_rng(C + N)
    dt, rows, pool = getattr(torch, dtype), 6, 8
    make = lambda *size, loc=0.0, sd=1.0: torch.from_numpy(rng.normal(loc, sd, size=size))  # noqa: E731
    both = make(rows, 3 * C + 2).to(dt).cuda()
    x, delta = both[:, 1:C + 1], both[:, C + 1:2 * C + 1]
    shared = make(rows, 2 * groups * N + 1).to(dt).cuda()
    b, c = (shared[:, 1 + i * groups * N:1 + (i + 1) * groups * N].unflatten(1, (groups, N)) for i in (0, 1))
    A, D, bias = -make(C, N).abs().float().cuda(), make(C).float().cuda(), make(C, loc=1.0).float().cuda()
    state = make(pool, C, N).float().cuda()
    slots = torch.tensor([7, -1, 0, 3, 8, 5], dtype=torch.int32, device="cuda")
    out = torch.full((rows, C + 2), 7.0, dtype=dt, device="cuda")
    before = state.clone()
    state_space.selective_step(x, delta, A, b, c, state, out[:, 1:C + 1], D, bias, slots, delta_kind=kind)
    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    h0 = f(before)[np.clip(slots.cpu().numpy(), 0, pool - 1)]
    want, h = scan(f(x)[:, None], f(delta)[:, None], f(A), f(b)[:, None], f(c)[:, None], f(D), f(bias), h0, np.ones(rows), kind)
    want, expect = want[:, 0], f(before)
    want[[1, 4]] = 0.0
    for i, s in enumerate(slots.tolist()):
        if 0 <= s < pool:
            expect[s] = h[i]
    close(out[:, 1:C + 1], want, dtype, ARITHMETIC)
    close(state, expect, "float32", ARITHMETIC)
    assert bool((out[:, 0] == 7).all()) and bool((out[:, C + 1] == 7).all())
    untouched = [i for i in range(pool) if i not in slots.tolist()]
    assert torch.equal(state[untouched], before[untouched])


def test_infinite_step_sizes_and_states():
    """A step of infinite size forgets everything: exp(-inf) is 0, with x = 0 nothing is taken in either way round; other channels do not see it."""
    import torch
    x, delta = torch.zeros(1, 9, 70, device="cuda"), torch.zeros(1, 9, 70, device="cuda")
    delta[0, 4, 3] = 1e30
    b = torch.ones(1, 9, 1, 4, device="cuda")
    h0 = torch.ones(1, 70, 4, device="cuda")
    layer = state_space.SelectiveScan(1, 9, 70, 4)
    out, last = layer.forward(x, delta, -torch.ones(70, 4, device="cuda"), b, b, initial=h0)
    assert bool((last[0, 3] == 0).all()) and bool((out[0, 4:, 3] == 0).all()) and bool((out[0, :, 4] > 0).all())
    assert bool(torch.isfinite(out).all())


def test_two_streams_graphs_and_equal_calls():
    import torch
    layer, (operands, d, given, h0, dl), _ = check(4, 300, 70, lengths="ragged", initial=True, seed=9)
    other = state_space.SelectiveScan(4, 300, 70, 16)
    run = lambda l, s=None: (*l.forward(*operands, initial=h0, stream=s, **given), *l.backward(*operands, d, grad_last=dl, stream=s, **given))  # noqa: E731
    eager = [t.clone() for t in run(layer)]
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        got = {s: run(l, s) for s, l in ((a, layer), (b, other))}
    torch.cuda.synchronize()
    for g in got.values():
        assert all(torch.equal(p, q) for p, q in zip(g, eager))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        results = run(layer)
    for _ in range(3):
        for t in results:
            t.fill_(float("nan"))
        other.forward(*operands, **given)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(results, eager))


@pytest.mark.parametrize("B,T,C,N", [(300, 72, 40, 16), (300, 40, 64, 8), (4, 130, 64, 16), (257, 9, 60, 3), (20, 200, 130, 16), (600, 33, 40, 16), (1, 128, 64, 16), (1, 129, 64, 16)])
def test_short_sequences_and_many_lines(B, T, C, N):
    """Sizes at which a line is a workgroup, of one block of pieces and of several, and some beside them."""
    check(B, T, C, N, lengths="ragged", initial=True, seed=T)
    check(B, T, C, N, dtype="bfloat16", D=False, seed=T + 1)


@pytest.mark.parametrize("T", [13, 16, 700])
def test_infinite_rates_of_decay(T):
    """A state that forgets everything at every position: what it takes in, exactly, at lengths that end inside a piece too; other states do not see it."""
    import torch
    torch.manual_seed(0)
    B, C, N = 2, 70, 4
    x, delta, d = (torch.randn(B, T, C, device="cuda") for _ in range(3))
    b, c = torch.randn(B, T, 1, N, device="cuda"), torch.randn(B, T, 1, N, device="cuda")
    A = -torch.rand(C, N, device="cuda")
    A[:, 2] = -float("inf")
    n = torch.tensor([T, T - 5], dtype=torch.int32, device="cuda")
    h0 = torch.randn(B, C, N, device="cuda")
    layer = state_space.SelectiveScan(B, T, C, N)
    out, last = layer.forward(x, delta, A, b, c, lengths=n, initial=h0)
    step = torch.nn.functional.softplus(delta.double())
    for i, k in enumerate(n.tolist()):
        want = (step[i, k - 1] * x[i, k - 1].double() * b[i, k - 1, 0, 2].double())
        assert float((last[i, :, 2].double() - want).abs().max()) <= 1e-6 * float(want.abs().max())
    grads = layer.backward(x, delta, A, b, c, d, lengths=n)
    assert all(bool(torch.isfinite(t).all()) for t in (out, last, *grads))
    assert not grads[-1][:, :, 2].any() and not grads[2][:, 2].any()


def test_a_batch_beyond_32_bits():
    """Two sequences 2.2e9 elements apart in x, delta and their gradients; states of b and c too."""
    import torch
    torch.manual_seed(0)
    T, C, N = 20, 64, 16
    far = 2_200_000_000
    x, delta, d, b, c = (torch.randn(2, T, n, device="cuda").half() for n in (C, C, C, N, N))
    A = -torch.rand(C, N, device="cuda")
    layer = state_space.SelectiveScan(2, T, C, N, dtype=torch.float16)
    want = [t.clone() for t in (*layer.forward(x, delta, A, b[:, :, None], c[:, :, None]), *layer.backward(x, delta, A, b[:, :, None], c[:, :, None], d))]
    big = torch.empty(far + 20000, dtype=torch.float16, device="cuda")
    at, views = 0, []
    for t in (x, delta, d, b, c, x, delta, b, c):
        v = big.as_strided(t.shape, (far, t.shape[2], 1), at)
        views.append(v)
        at += T * t.shape[2]
    for v, t in zip(views, (x, delta, d, b, c)):
        v.copy_(t)
    xs, ds, dd, bs, cs, gx, gd, gb, gc = views
    operands = (xs, ds, A, bs[:, :, None], cs[:, :, None])
    got = (*layer.forward(*operands), *layer.backward(*operands, dd, grad_x=gx, grad_delta=gd, grad_b=gb[:, :, None], grad_c=gc[:, :, None]))
    assert all(torch.equal(p.reshape(q.shape), q) for p, q in zip(got, want))


def test_pools_beyond_32_bits():
    import torch
    C, N, pool = 1024, 16, 140_000         # 2.3e9 states
    state = torch.zeros(pool, C, N, device="cuda")
    torch.manual_seed(0)
    x, delta, b, c = (torch.randn(3, *s, device="cuda") for s in ((C,), (C,), (1, N), (1, N)))
    A, out, near = -torch.rand(C, N, device="cuda"), torch.empty(3, C, device="cuda"), torch.zeros(3, C, N, device="cuda")
    slots = torch.tensor([pool - 1, 0, 131_073], dtype=torch.int32, device="cuda")
    for _ in range(2):
        state_space.selective_step(x, delta, A, b, c, state, out, slots=slots)
        one = out.clone()
        state_space.selective_step(x, delta, A, b, c, near, out)
    assert torch.equal(one, out) and torch.equal(state[slots.long()], near) and int((state != 0).any(2).any(1).sum()) == 3
