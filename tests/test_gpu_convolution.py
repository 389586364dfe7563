"""Short causal convolution on the GPU against its definition, position by position in 64 bits."""
import numpy as np
import pytest

from paper_1907_03329_amd import state_space
from tests.state_space_common import Given, close, convolution, ragged, silu

pytestmark = pytest.mark.gpu

# fp32 arithmetic before the rounding of a result.  An output is a sum of at most nine terms, each product and sum rounded to 2^-24 of the largest partial
# sum, then a sigmoid that is off by a few 2^-24, and silu's derivative is at most 1.1: below 2^-18 of the largest output or input gradient, for
# values of one size.  Gradients of weights are sums over positions: rounded at every addition, at most one for each of the run's and
# workgroups' positions, here some 2^-24 sqrt(positions), far below 2^-16 of the sum of magnitudes.
ARITHMETIC, SUMS = 2.0 ** -18, 2.0 ** -16


def check(B, T, C, K=4, act="silu", dtype="float32", time_major=False, lengths=None, initial=False, layout="plain", bias=True, own_places=False, seed=0):
    import torch
    rng = np.random.default_rng(seed)
    n = ragged(rng, B, T) if isinstance(lengths, str) else np.full(B, T) if lengths is None else np.asarray(lengths)
    g = Given(rng, B, T, dtype, time_major, None if lengths is None else n, layout)
    x, x64 = g.rows(C)
    d, d64 = g.rows(C)
    w, w64 = g.floats(C, K, sd=0.5)
    c, c64 = g.floats(C, sd=0.3) if bias else (None, np.zeros(C))
    first = torch.from_numpy(rng.normal(size=(B, K - 1, C))).to(g.dt) if initial else torch.zeros(B, K - 1, C, dtype=g.dt)
    dl, dl64 = g.floats(B, K - 1, C) if initial else (None, np.zeros((B, K - 1, C)))
    layer = state_space.ShortConvolution(B, T, C, K, activation=act, dtype=g.dt, time_major=time_major)
    for t in (layer.out, layer.last, layer.grad_x, layer.grad_weight, layer.grad_bias, layer.grad_initial):
        t.fill_(float("nan"))
    layer.workspace.fill_(255)
    lens = None if lengths is None else torch.from_numpy(n.astype(np.int32)).cuda()
    given = dict(bias=c, lengths=lens, initial=first.cuda() if initial else None)
    out, last = layer.forward(x, w, **given)
    place, untouched = g.places(C) if own_places else (None, lambda: True)
    gx, gw, gb, gi = layer.backward(x, w, d, grad_last=dl, grad_x=place, **given)
    want = convolution(x64, w64, c64, first.double().numpy(), n, act, d64, dl64)
    what = (B, T, C, K, act, dtype, time_major, layout)
    close(g.turn(out), want[0], dtype, ARITHMETIC, ("out",) + what)
    assert torch.equal(last.double().cpu(), torch.from_numpy(want[1])), ("last",) + what
    close(g.turn(gx), want[2], dtype, ARITHMETIC, ("grad_x",) + what)
    total = np.abs(d64).sum() / C + 1.0     # of the magnitudes that are added up for a channel
    close(gw, want[3], "float32", SUMS, ("grad_weight",) + what, 3.0 * total)
    close(gb, want[4], "float32", SUMS, ("grad_bias",) + what, total)
    close(gi, want[5], "float32", ARITHMETIC, ("grad_initial",) + what)
    assert untouched(), what
    if lengths is not None:
        for b in range(B):
            for t in (g.turn(out), g.turn(gx)):
                assert not t[b, n[b]:].any(), what
    return layer, (x, w, d, given, dl), (out, last, gx, gw, gb, gi)


@pytest.mark.parametrize("T", [1, 2, 3, 4, 7, 8, 9, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 255, 257, 1000])
def test_lengths_around_every_run(T):
    check(3, T, 68, initial=True, seed=T)


@pytest.mark.parametrize("K", [2, 3, 4, 5, 6, 7, 8])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_taps(K, dtype):
    check(2, 41, 72, K, dtype=dtype, initial=True, lengths="ragged", seed=K)
    check(3, K - 1, 72, K, dtype=dtype, initial=True, lengths="ragged", act="none", seed=K)


@pytest.mark.parametrize("C", [1, 2, 3, 4, 5, 7, 8, 9, 15, 16, 17, 31, 50, 63, 64, 65, 66, 67, 71, 127, 130, 200])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_channels(C, dtype):
    check(2, 37, C, dtype=dtype, initial=True, seed=C)


@pytest.mark.parametrize("layout", ["plain", "gaps", "slices"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("time_major", [False, True])
def test_strides_lengths_and_places(layout, dtype, time_major):
    check(9, 75, 50, dtype=dtype, time_major=time_major, lengths="ragged", initial=True, layout=layout, own_places=True, seed=5)


@pytest.mark.parametrize("lengths", [[0, 0, 0], [1, 0, 2], [0, 40, 3], [-5, 100, 40]])
def test_short_and_empty_sequences(lengths):
    n = np.clip(lengths, 0, 40)
    check(3, 40, 66, lengths=n, initial=True, seed=1)
    check(3, 40, 66, 8, lengths=n, initial=True, seed=2)


def test_lengths_outside_are_clamped():
    import torch
    layer = state_space.ShortConvolution(2, 10, 16)
    x, w = torch.randn(2, 10, 16, device="cuda"), torch.randn(16, 4, device="cuda")
    a = layer.forward(x, w, lengths=torch.tensor([-3, 99], dtype=torch.int32, device="cuda"))[0].clone()
    b = layer.forward(x, w, lengths=torch.tensor([0, 10], dtype=torch.int32, device="cuda"))[0]
    assert torch.equal(a, b)


def test_no_bias_many_sequences_and_long_ones():
    check(501, 30, 50, bias=False, lengths="ragged", seed=3)
    check(1, 20000, 16, dtype="bfloat16", initial=True, seed=4)
    check(2, 3000, 130, 3, act="none", seed=6)


def test_gradients_by_differences():
    """The sum of out times d changes with every operand as the gradients say."""
    import torch
    layer, (x, w, d, given, dl), (_, _, gx, gw, gb, gi) = check(2, 19, 20, 5, initial=True, lengths="ragged", seed=8)
    gx, gw, gb, gi = (t.clone() for t in (gx, gw, gb, gi))
    n = given["lengths"].tolist()
    mask = torch.zeros_like(x)
    for b, k in enumerate(n):
        mask[b, :k] = 1.0
    x = torch.where(mask > 0, x, 0.0)
    d = torch.where(mask > 0, d, 0.0)

    def value(x, w, c, first):
        out, last = layer.forward(x, w, c, lengths=given["lengths"], initial=first)
        return float((out.double() * d.double()).sum() + (last.double() * dl.double()).sum())

    eps = 1e-2      # (second order: a thousandth of the difference at most, for values of one size; fp32 sums 2^-20 / eps of it)
    for which, grad in (("x", gx), ("w", gw), ("c", gb), ("first", gi)):
        dirs = torch.randn_like(grad) * (mask if which == "x" else 1.0)
        args = {"x": x, "w": w, "c": given["bias"], "first": given["initial"]}
        up, down = ({**args, which: args[which] + s * eps * dirs} for s in (1, -1))
        got, want = (value(**up) - value(**down)) / (2 * eps), float((grad.double() * dirs.double()).sum())
        assert abs(got - want) <= 5e-3 * float((grad.double() * dirs.double()).abs().sum()), which


def test_whole_sequences_in_pieces_and_position_by_position():
    """A sequence cut in two with the window handed over, by the layer's own `last` too, and position by position: the same bits."""
    import torch
    torch.manual_seed(0)
    B, T, C, K = 5, 24, 50, 4
    x, w, c = torch.randn(B, T, C, device="cuda").bfloat16(), torch.randn(C, K, device="cuda"), torch.randn(C, device="cuda")
    whole = state_space.ShortConvolution(B, T, C, K, dtype=torch.bfloat16, training=False)
    out, last = (t.clone() for t in whole.forward(x, w, c))
    half = state_space.ShortConvolution(B, T // 2, C, K, dtype=torch.bfloat16, training=False)
    a, carried = half.forward(x[:, :T // 2], w, c)
    a = a.clone()
    b, end = half.forward(x[:, T // 2:], w, c, initial=carried)
    assert torch.equal(torch.cat([a, b], 1), out) and torch.equal(end, last)
    pool = torch.full((9, K - 1, C), 3.0, device="cuda", dtype=torch.bfloat16)
    slots = torch.tensor([4, 0, 8, 2, 5], dtype=torch.int32, device="cuda")
    pool[slots.long()] = 0.0
    one = torch.empty(B, C, dtype=torch.bfloat16, device="cuda")
    for t in range(T):
        state_space.convolution_step(x[:, t], w, pool, one, c, slots)
        close(one, out[:, t].double().cpu().numpy(), "bfloat16", 2.0 ** -20, t)
    assert torch.equal(pool[slots.long()], last)
    rest = [i for i in range(9) if i not in slots.tolist()]
    assert bool((pool[rest] == 3.0).all())


@pytest.mark.parametrize("C", [1, 3, 7, 8, 50, 1000, 2049])
@pytest.mark.parametrize("K", [2, 4, 8])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_single_positions(C, K, dtype):
    import torch
    rng = np.random.default_rng(C)
    dt, rows, pool = getattr(torch, dtype), 6, 8
    state = torch.from_numpy(rng.normal(size=(pool, K - 1, C))).to(dt).cuda()
    both = torch.from_numpy(rng.normal(size=(rows, 2 * C + 1))).to(dt).cuda()
    x, w, c = both[:, 1:C + 1], torch.from_numpy(rng.normal(size=(C, K))).float().cuda(), torch.from_numpy(rng.normal(size=C)).float().cuda()
    slots = torch.tensor([7, -1, 0, 3, 8, 5], dtype=torch.int32, device="cuda")
    out = torch.full((rows, C + 2), 7.0, dtype=dt, device="cuda")
    before = state.clone()
    state_space.convolution_step(x, w, state, out[:, 1:C + 1], c, slots)
    seen = torch.cat([before[slots.long().clamp(0, pool - 1)], x[:, None]], 1).double().cpu().numpy()
    want = silu(c.double().cpu().numpy() + np.einsum("rkc,ck->rc", seen, w.double().cpu().numpy()))[0]
    want[[1, 4]] = 0.0
    close(out[:, 1:C + 1], want, dtype, ARITHMETIC)
    assert bool((out[:, 0] == 7).all()) and bool((out[:, C + 1] == 7).all())
    expect = before.clone()
    for i, s in enumerate(slots.tolist()):
        if 0 <= s < pool:
            expect[s] = torch.cat([before[s, 1:], x[i:i + 1]])
    assert torch.equal(state, expect)


def test_infinite_outputs_stay_what_they_are():
    """x sigmoid(x) at infinities, and slopes there, in one row without touching the others."""
    import torch
    x = torch.zeros(1, 3, 8, device="cuda")
    x[0, 0, :4] = torch.tensor([float("inf"), float("-inf"), 200.0, -200.0])
    w = torch.zeros(8, 2, device="cuda")
    w[:, 1] = 1.0
    layer = state_space.ShortConvolution(1, 3, 8, 2)
    out = layer.forward(x, w)[0]
    assert float(out[0, 0, 0]) == float("inf") and out[0, 0, 1:4].tolist()[1] == 200.0 and float(out[0, 0, 3]) == 0.0 and float(out[0, 0, 1]) == 0.0


def test_two_streams_graphs_and_equal_calls():
    import torch
    layer, (x, w, d, given, dl), _ = check(4, 300, 70, lengths="ragged", initial=True, seed=9)
    other = state_space.ShortConvolution(4, 300, 70)
    eager = [t.clone() for t in (*layer.forward(x, w, **given), *layer.backward(x, w, d, grad_last=dl, **given))]
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    got = {}
    for _ in range(3):
        for s, l in ((a, layer), (b, other)):
            got[s] = (*l.forward(x, w, stream=s, **given), *l.backward(x, w, d, grad_last=dl, stream=s, **given))
    torch.cuda.synchronize()
    for g in got.values():
        assert all(torch.equal(p, q) for p, q in zip(g, eager))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        results = (*layer.forward(x, w, **given), *layer.backward(x, w, d, grad_last=dl, **given))
    for _ in range(3):
        for t in results:
            t.fill_(float("nan"))
        other.forward(x, w, **given)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(results, eager))


def test_windows_carried_from_batch_to_batch_in_training():
    """The layer's own last as the next initial: forward and reverse passes as with a copy of it; what has been overwritten since is refused."""
    import torch
    torch.manual_seed(0)
    B, T, C, K = 3, 10, 40, 4
    x, d, w = torch.randn(2, B, T, C, device="cuda").bfloat16(), torch.randn(B, T, C, device="cuda").bfloat16(), torch.randn(C, K, device="cuda")
    results = []
    for own in (True, False):
        layer = state_space.ShortConvolution(B, T, C, K, dtype=torch.bfloat16)
        last = layer.forward(x[0], w)[1]
        with pytest.raises(ValueError):
            layer.backward(x[0], w, d, initial=last)
        first = last if own else last.clone()
        out = layer.forward(x[1], w, initial=first)[0]
        grads = layer.backward(x[1], w, d, initial=first)
        again = layer.backward(x[1], w, d, initial=first, grad_last=grads[3])       # (its own grad_initial, copied before)
        results.append([t.clone() for t in (out, *grads, *again)])
    assert all(torch.equal(a, b) for a, b in zip(*results))


def test_a_batch_beyond_32_bits():
    """Two sequences 2.2e9 elements apart, and rows of one 5e8 apart."""
    import torch
    C, T = 64, 9
    w = torch.randn(C, 4, device="cuda")
    near = torch.randn(2, T, C, device="cuda").half()
    layer = state_space.ShortConvolution(2, T, C, dtype=torch.float16)
    want = [t.clone() for t in (layer.forward(near, w)[0], *layer.backward(near, w, near))]
    big = torch.empty(2 * 2_200_000_000 + 1000, dtype=torch.float16, device="cuda")
    for strides in ((2_200_000_000, C, 1), (C, 500_000_000, 1)):
        x = big.as_strided((2, T, C), strides) if strides[0] > C else big.as_strided((2, T - 1, C), strides)
        if strides[0] > C:
            x.copy_(near)
            got = (layer.forward(x, w)[0], *layer.backward(x, w, x))
            assert all(torch.equal(a, b) for a, b in zip(got, want))
        else:
            x.copy_(near[:, :T - 1])
            short = state_space.ShortConvolution(2, T - 1, C, dtype=torch.float16, training=False)
            assert torch.equal(short.forward(x, w)[0], want[0][:, :T - 1])
