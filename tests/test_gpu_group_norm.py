"""Group norm with activation on the GPU against its definition in 64 bits."""
import numpy as np
import pytest

from paper_1907_03329_amd import layers

pytestmark = pytest.mark.gpu

EPS = 1e-5
# Largest difference over the largest value of the array.  Results are rounded once (24, 8, 11 significant bits: at most 2^-24, 2^-8,
# 2^-11 of them).  Before that fp32 sums of n terms in pieces (errors of some 2^-24 of the sum of magnitudes, for a mean against values of
# its own size), a square root, a division, a sigmoid: 1e-5 of the largest value.  Sums over all positions (grad_scale, grad_shift)
# add up terms of both signs, so their error is measured against the sum of magnitudes.
ROUNDING = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
ARITHMETIC = 1e-5


def definition(x, scale, shift, G, act, lengths, d=None):
    """float64 numpy, sample by sample."""
    N, T, C = x.shape
    y, dx, dscale, dshift, most = np.zeros_like(x), np.zeros_like(x), np.zeros(C), np.zeros(C), [np.zeros(C), np.zeros(C)]
    for n, length in enumerate(lengths):
        if length == 0:
            continue
        part = x[n, :length].reshape(length, G, C // G)
        mean, var = part.mean((0, 2), keepdims=True), part.var((0, 2), keepdims=True)
        rstd = 1.0 / np.sqrt(var + EPS)
        xhat = ((part - mean) * rstd).reshape(length, C)
        u = xhat * scale + shift
        p = 1.0 / (1.0 + np.exp(-u)) if act == "silu" else np.ones_like(u)
        y[n, :length] = u * p
        if d is None:
            continue
        du = d[n, :length] * (p + u * p * (1 - p) if act == "silu" else 1.0)
        dshift += du.sum(0)
        dscale += (du * xhat).sum(0)
        most[0] += np.abs(du).sum(0)
        most[1] += np.abs(du * xhat).sum(0)
        t, xg = (du * scale).reshape(length, G, C // G), xhat.reshape(length, G, C // G)
        dx[n, :length] = (rstd * (t - t.mean((0, 2), keepdims=True) - xg * (t * xg).mean((0, 2), keepdims=True))).reshape(length, C)
    return (y, dx, dscale, dshift, most) if d is not None else y


def close(got, want, dtype, what, most=None):
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all(), what
    scale = np.abs(want).max() if most is None else most.max()
    assert np.abs(got - want).max() <= (ROUNDING[dtype] + ARITHMETIC) * scale, (what, np.abs(got - want).max(), scale)


def check(N, T, C, G, dtype="float32", act="silu", lengths=None, mean=0.3, seed=0, off=0):
    import torch
    rng = np.random.default_rng(seed)
    dt = getattr(torch, dtype)
    host = [torch.from_numpy(rng.normal(m, 1.2, size=(N, T, C))).to(dt) for m in (mean, 0.0)]
    ref = [t.double().numpy() for t in host]
    if isinstance(lengths, str):
        lengths = rng.integers(0, T + 1, N)
        lengths[rng.integers(N)] = T
        if N > 1:
            lengths[np.flatnonzero(lengths < T)[:1]] = 0
    n = np.full(N, T) if lengths is None else np.asarray(lengths)
    for i in range(N):      # what lies past a length must not matter
        for t in host:
            t[i, n[i]:] = float("nan") if i % 2 else float("inf")
    def place(t):           # `off`: elements by which an array misses the place that wide accesses like
        flat = torch.zeros(t.numel() + off, dtype=t.dtype, device="cuda")
        flat[off:].copy_(t.reshape(-1))
        return flat[off:].view(t.shape)
    x, d = (place(t) for t in host)
    scale, shift = (torch.from_numpy(rng.normal(m, 0.2, size=C)).float() for m in (1.0, 0.0))
    layer = layers.GroupNorm(N, T, C, G, activation=act, eps=EPS, dtype=dt)
    for t in (layer.out, layer.stats, layer.grad_x, layer.grad_scale, layer.grad_shift):
        t.fill_(float("nan"))
    layer.workspace.fill_(255)
    lens = None if lengths is None else torch.from_numpy(n.astype(np.int32)).cuda()
    given = x, place(scale), place(shift)
    out = layer.forward(*given, lengths=lens)
    grads = layer.backward(*given, d, lengths=lens)
    want = definition(ref[0], scale.double().numpy(), shift.double().numpy(), G, act, n, ref[1])
    what = (N, T, C, G, dtype, act)
    close(out, want[0], dtype, ("out",) + what)
    close(grads[0], want[1], dtype, ("grad_x",) + what)
    close(grads[1], want[2], "float32", ("grad_scale",) + what, want[4][1])
    close(grads[2], want[3], "float32", ("grad_shift",) + what, want[4][0])
    for i in range(N):
        assert not out[i, n[i]:].any() and not grads[0][i, n[i]:].any()
    plain = layers.GroupNorm(N, T, C, G, activation=act, eps=EPS, dtype=dt, training=False)
    assert torch.equal(plain.forward(*given, lengths=lens), out)
    return layer, given + (d, lens), (out,) + grads


@pytest.mark.parametrize("T", [1, 2, 3, 15, 16, 17, 72, 255, 256, 257, 1025, 3000])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_positions(T, dtype):
    check(3, T, 40, 4, dtype=dtype, seed=T)


@pytest.mark.parametrize("C,G", [(1, 1), (2, 2), (3, 1), (16, 16), (18, 2), (37, 1), (74, 2), (96, 32), (130, 13), (256, 32), (320, 32), (1000, 4),
                                 (1026, 2), (2048, 1), (4096, 4), (5000, 1)])
@pytest.mark.parametrize("T", [1, 9, 600])
def test_channels_and_groups(C, G, T):
    check(2, T, C, G, dtype="float16" if C % 2 else "float32", act="none" if C % 4 else "silu", seed=C + T)


@pytest.mark.parametrize("N,C,G", [(1, 64, 4), (5, 16, 1), (63, 48, 2), (1000, 40, 4), (3000, 512, 32), (777, 2048, 16), (100, 1000, 8), (130, 36, 36),
                                   (70, 999, 27), (300, 1536, 12), (65, 4096, 32), (40, 2050, 5)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_every_position_by_itself(N, C, G, dtype):
    check(N, 1, C, G, dtype=dtype, seed=N)
    check(N, 1, C, G, dtype=dtype, act="none", lengths=(np.arange(N) % 3 > 0).astype(int), seed=N + 1)


@pytest.mark.parametrize("N,T,C,G", [(2050, 5, 60, 3), (2048, 16, 64, 64), (700, 16, 200, 8), (2100, 2, 37, 1), (600, 4, 1000, 4), (600, 3, 1026, 6)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_many_short_samples(N, T, C, G, dtype):
    check(N, T, C, G, dtype=dtype, seed=C)
    check(N, T, C, G, dtype=dtype, act="none", lengths="ragged", seed=C + 1)


@pytest.mark.parametrize("T,C,G", [(50, 40, 4), (700, 96, 8), (2500, 64, 2), (9, 37, 1)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_ragged_lengths_with_garbage_behind_them(T, C, G, dtype):
    check(9, T, C, G, dtype=dtype, lengths="ragged", seed=T)
    check(3, T, C, G, dtype=dtype, lengths=[0, 1, 0], act="none", seed=T + 1)


def test_all_samples_empty():
    _, _, results = check(2, 30, 16, 4, lengths=[0, 0])
    assert not any(t.any() for t in results)


@pytest.mark.parametrize("off", [1, 2, 3])
@pytest.mark.parametrize("N,T", [(2, 100), (20, 1), (2, 2000)])
def test_arrays_that_wide_accesses_miss(off, N, T):
    check(N, T, 64, 4, dtype="bfloat16", off=off, seed=off)
    check(N, T, 64, 4, off=off, seed=off)


@pytest.mark.parametrize("N,T", [(2, 200), (40, 1), (2, 5000)])
def test_far_from_zero(N, T):
    """Mean 1000, deviation 1.2.  The values are fp32 numbers with a spacing of 6e-5, of which the mean keeps a part in 2^24 or so: an error
    of 1e-4 of a deviation, to which the output is proportional.  Sums of squares minus squared sums would be off by 0.1 or more."""
    import torch
    rng = np.random.default_rng(N)
    x = torch.from_numpy(rng.normal(1000.0, 1.2, size=(N, T, 64))).float()
    layer = layers.GroupNorm(N, T, 64, 2, activation="none", eps=EPS)
    out = layer.forward(x.cuda(), torch.ones(64, device="cuda"), torch.zeros(64, device="cuda"))
    want = definition(x.double().numpy(), np.ones(64), np.zeros(64), 2, "none", [T] * N)
    assert np.abs(out.double().cpu().numpy() - want).max() <= 2e-4 * np.abs(want).max()


@pytest.mark.parametrize("N,T", [(2, 40), (9, 1), (1, 3000)])
def test_constant_groups(N, T):
    """No variance: the normalised value is zero, the gradient that of a division by sqrt(eps)."""
    import torch
    x = torch.full((N, T, 32), 2.5, device="cuda")
    layer = layers.GroupNorm(N, T, 32, 4, eps=EPS)
    shift = torch.linspace(-1, 1, 32, device="cuda")
    out = layer.forward(x, torch.ones(32, device="cuda"), shift)
    want = shift * torch.sigmoid(shift)
    assert float((out - want).abs().max()) <= 1e-6
    assert all(t.isfinite().all() for t in layer.backward(x, torch.ones(32, device="cuda"), shift, x))


@pytest.mark.parametrize("N,T,C,G", [(2, 33, 12, 3), (6, 1, 24, 2), (1, 1500, 8, 2)])
def test_gradients_against_differences(N, T, C, G):
    import torch
    layer, (x, scale, shift, d, _), (_, gx, gs, gb) = check(N, T, C, G, seed=5)
    grads = gx.clone(), gs.clone(), gb.clone()
    value = lambda: float((layer.forward(x, scale, shift).double() * d.double()).sum())  # noqa: E731
    rng = np.random.default_rng(6)
    for t, grad in zip((x, scale, shift), grads):
        for _ in range(6):
            at = tuple(int(rng.integers(n)) for n in t.shape)
            step, old = 1e-2, float(t[at])
            t[at] = old + step
            up = value()
            t[at] = old - step
            down = value()
            t[at] = old
            # truncation: step^2 / 6 of a third derivative, of the size of the gradient; rounding: 6e-8 of outputs of up to 4 and gradients of
            # up to 5 in N T C terms of random sign, over 2e-2
            rounding = 6e-8 * 20 * (N * T * C) ** 0.5 / 2e-2
            assert abs((up - down) / (2 * step) - float(grad[at])) <= 1e-3 * max(1.0, float(grad.abs().max())) + rounding


@pytest.mark.parametrize("N,T,C,G", [(3, 70, 64, 8), (500, 1, 256, 4), (2, 4000, 64, 8)])
def test_equal_calls_are_equal_and_streams_and_graphs_do_not_matter(N, T, C, G):
    import torch
    layer, (x, scale, shift, d, lens), results = check(N, T, C, G, dtype="bfloat16", lengths="ragged", seed=11)
    want = [t.clone() for t in results]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    layer.forward(x, scale, shift, lengths=lens, stream=side)
    layer.backward(x, scale, shift, d, lengths=lens, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(results, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        layer.forward(x, scale, shift, lengths=lens)
        layer.backward(x, scale, shift, d, lengths=lens)
    for replay in range(3):
        scale.mul_(1.25)
        layer.forward(x, scale, shift, lengths=lens)
        layer.backward(x, scale, shift, d, lengths=lens)
        eager = [t.clone() for t in results]
        for t in results:
            t.zero_()
        layer.workspace.fill_(replay)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results, eager))


def test_refusals():
    import torch
    from paper_1907_03329_amd.binding import EsrnnError
    for args in ((2, 5, 8, 3), (0, 5, 8, 2), (2, 0, 8, 2), (2, 5, 0, 1), (2, 5, 8, 0)):
        with pytest.raises(EsrnnError) as e:
            layers.GroupNorm(*args)
        assert e.value.status == 2
    with pytest.raises(EsrnnError):
        layers.GroupNorm(2, 5, 8, 2, eps=0.0)
    with pytest.raises(ValueError):
        layers.GroupNorm(2, 5, 8, 2, activation="other")
    layer = layers.GroupNorm(2, 5, 8, 2)
    x, p = torch.zeros(2, 5, 8, device="cuda"), torch.zeros(8, device="cuda")
    with pytest.raises(EsrnnError) as e:
        layer.backward(x, p, p, x)
    assert e.value.status == 4
    for bad in (x[:1], x.half(), x.cpu(), torch.zeros(2, 8, 5, device="cuda").transpose(1, 2)):
        with pytest.raises(ValueError):
            layer.forward(bad, p, p)
    with pytest.raises(ValueError):
        layer.forward(x, p[:4], p)
    with pytest.raises(ValueError):
        layer.forward(x, p, p, lengths=torch.zeros(2, device="cuda"))
