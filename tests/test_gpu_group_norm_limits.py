"""Group norm on the GPU at the ends of its sizes."""
import numpy as np
import pytest

from paper_1907_03329_amd import layers
from tests.test_gpu_group_norm import ARITHMETIC, EPS, ROUNDING

pytestmark = pytest.mark.gpu


def test_more_groups_than_a_launch_has_workgroups():
    """2^24 + 192 groups of more than 512 positions: sums over groups by a workgroup of 256 threads each would be 2^32 threads.  17 GB an array, of which
    two positions of every sample exist (and all of the last sample)."""
    import torch
    N, T, C = (1 << 18) + 3, 513, 64
    free, _ = torch.cuda.mem_get_info()
    if free < 80 << 30:
        pytest.skip("needs 80 GB of device memory")
    generator = torch.Generator(device="cuda").manual_seed(3)
    x, d = (torch.empty((N, T, C), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for t in (x, d):
        t[:, :2].normal_(generator=generator)
        t[-1].normal_(generator=generator)
        t[:, 2:4] = float("nan")
        t[-1, 2:4] = 1.0
    lengths = torch.full((N,), 2, dtype=torch.int32, device="cuda")
    lengths[0], lengths[-1] = 0, T
    scale, shift = torch.linspace(0.5, 1.5, C, device="cuda"), torch.linspace(-1.0, 1.0, C, device="cuda")
    layer = layers.GroupNorm(N, T, C, C, activation="silu", eps=EPS, dtype=torch.bfloat16)
    layer.stats.fill_(float("nan"))
    out = layer.forward(x, scale, shift, lengths=lengths)
    gx, gs, gb = layer.backward(x, scale, shift, d, lengths=lengths)

    def definition(rows, length):
        f = lambda t: t[rows, :length].double()  # noqa: E731
        v = f(x)
        mean, var = v.mean(1, keepdim=True), v.var(1, unbiased=False, keepdim=True)
        rstd = 1.0 / (var + EPS).sqrt()
        xhat = (v - mean) * rstd
        u = xhat * scale + shift
        p = torch.sigmoid(u)
        du = f(d) * (p + u * p * (1 - p))
        g = du * scale
        return u * p, rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True)), du, du * xhat

    sums = [torch.zeros(2, C, dtype=torch.float64, device="cuda") for _ in range(2)]
    tolerance = ROUNDING["bfloat16"] + ARITHMETIC
    for rows, length in [(slice(k, min(k + (1 << 15), N - 1)), 2) for k in range(1, N - 1, 1 << 15)] + [(slice(N - 1, N), T)]:
        y, dx, du, along = definition(rows, length)
        assert float((out[rows, :length].double() - y).abs().max()) <= tolerance * float(y.abs().max())
        # (of two positions close to each other rstd is up to 300, and so is the gradient: against the largest of all)
        assert float((gx[rows, :length].double() - dx).abs().max()) <= tolerance * float(dx.abs().max())
        for s, v in zip(sums, (along, du)):
            s[0] += v.sum((0, 1))
            s[1] += v.abs().sum((0, 1))
    for got, s in zip((gs, gb), sums):
        assert float((got.double() - s[0]).abs().max()) <= ARITHMETIC * float(s[1].max())
    assert not out[0].any() and not gx[0].any()
    for t in (out, gx):     # zero behind the lengths
        assert not any(t[k:k + (1 << 15), 2:].any() for k in range(0, N - 1 - (1 << 15), 1 << 15))


@pytest.mark.parametrize("N,C,G", [(131072, 4096, 32), ((1 << 23) + 5, 64, 16), (600001, 8192, 2)])
def test_many_positions_by_themselves(N, C, G):
    """More samples times channels than the way for long samples takes, more than 2^25 groups, offsets beyond 2^32 elements in wide groups."""
    import torch
    free, _ = torch.cuda.mem_get_info()
    if free < 10 * N * C + (16 << 30):
        pytest.skip("needs more device memory")
    generator = torch.Generator(device="cuda").manual_seed(C)
    x, d = (torch.empty((N, 1, C), dtype=torch.bfloat16, device="cuda").normal_(generator=generator) for _ in range(2))
    scale, shift = torch.linspace(0.5, 1.5, C, device="cuda"), torch.linspace(-1.0, 1.0, C, device="cuda")
    lengths = (torch.arange(N, device="cuda") % 7 > 0).int()
    layer = layers.GroupNorm(N, 1, C, G, activation="silu", eps=EPS, dtype=torch.bfloat16)
    for t in (layer.out, layer.stats, layer.grad_x):
        t.fill_(float("nan"))
    out = layer.forward(x, scale, shift, lengths=lengths)
    gx, gs, gb = layer.backward(x, scale, shift, d, lengths=lengths)
    sums, tolerance = torch.zeros(4, C, dtype=torch.float64, device="cuda"), ROUNDING["bfloat16"] + ARITHMETIC
    rows = (1 << 26) // C
    for first in range(0, N, rows):
        at = slice(first, min(first + rows, N))
        v, exists = x[at, 0].double().unflatten(1, (G, C // G)), lengths[at].double()[:, None]
        mean, var = v.mean(2, keepdim=True), v.var(2, unbiased=False, keepdim=True)
        rstd = 1.0 / (var + EPS).sqrt()
        xhat = ((v - mean) * rstd).flatten(1)
        u = xhat * scale + shift
        p = torch.sigmoid(u)
        du = d[at, 0].double() * (p + u * p * (1 - p)) * exists
        g, xg = (du * scale).unflatten(1, (G, C // G)), xhat.unflatten(1, (G, C // G))
        dx = (rstd * (g - g.mean(2, keepdim=True) - xg * (g * xg).mean(2, keepdim=True))).flatten(1)
        for got, want in ((out, u * p * exists), (gx, dx)):
            assert float((got[at, 0].double() - want).abs().max()) <= tolerance * float(want.abs().max()), first
        along = du * xhat
        sums += torch.stack([along.sum(0), along.abs().sum(0), du.sum(0), du.abs().sum(0)])
    assert float((gs.double() - sums[0]).abs().max()) <= ARITHMETIC * float(sums[1].max())
    assert float((gb.double() - sums[2]).abs().max()) <= ARITHMETIC * float(sums[3].max())


@pytest.mark.parametrize("N,T,C,G", [(9, 1, 32, 4), (9, 1, 37, 1), (5, 1, 1024, 2), (5, 1, 2048, 1), (2, 40, 32, 4), (1, 3000, 32, 4)])
@pytest.mark.parametrize("eps", [1e-5, 1e-30, 1e-37, 1e-39, 1e-43])
def test_constant_groups_with_a_small_eps(N, T, C, G, eps):
    """No variance, so everything hangs on eps alone, which may be less than the smallest normal number."""
    import torch
    x = torch.full((N, T, C), 2.0, device="cuda")
    scale, shift = torch.linspace(0.5, 1.5, C, device="cuda"), torch.linspace(-1.0, 1.0, C, device="cuda")
    d = torch.randn(N, T, C, device="cuda", generator=torch.Generator(device="cuda").manual_seed(C))
    layer = layers.GroupNorm(N, T, C, G, activation="none", eps=eps)
    out = layer.forward(x, scale, shift)
    assert torch.equal(out, shift.expand_as(out))
    rstd = 1.0 / np.sqrt(np.float64(np.float32(eps)))
    assert float((layer.stats[..., 1].double() / rstd - 1).abs().max()) <= 1e-6
    gx, gs, gb = layer.backward(x, scale, shift, d)
    g = (d.double() * scale.double()).view(N, T, G, C // G)
    want = (rstd * (g - g.mean((1, 3), keepdim=True))).view(N, T, C)
    assert float((gx.double() - want).abs().max()) <= ARITHMETIC * float(want.abs().max())
    assert not gs.any() and float((gb.double() - d.double().sum((0, 1))).abs().max()) <= ARITHMETIC * float(d.double().abs().sum((0, 1)).max())
