"""Group norm on the GPU, group by group: small gradients and outputs are right by their own size, not only beside the largest of the array."""
import numpy as np
import pytest

from paper_1907_03329_amd import layers
from tests.test_gpu_group_norm import ARITHMETIC, EPS, ROUNDING, definition

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,T,C,G", [(18, 1, 96, 6), (18, 1, 37, 1), (18, 1, 1024, 2), (18, 1, 2048, 2), (18, 40, 48, 4), (2100, 4, 60, 3), (9, 2500, 40, 4)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("act", ["silu", "none"])
def test_every_group_has_its_own_digits(N, T, C, G, dtype, act):
    """Samples whose gradients lie eight powers of ten apart, and groups whose scales and shifts lie four apart.  Within a group the bound is that of
    tests/test_gpu_group_norm.py, against the group's largest value."""
    import torch
    rng = np.random.default_rng(C + T)
    dt, D = getattr(torch, dtype), C // G
    x = torch.from_numpy(rng.normal(0.3, 1.2, (N, T, C))).to(dt)
    d = torch.from_numpy(rng.normal(size=(N, T, C)) * 10.0 ** (np.arange(N) % 9 - 4)[:, None, None]).to(dt)
    factor = np.repeat(10.0 ** (np.arange(G) % 5 - 2.0), D)
    scale, shift = (torch.from_numpy(rng.normal(m, 0.2, C) * factor).float() for m in (1.0, 0.0))
    layer = layers.GroupNorm(N, T, C, G, activation=act, eps=EPS, dtype=dt)
    given = x.cuda(), scale.cuda(), shift.cuda()
    out = layer.forward(*given)
    gx, _, _ = layer.backward(*given, d.cuda())
    f = lambda t: t.double().numpy()  # noqa: E731
    want = definition(f(x), f(scale), f(shift), G, act, [T] * N, f(d))
    for name, got, w in (("out", out, want[0]), ("grad_x", gx, want[1])):
        off, most = (np.abs(v).reshape(N, T, G, D).max((1, 3)) for v in (got.double().cpu().numpy() - w, w))
        # (of a single position's group of few channels what is left of sums that cancel counts by the size of their terms: as large as the gradient
        # that goes in times scale and 1 / deviation)
        if name == "grad_x":
            rstd = 1.0 / np.sqrt(f(x).reshape(N, T, G, D).var((1, 3)) + EPS)
            most = np.maximum(most, rstd * np.abs(f(d) * f(scale)).reshape(N, T, G, D).max((1, 3)))
        assert (off <= (ROUNDING[dtype] + ARITHMETIC) * most).all(), (name, (off / most).max())
