"""AdamW on the GPU with gradients and hyper-parameters near the ends of their ranges."""
import numpy as np
import pytest

from paper_1907_03329_amd import layers

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("small", [1e-3, 1e-5, 1e-7, 1e-11, 1e-15])
def test_a_small_root_beside_a_large_one_keeps_the_smallest_code(small):
    """Codes of roots are one at least, whatever the block's largest is, so that no moment is divided by nothing later."""
    import torch
    n = 1024
    p, g = torch.zeros(n, device="cuda"), torch.full((n,), small, device="cuda")
    g[::256] = 1e6
    opt = layers.AdamW([p], [g], state_bits=8, seed=3, lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.0)
    for step in (1, 2):
        opt.step(step)
        assert bool((opt.r.view(torch.uint8) > 0).all()), step
    # a gradient of zero behind small ones moves no parameter by more than its share of the largest update, lr / (1 - beta1)
    for step in range(3, 200):
        g[::256] = small
        opt.step(step)
    before = p.clone()
    g.zero_()
    opt.step(200)
    assert bool((opt.r.view(torch.uint8) > 0).all()) and float((p - before).abs().max()) <= 1e-2


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [1e-37, 1e-38, 1e-40, 1e-44, 1e-50, 1e-300])
def test_eps_that_is_no_normal_number(bits, eps):
    """Gradients of zero: nothing but the decay, as 0 / eps is 0 for any eps; others: as with eps of 1e-30."""
    import torch
    results = []
    for e in (eps, 1e-30):
        p, g = torch.ones(512, device="cuda"), torch.zeros(512, device="cuda")
        g[:100] = torch.linspace(1e-12, 1.0, 100)
        opt = layers.AdamW([p], [g], state_bits=bits, lr=0.1, weight_decay=0.5, eps=e)
        for step in (1, 2):
            opt.step(step)
        results.append(p)
    assert bool((results[0][100:] - 0.95 ** 2).abs().max() <= 1e-6)
    assert torch.equal(results[0], results[1])


@pytest.mark.parametrize("clip", [1e-30, 1e-37, 1e-44, 1e-46, 1e-200])
def test_clipping_to_almost_nothing(clip):
    """A norm of 2 clipped to less than any number of fp32: the moments of a gradient of almost nothing, and a step of almost nothing of them."""
    import torch
    p, g = torch.ones(400, device="cuda"), torch.full((400,), 0.1, device="cuda")
    opt = layers.AdamW([p], [g], lr=0.1, weight_decay=0.0, clip_norm=clip, eps=1e-8)
    opt.step(1)
    assert abs(float(opt.grad_norm) - 2.0) <= 1e-5
    assert float(opt.m.abs().max()) <= 1e-31 and float((p - 1.0).abs().max()) <= 1e-6
