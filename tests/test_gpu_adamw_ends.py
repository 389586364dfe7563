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
