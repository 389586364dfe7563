"""Gradients of the network of linear_recurrence.py in 16 bits."""
import pytest

from tests.test_gpu_linear_recurrence import batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,unit", [("bfloat16", 2.0 ** -7), ("float16", 2.0 ** -10)])
def test_the_last_layers_gradient_is_that_of_the_weights_it_had(dtype, unit, monkeypatch):
    """Two halves of its weights that are one in 16 bits, and in 32 bits one and 0.45 units more: the forward pass cannot tell them apart, and what goes
    into the norm's reverse pass is the same for both."""
    import torch
    lr, (features, targets, lengths, exists) = batch(B=8)
    dt = getattr(torch, dtype)
    net = lr.Forecaster(8, targets.shape[1], channels=64, dtype=dt)
    net.params["w_out"][:32], net.params["w_out"][32:] = 1.0, 1.0 + 0.45 * unit
    net.weights["w_out"].copy_(net.params["w_out"])
    assert bool((net.weights["w_out"] == 1.0).all())
    given = []
    backward = net.norm.backward
    monkeypatch.setattr(net.norm, "backward", lambda *args, **kw: given.append(args[3].clone()) or backward(*args, **kw))
    net.train_step(features.to(dt), targets, lengths, exists)
    assert bool(given[0].any()) and torch.equal(given[0][..., :32], given[0][..., 32:])


def test_gradients_of_a_large_batch_in_fp16():
    """A batch of the size of the benchmark's: the error's share of an element of some 250 000 is below the smallest numbers of fp16.  Against the same network
    in fp32, parameter by parameter (Frobenius norms): values and gradients are rounded to 11 bits some six times on their way, 2^-11 each,
    weights once, and the roundings of many elements do not add up: 1e-2 has room for it, gradients that are lost do not."""
    import torch
    lr, (features, targets, lengths, exists) = batch(B=4096)
    grads = []
    for dtype in (torch.float32, torch.float16):
        net = lr.Forecaster(4096, targets.shape[1], channels=32, groups=4, dtype=dtype)
        net.train_step(features.to(dtype), targets, lengths, exists)
        grads.append({k: v.double() for k, v in net.grads.items()})
    for k, want in grads[0].items():
        assert float((grads[1][k] - want).norm()) <= 1e-2 * float(want.norm()), k
