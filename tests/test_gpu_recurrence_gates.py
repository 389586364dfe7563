"""Gated linear recurrence on the GPU with gates far from zero, where one of its two coefficients is near the end of fp32: every 16-bit number from
80 to 95 of either sign, NaN and infinities, in sequences of one block and of many, in reverse and position by position."""
import numpy as np
import pytest

from paper_1907_03329_amd import layers
from tests.test_gpu_recurrence import ARITHMETIC, ROUNDING, definition

pytestmark = pytest.mark.gpu

# What the coefficients may be off by: the large one by some 2^-23, so that a state kept over T positions is off by T 2^-23 at most;
# the small one, below 1e-34 here, may be zero where it is no normal number.  Elements of the result are compared one by one: with their
# own size, and an absolute 1e-30 for what the small coefficient makes of inputs of size one.
TINY = 1e-30


def gates(dtype, sign):
    """All numbers of the type from 80 to 95 (fp32: every 1/64)."""
    step = {"bfloat16": 0.5, "float16": 2.0 ** -4, "float32": 2.0 ** -6}[dtype]
    return sign * np.arange(80.0, 95.0 + step, step)


def close(got, want, dtype, T, what):
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all(), what
    bound = (ROUNDING[dtype] + ARITHMETIC + T * 2.0 ** -23) * np.abs(want) + TINY
    assert (np.abs(got - want) <= bound).all(), (what, got[np.abs(got - want) > bound][:4], want[np.abs(got - want) > bound][:4])


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("kind", ["smooth", "decay"])
@pytest.mark.parametrize("sign", [-1.0, 1.0])
@pytest.mark.parametrize("T", [5, 300])
def test_gates_far_from_zero(dtype, kind, sign, T):
    import torch
    g = gates(dtype, sign)
    rng = np.random.default_rng(T)
    C, dt = len(g), getattr(torch, dtype)
    # (values of size one, none near zero: of a sum of a few of either sign every element has to be right by itself)
    x, d = (torch.from_numpy(rng.uniform(0.5, 1.0, (1, T, C))).to(dt) for _ in range(2))
    gate = torch.from_numpy(np.broadcast_to(g, (1, T, C)).copy()).to(dt)
    assert (gate.double().numpy() == g).all()
    h0, dl = (torch.from_numpy(rng.uniform(0.5, 1.0, (1, C))).float() for _ in range(2))
    layer = layers.GatedRecurrence(1, T, C, kind=kind, dtype=dt)
    out, last = layer.forward(x.cuda(), gate.cuda(), initial=h0.cuda())
    gx, gg, gi = layer.backward(x.cuda(), gate.cuda(), d.cuda(), grad_last=dl.cuda())
    f = lambda t: t.double().numpy()  # noqa: E731
    want = definition(kind, f(x), f(gate), f(h0), np.array([T]), f(d), f(dl))
    for name, got, w, of in zip(("out", "last", "grad_x", "grad_gate", "grad_initial"), (out, last, gx, gg, gi), want,
                                (dtype, "float32", dtype, dtype, "float32")):
        close(got, w, of, T, (name, dtype, kind, sign, T))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("kind", ["smooth", "decay"])
@pytest.mark.parametrize("sign", [-1.0, 1.0])
def test_single_positions_with_gates_far_from_zero(dtype, kind, sign):
    import torch
    g = gates(dtype, sign)
    rng = np.random.default_rng(1)
    C, dt = len(g), getattr(torch, dtype)
    x, gate = torch.from_numpy(rng.uniform(0.5, 1.0, (1, C))).to(dt), torch.from_numpy(g[None]).to(dt)
    state = torch.from_numpy(rng.uniform(0.5, 1.0, (1, C))).float()
    want = definition(kind, x.double().numpy()[:, None], gate.double().numpy()[:, None], state.double().numpy(), np.array([1]))[1]
    out, state = torch.empty(1, C, dtype=dt, device="cuda"), state.cuda()
    layers.recurrence_step(x.cuda(), gate.cuda(), state, out, kind=kind)
    close(out, want, dtype, 1, ("out", dtype, kind, sign))
    close(state, want, "float32", 1, ("state", dtype, kind, sign))


@pytest.mark.parametrize("kind", ["smooth", "decay"])
def test_a_gate_that_is_not_a_number(kind):
    """Its channel is NaN from its position on, and its own gradients; the other channels are what they were."""
    import torch
    T = 300
    x, gate = torch.ones(1, T, 8, device="cuda"), torch.zeros(1, T, 8, device="cuda")
    layer = layers.GatedRecurrence(1, T, 8, kind=kind)
    clean = layer.forward(x, gate)[0].clone()
    gate[0, 150, 3] = float("nan")
    out, last = layer.forward(x, gate)
    gx, gg, gi = layer.backward(x, gate, x)
    assert out[0, 150:, 3].isnan().all() and torch.equal(out[0, :150], clean[0, :150]) and bool(last[0, 3].isnan())
    assert bool(gg[0, 150, 3].isnan()) and bool(gi[0, 3].isnan())
    others = [c for c in range(8) if c != 3]
    assert torch.equal(out[:, :, others], clean[:, :, others])
    assert all(bool(t[..., others].isfinite().all()) for t in (last, gx, gg, gi))
