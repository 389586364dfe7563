"""Gated linear recurrence on the GPU: arrays that overlap are refused, arrays that only lie between each other are not, and a layer's own last state
and gradient are its next call's."""
import numpy as np
import pytest

from paper_1907_03329_amd import layers
from tests.test_gpu_recurrence import close, definition, tensors

pytestmark = pytest.mark.gpu


def refused(call):
    from paper_1907_03329_amd.binding import EsrnnError
    with pytest.raises(EsrnnError) as e:
        call()
    return e.value.status == 2


def some(*shape):
    import torch
    return torch.randn(*shape, device="cuda")


@pytest.mark.parametrize("time_major", [False, True])
@pytest.mark.parametrize("B,T,C", [(3, 7, 8), (1, 7, 65), (3, 1, 5), (1, 1, 4), (2, 300, 67)])
def test_overlap_is_refused(B, T, C, time_major):
    lead = (T, B) if time_major else (B, T)
    layer = layers.GatedRecurrence(B, T, C, time_major=time_major)
    x, g, d = (some(*lead, C) for _ in range(3))
    assert refused(lambda: layer.forward(layer.out, g)) and refused(lambda: layer.forward(x, layer.out))
    layer.forward(x, g)
    for own in (x, g, d):
        assert refused(lambda: layer.backward(x, g, d, grad_x=own)) and refused(lambda: layer.backward(x, g, d, grad_gate=own))
    both = some(*lead, 2 * C)
    assert refused(lambda: layer.backward(x, g, d, grad_x=both[..., :C], grad_gate=both[..., :C]))
    # by one channel, in a row of their own and behind the last one of the others
    assert refused(lambda: layer.backward(x, g, d, grad_x=both[..., :C], grad_gate=both[..., C - 1:2 * C - 1]))
    assert refused(lambda: layer.backward(x, g, d, grad_x=both[..., C - 1:2 * C - 1], grad_gate=both[..., :C]))
    more = some(*(n + 1 for n in lead), C)
    for first, second in (((0, 0), (1, 1)), ((1, 0), (0, 1)), ((0, 1), (0, 0)), ((1, 0), (0, 0))):
        view = lambda at: more[at[0]:at[0] + lead[0], at[1]:at[1] + lead[1]]  # noqa: E731
        shares = abs(first[0] - second[0]) < lead[0] and abs(first[1] - second[1]) < lead[1]
        call = lambda: layer.backward(x, g, d, grad_x=view(first), grad_gate=view(second))  # noqa: E731
        if shares:
            assert refused(call)
        else:
            call()


@pytest.mark.parametrize("time_major", [False, True])
@pytest.mark.parametrize("B,T,C", [(3, 7, 8), (1, 7, 65), (3, 1, 5), (2, 300, 67)])
def test_five_parts_of_one_array(B, T, C, time_major):
    """x, gate, gradient of out and both gradients, row by row in one array."""
    import torch
    rng = np.random.default_rng(C)
    lead = (T, B) if time_major else (B, T)
    x, g, d, ref = tensors(rng, B, T, C, "float32", "smooth", time_major)
    for order in ((0, 1, 2, 3, 4), (4, 2, 0, 3, 1)):
        one = torch.full(lead + (5 * C,), float("nan"), device="cuda")
        parts = [one[..., i * C:(i + 1) * C] for i in order]
        for to, v in zip(parts, (x, g, d)):
            to.copy_(v)
        layer = layers.GatedRecurrence(B, T, C, time_major=time_major)
        layer.forward(*parts[:2])
        layer.backward(*parts[:3], grad_x=parts[3], grad_gate=parts[4])
        want = definition("smooth", ref["x"], ref["g"], np.zeros((B, C)), np.full(B, T), ref["d"], np.zeros((B, C)))
        turn = (lambda t: t.transpose(0, 1)) if time_major else (lambda t: t)
        close(turn(parts[3]), want[2])
        close(turn(parts[4]), want[3])
        assert torch.equal(parts[0], x) and torch.equal(parts[1], g) and torch.equal(parts[2], d)


@pytest.mark.parametrize("B,T,C", [(2, 40, 65), (5, 300, 67), (400, 20, 130), (3, 300, 64), (1, 3000, 193)])
@pytest.mark.parametrize("other_stream", [False, True])
def test_pieces_of_a_sequence_one_after_the_other(B, T, C, other_stream):
    """The layer's own last state is the next piece's initial one, and backwards its gradient likewise: as if the caller had copied them."""
    import torch
    x, g, d = some(3, B, T, C), some(3, B, T, C), some(3, B, T, C)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream() if other_stream else None
    results = []
    for copied in (True, False):
        layer = layers.GatedRecurrence(B, T, C)
        state, found = torch.zeros(B, C, device="cuda"), []
        gradient = torch.ones(B, C, device="cuda")
        for k in range(3):
            torch.cuda.synchronize()
            out, last = layer.forward(x[k], g[k], initial=state, stream=stream)
            grads = layer.backward(x[k], g[k], d[k], grad_last=gradient, stream=stream)
            torch.cuda.synchronize()
            found += [t.clone() for t in (out, last) + grads]
            state, gradient = (last.clone(), grads[2].clone()) if copied else (last, grads[2])
        results.append(found)
    assert all(torch.equal(a, b) for a, b in zip(*results))
