"""The network of state_space_network.py: convolution, scan and block norms together, in training and position by position."""
import numpy as np
import pytest

from paper_1907_03329_amd import synth

pytestmark = pytest.mark.gpu


def batch(B=96, ragged=True, dtype="float32"):
    import torch
    from paper_1907_03329_amd import linear_recurrence as lr, state_space_network as net
    cfg = synth.CONFIGS["quarterly"].with_(B=B)
    given = synth.make_inputs(cfg, seed=3, ragged=ragged)
    features, targets, lengths = lr.windows(given["y"], given["lengths"])
    exists = (np.arange(targets.shape[1])[None] < lengths[:, None]).astype(np.int32).ravel()
    features, targets, lengths, exists = [torch.from_numpy(t).cuda() for t in (features, targets, lengths, exists)]
    return net, [features.to(getattr(torch, dtype)), targets, lengths, exists]


def plain(torch, p, features, lengths, M, C, N, blocks, taps):
    """The network in elementary operations, position by position where it is a recurrence."""
    silu = lambda v: v * torch.sigmoid(v)  # noqa: E731
    rms = lambda v: v / (v.square().mean(-1, keepdim=True) + 1e-5).sqrt()  # noqa: E731
    B, P = features.shape[:2]
    stream = features @ p["w_in"]
    n = rms(stream) * p["entry"]
    for i in range(blocks):
        both = n @ p[f"{i}.w_both"]
        seen = torch.cat([torch.zeros(B, taps - 1, C, dtype=both.dtype), both[..., :C]], 1)
        u = silu(p[f"{i}.taps_bias"] + sum(seen[:, j:j + P] * p[f"{i}.taps"][:, j] for j in range(taps)))
        mixed = u @ p[f"{i}.w_scan"]
        step = torch.nn.functional.softplus(mixed[..., :C] + p[f"{i}.delta_bias"])
        b, c, A = mixed[..., C:C + N], mixed[..., C + N:], -torch.exp(p[f"{i}.log_rate"])
        h, ys = torch.zeros(B, C, N, dtype=both.dtype), []
        for t in range(P):
            h = torch.exp(step[:, t, :, None] * A) * h + (step[:, t] * u[:, t])[..., None] * b[:, t, None]
            ys.append((h * c[:, t, None]).sum(-1) + p[f"{i}.D"] * u[:, t])
        z = rms(torch.stack(ys, 1) * silu(both[..., C:])) * p[f"{i}.gated"]
        stream = stream + p[f"{i}.scale"] * (z @ p[f"{i}.w_back"])
        n = rms(stream) * p[f"{i}.pre"]
    return (n @ p["w_out"])[..., 0] + p["b_out"]


def test_gradients_of_the_whole_network():
    """Against torch's derivative of the same network written in elementary operations in 64 bits on the CPU."""
    import torch
    module, (features, targets, lengths, exists) = batch(B=6)
    P = targets.shape[1]
    net = module.Forecaster(6, P, width=16, channels=24, states=5, blocks=2)
    before = {k: v.detach().cpu().double().requires_grad_() for k, v in net.params.items()}
    loss = net.backward(features, targets, lengths, exists)
    t, e = targets.cpu().double(), exists.view(6, P).cpu().double()
    pred = plain(torch, before, features.cpu().double(), lengths, 16, 24, 5, 2, module.TAPS)
    want = ((pred - t) * e).square().sum() / e.sum()
    want.backward()
    want_loss = float(want.detach())
    assert abs(float(loss) - want_loss) <= 1e-5 * want_loss
    for k, g in net.grads.items():
        assert float((g.cpu().double() - before[k].grad).abs().max()) <= 2e-4 * float(before[k].grad.abs().max()), k


@pytest.mark.parametrize("dtype,bits", [("float32", 32), ("bfloat16", 8), ("float16", 32)])
def test_training_runs(dtype, bits):
    import torch
    module, (features, targets, lengths, exists) = batch(dtype=dtype)
    net = module.Forecaster(96, targets.shape[1], width=32, channels=64, dtype=getattr(torch, dtype), state_bits=bits)
    before = {k: v.clone() for k, v in net.params.items()}
    for _ in range(5):
        loss = net.train_step(features, targets, lengths, exists)
    assert bool(torch.isfinite(loss)) and all(bool(torch.isfinite(v).all()) for v in net.params.values())
    assert all(not torch.equal(v, before[k]) for k, v in net.params.items())


def test_positions_one_by_one_predict_what_the_whole_pass_predicts():
    import torch
    module, (features, targets, lengths, exists) = batch(B=20, ragged=False)
    P = targets.shape[1]
    net = module.Forecaster(20, P, width=32, channels=48, states=8)
    for _ in range(5):
        net.train_step(features, targets, lengths, exists)
    whole = net.predict(features, lengths, exists)
    pools, slots = net.pools(50), torch.arange(49, 29, -1, dtype=torch.int32, device="cuda")
    for p in range(P):
        one = net.step(features[:, p].contiguous(), pools, slots=slots)
        assert float((one - whole[:, p]).abs().max()) <= 1e-4 * float(whole.abs().max())
    for (windows, states), window, state in zip(pools, net.last_windows, net.last_states):
        assert float((states[slots.long()] - state).abs().max()) <= 1e-4 * float(state.abs().max())
        assert float((windows[slots.long()] - window).abs().max()) <= 1e-4 * float(window.abs().max())
        assert not states[:30].any() and not windows[:30].any()
    pools = [(w.clone(), s.clone()) for w, s in zip(net.last_windows, net.last_states)]
    ahead = net.forecast(features[:, -1], pools, 8)
    assert ahead.shape == (20, 8) and bool(ahead.isfinite().all())


def test_a_captured_training_pass():
    """Forward and reverse pass in a graph, replayed with eager work between: what the eager pass gives, every time."""
    import torch
    module, (features, targets, lengths, exists) = batch(B=40, dtype="bfloat16")
    net = module.Forecaster(40, targets.shape[1], width=32, channels=64, dtype=torch.bfloat16)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        net.backward(features, targets, lengths, exists)
    torch.cuda.synchronize()
    eager = {k: v.clone() for k, v in net.grads.items() if k != "b_out"}       # (its gradient is a sum of torch's over all positions)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        net.backward(features, targets, lengths, exists)
    for _ in range(3):
        for g in net.grads.values():
            g.fill_(float("nan"))
        net.predict(features, lengths, exists)
        graph.replay()
        torch.cuda.synchronize()
        for k, want in eager.items():
            assert float((net.grads[k] - want).abs().max()) <= 1e-5 * float(want.abs().max()), k


def test_command(capsys):
    from paper_1907_03329_amd import state_space_network
    state_space_network.main(["--batch", "64", "--channels", "64", "--width", "32", "--steps", "10"])
    assert "finite: True" in capsys.readouterr().out
    state_space_network.main(["--workload", "yearly", "--batch", "5", "--channels", "20", "--width", "12", "--states", "3", "--blocks", "1", "--steps", "1", "--dtype", "f32"])
    assert "finite: True" in capsys.readouterr().out


def test_no_steps_are_refused():
    from paper_1907_03329_amd import state_space_network
    with pytest.raises(SystemExit):
        state_space_network.main(["--batch", "16", "--steps", "0"])
