"""A small network of selective state space blocks, trained and served on the synthetic series of synth.py:

    python -m paper_1907_03329_amd.state_space_network [--workload quarterly --batch 512 --width 64 --channels 128 --states 16 --blocks 2 --steps 200 --dtype bf16]

At every position the last few log differences of a series are embedded into a residual stream; every block takes the stream's norm through a
projection, a short causal convolution with SiLU, the selective scan (whose steps, inputs and outputs come from another projection), a gated norm
and a projection back, and adds that to the stream; a linear layer on the last norm predicts the next log difference.  Training runs whole batches (the
operators, their reverse passes, AdamW over the parameter list); forecasting runs single positions on windows and states in pools.  The projections
are matrix products of torch; everything between them is the library's.
"""
from __future__ import annotations

import argparse
import math
import time

import numpy as np
import torch

from . import layers, state_space, synth
from .linear_recurrence import LAGS, following, windows

TAPS = 4        # of the convolution


class Forecaster:
    """Parameters, buffers and steps of the network for batches of B series of P positions: `width` channels of the stream, `channels` of a block with
    `states` states each."""

    def __init__(self, B: int, P: int, width: int = 64, channels: int = 128, states: int = 16, blocks: int = 2, dtype=torch.float32, state_bits: int = 32,
                 lr: float = 3e-3, seed: int = 0, device: str = "cuda"):
        self.B, self.P, self.M, self.C, self.N, self.blocks, self.dtype, self.device = B, P, width, channels, states, blocks, dtype, device
        M, C, N = width, channels, states
        g = torch.Generator(device="cpu").manual_seed(seed)
        normal = lambda *shape, sd: (torch.randn(*shape, generator=g) * sd).to(device)  # noqa: E731
        steps = torch.exp(torch.empty(C).uniform_(math.log(1e-3), math.log(1e-1), generator=g))        # where the projection gives zero
        rates = torch.log(torch.arange(1, N + 1, dtype=torch.float32)).repeat(C, 1)
        p = {"w_in": normal(LAGS, M, sd=0.5), "entry": torch.ones(M, device=device)}
        for i in range(blocks):
            p |= {f"{i}.w_both": normal(M, 2 * C, sd=M ** -0.5), f"{i}.taps": normal(C, TAPS, sd=TAPS ** -0.5), f"{i}.taps_bias": torch.zeros(C, device=device),
                  f"{i}.w_scan": normal(C, C + 2 * N, sd=C ** -0.5), f"{i}.log_rate": rates.to(device, copy=True), f"{i}.D": torch.ones(C, device=device),
                  f"{i}.delta_bias": (steps + torch.log(-torch.expm1(-steps))).to(device), f"{i}.gated": torch.ones(C, device=device),
                  f"{i}.w_back": normal(C, M, sd=C ** -0.5), f"{i}.scale": torch.full((M,), 0.5, device=device), f"{i}.pre": torch.ones(M, device=device)}
        p |= {"w_out": normal(M, 1, sd=0.02), "b_out": torch.zeros(1, device=device)}
        self.params, self.grads = p, {k: torch.zeros_like(v) for k, v in p.items()}
        # weights of the projections in the element type, renewed by the update itself
        self.weights = {k: v.to(dtype) if dtype != torch.float32 else v for k, v in p.items() if "w_" in k}
        copies = [self.weights.get(k) if dtype != torch.float32 else None for k in p]
        self.optimiser = layers.AdamW(list(p.values()), list(self.grads.values()), lr=lr, weight_decay=[0.01 if "w_" in k else 0.0 for k in p], clip_norm=1.0,
                                      state_bits=state_bits, seed=seed, copies=copies)
        self._whole, self._single = self._norms(B * P, True), self._norms(B, False)
        self.convolutions = [state_space.ShortConvolution(B, P, C, TAPS, dtype=dtype, device=device) for _ in range(blocks)]
        self.scans = [state_space.SelectiveScan(B, P, C, N, dtype=dtype, device=device) for _ in range(blocks)]
        self.steps = 0

    def _norms(self, rows, training):
        """The norm before the first block; for each block that of its gated result, and that of the stream behind it."""
        make = lambda width, **kw: state_space.BlockNorm(rows, width, dtype=self.dtype, stream_dtype=torch.float32, training=training, device=self.device, **kw)  # noqa: E731
        # (in the types of the layers: without a residual there is no stream)
        return (make(self.M, residual=False), [make(self.C, gate="before", residual=False, pre=False) for _ in range(self.blocks)],
                [make(self.M) for _ in range(self.blocks)])

    def _rate(self, i):
        return -torch.exp(self.params[f"{i}.log_rate"])

    def predict(self, features, lengths=None, exists=None):
        """Predictions [B, P] float32 of whole sequences; what backward() needs stays behind.  exists: int32 [B P], 0 past the lengths."""
        B, P, M, C, N, p, w = self.B, self.P, self.M, self.C, self.N, self.params, self.weights
        entry, gated, behind = self._whole
        embedded = features.view(-1, LAGS) @ w["w_in"]
        stream = embedded.float()
        _, n = entry.forward(embedded, pre_weight=p["entry"], exists=exists)
        self._kept, self.last_windows, self.last_states = [(embedded, stream)], [], []
        for i in range(self.blocks):
            both = (n @ w[f"{i}.w_both"]).view(B, P, 2 * C)
            u, window = self.convolutions[i].forward(both[..., :C], p[f"{i}.taps"], p[f"{i}.taps_bias"], lengths=lengths)
            mixed = (u.view(-1, C) @ w[f"{i}.w_scan"]).view(B, P, C + 2 * N)
            given = (u, mixed[..., :C], self._rate(i), mixed[..., None, C:C + N], mixed[..., None, C + N:])
            y, state = self.scans[i].forward(*given, D=p[f"{i}.D"], bias=p[f"{i}.delta_bias"], lengths=lengths)
            gate = both.view(-1, 2 * C)[:, C:]
            _, z = gated[i].forward(y.view(-1, C), gate, post_weight=p[f"{i}.gated"], exists=exists)
            back = z @ w[f"{i}.w_back"]
            self._kept.append((n, both, given, gate, z, back, stream))
            stream, n = behind[i].forward(back, residual=stream, scale=p[f"{i}.scale"], pre_weight=p[f"{i}.pre"], exists=exists)
            self.last_windows.append(window)
            self.last_states.append(state)
        self._n = n
        return (n @ w["w_out"]).float().view(B, P) + p["b_out"]

    def train_step(self, features, targets, lengths, exists):
        """One update; returns the mean squared error before it (a device scalar)."""
        loss = self.backward(features, targets, lengths, exists)
        self.steps += 1
        self.optimiser.step(self.steps)
        return loss

    def backward(self, features, targets, lengths, exists):
        """The gradients of the mean squared error, in `grads`; returns it."""
        B, P, C, N, p, w, g = self.B, self.P, self.C, self.N, self.params, self.weights, self.grads
        entry, gated, behind = self._whole
        mask = exists.view(B, P).float()
        share = 1.0 / mask.sum().clamp_min(1.0)
        error = (self.predict(features, lengths, exists) - targets) * mask
        # Gradients of the sum, not of the mean, until they are in 32 bits: a position's share of a large batch is too small for fp16.
        d = (2.0 * error).view(-1, 1)
        put = lambda name, value: torch.mul(value.view_as(g[name]), share, out=g[name])  # noqa: E731
        product = lambda a, b: a.float().t() @ b.float()  # noqa: E731  (over all positions, in 32 bits)
        put("b_out", d.sum(0))
        put("w_out", product(self._n, d))
        grad_n, grad_stream = (d @ w["w_out"].float().t()).to(self.dtype), None
        for i in reversed(range(self.blocks)):
            n, both, given, gate, z, back, stream = self._kept[i + 1]
            grad_back, _, grad_stream, _, grad_scale, grad_pre = behind[i].backward(back, grad_n, grad_stream, residual=stream, scale=p[f"{i}.scale"],
                                                                                     pre_weight=p[f"{i}.pre"], exists=exists)
            put(f"{i}.scale", grad_scale)
            put(f"{i}.pre", grad_pre)
            put(f"{i}.w_back", product(z, grad_back))
            y = self.scans[i].out.view(-1, C)
            grad_y, grad_gate, _, grad_gated, _, _ = gated[i].backward(y, grad_back @ w[f"{i}.w_back"].t(), gate=gate, post_weight=p[f"{i}.gated"], exists=exists)
            put(f"{i}.gated", grad_gated)
            grad_mixed = torch.empty((B, P, C + 2 * N), dtype=self.dtype, device=self.device)
            grad_u, _, grad_A, _, _, grad_D, grad_bias, _ = self.scans[i].backward(
                *given, grad_y.view(B, P, C), D=p[f"{i}.D"], bias=p[f"{i}.delta_bias"], lengths=lengths, grad_delta=grad_mixed[..., :C],
                grad_b=grad_mixed[..., None, C:C + N], grad_c=grad_mixed[..., None, C + N:])
            put(f"{i}.log_rate", grad_A * given[2])
            put(f"{i}.D", grad_D)
            put(f"{i}.delta_bias", grad_bias)
            flat = grad_mixed.view(-1, C + 2 * N)
            put(f"{i}.w_scan", product(given[0].view(-1, C), flat))
            grad_u = grad_u.view(-1, C) + flat @ w[f"{i}.w_scan"].t()
            grad_both = torch.empty_like(both)
            _, grad_taps, grad_taps_bias, _ = self.convolutions[i].backward(both[..., :C], p[f"{i}.taps"], grad_u.view(B, P, C), p[f"{i}.taps_bias"], lengths=lengths,
                                                                            grad_x=grad_both[..., :C])
            grad_both.view(-1, 2 * C)[:, C:] = grad_gate
            put(f"{i}.taps", grad_taps)
            put(f"{i}.taps_bias", grad_taps_bias)
            put(f"{i}.w_both", product(n, grad_both.view(-1, 2 * C)))
            grad_n = grad_both.view(-1, 2 * C) @ w[f"{i}.w_both"].t()
        embedded, _ = self._kept[0]
        grad_embedded, _, _, _, _, grad_entry = entry.backward(embedded, grad_n, pre_weight=p["entry"], exists=exists)
        put("entry", grad_entry)
        total = grad_embedded.float() + (grad_stream if grad_stream is not None else 0.0)
        put("w_in", product(features.view(-1, LAGS), total))
        return (error * error).sum() * share

    def pools(self, rows):
        """Windows and states of `rows` requests, all at the beginning."""
        return [(torch.zeros((rows, TAPS - 1, self.C), dtype=self.dtype, device=self.device), torch.zeros((rows, self.C, self.N), device=self.device))
                for _ in range(self.blocks)]

    def step(self, features, pools, slots=None):
        """The next log difference [B] float32 of B requests from features [B, LAGS], their windows and states moved on in the pools."""
        C, N, p, w = self.C, self.N, self.params, self.weights
        entry, gated, behind = self._single
        embedded = features @ w["w_in"]
        stream = embedded.float()
        _, n = entry.forward(embedded, pre_weight=p["entry"])
        for i, (windows_, states) in enumerate(pools):
            both = n @ w[f"{i}.w_both"]
            u, y = (torch.empty((self.B, C), dtype=self.dtype, device=self.device) for _ in range(2))
            state_space.convolution_step(both[:, :C], p[f"{i}.taps"], windows_, u, p[f"{i}.taps_bias"], slots)
            mixed = u @ w[f"{i}.w_scan"]
            state_space.selective_step(u, mixed[:, :C], self._rate(i), mixed[:, None, C:C + N], mixed[:, None, C + N:], states, y, p[f"{i}.D"], p[f"{i}.delta_bias"], slots)
            _, z = gated[i].forward(y, both[:, C:], post_weight=p[f"{i}.gated"])
            stream, n = behind[i].forward(z @ w[f"{i}.w_back"], residual=stream, scale=p[f"{i}.scale"], pre_weight=p[f"{i}.pre"], in_place=True)
        return (n @ w["w_out"]).float().view(-1) + p["b_out"]

    def forecast(self, features_last, pools, horizon: int):
        """`horizon` log differences [B, horizon] that follow, each fed back as an observation.  features_last: [B, LAGS], what the next position sees; pools:
        as the last position left them (predict's last_windows and last_states), moved on."""
        features, outs = features_last.clone(), []
        for _ in range(horizon):
            outs.append(self.step(features, pools))
            features = torch.cat([features[:, 1:], outs[-1][:, None].to(features.dtype)], 1)
        return torch.stack(outs, 1)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--workload", choices=synth.CONFIG_ORDER, default="quarterly")
    for name, value in (("batch", 512), ("width", 64), ("channels", 128), ("states", 16), ("blocks", 2), ("steps", 200)):
        ap.add_argument(f"--{name}", type=int, default=value)
    ap.add_argument("--dtype", choices=("f32", "bf16", "f16"), default="bf16")
    ap.add_argument("--bits", type=int, choices=(32, 8), default=8)
    args = ap.parse_args(argv)
    if args.steps < 1:
        ap.error("--steps has to be at least 1")
    dtype = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[args.dtype]
    cfg = synth.CONFIGS[args.workload].with_(B=args.batch)
    given = synth.make_inputs(cfg, seed=0, ragged=True)
    features, targets, lengths = windows(given["y"], given["lengths"])
    P = targets.shape[1]
    exists = (np.arange(P)[None] < lengths[:, None]).astype(np.int32).ravel()
    features, targets, lengths, exists = (torch.from_numpy(t).cuda() for t in (features, targets, lengths, exists))
    features = features.to(dtype)
    net = Forecaster(args.batch, P, args.width, args.channels, args.states, args.blocks, dtype=dtype, state_bits=args.bits)
    loss = net.train_step(features, targets, lengths, exists)
    first = float(loss)
    torch.cuda.synchronize()
    began = time.perf_counter()
    for _ in range(args.steps - 1):
        loss = net.train_step(features, targets, lengths, exists)
    torch.cuda.synchronize()
    ms = (time.perf_counter() - began) / max(1, args.steps - 1) * 1e3
    spread = float((targets[exists.view(-1, P) > 0]).square().mean())
    net.predict(features, lengths, exists)
    pools = [(window.clone(), state.clone()) for window, state in zip(net.last_windows, net.last_states)]
    ahead = net.forecast(following(features, targets, lengths), pools, cfg.H)
    print(f"{args.workload}, {args.batch} series, {P} positions, {args.blocks} blocks of {args.channels} channels x {args.states} states, {args.dtype}, moments in "
          f"{args.bits} bits: mean squared error {first:.5f} -> {float(loss):.5f} (mean square of the targets {spread:.5f}), {ms:.3f} ms a step; "
          f"forecasts {tuple(ahead.shape)}, finite: {bool(ahead.isfinite().all())}")


if __name__ == "__main__":
    main()
