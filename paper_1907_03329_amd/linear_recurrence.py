"""A small network of the layer operators, trained and served on the synthetic series of synth.py:

    python -m paper_1907_03329_amd.linear_recurrence [--workload quarterly --batch 512 --channels 128 --steps 200 --dtype bf16 --bits 8]

At every position the last few log differences of a series go through one projection to the input and the gate of a gated
recurrence (an exponential smoothing whose coefficient the network chooses, position by position); its states are
normalised by groups with SiLU, every position by itself, and a linear layer predicts the next log difference.  Training runs whole
batches (scan, group norm, their reverse passes, AdamW over the parameter list); forecasting runs single positions on states
in a pool.  The projections are matrix products of torch; everything between them is the library's.
"""
from __future__ import annotations

import argparse
import time

import numpy as np
import torch

from . import layers, synth

LAGS = 8        # log differences that a position sees


def windows(y: np.ndarray, lengths: np.ndarray):
    """Features [B, P, LAGS], targets [B, P] and positions that exist [B] of series y [T, B] (position p sees up to observation
    p + LAGS and predicts the log difference that follows)."""
    log = np.log(y.T.astype(np.float64))
    diff = np.diff(log, axis=1)                                     # [B, T - 1]
    P = diff.shape[1] - LAGS
    features = np.stack([diff[:, j:j + P] for j in range(LAGS)], axis=-1)
    contiguous = lambda v: np.ascontiguousarray(v, dtype=np.float32)  # noqa: E731
    return contiguous(features), contiguous(diff[:, LAGS:LAGS + P]), np.maximum(lengths - 1 - LAGS, 0).astype(np.int32)


def following(features, targets, lengths):
    """Features [B, LAGS] of the position behind the last one of each series: the last one's, moved on by its target, which is the last log
    difference that there is."""
    if int(lengths.min()) < 1:
        raise ValueError(f"series of fewer than {LAGS + 2} observations have no position to go on from")
    b, last = torch.arange(len(features), device=features.device), lengths.long() - 1
    return torch.cat([features[b, last, 1:], targets[b, last, None].to(features.dtype)], 1)


class Forecaster:
    """Parameters, buffers and steps of the network for batches of B series of P positions."""

    def __init__(self, B: int, P: int, channels: int = 128, groups: int = 8, dtype=torch.float32, state_bits: int = 32,
                 lr: float = 3e-3, seed: int = 0, device: str = "cuda"):
        self.B, self.P, self.C, self.dtype, self.device = B, P, channels, dtype, device
        C = channels
        g = torch.Generator(device="cpu").manual_seed(seed)
        normal = lambda *shape, sd: (torch.randn(*shape, generator=g) * sd).to(device)  # noqa: E731
        gate_bias = torch.linspace(-4.0, 1.0, C)        # memories of about one to fifty positions
        self.params = {"w_in": normal(LAGS, 2 * C, sd=0.5), "b_in": torch.cat([torch.zeros(C), gate_bias]).to(device),
                       "scale": torch.ones(C, device=device), "shift": torch.zeros(C, device=device), "w_out": normal(C, 1, sd=0.02),
                       "b_out": torch.zeros(1, device=device)}
        self.grads = {k: torch.zeros_like(v) for k, v in self.params.items()}
        # weights of the projections in the element type, renewed by the update itself
        self.weights = {k: self.params[k].to(dtype) if dtype != torch.float32 else self.params[k] for k in ("w_in", "w_out")}
        copies = [self.weights.get(k) if dtype != torch.float32 else None for k in self.params]
        decay = [0.01 if k.startswith("w") else 0.0 for k in self.params]
        self.optimiser = layers.AdamW(list(self.params.values()), list(self.grads.values()), lr=lr, weight_decay=decay, clip_norm=1.0,
                                      state_bits=state_bits, seed=seed, copies=copies)
        self.recurrence = layers.GatedRecurrence(B, P, C, kind="smooth", dtype=dtype, device=device)
        self.norm = layers.GroupNorm(B * P, 1, C, groups, activation="silu", dtype=dtype, device=device)
        self.norm_step = layers.GroupNorm(B, 1, C, groups, activation="silu", dtype=dtype, training=False, device=device)
        self.grad_both = torch.empty((B, P, 2 * C), dtype=dtype, device=device)
        self.steps = 0

    def predict(self, features, lengths=None, exists=None):
        """Predictions [B, P] float32 of whole sequences; what backward() needs stays behind.  exists: int32 [B P], 0 past the lengths."""
        self._both = torch.addmm(self.params["b_in"].to(self.dtype), features.view(-1, LAGS), self.weights["w_in"]).view(self.B, self.P, 2 * self.C)
        x, gate = self._both[..., :self.C], self._both[..., self.C:]
        states, self.last = self.recurrence.forward(x, gate, lengths=lengths)
        self._z = self.norm.forward(states.view(-1, 1, self.C), self.params["scale"], self.params["shift"], lengths=exists)
        return (self._z.view(-1, self.C) @ self.weights["w_out"]).float().view(self.B, self.P) + self.params["b_out"]

    def train_step(self, features, targets, lengths, exists):
        """One update; returns the mean squared error before it (a device scalar)."""
        B, P, C = self.B, self.P, self.C
        mask = exists.view(B, P).float()
        count = mask.sum().clamp_min(1.0)
        error = (self.predict(features, lengths, exists) - targets) * mask
        loss = (error * error).sum() / count
        # Gradients of the sum, not of the mean, until they are in 32 bits: a position's share of a large batch is too small for fp16.
        d, share = (2.0 * error).view(-1, 1), 1.0 / count
        g, z = self.grads, self._z.view(-1, C)
        torch.mul(d.sum(0), share, out=g["b_out"])
        torch.mul(z.float().t() @ d, share, out=g["w_out"])       # (products over all positions in 32 bits)
        grad_z = (d @ self.weights["w_out"].float().t()).to(self.dtype)     # (of the weights that the forward pass had)
        states, scale, shift = self.recurrence.out.view(-1, 1, C), self.params["scale"], self.params["shift"]
        grad_states, grad_scale, grad_shift = self.norm.backward(states, scale, shift, grad_z.view(-1, 1, C), lengths=exists)
        torch.mul(grad_scale, share, out=g["scale"])
        torch.mul(grad_shift, share, out=g["shift"])
        self.recurrence.backward(self._both[..., :C], self._both[..., C:], grad_states.view(B, P, C), lengths=lengths,
                                 grad_x=self.grad_both[..., :C], grad_gate=self.grad_both[..., C:])
        flat = self.grad_both.view(-1, 2 * C)
        flat = flat.float()
        torch.mul(features.view(-1, LAGS).float().t() @ flat, share, out=g["w_in"])
        torch.mul(flat.sum(0), share, out=g["b_in"])
        self.steps += 1
        self.optimiser.step(self.steps)
        return loss

    def step(self, features, state, slots=None):
        """The next log difference [rows] float32 of `rows` = B series from features [B, LAGS], their states updated in the pool."""
        both = torch.addmm(self.params["b_in"].to(self.dtype), features, self.weights["w_in"])
        out = torch.empty((self.B, self.C), dtype=self.dtype, device=self.device)
        layers.recurrence_step(both[:, :self.C], both[:, self.C:], state, out, slots=slots, kind="smooth")
        z = self.norm_step.forward(out.view(-1, 1, self.C), self.params["scale"], self.params["shift"])
        return (z.view(-1, self.C) @ self.weights["w_out"]).float().view(-1) + self.params["b_out"]

    def forecast(self, features_last, state, horizon: int):
        """`horizon` log differences [B, horizon] that follow, each fed back as an observation.  features_last: [B, LAGS], what the next
        position sees; state: [B, C], that of the last position."""
        features, outs = features_last.clone(), []
        for _ in range(horizon):
            outs.append(self.step(features, state))
            features = torch.cat([features[:, 1:], outs[-1][:, None].to(features.dtype)], 1)
        return torch.stack(outs, 1)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--workload", choices=synth.CONFIG_ORDER, default="quarterly")
    ap.add_argument("--batch", type=int, default=512)
    ap.add_argument("--channels", type=int, default=128)
    ap.add_argument("--steps", type=int, default=200)
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
    net = Forecaster(args.batch, P, args.channels, dtype=dtype, state_bits=args.bits)
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
    ahead = net.forecast(following(features, targets, lengths), net.last.clone(), cfg.H)
    print(f"{args.workload}, {args.batch} series, {P} positions, {args.channels} channels, {args.dtype}, moments in {args.bits} bits: "
          f"mean squared error {first:.5f} -> {float(loss):.5f} (mean square of the targets {spread:.5f}), {ms:.3f} ms a step; "
          f"forecasts {tuple(ahead.shape)}, finite: {bool(ahead.isfinite().all())}")


if __name__ == "__main__":
    main()
