"""Measurable cases of the operators of a selective state space layer: the short causal convolution, the selective scan, and the norms
around a block with its gate and residual.

A case is a dict of plain values.  Ops:

  conv, convtrain, convstep        the convolution over whole sequences, the same with gradients, one position of many requests
  select, selecttrain, selectstep  the scan over whole sequences, the same with gradients, one position of many requests
  block, blocktrain                gate, norm behind a block, residual, norm before the next block; the same with gradients

With `own` false, run() computes the operators in elementary torch operations in 32 bits; with `own` true it calls the package.
exact() computes them in 64 bits from their definitions.
"""
import math

import numpy as np
import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_SIZE = {"f32": 4, "bf16": 2, "f16": 2}
_EPS = 1e-5                                  # of the norms


def _named(c, name):
    return dict(c, name=name) if name else c


def _conv(op, B, T, C, taps, dtype, act="silu", ragged=False, initial=False, time_major=False, name=None):
    return _named({"op": op, "B": B, "T": T, "C": C, "taps": taps, "dtype": dtype, "act": act, "ragged": ragged, "initial": initial,
                   "time_major": time_major}, name)


def _convstep(rows, pool, C, taps, dtype, act="silu", name=None):
    return _named({"op": "convstep", "rows": rows, "pool": pool, "C": C, "taps": taps, "dtype": dtype, "act": act}, name)


def _select(op, B, T, C, N, groups, dtype, ragged=False, initial=False, time_major=False, name=None):
    return _named({"op": op, "B": B, "T": T, "C": C, "N": N, "groups": groups, "dtype": dtype, "ragged": ragged, "initial": initial,
                   "time_major": time_major}, name)


def _selectstep(rows, pool, C, N, groups, dtype, name=None):
    return _named({"op": "selectstep", "rows": rows, "pool": pool, "C": C, "N": N, "groups": groups, "dtype": dtype}, name)


def _block(op, rows, C, dtype, stream, gate="before", residual=True, ragged=False, name=None):
    return _named({"op": op, "rows": rows, "C": C, "dtype": dtype, "stream": stream, "gate": gate, "residual": residual, "ragged": ragged}, name)


def listed():
    return [
        # evaluation of one small batch of quarterly series at the network's hidden size: nothing but latency
        _conv("conv", 16, 72, 40, 4, "f32", name="conv_quarterly_16"),
        # training on ragged monthly series in the framework's time-major order: odd batch, hidden size 50, windows carried over from a batch before
        _conv("convtrain", 501, 240, 50, 4, "f32", ragged=True, initial=True, time_major=True, name="convtrain_monthly_501_ragged"),
        # an ordinary large training step of a wide layer
        _conv("convtrain", 8, 4096, 2048, 4, "bf16", name="convtrain_4096_wide"),
        # a token each for a handful of requests
        _convstep(7, 64, 1000, 4, "bf16", name="convstep_7"),
        # evaluation of one small batch of quarterly series
        _select("select", 16, 72, 40, 16, 1, "f32", name="select_quarterly_16"),
        # training on ragged monthly series, time-major, with states carried over
        _select("selecttrain", 501, 240, 50, 16, 1, "f32", ragged=True, initial=True, time_major=True, name="selecttrain_monthly_501_ragged"),
        # an ordinary large training step of a wide layer
        _select("selecttrain", 4, 4096, 2048, 16, 1, "bf16", name="selecttrain_4096_wide"),
        # one very long sequence of few channels: parallel over time or not at all
        _select("selecttrain", 1, 65536, 256, 16, 1, "bf16", initial=True, name="selecttrain_65536_single"),
        # a token each for a full server: the states of all requests are read and written
        _selectstep(1024, 2048, 2048, 16, 1, "bf16", name="selectstep_1024"),
        # a token each for a handful of requests, the residual stream in 32 bits
        _block("block", 7, 2048, "bf16", "f32", name="block_7"),
        # ragged monthly series at hidden size 50: many short rows, those past the lengths absent; the gated norm inside a block, no residual
        _block("blocktrain", 120240, 50, "f32", "f32", residual=False, ragged=True, name="blocktrain_monthly_501_ragged"),
        # an ordinary large training step of a wide layer, everything at once
        _block("blocktrain", 32768, 2048, "bf16", "bf16", gate="after", name="blocktrain_32768"),
    ]


def _log(rng, lo, hi):
    return round(math.exp(rng.uniform(math.log(lo), math.log(hi))))


def draw(rng):
    """One more case of the same ranges: sizes over their logarithm, as often odd as round."""
    most = {"conv": 8 * 4096 * 2048, "select": 4 * 4096 * 2048 * 16, "block": 32768 * 2048}
    size = lambda lo, hi, to: max(lo, _log(rng, lo, hi) // to * to if rng.random() < 0.5 else _log(rng, lo, hi))  # noqa: E731
    while True:
        op = rng.choice(["conv", "convtrain", "convtrain", "convstep", "select", "select", "selecttrain", "selecttrain", "selecttrain", "selectstep",
                         "block", "blocktrain", "blocktrain"])
        dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
        half = _SIZE[dtype] // 2
        if op in ("conv", "convtrain"):
            B, T, C = size(1, 512, 4), size(8, 65536, 64), size(16, 4096, 64)
            if not 4096 <= B * T * C * half <= most["conv"]:
                continue
            return _conv(op, B, T, C, rng.choice([2, 3, 4, 4, 4, 7, 8]), dtype, rng.choice(["silu", "silu", "none"]), rng.random() < 0.4 and B > 1,
                         rng.random() < 0.5, rng.random() < 0.3)
        if op == "convstep":
            rows = size(1, 2048, 8)
            return _convstep(rows, rows + _log(rng, 1, 4096), size(16, 4096, 64), rng.choice([2, 3, 4, 4, 8]), dtype)
        if op in ("select", "selecttrain"):
            B, T, C, N = size(1, 512, 4), size(8, 65536, 64), size(16, 4096, 64), rng.choice([4, 7, 8, 16, 16, 16, 16, 32])
            groups = rng.choice([1, 1, 1, 2, 4])
            if C % groups or not 65536 <= B * T * C * N * half <= most["select"]:
                continue
            return _select(op, B, T, C, N, groups, dtype, rng.random() < 0.4 and B > 1, rng.random() < 0.5, rng.random() < 0.3)
        if op == "selectstep":
            rows, C, groups = size(1, 1024, 8), size(16, 2048, 64), rng.choice([1, 1, 2])
            if C % groups:
                continue
            return _selectstep(rows, rows + _log(rng, 1, 1024), C, rng.choice([4, 7, 16, 16, 16, 32]), groups, dtype)
        rows, C = size(1, 200000, 64), size(16, 8192, 64)
        if not 4096 <= rows * C * half <= most["block"]:
            continue
        return _block(op, rows, C, dtype, rng.choice([dtype, "f32"]), rng.choice(["none", "before", "after"]), rng.random() < 0.7,
                      rng.random() < 0.3 and rows > 1)


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(g, shape, mean=0.0, sd=1.0, dtype=torch.float32):
    return torch.empty(shape, device="cuda").normal_(mean, sd, generator=g).to(dtype)


def _lengths(case, rows, T, seed):
    """Ragged lengths between a quarter of the longest and the longest, one of which is there and one empty row in larger batches."""
    if not case["ragged"]:
        return None
    rng = np.random.RandomState(seed)
    n = rng.randint(max(1, T // 4), T + 1, rows).astype(np.int32)
    n[rng.randint(rows)] = T
    if rows > 8:
        n[0 if n[0] < T else 1] = 0
    return torch.from_numpy(n).cuda()


def _scan_parameters(g, C, N):
    """Decay rates 1 .. N with some spread over the channels, step sizes of 0.001 to 0.1 where the projection gives zero."""
    rate = torch.arange(1, N + 1, device="cuda", dtype=torch.float32).repeat(C, 1) * _normal(g, (C, N), 0.0, 0.2).exp()
    dt = torch.exp(torch.empty(C, device="cuda").uniform_(math.log(1e-3), math.log(1e-1), generator=g))
    return {"A": -rate, "D": _normal(g, (C,), 1.0, 0.2), "bias": dt + torch.log(-torch.expm1(-dt))}


def _inputs(case, seed):
    """The operands of a case, before anything that belongs to one side only."""
    g, op, dt = _generator(seed), case["op"], _TYPES[case["dtype"]]
    if op in ("conv", "convtrain"):
        B, T, C, K = case["B"], case["T"], case["C"], case["taps"]
        shape = (T, B) if case["time_major"] else (B, T)
        # the half of a projection's result that the block's gate does not have
        both = torch.empty((*shape, 2 * C), device="cuda", dtype=dt)
        both.normal_(generator=g)
        s = {"x": both[..., :C], "weight": _normal(g, (C, K), 0.0, 1.0 / math.sqrt(K)), "bias": _normal(g, (C,), 0.0, 0.3),
             "lengths": _lengths(case, B, T, seed), "initial": _normal(g, (B, K - 1, C), dtype=dt) if case["initial"] else None}
        if op == "convtrain":
            s["grad_out"] = _normal(g, (*shape, C), dtype=dt)
            s["grad_last"] = _normal(g, (B, K - 1, C)) if case["initial"] else None
        return s
    if op == "convstep":
        rows, C, K = case["rows"], case["C"], case["taps"]
        both = _normal(g, (rows, 2 * C), dtype=dt)
        return {"x": both[:, :C], "weight": _normal(g, (C, K), 0.0, 1.0 / math.sqrt(K)), "bias": _normal(g, (C,), 0.0, 0.3),
                "state": _normal(g, (case["pool"], K - 1, C), dtype=dt),
                "slots": torch.from_numpy(np.random.RandomState(seed).permutation(case["pool"])[:rows].astype(np.int32)).cuda()}
    if op in ("select", "selecttrain"):
        B, T, C, N, G = case["B"], case["T"], case["C"], case["N"], case["groups"]
        shape = (T, B) if case["time_major"] else (B, T)
        mixed = _normal(g, (*shape, 2 * G * N), dtype=dt)       # B and C of a position from one projection
        s = {"x": _normal(g, (*shape, C), dtype=dt), "delta": _normal(g, (*shape, C), 0.0, 0.7, dt), **_scan_parameters(g, C, N),
             "B": mixed[..., :G * N].unflatten(-1, (G, N)), "C": mixed[..., G * N:].unflatten(-1, (G, N)), "lengths": _lengths(case, B, T, seed),
             "initial": _normal(g, (B, C, N)) if case["initial"] else None}
        if op == "selecttrain":
            s["grad_out"] = _normal(g, (*shape, C), dtype=dt)
            s["grad_last"] = _normal(g, (B, C, N)) if case["initial"] else None
        return s
    if op == "selectstep":
        rows, C, N, G = case["rows"], case["C"], case["N"], case["groups"]
        mixed = _normal(g, (rows, 2 * G * N), dtype=dt)
        return {"x": _normal(g, (rows, C), dtype=dt), "delta": _normal(g, (rows, C), 0.0, 0.7, dt), **_scan_parameters(g, C, N),
                "B": mixed[:, :G * N].unflatten(-1, (G, N)), "C": mixed[:, G * N:].unflatten(-1, (G, N)), "state": _normal(g, (case["pool"], C, N)),
                "slots": torch.from_numpy(np.random.RandomState(seed).permutation(case["pool"])[:rows].astype(np.int32)).cuda()}
    rows, C, train, stream = case["rows"], case["C"], op == "blocktrain", _TYPES[case["stream"]]
    s = {"y": _normal(g, (rows, C), 0.0, 0.8, dt), "post": _normal(g, (C,), 1.0, 0.2), "exists": None, "gate": None, "residual": None, "scale": None,
         "pre": None}
    if case["gate"] != "none":
        s["gate"] = _normal(g, (rows, C), dtype=dt)
    if case["residual"]:
        s |= {"residual": _normal(g, (rows, C), 0.0, 2.0, stream), "scale": _normal(g, (C,), 0.5, 0.1), "pre": _normal(g, (C,), 1.0, 0.2)}
    if case["ragged"]:
        s["exists"] = torch.from_numpy((np.random.RandomState(seed).random(rows) < 0.7).astype(np.int32)).cuda()
    if train:
        s["grad_out"] = _normal(g, (rows, C), dtype=dt)
        s["grad_sum"] = _normal(g, (rows, C), dtype=stream) if case["residual"] else None
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if not own:
        return s
    from paper_1907_03329_amd import state_space
    op, dt = case["op"], _TYPES[case["dtype"]]
    if op in ("conv", "convtrain"):
        s["layer"] = state_space.ShortConvolution(case["B"], case["T"], case["C"], case["taps"], activation=case["act"], dtype=dt,
                                                  time_major=case["time_major"], training=op == "convtrain")
    elif op in ("select", "selecttrain"):
        s["layer"] = state_space.SelectiveScan(case["B"], case["T"], case["C"], case["N"], groups=case["groups"], dtype=dt,
                                               time_major=case["time_major"], training=op == "selecttrain")
    elif op in ("block", "blocktrain"):
        s["layer"] = state_space.BlockNorm(case["rows"], case["C"], gate=case["gate"], residual=case["residual"], pre=case["residual"], eps=_EPS,
                                           dtype=dt, stream_dtype=_TYPES[case["stream"]], training=op == "blocktrain")
    else:
        s["out"] = torch.empty((case["rows"], case["C"]), dtype=dt, device="cuda")
        s["call"] = state_space.convolution_step if op == "convstep" else state_space.selective_step
    return s


# ---------------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        return {"conv": _plain_conv, "convtrain": _plain_conv, "convstep": _plain_convstep, "select": _plain_select, "selecttrain": _plain_select,
                "selectstep": _plain_selectstep, "block": _plain_block, "blocktrain": _plain_block}[op](s)
    if op == "convstep":
        s["call"](s["x"], s["weight"], s["state"], s["out"], bias=s["bias"], slots=s["slots"], activation=case["act"])
        return {"out": s["out"], "state": s["state"]}
    if op == "selectstep":
        s["call"](s["x"], s["delta"], s["A"], s["B"], s["C"], s["state"], s["out"], D=s["D"], bias=s["bias"], slots=s["slots"])
        return {"out": s["out"], "state": s["state"]}
    layer = s["layer"]
    if op in ("conv", "convtrain"):
        out, last = layer.forward(s["x"], s["weight"], s["bias"], lengths=s["lengths"], initial=s["initial"])
        if op == "conv":
            return {"out": out, "last": last}
        gx, gw, gb, gi = layer.backward(s["x"], s["weight"], s["grad_out"], bias=s["bias"], lengths=s["lengths"], initial=s["initial"],
                                        grad_last=s["grad_last"])
        return {"out": out, "last": last, "grad_x": gx, "grad_weight": gw, "grad_bias": gb, "grad_initial": gi}
    if op in ("select", "selecttrain"):
        given = [s[k] for k in ("x", "delta", "A", "B", "C")]
        out, last = layer.forward(*given, D=s["D"], bias=s["bias"], lengths=s["lengths"], initial=s["initial"])
        if op == "select":
            return {"out": out, "last": last}
        grads = layer.backward(*given, s["grad_out"], D=s["D"], bias=s["bias"], lengths=s["lengths"], grad_last=s["grad_last"])
        return {"out": out, "last": last} | dict(zip(("grad_x", "grad_delta", "grad_A", "grad_B", "grad_C", "grad_D", "grad_bias", "grad_initial"), grads))
    given = {k: s[k] for k in ("gate", "residual", "scale", "exists")} | {"post_weight": s["post"], "pre_weight": s["pre"]}
    total, out = layer.forward(s["y"], **given)
    r = {"out": out} | ({"sum": total} if case["residual"] else {})
    if op == "block":
        return r
    grads = layer.backward(s["y"], s["grad_out"], grad_sum=s["grad_sum"], **given)
    names = ("grad_y", "grad_gate", "grad_residual", "grad_post_weight", "grad_scale", "grad_pre_weight")
    return r | {k: v for k, v in zip(names, grads) if v is not None}


def _turn(case, t):
    """[B, T, ...] of an array in the case's order, and back."""
    return t.transpose(0, 1) if case["time_major"] else t


def _valid(s, T):
    return None if s["lengths"] is None else torch.arange(T, device="cuda")[None] < s["lengths"][:, None]


def _keep(mask, t, instead=0.0):
    return t if mask is None else torch.where(mask.view(mask.shape + (1,) * (t.dim() - mask.dim())), t, instead)


def _plain_conv(s):
    case = s["case"]
    dt, K, silu = _TYPES[case["dtype"]], case["taps"], case["act"] == "silu"
    x = _turn(case, s["x"]).float()
    B, T, C = x.shape
    valid = _valid(s, T)
    x = _keep(valid, x)
    first = s["initial"].float() if s["initial"] is not None else torch.zeros((B, K - 1, C), device="cuda")
    seen = torch.cat([first, x], 1)                             # [B, K - 1 + T, C]
    u = s["bias"] + sum(seen[:, j:j + T] * s["weight"][:, j] for j in range(K))
    p = torch.sigmoid(u) if silu else None
    out = _turn(case, _keep(valid, u * p if silu else u).to(dt))
    at = torch.arange(K - 1, device="cuda")[None] + (s["lengths"][:, None].long() if s["lengths"] is not None else T)
    at = at.expand(B, K - 1)[..., None].expand(B, K - 1, C)
    r = {"out": out, "last": seen.gather(1, at).to(dt)}
    if case["op"] == "conv":
        return r
    du = _keep(valid, _turn(case, s["grad_out"]).float())
    if silu:
        du = du * (p * (1.0 + u * (1.0 - p)))
    dseen = torch.zeros_like(seen)
    for j in range(K):
        dseen[:, j:j + T] += du * s["weight"][:, j]
    if s["grad_last"] is not None:
        dseen.scatter_add_(1, at, s["grad_last"])
    r["grad_weight"] = torch.stack([(du * seen[:, j:j + T]).sum((0, 1)) for j in range(K)], 1)
    r["grad_bias"] = du.sum((0, 1))
    r["grad_x"] = _turn(case, _keep(valid, dseen[:, K - 1:]).to(dt))
    r["grad_initial"] = dseen[:, :K - 1].contiguous()
    return r


def _plain_convstep(s):
    case = s["case"]
    at = s["slots"].long()
    seen = torch.cat([s["state"][at].float(), s["x"].float()[:, None]], 1)
    u = s["bias"] + (seen * s["weight"].t()).sum(1)
    s["state"][at] = seen[:, 1:].to(s["state"].dtype)
    return {"out": (u * torch.sigmoid(u) if case["act"] == "silu" else u).to(_TYPES[case["dtype"]]), "state": s["state"]}


def _softplus(v):
    return v.clamp_min(0.0) + torch.log1p(torch.exp(-v.abs()))


def _prefixes(a, b):
    """h_t = a_t h_{t-1} + b_t along dimension 1 for all t at once, as (A, B) with h_t = A_t h_{-1} + B_t: the pairs of spans of
    1, 2, 4, ... positions are put together."""
    T, reach = a.shape[1], 1
    while reach < T:
        b = torch.cat([b[:, :reach], b[:, reach:] + a[:, reach:] * b[:, :-reach]], 1)
        a = torch.cat([a[:, :reach], a[:, reach:] * a[:, :-reach]], 1)
        reach *= 2
    return a, b


def _wide(t, C):
    """[.., G, N] for each of C channels: [.., C, N]."""
    return t.repeat_interleave(C // t.shape[-2], -2)


def _narrow(t, G):
    """Sums of [.., C, N] over the channels of each group: [.., G, N]."""
    return t.unflatten(-2, (G, t.shape[-2] // G)).sum(-2)


def _plain_select(s):
    case = s["case"]
    dt, N, G = _TYPES[case["dtype"]], case["N"], case["groups"]
    x, v = _turn(case, s["x"]).float(), _turn(case, s["delta"]).float() + s["bias"]
    B, T, C = x.shape
    valid = _valid(s, T)
    x, v = _keep(valid, x), _keep(valid, v)
    Bm, Cm = (_wide(_keep(valid, _turn(case, s[k]).float()), C) for k in ("B", "C"))
    delta = _keep(valid, _softplus(v))                          # (no step past the length: the state rests there)
    a = torch.exp(delta[..., None] * s["A"])                    # [B, T, C, N]
    u = delta * x
    first = s["initial"] if s["initial"] is not None else torch.zeros((B, C, N), device="cuda")
    P, h = _prefixes(a, u[..., None] * Bm)
    h = h + P * first[:, None]
    del P
    r = {"out": _turn(case, _keep(valid, (h * Cm).sum(-1) + s["D"] * x).to(dt)), "last": h[:, -1].clone()}
    if case["op"] == "select":
        return r
    dy = _keep(valid, _turn(case, s["grad_out"]).float())
    d = dy[..., None] * Cm
    if s["grad_last"] is not None:
        d[:, -1] += s["grad_last"]
    after = torch.cat([a[:, 1:], torch.ones_like(a[:, :1])], 1)
    L = _prefixes(after.flip(1), d.flip(1))[1].flip(1)          # of the state at each position
    del after, d
    before = torch.cat([first[:, None], h[:, :-1]], 1)
    g = L * a * before
    lb = (L * Bm).sum(-1)
    ddelta = _keep(valid, (g * s["A"]).sum(-1) + lb * x)
    dv = ddelta * torch.sigmoid(v)
    r["grad_x"] = _turn(case, _keep(valid, lb * delta + s["D"] * dy).to(dt))
    r["grad_delta"] = _turn(case, _keep(valid, dv).to(dt))
    r["grad_A"] = (g * delta[..., None]).sum((0, 1))
    r["grad_B"] = _turn(case, _keep(valid, _narrow(L * u[..., None], G)).to(dt))
    r["grad_C"] = _turn(case, _narrow(h * dy[..., None], G).to(dt))
    r["grad_D"] = (dy * x).sum((0, 1))
    r["grad_bias"] = _keep(valid, dv).sum((0, 1))
    r["grad_initial"] = a[:, 0] * L[:, 0]
    return r


def _plain_selectstep(s):
    case = s["case"]
    at, C = s["slots"].long(), case["C"]
    x, delta = s["x"].float(), _softplus(s["delta"].float() + s["bias"])
    h = torch.exp(delta[..., None] * s["A"]) * s["state"][at] + (delta * x)[..., None] * _wide(s["B"].float(), C)
    s["state"][at] = h
    return {"out": ((h * _wide(s["C"].float(), C)).sum(-1) + s["D"] * x).to(_TYPES[case["dtype"]]), "state": s["state"]}


def _plain_block(s):
    case = s["case"]
    dt, stream = _TYPES[case["dtype"]], _TYPES[case["stream"]]
    there = None if s["exists"] is None else s["exists"] != 0
    keep = lambda t: _keep(there, t)  # noqa: E731
    mean = lambda t: t.mean(1, keepdim=True)  # noqa: E731
    y = keep(s["y"].float())
    q = keep(s["gate"].float()) if s["gate"] is not None else None
    sig = torch.sigmoid(q) if q is not None else None
    act = q * sig if q is not None else None
    v = y * act if case["gate"] == "before" else y
    r1 = torch.rsqrt(mean(v * v) + _EPS)
    vhat = v * r1
    p = vhat * s["post"]
    e = p * act if case["gate"] == "after" else p
    r = {}
    if case["residual"]:
        t = keep(s["residual"].float()) + s["scale"] * e
        r2 = torch.rsqrt(mean(t * t) + _EPS)
        that = t * r2
        r["sum"], r["out"] = keep(t).to(stream), keep(that * s["pre"]).to(dt)
    else:
        r["out"] = keep(e).to(dt)
    if case["op"] == "block":
        return r
    d = keep(s["grad_out"].float())
    if case["residual"]:
        dt_hat = d * s["pre"]
        r["grad_pre_weight"] = (d * that).sum(0)
        total = keep(s["grad_sum"].float()) + r2 * (dt_hat - that * mean(dt_hat * that))
        r["grad_residual"] = keep(total).to(stream)
        r["grad_scale"] = (total * e).sum(0)
        d = total * s["scale"]
    dact = None
    if case["gate"] == "after":
        dact = d * p
        d = d * act
    r["grad_post_weight"] = (d * vhat).sum(0)
    dv_hat = d * s["post"]
    dv = r1 * (dv_hat - vhat * mean(dv_hat * vhat))
    if case["gate"] == "before":
        dact = dv * y
        dv = dv * act
    r["grad_y"] = keep(dv).to(dt)
    if q is not None:
        r["grad_gate"] = keep(dact * (sig * (1.0 + q * (1.0 - sig)))).to(dt)
    return r


# ---------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------------
def work(case):
    op, e = case["op"], _SIZE[case["dtype"]]
    if op in ("conv", "convtrain"):
        n, rows, K = case["B"] * case["T"] * case["C"], case["B"] * case["C"] * (case["taps"] - 1), case["taps"]
        small = 4 * case["C"] * (K + 1) + e * rows * (1 + case["initial"]) + 4 * case["B"] * case["ragged"]
        if op == "conv":
            return {"bytes": 2 * e * n + small, "flops": (2 * K + 5) * n}
        return {"bytes": 4 * e * n + small + 4 * case["C"] * (K + 1) + 4 * rows * (1 + case["initial"]), "flops": (6 * K + 15) * n}    # x, grad_out; out, grad_x
    if op == "convstep":
        n, K = case["rows"] * case["C"], case["taps"]
        return {"bytes": 2 * e * n * K + 4 * case["C"] * (K + 1) + 4 * case["rows"], "flops": (2 * K + 5) * n}
    if op in ("select", "selecttrain"):
        positions, C, N, G = case["B"] * case["T"], case["C"], case["N"], case["groups"]
        n, m, states = positions * C, positions * G * N, 4 * case["B"] * C * N
        small = 4 * C * (N + 2) + states * (1 + case["initial"]) + 4 * case["B"] * case["ragged"]
        if op == "select":
            return {"bytes": e * (3 * n + 2 * m) + small, "flops": n * (7 * N + 10)}
        # x, delta, grad_out, B, C; out, grad_x, grad_delta and the gradients of B and C
        return {"bytes": e * (6 * n + 4 * m) + small + 4 * C * (N + 2) + states * (1 + case["initial"]), "flops": n * (25 * N + 30)}
    if op == "selectstep":
        rows, C, N, G = case["rows"], case["C"], case["N"], case["groups"]
        return {"bytes": rows * (e * (3 * C + 2 * G * N) + 8 * C * N + 4) + 4 * C * (N + 2), "flops": rows * C * (7 * N + 10)}
    n, r = case["rows"] * case["C"], _SIZE[case["stream"]]
    gate, residual = case["gate"] != "none", case["residual"]
    small = 4 * case["C"] * (1 + 2 * residual) + 4 * case["rows"] * case["ragged"]
    forward = n * (e * (2 + gate) + 2 * r * residual)
    if op == "block":
        return {"bytes": forward + small, "flops": n * (5 + 6 * gate + 6 * residual)}
    # (what the forward pass read is not counted again) grad_out, grad_sum; the gradients of y, gate and residual
    return {"bytes": forward + n * (e * (2 + gate) + 2 * r * residual) + 2 * small, "flops": n * (17 + 18 * gate + 20 * residual)}


# ---------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def _states64(a, b, first):
    """h_t = a_t h_{t-1} + b_t along dimension 1 (in b's place): position by position within pieces that run side by side, then the pieces one
    behind the other."""
    B, T = a.shape[:2]
    rest = a.shape[2:]
    piece = max(1, math.isqrt(T))
    whole = T // piece * piece
    h = torch.empty_like(b)
    local, decay = b[:, :whole].unflatten(1, (-1, piece)), a[:, :whole].unflatten(1, (-1, piece)).clone()
    H = torch.zeros((B, whole // piece, *rest), dtype=a.dtype, device=a.device)
    out = torch.empty_like(local)
    for t in range(piece):
        H = decay[:, :, t] * H + local[:, :, t]
        out[:, :, t] = H
        if t:
            decay[:, :, t] *= decay[:, :, t - 1]
    state = first
    for k in range(whole // piece):
        out[:, k] += decay[:, k] * state[:, None]
        state = out[:, k, -1]
    h[:, :whole] = out.flatten(1, 2)
    for t in range(whole, T):
        state = a[:, t] * state + b[:, t]
        h[:, t] = state
    return h


def _inside(s, B, T):
    n = s["lengths"].long() if s["lengths"] is not None else torch.full((B,), T, device="cuda")
    return n, (torch.arange(T, device="cuda") < n[:, None])[:, :, None]


def _silu_slope(u):
    p = 1.0 / (1.0 + torch.exp(-u))
    return p + u * p * (1.0 - p)


def _exact_conv(case, s):
    K = case["taps"]
    x, w, bias = _turn(case, s["x"]).double(), s["weight"].double(), s["bias"].double()
    B, T, C = x.shape
    n, inside = _inside(s, B, T)
    silu = case["act"] == "silu"
    past = s["initial"].double() if s["initial"] is not None else x.new_zeros((B, K - 1, C))
    # lag k reaches k positions back, the last tap has lag 0
    def lagged(k):
        return torch.cat([past[:, K - 1 - k:], x[:, :T - k]], 1)[:, :T] if k else x
    u = torch.zeros_like(x) + bias
    for k in range(K):
        u += w[:, K - 1 - k] * lagged(k)
    r = {"out": _turn(case, torch.where(inside, u / (1.0 + torch.exp(-u)) if silu else u, 0.0))}
    last, everything = torch.empty_like(past), torch.cat([past, x], 1)
    for b, length in enumerate(n.tolist()):
        last[b] = everything[b, length:length + K - 1]
    r["last"] = last
    if case["op"] == "conv":
        return r
    du = torch.where(inside, _turn(case, s["grad_out"]).double() * (_silu_slope(u) if silu else 1.0), 0.0)
    dall = torch.zeros_like(everything)
    for k in range(K):
        dall[:, K - 1 - k:K - 1 - k + T] += du * w[:, K - 1 - k]
    if s["grad_last"] is not None:
        for b, length in enumerate(n.tolist()):
            dall[b, length:length + K - 1] += s["grad_last"][b].double()
    # (garbage past a length meets a zero)
    r["grad_weight"] = torch.stack([(du * everything[:, j:j + T]).sum((0, 1)) for j in range(K)], 1)
    r["grad_bias"] = du.sum((0, 1))
    r["grad_x"] = _turn(case, torch.where(inside, dall[:, K - 1:], 0.0))
    r["grad_initial"] = dall[:, :K - 1]
    return r


def _exact_select(case, s):
    """All channels of a few sequences at a time."""
    C, N, G = case["C"], case["N"], case["groups"]
    x, raw, Bm, Cm = (_turn(case, s[k]) for k in ("x", "delta", "B", "C"))
    B, T = x.shape[:2]
    n, inside = _inside(s, B, T)
    A, D, bias = s["A"].double(), s["D"].double(), s["bias"].double()
    train = case["op"] == "selecttrain"
    some = max(1, 2 ** 28 // (T * C * N))
    got = []
    dA, dD, dbias = torch.zeros_like(A), torch.zeros_like(D), torch.zeros_like(bias)
    of_channel = torch.arange(C, device="cuda") // (C // G)
    for lo in range(0, B, some):
        part = slice(lo, min(lo + some, B))
        ok = inside[part]
        xs, v = x[part].double(), raw[part].double() + bias
        step = torch.where(ok, torch.logaddexp(v, torch.zeros_like(v)), 0.0)
        bs, cs = Bm[part].double()[:, :, of_channel], Cm[part].double()[:, :, of_channel]
        a = torch.exp(step[..., None] * A)
        first = s["initial"][part].double() if s["initial"] is not None else torch.zeros((xs.shape[0], C, N), dtype=torch.float64, device="cuda")
        h = _states64(a, (step * xs)[..., None] * bs, first)
        r = {"out": torch.where(ok, torch.einsum("btcn,btcn->btc", h, cs) + D * xs, 0.0), "last": h[:, -1].clone()}
        if train:
            dy = torch.where(ok, _turn(case, s["grad_out"])[part].double(), 0.0)
            end = s["grad_last"][part].double() if s["grad_last"] is not None else torch.zeros_like(first)
            # mu_t = a_t lambda_t from the end, lambda_t = dy_t C_t + mu_{t+1}
            d = dy[..., None] * cs
            mu = _states64(a.flip(1), (a * d).flip(1), end).flip(1)
            d[:, :-1] += mu[:, 1:]
            d[:, -1] += end
            lam = d
            del cs
            r["grad_C"] = (h * dy[..., None]).unflatten(2, (G, C // G)).sum(3)
            h = torch.cat([first[:, None], h[:, :-1]], 1)
            r["grad_B"] = torch.where(ok[..., None], (lam * (step * xs)[..., None]).unflatten(2, (G, C // G)).sum(3), 0.0)
            through = (lam * bs).sum(-1)
            r["grad_x"] = torch.where(ok, through * step + D * dy, 0.0)
            mu *= h
            dA += (mu * step[..., None]).sum((0, 1))
            dv = torch.where(ok, ((mu * A).sum(-1) + through * xs) / (1.0 + torch.exp(-v)), 0.0)
            r["grad_delta"] = dv
            dbias += dv.sum((0, 1))
            dD += (dy * xs).sum((0, 1))
            r["grad_initial"] = a[:, 0] * lam[:, 0]
            del lam, mu, d
        got.append(r)
        del a, h, bs
    out = {}
    for k in got[0]:
        whole = torch.cat([r[k] for r in got])
        out[k] = whole if k in ("last", "grad_initial") else _turn(case, whole)
    return out | ({"grad_A": dA, "grad_D": dD, "grad_bias": dbias} if train else {})


def _exact_block(case, s):
    f = lambda k: None if s[k] is None else s[k].double()  # noqa: E731
    y, gate, res, scale, w1, w2 = (f(k) for k in ("y", "gate", "residual", "scale", "post", "pre"))
    rows, C = y.shape
    there = torch.ones((rows, 1), dtype=torch.bool, device="cuda") if s["exists"] is None else (s["exists"] != 0)[:, None]
    silu = gate / (1.0 + torch.exp(-gate)) if gate is not None else torch.ones_like(y)
    before, after = (silu if case["gate"] == k else torch.ones_like(y) for k in ("before", "after"))
    v = y * before
    root1 = torch.sqrt(v.square().sum(1, keepdim=True) / C + _EPS)
    normed = v / root1
    e = normed * w1 * after
    out, r = e, {}
    if res is not None:
        total = res + scale * e
        root2 = torch.sqrt(total.square().sum(1, keepdim=True) / C + _EPS)
        out = total / root2 * w2
        r["sum"] = torch.where(there, total, 0.0)
    r["out"] = torch.where(there, out, 0.0)
    if case["op"] == "block":
        return r
    d = torch.where(there, s["grad_out"].double(), 0.0)
    if res is not None:
        r["grad_pre_weight"] = (d * total / root2).sum(0)
        d = d * w2
        d = (d - total * (d * total).sum(1, keepdim=True) / (C * root2.square())) / root2 + torch.where(there, s["grad_sum"].double(), 0.0)
        r["grad_residual"], r["grad_scale"] = d, (d * e).sum(0)
        d = d * scale
    r["grad_post_weight"] = (d * after * normed).sum(0)
    dn = d * after * w1
    dv = (dn - normed * (dn * normed).sum(1, keepdim=True) / C) / root1
    r["grad_y"] = dv * before
    if gate is not None:
        r["grad_gate"] = (dv * y if case["gate"] == "before" else d * normed * w1) * _silu_slope(gate)
    return r


def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op == "convstep":
        at, K, w = s["slots"].long(), case["taps"], s["weight"].double()
        state = s["state"].double()
        u = s["bias"].double() + s["x"].double() * w[:, K - 1]
        for j in range(K - 1):
            u = u + state[at, j] * w[:, j]
        state[at] = torch.cat([state[at, 1:], s["x"].double()[:, None]], 1)
        return {"out": u / (1.0 + torch.exp(-u)) if case["act"] == "silu" else u, "state": state}
    if op == "selectstep":
        at, of_channel = s["slots"].long(), torch.arange(case["C"], device="cuda") // (case["C"] // case["groups"])
        x, v, state = s["x"].double(), s["delta"].double() + s["bias"].double(), s["state"].double()
        step = torch.logaddexp(v, torch.zeros_like(v))
        h = state[at] * torch.exp(step[..., None] * s["A"].double()) + s["B"].double()[:, of_channel] * (step * x)[..., None]
        state[at] = h
        return {"out": (h * s["C"].double()[:, of_channel]).sum(-1) + s["D"].double() * x, "state": state}
    if op in ("conv", "convtrain"):
        return _exact_conv(case, s)
    return _exact_select(case, s) if op in ("select", "selecttrain") else _exact_block(case, s)
