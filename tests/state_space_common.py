"""Plain 64-bit definitions of the operators of a selective state space layer, position by position, and what the tests of their kernels share."""
import numpy as np

# An element is rounded to its type once: half a unit in the last place, relative to the value.
ROUNDING = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
TINY = {"float32": 2.0 ** -149, "bfloat16": 2.0 ** -133, "float16": 2.0 ** -24}


def sigmoid(v):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-v))


def silu(v):
    """silu(v) and its derivative."""
    p = sigmoid(v)
    return v * p, p * (1.0 + v * (1.0 - p))


def close(got, want, dtype, arithmetic, what="", scale=None):
    """|got - want| <= rounding |want| + arithmetic scale, elementwise: one rounding to the type, and fp32 arithmetic whose errors go by the size of
    what is added up (`scale`: an array of that, or the largest value)."""
    got = got.double().cpu().numpy()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    if not want.size:
        return
    assert np.isfinite(got).all(), what
    scale = np.abs(want).max() if scale is None else scale
    room = (ROUNDING[dtype] * (1.0 + 2.0 ** -10)) * np.abs(want) + arithmetic * scale + TINY[dtype]
    err = np.abs(got - want)
    worst = np.unravel_index(np.argmax(err - room), err.shape)
    assert (err <= room).all(), (what, worst, got[worst], want[worst], err[worst], room[worst])


def convolution(x, w, bias, first, lengths, act, d=None, dlast=None):
    """All in float64 numpy, x [B, T, C], first [B, K - 1, C]."""
    B, T, C = x.shape
    K = w.shape[1]
    out, last = np.zeros_like(x), np.zeros_like(first)
    gx, gw, gb, gi = np.zeros_like(x), np.zeros_like(w), np.zeros(C), np.zeros_like(first)
    for b in range(B):
        n = int(lengths[b])
        seen = np.concatenate([first[b], x[b, :n]])
        last[b] = seen[n:n + K - 1]
        grad = np.zeros_like(seen)
        if d is not None:
            grad[n:n + K - 1] += dlast[b]
        for t in range(n):
            u = bias + (w.T * seen[t:t + K]).sum(0)
            y, slope = silu(u) if act == "silu" else (u, np.ones_like(u))
            out[b, t] = y
            if d is not None:
                du = d[b, t] * slope
                gw += du[:, None] * seen[t:t + K].T
                gb += du
                grad[t:t + K] += w.T * du
        gi[b], gx[b, :n] = grad[:K - 1], grad[K - 1:]
    return (out, last) if d is None else (out, last, gx, gw, gb, gi)


def softplus(v):
    return np.logaddexp(v, 0.0)


def scan(x, delta, A, b, c, D, bias, h0, lengths, kind, d=None, dlast=None):
    """All in float64 numpy: x, delta [B, T, C], b, c [B, T, G, N], h0 [B, C, N]; the reverse pass written down from the forward one."""
    B, T, C = x.shape
    G = b.shape[2]
    of = np.arange(C) // (C // G)
    v = delta + bias
    step = softplus(v) if kind == "softplus" else v
    slope = sigmoid(v) if kind == "softplus" else np.ones_like(v)
    out, before, h = np.zeros_like(x), np.zeros((B, T) + h0.shape[1:]), h0.copy()
    for t in range(T):
        on = (t < lengths)[:, None]
        before[:, t] = h
        bt, ct = b[:, t, of], c[:, t, of]
        new = np.exp(step[:, t, :, None] * A) * h + (step[:, t] * x[:, t])[..., None] * bt
        h = np.where(on[..., None], new, h)
        out[:, t] = np.where(on, (h * ct).sum(-1) + D * x[:, t], 0.0)
    if d is None:
        return out, h
    mu = dlast.copy()
    gx, gd, gb, gc = np.zeros_like(x), np.zeros_like(x), np.zeros_like(b), np.zeros_like(c)
    gA, gD, gbias = np.zeros_like(A), np.zeros(C), np.zeros(C)
    for t in range(T - 1, -1, -1):
        on = (t < lengths)[:, None]
        bt, ct, s, g = b[:, t, of], c[:, t, of], step[:, t], np.where(on, d[:, t], 0.0)
        a = np.exp(s[..., None] * A)
        after = a * before[:, t] + (s * x[:, t])[..., None] * bt
        lam = np.where(on[..., None], g[..., None] * ct + mu, 0.0)
        through = (lam * bt).sum(-1)
        m = lam * a * before[:, t]
        ds = (m * A).sum(-1) + through * x[:, t]
        gx[:, t] = np.where(on, s * through + D * g, 0.0)
        gd[:, t] = np.where(on, ds * slope[:, t], 0.0)
        gA += (m * s[..., None]).sum(0)
        gD += (g * np.where(on, x[:, t], 0.0)).sum(0)
        gbias += gd[:, t].sum(0)
        for k in range(G):
            gb[:, t, k] = (lam * (s * x[:, t])[..., None])[:, of == k].sum(1)
            gc[:, t, k] = np.where(on[..., None], after * g[..., None], 0.0)[:, of == k].sum(1)
        mu = np.where(on[..., None], a * lam, mu)
    return out, h, gx, gd, gA, gb, gc, gD, gbias, mu


def block(y, gate, place, residual, exists, post, scale, pre, eps, d=None, dsum=None):
    """All in float64 numpy, rows [R, C]; operands that are None are left out.  A dict of everything, and one of how large what each is added up from is: the
    same with magnitudes in the place of terms, so that what two terms of one size leave of each other is measured by them."""
    on = exists[:, None]
    y = np.where(on, y, 0.0)
    g = np.where(on, gate, 0.0) if gate is not None else np.zeros_like(y)
    act, slope = silu(g) if gate is not None else (np.ones_like(y), np.zeros_like(y))
    steep = sigmoid(g) * (1.0 + np.abs(g) * sigmoid(-g))
    before, after = (act if place == k else np.ones_like(y) for k in ("before", "after"))
    mean = lambda t: t.mean(1, keepdims=True)  # noqa: E731
    w1, s, w2 = (np.ones(y.shape[1]) if t is None else t for t in (post, scale, pre))
    v = y * before
    r1 = 1.0 / np.sqrt(mean(v * v) + eps) if post is not None else 1.0
    vhat = v * r1
    p = vhat * w1
    e = p * after
    res = np.where(on, residual, 0.0) if residual is not None else np.zeros_like(y)
    total, total_size = res + s * e, np.abs(res) + np.abs(s * e)
    r2 = 1.0 / np.sqrt(mean(total * total) + eps) if pre is not None else 1.0
    that, that_size = total * r2, total_size * r2
    r = {"sum": np.where(on, total, 0.0), "out": np.where(on, that * w2, 0.0)}
    z = {"sum": total_size, "out": that_size * np.abs(w2)}
    d = np.zeros_like(y) if d is None else np.where(on, d, 0.0)
    ds = np.zeros_like(y) if dsum is None else np.where(on, dsum, 0.0)
    size = np.abs(ds)
    if pre is not None:
        r["pre"], z["pre"] = (d * that).sum(0), (np.abs(d) * that_size).sum(0)
        dh = d * w2
        ds = ds + r2 * (dh - that * mean(dh * that))
        size = size + r2 * (np.abs(dh) + that_size * mean(np.abs(dh) * that_size))
    elif residual is None:
        ds, size = d, np.abs(d)
    r["residual"], z["residual"] = np.where(on, ds, 0.0), size
    r["scale"], z["scale"] = (ds * e).sum(0), (size * np.abs(e)).sum(0)
    de, de_size = ds * s, size * np.abs(s)
    dp, dp_size = de * after, de_size * np.abs(after)
    r["post"], z["post"] = (dp * vhat).sum(0), (dp_size * np.abs(vhat)).sum(0)
    dh, dh_size = dp * w1, dp_size * np.abs(w1)
    dv = r1 * (dh - vhat * mean(dh * vhat)) if post is not None else dh
    dv_size = r1 * (dh_size + np.abs(vhat) * mean(dh_size * np.abs(vhat))) if post is not None else dh_size
    r["y"], z["y"] = np.where(on, dv * before, 0.0), dv_size * np.abs(before)
    r["gate"] = np.where(on, (dv * y if place == "before" else de * p) * slope, 0.0)
    z["gate"] = (dv_size * np.abs(y) if place == "before" else de_size * np.abs(p)) * steep
    return r, z


def ragged(rng, B, T):
    """Lengths from zero to T: one whole, one empty."""
    n = rng.integers(0, T + 1, B)
    n[rng.integers(B)] = T
    if B > 1:
        n[np.flatnonzero(n < T)[:1]] = 0
    return n


class Given:
    """Tensors as a caller's program has them, and the same values in float64 [B, T, ..].  layout "gaps": every array with gaps between its rows, from a place
    that no wide access likes; "slices": out of one wider array.  Behind lengths there is garbage."""

    def __init__(self, rng, B, T, dtype, time_major, lengths, layout):
        import torch
        self.rng, self.B, self.T, self.dt, self.time_major, self.lengths, self.layout, self.torch = rng, B, T, getattr(torch, dtype), time_major, lengths, layout, torch

    def turn(self, t):
        return t.transpose(0, 1) if self.time_major else t

    def rows(self, *tail, loc=0.0, sd=1.0, garbage=True):
        torch, n = self.torch, int(np.prod(tail))
        host = torch.from_numpy(self.rng.normal(loc, sd, size=(self.B, self.T, n))).to(self.dt)
        ref = host.double().numpy().reshape(self.B, self.T, *tail)
        if self.lengths is not None and garbage:
            for b, k in enumerate(self.lengths):
                host[b, k:] = float("nan") if b % 2 else float("inf")
        host = host.transpose(0, 1) if self.time_major else host
        lead = host.shape[:2]
        if self.layout == "gaps":
            flat = torch.full((lead[0], lead[1] + 2, n + 3), float("nan"), dtype=self.dt, device="cuda")
            view = flat[:, 1:-1, 1:n + 1]
        elif self.layout == "slices":
            view = torch.full((lead[0], lead[1], 2 * n), float("nan"), dtype=self.dt, device="cuda")[..., n:]
        else:
            view = torch.empty((lead[0], lead[1], n), dtype=self.dt, device="cuda")
        view.copy_(host)
        return view.unflatten(-1, tail) if len(tail) > 1 else view, ref

    def floats(self, *size, loc=0.0, sd=1.0):
        t = self.torch.from_numpy(self.rng.normal(loc, sd, size=size)).float()
        return t.cuda(), t.double().numpy()

    def places(self, *tail):
        """An output of the caller's, strided as the layout is, and whether what lies around it is as it was."""
        torch, n = self.torch, int(np.prod(tail))
        lead = (self.T, self.B) if self.time_major else (self.B, self.T)
        flat = torch.full((lead[0], lead[1] + 2, n + 3), 7.0, dtype=self.dt, device="cuda")
        view = flat[:, 1:-1, 1:n + 1]

        def untouched():
            kept = flat.clone()
            kept[:, 1:-1, 1:n + 1] = 7.0
            return bool((kept == 7.0).all())
        return view.unflatten(-1, tail) if len(tail) > 1 else view, untouched
