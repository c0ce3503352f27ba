"""The norms and gates on a residual stream in 64 bits on the CPU, with a bound for how far results may be from it.

A bound follows the fp32 computation from the inputs on, an error beside every value: an operation adds 2^-24 of its result, a sum
DEPTH * 2^-24 of the sum of its terms' sizes: its longest chain is a thread's 8 columns (7 additions, one more for each further
8192), 6 steps over a wave, 15 over a workgroup's waves; or, over rows, the 16 rows that a run has at the sizes tested, 16 runs of a thread
and 5 steps, and the few of several waves' rows: below 48 in any case, and 16 for the terms' own roundings.  A square root and a
division are rounded correctly."""
import torch

from feed_forward_util import EPS32, half, tiny

DEPTH = 64


class V:
    """Values and how far they may be off."""

    def __init__(self, v, e=None):
        self.v, self.e = v, torch.zeros_like(v) if e is None else e

    def __add__(self, o):
        r = self.v + o.v
        return V(r, self.e + o.e + EPS32 * r.abs())

    def __sub__(self, o):
        r = self.v - o.v
        return V(r, self.e + o.e + EPS32 * r.abs())

    def __mul__(self, o):
        if not isinstance(o, V):
            o = V(torch.full_like(self.v, o))
        r = self.v * o.v
        e = self.e * o.v.abs() + self.v.abs() * o.e + self.e * o.e
        return V(r, e + EPS32 * (r.abs() + e))

    def total(self, dim):
        e = self.e.sum(dim, keepdim=True)
        return V(self.v.sum(dim, keepdim=True), e + DEPTH * EPS32 * (self.v.abs().sum(dim, keepdim=True) + e))

    def mean(self):
        t, n = self.total(1), self.v.shape[1]
        return V(t.v / n, t.e / n + EPS32 * t.v.abs() / n)

    def rounded(self, dtype):
        return self.v, self.e + half(dtype) * (self.v.abs() + self.e) + tiny(dtype)


def exactly(t):
    return V(t.double())


def stats(kind, v, eps):
    """The normalised rows and their factor."""
    if kind == "layer":
        v = v - v.mean()
    q = (v * v).mean()
    q = V(q.v + eps, q.e + EPS32 * (q.v + eps))
    r = 1 / q.v.sqrt()
    # d(1/sqrt q) = r / 2 of the relative error of q, and two roundings; an error of all of q leaves no bound
    rel = (q.e / q.v).clamp(max=0.5)
    rstd = V(r, r * (rel / 2 + rel * rel + 3 * EPS32))
    return v * rstd, rstd


def normed(n, w, c):
    y = n if w is None else n * exactly(w)
    return y if c is None else y + exactly(c)


def gate_rows(gate, rows, M):
    return exactly(gate.repeat_interleave(rows, 0)[:M])


def forward(before, after, rows, eps, scale, r, b, gate, w_after, c_after, w_before, c_before):
    s = exactly(r)
    if b is not None:
        p = exactly(b)
        if after != "none":
            p = normed(stats(after, p, eps)[0], w_after, c_after)
        if gate is not None:
            p = p * gate_rows(gate, rows, len(r))
        s = s + p * scale
    out = dict(s=s.rounded(r.dtype))
    if before != "none":
        out["h"] = normed(stats(before, s, eps)[0], w_before, c_before).rounded(r.dtype)
    return out


def _back(kind, d, n, rstd):
    t = d - n * (d * n).mean()
    return (t - d.mean() if kind == "layer" else t) * rstd


def backward(before, after, rows, eps, scale, s, b, gate, w_after, c_after, w_before, ds, dh):
    dt, M = s.dtype, len(s)
    out = {}
    total = exactly(ds) if ds is not None else None
    if dh is not None:
        d = exactly(dh)
        n, rstd = stats(before, exactly(s), eps)
        back = _back(before, normed(d, w_before, None), n, rstd)
        total = back if total is None else total + back
        out.update(dw_before=(d * n).total(0), dc_before=d.total(0))
    out["dr"] = total
    if b is not None:
        dp, p = total * scale, exactly(b)
        if after != "none":
            n, rstd = stats(after, p, eps)
            p = normed(n, w_after, c_after)
        if gate is not None:
            t = dp * p
            groups = -(-M // rows)
            pad = torch.zeros(groups * rows - M, s.shape[1], dtype=torch.float64)
            parts = V(torch.cat([t.v, pad]).view(groups, rows, -1), torch.cat([t.e, pad]).view(groups, rows, -1)).total(1)
            out["dgate"] = V(parts.v[:, 0], parts.e[:, 0])
            dp = dp * gate_rows(gate, rows, M)
        if after != "none":
            out.update(dw_after=(dp * n).total(0), dc_after=dp.total(0))
            dp = _back(after, normed(dp, w_after, None), n, rstd)
        out["db"] = dp
    for k in ("dw_before", "dc_before", "dw_after", "dc_after"):
        if k in out:
            out[k] = V(out[k].v[0], out[k].e[0])
    return {k: v.rounded(dt) for k, v in out.items()}
