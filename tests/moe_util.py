"""A layer of experts in 64 bits on the CPU, with a bound for how far results may be from it: feed_forward_util.py's of the
gated products; a weight's exponentials (arguments of up to 40 with a rounding each, 2^-24 * 40, and a few of the sum and the
division: below 1e-5); weight * h as two terms of the type, which keep it to half a step of half a step; and the fp32 sums over
all chosen experts' features, two products each."""
import torch

import feed_forward_util as ff

WEIGHT_ERR = 1e-5


def route(x, router, k, normalize):
    """Logits as fp32, the chosen experts (largest first, ties to the lower, NaN last), their weights."""
    logits = (x.double() @ router.double().t()).float()
    T, E = logits.shape
    keys = [sorted(range(E), key=lambda e: (bool(torch.isnan(logits[t, e])), -float(logits[t, e].nan_to_num(0.0)), e)) for t in range(T)]
    chosen = torch.tensor([r[:k] for r in keys])
    v = logits.double()
    e = torch.exp(v - v.gather(1, chosen[:, :1]))
    top = e.gather(1, chosen)
    return logits, chosen, top / (top if normalize else e).sum(1, keepdim=True)


def forward(act, x, router, wg, wu, wd, k, normalize, residual):
    dt, (T, D) = x.dtype, x.shape
    _, chosen, weights = route(x, router, k, normalize)
    y = torch.zeros(T, D, dtype=torch.float64)
    err, size = y.clone(), y.clone()
    for e in chosen.unique().tolist():
        t, j = (chosen == e).nonzero(as_tuple=True)
        (g, eg), (u, eu) = ff.product(x[t], wg[e]), ff.product(x[t], wu[e])
        a = ff.act64(act, g)[0]
        ea = ff.SLOPE * eg + ff.ACT_ERR * a.abs()
        w = weights[t, j][:, None]
        h = w * a * u
        eh = w * (ea * u.abs() + a.abs() * eu + ea * eu) + (WEIGHT_ERR + 3 * ff.EPS32) * h.abs()
        eh = eh + (0.0 if dt is torch.float32 else ff.half(dt) ** 2) * (h.abs() + eh) + (0.0 if dt is torch.float32 else ff.tiny(dt))
        v = wd[e].double()
        y[t] += h @ v.t()
        err[t] += eh @ v.abs().t()
        size[t] += (h.abs() + eh) @ v.abs().t()
    err = err + (2 * k * wd.shape[2] + 8) * ff.EPS32 * size
    if residual is not None:
        y = y + residual.double()
        err = err + ff.EPS32 * y.abs()
    return ff.rounded(y, err, dt), chosen, weights
