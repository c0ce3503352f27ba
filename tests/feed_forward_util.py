"""The feed-forward operators in 64 bits on the CPU, with a bound for how far results may be from it.

A bound is made of: half a step of the result's type (finfo.eps / 2 of its value); the fp32 sums, at most (terms + 8) * 2^-24
of the sum of the products' sizes whatever their order; the activations in fp32, whose exponentials' arguments of up to 40
carry three roundings (40 * 3 * 2^-24 < 1e-5 relative); and the rounding of dz, dg and du to the tensors' type."""
import torch

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ACTS = ["none", "relu", "silu", "gelu", "gelu_tanh"]
EPS32 = 2.0 ** -24
ACT_ERR = 1e-5
SLOPE = 1.13          # the largest |act'|, of gelu and silu


def half(dtype):
    return torch.finfo(dtype).eps / 2


def tiny(dtype):
    """Half the distance of the smallest numbers of a type."""
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2


def rand(g, rows, cols, dtype, std=1.0, pad=0, offset=0):
    """rows x cols on the CPU, cols + pad apart, `offset` values behind the buffer's beginning."""
    flat = (torch.randn(rows * (cols + pad) + offset, generator=g) * std).to(dtype)
    return flat[offset:].view(rows, cols + pad)[:, :cols]


def to_gpu(t):
    """The same values with the same strides and the same offset to an aligned address."""
    off = t.storage_offset()
    flat = torch.zeros(off + (t.shape[0] - 1) * t.stride(0) + t.shape[1] if t.numel() else 0, dtype=t.dtype)
    base = flat.as_strided(t.shape, t.stride(), off) if t.numel() else flat.view(t.shape)
    base.copy_(t)
    gpu = flat.cuda()
    return gpu.as_strided(t.shape, t.stride(), off) if t.numel() else gpu.view(t.shape)


def empty_gpu(rows, cols, dtype, pad=0):
    """NaN everywhere, also between the rows, to see what is written."""
    t = torch.full((max(rows, 1), cols + pad), float("nan"), dtype=dtype, device="cuda")
    return t[:rows, :cols]


def untouched(t, cols):
    """Whether nothing was written between the rows of a tensor made by empty_gpu."""
    base = t._base
    return base is None or base.shape[1] == cols or bool(torch.isnan(base[:, cols:]).all())


def act64(act, z):
    """act(z) and its derivative."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return z.clamp(min=0), (z > 0).double()
    if act == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s))
    if act == "gelu":
        cdf = torch.special.ndtr(z)
        return z * cdf, cdf + z * torch.exp(-z * z / 2) * 0.3989422804014327
    c = 0.7978845608028654
    t = torch.tanh(c * (z + 0.044715 * z ** 3))
    return z * (1 + t) / 2, (1 + t) / 2 + z * (1 - t * t) / 2 * c * (1 + 3 * 0.044715 * z * z)


def product(x, w, bias=None):
    """x w^T + bias and its bound (of the fp32 sum)."""
    x, w = x.double(), w.double()
    z = x @ w.t()
    size = x.abs() @ w.abs().t()
    if bias is not None:
        z, size = z + bias.double(), size + bias.double().abs()
    return z, (x.shape[1] + 8) * EPS32 * size


def rounded(v, err, dtype):
    return v, err + half(dtype) * (v.abs() + err) + tiny(dtype)


def linear_forward(act, x, w, bias, residual):
    dt = x.dtype
    z, ez = product(x, w, bias)
    a, _ = act64(act, z)
    e = SLOPE * ez + ACT_ERR * a.abs()
    y = a if residual is None else a + residual.double()
    return rounded(y, e + EPS32 * y.abs(), dt), rounded(z, ez, dt)


def _grad_product(dz, ez, b, dt):
    """dz^T-free product dz b with dz known to ez."""
    b = b.double()
    v, size = dz @ b, dz.abs() @ b.abs()
    return v, ez @ b.abs() + (dz.shape[1] + 8) * EPS32 * (size + ez @ b.abs())


def linear_backward(act, x, w, z, dy):
    dt = x.dtype
    d = act64(act, z.double())[1] if act != "none" else torch.ones_like(dy.double())
    dz = dy.double() * d
    exact = act in ("none", "relu")
    ez32 = torch.zeros_like(dz) if exact else (ACT_ERR + EPS32) * dy.double().abs() * (d.abs() + 1)
    ez = ez32 if exact else ez32 + half(dt) * (dz.abs() + ez32) + tiny(dt)
    dx = rounded(*_grad_product(dz, ez, w, dt), dt)
    dw = rounded(*_grad_product(dz.t(), ez.t(), x, dt), dt)
    db = dz.sum(0)
    edb = ez32.sum(0) + (dz.shape[0] + 8) * EPS32 * (dz.abs() + ez32).sum(0)
    return dx, dw, rounded(db, edb, dt)


def gated_forward(act, x, wg, wu):
    dt = x.dtype
    (g, eg), (u, eu) = product(x, wg), product(x, wu)
    a, _ = act64(act, g)
    ea = SLOPE * eg + ACT_ERR * a.abs()
    h = a * u
    return rounded(h, ea * u.abs() + a.abs() * eu + ea * eu + EPS32 * h.abs(), dt), rounded(g, eg, dt), rounded(u, eu, dt)


def gated_backward(act, x, wg, wu, g, u, dh):
    dt = x.dtype
    a, d = act64(act, g.double())
    dh64, u64 = dh.double(), u.double()
    dg, du = dh64 * u64 * d, dh64 * a

    def spread(v, e):
        return e + half(dt) * (v.abs() + e) + tiny(dt)
    eg = spread(dg, (ACT_ERR + 3 * EPS32) * (dh64 * u64).abs() * (d.abs() + 1))
    eu = spread(du, (ACT_ERR + 2 * EPS32) * du.abs())
    one, two = _grad_product(dg, eg, wg, dt), _grad_product(du, eu, wu, dt)
    both = dg.abs() @ wg.double().abs() + du.abs() @ wu.double().abs()
    dx = rounded(one[0] + two[0], one[1] + two[1] + (dg.shape[1] + 8) * EPS32 * both, dt)
    return (dx, rounded(*_grad_product(dg.t(), eg.t(), x, dt), dt), rounded(*_grad_product(du.t(), eu.t(), x, dt), dt))


def check(name, got, want):
    value, bound = want
    over = value.abs() >= torch.finfo(got.dtype).max * (1 + half(got.dtype) / 2)   # rounds to an infinity
    got = got.detach().cpu().double()
    assert got.shape == value.shape, (name, got.shape, value.shape)
    assert torch.equal(got[over], value[over].sign() * float("inf")), name
    got, value = got.masked_fill(over, 0.0), value.masked_fill(over, 0.0)
    assert bool(torch.isfinite(got).all()), "%s: %d results are not finite" % (name, int((~torch.isfinite(got)).sum()))
    off = (got - value).abs() - bound
    if got.numel() and float(off.max()) > 0:
        at = int(off.argmax())
        raise AssertionError("%s: %d of %d out of bound; the worst at %d: %.9g, expected %.9g +- %.3g" % (
            name, int((off > 0).sum()), got.numel(), at, got.flatten()[at], value.flatten()[at], bound.flatten()[at]))
