"""Microscaled 4-bit floating point on the CPU, in 64 bits and by tables."""
import torch

VALUES = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def blocks_of(cols):
    return -(-cols // 32)


def exponents(most):
    """floor(log2(most)) - 2, at least -127; most > 0 finite."""
    return (torch.frexp(most)[1] - 3).clamp(min=-127)


def quantize(x):
    """Codes (a byte each, rows x whole blocks) and scales (rows x blocks)."""
    rows, cols = x.shape
    n = blocks_of(cols)
    v = torch.zeros(rows, n * 32, dtype=torch.float64)
    v[:, :cols] = x.double()
    v = v.view(rows, n, 32)
    odd = ~torch.isfinite(v).all(2)
    v = v.masked_fill(odd[:, :, None], 0.0)
    most = v.abs().amax(2)
    e = torch.where(most > 0, exponents(most), torch.full_like(most, -127).int())
    a = torch.ldexp(v.abs(), -e[:, :, None])
    # the nearest of the eight; from two as near the one of even number
    off = (a[..., None] - VALUES).abs()
    near = off == off.amin(-1, keepdim=True)
    even = near & (torch.arange(8) % 2 == 0)
    code = torch.where(even.any(-1), even.int().argmax(-1), near.int().argmax(-1))
    code = code + 8 * torch.signbit(v).int()
    code = code.masked_fill(odd[:, :, None], 0)
    scale = torch.where(odd, 255, e + 127)
    return code.view(rows, n * 32).to(torch.uint8), scale.to(torch.uint8)


def pack(code):
    return code[:, 0::2] | code[:, 1::2] << 4


def unpack(codes):
    return torch.stack([codes & 15, codes >> 4], 2).view(codes.shape[0], -1)


def values(code, scale, cols):
    """What codes (a byte each) and scales stand for, 64 bits."""
    rows = code.shape[0]
    v = VALUES[(code & 7).long()] * torch.where(code >= 8, -1.0, 1.0)
    s = torch.ldexp(torch.ones(scale.shape, dtype=torch.float64), scale.int() - 127)
    s = torch.where(scale == 255, float("nan"), s)
    return (v.view(rows, -1, 32) * s[:, :, None]).view(rows, -1)[:, :cols]
