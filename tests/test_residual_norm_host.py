"""The norms and gates on a residual stream without a device: what the entry points refuse, and the tests' own formulas against
automatic differentiation in 64 bits."""
import ctypes

import pytest
import torch

import residual_norm_util as rn

P = 4096          # an address that is only compared and aligned, never read


@pytest.fixture(scope="module")
def B():
    from paper_1504_04343_amd import binding
    return binding


@pytest.mark.parametrize("bad", [dict(M=-1), dict(D=0), dict(D=-3), dict(type=3), dict(type=-1), dict(before=3), dict(after=-1),
                                 dict(gate_rows=0), dict(gate_rows=-2), dict(eps=-1e-6), dict(eps=float("nan")),
                                 dict(eps=float("inf")), dict(scale=float("nan")), dict(scale=float("-inf"))])
def test_descriptors(B, bad):
    d = B.make_residual_norm_desc(**dict(dict(M=8, D=16, type=1), **bad))
    with pytest.raises(B.CctError) as e:
        B.cct_residual_norm_workspace_bytes(d)
    assert e.value.code == B.EINVAL
    assert forward(B, d) == B.EINVAL and backward(B, d) == B.EINVAL
    assert B._lib.cct_residual_norm_workspace_bytes(None, ctypes.byref(ctypes.c_size_t())) == B.EINVAL


def test_sizes(B):
    for M, D, type in ((2 ** 31 - 255, 1, 0), (1, 2 ** 31 - 1, 1), (1 << 20, 1 << 18, 1), (1 << 19, 1 << 18, 0)):
        with pytest.raises(B.CctError) as e:
            B.cct_residual_norm_workspace_bytes(B.make_residual_norm_desc(M, D, type))
        assert e.value.code == B.EUNSUPPORTED
    for M, D, rows in ((2 ** 31 - 256, 8, 1), (2 ** 31 - 256, 8, 2 ** 31 - 1), (1, 2 ** 31 - 256, 1), (1 << 19, 1 << 18, 1 << 18),
                       (0, 8, 1), (1, 1, 2 ** 31 - 1)):
        for type in (1, 2):
            n = B.cct_residual_norm_workspace_bytes(B.make_residual_norm_desc(M, D, type, gate_rows=rows))
            assert 256 <= n < 1 << 45


def forward(B, d, **k):
    a = dict(r=P, ldr=64, b=P, ldb=64, gate=P, ldgate=64, w_after=P, c_after=P, w_before=P, c_before=P, s=P, lds=64, h=P, ldh=64)
    a.update(k)
    return B._lib.cct_residual_norm_forward(ctypes.byref(d), *a.values(), None)


def backward(B, d, **k):
    a = dict(s=P, lds=64, b=P, ldb=64, gate=P, ldgate=64, w_after=P, c_after=P, w_before=P, ds=P, ldds=64, dh=P, lddh=64, dr=P,
             lddr=64, db=P, lddb=64, dgate=P, lddgate=64, dw_after=P, dc_after=P, dw_before=P, dc_before=P, ws=P, n=1 << 40)
    a.update(k)
    return B._lib.cct_residual_norm_backward(ctypes.byref(d), *a.values(), None)


def test_forward_refuses(B):
    d = B.make_residual_norm_desc(8, 32, B.TYPE_BF16, B.NORM_RMS, B.NORM_LAYER, 3)
    names = ("r", "b", "gate", "s", "h")
    for bad in [dict(r=None)] + [{n: P + 1} for n in names] + [{"ld" + n: 31} for n in names] + [dict(ldr=-64)] + \
            [{v: P + 1} for v in ("w_after", "c_after", "w_before", "c_before")] + \
            [dict(b=None), dict(b=None, gate=None), dict(b=None, gate=None, w_after=None)]:
        assert forward(B, d, **bad) == B.EINVAL, bad
    assert B._lib.cct_residual_norm_forward(None, *[P, 64] * 3, *[P] * 4, *[P, 64] * 2, None) == B.EINVAL
    none = B.make_residual_norm_desc(8, 32, B.TYPE_BF16, B.NORM_NONE, B.NORM_NONE, 3)
    off = dict(w_after=None, c_after=None, w_before=None, c_before=None, h=None)
    for n in off:
        assert forward(B, none, **dict(off, **{n: P})) == B.EINVAL, n
    assert forward(B, none, **dict(off, s=None)) == B.OK                                     # nothing is asked for
    assert forward(B, B.make_residual_norm_desc(0, 32, B.TYPE_BF16, after=1), r=None, s=None) == B.OK   # no rows


def test_backward_refuses(B):
    d = B.make_residual_norm_desc(8, 32, B.TYPE_F16, B.NORM_RMS, B.NORM_LAYER, 3)
    names = ("s", "b", "gate", "ds", "dh", "dr", "db", "dgate")
    for bad in [{n: P + 1} for n in names] + [{"ld" + n: 31} for n in names] + \
            [{v: P + 1} for v in ("w_after", "c_after", "w_before", "dw_after", "dc_after", "dw_before", "dc_before")] + \
            [dict(s=None), dict(b=None), dict(gate=None), dict(ds=None, dh=None), dict(ws=None), dict(ws=P + 128)]:
        assert backward(B, d, **bad) == B.EINVAL, bad
    assert backward(B, d, n=B.cct_residual_norm_workspace_bytes(d) - 1) == B.EWORKSPACE
    none = B.make_residual_norm_desc(8, 32, B.TYPE_F16, B.NORM_NONE, B.NORM_NONE, 3)
    off = dict(w_after=None, c_after=None, w_before=None, dh=None, dw_after=None, dc_after=None, dw_before=None, dc_before=None)
    for n in off:
        assert backward(B, none, **dict(off, **{n: P})) == B.EINVAL, n
    assert backward(B, none, **dict(off, b=None)) == B.EINVAL                                # dgate needs it


def test_the_binding_looks_at_tensors(B):
    d = B.make_residual_norm_desc(4, 16, B.TYPE_F32)
    cpu = torch.zeros(4, 16)
    with pytest.raises(TypeError):
        B.cct_residual_norm_forward(d, cpu, None, None, None, None, None, None, None, cpu)
    with pytest.raises(ValueError):
        B.cct_residual_norm_forward(d, None, None, None, None, None, None, None, None, None)


def definition(before, after, rows, eps, scale, r, b, gate, w_after, c_after, w_before, c_before):
    def norm(kind, v, w, c):
        if kind == "none":
            return v
        if kind == "layer":
            return torch.nn.functional.layer_norm(v, v.shape[1:], w, c, eps)
        return v / ((v ** 2).mean(1, keepdim=True) + eps).sqrt() * w + c
    p = norm(after, b, w_after, c_after) * gate[torch.arange(len(r)) // rows]
    s = r + scale * p
    return s, norm(before, s, w_before, c_before)


@pytest.mark.parametrize("before", ["rms", "layer", "none"])
@pytest.mark.parametrize("after", ["rms", "layer", "none"])
@pytest.mark.parametrize("rows", [1, 3, 7, 100])
def test_formulas(before, after, rows):
    g = torch.Generator().manual_seed(rows)
    M, D, eps, scale = 7, 12, 1e-3, -0.7
    t = {n: torch.randn(M, D, generator=g, dtype=torch.float64) for n in ("r", "b", "ds", "dh")}
    gate = torch.randn(-(-M // rows), D, generator=g, dtype=torch.float64).requires_grad_()
    w = {n: torch.randn(D, generator=g, dtype=torch.float64).requires_grad_() for n in ("w_after", "c_after", "w_before", "c_before")}
    t["r"].requires_grad_()
    t["b"].requires_grad_()
    s, h = definition(before, after, rows, eps, scale, t["r"], t["b"], gate, **w)
    no_h, no_n = before == "none", after == "none"
    leaves = dict(dr=t["r"], db=t["b"], dgate=gate)
    if not no_n:
        leaves.update(dw_after=w["w_after"], dc_after=w["c_after"])
    if not no_h:
        leaves.update(dw_before=w["w_before"], dc_before=w["c_before"])
    want = dict(zip(leaves, torch.autograd.grad([s] + [h] * (not no_h), list(leaves.values()), [t["ds"]] + [t["dh"]] * (not no_h))))
    w = {k: v.detach() for k, v in w.items()}
    if no_n:
        w.update(w_after=None, c_after=None)
    if no_h:
        w.update(w_before=None, c_before=None)
    s, h, b, gate = s.detach(), h.detach(), t["b"].detach(), gate.detach()
    out = rn.forward(before, after, rows, eps, scale, t["r"].detach(), b, gate, **w)
    assert torch.allclose(out["s"][0], s, rtol=1e-12, atol=1e-12) and (no_h or torch.allclose(out["h"][0], h, rtol=1e-12, atol=1e-12))
    c_before = w.pop("c_before")
    got = rn.backward(before, after, rows, eps, scale, s, b, gate, ds=t["ds"], dh=None if no_h else t["dh"], **w)
    assert set(got) == set(want) and (c_before is None) == no_h
    for k in want:
        assert torch.allclose(got[k][0], want[k], rtol=1e-10, atol=1e-12), k
