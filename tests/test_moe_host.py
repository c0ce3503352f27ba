"""What a layer of experts refuses, on the host, and the tests' own routing."""
import ctypes

import pytest
import torch

import moe_util as moe

P = 4096          # an address that is only compared and aligned, never read


@pytest.fixture(scope="module")
def B():
    from paper_1504_04343_amd import binding
    return binding


def call(B, d, **k):
    a = dict(x=P, ldx=64, router=P, ldrouter=64, wg=P, ldwg=64, wg_e=4096, wu=P, ldwu=64, wu_e=4096, wd=P, ldwd=64, wd_e=4096, r=None, ldr=0,
             y=P, ldy=64, chosen=None, weights=None, ws=P, n=1 << 40)
    a.update(k)
    return B._lib.cct_moe_forward(ctypes.byref(d), *a.values(), None)


BASE = dict(tokens=8, experts=6, chosen=2, D=32, F=48, type=1, activation=2)


@pytest.mark.parametrize("bad", [dict(tokens=-1), dict(experts=0), dict(chosen=0), dict(chosen=7), dict(D=0), dict(F=-1), dict(type=3),
                                 dict(activation=5), dict(activation=-1)])
def test_descriptors(B, bad):
    d = B.make_moe_desc(**dict(BASE, **bad))
    assert call(B, d) == B.EINVAL
    with pytest.raises(B.CctError) as e:
        B.cct_moe_workspace_bytes(d)
    assert e.value.code == B.EINVAL


@pytest.mark.parametrize("big", [dict(tokens=65), dict(experts=513), dict(experts=40, chosen=17), dict(D=(1 << 24) + 1), dict(F=(1 << 24) + 1),
                                 dict(D=1 << 20, F=1 << 20)])
def test_sizes(B, big):
    d = B.make_moe_desc(**dict(BASE, **big))
    assert call(B, d, ldx=1 << 25, ldrouter=1 << 25) == B.EUNSUPPORTED
    with pytest.raises(B.CctError) as e:
        B.cct_moe_workspace_bytes(d)
    assert e.value.code == B.EUNSUPPORTED


def test_refuses(B):
    d = B.make_moe_desc(**BASE)
    for bad in [{n: None} for n in ("x", "router", "wg", "wu", "wd", "y", "ws")] + [{n: P + 1} for n in ("x", "router", "wg", "wu", "wd", "y")] + \
            [dict(ldx=31), dict(ldrouter=31), dict(ldwg=31), dict(ldwu=31), dict(ldwd=47), dict(ldy=31), dict(wg_e=64 * 47 + 31),
             dict(wu_e=0), dict(wd_e=64 * 31 + 47), dict(wg_e=-1), dict(ldwd=1 << 39, wd_e=1 << 62), dict(r=P, ldr=31), dict(r=P + 1, ldr=32),
             dict(chosen=P + 2), dict(weights=P + 1), dict(ws=P + 128)]:
        assert call(B, d, **bad) == B.EINVAL, bad
    assert call(B, d, n=B.cct_moe_workspace_bytes(d) - 1) == B.EWORKSPACE
    assert B._lib.cct_moe_forward(None, *[P, 64] * 2, *[P, 64, 64] * 3, None, 0, P, 64, None, None, P, 1 << 40, None) == B.EINVAL
    assert B._lib.cct_moe_workspace_bytes(ctypes.byref(d), None) == B.EINVAL
    assert call(B, B.make_moe_desc(**dict(BASE, tokens=0)), x=None, y=None) == B.OK


def test_workspace(B):
    """h in two terms of 16 bits or one of 32: the same bytes, in rows of whole steps."""
    for type in (0, 1, 2):
        n = B.cct_moe_workspace_bytes(B.make_moe_desc(64, 512, 16, 1 << 12, 1531, type))
        assert 0 <= n - (64 * 16 * 1536 * 4 + 64 * 512 * 4 + 64 * 16 * (2 + 4) + 512 * (8 + 64 * 2) + 64 * 16 * 4096 * 4) < 8 * 256
    assert B.cct_moe_workspace_bytes(B.make_moe_desc(0, 4, 2, 8, 8)) == 256


def test_the_binding_looks_at_tensors(B):
    d = B.make_moe_desc(2, 3, 1, 8, 16, B.TYPE_F32)
    cpu = torch.zeros(2, 8)
    with pytest.raises(TypeError):
        B.cct_moe_forward(d, cpu, cpu, None, None, None, None, cpu, None, None, cpu)


def test_routing():
    x = torch.tensor([[1.0, 0.0], [0.0, 1.0], [1.0, 1.0]])
    router = torch.tensor([[1.0, 3.0], [2.0, 3.0], [2.0, float("nan")], [-1.0, 3.0]])
    logits, chosen, weights = moe.route(x, router, 2, True)
    assert chosen[0].tolist() == [1, 0]                      # of 1, 2, NaN (0 * NaN is one) and -1
    assert chosen[1].tolist() == [0, 1] and torch.allclose(weights[1], torch.tensor([0.5, 0.5], dtype=torch.float64))
    assert chosen[2].tolist() == [1, 0]
