"""What the feed-forward operators, the gradient norm and the weight update refuse, on the host: nothing here has a device, and a
call that got past its checks would end with CCT_EHIP at the latest."""
import ctypes

import pytest

P = 4096          # an address that is only compared and aligned, never read


@pytest.fixture(scope="module")
def B():
    from paper_1504_04343_amd import binding
    return binding


@pytest.mark.parametrize("bad", [dict(M=-1), dict(N=0), dict(K=0), dict(N=-4), dict(type=3), dict(type=-1), dict(activation=5),
                                 dict(activation=-1)])
def test_descriptors(B, bad):
    base = dict(M=8, N=8, K=8, type=1, activation=1)
    base.update(bad)
    d = B.make_linear_desc(**base)
    g = B.make_gated_desc(base["M"], base["N"], base["K"], base["type"], base["activation"])
    for p in (B.PASS_FORWARD, B.PASS_BACKWARD):
        for f, desc in ((B.cct_linear_workspace_bytes, d), (B.cct_gated_workspace_bytes, g)):
            with pytest.raises(B.CctError) as e:
                f(desc, p)
            assert e.value.code == B.EINVAL
    lib = B._lib
    assert lib.cct_linear_forward(ctypes.byref(d), P, 8, P, 8, None, None, 0, P, 8, None, 0, P, 1 << 40, None) == B.EINVAL


def test_sizes_beyond_a_launch(B):
    for sizes in ((2 ** 31 - 256, 2 ** 31 - 256, 8), (2 ** 31 - 1, 8, 8), (8, 2 ** 31 - 1, 8), (8, 8, 2 ** 31 - 255)):
        for make, ask in ((B.make_linear_desc, B.cct_linear_workspace_bytes), (B.make_gated_desc, B.cct_gated_workspace_bytes)):
            for p in (B.PASS_FORWARD, B.PASS_BACKWARD):
                with pytest.raises(B.CctError) as e:
                    ask(make(*sizes, B.TYPE_BF16), p)
                assert e.value.code == B.EUNSUPPORTED
    B.cct_linear_workspace_bytes(B.make_linear_desc(2 ** 31 - 256, 8, 8, B.TYPE_F32), B.PASS_FORWARD)


def linear(B, d, **k):
    a = dict(x=P, ldx=64, w=P, ldw=64, bias=None, r=None, ldr=0, y=P, ldy=64, z=None, ldz=0, ws=P, n=1 << 40)
    a.update(k)
    return B._lib.cct_linear_forward(ctypes.byref(d), a["x"], a["ldx"], a["w"], a["ldw"], a["bias"], a["r"], a["ldr"], a["y"],
                                     a["ldy"], a["z"], a["ldz"], a["ws"], a["n"], None)


def test_linear_forward_refuses(B):
    d = B.make_linear_desc(8, 16, 32, B.TYPE_BF16, B.ACT_GELU)
    for bad in (dict(x=None), dict(w=None), dict(y=None), dict(x=P + 1), dict(w=P + 1), dict(bias=P + 1), dict(ldx=31), dict(ldw=0),
                dict(ldy=15), dict(r=P, ldr=15), dict(r=P + 1, ldr=16), dict(z=P, ldz=3), dict(ws=None), dict(ws=P + 16),
                dict(ldx=-64)):
        assert linear(B, d, **bad) == B.EINVAL, bad
    assert linear(B, d, n=B.cct_linear_workspace_bytes(d, B.PASS_FORWARD) - 1) == B.EWORKSPACE
    assert B._lib.cct_linear_forward(None, P, 64, P, 64, None, None, 0, P, 64, None, 0, P, 1 << 40, None) == B.EINVAL
    assert linear(B, B.make_linear_desc(0, 16, 32, B.TYPE_BF16), x=None, y=None) == B.OK     # an empty batch


def test_linear_backward_refuses(B):
    def call(d, **k):
        a = dict(x=P, ldx=64, w=P, ldw=64, z=P, ldz=64, dy=P, lddy=64, dx=P, lddx=64, dw=P, lddw=64, db=None, ws=P, n=1 << 40)
        a.update(k)
        return B._lib.cct_linear_backward(ctypes.byref(d), *(a[i] for i in (
            "x", "ldx", "w", "ldw", "z", "ldz", "dy", "lddy", "dx", "lddx", "dw", "lddw", "db", "ws", "n")), None)
    d = B.make_linear_desc(8, 16, 32, B.TYPE_F32, B.ACT_RELU)
    for bad in (dict(x=None), dict(w=None), dict(z=None), dict(dy=None), dict(x=P + 2), dict(dx=P + 2), dict(dw=P + 1), dict(db=P + 2),
                dict(ldx=31), dict(ldw=31), dict(ldz=15), dict(lddy=15), dict(lddx=31), dict(lddw=31), dict(ws=None),
                dict(ws=P + 128)):
        assert call(d, **bad) == B.EINVAL, bad
    assert call(d, n=B.cct_linear_workspace_bytes(d, B.PASS_BACKWARD) - 1) == B.EWORKSPACE


def test_gated_refuses(B):
    def forward(d, **k):
        a = dict(x=P, ldx=64, wg=P, ldwg=64, wu=P, ldwu=64, h=P, ldh=64, g=None, ldg=64, u=None, ldu=64, ws=P, n=1 << 40)
        a.update(k)
        return B._lib.cct_gated_forward(ctypes.byref(d), *a.values(), None)

    def backward(d, **k):
        a = dict(x=P, ldx=64, wg=P, ldwg=64, wu=P, ldwu=64, g=P, ldg=64, u=P, ldu=64, dh=P, lddh=64, dx=P, lddx=64, dwg=P, lddwg=64,
                 dwu=P, lddwu=64, ws=P, n=1 << 40)
        a.update(k)
        return B._lib.cct_gated_backward(ctypes.byref(d), *a.values(), None)
    d = B.make_gated_desc(8, 16, 32, B.TYPE_F16, B.ACT_SILU)
    for bad in (dict(x=None), dict(wg=None), dict(wu=None), dict(h=None), dict(g=P), dict(u=P), dict(g=P, u=P, ldg=1),
                dict(g=P, u=P + 1), dict(ldx=31), dict(ldwu=31), dict(ldh=15), dict(ws=None), dict(ws=P + 8)):
        assert forward(d, **bad) == B.EINVAL, bad
    assert forward(d, n=B.cct_gated_workspace_bytes(d, B.PASS_FORWARD) - 1) == B.EWORKSPACE
    for bad in (dict(x=None), dict(wg=None), dict(wu=None), dict(g=None), dict(u=None), dict(dh=None), dict(dwg=None), dict(dwu=None),
                dict(dx=P + 1), dict(lddx=31), dict(lddwg=31), dict(lddwu=31), dict(ldg=15), dict(ldu=15), dict(lddh=15),
                dict(ws=None)):
        assert backward(d, **bad) == B.EINVAL, bad
    assert backward(d, n=B.cct_gated_workspace_bytes(d, B.PASS_BACKWARD) - 1) == B.EWORKSPACE
    assert backward(d, dx=None, dwg=None, dwu=None) == B.OK                                   # nothing is asked for


def test_lists_refuse(B):
    def lst(*ts):
        return (B.Tensor * max(1, len(ts)))(*(B.Tensor(*t, 0) for t in ts))
    lib, n = B._lib, ctypes.c_size_t()
    good, w = lst((P, 100, 1), (P, 7, 0)), lst((P, 100, 0), (P, 7, 0))
    assert lib.cct_grad_norm_workspace_bytes(good, 2, ctypes.byref(n)) == B.OK and n.value >= 16
    assert lib.cct_grad_norm(good, 2, 1.0, P, P, n.value - 1, None) == B.EWORKSPACE
    for bad in (lst((P, -1, 0), (P, 7, 0)), lst((None, 3, 0), (P, 7, 0)), lst((P, 3, 5), (P, 7, 0)), lst((P + 2, 3, 0), (P, 7, 0)),
                lst((P + 1, 3, 1), (P, 7, 0))):
        assert lib.cct_grad_norm_workspace_bytes(bad, 2, ctypes.byref(n)) == B.EINVAL
        assert lib.cct_grad_norm(bad, 2, 1.0, P, P, 1 << 30, None) == B.EINVAL
        assert lib.cct_grad_scale(bad, 2, P, bad, None) == B.EINVAL
        assert lib.cct_grad_scale(good, 2, P, bad, None) == B.EINVAL
        assert lib.cct_sgd_update(good, 2, P, bad, w, None, 0.1, 0.9, 0.0, None) == B.EINVAL
        assert lib.cct_sgd_update(good, 2, P, w, w, bad, 0.1, 0.9, 0.0, None) == B.EINVAL
    nan = float("nan")
    for limit in (0.0, -1.0, nan):
        assert lib.cct_grad_norm(good, 2, limit, P, P, 1 << 30, None) == B.EINVAL
    for args in ((good, 2, 1.0, None, P, 1 << 30), (good, 2, 1.0, P, None, 1 << 30), (good, 2, 1.0, P, P + 8, 1 << 30),
                 (good, -1, 1.0, P, P, 1 << 30), (None, 2, 1.0, P, P, 1 << 30)):
        assert lib.cct_grad_norm(*args, None) == B.EINVAL
    assert lib.cct_grad_scale(good, 2, None, good, None) == B.EINVAL
    assert lib.cct_grad_scale(good, 2, P, w, None) == B.EINVAL                        # another type
    assert lib.cct_sgd_update(good, 2, P, lst((P, 99, 0), (P, 7, 0)), w, None, 0.1, 0.9, 0.0, None) == B.EINVAL
    assert lib.cct_sgd_update(good, 2, P, good, w, None, 0.1, 0.9, 0.0, None) == B.EINVAL   # weights are fp32
    for rule in ((nan, 0.9, 0.0), (0.1, nan, 0.0), (0.1, 0.9, float("inf"))):
        assert lib.cct_sgd_update(good, 2, P, w, w, None, *rule, None) == B.EINVAL


def test_the_binding_looks_at_tensors(B):
    import torch
    d = B.make_linear_desc(4, 8, 16, B.TYPE_BF16)
    cpu = torch.zeros(4, 16, dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        B.cct_linear_forward(d, cpu, cpu, None, None, cpu, None, cpu)
    with pytest.raises(ValueError):
        B.cct_linear_forward(d, None, cpu, None, None, cpu, None, cpu)
    with pytest.raises(TypeError):
        B.make_tensor_list([cpu])
    with pytest.raises(B.CctError):
        B.cct_linear_forward(B.make_linear_desc(4, 8, 16, 9), cpu, cpu, None, None, cpu, None, cpu)


def test_sizes_of_matrices_that_fit_a_card(B):
    """What is refused is a matrix that no card holds, not two sizes that no matrix has."""
    def ask(M, N, K, type):
        out = set()
        for make, f in ((B.make_linear_desc, B.cct_linear_workspace_bytes), (B.make_gated_desc, B.cct_gated_workspace_bytes)):
            for p in (B.PASS_FORWARD, B.PASS_BACKWARD):
                try:
                    assert f(make(M, N, K, type), p) > 0
                    out.add(B.OK)
                except B.CctError as e:
                    out.add(e.code)
        assert len(out) == 1
        return out.pop()
    for type in (B.TYPE_F32, B.TYPE_BF16, B.TYPE_F16):
        for sizes in ((8, 3000000, 8), (8, 8, 3000000), (1, 2 ** 31 - 256, 8), (2 ** 31 - 256, 1, 1), (1, 1, 2 ** 31 - 256),
                      (1 << 24, 64, 1 << 12)):
            assert ask(*sizes, type) == B.OK, sizes
        for sizes in ((1 << 20, 1 << 20, 8), (8, 1 << 20, 1 << 20), (1 << 20, 8, 1 << 20)):
            assert ask(*sizes, type) == B.EUNSUPPORTED, sizes
    assert ask(1 << 19, 1 << 18, 8, B.TYPE_BF16) == B.OK
    assert ask(1 << 19, 1 << 18, 8, B.TYPE_F32) == B.EUNSUPPORTED


def test_tensors_beyond_a_launch(B):
    """A launch takes 2^24 - 1 workgroups of 8192 values (the update: 4096); more in one tensor are refused, in several not."""
    lib, n = B._lib, ctypes.c_size_t()

    def lst(*sizes, type=1):
        return (B.Tensor * len(sizes))(*(B.Tensor(P, s, type, 0) for s in sizes))
    most = ((1 << 24) - 1) * 8192
    assert lib.cct_grad_norm_workspace_bytes(lst(most), 1, ctypes.byref(n)) == B.OK and n.value == 8 * ((1 << 24) - 1)
    assert lib.cct_grad_norm_workspace_bytes(lst(most, most), 2, ctypes.byref(n)) == B.OK
    for more in (most + 1, 1 << 40):
        assert lib.cct_grad_norm_workspace_bytes(lst(5, more), 2, ctypes.byref(n)) == B.EUNSUPPORTED
        assert lib.cct_grad_norm(lst(5, more), 2, 1.0, P, P, 1 << 60, None) == B.EUNSUPPORTED
        assert lib.cct_grad_scale(lst(5, more), 2, P, lst(5, more), None) == B.EUNSUPPORTED
    w = lst(most // 2 + 1, type=0)
    assert lib.cct_sgd_update(lst(most // 2 + 1), 1, P, w, w, None, 0.1, 0.9, 0.0, None) == B.EUNSUPPORTED


def test_workspace_is_what_a_call_may_need(B):
    """A forward pass of up to 16 rows (fp32: 32) copies nothing, whatever its operands' addresses; an fp32 gradient whose
    contraction is not cut is stored without partial sums."""
    def linear(M, N, K, type, p):
        return B.cct_linear_workspace_bytes(B.make_linear_desc(M, N, K, type, B.ACT_RELU), p)

    def gated(M, N, K, type, p):
        return B.cct_gated_workspace_bytes(B.make_gated_desc(M, N, K, type), p)
    for type, most in ((B.TYPE_BF16, 16), (B.TYPE_F16, 16), (B.TYPE_F32, 32)):
        for M in (1, most):
            assert linear(M, 4096, 4096, type, B.PASS_FORWARD) == 256
            assert gated(M, 8192, 4096, type, B.PASS_FORWARD) == 256
    assert linear(17, 4096, 4096, B.TYPE_BF16, B.PASS_FORWARD) >= (17 + 4096) * 4096 * 2   # copies
    # partial sums of few columns of long rows
    assert linear(16, 64, 9216, B.TYPE_BF16, B.PASS_FORWARD) > 256
    # dz, its column sums (one row of 64), a packed operand of three terms
    n = 8192 * 8192
    assert 0 <= linear(8192, 8192, 8192, B.TYPE_F32, B.PASS_BACKWARD) - (4 * n + 4 * n // 64 + 6 * n) < 1024


def test_workspace_of_the_largest_sizes(B):
    """Counts of workgroups and of rows of partial sums next to 2^31: negative ones made the workspace smaller."""
    for type, size in ((B.TYPE_F32, 4), (B.TYPE_BF16, 2)):
        for n in ((1 << 30) - 8, (1 << 30) + 104, (1 << 31) - 2048, (1 << 31) - 1024, (1 << 31) - 512, (1 << 31) - 256):
            for i in range(3):
                dims = [n if k == i else 1 for k in range(3)]
                for p in (B.PASS_FORWARD, B.PASS_BACKWARD):
                    assert B.cct_gated_workspace_bytes(B.make_gated_desc(*dims, type), p) >= 256
                # dz in rows of 8 values
                assert B.cct_linear_workspace_bytes(B.make_linear_desc(*dims, type), B.PASS_BACKWARD) >= \
                    dims[0] * -(-dims[1] // 8) * 8 * size, dims
            rows = 64                   # of a workgroup of dz, which leaves one of column sums; of these at most 2^21
            while -(-n // rows) > 1 << 21:
                rows *= 2
            # dz, the sums, and x's copy in such rows or 2^30 bytes of dz as three terms of 32 steps, 64 rows at a time
            least = n * 8 * size + -(-n // rows) * 4 + (n * 8 * size if size == 2 else (1 << 30) // 192 // 64 * 64 * 192)
            total = B.cct_linear_workspace_bytes(B.make_linear_desc(n, 1, 1, type), B.PASS_BACKWARD)
            assert least <= total < least + (1 << 16), (n, type, total, least)
