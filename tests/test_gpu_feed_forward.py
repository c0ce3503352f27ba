"""The products of feed-forward blocks (cct_linear_*, cct_gated_*) against 64 bits on the CPU, within bounds derived from the
types (feed_forward_util.py): every type and activation, one row to several hundred, odd sizes, strides and addresses, empty
batches, values that are not finite, captured graphs, another stream, offsets beyond 32 bits, and differences."""
import pytest
import torch

import feed_forward_util as ff

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available()
    from paper_1504_04343_amd import binding
    return binding


def consts(B, type, act):
    return (dict(f32=B.TYPE_F32, bf16=B.TYPE_BF16, f16=B.TYPE_F16)[type],
            dict(none=B.ACT_NONE, relu=B.ACT_RELU, silu=B.ACT_SILU, gelu=B.ACT_GELU, gelu_tanh=B.ACT_GELU_TANH)[act])


def linear_forward(B, type, act, x, w, bias, residual, save, pad=0):
    M, K = x.shape
    N = w.shape[0]
    t, a = consts(B, type, act)
    d = B.make_linear_desc(M, N, K, t, a)
    y = ff.empty_gpu(M, N, x.dtype, pad)
    z = ff.empty_gpu(M, N, x.dtype, pad) if save else None
    B.cct_linear_forward(d, ff.to_gpu(x), ff.to_gpu(w), None if bias is None else bias.cuda(),
                         None if residual is None else ff.to_gpu(residual), y, z, B.alloc_linear_workspace(d, B.PASS_FORWARD))
    torch.cuda.synchronize()
    assert ff.untouched(y, N) and (z is None or ff.untouched(z, N))
    return y, z


def linear_backward(B, type, act, x, w, z, dy, pad=0, want=("dx", "dw", "dbias")):
    (M, K), N = x.shape, w.shape[0]
    t, a = consts(B, type, act)
    d = B.make_linear_desc(M, N, K, t, a)
    dx = ff.empty_gpu(M, K, x.dtype, pad) if "dx" in want else None
    dw = ff.empty_gpu(N, K, x.dtype, pad) if "dw" in want else None
    db = torch.full((N,), float("nan"), dtype=x.dtype, device="cuda") if "dbias" in want else None
    ws = B.alloc_linear_workspace(d, B.PASS_BACKWARD)
    ws.fill_(0xff)   # nothing that a workspace holds before the call may matter
    B.cct_linear_backward(d, ff.to_gpu(x) if dw is not None else None, ff.to_gpu(w) if dx is not None else None,
                          None if z is None else ff.to_gpu(z), ff.to_gpu(dy), dx, dw, db, ws)
    torch.cuda.synchronize()
    assert (dx is None or ff.untouched(dx, K)) and (dw is None or ff.untouched(dw, K))
    return dx, dw, db


def gated_forward(B, type, act, x, wg, wu, save, pad=0):
    (M, K), F = x.shape, wg.shape[0]
    t, a = consts(B, type, act)
    d = B.make_gated_desc(M, F, K, t, a)
    h = ff.empty_gpu(M, F, x.dtype, pad)
    g, u = (ff.empty_gpu(M, F, x.dtype, pad), ff.empty_gpu(M, F, x.dtype, pad)) if save else (None, None)
    ws = B.alloc_gated_workspace(d, B.PASS_FORWARD)
    ws.fill_(0xff)
    B.cct_gated_forward(d, ff.to_gpu(x), ff.to_gpu(wg), ff.to_gpu(wu), h, g, u, ws)
    torch.cuda.synchronize()
    assert ff.untouched(h, F)
    return h, g, u


def gated_backward(B, type, act, x, wg, wu, g, u, dh, pad=0):
    (M, K), F = x.shape, wg.shape[0]
    t, a = consts(B, type, act)
    d = B.make_gated_desc(M, F, K, t, a)
    dx, dwg, dwu = (ff.empty_gpu(r, K, x.dtype, pad) for r in (M, F, F))
    ws = B.alloc_gated_workspace(d, B.PASS_BACKWARD)
    ws.fill_(0xff)
    B.cct_gated_backward(d, *(ff.to_gpu(t) for t in (x, wg, wu, g, u, dh)), dx, dwg, dwu, ws)
    torch.cuda.synchronize()
    assert all(ff.untouched(t, K) for t in (dx, dwg, dwu))
    return dx, dwg, dwu


# M, N, K, elements between the rows' ends and beginnings, elements in front of the first row
SHAPES = [(1, 1, 1, 0, 0), (1, 7, 3, 0, 0), (1, 64, 256, 0, 0), (2, 33, 1000, 0, 0), (3, 130, 515, 1, 1), (5, 300, 72, 8, 0),
          (16, 48, 2048, 0, 0), (17, 257, 129, 0, 0), (31, 64, 40, 64, 8), (33, 520, 136, 0, 2), (64, 96, 1024, 0, 0),
          (65, 72, 7, 5, 0), (100, 1000, 64, 0, 0), (128, 128, 128, 0, 0), (129, 136, 264, 8, 8), (257, 300, 70, 3, 1),
          (300, 520, 512, 0, 0), (513, 264, 72, 0, 0)]
IDS = ["%dx%dx%d+%d@%d" % s for s in SHAPES]


@pytest.mark.parametrize("type", list(ff.TYPES))
@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
def test_linear(B, type, shape):
    M, N, K, pad, off = shape
    i = SHAPES.index(shape)
    g = torch.Generator().manual_seed(i)
    dt = ff.TYPES[type]
    act = ff.ACTS[i % 5]
    x, w = ff.rand(g, M, K, dt, 1.0, pad, off), ff.rand(g, N, K, dt, K ** -0.5, pad, off)
    bias = ff.rand(g, 1, N, dt, 0.3).view(N) if i % 3 else None
    residual = ff.rand(g, M, N, dt, 1.0, pad, off) if i % 2 else None
    y, z = linear_forward(B, type, act, x, w, bias, residual, True, pad)
    want = ff.linear_forward(act, x, w, bias, residual)
    ff.check("y", y, want[0])
    ff.check("z", z, want[1])
    y2, _ = linear_forward(B, type, act, x, w, bias, residual, False, pad)
    assert torch.equal(y, y2)
    dy = ff.rand(g, M, N, dt, 0.3, pad, off)
    zs = z.cpu() if act != "none" else None
    got = linear_backward(B, type, act, x, w, zs, dy, pad)
    for name, t, v in zip(("dx", "dw", "dbias"), got, ff.linear_backward(act, x, w, zs, dy)):
        ff.check(name, t, v)
    again = linear_backward(B, type, act, x, w, zs, dy, pad)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    # one at a time, and what is not needed left out
    for name, t in zip(("dx", "dw", "dbias"), got):
        alone = linear_backward(B, type, act, x, w, zs, dy, pad, (name,))
        assert torch.equal(alone[("dx", "dw", "dbias").index(name)], t), name


@pytest.mark.parametrize("type", list(ff.TYPES))
@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
def test_gated(B, type, shape):
    M, F, K, pad, off = shape
    i = SHAPES.index(shape)
    gen = torch.Generator().manual_seed(100 + i)
    dt = ff.TYPES[type]
    act = ff.ACTS[(i + 2) % 5]
    x = ff.rand(gen, M, K, dt, 1.0, pad, off)
    wg, wu = (ff.rand(gen, F, K, dt, K ** -0.5, pad, off) for _ in range(2))
    h, g, u = gated_forward(B, type, act, x, wg, wu, True, pad)
    for name, t, v in zip("hgu", (h, g, u), ff.gated_forward(act, x, wg, wu)):
        ff.check(name, t, v)
    h2, _, _ = gated_forward(B, type, act, x, wg, wu, False, pad)
    assert torch.equal(h, h2)
    dh = ff.rand(gen, M, F, dt, 0.3, pad, off)
    g, u = g.cpu(), u.cpu()
    got = gated_backward(B, type, act, x, wg, wu, g, u, dh, pad)
    for name, t, v in zip(("dx", "dwg", "dwu"), got, ff.gated_backward(act, x, wg, wu, g, u, dh)):
        ff.check(name, t, v)
    again = gated_backward(B, type, act, x, wg, wu, g, u, dh, pad)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("type", list(ff.TYPES))
@pytest.mark.parametrize("act", ff.ACTS)
def test_every_activation(B, type, act):
    """Far into both tails: K = 1 and weights of 1 make z the input itself."""
    dt = ff.TYPES[type]
    z = torch.cat([torch.linspace(-30, 30, 241), torch.tensor([0.0, -0.0, 1e-4, -1e-4, 6e4, -6e4])]).to(dt).view(-1, 1)
    w, dy = torch.ones(1, 1, dtype=dt), torch.ones(z.shape, dtype=dt)
    y, zz = linear_forward(B, type, act, z, w, None, None, True)
    ff.check("y", y, ff.linear_forward(act, z, w, None, None)[0])
    assert torch.equal(zz.cpu(), z)
    dx, _, _ = linear_backward(B, type, act, z, w, z, dy)
    ff.check("dx", dx, ff.linear_backward(act, z, w, z, dy)[0])
    h, _, _ = gated_forward(B, type, act, z, w, torch.full((1, 1), 0.001, dtype=dt), False)
    ff.check("h", h, ff.gated_forward(act, z, w, torch.full((1, 1), 0.001, dtype=dt))[0])


@pytest.mark.parametrize("type", list(ff.TYPES))
def test_larger_sums(B, type):
    """More than one tile and stage each way, and a contraction that may be split."""
    dt = ff.TYPES[type]
    for M, N, K in ((200, 384, 4096), (16, 64, 9216), (1, 100, 16384), (520, 300, 2056)):
        print("larger", type, M, N, K, flush=True)
        g = torch.Generator().manual_seed(M)
        x, w = ff.rand(g, M, K, dt), ff.rand(g, N, K, dt, K ** -0.5)
        bias = ff.rand(g, 1, N, dt).view(N)
        y, z = linear_forward(B, type, "gelu", x, w, bias, None, True)
        want = ff.linear_forward("gelu", x, w, bias, None)
        ff.check("y", y, want[0])
        ff.check("z", z, want[1])
        dy = ff.rand(g, M, N, dt)
        for name, t, v in zip(("dx", "dw", "dbias"), linear_backward(B, type, "gelu", x, w, z.cpu(), dy),
                              ff.linear_backward("gelu", x, w, z.cpu(), dy)):
            ff.check(name, t, v)


@pytest.mark.parametrize("type", list(ff.TYPES))
@pytest.mark.parametrize("M", [1, 40, 300])
def test_what_is_not_finite_stays_where_it_is(B, type, M):
    """A row of x with an infinity or a NaN touches its own row of results only, and with the sums that fp32 has: an infinity
    times a number is an infinity of its sign."""
    dt = ff.TYPES[type]
    N, K = 136, 264
    g = torch.Generator().manual_seed(M)
    x, w = ff.rand(g, M, K, dt), ff.rand(g, N, K, dt)
    clean, _ = linear_forward(B, type, "none", x, w, None, None, False)
    x = x.clone()
    x[M // 2, 7] = float("inf")
    y, _ = linear_forward(B, type, "none", x, w, None, None, False)
    want = torch.where(w[:, 7] > 0, float("inf"), -float("inf")).to(dt)
    assert not bool((w[:, 7] == 0).any())
    assert torch.equal(y[M // 2].cpu(), want)
    rest = torch.arange(M) != M // 2
    assert torch.equal(y[rest], clean[rest])
    x[M // 2, 9] = float("nan")
    y, _ = linear_forward(B, type, "relu", x, w, None, None, False)
    assert bool(torch.isnan(y[M // 2]).all()) and bool(torch.isfinite(y[rest]).all())
    # the last column, which a tile's padding lies next to
    x[M // 2, 7] = x[M // 2, 9] = 1.0
    x[M // 2, K - 1] = float("nan")
    y, _ = linear_forward(B, type, "none", x, w, None, None, False)
    assert bool(torch.isnan(y[M // 2]).all()) and torch.equal(y[rest], clean[rest])
    # backward: an infinite dy touches its row of dx and its row of dw
    dy = ff.rand(g, M, N, dt)
    x = ff.rand(g, M, K, dt)
    dy[M // 2, 5] = float("inf")
    dx, dw, db = linear_backward(B, type, "none", x, w, None, dy)
    assert torch.equal(dx[M // 2].cpu(), torch.where(w[5] > 0, float("inf"), -float("inf")).to(dt))
    assert bool(torch.isfinite(dx[rest]).all())
    assert torch.equal(dw[5].cpu(), torch.where(x[M // 2] > 0, float("inf"), -float("inf")).to(dt))
    assert bool(torch.isfinite(dw[torch.arange(N) != 5]).all()) and float(db[5]) == float("inf")


def test_fp32_ends_of_the_range(B):
    """Sums of products whose factors lie at the ends of fp32's range."""
    g = torch.Generator().manual_seed(3)
    for M in (3, 150):
        for sx, sw in ((1e-38, 1e30), (1e30, 1e-38), (1e37, 1e-30), (1e-20, 1e-12), (3e38 / 8, 1e-3)):
            print("range", M, sx, sw, flush=True)
            x, w = (torch.rand(M, 72, generator=g) - 0.5) * sx, (torch.rand(140, 72, generator=g) - 0.5) * sw
            y, _ = linear_forward(B, "f32", "none", x, w, None, None, False)
            ff.check("y", y, ff.linear_forward("none", x, w, None, None)[0])


@pytest.mark.parametrize("type", ["bf16", "f16"])
def test_numbers_below_the_normal_ones(B, type):
    """Operands, and results, that a type holds only as subnormal numbers: products of powers of two, exact."""
    dt = ff.TYPES[type]
    low = -132 if type == "bf16" else -23          # subnormal: bf16 below 2^-126, fp16 below 2^-14
    for M in (2, 90):
        print("subnormal", type, M, flush=True)
        x = torch.zeros(M, 16, dtype=torch.float64)
        x[:, 3] = 2.0 ** low
        x[:, 4] = 3 * 2.0 ** low
        w = torch.zeros(24, 16, dtype=torch.float64)
        w[:, 3], w[:, 4] = 2.0 ** 12, 2.0 ** 12
        w[1, 3:5], w[2, 3:5], w[3, 3:5] = 1.0, -1.0, 0.5
        want = (x @ w.t()).to(dt)
        y, _ = linear_forward(B, type, "none", x.to(dt), w.to(dt), None, None, False)
        assert torch.equal(y.cpu(), want)
        dx, dw, _ = linear_backward(B, type, "none", w.to(dt)[:, :16], x.to(dt)[:24], None,
                                    torch.eye(24, min(M, 24), dtype=dt))
        assert torch.equal(dx.cpu(), x.to(dt)[:24] if M >= 24 else torch.cat([x.to(dt), torch.zeros(24 - M, 16, dtype=dt)]))


@pytest.mark.parametrize("type", list(ff.TYPES))
def test_empty_batch(B, type):
    dt = ff.TYPES[type]
    w, x = torch.ones(24, 16, dtype=dt), torch.ones(0, 16, dtype=dt)
    y, z = linear_forward(B, type, "gelu", x, w, None, None, True)
    dx, dw, db = linear_backward(B, type, "gelu", x, w, z.cpu(), torch.ones(0, 24, dtype=dt))
    assert not bool(dw.any()) and not bool(db.any()) and dw.shape == (24, 16)
    empty = torch.ones(0, 24, dtype=dt)
    _, dwg, dwu = gated_backward(B, type, "silu", x, w, w, empty, empty, empty)
    assert not bool(dwg.any()) and not bool(dwu.any())


def test_residual_in_place(B):
    g = torch.Generator().manual_seed(9)
    for type in ff.TYPES:
        for M in (1, 20, 200):
            dt = ff.TYPES[type]
            x, w, r = ff.rand(g, M, 96, dt), ff.rand(g, 160, 96, dt, 0.1), ff.rand(g, M, 160, dt)
            want, _ = linear_forward(B, type, "silu", x, w, None, r, False)
            t, a = consts(B, type, "silu")
            d = B.make_linear_desc(M, 160, 96, t, a)
            s = r.cuda()
            B.cct_linear_forward(d, x.cuda(), w.cuda(), None, s, s, None, B.alloc_linear_workspace(d, B.PASS_FORWARD))
            assert torch.equal(s, want)


def test_offsets_beyond_32_bits(B):
    """Rows that lie more than 2^31 values, or 2^32 bytes, apart in one tensor."""
    K, N, ld = 72, 40, (1 << 30) + 24
    g = torch.Generator().manual_seed(11)
    for M in (5, 70):
        ld_m = ld if M == 5 else (1 << 26) + 8
        flat = torch.empty((M - 1) * ld_m + K, dtype=torch.bfloat16, device="cuda")
        x, w = ff.rand(g, M, K, torch.bfloat16), ff.rand(g, N, K, torch.bfloat16)
        gx = flat.as_strided((M, K), (ld_m, 1))
        gx.copy_(x)
        d = B.make_linear_desc(M, N, K, B.TYPE_BF16)
        y = ff.empty_gpu(M, N, torch.bfloat16)
        B.cct_linear_forward(d, gx, w.cuda(), None, None, y, None, B.alloc_linear_workspace(d, B.PASS_FORWARD))
        ff.check("y", y, ff.linear_forward("none", x, w, None, None)[0])
        # the same rows as dx and as dy
        dy = ff.rand(g, M, N, torch.bfloat16)
        dw = ff.empty_gpu(N, K, torch.bfloat16)
        dx = flat.as_strided((M, K), (ld_m, 1))
        ws = B.alloc_linear_workspace(d, B.PASS_BACKWARD)
        B.cct_linear_backward(d, gx, None, None, dy.cuda(), None, dw, None, ws)
        want = ff.linear_backward("none", x, w, None, dy)
        ff.check("dw", dw, want[1])
        B.cct_linear_backward(d, None, w.cuda(), None, dy.cuda(), dx, None, None, ws)
        ff.check("dx", dx, want[0])
        del flat, gx, dx


def test_fp32_rows_too_far_apart_for_the_split_product(B):
    """Rows 2^22 values apart and more, each of x, w and the gradients: the general kernel."""
    g = torch.Generator().manual_seed(12)
    M, N, K, ld = 70, 40, 72, (1 << 22) + 5
    flat = torch.empty((M - 1) * ld + K, device="cuda")
    far = lambda r, c: flat.as_strided((r, c), (ld, 1))  # noqa: E731
    x, w, u = ff.rand(g, M, K, torch.float32), ff.rand(g, N, K, torch.float32, 0.1), ff.rand(g, N, K, torch.float32, 0.1)
    bias, r = ff.rand(g, 1, N, torch.float32).view(N), ff.rand(g, M, N, torch.float32)
    d = B.make_linear_desc(M, N, K, B.TYPE_F32, B.ACT_GELU)
    y, z = ff.empty_gpu(M, N, torch.float32), ff.empty_gpu(M, N, torch.float32)
    far(N, K).copy_(w)
    B.cct_linear_forward(d, x.cuda(), far(N, K), bias.cuda(), r.cuda(), y, z, B.alloc_linear_workspace(d, B.PASS_FORWARD))
    want = ff.linear_forward("gelu", x, w, bias, r)
    ff.check("y", y, want[0])
    ff.check("z", z, want[1])
    dy = ff.rand(g, M, N, torch.float32)
    dx, dw = ff.empty_gpu(M, K, torch.float32), ff.empty_gpu(N, K, torch.float32)
    ws = B.alloc_linear_workspace(d, B.PASS_BACKWARD)
    B.cct_linear_backward(d, None, far(N, K), z, dy.cuda(), dx, None, None, ws)
    far(M, K).copy_(x)
    B.cct_linear_backward(d, far(M, K), None, z, dy.cuda(), None, dw, None, ws)
    want = ff.linear_backward("gelu", x, w, z.cpu(), dy)
    ff.check("dx", dx, want[0])
    ff.check("dw", dw, want[1])
    e = B.make_gated_desc(M, N, K, B.TYPE_F32, B.ACT_SILU)
    far(N, K).copy_(w)
    h = ff.empty_gpu(M, N, torch.float32)
    B.cct_gated_forward(e, x.cuda(), far(N, K), u.cuda(), h, None, None, B.alloc_gated_workspace(e, B.PASS_FORWARD))
    ff.check("h", h, ff.gated_forward("silu", x, w, u)[0])


@pytest.mark.parametrize("type", list(ff.TYPES))
def test_few_rows_and_columns_of_long_rows(B, type):
    """The contraction of a forward product of few rows in splits, whole and not, at any address."""
    dt = ff.TYPES[type]
    for M, N, K, pad in ((1, 10, 8192, 0), (3, 33, 9001, 1), (16, 72, 20000, 0), (30, 100, 12288, 3), (50, 40, 8200, 5)):
        print("splits", type, M, N, K, flush=True)
        g = torch.Generator().manual_seed(N)
        x, w, u = (ff.rand(g, r, K, dt, s, pad) for r, s in ((M, 1.0), (N, K ** -0.5), (N, K ** -0.5)))
        bias, r = ff.rand(g, 1, N, dt).view(N), ff.rand(g, M, N, dt)
        y, z = linear_forward(B, type, "gelu", x, w, bias, r, True)
        want = ff.linear_forward("gelu", x, w, bias, r)
        ff.check("y", y, want[0])
        ff.check("z", z, want[1])
        h, gg, uu = gated_forward(B, type, "silu", x, w, u, True)
        for name, t, v in zip("hgu", (h, gg, uu), ff.gated_forward("silu", x, w, u)):
            ff.check(name, t, v)


@pytest.mark.parametrize("type", list(ff.TYPES))
def test_few_rows_at_odd_addresses(B, type):
    """Rows of 16-bit values that begin between multiples of four bytes, all of them or every other one, in x, in the weights
    or in one weight only; NaN in front of each row, which the loads may touch."""
    dt = ff.TYPES[type]
    for M, N, K, pad, off in ((1, 33, 96, 1, 1), (3, 100, 515, 2, 1), (16, 40, 8224, 1, 0), (17, 50, 130, 3, 1),
                              (32, 20, 264, 1, 3), (64, 72, 520, 2, 1), (60, 90, 1024, 1, 0)):
        print("odd", type, M, N, K, pad, off, flush=True)
        g = torch.Generator().manual_seed(K)

        def rows(r, std, pad, off):
            v = ff.rand(g, r, K, dt, std)
            flat = torch.full((off + r * (K + pad),), float("nan"), dtype=dt, device="cuda")
            t = flat[off:].view(r, K + pad)[:, :K]
            t.copy_(v)
            return v, t

        for odd_x, odd_w, odd_u in ((1, 1, 1), (1, 0, 0), (0, 1, 0), (0, 0, 1)):
            (x, xg), (w, wg), (u, ug) = (rows(r, s, pad if o else 8, off if o else 0)
                                         for r, s, o in ((M, 1.0, odd_x), (N, K ** -0.5, odd_w), (N, K ** -0.5, odd_u)))
            y, z = ff.empty_gpu(M, N, dt), ff.empty_gpu(M, N, dt)
            d = B.make_linear_desc(M, N, K, getattr(B, "TYPE_" + type.upper()), B.ACT_GELU)
            B.cct_linear_forward(d, xg, wg, None, None, y, z, B.alloc_linear_workspace(d, B.PASS_FORWARD))
            for name, t, v in zip("yz", (y, z), ff.linear_forward("gelu", x, w, None, None)):
                ff.check(name, t, v)
            h, gg, uu = (ff.empty_gpu(M, N, dt) for _ in range(3))
            e = B.make_gated_desc(M, N, K, getattr(B, "TYPE_" + type.upper()), B.ACT_SILU)
            B.cct_gated_forward(e, xg, wg, ug, h, gg, uu, B.alloc_gated_workspace(e, B.PASS_FORWARD))
            for name, t, v in zip("hgu", (h, gg, uu), ff.gated_forward("silu", x, w, u)):
                ff.check(name, t, v)


@pytest.mark.parametrize("type", ["bf16", "f16"])
def test_backward_products_in_one_launch(B, type):
    """Sizes whose products share a launch, in tiles of 64, 64 x 128 and 128, ragged, with the sum of columns beside them (by
    one workgroup of rows, by several) and without, whole and in splits; every result alone and in pairs has the same bits."""
    dt = ff.TYPES[type]
    for M, N, K, pad, off in ((20, 100, 300, 0, 0), (33, 72, 136, 1, 1), (500, 300, 500, 5, 0), (1030, 1023, 1030, 0, 0),
                              (1531, 1000, 2049, 3, 0), (2000, 1500, 700, 0, 0),
                              # long contractions of few results, cut into splits: dx, dw, all
                              (60, 1301, 64, 0, 0), (1, 1565, 32, 8, 0), (2799, 10, 406, 1, 1), (700, 650, 40, 0, 0)):
        print("together", type, M, N, K, flush=True)
        g = torch.Generator().manual_seed(M)
        x, w, u = (ff.rand(g, r, K, dt, s, pad, off) for r, s in ((M, 1.0), (N, K ** -0.5), (N, K ** -0.5)))
        z, dy, uu = (ff.rand(g, M, N, dt, 1.0, pad, off) for _ in range(3))
        names = ("dx", "dw", "dbias")
        got = linear_backward(B, type, "gelu", x, w, z, dy, pad)
        for name, t, v in zip(names, got, ff.linear_backward("gelu", x, w, z, dy)):
            ff.check(name, t, v)
        for want in (("dx", "dw"), ("dx", "dbias"), ("dw", "dbias"), ("dx",), ("dw",), ("dbias",)):
            some = linear_backward(B, type, "gelu", x, w, z, dy, pad, want)
            assert all(torch.equal(some[i], got[i]) for i in range(3) if names[i] in want), want
        for name, t, v in zip(("dx", "dwg", "dwu"), gated_backward(B, type, "silu", x, w, u, z, uu, dy, pad),
                              ff.gated_backward("silu", x, w, u, z, uu, dy)):
            ff.check(name, t, v)


@pytest.mark.parametrize("type", ["bf16", "f16"])
def test_every_tile_and_split(B, type):
    """Sizes that the plan cuts into tiles of 256, 192 x 256, 128, 64 x 128 and 64, each direction, with one split and with
    several, and with a remainder in a launch of its own."""
    dt = ff.TYPES[type]
    for M, N, K in ((3600, 3592, 136), (3600, 136, 3592), (136, 3600, 3592), (2500, 4096, 136), (2500, 136, 4096),
                    (136, 2500, 4096), (4104, 4104, 200), (4104, 200, 4104), (200, 4104, 4104), (2050, 520, 72), (1032, 1536, 600), (520, 300, 2056), (72, 136, 8200), (264, 1100, 1032)):
        print("tiles", type, M, N, K, flush=True)
        g = torch.Generator().manual_seed(K)
        x, w, u = ff.rand(g, M, K, dt), ff.rand(g, N, K, dt, K ** -0.5), ff.rand(g, N, K, dt, K ** -0.5)
        y, z = linear_forward(B, type, "silu", x, w, None, None, True)
        want = ff.linear_forward("silu", x, w, None, None)
        ff.check("y", y, want[0])
        dy, z = ff.rand(g, M, N, dt), z.cpu()
        for name, t, v in zip(("dx", "dw", "dbias"), linear_backward(B, type, "silu", x, w, z, dy),
                              ff.linear_backward("silu", x, w, z, dy)):
            ff.check(name, t, v)
        h, gg, uu = gated_forward(B, type, "gelu_tanh", x, w, u, True)
        for name, t, v in zip("hgu", (h, gg, uu), ff.gated_forward("gelu_tanh", x, w, u)):
            ff.check(name, t, v)


def test_weights_of_a_gated_block_with_other_strides(B):
    """wg and wu in rows of different lengths, as two slices of different tensors."""
    g = torch.Generator().manual_seed(31)
    for type in ff.TYPES:
        for M in (5, 90):
            dt = ff.TYPES[type]
            x, wg, wu = ff.rand(g, M, 64, dt), ff.rand(g, 96, 64, dt, 0.1, 8), ff.rand(g, 96, 64, dt, 0.1, 24)
            h, gg, uu = gated_forward(B, type, "silu", x, wg, wu, True)
            for name, t, v in zip("hgu", (h, gg, uu), ff.gated_forward("silu", x, wg, wu)):
                ff.check(name, t, v)
            dh = ff.rand(g, M, 96, dt)
            got = gated_backward(B, type, "silu", x, wg, wu, gg.cpu(), uu.cpu(), dh)
            for name, t, v in zip(("dx", "dwg", "dwu"), got, ff.gated_backward("silu", x, wg, wu, gg.cpu(), uu.cpu(), dh)):
                ff.check(name, t, v)


@pytest.mark.parametrize("type", ["f32", "bf16"])
def test_gradients_against_differences(B, type):
    """<dx, s> and <dw, s> against how the loss changes along a direction s.  The loss is taken in 64 bits from the operator's
    own z and residual-free y in fp32 inputs, so that the differences carry the products' error only: with a step of 1/64 the
    third derivative's share is (1/64)^2 / 6 of sums of order one per value and the fp32 error 64 * 2^-22 of them."""
    g = torch.Generator().manual_seed(21)
    M, N, K = 37, 41, 29
    dt = ff.TYPES[type]
    if type == "bf16":   # the values of a bf16 pass, whose gradient is compared with the fp32 operator's differences
        x, w, dy = ff.rand(g, M, K, dt).float(), ff.rand(g, N, K, dt, 0.2).float(), ff.rand(g, M, N, dt).float()
    else:
        x, w, dy = ff.rand(g, M, K, dt), ff.rand(g, N, K, dt, 0.2), ff.rand(g, M, N, dt)
    for act in ("silu", "gelu", "gelu_tanh"):
        _, z = linear_forward(B, "f32", act, x, w, None, None, True)
        dx, dw, _ = linear_backward(B, type, act, x.to(dt), w.to(dt), z.cpu().to(dt), dy.to(dt))

        def loss(x_, w_):
            y, _ = linear_forward(B, "f32", act, x_, w_, None, None, False)
            return float((y.cpu().double() * dy.double()).sum())
        sx, sw = torch.randn(M, K, generator=g) / K, torch.randn(N, K, generator=g) / K
        h = 1.0 / 64
        for got, s, diff in ((dx, sx, loss(x + h * sx, w) - loss(x - h * sx, w)),
                             (dw, sw, loss(x, w + h * sw) - loss(x, w - h * sw))):
            terms = got.cpu().double() * s.double()
            # bf16: z, dz and the result are off by 2^-8 each at most, errors of either sign over the terms
            tol = (2.0 ** -7 if type == "bf16" else 2.0 ** -12) * float(terms.norm()) * 8
            assert abs(diff / (2 * h) - float(terms.sum())) <= tol


@pytest.mark.parametrize("type", list(ff.TYPES))
def test_on_another_stream_and_in_a_graph(B, type):
    """Captured once and replayed with new inputs, with eager work and synchronizations in between: the eager bits."""
    dt = ff.TYPES[type]
    gen = torch.Generator(device="cuda").manual_seed(5)
    for M in (1, 24, 260):
        print("graph", type, M, flush=True)
        F, K = 200, 328
        t, _ = consts(B, type, "silu")
        dg, dl = B.make_gated_desc(M, F, K, t, B.ACT_SILU), B.make_linear_desc(M, K, F, t, B.ACT_GELU)
        new = lambda r, c: torch.randn(r, c, generator=gen, device="cuda").to(dt)  # noqa: E731
        x, dy = new(M, K), new(M, K)
        wg, wu, w, bias = new(F, K), new(F, K), new(K, F), new(1, K).view(K)
        o = {n: torch.empty(r, c, dtype=dt, device="cuda") for n, r, c in (
            ("h", M, F), ("g", M, F), ("u", M, F), ("y", M, K), ("z", M, K), ("dh", M, F), ("dw", K, F), ("dx", M, K),
            ("dwg", F, K), ("dwu", F, K))}
        o["db"] = torch.empty(K, dtype=dt, device="cuda")
        ws = [B.alloc_gated_workspace(dg, 0), B.alloc_linear_workspace(dl, 0), B.alloc_linear_workspace(dl, 3),
              B.alloc_gated_workspace(dg, 3)]

        def block():
            B.cct_gated_forward(dg, x, wg, wu, o["h"], o["g"], o["u"], ws[0])
            B.cct_linear_forward(dl, o["h"], w, bias, x, o["y"], o["z"], ws[1])
            B.cct_linear_backward(dl, o["h"], w, o["z"], dy, o["dh"], o["dw"], o["db"], ws[2])
            B.cct_gated_backward(dg, x, wg, wu, o["g"], o["u"], o["dh"], o["dx"], o["dwg"], o["dwu"], ws[3])

        block()
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            block()
            torch.cuda.synchronize()
            with torch.cuda.graph(graph, stream=side):
                block()
        torch.cuda.synchronize()
        for r in range(3):
            x.copy_(new(M, K))
            dy.copy_(new(M, K))
            torch.cuda.synchronize()
            block()
            torch.cuda.synchronize()
            eager = {n: v.clone() for n, v in o.items()}
            for v in o.values():
                v.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            for n, v in o.items():
                assert torch.equal(v, eager[n]), (n, r)
