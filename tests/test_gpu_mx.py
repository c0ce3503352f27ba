"""Microscaled 4-bit floating point (cct_mx_*): codes, scales and values bit by bit against tables on the CPU; products against 64
bits, within the bound of fp32 sums of exact products (feed_forward_util.py)."""
import pytest
import torch

import feed_forward_util as ff
import mx_util as mx

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available()
    from paper_1504_04343_amd import binding
    return binding


def matrix(B, rows, cols, pad=0, fill=0xee):
    """A matrix whose rows have room behind them, all bytes `fill`."""
    n = mx.blocks_of(cols)
    wide, high = n * 16, -(-n // 4) * 4
    codes = torch.full((max(rows, 1), wide + 16 * pad), fill, dtype=torch.uint8, device="cuda")
    scales = torch.full((max(rows, 1), high + 4 * pad), fill, dtype=torch.uint8, device="cuda")
    return B.MxMatrix(rows, cols, codes[:rows, :wide], scales[:rows, :high]), codes, scales


def given(B, code, scale, cols, pad=0):
    """A matrix of codes (a byte each) and scales; scales that are no block's are NaN."""
    m, codes, scales = matrix(B, len(code), cols, pad, 255)
    m.codes.copy_(mx.pack(code).cuda())
    m.scales[:, :scale.shape[1]] = scale.cuda()
    return m


def check_quantized(B, x, pad=0):
    rows, cols = x.shape
    m, codes, scales = matrix(B, rows, cols, pad)
    B.cct_mx_quantize(ff.to_gpu(x), m)
    code, scale = mx.quantize(x)
    assert torch.equal(m.codes.cpu(), mx.pack(code))
    assert torch.equal(m.scales.cpu()[:, :scale.shape[1]], scale)
    assert bool((codes[:, m.codes.shape[1]:] == 0xee).all()) and bool((scales[:, m.scales.shape[1]:] == 0xee).all())
    out = ff.empty_gpu(rows, cols, x.dtype, pad)
    B.cct_mx_dequantize(m, out)
    want = mx.values(code, scale, cols).to(x.dtype)
    assert torch.equal(out.cpu().nan_to_num(77.0), want.nan_to_num(77.0)) and ff.untouched(out, cols)


@pytest.mark.parametrize("type", list(ff.TYPES))
@pytest.mark.parametrize("shape", [(1, 1, 0, 0), (1, 31, 0, 0), (1, 4096, 0, 0), (2, 33, 1, 1), (3, 7, 5, 0), (5, 1000, 3, 1), (17, 2049, 0, 0),
                                   (64, 96, 8, 8), (300, 65, 0, 3), (1531, 264, 1, 0), (70000, 40, 0, 0)], ids=str)
def test_quantize(B, type, shape):
    M, D, pad, off = shape
    g = torch.Generator().manual_seed(M + D)
    x = ff.rand(g, M, D, ff.TYPES[type], 1.0, pad, off)
    x *= torch.exp2(torch.randint(-9, 6, (M, 1), generator=g).float()).to(x.dtype)
    check_quantized(B, x, pad)


@pytest.mark.parametrize("type", list(ff.TYPES))
def test_every_rounding(B, type):
    """Middles between neighbours and the numbers next to them, all signs, in blocks of every scale that the type reaches."""
    dt = ff.TYPES[type]
    lo, hi = dict(f32=(-149, 127), bf16=(-133, 127), f16=(-24, 15))[type]
    at = torch.tensor([4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 0.5, 1.0, 1.5, 2.0, 3.0])
    step = {"f32": 2.0 ** -21, "bf16": 2.0 ** -5, "f16": 2.0 ** -8}[type]
    row = torch.cat([at, at * (1 + step), at * (1 - step / 2)])
    rows = []
    for e in range(lo, hi + 1):
        v = torch.ldexp(row.double(), torch.tensor(e - 2)).clamp(max=float(torch.finfo(dt).max)).to(dt)
        first = torch.ldexp(torch.tensor(1.0, dtype=torch.float64), torch.tensor(e)).to(dt)   # its block's largest power of two
        v = v[v < 2 * first] if e < hi else v
        v = torch.cat([first[None], v, v.new_zeros(62)])[:62]
        rows.append(torch.cat([first[None], v[1:32], first[None], -v[31:]])[:64])
    check_quantized(B, torch.stack(rows))


@pytest.mark.parametrize("type", list(ff.TYPES))
def test_blocks_that_are_not_finite(B, type):
    x = ff.rand(torch.Generator().manual_seed(1), 6, 200, ff.TYPES[type])
    x[1, 40], x[2, 199], x[3, 0], x[3, 64] = float("nan"), float("inf"), -float("inf"), float("nan")
    x[4, 32:64], x[5] = 0.0, -0.0
    check_quantized(B, x)


@pytest.mark.parametrize("type", list(ff.TYPES))
def test_dequantize_everything(B, type):
    """Every code at every scale; fp16 rounds, and to infinities beyond its range."""
    code = torch.arange(32, dtype=torch.uint8).view(1, 32).expand(256, 32) & 15
    scale = torch.arange(256, dtype=torch.uint8).view(256, 1)
    m = given(B, code.contiguous(), scale, 32)
    out = torch.empty(256, 32, dtype=ff.TYPES[type], device="cuda")
    B.cct_mx_dequantize(m, out)
    want = mx.values(code, scale, 32).to(ff.TYPES[type])
    assert torch.equal(torch.isnan(out.cpu()), torch.isnan(want))
    assert torch.equal(out.cpu().nan_to_num(1.0, 7e4, -7e4).float(), want.nan_to_num(1.0, 7e4, -7e4).float())


def operand(g, rows, cols, low=-2, high=3):
    """Codes and scales of a matrix, and its values."""
    code = torch.randint(0, 16, (rows, mx.blocks_of(cols) * 32), generator=g, dtype=torch.uint8)
    code[:, cols:] = 0
    scale = (torch.randint(low, high, (rows, mx.blocks_of(cols)), generator=g) + 127).to(torch.uint8)
    return code, scale, mx.values(code, scale, cols)


def run(B, type, act, x, w, bias, residual, save, M, N, K, pad=0, quantize=False):
    t = dict(f32=B.TYPE_F32, bf16=B.TYPE_BF16, f16=B.TYPE_F16)[type]
    d = B.make_linear_desc(M, N, K, t, ff.ACTS.index(act))
    y = ff.empty_gpu(M, N, ff.TYPES[type], pad)
    z = ff.empty_gpu(M, N, ff.TYPES[type], pad) if save else None
    ws = B.alloc_mx_linear_workspace(d, quantize)
    ws.fill_(0xff)   # nothing that a workspace holds before the call may matter
    B.cct_mx_linear_forward(d, x, w, None if bias is None else bias.cuda(), None if residual is None else ff.to_gpu(residual), y, z, ws)
    torch.cuda.synchronize()
    assert ff.untouched(y, N) and (z is None or ff.untouched(z, N))
    return y, z


def expect(act, xv, wv, bias, residual, dt):
    z, ez = ff.product(xv, wv, bias)
    a, _ = ff.act64(act, z)
    y = a if residual is None else a + residual.double()
    return ff.rounded(y, ff.SLOPE * ez + ff.ACT_ERR * a.abs() + ff.EPS32 * y.abs(), dt), ff.rounded(z, ez, dt)


# M, N, K, elements between the rows of y (and blocks between those of codes), elements in front
SHAPES = [(1, 1, 1, 0, 0), (1, 16, 32, 0, 0), (1, 64, 4096, 0, 0), (2, 33, 1000, 0, 0), (3, 130, 515, 1, 1), (16, 48, 2048, 0, 0),
          (17, 257, 129, 0, 0), (31, 64, 40, 64, 8), (33, 520, 136, 0, 2), (64, 96, 1024, 0, 0), (65, 72, 7, 5, 0), (100, 1000, 64, 0, 0),
          (128, 128, 128, 0, 0), (129, 136, 264, 8, 8), (257, 300, 300, 3, 1), (300, 520, 512, 0, 0), (513, 264, 776, 0, 0),
          (256, 256, 256, 0, 0), (700, 700, 1300, 1, 0), (5, 40, 70000, 0, 0), (70, 24, 33000, 3, 0), (1, 6, 16384, 0, 0)]


@pytest.mark.parametrize("type", list(ff.TYPES))
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "%dx%dx%d+%d@%d" % s)
def test_product(B, type, shape):
    M, N, K, pad, off = shape
    i = SHAPES.index(shape)
    g, dt, act = torch.Generator().manual_seed(i), ff.TYPES[type], ff.ACTS[i % 5]
    xc, xs, xv = operand(g, M, K)
    wc, ws, wv = operand(g, N, K, -6, -1)
    bias = ff.rand(g, 1, N, dt, 0.3).view(N) if i % 3 else None
    residual = ff.rand(g, M, N, dt, 1.0, pad, off) if i % 2 else None
    x, w = given(B, xc, xs, K, pad), given(B, wc, ws, K, pad)
    y, z = run(B, type, act, x, w, bias, residual, True, M, N, K, pad)
    want = expect(act, xv, wv, bias, residual, dt)
    ff.check("y", y, want[0])
    ff.check("z", z, want[1])
    assert torch.equal(y, run(B, type, act, x, w, bias, residual, False, M, N, K, pad)[0])
    # x as values: the same as if it were quantised before
    v = ff.rand(g, M, K, dt, 1.0, pad, off)
    q, _, _ = matrix(B, M, K)
    B.cct_mx_quantize(ff.to_gpu(v), q)
    a = run(B, type, act, q, w, bias, residual, False, M, N, K, pad)[0]
    b = run(B, type, act, ff.to_gpu(v), w, bias, residual, False, M, N, K, pad, True)[0]
    assert torch.equal(a, b)
    ff.check("y", a, expect(act, mx.values(*mx.quantize(v), K), wv, bias, residual, dt)[0])


@pytest.mark.parametrize("type", list(ff.TYPES))
@pytest.mark.parametrize("M", [1, 4, 5])
def test_what_is_quantised_on_the_way(B, type, M):
    """A product with the identity gives the values that x was rounded to, also where the workgroups that multiply round it: rows of
    every scale of the type, its smallest numbers, infinities and NaN."""
    K, dt = 96, ff.TYPES[type]
    g = torch.Generator().manual_seed(M)
    code = torch.eye(K).byte() * 2                        # 1.0
    eye = given(B, code, torch.full((K, 3), 127, dtype=torch.uint8), K)
    lo, hi = dict(f32=(-149, 125), bf16=(-133, 125), f16=(-24, 13))[type]
    for e in range(lo, hi, 7):
        # up to just below 8 times 2^e, so that every rounding is met; a row of the middles between neighbours
        x = torch.ldexp((torch.rand(M, K, generator=g) * 16 - 8).double(), torch.tensor(e)).to(dt)
        x[M - 1, :15] = torch.ldexp(torch.tensor([4, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, 6, 7, .5, 1, 1.5, 2, 3]).double(), torch.tensor(e)).to(dt)
        x[0, 64:] = 0
        y, _ = run(B, type, "none", ff.to_gpu(x), eye, None, None, False, M, K, K, 0, True)
        want = mx.values(*mx.quantize(x), K)
        # (what is below fp32's normal numbers may be lost in the sum of its products)
        off = (y.cpu().double() - want).abs()
        assert bool((off <= (2.0 ** -126 if type != "f16" else 0.0)).all()), e
    x = ff.rand(g, M, K, dt)
    x[0, 5], x[M - 1, 70] = float("inf"), float("nan")
    y = run(B, type, "none", ff.to_gpu(x), eye, None, None, False, M, K, K, 0, True)[0].cpu()
    assert torch.isnan(y[0]).all() and torch.isnan(y[M - 1]).all()        # 0 * NaN
    assert M < 3 or torch.equal(y[1:M - 1].double(), mx.values(*mx.quantize(x), K)[1:M - 1])


@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("act", ff.ACTS)
@pytest.mark.parametrize("M", [1, 300])
def test_activations_of_all_numbers(B, type, act, M):
    """Of every number of the type: a product of zeros, and the number as bias."""
    dt, N = ff.TYPES[type], 65536
    z = torch.arange(N, dtype=torch.int32).to(torch.uint16).view(dt)
    zeros = lambda rows: given(B, torch.zeros(rows, 32, dtype=torch.uint8), torch.full((rows, 1), 127, dtype=torch.uint8), 32)
    y, _ = run(B, type, act, zeros(M), zeros(N), z, None, False, M, N, 32)
    y = y.cpu()
    assert torch.equal(y.view(torch.int16), y[:1].view(torch.int16).expand(M, N)) or act != "none" and \
        torch.equal(y.nan_to_num(1.0), y[:1].nan_to_num(1.0).expand(M, N))
    y, z = y[:1], z.double().view(1, N)
    plus, bad = z == float("inf"), torch.isnan(z)
    assert bool((y[plus] == float("inf")).all()) and bool(torch.isnan(y[bad]).all())
    there = torch.isfinite(z)
    z = z[there].view(1, -1)
    # 1 + erf and 1 + tanh have nothing of the left tails in 64 bits: erfc and the logistic function do
    if act == "gelu":
        a = z * 0.5 * torch.special.erfc(-z * 0.5 ** 0.5)
    elif act == "gelu_tanh":
        a = z * torch.sigmoid(2 * 0.7978845608028654 * (z + 0.044715 * z ** 3))
    else:
        a = ff.act64(act, z)[0]
    ff.check("y", y[there].view(1, -1), ff.rounded(a, ff.ACT_ERR * a.abs(), dt))


@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("act,least,bound", [("silu", -60.0, 2.0 ** -21), ("gelu", -4.0, 2.0 ** -19.7), ("gelu_tanh", -1.0, 2.0 ** -20.5)],
                         ids=["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("M", [1, 300])
def test_activations_before_they_are_rounded(B, type, act, least, bound, M):
    """The rounded activation as a residual that is taken away leaves act(z)'s own digits.  In units of 2^-23, a place of the hardware's
    exp2 and reciprocal at the most, half of one an operation's rounding: SiLU 1 of each, 1 + e, the product and the power's argument:
    3.2, 2^-21.3.  GELU: the polynomial 1.4, t (1.5 places at a = 3.2, where the function goes with its power 1.84; 1 of power 2.6 at
    a = 0) 2.8, Horner's steps 1, exp2 1.5 with its argument, whose constant is short of 0.9 at a = 4, three products 1.5: 9.1, 2^-19.8.
    GELU_TANH down to -1: an argument of 1.7 with two roundings and its constant's 1.8, the rest as SiLU: 5, 2^-20.6."""
    dt, N = ff.TYPES[type], 65536
    z = torch.arange(N, dtype=torch.int32).to(torch.uint16).view(dt)
    z = z.masked_fill(~torch.isfinite(z), 0.0)
    v = z.double()
    if act == "gelu":
        a = v * 0.5 * torch.special.erfc(-v * 0.5 ** 0.5)
    else:
        a = v * torch.sigmoid(v if act == "silu" else 2 * 0.7978845608028654 * (v + 0.044715 * v ** 3))
    near = -a.to(dt)
    zeros = lambda rows: given(B, torch.zeros(rows, 32, dtype=torch.uint8), torch.full((rows, 1), 127, dtype=torch.uint8), 32)
    y, _ = run(B, type, act, zeros(M), zeros(N), z, near.expand(M, N).contiguous(), False, M, N, 32)
    there = (v >= least) & (a.abs() > 2.0 ** -100)
    value = (a + near.double())[there].expand(M, -1)
    ff.check("y", y[:, there.cuda()], ff.rounded(value, bound * a[there].abs().expand(M, -1), dt))


@pytest.mark.parametrize("M", [1, 20, 300])
def test_whole_numbers(B, M):
    """Sums of whole numbers below 2^24 are exact, whatever their order."""
    N, K = 310, 5000
    g = torch.Generator().manual_seed(M)
    xc, xs, xv = operand(g, M, K, 1, 3)
    wc, ws, wv = operand(g, N, K, 1, 3)
    y, _ = run(B, "f32", "none", given(B, xc, xs, K), given(B, wc, ws, K), None, None, False, M, N, K)
    assert torch.equal(y.cpu().double(), xv @ wv.t())


PLANS = [(3, 160, 1000, "mx_rows_kernel"), (16, 24, 40000, "mx_rows_kernel"),
         (300, 200, 1100, "mx_tile_kernel<64x64, 1 splits, 4 stages>"), (40, 16384, 4000, "mx_tile_kernel<64x64, 1 splits, 4 stages>"),
         (300, 200, 10880, "mx_tile_kernel<64x64, 9 splits, 4 stages>"), (1000, 1000, 200, "mx_tile_kernel<64x64, 1 splits, 2 stages>"),
         (4182, 1, 13105, "mx_tile_kernel<64x64, 13 splits, 2 stages>"), (2100, 2100, 1100, "mx_tile_kernel<64x128, 1 splits, 2 stages>"),
         (70, 1814, 19797, "mx_tile_kernel<64x128, 8 splits, 2 stages>"), (1500, 1500, 4100, "mx_tile_kernel<128x128, 1 splits, 2 stages>"),
         (1030, 1000, 20000, "mx_tile_kernel<128x128, 3 splits, 2 stages>"), (4096, 4090, 1500, "mx_tile_kernel<256x256, 1 splits, 2 stages>"),
         (7000, 8000, 200, "mx_tile_kernel<256x256, 1 splits, 2 stages>")]


@pytest.mark.parametrize("M,N,K,kernel", PLANS)
def test_every_plan(B, M, N, K, kernel):
    """Which kernel ran, and whole numbers, whose sums are exact: terms of up to 144 * 4, at most 40000 of them."""
    g = torch.Generator().manual_seed(M)
    (xc, xs, _), (wc, ws, _) = operand(g, M, K, 1, 3), operand(g, N, K, 1, 2)   # multiples of 1: halves times two or more
    x, w = given(B, xc, xs, K, 1), given(B, wc, ws, K)
    residual = torch.randint(-9, 9, (M, N), generator=g).float()
    B.cct_profile_enable(True)
    try:
        y, _ = run(B, "f32", "none", x, w, None, residual, False, M, N, K)
        names = [e["name"] for e in B.cct_profile_read() if e["name"].startswith("mx")]
    finally:
        B.cct_profile_enable(False)
    assert names == [kernel]
    values = [torch.empty(r, K, device="cuda") for r in (M, N)]
    for m, v in zip((x, w), values):
        B.cct_mx_dequantize(m, v)
    assert torch.equal(y.double(), values[0].double() @ values[1].double().t() + residual.double().cuda())
    # rows too far apart for a tile's offsets
    if M <= 300 and N <= 200:
        far = torch.empty((N - 1) * (1 << 23) + w.codes.shape[1], dtype=torch.uint8, device="cuda").as_strided(w.codes.shape, (1 << 23, 1))
        far.copy_(w.codes)
        assert torch.equal(y, run(B, "f32", "none", x, B.MxMatrix(N, K, far, w.scales), None, residual, False, M, N, K)[0])


@pytest.mark.parametrize("M", [1, 40, 200, 600])
def test_scales_from_end_to_end(B, M):
    """Products far up and far down: results in fp32's range are right to the sum's bound, or what its smallest numbers lose."""
    N, K = 70, 256
    g = torch.Generator().manual_seed(5)
    xc, _, _ = operand(g, M, K)
    wc, _, _ = operand(g, N, K)
    for sx, sw in ((0, 254), (254, 0), (1, 127), (60, 70), (200, 180), (127, 250)):
        a, b = torch.full((M, 8), sx, dtype=torch.uint8), torch.full((N, 8), sw, dtype=torch.uint8)
        y, _ = run(B, "f32", "none", given(B, xc, a, K), given(B, wc, b, K), None, None, False, M, N, K)
        xv, wv = mx.values(xc, a, K), mx.values(wc, b, K)
        value, bound = expect("none", xv, wv, None, None, torch.float32)[0]
        # a partial sum lies within the sum of the terms' sizes: only where that passes fp32's range can one become an infinity
        # although the result is none (256 products of up to 36 * 2^123), which the sum then stays or turns into NaN
        free = xv.abs() @ wv.abs().t() * (1 + K * ff.EPS32) >= torch.finfo(torch.float32).max
        assert bool((free & torch.isfinite(y.cpu()) & ((y.cpu().double() - value).abs() > bound + K * 2.0 ** -126)).any()) is False
        ff.check("y", y.masked_fill(free.cuda(), 0.0), (value.masked_fill(free, 0.0), bound + K * 2.0 ** -126))
        assert (sx, sw) in ((200, 180), (127, 250)) or not free.any()   # 2^126 and 2^123 times up to 36 * 256


@pytest.mark.parametrize("M", [1, 40, 300])
def test_nan_blocks(B, M):
    """A block that is NaN makes its row's (or column's) results NaN and no others, also where its codes are zeros."""
    N, K = 150, 700
    g = torch.Generator().manual_seed(6)
    xc, xs, xv = operand(g, M, K)
    wc, ws, wv = operand(g, N, K)
    xs[M // 2, 21] = 255                    # the last block, which is not whole
    ws[3, 0] = 255
    wc[3, :32] = 0
    y, _ = run(B, "f32", "none", given(B, xc, xs, K), given(B, wc, ws, K), None, None, False, M, N, K)
    nan = torch.zeros(M, N, dtype=torch.bool)
    nan[M // 2] = True
    nan[:, 3] = True
    assert torch.equal(torch.isnan(y.cpu()), nan)
    value, bound = expect("none", xv, wv, None, None, torch.float32)[0]
    ff.check("y", y.masked_fill(nan.cuda(), 0.0), (value.masked_fill(nan, 0.0), bound.nan_to_num(0.0) + nan.double()))


@pytest.mark.parametrize("M", [1, 40, 300])
def test_rows_far_apart(B, M):
    """Weight rows whose offsets pass 32 bits."""
    N, K = 5, 300
    g = torch.Generator().manual_seed(7)
    xc, xs, xv = operand(g, M, K)
    wc, ws, wv = operand(g, N, K)
    ld = (1 << 30) + 16
    far = torch.empty((N - 1) * ld + 160, dtype=torch.uint8, device="cuda").as_strided((N, 160), (ld, 1))
    far.copy_(mx.pack(wc).cuda())
    scales = torch.zeros(N, 12, dtype=torch.uint8, device="cuda")
    scales[:, :10] = ws.cuda()
    x = given(B, xc, xs, K)
    y, _ = run(B, "f32", "none", x, B.MxMatrix(N, K, far, scales), None, None, False, M, N, K)
    near, _ = run(B, "f32", "none", x, given(B, wc, ws, K), None, None, False, M, N, K)
    ff.check("y", y, expect("none", xv, wv, None, None, torch.float32)[0])
    ff.check("y", near, expect("none", xv, wv, None, None, torch.float32)[0])


@pytest.mark.parametrize("M,N,K", [(1, 300, 1000), (40, 96, 9000), (3, 20, 30000), (300, 400, 512)])
def test_replayed_from_a_graph_and_on_another_stream(B, M, N, K):
    g = torch.Generator().manual_seed(8)
    w = given(B, *operand(g, N, K)[:2], K)
    x = torch.randn(M, K, device="cuda").bfloat16()
    d = B.make_linear_desc(M, N, K, B.TYPE_BF16, B.ACT_SILU)
    residual = torch.randn(M, N, device="cuda").bfloat16()
    y, ws = torch.empty_like(residual), B.alloc_mx_linear_workspace(d, True)
    q, values = B.MxMatrix(M, K), torch.empty_like(x)

    def step():
        B.cct_mx_linear_forward(d, x, w, None, residual, y, None, ws)
        B.cct_mx_quantize(x, q)
        B.cct_mx_dequantize(q, values)
    step()
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step()
    for i in range(3):
        x.normal_()
        step()
        want = y.clone(), values.clone()
        for again in (graph.replay, step):
            y.fill_(float("nan"))
            values.fill_(float("nan"))
            torch.cuda.synchronize()
            with torch.cuda.stream(side):
                again()
            torch.cuda.synchronize()
            assert torch.equal(want[0], y) and torch.equal(want[1], values), i


def test_no_rows(B):
    e = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    q = B.MxMatrix(0, 64)
    B.cct_mx_quantize(e, q)
    B.cct_mx_dequantize(q, e)
    d = B.make_linear_desc(0, 8, 64, B.TYPE_BF16)
    w = given(B, *operand(torch.Generator().manual_seed(9), 8, 64)[:2], 64)
    B.cct_mx_linear_forward(d, e, w, None, None, torch.empty(0, 8, dtype=torch.bfloat16, device="cuda"), None,
                            B.alloc_mx_linear_workspace(d, True))
