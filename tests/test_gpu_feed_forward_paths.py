"""Which kernels the products of feed-forward blocks run on, and that every one of them is right: whole numbers, whose sums are
exact in fp32 in any order, so that a step of a contraction that is lost, repeated or taken from another row shows in the
results' bits.  The reference is a product in 64 bits of the same numbers; the names are those of the profile."""
import pytest
import torch

import feed_forward_util as ff

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available()
    from paper_1504_04343_amd import binding
    return binding


@pytest.fixture(autouse=True)
def memory():
    """Tensors of tens of gigabytes are given back, not kept for the next test."""
    yield
    torch.cuda.empty_cache()


def consts(B, type):
    return dict(f32=B.TYPE_F32, bf16=B.TYPE_BF16, f16=B.TYPE_F16)[type], ff.TYPES[type]


def numbers(g, rows, cols, dt, most=1, pad=0):
    """Whole numbers from -most to most, rows cols + pad apart."""
    flat = torch.empty(rows, cols + pad, dtype=dt, device="cuda")
    for r in range(0, rows, max(1, (1 << 28) // (cols + pad))):     # in parts: whole int64 tensors would not fit
        part = flat[r:r + max(1, (1 << 28) // (cols + pad))]
        part.copy_(torch.randint(-most, most + 1, part.shape, generator=g, device="cuda", dtype=torch.int8))
    return flat[:, :cols]


def product(a, b, step=1 << 20):
    """a b^T in 64 bits, `step` steps of the contraction at a time."""
    out = torch.zeros(a.shape[0], b.shape[0], dtype=torch.float64, device="cuda")
    for k in range(0, a.shape[1], step):
        out += a[:, k:k + step].double() @ b[:, k:k + step].double().t()
    assert out.numel() == 0 or float(out.abs().max()) < 2 ** 24
    return out


def column_product(a, b):
    """a^T b in 64 bits for long columns, 2^14 of their values at a time."""
    n = a.shape[0] >> 14 << 14
    out = a[n:].double().t() @ b[n:].double()
    if n:
        tall = [t[:n].double().view(-1, 1 << 14, t.shape[1]) for t in (a, b)]
        out += torch.bmm(tall[0].transpose(1, 2).contiguous(), tall[1]).sum(0)
    return out


def empty(rows, cols, dt, pad=0):
    return ff.empty_gpu(rows, cols, dt, pad)


def profiled(B, call):
    """The names of what a call launches, in order of their first launch."""
    torch.cuda.synchronize()
    B.cct_profile_enable(True)
    try:
        call()
        torch.cuda.synchronize()
    finally:
        B.cct_profile_enable(False)
    return [e["name"] for e in B.cct_profile_read(64) for _ in range(e["launches"])]


def same(name, got, want):
    """Bit for bit the value rounded once to the type."""
    want = want.to(got.dtype)
    if not torch.equal(got, want):
        bad = got != want
        at = tuple(int(i) for i in bad.nonzero()[0])
        raise AssertionError("%s: %d of %d differ; the first at %s: %g, expected %g" % (
            name, int(bad.sum()), got.numel(), at, float(got[at]), float(want[at])))


@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("N,K,kernel", [(130, 1 << 24, "ff_tile_kernel<64x64"), (70, (1 << 24) + (1 << 19), "ff_general_kernel")])
def test_rows_longer_than_a_tile_reaches(B, type, N, K, kernel):
    """A tile's loads have 32 bits for its rows: 128 rows of 2^24 values are beyond them, 64 of somewhat more too."""
    t, dt = consts(B, type)
    g = torch.Generator(device="cuda").manual_seed(N)
    x, w = numbers(g, N, K, dt), numbers(g, N, K, dt)
    bias = numbers(g, 1, N, dt).view(N)
    d = B.make_linear_desc(N, N, K, t, B.ACT_RELU)
    y, z = empty(N, N, dt), empty(N, N, dt)
    ws = B.alloc_linear_workspace(d, B.PASS_FORWARD)
    assert any(n.startswith(kernel) for n in profiled(B, lambda: B.cct_linear_forward(d, x, w, bias, None, y, z, ws)))
    del ws
    want = product(x, w) + bias.double()
    same("z", z, want)
    same("y", y, want.clamp(min=0))
    e = B.make_gated_desc(N, N // 2, K, t, B.ACT_RELU)
    h, gg, uu = (empty(N, N // 2, dt) for _ in range(3))
    B.cct_gated_forward(e, x, w[:N // 2], w[N // 2:N // 2 * 2], h, gg, uu, B.alloc_gated_workspace(e, B.PASS_FORWARD))
    both = product(x, w)
    same("g", gg, both[:, :N // 2])
    same("u", uu, both[:, N // 2:N // 2 * 2])
    # act(g) * u of the fp32 sums may need more than 24 bits: rounded to fp32 first, then to the type
    same("h", h, (both[:, :N // 2].clamp(min=0) * both[:, N // 2:N // 2 * 2]).float())


@pytest.mark.parametrize("type", ["bf16", "f16"])
def test_gradients_of_rows_longer_than_a_tile_reaches(B, type):
    """Weights and inputs of such rows across the contraction, 64 steps of which are a stage."""
    t, dt = consts(B, type)
    M, N, K = 70, 66, (1 << 24) + (1 << 19)
    g = torch.Generator(device="cuda").manual_seed(7)
    x, w, dy, z = numbers(g, M, K, dt), numbers(g, N, K, dt), numbers(g, M, N, dt), numbers(g, M, N, dt)
    d = B.make_linear_desc(M, N, K, t, B.ACT_RELU)
    dx, dw = empty(M, K, dt), empty(N, K, dt)
    db = torch.full((N,), float("nan"), dtype=dt, device="cuda")
    ws = B.alloc_linear_workspace(d, B.PASS_BACKWARD)
    names = profiled(B, lambda: B.cct_linear_backward(d, x, w, z, dy, dx, dw, db, ws))
    assert names.count("ff_general_kernel") == 2, names
    dy.mul_(z > 0)
    same("dbias", db, dy.double().sum(0))
    for k in range(0, K, 1 << 21):
        part = slice(k, k + (1 << 21))
        same("dx", dx[:, part], product(dy, w[:, part].t()))
        same("dw", dw[:, part], product(dy.t(), x[:, part].t()))


def test_more_rows_than_threads_of_a_launch(B):
    """2^30 rows of 8 values: in tiles of 64, or 64 rows to a workgroup of dz, more than the 2^32 threads that a launch takes."""
    t, dt = consts(B, "bf16")
    M, N, K = (1 << 30) + 100, 8, 8
    if torch.cuda.mem_get_info()[0] < 150e9:
        pytest.skip("needs 150 GB")
    g = torch.Generator(device="cuda").manual_seed(3)
    x, w = numbers(g, M, K, dt), numbers(g, N, K, dt)
    d = B.make_linear_desc(M, N, K, t, B.ACT_RELU)
    y, z = (torch.empty(M, N, dtype=dt, device="cuda") for _ in range(2))
    ws = B.alloc_linear_workspace(d, B.PASS_FORWARD)
    B.cct_linear_forward(d, x, w, None, None, y, z, ws)
    del ws
    parts = [slice(m, min(m + (1 << 26), M)) for m in range(0, M, 1 << 26)]
    for p in parts:
        want = product(x[p], w)
        same("z", z[p], want)
        same("y", y[p], want.clamp_(min=0))
    del want
    dy, dx, dw = y, torch.empty(M, K, dtype=dt, device="cuda"), empty(N, K, dt)
    for p in parts:
        dy[p].copy_(torch.randint(-1, 2, dy[p].shape, generator=g, device="cuda", dtype=torch.int8))
    db = torch.full((N,), float("nan"), dtype=dt, device="cuda")
    ws = B.alloc_linear_workspace(d, B.PASS_BACKWARD)
    B.cct_linear_backward(d, x, w, z, dy, dx, dw, db, ws)
    del ws
    want_w, want_b = torch.zeros(N, K, dtype=torch.float64, device="cuda"), torch.zeros(N, dtype=torch.float64, device="cuda")
    for p in parts:
        dz = dy[p].mul_(z[p] > 0)
        same("dx", dx[p], product(dz, w.t()))
        want_w += column_product(dz, x[p])
        want_b += dz.double().sum(0)
    same("dw", dw, want_w)
    same("dbias", db, want_b)


def test_more_joined_results_than_threads_of_a_launch(B):
    """fp32 results with an activation go through the workspace: 2^34 of them, four to a thread."""
    M, N, K = (1 << 22) + 40, 4096, 4
    if torch.cuda.mem_get_info()[0] < 160e9:
        pytest.skip("needs 160 GB")
    g = torch.Generator(device="cuda").manual_seed(4)
    x, w = numbers(g, M, K, torch.float32, 3), numbers(g, N, K, torch.float32, 3)
    d = B.make_linear_desc(M, N, K, B.TYPE_F32, B.ACT_RELU)
    y = torch.empty(M, N, device="cuda")
    ws = B.alloc_linear_workspace(d, B.PASS_FORWARD)
    B.cct_linear_forward(d, x, w, None, None, y, None, ws)
    for m in range(0, M, 1 << 17):
        p = slice(m, min(m + (1 << 17), M))
        want = x[p] @ w.t()          # exact in any precision that holds 36
        same("y", y[p], want.clamp_(min=0))


@pytest.mark.parametrize("type", ["bf16", "f16"])
def test_gradients_of_more_outputs_than_a_tile_reaches(B, type):
    """17 million outputs: dz's rows, along the contraction of dx and across that of dw."""
    t, dt = consts(B, type)
    M, N, K = 70, (1 << 24) + (1 << 21), 16
    g = torch.Generator(device="cuda").manual_seed(7)
    x, w, dy, z = numbers(g, M, K, dt), numbers(g, N, K, dt), numbers(g, M, N, dt), numbers(g, M, N, dt)
    d = B.make_linear_desc(M, N, K, t, B.ACT_RELU)
    dx, dw = empty(M, K, dt), empty(N, K, dt)
    db = torch.full((N,), float("nan"), dtype=dt, device="cuda")
    ws = B.alloc_linear_workspace(d, B.PASS_BACKWARD)
    assert "ff_general_kernel" in profiled(B, lambda: B.cct_linear_backward(d, x, w, z, dy, dx, dw, db, ws))
    dy.mul_(z > 0)
    same("dx", dx, product(dy, w.t()))
    for n in range(0, N, 1 << 21):
        cols = dy[:, n:n + (1 << 21)]
        same("dw", dw[n:n + (1 << 21)], product(cols.t(), x.t()))
        same("dbias", db[n:n + (1 << 21)], cols.double().sum(0))


@pytest.mark.parametrize("type", list(ff.TYPES))
def test_three_million_outputs(B, type):
    """More outputs than their square allows, of few inputs."""
    t, dt = consts(B, type)
    M, N, K = 8, 3000000, 8
    g = torch.Generator(device="cuda").manual_seed(9)
    x, w, bias, dy = numbers(g, M, K, dt), numbers(g, N, K, dt), numbers(g, 1, N, dt).view(N), numbers(g, M, N, dt)
    d = B.make_linear_desc(M, N, K, t, B.ACT_RELU)
    y, z, dx, dw = empty(M, N, dt), empty(M, N, dt), empty(M, K, dt), empty(N, K, dt)
    db = torch.full((N,), float("nan"), dtype=dt, device="cuda")
    B.cct_linear_forward(d, x, w, bias, None, y, z, B.alloc_linear_workspace(d, B.PASS_FORWARD))
    want = product(x, w) + bias.double()
    same("z", z, want)
    same("y", y, want.clamp(min=0))
    B.cct_linear_backward(d, x, w, z, dy, dx, dw, db, B.alloc_linear_workspace(d, B.PASS_BACKWARD))
    dy.mul_(z > 0)
    same("dx", dx, product(dy, w.t()))
    same("dw", dw, product(dy.t(), x.t()))
    same("dbias", db, dy.double().sum(0))
    e = B.make_gated_desc(M, N, K, t, B.ACT_RELU)
    dx, dwg, dwu, h, gg, uu = empty(M, K, dt), empty(N, K, dt), empty(N, K, dt), empty(M, N, dt), empty(M, N, dt), empty(M, N, dt)
    wu = numbers(g, N, K, dt)
    B.cct_gated_forward(e, x, w, wu, h, gg, uu, B.alloc_gated_workspace(e, B.PASS_FORWARD))
    want_g, want_u = product(x, w), product(x, wu)
    same("g", gg, want_g)
    same("u", uu, want_u)
    same("h", h, want_g.clamp(min=0) * want_u)
    B.cct_gated_backward(e, x, w, wu, gg, uu, dy, dx, dwg, dwu, B.alloc_gated_workspace(e, B.PASS_BACKWARD))
    dg, du = dy.double() * want_u * (want_g > 0), dy.double() * want_g.clamp(min=0)
    same("dx", dx, product(dg, w.t()) + product(du, wu.t()))
    same("dwg", dwg, product(dg.t(), x.t()))
    same("dwu", dwu, product(du.t(), x.t()))


@pytest.mark.parametrize("type,N", [("f32", (1 << 26) + 80), ("bf16", (1 << 27) + 80)])
def test_few_rows_of_more_outputs_than_threads_of_a_launch(B, type, N):
    """16 outputs to a workgroup of the kernel for few rows would be 2^32 threads."""
    t, dt = consts(B, type)
    M, K = 2, 8
    g = torch.Generator(device="cuda").manual_seed(10)
    x, w = numbers(g, M, K, dt), numbers(g, N, K, dt)
    d = B.make_linear_desc(M, N, K, t, B.ACT_RELU)
    y = empty(M, N, dt)
    ws = B.alloc_linear_workspace(d, B.PASS_FORWARD)
    assert "ff_rows_kernel" not in profiled(B, lambda: B.cct_linear_forward(d, x, w, None, None, y, None, ws))
    for n in range(0, N, 1 << 24):
        same("y", y[:, n:n + (1 << 24)], product(x, w[n:n + (1 << 24)]).clamp(min=0))
    small = B.make_linear_desc(M, 4096, K, t, B.ACT_RELU)
    assert "ff_rows_kernel" in profiled(B, lambda: B.cct_linear_forward(small, x, w[:4096], None, None, empty(M, 4096, dt), None, ws))


def test_column_sums_of_more_outputs_than_threads_of_a_launch(B):
    """The sum of columns takes 16 of them and 1024 threads to a workgroup, in two launches."""
    t, dt = consts(B, "bf16")
    M, N, K = 70, (1 << 26) + 80, 8      # more rows than one workgroup of dz takes
    if torch.cuda.mem_get_info()[0] < 60e9:
        pytest.skip("needs 60 GB")
    g = torch.Generator(device="cuda").manual_seed(11)
    x, w, dy, z = numbers(g, M, K, dt), numbers(g, N, K, dt), numbers(g, M, N, dt), numbers(g, M, N, dt)
    d = B.make_linear_desc(M, N, K, t, B.ACT_RELU)
    dx, dw = empty(M, K, dt), empty(N, K, dt)
    db = torch.full((N,), float("nan"), dtype=dt, device="cuda")
    ws = B.alloc_linear_workspace(d, B.PASS_BACKWARD)
    B.cct_linear_backward(d, x, w, z, dy, dx, dw, db, ws)
    dy.mul_(z > 0)
    same("dx", dx, product(dy, w.t()))
    for n in range(0, N, 1 << 22):
        cols = dy[:, n:n + (1 << 22)]
        same("dw", dw[n:n + (1 << 22)], product(cols.t(), x.t()))
        same("dbias", db[n:n + (1 << 22)], cols.double().sum(0))


def test_fp32_rows_longer_than_the_split_product_addresses(B):
    """Weights of 2^22 values a row and more run on the general kernel, in splits of the contraction."""
    M, N, K = 40, 48, (1 << 22) + 8
    g = torch.Generator(device="cuda").manual_seed(12)
    x, w, u = (numbers(g, r, K, torch.float32) for r in (M, N, N))
    d = B.make_linear_desc(M, N, K, B.TYPE_F32, B.ACT_RELU)
    y, z = empty(M, N, torch.float32), empty(M, N, torch.float32)
    ws = B.alloc_linear_workspace(d, B.PASS_FORWARD)
    ws.fill_(0xff)
    assert profiled(B, lambda: B.cct_linear_forward(d, x, w, None, None, y, z, ws)) == ["ff_general_kernel"]
    want = product(x, w)
    same("z", z, want)
    same("y", y, want.clamp(min=0))
    e = B.make_gated_desc(M, N, K, B.TYPE_F32, B.ACT_RELU)
    h, gg, uu = (empty(M, N, torch.float32) for _ in range(3))
    ws = B.alloc_gated_workspace(e, B.PASS_FORWARD)
    ws.fill_(0xff)
    B.cct_gated_forward(e, x, w, u, h, gg, uu, ws)
    same("g", gg, want)
    same("u", uu, product(x, u))
    same("h", h, (want.clamp(min=0) * product(x, u)).float())
    dz = numbers(g, M, N, torch.float32)
    dx, dw = empty(M, K, torch.float32), empty(N, K, torch.float32)
    l = B.make_linear_desc(M, N, K, B.TYPE_F32)
    B.cct_linear_backward(l, x, w, None, dz, dx, dw, None, B.alloc_linear_workspace(l, B.PASS_BACKWARD))
    same("dx", dx, product(dz, w.t()))
    same("dw", dw, product(dz.t(), x.t()))


# What is computed; the tile; whether the contraction is split; what of the results is left for a launch of its own; M, N, K in
# multiples of 8, whose operands are taken in place, and otherwise, copied.
ALONE = [
    ("linear", "256x256", False, None, (8121, 1312, 144), (8121, 1305, 141)),
    ("linear", "256x256", False, "columns", (3082, 5144, 264), (3082, 5139, 259)),
    ("linear", "256x256", False, "rows", (5470, 2952, 264), (7223, 2207, 261)),
    ("linear", "192x256", False, None, (3349, 2328, 136), (2307, 3345, 139)),
    ("linear", "128x128", True, None, (328, 648, 3360), (328, 647, 3357)),
    ("linear", "128x128", False, None, (1677, 1176, 136), (1685, 1157, 141)),
    ("linear", "64x128", True, None, (264, 392, 2016), (399, 257, 2001)),
    ("linear", "64x128", False, None, (1220, 784, 136), (1220, 769, 143)),
    ("linear", "64x64", True, None, (136, 136, 1224), (136, 137, 1217)),
    ("linear", "64x64", False, None, (137, 136, 144), (136, 139, 139)),
    ("gated", "256x256", False, None, (580, 8288, 144), (580, 8283, 137)),
    ("gated", "256x256", False, "columns", (2949, 2696, 264), (2949, 2693, 263)),
    ("gated", "256x256", False, "rows", (2331, 3424, 272), (2818, 2857, 257)),
    ("gated", "192x256", False, None, (385, 8200, 144), (385, 8197, 143)),
    ("gated", "128x128", True, None, (258, 400, 3360), (258, 399, 3357)),
    ("gated", "128x128", False, None, (833, 1176, 136), (769, 1251, 139)),
    ("gated", "64x128", True, None, (139, 328, 2008), (258, 195, 2001)),
    ("gated", "64x128", False, None, (774, 616, 136), (644, 737, 137)),
    ("gated", "64x64", True, None, (136, 136, 1224), (136, 137, 1217)),
    ("gated", "64x64", False, None, (137, 136, 144), (136, 139, 139)),
    ("dx", "256x256", False, None, (1613, 144, 8888), (1613, 139, 8883)),
    ("dx", "256x256", False, "columns", (3723, 152, 5328), (3723, 147, 5321)),
    ("dx", "256x256", False, "rows", (8667, 400, 2000), (8666, 385, 1935)),
    ("dx", "192x256", False, None, (1737, 272, 6168), (1735, 265, 6177)),
    ("dx", "128x128", True, None, (403, 6008, 1960), (403, 6005, 1953)),
    ("dx", "128x128", False, None, (784, 776, 8592), (784, 775, 8587)),
    ("dx", "64x128", True, None, (139, 6296, 2440), (139, 6291, 2437)),
    ("dx", "64x128", False, None, (398, 4912, 8984), (398, 4909, 8979)),
    ("dx", "64x64", True, None, (174, 6264, 5408), (174, 6257, 5401)),
    ("dx", "64x64", False, None, (272, 1760, 6024), (272, 1755, 6019)),
    ("dw", "256x256", False, None, (141, 1608, 8840), (141, 1605, 8839)),
    ("dw", "256x256", False, "columns", (145, 3744, 5272), (152, 3713, 5255)),
    ("dw", "256x256", False, "rows", (410, 8688, 1968), (410, 8681, 1963)),
    ("dw", "192x256", False, None, (272, 1760, 6024), (272, 1755, 6019)),
    ("dw", "128x128", True, None, (5958, 400, 1928), (5995, 395, 1923)),
    ("dw", "128x128", False, None, (784, 776, 8592), (784, 775, 8587)),
    ("dw", "64x128", True, None, (6292, 144, 2456), (6292, 139, 2449)),
    ("dw", "64x128", False, None, (5511, 408, 8968), (5511, 401, 8967)),
    ("dw", "64x64", True, None, (6179, 176, 5440), (6214, 183, 5417)),
    ("dw", "64x64", False, None, (1737, 272, 6168), (1735, 265, 6177)),
    ("gated dx", "256x256", False, None, (1348, 776, 8928), (1348, 773, 8925)),
    ("gated dx", "256x256", False, "columns", (1794, 840, 8232), (1794, 833, 8229)),
    ("gated dx", "256x256", False, "rows", (1834, 792, 8824), (1813, 841, 8549)),
    ("gated dx", "192x256", False, None, (1026, 776, 8928), (1026, 775, 8923)),
    ("gated dx", "128x128", True, None, (387, 5696, 1928), (387, 5695, 1929)),
    ("gated dx", "128x128", False, None, (925, 920, 8032), (925, 917, 8027)),
    ("gated dx", "64x128", True, None, (138, 2960, 5352), (136, 3013, 5271)),
    ("gated dx", "64x128", False, None, (398, 4912, 8984), (398, 4909, 8979)),
    ("gated dx", "64x64", True, None, (20, 4112, 6408), (20, 4113, 6405)),
    ("gated dw", "256x256", False, None, (136, 4168, 3776), (136, 4161, 3773)),
    ("gated dw", "256x256", False, "columns", (408, 8992, 1960), (408, 8985, 1955)),
    ("gated dw", "256x256", False, "rows", (151, 5072, 3976), (151, 5065, 3975)),
    ("gated dw", "192x256", False, None, (387, 5696, 1928), (387, 5695, 1929)),
    ("gated dw", "128x128", True, None, (5349, 1776, 2216), (5349, 1769, 2213)),
    ("gated dw", "128x128", False, None, (925, 920, 8032), (925, 917, 8027)),
    ("gated dw", "64x128", True, None, (8987, 16, 8992), (8987, 15, 8987)),
]
# The backward pass of; the tile that its products share; whether dx's contraction is split, and the weights'; sizes as above.
TOGETHER = [
    ("linear", "128x128", (False, False), (144, 136, 5416), (144, 137, 5409)),
    ("linear", "128x128", (False, True), (5470, 144, 136), (5472, 139, 137)),
    ("linear", "128x128", (True, False), (137, 5512, 144), (137, 5505, 139)),
    ("linear", "128x128", (True, True), (1805, 520, 136), (1805, 515, 137)),
    ("linear", "64x128", (False, False), (136, 144, 2752), (136, 137, 2753)),
    ("linear", "64x128", (False, True), (4313, 144, 136), (4286, 137, 137)),
    ("linear", "64x128", (True, False), (138, 4312, 136), (141, 4161, 137)),
    ("linear", "64x128", (True, True), (265, 2288, 136), (258, 2261, 139)),
    ("linear", "64x64", (False, False), (137, 136, 144), (136, 139, 139)),
    ("linear", "64x64", (False, True), (775, 144, 144), (777, 137, 137)),
    ("linear", "64x64", (True, False), (137, 792, 144), (137, 789, 139)),
    ("linear", "64x64", (True, True), (266, 816, 136), (771, 257, 141)),
    ("gated", "128x128", (False, False), (197, 136, 4880), (197, 137, 4877)),
    ("gated", "128x128", (False, True), (7391, 144, 136), (6981, 143, 137)),
    ("gated", "128x128", (True, False), (141, 2768, 136), (138, 2717, 137)),
    ("gated", "128x128", (True, True), (1540, 264, 144), (1548, 261, 143)),
    ("gated", "64x128", (False, False), (136, 144, 3464), (136, 141, 3463)),
    ("gated", "64x128", (False, True), (1547, 136, 456), (1093, 137, 643)),
    ("gated", "64x128", (True, False), (137, 2056, 144), (137, 2055, 139)),
    ("gated", "64x128", (True, True), (259, 1104, 136), (259, 1101, 137)),
    ("gated", "64x64", (False, False), (137, 136, 144), (136, 139, 139)),
    ("gated", "64x64", (False, True), (1096, 136, 200), (1097, 137, 193)),
    ("gated", "64x64", (True, False), (136, 392, 144), (136, 387, 143)),
    ("gated", "64x64", (True, True), (265, 392, 136), (265, 387, 137)),
]


def forms(rows):
    """Each with its sizes in multiples of 8, in rows that are further apart, in bf16, and with the others in fp16."""
    return [pytest.param(*r[:-2], r[-2 + i], t, 8 * (1 - i), id="-".join(str(v).replace(" ", "_") for v in (*r[:-2], t)))
            for r in rows for i, t in enumerate(("bf16", "f16"))]


def check_launches(names, tile, split, cut, products=1):
    tiles = [n for n in names if n.startswith("ff_tile_kernel")]
    assert len(tiles) == products * (2 if cut else 1), names
    first = [n for n in tiles if n.startswith("ff_tile_kernel<%s, " % tile)]
    assert first and (", 1 splits>" in first[0]) == (not split), names


def forward_case(B, kind, tile, split, cut, sizes, type, pad):
    t, dt = consts(B, type)
    M, N, K = sizes
    g = torch.Generator(device="cuda").manual_seed(M + N + K)
    x, w = numbers(g, M, K, dt, 1, pad), numbers(g, N, K, dt, 1, pad)
    if kind == "linear":
        bias, r = numbers(g, 1, N, dt, 5).view(N), numbers(g, M, N, dt, 5, 3)
        d = B.make_linear_desc(M, N, K, t, B.ACT_RELU)
        y, z = empty(M, N, dt, 3), empty(M, N, dt, 3)
        ws = B.alloc_linear_workspace(d, B.PASS_FORWARD)
        ws.fill_(0xff)
        check_launches(profiled(B, lambda: B.cct_linear_forward(d, x, w, bias, r, y, z, ws)), tile, split, cut)
        want = product(x, w) + bias.double()
        same("z", z, want)
        same("y", y, want.clamp(min=0) + r.double())
        assert ff.untouched(y, N) and ff.untouched(z, N)
        return
    wu = numbers(g, N, K, dt, 1, pad)
    e = B.make_gated_desc(M, N, K, t, B.ACT_RELU)
    h, gg, uu = (empty(M, N, dt, 3) for _ in range(3))
    ws = B.alloc_gated_workspace(e, B.PASS_FORWARD)
    ws.fill_(0xff)
    check_launches(profiled(B, lambda: B.cct_gated_forward(e, x, w, wu, h, gg, uu, ws)), tile, split, cut)
    want_g, want_u = product(x, w), product(x, wu)
    same("g", gg, want_g)
    same("u", uu, want_u)
    same("h", h, want_g.clamp(min=0) * want_u)
    assert all(ff.untouched(v, N) for v in (h, gg, uu))


class Backward:
    """The backward pass of a linear layer or a gated block with ReLU, z (g, u) and dy of -1, 0 and 1: dz, dg and du are
    whole numbers too."""

    def __init__(self, B, gated, sizes, type, pad):
        self.B, self.gated = B, gated
        t, dt = consts(B, type)
        M, N, K = self.sizes = sizes
        g = torch.Generator(device="cuda").manual_seed(M + N + K)
        self.dt = dt
        self.x = numbers(g, M, K, dt, 1, pad)
        self.w = [numbers(g, N, K, dt, 1, pad) for _ in range(1 + gated)]
        self.z = [numbers(g, M, N, dt, 1, pad) for _ in range(1 + gated)]
        self.dy = numbers(g, M, N, dt, 1, pad)
        self.d = (B.make_gated_desc if gated else B.make_linear_desc)(M, N, K, t, B.ACT_RELU)
        self.ws = (B.alloc_gated_workspace if gated else B.alloc_linear_workspace)(self.d, B.PASS_BACKWARD)

    def run(self, dx=True, dw=True, db=True):
        """Results, and the names of the launches."""
        M, N, K = self.sizes
        self.ws.fill_(0xff)
        dx = empty(M, K, self.dt, 3) if dx else None
        dw = [empty(N, K, self.dt, 3) for _ in self.w] if dw else [None] * len(self.w)
        if self.gated:
            names = profiled(self.B, lambda: self.B.cct_gated_backward(self.d, self.x, *self.w, *self.z, self.dy, dx, *dw, self.ws))
            return [dx, *dw], names
        db = torch.full((N,), float("nan"), dtype=self.dt, device="cuda") if db else None
        names = profiled(self.B, lambda: self.B.cct_linear_backward(self.d, self.x, self.w[0], self.z[0], self.dy, dx, dw[0], db, self.ws))
        return [dx, *dw, db], names

    def check(self, got):
        K, dy = self.sizes[2], self.dy.double()
        g = self.z[0].double()
        if self.gated:
            dz = [dy * self.z[1].double() * (g > 0), dy * g.clamp(min=0)]
        else:
            dz = [dy * (g > 0)]
        for name, t, v in zip(("dx", "dw", "du"), got, [sum(product(a, w.t()) for a, w in zip(dz, self.w))] +
                              [product(a.t(), self.x.t()) for a in dz]):
            same(name, t, v)
            assert ff.untouched(t, K)
        if not self.gated:
            same("dbias", got[2], dz[0].sum(0))


@pytest.mark.parametrize("what,tile,split,cut,sizes,type,pad", forms([r for r in ALONE if r[0] in ("linear", "gated")]))
def test_forward_tiles(B, what, tile, split, cut, sizes, type, pad):
    forward_case(B, what, tile, split, cut, sizes, type, pad)


@pytest.mark.parametrize("what,tile,split,cut,sizes,type,pad", forms([r for r in ALONE if r[0] not in ("linear", "gated")]))
def test_backward_tiles(B, what, tile, split, cut, sizes, type, pad):
    """Products in launches of their own; each gradient alone has the same bits."""
    b = Backward(B, what.startswith("gated"), sizes, type, pad)
    got, names = b.run()
    assert not any(n.startswith("ff_tile_kernel_together") for n in names), names
    b.check(got)
    dx, names_x = b.run(True, False, False)
    dw, names_w = b.run(False, True, False)
    assert torch.equal(dx[0], got[0]) and all(torch.equal(v, u) for v, u in zip(dw[1:1 + len(b.w)], got[1:]))
    if what.endswith("dx"):
        check_launches(names_x, tile, split, cut)
    else:
        check_launches(names_w, tile, split, cut, len(b.w))


@pytest.mark.parametrize("what,tile,splits,sizes,type,pad", forms(TOGETHER))
def test_backward_products_that_share_a_launch(B, what, tile, splits, sizes, type, pad):
    b = Backward(B, what == "gated", sizes, type, pad)
    got, names = b.run()
    shared = "ff_tile_kernel_together<%s, %d products" % (tile, 1 + len(b.w))
    assert [n for n in names if n.startswith("ff_tile_kernel")][0].startswith(shared), names
    b.check(got)
    for i, want in enumerate(((True, False, False), (False, True, False))):
        some, names = b.run(*want)
        assert all(torch.equal(u, v) for u, v in zip(some, got) if u is not None)
        mine = [n for n in names if n.startswith("ff_tile_kernel_together<" + tile)]
        assert len(mine) == 1 and (", 1 splits>" in mine[0]) == (not splits[i]), names


def test_every_plan_has_a_case():
    """Of the tiles and splits that ff_product.hip chooses from, with what is left over of the large ones."""
    plans = {(t, s, None) for t in ("128x128", "64x128", "64x64") for s in (False, True)}
    plans |= {("256x256", False, c) for c in (None, "rows", "columns")} | {("192x256", False, None)}
    have = {}
    for what, tile, split, cut, *_ in ALONE:
        have.setdefault(what, set()).add((tile, split, cut))
    for what in ("linear", "gated", "dx", "dw"):
        assert have[what] == plans, what
    assert len(TOGETHER) == 24


@pytest.mark.parametrize("type", list(ff.TYPES))
@pytest.mark.parametrize("M", [1, 16, 17, 32, 33, 64])
def test_few_rows_of_ragged_contractions(B, type, M):
    """No step lost or repeated at the ends of steps, waves and splits, in rows at any address."""
    t, dt = consts(B, type)
    rows = 0
    for N in (10, 72, 1100):
        for K in (1, 31, 33, 255, 1025, 8193, 20005):
            for pad in (0, 1, 2, 8 - K % 8):
                g = torch.Generator(device="cuda").manual_seed(K)
                x, w, u = numbers(g, M, K, dt, 1, pad), numbers(g, N, K, dt, 1, pad), numbers(g, N, K, dt, 1, pad)
                bias, r = numbers(g, 1, N, dt, 5).view(N), numbers(g, M, N, dt, 5)
                d = B.make_linear_desc(M, N, K, t, B.ACT_RELU)
                y, z = empty(M, N, dt, 1), empty(M, N, dt, 1)
                ws = B.alloc_linear_workspace(d, B.PASS_FORWARD)
                ws.fill_(0xff)
                rows += "ff_rows_kernel" in profiled(B, lambda: B.cct_linear_forward(d, x, w, bias, r, y, z, ws))
                want = product(x, w) + bias.double()
                same("z", z, want)
                same("y", y, want.clamp(min=0) + r.double())
                e = B.make_gated_desc(M, N, K, t, B.ACT_RELU)
                h, gg, uu = (empty(M, N, dt, 1) for _ in range(3))
                ws = B.alloc_gated_workspace(e, B.PASS_FORWARD)
                ws.fill_(0xff)
                B.cct_gated_forward(e, x, w, u, h, gg, uu, ws)
                want_g, want_u = product(x, w), product(x, u)
                same("g", gg, want_g)
                same("u", uu, want_u)
                same("h", h, want_g.clamp(min=0) * want_u)
    cases = 3 * 7 * 4
    assert rows == (cases if M <= (32 if type == "f32" else 16) else 0) or (type != "f32" and 0 < rows < cases)


def split_launches(names):
    """How many fp32 products ran, and whether partial sums were joined."""
    return sum(n.startswith("gemm_split") for n in names), "ff_join_kernel" in names


def test_fp32_products_in_several_parts_of_rows(B):
    """The packed operand of more than 19392 rows of 9216 values is more than 2^30 bytes: one part after the other, the last one
    smaller, stored directly, with an activation, in splits, and of a gated block."""
    dt = torch.float32
    M, N, K = 19600, 4096, 9216
    g = torch.Generator(device="cuda").manual_seed(13)
    x, w, bias, r = numbers(g, M, K, dt), numbers(g, N, K, dt), numbers(g, 1, N, dt, 5).view(N), numbers(g, M, N, dt, 5, 3)
    want = product(x, w)
    plain, act = (B.make_linear_desc(M, N, K, B.TYPE_F32, a) for a in (B.ACT_NONE, B.ACT_RELU))
    ws = B.alloc_linear_workspace(act, B.PASS_FORWARD)
    ws.fill_(0xff)
    y, z = empty(M, N, dt, 3), empty(M, N, dt, 3)
    assert split_launches(profiled(B, lambda: B.cct_linear_forward(plain, x, w, bias, None, y, None, ws))) == (2, False)
    same("y", y, want + bias.double())
    ws.fill_(0xff)
    assert split_launches(profiled(B, lambda: B.cct_linear_forward(act, x, w, bias, r, y, z, ws))) == (2, True)
    same("z", z, want + bias.double())
    same("y", y, (want + bias.double()).clamp(min=0) + r.double())
    few = B.make_linear_desc(M, 72, K, B.TYPE_F32)                       # the contraction in splits
    y = empty(M, 72, dt)
    ws.fill_(0xff)
    assert split_launches(profiled(B, lambda: B.cct_linear_forward(few, x, w[:72], None, None, y, None, ws))) == (2, True)
    same("y", y, want[:, :72])
    del ws, y, z, r
    F = 264
    e = B.make_gated_desc(M, F, K, B.TYPE_F32, B.ACT_RELU)
    h, gg, uu = (empty(M, F, dt, 3) for _ in range(3))
    ws = B.alloc_gated_workspace(e, B.PASS_FORWARD)
    ws.fill_(0xff)
    assert split_launches(profiled(B, lambda: B.cct_gated_forward(e, x, w[:F], w[F:2 * F], h, gg, uu, ws))) == (4, True)
    same("g", gg, want[:, :F])
    same("u", uu, want[:, F:2 * F])
    same("h", h, want[:, :F].clamp(min=0) * want[:, F:2 * F])


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("K,splits", [(264, True), (2048, False)])
def test_fp32_gradients_in_several_parts_of_rows(B, gated, K, splits):
    """dx of 19600 rows and 9216 outputs, and dw of 9216 rows and a contraction of 19600 steps."""
    b = Backward(B, gated, (19600, 9216, K), "f32", 0)
    got, names = b.run()
    assert split_launches(names) == (8 if gated else 4, splits or gated), names
    b.check(got)
    dx, names = b.run(True, False, False)
    assert split_launches(names)[0] == (4 if gated else 2) and torch.equal(dx[0], got[0])


@pytest.mark.parametrize("type", list(ff.TYPES))
@pytest.mark.parametrize("which", range(3), ids=["rows", "outputs", "inputs"])
def test_sizes_at_the_limit(B, type, which):
    """2^31 - 256 rows, outputs or inputs, of one value each."""
    t, dt = consts(B, type)
    if torch.cuda.mem_get_info()[0] < 150e9:
        pytest.skip("needs 150 GB")
    M, N, K = [(1 << 31) - 256 if i == which else 1 for i in range(3)]
    g = torch.Generator(device="cuda").manual_seed(which)

    def values(r, c):
        return numbers(g, 1, r * c, dt).view(r, c) if r > 1 else numbers(g, r, c, dt)
    x, w = values(M, K), values(N, K)
    d = B.make_linear_desc(M, N, K, t, B.ACT_RELU)
    y, z = (torch.full((M, N), float("nan"), dtype=dt, device="cuda") for _ in range(2))
    ws = B.alloc_linear_workspace(d, B.PASS_FORWARD)
    print("forward", type, M, N, K, flush=True)
    B.cct_linear_forward(d, x, w, None, None, y, z, ws)
    torch.cuda.synchronize()
    del ws
    # with one input, z is x w whatever the shape; with one row and output, a sum
    step = 1 << 26
    flat = [v.reshape(-1) for v in (x, w, y, z)]

    def part(v, p):
        return v[p] if v.numel() > 1 else v
    spans = [slice(i, min(i + step, (1 << 31) - 256)) for i in range(0, (1 << 31) - 256, step)]
    if which == 2:
        want = sum(float((flat[0][p].double() * flat[1][p].double()).sum()) for p in spans)
        assert float(z) == float(torch.tensor(want, dtype=torch.float64).to(dt)) and float(y) == max(0.0, float(z))
    else:
        for p in spans:
            want = part(flat[0], p) * part(flat[1], p)
            same("z", flat[3][p], want)
            same("y", flat[2][p], want.clamp_(min=0))
    del y, want
    flat = flat[:2]
    z.fill_(1.0)                     # half of dy is kept
    z.view(-1)[::2] = -1.0 if which < 2 else 1.0
    dy = values(M, N)
    dx, dw = (torch.full(v.shape, float("nan"), dtype=dt, device="cuda") for v in (x, w))
    db = torch.full((N,), float("nan"), dtype=dt, device="cuda")
    ws = B.alloc_linear_workspace(d, B.PASS_BACKWARD)
    print("backward", type, M, N, K, flush=True)
    B.cct_linear_backward(d, x, w, z, dy, dx, dw, db, ws)
    torch.cuda.synchronize()
    del ws
    dz, f = dy.view(-1), [v.reshape(-1) for v in (dx, dw, x, w)]
    sums = [0.0, 0.0, 0.0]           # of dx, dw, dbias where each is one value
    for p in spans:
        v = part(dz, p) * (part(z.view(-1), p) > 0)
        for i, other in ((0, f[3]), (1, f[2])):
            term = v * part(other, p)
            if f[i].numel() > 1:
                same(("dx", "dw")[i], f[i][p], term.expand_as(f[i][p]))
            else:
                sums[i] += float(term.double().sum())
        if N > 1:
            same("dbias", db[p], v)
        elif M > 1:
            sums[2] += float(v.double().sum())
        else:
            sums[2] = float(v)
    for i, got in ((0, dx), (1, dw), (2, db)):
        if got.numel() == 1:
            assert float(got) == float(torch.tensor(sums[i], dtype=torch.float64).to(dt)), i


@pytest.mark.parametrize("type", ["bf16", "f16"])
def test_copied_rows_keep_their_smallest_numbers(B, type):
    """Rows of 17 values are copied for the tiles: subnormal ones too, as they are."""
    t, dt = consts(B, type)
    M, N, K = 90, 40, 17
    low = 2.0 ** (-133 if type == "bf16" else -24)
    g = torch.Generator(device="cuda").manual_seed(2)
    x = (numbers(g, M, K, torch.float64, 3) * low).to(dt)
    w = numbers(g, N, K, dt, 2) * 2.0 ** 12
    d = B.make_linear_desc(M, N, K, t)
    y = empty(M, N, dt)
    names = profiled(B, lambda: B.cct_linear_forward(d, x, w, None, None, y, None, B.alloc_linear_workspace(d, B.PASS_FORWARD)))
    assert any(n.startswith("ff_dz_kernel") for n in names)
    same("y", y, x.double() @ w.double().t())
    dy = torch.eye(M, N, device="cuda").to(dt)       # dw is x's first rows
    dw = empty(N, K, dt)
    B.cct_linear_backward(d, x, None, None, dy, None, dw, None, B.alloc_linear_workspace(d, B.PASS_BACKWARD))
    same("dw", dw, x[:N])
