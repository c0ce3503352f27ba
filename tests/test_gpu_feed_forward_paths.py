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
