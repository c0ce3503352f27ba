"""A layer of experts for a few tokens (cct_moe_forward) against 64 bits on the CPU, within bounds derived from the types
(moe_util.py): types and activations, one token to 64, one expert to 512, odd sizes, strides and addresses, ties, experts that
are not chosen, values that are not finite, captured graphs, another stream, offsets beyond 32 bits."""
import pytest
import torch

import feed_forward_util as ff
import moe_util as moe

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available()
    from paper_1504_04343_amd import binding
    return binding


def experts(g, E, rows, cols, dt, pad=0, off=0):
    """E matrices on the CPU, rows cols + pad apart, `off` values in front of the first and between them."""
    ld, e = cols + pad, rows * (cols + pad) + off
    flat = (torch.randn(E * e + off, generator=g) * cols ** -0.5).to(dt)
    return flat.as_strided((E, rows, cols), (e, ld, 1), off)


def to_gpu(t):
    """The same values, strides and offset."""
    flat = torch.empty(t.untyped_storage().nbytes() // t.element_size(), dtype=t.dtype)
    flat.copy_(t.as_strided((len(flat),), (1,), 0))
    return flat.cuda().as_strided(t.shape, t.stride(), t.storage_offset())


class Case:
    def __init__(self, T, E, k, D, F, type, act="silu", normalize=True, residual=False, pad=0, off=0, seed=0):
        g, dt = torch.Generator().manual_seed(seed), ff.TYPES[type]
        self.sizes, self.type, self.act, self.normalize, self.pad = (T, E, k, D, F), type, act, normalize, pad
        self.x, self.router = ff.rand(g, T, D, dt, 1.0, pad, off), ff.rand(g, E, D, dt, D ** -0.5, pad, off)
        self.wg, self.wu, self.wd = experts(g, E, F, D, dt, pad, off), experts(g, E, F, D, dt, pad, off), experts(g, E, D, F, dt, pad, off)
        self.residual = ff.rand(g, T, D, dt, 1.0, pad, off) if residual else None

    def desc(self, B):
        t = dict(f32=B.TYPE_F32, bf16=B.TYPE_BF16, f16=B.TYPE_F16)[self.type]
        return B.make_moe_desc(*self.sizes, t, ff.ACTS.index(self.act), self.normalize)

    def run(self, B, outs=True, in_place=False):
        T, E, k, D, F = self.sizes
        d = self.desc(B)
        residual = None if self.residual is None else ff.to_gpu(self.residual)
        y = residual if in_place else ff.empty_gpu(T, D, self.x.dtype, self.pad)
        chosen = torch.full((T, k), -7, dtype=torch.int32, device="cuda") if outs else None
        weights = torch.full((T, k), float("nan"), device="cuda") if outs else None
        ws = B.alloc_moe_workspace(d)
        ws.fill_(0xff)   # nothing that a workspace holds before the call may matter
        B.cct_moe_forward(d, ff.to_gpu(self.x), ff.to_gpu(self.router), to_gpu(self.wg), to_gpu(self.wu), to_gpu(self.wd), residual, y, chosen,
                          weights, ws)
        torch.cuda.synchronize()
        assert in_place or ff.untouched(y, D)
        return y, chosen, weights

    def want(self):
        return moe.forward(self.act, self.x, self.router, self.wg, self.wu, self.wd, self.sizes[2], self.normalize, self.residual)

    def check(self, B, rows=slice(None)):
        (y, chosen, weights), (value, which, exact) = self.run(B), self.want()
        assert torch.equal(chosen.cpu().long()[rows], which[rows])
        assert bool(((weights.cpu().double() - exact).abs() <= (moe.WEIGHT_ERR + ff.EPS32) * exact)[rows].all())
        ff.check("y", y[rows], (value[0][rows], value[1][rows]))
        return y


# tokens, experts, chosen, D, F, elements between rows, elements in front
SHAPES = [(1, 1, 1, 1, 1, 0, 0), (1, 4, 2, 7, 3, 0, 0), (1, 8, 2, 256, 512, 0, 0), (2, 3, 3, 33, 100, 1, 1), (3, 16, 4, 1000, 515, 0, 0),
          (5, 64, 8, 72, 40, 8, 0), (16, 8, 2, 128, 264, 0, 2), (17, 6, 2, 136, 96, 0, 0), (16, 20, 3, 2049, 31, 0, 0), (32, 4, 1, 64, 520, 3, 1),
          (33, 2, 2, 48, 72, 0, 0), (64, 7, 3, 96, 130, 64, 8), (64, 1, 1, 40, 24, 0, 0), (50, 512, 16, 24, 16, 0, 0), (64, 130, 5, 31, 33, 5, 0),
          (9, 256, 1, 64, 64, 0, 0),
          # a token's experts side by side; contractions of 2, 4 and 8 waves, of whole steps or not
          (1, 6, 5, 72, 1100, 0, 0), (1, 9, 3, 513, 2100, 1, 1), (35, 3, 2, 520, 250, 0, 0), (64, 2, 1, 300, 700, 3, 0), (20, 5, 2, 768, 32, 0, 0)]


@pytest.mark.parametrize("type", list(ff.TYPES))
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "%d-%d-%d-%dx%d+%d@%d" % s)
def test_forward(B, type, shape):
    i = SHAPES.index(shape)
    c = Case(*shape[:5], type, ff.ACTS[i % 5], i % 3 != 0, i % 2 == 0, *shape[5:], seed=i)
    y = c.check(B)
    assert torch.equal(y, c.run(B, outs=False)[0])
    if c.residual is not None:
        assert torch.equal(y, c.run(B, in_place=True)[0])


@pytest.mark.parametrize("T", [1, 20, 64])
def test_experts_that_are_not_chosen_are_not_read(B, T):
    c = Case(T, 40, 2, 100, 72, "bf16", seed=T)
    y = c.check(B)
    _, which, _ = c.want()
    other = torch.tensor([e for e in range(40) if e not in which])
    assert len(other) or T > 20
    for w in (c.wg, c.wu, c.wd):
        w[other] = float("nan")
    assert torch.equal(y, c.run(B)[0])


@pytest.mark.parametrize("normalize", [True, False])
def test_ties_go_to_the_lower_expert(B, normalize):
    """Whole numbers, so that logits are exact; many equal ones, zeros of both signs among them."""
    g = torch.Generator().manual_seed(3)
    c = Case(30, 100, 6, 64, 48, "f32", normalize=normalize)
    c.x.copy_(torch.randint(-1, 2, c.x.shape, generator=g))
    c.router.copy_(torch.randint(0, 2, c.router.shape, generator=g) * (torch.arange(64) < 3) * -1.0)
    c.x[4] = 0
    c.x[5] = -0.0
    c.check(B)


def test_values_that_are_not_finite(B):
    """A token with one is alone with it; an expert's infinite weights reach its tokens only; NaN logits come last."""
    c = Case(20, 8, 2, 96, 64, "f32", seed=4)
    clean, which, _ = c.run(B)
    c.x[3, 5], c.x[9, 0] = float("nan"), float("inf")
    y, _, weights = c.run(B)
    keep = [t for t in range(20) if t not in (3, 9)]
    assert torch.equal(y[keep], clean[keep]) and torch.isnan(y[3]).all() and not torch.isfinite(y[9]).any() and torch.isnan(weights[3]).all()
    c = Case(20, 8, 2, 96, 64, "f32", seed=4)
    e = int(which[0, 0])
    c.wd[e] = float("inf")
    c.wg[e, 3] = float("nan")
    y, _, _ = c.run(B)
    theirs = (which == e).any(1)
    assert theirs.any() and not theirs.all()
    assert torch.equal(y[~theirs], clean[~theirs]) and torch.isnan(y[theirs]).all()
    c = Case(6, 5, 3, 32, 16, "bf16", seed=5)
    c.router[1] = float("nan")
    c.check(B)                                            # three of the other four
    c = Case(6, 5, 5, 32, 16, "f32", seed=5)
    c.router[1] = float("nan")
    _, which, weights = c.run(B)
    assert (which[:, 4] == 1).all() and torch.isnan(weights).all()


def test_large_and_small_logits(B):
    c = Case(4, 9, 3, 32, 16, "f32", normalize=False, seed=6)
    c.router *= 30.0
    (y, chosen, weights), (value, which, exact) = c.run(B), c.want()
    assert torch.equal(chosen.cpu().long(), which) and float(exact.max()) > 0.99
    # an argument's rounding is 2^-24 of it, up to 200 here
    assert bool(((weights.cpu().double() - exact).abs() <= 3e-5 * exact + 1e-37).all())


@pytest.mark.parametrize("type", ["bf16", "f32"])
def test_experts_far_apart(B, type):
    """Experts and rows whose offsets pass 32 bits."""
    c = Case(3, 3, 3, 40, 24, type, seed=7)
    want = c.run(B)[0]
    d, ws = c.desc(B), B.alloc_moe_workspace(c.desc(B))

    def far(t, e, ld):
        out = torch.empty(2 * e + (t.shape[1] - 1) * ld + t.shape[2], dtype=t.dtype, device="cuda").as_strided(t.shape, (e, ld, 1))
        return out.copy_(t)
    wg, wu, wd = far(c.wg, (1 << 31) + 7, 40), far(c.wu, 24 << 27, 1 << 27), far(c.wd, (1 << 31) + 1, 25)
    y = torch.empty_like(want)
    B.cct_moe_forward(d, ff.to_gpu(c.x), ff.to_gpu(c.router), wg, wu, wd, None, y, None, None, ws)
    assert torch.equal(y, want)


@pytest.mark.parametrize("T,E,k,D,F", [(1, 16, 2, 512, 768), (1, 8, 3, 256, 2100), (40, 12, 3, 100, 50), (16, 64, 4, 256, 256)])
def test_replayed_from_a_graph_and_on_another_stream(B, T, E, k, D, F):
    c = Case(T, E, k, D, F, "bf16", residual=True, seed=8)
    d = c.desc(B)
    x, router, residual = ff.to_gpu(c.x), ff.to_gpu(c.router), ff.to_gpu(c.residual)
    w = [to_gpu(t) for t in (c.wg, c.wu, c.wd)]
    outs = [torch.empty(T, D, dtype=torch.bfloat16, device="cuda"), torch.empty(T, k, dtype=torch.int32, device="cuda"),
            torch.empty(T, k, device="cuda")]
    ws = B.alloc_moe_workspace(d)

    def step():
        B.cct_moe_forward(d, x, router, *w, residual, *outs, ws)
    step()
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step()
    for i in range(3):
        x.normal_()
        step()
        want = [t.clone() for t in outs]
        for again in (graph.replay, step):
            for t in outs:
                t.zero_()
            torch.cuda.synchronize()
            with torch.cuda.stream(side):
                again()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, outs)), i


def test_no_tokens(B):
    c = Case(1, 4, 2, 16, 8, "bf16")
    d = B.make_moe_desc(0, 4, 2, 16, 8, B.TYPE_BF16)
    e = torch.empty(0, 16, dtype=torch.bfloat16, device="cuda")
    B.cct_moe_forward(d, e, ff.to_gpu(c.router), to_gpu(c.wg), to_gpu(c.wu), to_gpu(c.wd), None, e, None, None, B.alloc_moe_workspace(d))
