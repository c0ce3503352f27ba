"""The operators of a residual block as a program runs them one after the other: a training step (norms and a gate around a gated
feed-forward block, its gradients) against automatic differentiation in 64 bits, and a serving step (norm, experts, gate and
norm, a 4-bit product) against the same steps in 64 bits, eager and replayed from a graph."""
import pytest
import torch
import torch.nn.functional as F

import moe_util as moe
import mx_util as mx
from gpu_util import TOL_F32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available()
    from paper_1504_04343_amd import binding
    return binding


def norm64(v, w, eps):
    return v / ((v ** 2).mean(1, keepdim=True) + eps).sqrt() * w


class Training:
    """x -> h = N0(x); b = (silu(h wg^T) * (h wu^T)) wd^T; s = x + scale * gate * N1(b), y = N2(s), M rows of D, F wide, fp32."""
    EPS, SCALE = 1e-5, 0.5

    def __init__(self, B, M, D, width, rows):
        g = torch.Generator().manual_seed(M)
        self.B, self.M, self.D, self.F, self.rows = B, M, D, width, rows

        def make(*shape, std=1.0, mean=0.0):
            return (torch.randn(*shape, generator=g) * std + mean).cuda()
        self.x = make(M, D)
        self.leaves = dict(w0=make(D, std=0.2, mean=1), wg=make(width, D, std=D ** -0.5), wu=make(width, D, std=D ** -0.5),
                           wd=make(D, width, std=width ** -0.5), w1=make(D, std=0.2, mean=1), gate=make(-(-M // rows), D, std=0.5, mean=1),
                           w2=make(D, std=0.2, mean=1))
        self.ds, self.dy = make(M, D), make(M, D)
        self.grads = {k: torch.empty_like(t) for k, t in self.leaves.items()}
        self.dx = torch.empty_like(self.x)
        new = torch.empty_like
        wide = torch.empty(M, width, device="cuda")
        self.t = dict(h=new(self.x), g=new(wide), u=new(wide), a=new(wide), b=new(self.x), s=new(self.x), y=new(self.x), db=new(self.x),
                      da=new(wide), dh=new(self.x), dr=new(self.x))
        self.first = B.make_residual_norm_desc(M, D, B.TYPE_F32, B.NORM_RMS, B.NORM_NONE, 1, self.EPS)
        self.last = B.make_residual_norm_desc(M, D, B.TYPE_F32, B.NORM_RMS, B.NORM_RMS, rows, self.EPS, self.SCALE)
        self.gated, self.down = B.make_gated_desc(M, width, D, B.TYPE_F32, B.ACT_SILU), B.make_linear_desc(M, D, width, B.TYPE_F32)
        self.ws = [B.alloc_residual_norm_workspace(self.first), B.alloc_residual_norm_workspace(self.last),
                   *(B.alloc_gated_workspace(self.gated, p) for p in (B.PASS_FORWARD, B.PASS_BACKWARD)),
                   *(B.alloc_linear_workspace(self.down, p) for p in (B.PASS_FORWARD, B.PASS_BACKWARD))]

    def step(self):
        B, t, w, d = self.B, self.t, self.leaves, self.grads
        B.cct_residual_norm_forward(self.first, self.x, None, None, None, None, w["w0"], None, None, t["h"])
        B.cct_gated_forward(self.gated, t["h"], w["wg"], w["wu"], t["a"], t["g"], t["u"], self.ws[2])
        B.cct_linear_forward(self.down, t["a"], w["wd"], None, None, t["b"], None, self.ws[4])
        B.cct_residual_norm_forward(self.last, self.x, t["b"], w["gate"], w["w1"], None, w["w2"], None, t["s"], t["y"])
        B.cct_residual_norm_backward(self.last, t["s"], t["b"], w["gate"], w["w1"], None, w["w2"], self.ds, self.dy, t["dr"], t["db"],
                                     d["gate"], d["w1"], None, d["w2"], None, self.ws[1])
        B.cct_linear_backward(self.down, t["a"], w["wd"], None, t["db"], t["da"], d["wd"], None, self.ws[5])
        B.cct_gated_backward(self.gated, t["h"], w["wg"], w["wu"], t["g"], t["u"], t["da"], t["dh"], d["wg"], d["wu"], self.ws[3])
        # the stream reaches the block and what follows: both gradients meet here
        B.cct_residual_norm_backward(self.first, self.x, None, None, None, None, w["w0"], t["dr"], t["dh"], self.dx, None, None, None,
                                     None, d["w0"], None, self.ws[0])

    def definition(self):
        w = {k: t.cpu().double().requires_grad_() for k, t in self.leaves.items()}
        x = self.x.cpu().double().requires_grad_()
        h = norm64(x, w["w0"], self.EPS)
        b = F.linear(F.silu(F.linear(h, w["wg"])) * F.linear(h, w["wu"]), w["wd"])
        s = x + self.SCALE * w["gate"][torch.arange(self.M) // self.rows] * norm64(b, w["w1"], self.EPS)
        y = norm64(s, w["w2"], self.EPS)
        grads = torch.autograd.grad([s, y], [x, *w.values()], [self.ds.cpu().double(), self.dy.cpu().double()])
        return s, y, grads[0], dict(zip(w, grads[1:]))


def close(name, got, want):
    want = want.detach()
    off = float((got.cpu().double() - want).abs().max() / want.abs().max())
    assert off <= TOL_F32, (name, off)


@pytest.mark.parametrize("M,D,width,rows", [(5, 72, 100, 2), (130, 264, 520, 130), (64, 600, 96, 1)])
def test_a_training_step(B, M, D, width, rows):
    """Within the library's fp32 tolerance of 1e-4 of the largest value."""
    t = Training(B, M, D, width, rows)
    t.step()
    s, y, dx, grads = t.definition()
    close("s", t.t["s"], s)
    close("y", t.t["y"], y)
    close("dx", t.dx, dx)
    for k, v in grads.items():
        close(k, t.grads[k], v)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            t.step()
    for _ in range(3):
        t.x.normal_()
        t.step()
        want = [v.clone() for v in (t.dx, t.t["y"], *t.grads.values())]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (t.dx, t.t["y"], *t.grads.values())))


@pytest.mark.parametrize("T", [1, 7, 40])
def test_a_serving_step(B, T):
    """h = N0(x); b = experts(h); s = x + gate * N1(b), q = N2(s); z = q w^T, q and w in 4 bits.  Each operator against 64 bits from
    what it was given, so that a step's rounding is not the next one's error."""
    g, dt = torch.Generator().manual_seed(T), torch.bfloat16
    D, width, E, k, N = 160, 96, 6, 2, 200

    def make(*shape, std=1.0, mean=0.0):
        return (torch.randn(*shape, generator=g) * std + mean).to(dt).cuda()
    x, w0, w1, w2, gate = make(T, D), make(D, std=0.2, mean=1), make(D, std=0.2, mean=1), make(D, std=0.2, mean=1), make(1, D, mean=1)
    router, wg, wu, wd = make(E, D, std=D ** -0.5), make(E, width, D, std=0.1), make(E, width, D, std=0.1), make(E, D, width, std=0.1)
    w = B.MxMatrix(N, D)
    B.cct_mx_quantize(make(N, D), w)
    h, b, s, q, z = (torch.empty(T, n, dtype=dt, device="cuda") for n in (D, D, D, D, N))
    first = B.make_residual_norm_desc(T, D, B.TYPE_BF16, B.NORM_RMS)
    last = B.make_residual_norm_desc(T, D, B.TYPE_BF16, B.NORM_RMS, B.NORM_RMS, T)
    layer, product = B.make_moe_desc(T, E, k, D, width, B.TYPE_BF16), B.make_linear_desc(T, N, D, B.TYPE_BF16)
    ws, ws2 = B.alloc_moe_workspace(layer), B.alloc_mx_linear_workspace(product)

    def step():
        B.cct_residual_norm_forward(first, x, None, None, None, None, w0, None, None, h)
        B.cct_moe_forward(layer, h, router, wg, wu, wd, None, b, None, None, ws)
        B.cct_residual_norm_forward(last, x, b, gate, w1, None, w2, None, s, q)
        B.cct_mx_linear_forward(product, q, w, None, None, z, None, ws2)
    step()
    import feed_forward_util as ff
    import residual_norm_util as rn
    c = {n: t.cpu() for n, t in dict(x=x, w0=w0, w1=w1, w2=w2, gate=gate, h=h, b=b, s=s, q=q, router=router, wg=wg, wu=wu, wd=wd).items()}
    ff.check("h", h, rn.forward("rms", "none", 1, 1e-6, 1.0, c["x"], None, None, None, None, c["w0"], None)["h"])
    ff.check("b", b, moe.forward("silu", c["h"], c["router"], c["wg"], c["wu"], c["wd"], k, True, None)[0])
    both = rn.forward("rms", "rms", T, 1e-6, 1.0, c["x"], c["b"], c["gate"], c["w1"], None, c["w2"], None)
    ff.check("s", s, both["s"])
    ff.check("q", q, both["h"])
    wide = mx.unpack(w.codes.cpu())
    values = mx.values(wide, w.scales.cpu()[:, :mx.blocks_of(D)], D)
    ff.check("z", z, ff.rounded(*ff.product(mx.values(*mx.quantize(c["q"]), D), values), dt))
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step()
    for _ in range(3):
        x.normal_()
        step()
        want = [t.clone() for t in (b, s, q, z)]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b_) for a, b_ in zip(want, (b, s, q, z)))
