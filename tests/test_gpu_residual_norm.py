"""Norms and gates on a residual stream (cct_residual_norm_*) against 64 bits on the CPU, within bounds that follow the fp32
computation (residual_norm_util.py): types, norms, gates of one row to all, odd sizes, strides and addresses, long rows, missing
operands, in place, values that are not finite, empty batches, captured graphs, another stream, and differences."""
import pytest
import torch

import feed_forward_util as ff
import residual_norm_util as rn

pytestmark = pytest.mark.gpu

NORMS = ["none", "rms", "layer"]
GRADS = ("dr", "db", "dgate", "dw_after", "dc_after", "dw_before", "dc_before")


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available()
    from paper_1504_04343_amd import binding
    return binding


def desc_of(B, M, D, type, before, after, rows, eps, scale):
    t = dict(f32=B.TYPE_F32, bf16=B.TYPE_BF16, f16=B.TYPE_F16)[type]
    return B.make_residual_norm_desc(M, D, t, NORMS.index(before), NORMS.index(after), rows, eps, scale)


def vec(t):
    return None if t is None else t.cuda()


def mat(t):
    return None if t is None else ff.to_gpu(t)


class Case:
    """Operands on the CPU, and the calls."""

    def __init__(self, B, M, D, type, before="rms", after="rms", rows=1, gate=True, affine=True, pad=0, off=0, eps=1e-5, scale=0.7,
                 seed=0, block=True):
        g, dt = torch.Generator().manual_seed(seed), ff.TYPES[type]
        self.B, self.M, self.D, self.dt, self.pad, self.rows = B, M, D, dt, pad, rows
        self.how = (before, after, rows, eps, scale)
        self.desc = desc_of(B, M, D, type, *self.how)
        self.groups = -(-M // rows)

        def vector(std, mean, there):
            return (torch.randn(D, generator=g) * std + mean).to(dt) if there else None
        self.r, self.b = ff.rand(g, M, D, dt, 2.0, pad, off), ff.rand(g, M, D, dt, 1.0, pad, off) if block else None
        self.gate = ff.rand(g, self.groups, D, dt, 1.0, pad, off) if gate and block else None
        self.w_after, self.c_after = vector(0.3, 1.0, block and after != "none"), vector(0.5, 0.0, block and affine and after != "none")
        self.w_before, self.c_before = vector(0.3, 1.0, before != "none"), vector(0.5, 0.0, affine and before != "none")
        self.s = ff.rand(g, M, D, dt, 2.0, pad, off)
        self.ds = ff.rand(g, M, D, dt, 1.0, pad, off)
        self.dh = ff.rand(g, M, D, dt, 1.0, pad, off) if before != "none" else None

    def forward(self, want=("s", "h"), in_place=False):
        r = mat(self.r)
        s = r if in_place else ff.empty_gpu(self.M, self.D, self.dt, self.pad) if "s" in want else None
        h = ff.empty_gpu(self.M, self.D, self.dt, self.pad) if "h" in want and self.how[0] != "none" else None
        self.B.cct_residual_norm_forward(self.desc, r, mat(self.b), mat(self.gate), vec(self.w_after), vec(self.c_after),
                                         vec(self.w_before), vec(self.c_before), s, h)
        torch.cuda.synchronize()
        out = {k: t for k, t in (("s", s), ("h", h)) if t is not None}
        assert in_place or all(ff.untouched(t, self.D) for t in out.values())
        return out

    def forward64(self):
        return rn.forward(*self.how, self.r, self.b, self.gate, self.w_after, self.c_after, self.w_before, self.c_before)

    def backward(self, want=GRADS, in_place=False):
        ds = mat(self.ds)
        out = {}
        for k in want:
            there = {"db": self.b is not None, "dgate": self.gate is not None, "dw_after": self.w_after is not None,
                     "dc_after": self.w_after is not None, "dw_before": self.dh is not None, "dc_before": self.dh is not None}
            if not there.get(k, True):
                continue
            if k == "dr" and in_place:
                out[k] = ds
            elif k in ("dr", "db", "dgate"):
                out[k] = ff.empty_gpu(self.groups if k == "dgate" else self.M, self.D, self.dt, self.pad)
            else:
                out[k] = torch.full((self.D,), float("nan"), dtype=self.dt, device="cuda")
        ws = self.B.alloc_residual_norm_workspace(self.desc)
        ws.fill_(0xff)   # nothing that a workspace holds before the call may matter
        self.B.cct_residual_norm_backward(self.desc, mat(self.s), mat(self.b), mat(self.gate), vec(self.w_after), vec(self.c_after),
                                          vec(self.w_before), ds, mat(self.dh), *(out.get(k) for k in GRADS), ws)
        torch.cuda.synchronize()
        assert all(t.dim() == 1 or (k == "dr" and in_place) or ff.untouched(t, self.D) for k, t in out.items())
        return out

    def backward64(self):
        return rn.backward(*self.how, self.s, self.b, self.gate, self.w_after, self.c_after, self.w_before, self.ds, self.dh)


# M, D, before, after, gate rows (0: no gate), biases, elements between rows, elements in front
SHAPES = [(1, 1, "rms", "rms", 1, True, 0, 0), (1, 7, "layer", "rms", 1, True, 0, 0), (1, 64, "rms", "none", 0, False, 0, 0),
          (2, 513, "rms", "layer", 2, True, 0, 1), (3, 1000, "layer", "layer", 1, True, 1, 1), (5, 512, "none", "rms", 2, False, 0, 0),
          (16, 8192, "rms", "rms", 16, False, 0, 0), (17, 2049, "layer", "rms", 4, True, 3, 0), (33, 130, "rms", "layer", 33, True, 5, 2),
          (64, 4096, "layer", "none", 64, False, 8, 8), (129, 1025, "rms", "rms", 1, True, 0, 0), (300, 72, "layer", "layer", 7, True, 0, 0),
          (700, 24, "rms", "rms", 300, False, 0, 0), (1531, 264, "rms", "rms", 1000, True, 0, 0), (2100, 40, "layer", "layer", 5, True, 0, 0),
          (2100, 520, "rms", "none", 2100, False, 0, 0), (40, 8200, "rms", "layer", 13, True, 0, 0), (9, 16387, "layer", "rms", 1, True, 1, 1),
          (2, 33000, "rms", "none", 2, False, 0, 0), (6, 3000, "none", "none", 3, False, 0, 0), (4, 1536, "none", "layer", 0, True, 2, 0),
          (37, 5000, "layer", "rms", 5, True, 3, 1), (300, 4104, "rms", "layer", 300, True, 0, 0), (70, 8191, "rms", "rms", 9, False, 0, 0),
          (4, 500, "rms", "rms", 4, True, 0, 0), (3, 4200, "layer", "layer", 5, True, 0, 0), (2049, 512, "rms", "layer", 700, True, 0, 0),
          # two rows at a time: runs that end in the first, in the second and within a gate row
          (2, 2300, "layer", "rms", 1, True, 0, 0), (301, 2500, "layer", "layer", 3, True, 5, 1), (1100, 2560, "rms", "rms", 1100, False, 0, 0),
          (1027, 2816, "rms", "layer", 2, True, 8, 0), (205, 2049, "layer", "layer", 37, True, 3, 3), (13, 2568, "none", "rms", 6, True, 0, 0)]
IDS = ["%dx%d-%s-%s-%d+%d@%d" % (s[:5] + s[6:]) for s in SHAPES]


@pytest.mark.parametrize("type", list(ff.TYPES))
@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
def test_forward(B, type, shape):
    M, D, before, after, rows, affine, pad, off = shape
    c = Case(B, M, D, type, before, after, max(rows, 1), rows > 0, affine, pad, off, seed=SHAPES.index(shape))
    got, want = c.forward(), c.forward64()
    assert set(got) == set(want)
    for k in got:
        ff.check(k, got[k], want[k])
        assert torch.equal(got[k], c.forward((k,))[k]), k
    again = c.forward(in_place=True)
    assert all(torch.equal(got[k], again[k]) for k in got)


@pytest.mark.parametrize("type", list(ff.TYPES))
@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
def test_backward(B, type, shape):
    M, D, before, after, rows, affine, pad, off = shape
    c = Case(B, M, D, type, before, after, max(rows, 1), rows > 0, affine, pad, off, seed=100 + SHAPES.index(shape))
    got, want = c.backward(), c.backward64()
    assert set(got) == set(want)
    for k in got:
        ff.check(k, got[k], want[k])
    for k in got:                      # one at a time
        assert torch.equal(got[k], c.backward((k,))[k]), k
    again = c.backward(in_place=True)
    assert all(torch.equal(got[k], again[k]) for k in got)


@pytest.mark.parametrize("D", [24, 1000, 9000])
def test_parts_that_are_not_there(B, D):
    """No block yet; no vectors; only one of the two gradients."""
    c = Case(B, 5, D, "f32", block=False)
    got, want = c.forward(), c.forward64()
    assert torch.equal(got["s"].cpu(), c.r)
    ff.check("h", got["h"], want["h"])
    for k, t in c.backward().items():
        ff.check(k, t, c.backward64()[k])
    c = Case(B, 5, D, "f32", "layer", "rms")
    c.w_after = c.c_after = c.w_before = c.c_before = None
    for k, t in c.forward().items():
        ff.check(k, t, c.forward64()[k])
    for k, t in c.backward(("dr", "db", "dgate")).items():
        ff.check(k, t, c.backward64()[k])
    for missing in ("ds", "dh"):
        c = Case(B, 5, D, "bf16", "rms", "layer", rows=2)
        setattr(c, missing, None)
        want = c.backward64()
        if missing == "ds":
            got = c.backward()
        else:   # sums over what does not come are zero
            want.update(dw_before=None, dc_before=None)
            c.dh = None
            got = {}
            for k in GRADS:
                got[k] = torch.full((D,) if k[1] in "wc" else (c.groups if k == "dgate" else 5, D), float("nan"), dtype=c.dt, device="cuda")
            B.cct_residual_norm_backward(c.desc, None, mat(c.b), mat(c.gate), vec(c.w_after), vec(c.c_after), vec(c.w_before), mat(c.ds),
                                         None, *got.values(), B.alloc_residual_norm_workspace(c.desc))
            assert not got["dw_before"].any() and not got["dc_before"].any()
        for k in got:
            if want[k] is not None:
                ff.check(k, got[k], want[k])


@pytest.mark.parametrize("type", list(ff.TYPES))
@pytest.mark.parametrize("D", [24, 512, 520, 768, 1000, 2049, 2560, 4100, 8185, 9000])
def test_layer_norms_without_weights_or_gate(B, D, type):
    """Nothing but the norms themselves, whose level (the mean of dh, far from zero here) must not reach columns that a row has not."""
    for none in (("w_after", "c_after", "w_before", "c_before"), ("w_after", "c_after"), ("w_before", "c_before")):
        c = Case(B, 9, D, type, "layer", "layer", gate=False, seed=D)
        for n in none:
            setattr(c, n, None)
        c.dh = (c.dh.float() + 1.5).to(c.dt)
        got, want = c.forward(), c.forward64()
        back, want_back = c.backward(), c.backward64()
        for k in got:
            ff.check(k, got[k], want[k])
        for k in back:
            ff.check(k, back[k], want_back[k])
        assert torch.equal(back["db"], c.backward(("db",))["db"])


def test_b_is_not_needed_without_its_norm(B):
    c = Case(B, 6, 100, "f32", "rms", "none", rows=2)
    want = c.backward64()
    db = ff.empty_gpu(6, 100, c.dt)
    B.cct_residual_norm_backward(c.desc, mat(c.s), None, mat(c.gate), None, None, vec(c.w_before), mat(c.ds), mat(c.dh), None, db, None,
                                 None, None, None, None, B.alloc_residual_norm_workspace(c.desc))
    ff.check("db", db, want["db"])


@pytest.mark.parametrize("D", [40, 9000])
def test_no_rows(B, D):
    d = B.make_residual_norm_desc(0, D, B.TYPE_BF16, B.NORM_RMS, B.NORM_RMS, 4)
    e = torch.empty(0, D, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(D, dtype=torch.bfloat16, device="cuda")
    B.cct_residual_norm_forward(d, e, e, e, w, None, w, None, e, e)
    grads = [torch.full((D,), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    B.cct_residual_norm_backward(d, e, e, e, w, None, w, e, e, e, e, e, *grads, B.alloc_residual_norm_workspace(d))
    assert not any(t.any() for t in grads)


@pytest.mark.parametrize("D", [100, 2100, 9000])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_values_that_are_not_finite(B, D, kind):
    """A row that holds one, and no other, is not finite."""
    c = Case(B, 9, D, "f32", kind, kind, rows=3)
    clean, back = c.forward(), c.backward()
    for t, where in ((c.r, 1), (c.b, 4), (c.s, 1), (c.dh, 4)):
        t[where, D // 2] = float("nan") if where == 1 else float("inf")
    for a, b in ((clean, c.forward()), (back, {k: v for k, v in c.backward(("dr", "db")).items()})):
        for k, t in b.items():
            rows = torch.tensor([i for i in range(9) if i not in (1, 4)])
            assert torch.equal(a[k][rows], t[rows]), k
            assert torch.isnan(t[1]).any() and not torch.isfinite(t[4]).all(), k


def test_rows_of_zeros(B):
    c = Case(B, 3, 64, "f32", "rms", "layer", affine=False)
    c.r[1] = 0
    c.b[1] = 0
    got, want = c.forward(), c.forward64()
    ff.check("s", got["s"], want["s"])
    assert not got["s"][1].any() and not got["h"][1].any()
    c.how = ("rms", "layer", 1, 0.0, 0.7)
    c.desc = desc_of(B, 3, 64, "f32", *c.how)
    got = c.forward()
    assert torch.isnan(got["s"][1]).all() and torch.isfinite(got["s"][0]).all()          # 0 / 0, as the formula says


def test_rows_far_apart(B):
    """Rows whose offsets pass 32 bits."""
    M, D, ld = 5, 70, (1 << 30) + 8
    c = Case(B, M, D, "bf16", "rms", "none", gate=False, affine=False)
    base = torch.empty((M - 1) * ld + D, dtype=torch.bfloat16, device="cuda")
    far = base.as_strided((M, D), (ld, 1))
    far.copy_(c.r)
    got = c.forward()
    s, h = torch.empty_like(far[:, :], memory_format=torch.contiguous_format), ff.empty_gpu(M, D, c.dt)
    B.cct_residual_norm_forward(c.desc, far, mat(c.b), None, None, None, vec(c.w_before), None, s, h)
    assert torch.equal(s, got["s"]) and torch.equal(h, got["h"])
    far.copy_(c.s)
    got = c.backward()
    dr = torch.empty_like(s)
    B.cct_residual_norm_backward(c.desc, far, mat(c.b), None, None, None, vec(c.w_before), mat(c.ds), mat(c.dh), dr, None, None, None,
                                 None, None, None, B.alloc_residual_norm_workspace(c.desc))
    assert torch.equal(dr, got["dr"])


def test_rows_of_134_million_columns(B):
    """More columns than a launch's second and third dimension take workgroups of them: against 64 bits on the GPU."""
    D = 65535 * 2048 + 1000
    g = torch.Generator(device="cuda").manual_seed(1)
    r, w, ds, dh = (torch.randn(1, D, generator=g, device="cuda").to(torch.bfloat16) for _ in range(4))
    d = B.make_residual_norm_desc(1, D, B.TYPE_BF16, B.NORM_RMS)
    h, dr, dw = (torch.full_like(r, float("nan")) for _ in range(3))
    B.cct_residual_norm_forward(d, r, None, None, None, None, w[0], None, None, h)
    B.cct_residual_norm_backward(d, r, None, None, None, None, w[0], ds, dh, dr, None, None, None, None, dw[0], None,
                                 B.alloc_residual_norm_workspace(d))
    v, e, u = r.double(), dh.double(), w.double()
    rstd = 1 / ((v * v).mean() + 1e-6).sqrt()
    n = v * rstd
    # A thread adds 16384 times, its workgroup 10 more: a sum is off by 16400 x 2^-24 < 2^-9.99 of its terms' sizes, rstd by half of
    # that, n slope by 2.5 times that: all below 2^-8.6.  The result's rounding is half a step of bf16.
    slope, most = (e * u * n).mean(), (e * u * n).abs().mean()
    for got, want, size in ((h, n * u, (n * u).abs()), (dw, e * n, (e * n).abs()),
                            (dr, ds.double() + (e * u - n * slope) * rstd, ((e * u).abs() + n.abs() * most) * rstd)):
        assert bool(((got.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -8.6 * (1 + 2.0 ** -8) * size + 1e-30).all())


@pytest.mark.parametrize("M,D,rows", [(50, 600, 7), (1, 4096, 1), (30, 6000, 4), (600, 96, 600), (20, 9000, 20)])
def test_replayed_from_a_graph_and_on_another_stream(B, M, D, rows):
    c = Case(B, M, D, "bf16", "rms", "rms", rows)
    args = [mat(c.b), mat(c.gate), vec(c.w_after), vec(c.c_after), vec(c.w_before)]
    r, ds, dh, c_before = mat(c.r), mat(c.ds), mat(c.dh), vec(c.c_before)
    s, h = torch.empty_like(r), torch.empty_like(r)
    grads = [torch.empty_like(t) for t in (r, r, args[1], args[2], args[2], args[2], args[2])]
    ws = B.alloc_residual_norm_workspace(c.desc)

    def step():
        B.cct_residual_norm_forward(c.desc, r, *args, c_before, s, h)
        B.cct_residual_norm_backward(c.desc, s, *args, ds, dh, *grads, ws)
    step()
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step()
    for i in range(3):
        r.normal_()
        dh.normal_()
        step()
        want = [t.clone() for t in [s, h] + grads]
        for t in [s, h] + grads:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, [s, h] + grads)), i
        for t in [s, h] + grads:
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            step()
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, [s, h] + grads)), i


@pytest.mark.parametrize("D", [33, 700])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_gradients_against_differences(B, D, kind):
    """<gradient, v> against (L(+t v) - L(-t v)) / 2t of L = <ds, s> + <dh, h>: apart by the differences' own error, which 64 bits
    tell, and by the roundings that the bounds tell."""
    M, rows, t = 6, 4, 2.0 ** -6
    c = Case(B, M, D, "f32", kind, kind, rows, seed=3)
    ds, dh = c.ds.double(), c.dh.double()
    names = ("r", "b", "gate", "w_after", "c_after", "w_before", "c_before")
    keep = {n: getattr(c, n) for n in names}
    c.s = c.forward()["s"].cpu()
    grads, grads64 = c.backward(), c.backward64()

    def loss(out):
        return float((ds * out["s"].double().cpu()).sum() + (dh * out["h"].double().cpu()).sum())
    for n in names:
        v = torch.randn(keep[n].shape, generator=torch.Generator().manual_seed(9))
        got, exact, noise = 0.0, 0.0, 0.0
        for sign in (1, -1):
            setattr(c, n, keep[n] + sign * t * v)
            want = c.forward64()
            got += sign * loss(c.forward()) / (2 * t)
            exact += sign * loss({k: w[0] for k, w in want.items()}) / (2 * t)
            noise += float((ds.abs() * want["s"][1]).sum() + (dh.abs() * want["h"][1]).sum()) / (2 * t)
        # the points themselves are rounded to fp32
        noise += float((grads64["d" + n][0].abs() * (keep[n].double().abs() + t * v.double().abs())).sum()) * 2 * ff.EPS32 / t
        setattr(c, n, keep[n])
        value, bound = grads64["d" + n]
        slope = float((grads["d" + n].double().cpu() * v.double()).sum())
        short = abs(exact - float((value * v.double()).sum()))
        assert abs(got - slope) <= 1.01 * (noise + short + float((bound * v.double().abs()).sum())), n
        assert short <= 0.05 * abs(exact) + 0.5, n      # else the comparison says nothing
