"""What reaches the experts' second product: every bit of fp32's weight * h, whatever its size and the tensors' type.

Whole numbers, where the results are exact or wrong; small numbers of fp16 within a bound without any absolute part of their own; and
infinities, which are the formula's."""
import pytest
import torch

import feed_forward_util as ff
import moe_util as moe
from test_gpu_moe import Case, B  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


# tokens, experts, chosen, D, F: a single token's experts in one contraction and side by side; every count of blocks of columns, full
# and with one token more; several passes over the weights (few tokens on average, all on the same experts)
WHOLE = [(1, 3, 1, 512, 264), (1, 4, 4, 512, 264), (1, 4, 4, 520, 1400), (2, 4, 2, 512, 100), (5, 32, 1, 512, 72), (6, 4, 2, 500, 72),
         (10, 16, 1, 512, 130), (11, 9, 4, 512, 96), (16, 16, 2, 512, 264), (17, 1, 1, 512, 264), (33, 64, 2, 512, 1030), (40, 4, 4, 512, 64),
         (64, 256, 1, 512, 264), (64, 1, 1, 512, 264), (64, 2, 2, 264, 1400)]


@pytest.mark.parametrize("type", list(ff.TYPES))
@pytest.mark.parametrize("sizes", WHOLE, ids=lambda s: "%d-%d-%d-%dx%d" % s)
def test_whole_numbers(B, type, sizes):  # noqa: F811
    """Features come in pairs with the same g and u one apart, so that h differs by g: y is that difference, between numbers of up to
    20 bits.  Logits are all the same: the first experts, of weight 1 / chosen, a power of two."""
    T, E, k, D, F = sizes
    g = torch.Generator().manual_seed(F)
    c = Case(T, E, k, D, F, type, act="none")
    for t in (c.x, c.router, c.wg, c.wu, c.wd):
        t.zero_()
    c.x.copy_(torch.randint(0, 3, (T, D), generator=g))
    c.x[:, 0] = 1
    pairs = min(F // 2, D)
    even, odd = torch.arange(pairs) * 2, torch.arange(pairs) * 2 + 1
    gates = torch.randint(-3, 4, (E, pairs, D), generator=g) * (torch.rand(E, pairs, D, generator=g) < 8 / D)
    up = torch.randint(0, 127, (E, pairs, D), generator=g)
    c.wg[:, even], c.wg[:, odd] = gates.to(c.x.dtype), gates.to(c.x.dtype)
    c.wu[:, even], c.wu[:, odd] = (up + (torch.arange(D) == 0)).to(c.x.dtype), up.to(c.x.dtype)
    c.wd[:, torch.arange(pairs), even], c.wd[:, torch.arange(pairs), odd] = 1, -1
    x = c.x.double()
    want = torch.zeros(T, D, dtype=torch.float64)
    want[:, :pairs] = sum(x @ gates[e].double().t() for e in range(k)) / k
    most = max(float(((x @ gates[e].double().t()) * (x @ up[e].double().t())).abs().max()) for e in range(k))
    assert 2 ** 17 < most < 2 ** 23 and torch.equal(want.to(c.x.dtype).double(), want)   # every sum of fp32 is exact, and so is y
    y, chosen, weights = c.run(B)
    assert torch.equal(chosen.cpu(), torch.arange(k, dtype=torch.int32).expand(T, k)) and bool((weights == 1 / k).all())
    assert torch.equal(y.cpu().double(), want)


def forward64(c):
    """moe_util.forward, with the bound of weight * h as fp32 holds it: to 2^-24."""
    T, E, k, D, F = c.sizes
    _, chosen, weights = moe.route(c.x, c.router, k, c.normalize)
    y = torch.zeros(T, D, dtype=torch.float64)
    err, size = y.clone(), y.clone()
    for e in chosen.unique().tolist():
        t, j = (chosen == e).nonzero(as_tuple=True)
        (g, eg), (u, eu) = ff.product(c.x[t], c.wg[e]), ff.product(c.x[t], c.wu[e])
        a, w = ff.act64(c.act, g)[0], weights[t, j][:, None]
        ea = ff.SLOPE * eg + ff.ACT_ERR * a.abs()
        h = w * a * u
        eh = w * (ea * u.abs() + a.abs() * eu + ea * eu) + (moe.WEIGHT_ERR + 3 * ff.EPS32) * h.abs()
        v = c.wd[e].double()
        y[t] += h @ v.t()
        err[t] += eh @ v.abs().t()
        size[t] += (h.abs() + eh) @ v.abs().t()
    # three terms of a value at the most, two of a weight
    return ff.rounded(y, err + (6 * k * F + 16) * ff.EPS32 * size, c.x.dtype)


# tokens, experts, chosen, D, F, whether the chosen experts' weights add up to one
SMALL = [(1, 4, 2, 64, 40, True), (1, 6, 5, 64, 1100, True), (3, 200, 8, 64, 24, False), (20, 8, 2, 64, 40, True), (64, 4, 2, 48, 33, False)]


@pytest.mark.parametrize("type", list(ff.TYPES))
@pytest.mark.parametrize("sizes", SMALL, ids=lambda s: "%d-%d-%d-%dx%d-%s" % s)
def test_small_values(B, type, sizes):  # noqa: F811
    """h of 1e-6 and less, below fp16's normal numbers, and weights wd that bring it back."""
    c = Case(*sizes[:5], type, "silu", sizes[5], seed=11)
    c.wg *= 2.0 ** -9
    c.wu *= 2.0 ** -10
    c.wd *= 2.0 ** 13
    want = forward64(c)
    y, chosen, _ = c.run(B)
    assert float(want[0].abs().max()) > 2.0 ** -10
    ff.check("y", y, want)


@pytest.mark.parametrize("type", list(ff.TYPES))
@pytest.mark.parametrize("T", [1, 9, 40])
def test_infinite_weights(B, T, type):  # noqa: F811
    """An infinity or a NaN in wd makes the results of its row what the formula says, and no others."""
    c = Case(T, 6, 2, 72, 300, type, "silu", seed=T)
    c.wd[:, 3, 5] = float("inf")
    c.wd[2, 7, 299] = -float("inf")
    c.wd[1, 20, 0] = float("nan")
    c.wd[:, 70, 9], c.wd[:, 70, 250] = float("inf"), -float("inf")
    y = c.run(B)[0].cpu()
    _, chosen, weights = moe.route(c.x, c.router, 2, True)
    exact = torch.zeros(T, 72, dtype=torch.float64)
    for t in range(T):
        for j in range(2):
            e = int(chosen[t, j])
            g, u = c.wg[e].double() @ c.x[t].double(), c.wu[e].double() @ c.x[t].double()
            exact[t] += (c.wd[e].double() * (weights[t, j] * ff.act64("silu", g)[0] * u)).sum(1)
    assert torch.equal(torch.isnan(y), torch.isnan(exact)) and torch.equal(torch.isinf(y), torch.isinf(exact))
    at = torch.isinf(exact)
    assert bool(at[:, 3].any()) and torch.equal(y[at].double(), exact[at])
    c.wd[~torch.isfinite(c.wd)] = 0
    value, bound = forward64(c)
    rows = [d for d in range(72) if d not in (3, 7, 20, 70)]
    ff.check("y", y[:, rows], (value[:, rows], bound[:, rows]))


@pytest.mark.parametrize("type", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 7])
def test_h_beyond_the_range(B, T, type):  # noqa: F811
    """g u passes fp32's range: an infinity, with the sign of wd."""
    c = Case(T, 3, 2, 40, 33, type, "none", seed=2)
    c.x.copy_(c.x.float().abs() + 0.5)
    c.router *= 2.0 ** -10
    c.wg.copy_(c.wg.float().abs() * 2.0 ** 70 + 2.0 ** 70)
    c.wu.copy_(c.wg)
    c.wd.copy_(torch.where(torch.arange(40)[:, None] % 2 == 0, 1.0, -1.0) * (c.wd.float().abs() + 2.0 ** -5))
    y = c.run(B)[0].cpu()
    assert torch.equal(y.float(), torch.where(torch.arange(40) % 2 == 0, 1.0, -1.0).expand(T, 40) * float("inf"))
