"""SiLU and tanh-GELU, and their derivatives, where the logistic function in them is no normal number any more and its product
with the argument still is, relative to the value: 1e-5 for the fp32 function (an exponential's argument of up to 105 carries
three roundings: 105 * 3 * 2^-24 < 2e-5; twice that is allowed to the derivatives, whose parts have two such factors), half a step
of the type, and half the distance of its smallest numbers."""
import pytest
import torch

import feed_forward_util as ff
from test_gpu_feed_forward import B, gated_forward, linear_backward, linear_forward  # noqa: F401  (B: the fixture)

pytestmark = pytest.mark.gpu
ERR = 2e-5


def tail(act, dt):
    """Arguments from -60 down to where the results of fp32 end: of tanh-GELU's z those that take its logistic function there."""
    z = torch.linspace(-8.5, -11.0, 501) if act == "gelu_tanh" else torch.linspace(-60.0, -105.0, 901)
    return z.to(dt).view(-1, 1)


def bound(v, dt, err):
    return v, (err + ff.half(dt)) * v.abs() + ff.tiny(dt) + ff.tiny(torch.float32)


@pytest.mark.parametrize("type", list(ff.TYPES))
@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
def test_the_lower_tail(B, type, act):  # noqa: F811
    dt = ff.TYPES[type]
    z = tail(act, dt)
    w = torch.ones(1, 1, dtype=dt)
    z64 = z.double()
    if act == "silu":
        a, d = z64 * torch.sigmoid(z64), torch.sigmoid(z64) * (1 + z64 * torch.sigmoid(-z64))
    else:
        c = 2 * 0.7978845608028654
        s = torch.sigmoid(c * (z64 + 0.044715 * z64 ** 3))
        a, d = z64 * s, s + z64 * s * (1 - s) * c * (1 + 3 * 0.044715 * z64 ** 2)
    # tanh-GELU's argument is a sum of two rounded terms, up to 3 * 2^-24 of -105 each
    err = ERR * (2 if act == "gelu_tanh" else 1)
    y, _ = linear_forward(B, type, act, z, w, None, None, True)
    ff.check("y", y, bound(a, dt, err))
    few, _ = linear_forward(B, type, act, z[:16], w, None, None, True)
    assert torch.equal(few, y[:16])
    if type == "f16":        # whose smallest number is 2^-24
        return
    big = 2.0 ** 100
    dx, _, _ = linear_backward(B, type, act, z, w, z, torch.full(z.shape, big, dtype=dt))
    # dz is rounded to the type, and its product with 1 is
    ff.check("dx", dx, bound(d * big, dt, 2 * err + 2 * ff.half(dt)))
    h, _, u = gated_forward(B, type, act, z, w, torch.full((1, 1), big, dtype=dt), True)
    ff.check("h", h, bound(a * z64 * big, dt, err))
