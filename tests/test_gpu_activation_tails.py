"""The exact GELU and its slope element by element, far into the tail, in fp32.

Tolerance, derived before the first run (u = 2^-24).  Phi(x) for x < 0 is half a
complementary error function, t P(t) exp(-x^2 / 2): the exponent's argument x^2 / 2
is rounded three times, which moves the exponential by 3 u x^2 / 2 of itself; ex2,
the reciprocal (twice that in t P) and the last steps of the polynomial add 1 to 2 u each,
12 u in all, and the polynomial's own fit 4 u.  Near 0, 1/2 + x S(x^2) is off by less.
Bound of Phi: (16 + 1.5 x^2) u relative; of x Phi one rounding more.  The slope
Phi + x phi is held against |Phi| + |x phi|.  Values are kept ones, so the argument is
exact.  Exponentials below 2^-126 may be flushed before they are multiplied by x."""
import math

import pytest
import torch

from tests import worker_step_reference as R

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def B():
    from paper_2512_09685_b200 import binding
    return binding


def grid():
    """Values that 8 bits hold, every 1/16 up to 8 and every 1/8 up to 15, in blocks of one sign."""
    fine, wide = torch.arange(0, 128) / 16.0, torch.arange(0, 128) / 8.0
    x = torch.cat([fine, -fine, wide, -wide]).view(-1, 32)
    return x.cuda()


def phi(x):
    return torch.exp(-0.5 * x * x) / math.sqrt(2 * math.pi)


@pytest.mark.parametrize("pad", [0, 3])
def test_exact_gelu(B, pad):
    x = torch.zeros((16, 32 + pad), device="cuda")[:, :32]
    x.copy_(grid())
    codes, scales = B.star_checkpoint_empty(16, 32)
    h, dx = torch.empty_like(x), torch.empty_like(x)
    out = torch.zeros((16, 32 + pad), device="cuda")[:, :32]
    B.star_checkpoint_pack(codes, scales, x, act="gelu_erf", act_out=out)
    B.star_checkpoint_unpack(h, codes, scales)
    assert torch.equal(h, x)
    v = x.double()
    bound, tiny = (17 + 1.5 * v * v) * U, (1 + v.abs()) * 2.0 ** -126
    cdf = 0.5 * torch.erfc(-v / math.sqrt(2))
    err = (out.double() - v * cdf).abs()
    assert bool((err <= bound * (v * cdf).abs() + tiny).all()), float((err / ((v * cdf).abs() + tiny) / bound).max())
    B.star_checkpoint_unpack(out, codes, scales, act="gelu_erf")
    assert bool(((out.double() - v * cdf).abs() <= bound * (v * cdf).abs() + tiny).all())
    dy = torch.zeros((16, 32 + pad), device="cuda")[:, :32]
    dy.fill_(1.0)
    B.star_checkpoint_act_backward(out, dy, codes, scales, "gelu_erf")
    err = (out.double() - (cdf + v * phi(v))).abs()
    assert bool((err <= bound * (cdf + (v * phi(v)).abs()) + tiny).all())


def test_error_in_norm(B):
    """Activations as they come, Gaussian: near 0 some four roundings of 0.3 u each on average, twice
    that in the slope's sum, 3.6e-8 to 5e-8 of the whole (the same in elementary binary32
    operations).  Bound 7e-8."""
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((512, 1024), generator=g, device="cuda")
    codes, scales = B.star_checkpoint_empty(512, 1024)
    B.star_checkpoint_pack(codes, scales, x)
    v = torch.empty_like(x)
    B.star_checkpoint_unpack(v, codes, scales)
    out, dy = torch.empty_like(x), torch.randn((512, 1024), generator=g, device="cuda")
    B.star_checkpoint_unpack(out, codes, scales, act="gelu_erf")
    assert R.rel(out, R.act(v.double(), "gelu_erf")) <= 7e-8
    B.star_checkpoint_act_backward(out, dy, codes, scales, "gelu_erf")
    assert R.rel(out, dy.double() * R.act_slope(v.double(), "gelu_erf")) <= 7e-8


def test_exact_gelu_in_bf16(B):
    """A bf16 result is rounded by up to 2^-8 of itself.  Beside that the formula may be off by a
    thousandth of it, 4e-6, and the exponential by 1.5 x^2 u as above."""
    x = grid().to(torch.bfloat16)
    codes, scales = B.star_checkpoint_empty(16, 32)
    out, dy = torch.empty_like(x), torch.ones_like(x)
    B.star_checkpoint_pack(codes, scales, x, act="gelu_erf", act_out=out)
    v = x.double()
    bound, tiny = 2.0 ** -8 + 4e-6 + 1.5 * v * v * U, (1 + v.abs()) * 2.0 ** -126
    cdf = 0.5 * torch.erfc(-v / math.sqrt(2))
    assert bool(((out.double() - v * cdf).abs() <= bound * (v * cdf).abs() + tiny).all())
    B.star_checkpoint_act_backward(out, dy, codes, scales, "gelu_erf")
    slope = cdf + v * phi(v)
    assert bool(((out.double() - slope).abs() <= 2.0 ** -8 * slope.abs() + (bound - 2.0 ** -8) * (cdf + (v * phi(v)).abs()) * 1.01 + tiny).all())
