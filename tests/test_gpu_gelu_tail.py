"""GELU and its slope far to the left in 16-bit types: x Phi(x) is small there, and is fp32 arithmetic rounded once all the same."""
import math

import pytest
import torch

import paper_2503_10017_amd as fnn
from net_helpers import DEV, F32, TYPES, assert_within, rounding

pytestmark = pytest.mark.gpu


def tail_off(x):
    """Relative error of Phi(-|x|): 1.2e-6 of the rational fit, exp2 of x^2 / 2 with three roundings of its exponent, and 16 of the rest."""
    return 1.2e-6 + F32 * (3 * x * x / 2 + 16)


def phi_left(x):
    """Phi(x) for x <= 0 with all its digits."""
    return 0.5 * torch.special.erfcx(-x / math.sqrt(2)) * torch.exp(-x * x / 2)


def points(kind):
    dtype = TYPES[kind]
    low = -5.5 if kind == "f16" else -12.5        # below, the result is under the type's normal range (the exponential under fp32's)
    return torch.linspace(low, 0, 20001, dtype=torch.float64).to(dtype).to(DEV)


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("rows", [8, 20001])
def test_value(kind, rows):
    p = points(kind)[:, None].contiguous()
    one = torch.ones((1, 1), dtype=p.dtype, device=DEV)
    got = torch.cat([fnn.fnn_linear(part.contiguous(), one, act="gelu")[0] for part in p.split(rows)][:2500])
    x = p[:len(got)].double()
    want = x * phi_left(x)
    assert_within(got, want, tail_off(x) * want.abs() + rounding(want, p.dtype))


@pytest.mark.parametrize("kind", ["f16", "bf16"])
def test_slope(kind):
    p = points(kind)[:, None].contiguous()
    one = torch.ones((1, 1), dtype=p.dtype, device=DEV)
    got = fnn.fnn_linear_backward(torch.ones_like(p), p, one, p, act="gelu")[0]
    x = p.double()
    phi, density = phi_left(x), torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    want = phi + x * density
    # rounded to the type before it is multiplied by 1
    assert_within(got, want, tail_off(x) * (phi + x.abs() * density) + rounding(want, p.dtype))
