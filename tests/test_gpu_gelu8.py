"""Gaussian error units in 8 bits on the GPU, in their lower tail, where 1 + erf in any precision has lost them: against x erfc(-x / sqrt 2) / 2 in 64 bits."""
import math

import pytest
import torch

import paper_2210_02574_amd as pkg
import workloads as wl

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def he():
    assert torch.cuda.is_available(), "this test needs the MI355X"
    return pkg.HE.from_params(wl.C1B, device=0)


def gelu(x):
    """(value, relative error granted) of x Phi(x)."""
    x = x.double().cpu()
    return 0.5 * x * torch.special.erfc(x * -math.sqrt(0.5)), 2.0**-20 * (1 + x * x / 8)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_units_of_single_numbers(he, dtype):
    """Rows of one number: its unit is the scale times 127, with two roundings to 32 bits."""
    if dtype == F32:
        x = torch.cat([torch.linspace(-13, 13, 400001, dtype=torch.float64), torch.tensor([-1e-3, -1e-30, 1e-30, 1e30, 3e38])]).float()
    else:  # all numbers of the type
        x = torch.arange(-(2**15), 2**15).to(torch.int16).view(dtype)
    x = x[torch.isfinite(x) & (x.float() >= -13)]
    x8, scale = he.quantize8(x.cuda()[:, None], gelu=True)
    f, e = gelu(x)
    want = (f.abs() / 127).clamp(max=torch.finfo(F32).max)
    # (a unit below 2^-126 and a scale below 2^-126 are off by 2^-150 each, and t 2^(..) by as much times |x| <= 13: 2^-145 in all)
    assert ((scale.cpu().double() - want).abs() <= want * (e + 2.0**-23) + 2.0**-145).all()
    some = scale.cpu() > 0
    assert torch.equal(x8.cpu()[some, 0].double(), 127 * torch.sign(f[some])) and not x8.cpu()[~some].any()
    assert (f[~some].abs() <= 2.0**-138).all()  # a scale of zero: less than 127 2^-149


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("rows,width", [(3, 7), (40, 100), (17, 768), (5, 1021), (3, 4096), (2, 10001)])
@pytest.mark.parametrize("low,high", [(-12.0, -4.0), (-13.0, -11.0), (-6.0, -0.5)])
def test_rows_of_the_lower_tail(he, rows, width, dtype, low, high):
    """Rows whose largest unit is itself one of the tail, so that it decides scale and integers."""
    g = torch.Generator().manual_seed(width)
    x = (low + (high - low) * torch.rand(rows, width, generator=g, dtype=torch.float64)).to(dtype).clamp(low, high)
    x8, scale = he.quantize8(x.cuda(), gelu=True)
    f, e = gelu(x)
    t, at = f.abs().max(1, keepdim=True)
    et = e.gather(1, at)
    q = 127 * f / t
    # an integer is the nearest to a quotient that is 2^-17 off; 2^-149 at most is lost to subnormal numbers of 13 2^-126 and less
    assert ((x8.cpu().double() - q).abs() <= 0.5 + 2.0**-16 + q.abs() * (e + et + 2.0**-145 / t)).all()
    assert ((scale.cpu().double() - t[:, 0] / 127).abs() <= t[:, 0] / 127 * (et[:, 0] + 2.0**-23) + 2.0**-145).all()
    assert (scale > 0).all() and (x8.cpu().min(1)[0] == -127).all()


def test_units_that_vanish(he):
    """Below -13 units are within 2^-123 of zero, and so are the kernel's."""
    x = -torch.cat([torch.linspace(13, 40, 20001), torch.logspace(1.6, 38, 1000)])
    x8, scale = he.quantize8(x.cuda()[:, None], gelu=True)
    assert (scale >= 0).all() and (scale * 127 <= 2.0**-123).all() and torch.isfinite(scale).all()
