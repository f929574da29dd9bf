"""Root-mean-square norm, rows in 8 bits and their products on the GPU: against 64 bits with the bounds of rows8_reference."""
import numpy as np
import pytest
import torch

import encoder_reference as eref
import paper_2210_02574_amd as pkg
import rows8_reference as ref
import workloads as wl

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
WIDTHS = [(1, 1), (3, 7), (33, 16), (5, 250), (9, 256), (17, 257), (64, 768), (23, 1000), (7, 1021), (2050, 96), (6, 2048), (5, 2056), (3, 4096), (2, 5000), (3, 8192),
          (2, 10001), (2, 16384)]


@pytest.fixture(scope="module")
def he():
    assert torch.cuda.is_available(), "this test needs the MI355X"
    return pkg.HE.from_params(wl.C1B, device=0)


def rand(seed, *shape, dtype=F32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(*shape, generator=g)).to(dtype).cuda()


def integers(seed, rows, width, pad=0):
    """8-bit rows of any integers, with others behind them up to a multiple of 16."""
    g = torch.Generator().manual_seed(seed)
    return torch.randint(-128, 128, (rows, (width + 15) // 16 * 16 + pad), generator=g, dtype=torch.int8).cuda()[:, :width]


# ---- root-mean-square norm --------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype,wtype", [(F32, F32), (F16, F16), (F16, F32), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("rows,width", WIDTHS)
def test_rms_norm(he, rows, width, dtype, wtype):
    x, r, dy, ds = (rand(i, rows, width, dtype=dtype) for i in (1, 2, 3, 4))
    w = 1 + rand(5, width, dtype=wtype, scale=0.2)
    for residual, extra in ((None, None), (r, ds)):
        want = ref.rms_norm(x, w, residual, dy=dy, ds=extra)
        y, s, rstd = he.rms_norm(x, w, residual=residual)
        dx, dw = he.rms_norm_backward(dy, s, w, rstd, ds=extra)
        assert dw.dtype == wtype and dx.dtype == dtype
        for name, got in (("y", y), ("s", s), ("rstd", rstd), ("dx", dx), ("dw", dw)):
            eref.check(got, want[name], f"{name}, residual {residual is not None}")


def test_rms_norm_of_strided_and_unaligned_rows(he):
    big = rand(1, 40, 3, 264, dtype=BF16)
    w = rand(2, 256)
    for x in (big[:, 1, :256], big[:, 2, 1:257], big[3:, 0, 3:259], big[::2, 1, 8:]):
        want = ref.rms_norm(x, w, dy=x)
        out = torch.full((x.shape[0], 2, 256), 7.0, dtype=BF16, device="cuda")
        y, s, rstd = he.rms_norm(x, w, out=out[:, 1])
        eref.check(y, want["y"], "y")
        assert (out[:, 0] == 7).all() and s.data_ptr() == x.data_ptr()
        for name, got in zip(("dx", "dw"), he.rms_norm_backward(x, s, w, rstd)):
            eref.check(got, want[name], name)


def test_rms_norm_of_no_rows(he):
    x, w = torch.zeros(0, 64, dtype=BF16, device="cuda"), rand(1, 64)
    y, s, rstd = he.rms_norm(x, w)
    dx, dw = he.rms_norm_backward(x, s, w, rstd)
    assert y.shape == dx.shape == (0, 64) and not dw.any()
    y8, scale, _ = he.rms_norm8(x, w)
    assert y8.shape == (0, 64) and scale.shape == (0,)
    x8, scale = he.quantize8(x)
    o = he.linear8(x8, scale, *he.quantize8(rand(2, 5, 64)))
    assert o.shape == (0, 5)


# ---- rows in 8 bits ----------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("rows,width", WIDTHS)
def test_quantize(he, rows, width, dtype):
    x = rand(1, rows, width, dtype=dtype)
    x8, scale = he.quantize8(x)
    assert x8.dtype == torch.int8 and x8.shape == x.shape and x8.stride(0) % 64 == 0
    q, t = ref.quotients(x.double().cpu())
    assert torch.equal(x8.cpu().double(), torch.round(q))  # every x is a number of 32 bits: exact
    assert torch.equal(scale.cpu(), (t / 127).float())
    x8, scale = he.quantize8(x, gelu=True)
    f, e = ref.gelu(x)
    q, t = ref.quotients(f)
    et = e.gather(1, f.abs().argmax(1, keepdim=True))
    assert ((x8.cpu().double() - q).abs() <= 0.5 + 2.0**-15 + q.abs() * (e + et)).all()
    assert ((scale.cpu().double() - t / 127).abs() <= t / 127 * (et[:, 0] + 2.0**-23) + 1e-40).all()


@pytest.mark.parametrize("dtype,wtype", [(F32, F32), (F16, F16), (F16, F32), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("rows,width", WIDTHS)
def test_rms_norm_in_8_bits(he, rows, width, dtype, wtype):
    x, r = rand(1, rows, width, dtype=dtype), rand(2, rows, width, dtype=dtype)
    w = 1 + rand(5, width, dtype=wtype, scale=0.2)
    for residual in (None, r):
        y8, scale, s = he.rms_norm8(x, w, residual=residual)
        want = ref.rms_norm(x, w, residual)
        eref.check(s, want["s"], "s")
        q, t = ref.quotients(s.double().cpu() * w.double().cpu())
        if dtype == wtype and dtype != F32:
            assert torch.equal(y8.cpu().double(), torch.round(q))
        else:
            assert ((y8.cpu().double() - q).abs() <= 0.5 + 2.0**-15).all()
        rstd, bound = want["rstd"]
        assert ((scale.cpu().double() - t * rstd / 127).abs() <= t / 127 * (bound + 2.0**-22 * rstd)).all()


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_integers_on_the_border(he, dtype):
    """Rows whose quotients 127 x / t lie on k + 1/2 exactly: the even neighbour."""
    k = torch.arange(-127, 127, dtype=torch.float64) + 0.5
    for t in (127.0, 254.0, 63.5, 15.875):  # times an integer and a half, all of them numbers of 8 bits or more ..
        x = torch.cat([k * t / 127, torch.tensor([t], dtype=torch.float64)])
        keep = x.to(dtype).double() == x  # .. where the type has them
        row = x[keep].to(dtype).cuda()[None]
        assert keep.sum() > 100
        x8, scale = he.quantize8(row)
        assert torch.equal(x8.cpu().double()[0], torch.round(127 * row[0].double().cpu() / t))
        y8, _, _ = he.rms_norm8(row, torch.ones(row.shape[1], dtype=dtype, device="cuda"))
        assert torch.equal(x8, y8)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_integers_of_all_ratios(he, dtype):
    """All numbers of a type's significand against many maxima: exact."""
    bits = {F32: 12, F16: 11, BF16: 8}[dtype]
    x = torch.arange(2 ** (bits - 1), 2**bits, dtype=torch.float64)
    x = torch.cat([x, x / 2, x / 4, x / 16, x / 128, -x / 3])
    tops = 2.0**bits * (1 + torch.arange(0, 2 ** (bits - 1), max(1, 2 ** (bits - 8)), dtype=torch.float64) / 2 ** (bits - 1))
    rows = torch.cat([x.expand(len(tops), -1), tops[:, None]], 1).to(dtype).cuda()
    x8, scale = he.quantize8(rows)
    q, t = ref.quotients(rows.double().cpu())
    assert torch.equal(x8.cpu().double(), torch.round(q)) and torch.equal(scale.cpu(), (t / 127).float())


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_rows_of_any_size_in_8_bits(he, dtype):
    """From the smallest number of the type to the largest."""
    top, small = torch.finfo(dtype).max, {F32: 2.0**-149, F16: 2.0**-24, BF16: 2.0**-133}[dtype]
    base = torch.linspace(-1, 1, 333, dtype=torch.float64)
    for m in (top, top / 2, 2.0**-13, 2.0**-14, 100 * small, 3 * small, small):
        x = (base * m).to(dtype)
        x8, scale = he.quantize8(x.cuda()[None])
        q, t = ref.quotients(x.double()[None])
        assert torch.equal(x8.cpu().double(), torch.round(q)), m
        assert torch.equal(scale.cpu(), (t / 127).float()), m


def test_rows_that_are_not_finite_or_zero(he):
    nan, inf = float("nan"), float("inf")
    for dtype in (F32, F16, BF16):
        x = rand(1, 8, 300, dtype=dtype)
        w = 1 + rand(2, 300, dtype=dtype, scale=0.1)
        x[1, 5], x[2, 299], x[3, 0], x[5] = nan, inf, -inf, 0
        x[6] = -x[6].abs()
        good = [0, 4, 5, 6, 7]
        for x8, scale in (he.quantize8(x), he.quantize8(x, gelu=True), he.rms_norm8(x, w)[:2]):
            assert torch.isnan(scale[1:4]).all() and not x8[1:4].any()
            assert torch.isfinite(scale[good]).all() and (scale[[0, 4, 6, 7]] > 0).all()
            assert scale[5] == 0 and not x8[5].any()
            w8, ws = he.quantize8(rand(3, 40, 300))
            o = he.linear8(x8, scale, w8, ws)
            assert torch.isnan(o[1:4]).all() and torch.isfinite(o[good]).all() and not o[5].any()
        other = he.quantize8(x)
        x[1, 5], x[2, 299], x[3, 0] = 1, 1, 1
        again = he.quantize8(x)
        assert torch.equal(other[0][good], again[0][good]) and torch.equal(other[1][good], again[1][good])


def test_quantize_of_strided_and_unaligned_rows(he):
    big = rand(1, 40, 3, 264, dtype=BF16)
    for x in (big[:, 1, :256], big[:, 2, 1:257], big[3:, 0, 3:258], big[::2, 1, 8:]):
        x8, scale = he.quantize8(x)
        y8, y_scale = he.quantize8(x.contiguous())
        assert torch.equal(x8, y8) and torch.equal(scale, y_scale)


# ---- products --------------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("rows,width,channels", [
    (1, 1, 1), (1, 16, 16), (2, 15, 17), (15, 64, 3), (16, 65, 16), (17, 127, 33), (23, 768, 768), (31, 1021, 50), (32, 128, 257), (33, 100, 64), (48, 300, 31),
    (64, 2048, 65), (65, 64, 64), (65, 1, 1), (65, 129, 200), (100, 768, 100), (127, 1000, 129), (128, 130, 128), (129, 16, 63), (200, 257, 1021), (300, 113, 300),
    (1000, 384, 777), (1, 8192, 20), (40, 65536, 17), (70, 65535, 66), (700, 300, 700), (600, 1400, 800), (1100, 700, 1000), (2050, 200, 1500), (3100, 144, 4000), (3333, 1040, 4001), (1024, 129, 12400)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_product(he, rows, width, channels, dtype):
    x8, w8 = integers(1, rows, width, 32), integers(2, channels, width)
    size = 1 / (74 * 74 * width**0.5)  # results of about one
    scale, w_scale = size * (1 + rand(3, rows).abs()), 1 + rand(4, channels).abs()
    for bias in (None, rand(5, channels), rand(6, channels, dtype=dtype)):
        want = ref.linear8(x8, scale, w8, w_scale, bias, dtype)
        o = he.linear8(x8, scale, w8, w_scale, bias=bias, dtype=dtype)
        assert o.dtype == dtype
        assert ((o.double() - want[0]).abs() <= want[1]).all()
    out = torch.full((rows + 2, channels + 5), 7.0, dtype=dtype, device="cuda")  # rows that begin anywhere, and what is around them
    r = he.linear8(x8, scale, w8, w_scale, bias=bias, dtype=dtype, out=out[1:-1, 2:-3])
    assert torch.equal(r, o) and (out[0] == 7).all() and (out[-1] == 7).all() and (out[:, :2] == 7).all() and (out[:, -3:] == 7).all()


def test_product_of_the_largest_integers(he):
    """65536 products of -128 and -128 each: 2^30."""
    for rows in (3, 70):
        x8 = torch.full((rows, 65536), -128, dtype=torch.int8, device="cuda")
        w8 = torch.full((66, 65536), -128, dtype=torch.int8, device="cuda")
        one = torch.ones(rows, device="cuda"), torch.ones(66, device="cuda")
        assert (he.linear8(x8, one[0], w8, one[1], dtype=F32) == 2.0**30).all()


def test_product_of_views(he):
    big = integers(1, 90, 3 * 256)
    w8, ws = integers(2, 50, 256), rand(3, 50).abs()
    for rows in (90, 20):
        x8, scale = big[:rows, 256:512], rand(4, rows).abs()
        want = he.linear8(x8.contiguous(), scale, w8, ws, dtype=F32)
        assert torch.equal(he.linear8(x8, scale, w8, ws, dtype=F32), want)
        assert torch.equal(he.linear8(big[:2 * (rows // 2):2, 256:512], scale[::2].contiguous(), w8, ws, dtype=F32), want[::2])
        with pytest.raises(pkg.HeError, match="EINVAL"):  # rows in one place, as everywhere
            he.linear8(big[:1, 256:512].expand(rows, -1), scale, w8, ws, dtype=F32)
