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
          (2, 10001), (2, 16384), (32, 100), (33, 100), (31, 513), (17, 768), (70, 40), (65, 64), (37, 65), (140, 31), (99, 128)]


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


def offsets_of(lengths):
    return torch.tensor(np.concatenate([[0], np.cumsum(lengths)]).tolist(), dtype=torch.int32, device="cuda")


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
    (1000, 384, 777), (1, 8192, 20), (40, 65536, 17), (70, 65535, 66), (700, 300, 700), (600, 1400, 800), (1100, 700, 1000), (2050, 200, 1500), (3100, 144, 4000), (3333, 1040, 4001), (1024, 129, 12400),
    (1000, 1101, 777), (1, 2048, 1), (17, 5001, 100), (16, 33, 4000), (40, 7777, 31), (500, 2000, 1000), (33, 4097, 700),
    (2900, 130, 3301), (700, 1040, 12001), (8000, 1030, 2896)])
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


@pytest.mark.parametrize("rows,width,channels", [(600000, 8192, 40), (600001, 16, 4096), (70000, 32, 33000)])
def test_product_far_into_long_buffers(he, rows, width, channels):
    """Rows of x8, and of results, that begin behind 2^32 bytes and 2^31 elements."""
    x8 = torch.randint(-127, 128, (rows, width), dtype=torch.int8, device="cuda")
    scale, w8, ws = torch.rand(rows, device="cuda") / width, integers(2, channels, width), rand(3, channels).abs()
    o = he.linear8(x8, scale, w8, ws)
    for at in (0, rows // 2, rows - 300):
        want = ref.linear8(x8[at:at + 300], scale[at:at + 300], w8, ws, None, BF16)
        assert ((o[at:at + 300].double() - want[0]).abs() <= want[1]).all(), at


@pytest.mark.parametrize("dtype,width", [(BF16, 768), (F16, 64), (F32, 128), (BF16, 100), (F32, 1021)])
def test_results_are_the_same_however_they_are_written(he, dtype, width):
    """Rows do not hang on one another: a call that moves more than the last-level cache holds, rows of it alone, and rows that begin inside lines, bit for bit."""
    rows = 300 * 2**20 // (width * torch.finfo(dtype).bits // 8) // 3
    x, r, w = rand(1, rows, width, dtype=dtype), rand(2, rows, width, dtype=dtype), rand(3, width, dtype=dtype)
    y, s, rstd = he.rms_norm(x, w, residual=r)
    alone, _, rstd1 = he.rms_norm(x, w)
    y8, scale, s8 = he.rms_norm8(x, w, residual=r)
    q8, q = he.quantize8(x)
    dx, _ = he.rms_norm_backward(r, s, w, rstd, ds=x)
    assert torch.equal(s, x + r) and torch.equal(s8, s)
    for at in (0, rows // 3, rows - 1000):
        i = slice(at, at + 1000)
        small = he.rms_norm(x[i], w, residual=r[i])
        assert torch.equal(small[0], y[i]) and torch.equal(small[2], rstd[i])
        buf = torch.full((1002, width + 64 * 4), 7.0, dtype=dtype, device="cuda")
        for out in (buf[1:-1, 64:64 + width], buf[1:-1, 1:1 + width]):
            out.fill_(0)
            assert he.rms_norm(x[i], w, out=out)[0] is out and torch.equal(out, alone[i])
            out.fill_(7)
        assert (buf == 7).all()
        small8 = he.rms_norm8(x[i], w, residual=r[i])
        assert torch.equal(small8[0], y8[i]) and torch.equal(small8[1], scale[i])
        small8 = he.quantize8(x[i])
        assert torch.equal(small8[0], q8[i]) and torch.equal(small8[1], q[i])
        assert torch.equal(he.rms_norm_backward(r[i], s[i], w, rstd[i], ds=x[i])[0], dx[i])
    assert torch.equal(rstd1[:9], he.rms_norm(x[:9], w)[2])


def test_more_rows_than_a_launch_holds(he):
    """2^32 threads are too many, and eight of them are a row's here.  Every row has the same numbers in another order of its two halves."""
    rows, row, w = (1 << 28) + 37, rand(1, 8, dtype=BF16), torch.ones(8, device="cuda")
    x = row.expand(rows, 8).contiguous()
    x[1::2] = row.roll(4)
    y, _, rstd = he.rms_norm(x, w)
    small = he.rms_norm(x[:2], w)
    for k in range(2):
        assert (y[k::2] == small[0][k]).all() and (rstd[k::2] == small[2][k]).all()
    del y, rstd
    x8, scale = he.quantize8(x)
    small = he.quantize8(x[:2])
    for k in range(2):
        assert (x8[k::2] == small[0][k]).all() and (scale[k::2] == small[1][k]).all()


def test_rms_norm_weight_gradient_of_many_rows_repeats(he):
    x, dy = rand(1, 70001, 64, dtype=F16), rand(2, 70001, 64, dtype=F16)
    w = rand(3, 64)
    _, s, rstd = he.rms_norm(x, w)
    a, b = he.rms_norm_backward(dy, s, w, rstd), he.rms_norm_backward(dy, s, w, rstd)
    want = ref.rms_norm(x, w, dy=dy)
    for name, u, v in zip(("dx", "dw"), a, b):
        assert torch.equal(u, v)
        eref.check(u, want[name], name)


# ---- arguments -----------------------------------------------------------------------------------------------------------------------


def test_refusals_on_the_device(he):
    x, w = rand(1, 8, 64, dtype=BF16), rand(2, 64)
    x8, s = he.quantize8(x)
    w8, ws = he.quantize8(rand(3, 5, 64))
    flat = torch.zeros(400, dtype=torch.int8, device="cuda")
    for f in (lambda: he.rms_norm(x, w[:63]), lambda: he.rms_norm(x, w, residual=x[:4]), lambda: he.rms_norm(x, w, residual=x.float()), lambda: he.rms_norm(x.double(), w),
              lambda: he.rms_norm(x, w, out=x.float()), lambda: he.rms_norm8(x, w.cpu()), lambda: he.rms_norm_backward(x, x, w, rand(1, 7)), lambda: he.quantize8(x[0]),
              lambda: he.quantize8(x.t()), lambda: he.quantize8(x.cpu()), lambda: he.quantize8(x8), lambda: he.linear8(x, s, w8, ws), lambda: he.linear8(x8, s[:7], w8, ws),
              lambda: he.linear8(x8, s, w8, ws[:4]), lambda: he.linear8(x8, s, w8[:, :48], ws), lambda: he.linear8(x8, s, w8, ws, bias=rand(1, 4)),
              lambda: he.linear8(x8, s, w8, ws, dtype=torch.float64), lambda: he.linear8(x8, s, w8, ws, dtype=5), lambda: he.linear8(x8, s, w8, ws, out=torch.zeros(8, 4, device="cuda")),
              lambda: he.linear8(x8, s, w8, ws, dtype=F32, out=torch.zeros(8, 5, device="cuda", dtype=BF16)), lambda: he.linear8(x8.cpu(), s, w8, ws),
              lambda: he.linear8(x8[:, 1:17], s, w8[:, :16], ws), lambda: he.linear8(flat[:144].view(8, 18)[:, :16], s, w8[:, :16], ws),
              lambda: he.linear8(flat[:136].view(8, 17), s, w8[:, :17], ws),  # rows at no multiples of 16 bytes, and a last piece that the buffer does not hold
              lambda: he.linear8(torch.zeros(7 * 32 + 20, dtype=torch.int8, device="cuda").as_strided((8, 20), (32, 1)), s, w8[:, :20], ws)):
        with pytest.raises(ValueError):
            f()
    wide = torch.zeros(2, 16385, device="cuda")
    for f in (lambda: he.rms_norm(x, w, eps=-1.0), lambda: he.rms_norm(x, rand(2, 64, dtype=F16)), lambda: he.rms_norm8(wide, wide[0]), lambda: he.quantize8(wide),
              lambda: he.quantize8(wide[:, :0]), lambda: he.linear8(x8, s, w8[:0], ws[:0]), lambda: he.linear8(x8, s, w8, ws, bias=rand(1, 5, dtype=F16)),
              lambda: he.linear8(torch.zeros(2, 65552, dtype=torch.int8, device="cuda"), s[:2], torch.zeros(2, 65552, dtype=torch.int8, device="cuda"), s[:2]),
              lambda: he.linear8(torch.zeros(2, 1 << 23, dtype=torch.int8, device="cuda")[:, :64], s[:2], w8, ws)):
        with pytest.raises(pkg.HeError, match="EINVAL"):
            f()


def test_buffers_to_write_to(he):
    """They get another version, are refused where autograd tracks them or where they overlap what the call reads, and taken beside it."""
    buf = rand(1, 2048)
    x, w = buf[:512].view(8, 64), rand(2, 64)
    x8, s = he.quantize8(x)
    w8, ws = he.quantize8(rand(3, 64, 64))
    calls = (lambda out: he.rms_norm(x, w, out=out), lambda out: he.linear8(x8, s, w8, ws, out=out))
    for f in calls:
        out, t = torch.ones(8, 64, device="cuda"), torch.ones(8, 64, device="cuda", requires_grad=True)
        y = (t * out).sum()
        f(out)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()
        with pytest.raises(ValueError, match="require gradients"):
            f(torch.ones(8, 64, device="cuda", requires_grad=True))
    for f in (lambda: he.rms_norm(x, w, out=x), lambda: he.rms_norm(x, buf[1024:1088], out=buf[1000:1512].view(8, 64)),
              lambda: he.linear8(x8, buf[600:608], w8, ws, out=buf[512:1024].view(8, 64)), lambda: he.linear8(x8, s, w8, ws, bias=buf[:64], out=x)):
        with pytest.raises(ValueError, match="overlap"):
            f()
    both = torch.cat([x, torch.zeros_like(x)], 1)
    assert torch.equal(he.rms_norm(both[:, :64], w, out=both[:, 64:])[0], he.rms_norm(x, w)[0]) and torch.equal(both[:, :64], x)


# ---- streams, graphs, together ---------------------------------------------------------------------------------------------------------


def _everything(he, x, r, w, dy, w8, ws, b):
    y, s, rstd = he.rms_norm(x, w, residual=r)
    y8, scale, _ = he.rms_norm8(x, w, residual=r)
    u8, u_scale = he.quantize8(y, gelu=True)
    return (y, s, rstd, y8.clone(), scale, u8.clone(), u_scale, he.linear8(y8, scale, w8, ws, bias=b), he.linear8(y8[:40], scale[:40], w8, ws, bias=b),
            he.linear8(u8, u_scale, w8[:100], ws[:100], dtype=F32), *he.rms_norm_backward(dy, s, w, rstd, ds=r))


def _inputs(he, seed, rows=3000, width=328, channels=4100):
    w8, ws = he.quantize8(rand(seed, channels, width))
    return [rand(seed + 1, rows, width, dtype=BF16), rand(seed + 2, rows, width, dtype=BF16), rand(seed + 3, width), rand(seed + 4, rows, width, dtype=BF16), w8, ws,
            rand(seed + 5, channels)]


def test_repeats_bit_for_bit_on_two_streams_at_once(he):
    ins = [_inputs(he, 10), _inputs(he, 20)]
    want = [[t.clone() for t in _everything(he, *i)] for i in ins]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], [None, None]
    for rep in range(3):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                got[k] = _everything(he, *ins[k])
        torch.cuda.synchronize()
        for k in range(2):
            assert all(torch.equal(a, b) for a, b in zip(got[k], want[k])), (rep, k)


def test_two_captured_graphs(he):
    """Two graphs captured on one stream and replayed on two at once; inputs change between replays."""
    ins, fresh = [_inputs(he, 30), _inputs(he, 40)], [_inputs(he, 50), _inputs(he, 60)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for i in ins:
            _everything(he, *i)
    torch.cuda.synchronize()
    graphs, outs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()], [None, None]
    for k in range(2):
        with torch.cuda.graph(graphs[k], stream=side):
            outs[k] = _everything(he, *ins[k])
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for rep in range(4):
        if rep == 2:
            for k in range(2):
                for a, b in zip(ins[k], fresh[k]):
                    a.copy_(b)
        want = [[t.clone() for t in _everything(he, *i)] for i in ins]  # eager work between the replays
        torch.cuda.synchronize()
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                graphs[k].replay()
        torch.cuda.synchronize()
        for k in range(2):
            assert all(torch.equal(a, b) for a, b in zip(outs[k], want[k])), (rep, k)


def test_rms_norm_gradients_against_differences(he):
    """Along random directions: central differences with step h are off by h^2 and by 2^-24 |f| / h."""
    from paper_2210_02574_amd.embedding import rms_norm

    x, c, e = [rand(1, 39, 128), rand(2, 39, 128), rand(3, 128)], rand(4, 39, 128).double(), rand(5, 39, 128).double()

    def f(x, r, w):
        y, s = rms_norm(he, x, w, residual=r)
        return (y.double() * c + s.double() * e).sum()

    leaves = [t.requires_grad_(True) for t in x]
    grads = torch.autograd.grad(f(*leaves), leaves)
    h = 2.0**-7
    for i in range(3):
        d = rand(10 + i, *x[i].shape)
        d = d / d.norm()
        with torch.no_grad():
            a = [t + h * d if j == i else t for j, t in enumerate(x)]
            b = [t - h * d if j == i else t for j, t in enumerate(x)]
            diff = float(f(*a) - f(*b)) / (2 * h)
        want = float((grads[i] * d).sum())
        assert abs(diff - want) < 2.0**-11 * (1 + float(grads[i].norm())), (i, diff, want)


def test_rms_norm_passes_gradients_of_either_result_alone(he):
    from paper_2210_02574_amd.embedding import rms_norm

    x, r, w = (t.requires_grad_(True) for t in (rand(1, 6, 64), rand(2, 6, 64), rand(3, 64)))
    _, s = rms_norm(he, x, w, residual=r)
    s.sum().backward()
    assert (x.grad == 1).all() and (r.grad == 1).all() and w.grad is None
    y, same = rms_norm(he, x, w)
    assert same is x
    g, = torch.autograd.grad(y.square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        g.sum().backward()


def _plain_encoder(layers, last, x, off, heads, pool):
    """A pre-norm encoder in 64 bits by torch's differentiable elementary operations."""
    x = x.double()
    norm = lambda t, w: t * (t.pow(2).mean(1, keepdim=True) + 1e-5).rsqrt() * w  # noqa: E731
    o = off.tolist()
    for w in layers:
        w = {k: v.double() for k, v in w.items()}
        times = lambda t, n: t @ w[n].T + w[n + "_bias"]  # noqa: E731, B023
        d = x.shape[1] // heads
        qkv = times(norm(x, w["norm1"]), "qkv").view(-1, 3 * heads, d)
        rows = []
        for b, e in zip(o[:-1], o[1:]):
            q, k, v = (qkv[b:e, i * heads:(i + 1) * heads].transpose(0, 1) for i in range(3))
            rows.append((torch.softmax(q @ k.transpose(1, 2) * d**-0.5, -1) @ v).transpose(0, 1).flatten(1))
        x = x + times(torch.cat(rows), "out")
        x = x + times(torch.nn.functional.gelu(times(norm(x, w["norm2"]), "up")), "down")
    x = norm(x, last.double())
    take = (lambda b, e: x[b:e].mean(0)) if pool == "mean" else lambda b, e: x[b]
    return torch.stack([take(b, e) if e > b else x[:1].sum(0) * 0 for b, e in zip(o[:-1], o[1:])])


@pytest.mark.parametrize("pool", ["mean", "first"])
def test_encoder_with_root_mean_square_norms_and_its_gradients(he, pool):
    """All operators together in 32 bits.  Errors of single operations are near 2^-24 of their operands, a few hundred of them follow one another
    over two layers, norms multiply by at most rstd ~ 1: 2^-14 of the largest element is granted."""
    from paper_2210_02574_amd.embedding import SentenceEncoder

    layers = [SentenceEncoder.random_layer(64, 2, 96, 5 + i, F32, "cuda", std=0.1) for i in range(2)]
    layers = [{k: v for k, v in w.items() if k not in ("norm1_bias", "norm2_bias")} for w in layers]
    states, off, de, last = rand(1, 60, 64), offsets_of([20, 0, 1, 39]), rand(2, 4, 64), 1 + rand(3, 64, scale=0.1)
    leaves = [states, last] + [v for w in layers for v in w.values()]
    for t in leaves:
        t.requires_grad_(True)
    e = SentenceEncoder(he, layers, 2, pool=pool, norm="rms", last=last)(states, off)
    got = torch.autograd.grad(e, leaves, de)
    plain = _plain_encoder(layers, last, states, off, 2, pool)
    want = torch.autograd.grad(plain, leaves, de.double())
    assert e.dtype == F32 and (e - plain).abs().max() <= 2.0**-14 * plain.abs().max()
    for g, w in zip(got, want):
        assert (g - w).abs().max() <= 2.0**-14 * max(1.0, float(w.abs().max())), g.shape


@pytest.mark.parametrize("pool", ["mean", "first"])
@pytest.mark.parametrize("norm", ["layer", "rms"])
@pytest.mark.parametrize("width,inner", [(64, 96), (80, 100)])
def test_encoder_in_8_bits(he, norm, pool, width, inner):
    """Against the calls of the operators one by one, equal, and against the encoder that it comes from.  A row of a hundred values has its largest at about 2.6 times their mean
    size, so a step of 1/127 of it is off by 0.006 of that size in the mean (a step over root 12); a product has two such factors, a layer four products that add up or follow
    one another: 0.006 root 2 root 8 = 0.024 over two layers, of which the norms at the end keep what stands across the sum; three times that is granted."""
    from paper_2210_02574_amd.embedding import SentenceEncoder, SentenceEncoder8

    layers = [SentenceEncoder.random_layer(width, 2, inner, 5 + i, F32, "cuda", std=0.1) for i in range(2)]
    last = 1 + rand(3, width, scale=0.1) if norm == "rms" else None
    states, off = rand(1, 60, width), offsets_of([20, 0, 1, 39])
    enc = SentenceEncoder(he, layers, 2, pool=pool, norm=norm, last=last)
    enc8 = enc.in_8_bits()
    assert isinstance(enc8, SentenceEncoder8) and enc8.in_8_bits() is enc8
    e, e8 = enc(states, off), enc8(states, off)
    assert e8.dtype == F32 and not e8[1].any()
    some = [0, 2, 3]
    assert (e8 - e)[some].norm() <= 0.072 * e[some].norm()

    times = lambda a, w, n: he.linear8(*a, *he.quantize8(w[n]), bias=w[n + "_bias"], dtype=F32)  # noqa: E731
    x, f = states, None
    for w in layers:
        if norm == "rms":
            x8, s, x = he.rms_norm8(x, w["norm1"]) if f is None else he.rms_norm8(f, w["norm1"], residual=x)
            a = x8, s
        else:
            a = he.quantize8(x)
        qkv = times(a, w, "qkv").view(60, 6, -1)
        o, _ = he.attention(qkv[:, :2], qkv[:, 2:4], qkv[:, 4:], off)
        f = times(he.quantize8(o.flatten(1)), w, "out")
        if norm == "rms":
            x8, s, x = he.rms_norm8(f, w["norm2"], residual=x)
            a = x8, s
        else:
            x = he.layer_norm(f, w["norm1"], w["norm1_bias"], residual=x)[0]
            a = he.quantize8(x)
        f = times(he.quantize8(times(a, w, "up"), gelu=True), w, "down")
        if norm == "layer":
            x = he.layer_norm(f, w["norm2"], w["norm2_bias"], residual=x)[0]
    if norm == "rms":
        x = he.rms_norm(f, last, residual=x)[0]
    if pool == "mean":
        assert torch.equal(e8, he.pool_mean(x, off))
    else:  # the same rows in another product, and an attention of lone queries
        assert (e8[some] - x[[0, 20, 21]]).abs().max() <= 0.02 * x.abs().max()
    assert enc8(states[:0], offsets_of([0, 0])).shape == (2, width)
    with pytest.raises(ValueError, match="no gradients"):
        enc8(states.clone().requires_grad_(True), off)


@pytest.mark.parametrize("norm", ["layer", "rms"])
def test_encoder_in_8_bits_keeps_sentences_and_padding_apart(he, norm):
    """A padded batch whose padding holds NaN and infinities, against the same sentences packed: every operator works on rows or sequences alone; attention's tiles lie elsewhere,
    which is a rounding of 2^-24 here, and a neighbouring integer now and then."""
    from paper_2210_02574_amd.embedding import SentenceEncoder

    layers = [SentenceEncoder.random_layer(64, 2, 96, 5 + i, F32, "cuda", std=0.1) for i in range(2)]
    enc = SentenceEncoder(he, layers, 2, norm=norm, last=rand(3, 64) if norm == "rms" else None).in_8_bits()
    lengths, packed = [20, 0, 1, 39], rand(1, 60, 64)
    padded, at = torch.full((4 * 40, 64), float("nan"), device="cuda"), 0
    padded[30] = float("inf")
    for i, n in enumerate(lengths):
        padded[40 * i:40 * i + n] = packed[at:at + n]
        at += n
    begin = torch.arange(0, 160, 40, dtype=torch.int32, device="cuda")
    a, b = enc(packed, offsets_of(lengths)), enc(padded, (begin, begin + torch.tensor(lengths, dtype=torch.int32, device="cuda")))
    assert torch.isfinite(b).all() and (a - b).abs().max() <= 0.02 * a.abs().max()
    packed[5, 7] = float("nan")  # of the first sentence
    c = enc(packed, offsets_of(lengths))
    assert torch.isnan(c[0]).all() and torch.equal(a[1:], c[1:])


def test_two_threads_at_once(he):
    import threading

    ins = [_inputs(he, 70, 400, 200, 300), _inputs(he, 80, 20, 1000, 90)]
    want = [[t.clone() for t in _everything(he, *i)] for i in ins]
    torch.cuda.synchronize()
    bad, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]

    def work(k):
        with torch.cuda.stream(streams[k]):
            for _ in range(50):
                got = _everything(he, *ins[k])
            streams[k].synchronize()
            if not all(torch.equal(a, b) for a, b in zip(got, want[k])):
                bad.append(k)

    threads = [threading.Thread(target=work, args=(k,)) for k in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad


def test_encoder_in_8_bits_in_a_graph(he):
    from paper_2210_02574_amd.embedding import SentenceEncoder

    layers = [SentenceEncoder.random_layer(768, 12, 1000, 5 + i, BF16, "cuda") for i in range(2)]
    enc = SentenceEncoder(he, layers, 12, norm="rms", last=torch.ones(768, dtype=BF16, device="cuda")).in_8_bits()
    states, off = rand(1, 700, 768, dtype=BF16), offsets_of([20, 0, 1, 39, 500, 140])
    enc(states, off)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = enc(states, off)
    for rep in range(3):
        states.copy_(rand(10 + rep, 700, 768, dtype=BF16))
        off.copy_(offsets_of([20 + rep, 0, 1, 39 - rep, 400, 240]))
        want = enc(states, off).clone()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), rep


def test_sentences_in_8_bits_to_encrypted_logits(he):
    """Token states -> 8-bit encoder -> packed, encrypted -> encrypted classifier -> logits, against the same in the clear."""
    from paper_2210_02574_amd.classifier import EncryptedInference, logits_from_slots
    from paper_2210_02574_amd.embedding import SentenceEncoder

    layers = [SentenceEncoder.random_layer(768, 12, 1024, 7 + i, BF16, "cuda") for i in range(2)]
    enc = SentenceEncoder(he, layers, 12).in_8_bits()
    lengths = [17, 1, 64]
    states, off = rand(9, sum(lengths), 768, dtype=BF16), offsets_of(lengths)
    W = wl.weights(11)
    level, scale = 3, 2.0**30
    inf = EncryptedInference(he, level)
    sk = he.keygen_secret(12)
    keys = inf.make_keys(sk, 13)
    cts = inf.encrypt_sentences(sk, enc, states, off, scale, 14)
    e = enc(states, off).double().cpu().numpy()
    pts = inf.encode_weights(W)
    got = np.concatenate([logits_from_slots(he.decrypt(sk, he.to_host(inf.run(ct, pts, keys)), scale)) for ct in cts])
    assert np.abs(got[:3] - e @ W.T).max() < 2.0**-8  # scale 2^30 on the smallest ring
