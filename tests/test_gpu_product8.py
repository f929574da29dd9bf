"""Products of 8-bit rows and weights on the GPU, in every variant, against 64 bits with the bounds of rows8_reference."""
import pytest
import torch

import paper_2210_02574_amd as pkg
import rows8_reference as ref
import workloads as wl
from product8_shapes import PITCH, VARIANTS

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
# rows, width, channels: tiles of 16 with four and eight groups of waves, of 32, of 64 with one and four groups, of 128, of 256 by 192, of 256
SHAPES = [(23, 768, 768), (17, 2100, 100), (500, 768, 768), (1000, 300, 1000), (1000, 1040, 1000), (5284, 200, 768), (16380, 144, 768), (4090, 300, 4096)]


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


@pytest.mark.parametrize("rows,width,channels", SHAPES)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scales_at_the_ends_of_the_range(he, rows, width, channels, dtype):
    """Sums of up to 2^20 times the scale of a row of large values leave 32 bits, results do not: x_scale up to 2^120, w_scale about 2^-110; and the other way round.  Rows beside
    them are ordinary, one is zero, and one's results leave the range."""
    x8, w8, bias = integers(1, rows, width), integers(2, channels, width), rand(3, channels)
    x8[1] = 0
    w8[5] = 0
    e = torch.arange(rows) % 5
    scale = (1 + rand(4, rows).abs()) * torch.tensor([2.0**120, 1.0, 2.0**63, 2.0**64, 2.0**100])[e].cuda()
    w_scale = (1 + rand(5, channels).abs()) * 2.0**-110
    scale[1] = 2.0**126
    for xs, ws in ((scale, w_scale), (scale * 2.0**-110, w_scale * 2.0**110), (scale * 2.0**-120, w_scale * 2.0**120)):
        for b in (None, bias):
            want, bound = ref.linear8(x8, xs, w8, ws, b, dtype)
            assert want.abs().max() < 2.0**127
            o = he.linear8(x8, xs, w8, ws, bias=b, dtype=dtype).double()
            assert ((o - want).abs() <= bound).all()
    xs = torch.full_like(scale, 2.0**120)
    o = he.linear8(x8, xs, w8, torch.full_like(w_scale, 2.0**20), bias=bias, dtype=F32)
    sums = x8.double() @ w8.double().t()
    assert torch.equal(o.double(), torch.where(sums == 0, bias.double(), sums * float("inf")))


@pytest.mark.parametrize("rows,width,channels", list(VARIANTS))
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_results_that_fill_whole_lines(he, rows, width, channels, dtype):
    """Rows of results that begin at multiples of 128 bytes, the last tile of rows ragged: alone, and in a wider buffer with channels that no vector divides, where a row's last piece is
    written element by element behind whole ones.  What stands around the results stays."""
    x8, w8 = integers(1, rows, width, 32), integers(2, channels, width)
    scale, w_scale = (1 + rand(3, rows).abs()) / (74 * 74 * width**0.5), 1 + rand(4, channels).abs()  # results of about one
    bias = rand(5, channels, dtype=dtype)
    want, bound = ref.linear8(x8, scale, w8, w_scale, bias, dtype)
    o = he.linear8(x8, scale, w8, w_scale, bias=bias, dtype=dtype)
    assert channels % PITCH == 0 and o.data_ptr() % 128 == 0
    assert ((o.double() - want).abs() <= bound).all()
    for fewer, pitch in ((0, channels + PITCH), (3, channels), (11, channels + 2 * PITCH)):
        n = channels - fewer
        buf = torch.full((rows + 2, pitch), 7.0, dtype=dtype, device="cuda")
        r = he.linear8(x8, scale, w8[:n], w_scale[:n], bias=bias[:n], dtype=dtype, out=buf[1:-1, :n])
        assert r.data_ptr() % 128 == 0
        assert torch.equal(r, o[:, :n])
        assert (buf[0] == 7).all() and (buf[-1] == 7).all() and (buf[:, n:] == 7).all()


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_rows_and_channels_do_not_hang_on_those_beside_them(he, dtype):
    """The same rows and channels in calls of every variant, bit for bit: sums are exact, and each result is rounded to 32 bits before its type."""
    rows, width, channels = 16380, 1040, 4096
    x8, w8 = integers(1, rows, width), integers(2, channels, width)
    scale, w_scale, bias = (1 + rand(3, rows).abs()) / (74 * 74 * width**0.5), 1 + rand(4, channels).abs(), rand(5, channels, dtype=dtype)
    call = lambda m, n: he.linear8(x8[:m], scale[:m], w8[:n], w_scale[:n], bias=bias[:n], dtype=dtype)  # noqa: E731
    whole = call(rows, channels)
    for m, n in ((rows, 768), (rows, 765), (4001, 4032), (5284, 700), (1000, 1024), (1000, 2000), (500, 768), (23, 765), (1, 100)):
        assert torch.equal(call(m, n), whole[:m, :n]), (m, n)
    eight = he.linear8(x8[:20, :400], scale[:20], w8[:50, :400], w_scale[:50], bias=bias[:50], dtype=dtype)
    assert torch.equal(he.linear8(x8[:3000, :400], scale[:3000], w8[:3000, :400], w_scale[:3000], bias=bias[:3000], dtype=dtype)[:20, :50], eight)
