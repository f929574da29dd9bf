"""Root-mean-square norm and its gradients on rows with infinities, NaN, squares beyond 32 bits and nothing but zeros, beside good rows: what such a row gives, and that it
reaches no other row."""
import pytest
import torch

import encoder_reference as eref
import paper_2210_02574_amd as pkg
import rows8_reference as ref
import workloads as wl

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
NAN, INF = float("nan"), float("inf")
# below a vector, multiples of one and not, threads of a part of a wave, a wave and several
WIDTHS = [5, 64, 77, 768, 1021, 2050, 5000, 8192]


@pytest.fixture(scope="module")
def he():
    assert torch.cuda.is_available(), "this test needs the MI355X"
    return pkg.HE.from_params(wl.C1B, device=0)


def rand(seed, *shape, dtype=F32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(*shape, generator=g)).to(dtype).cuda()


@pytest.mark.parametrize("dtype,wtype", [(F32, F32), (F16, F32), (BF16, BF16)])
@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("rows", [8, 300])
def test_rows_that_are_not_finite(he, rows, width, dtype, wtype):
    """Rows 1 (a NaN), 2 (an infinity in the last place), 3 (a negative one in the first) and 4 (values whose squares leave 32 bits; fp16 has none) against the definition; all others
    are bit for bit what they are without them."""
    x, dy, ds, w = rand(1, rows, width, dtype=dtype), rand(2, rows, width, dtype=dtype), rand(3, rows, width, dtype=dtype), 1 + rand(4, width, dtype=wtype, scale=0.2)
    plain = x.clone()
    plain_y, _, plain_rstd = he.rms_norm(plain, w)
    x[1, width // 2], x[2, -1], x[3, 0] = NAN, INF, -INF
    if dtype != F16:
        x[4] = 1e30 * torch.sign(x[4].float()).to(dtype)
    bad = [1, 2, 3] if dtype == F16 else [1, 2, 3, 4]
    good = [r for r in range(rows) if r not in bad]
    y, s, rstd = he.rms_norm(x, w)
    assert torch.equal(y[good], plain_y[good]) and torch.equal(rstd[good], plain_rstd[good])
    assert torch.isnan(rstd[1]) and torch.isnan(y[1]).all()
    assert not rstd[bad[1:]].any()
    want = x[bad[1:]].float() * 0  # y = s 0 w: zeros, and NaN at infinities
    assert torch.equal(torch.isnan(y[bad[1:]]), torch.isnan(want)) and not torch.nan_to_num(y[bad[1:]]).any()

    dx, dw = he.rms_norm_backward(dy, s, w, rstd, ds=ds)
    plain_dx, _ = he.rms_norm_backward(dy, plain, w, plain_rstd, ds=ds)
    assert torch.equal(dx[good], plain_dx[good])
    assert torch.isnan(dx[1:4]).all()  # mean(g s) of such a row is not a number
    if dtype != F16:
        assert torch.equal(dx[4], ds[4])  # rstd = 0: the gradient of y = 0
    assert torch.isnan(dw).all()  # row 1 has no number in any column

    zero = dy.clone()
    zero[1] = 0
    assert torch.isnan(he.rms_norm_backward(zero, s, w, rstd)[1]).all()  # 0 times NaN too
    # without row 1: the columns of the two infinities alone, and elsewhere the sum over the good rows
    x[1], rstd[1] = plain[1], plain_rstd[1]
    dx, dw = he.rms_norm_backward(dy, x, w, rstd)
    keep = [r for r in range(rows) if r not in bad[1:]]
    assert torch.isnan(dw[[0, -1]]).all()
    want = ref.rms_norm(plain[keep], w, dy=dy[keep])["dw"]
    eref.check(dw[1:-1], (want[0][1:-1], want[1][1:-1]), "dw")


@pytest.mark.parametrize("dtype,wtype", [(F32, F32), (F16, F32), (BF16, BF16)])
@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("rows", [8, 300])
def test_gradients_that_are_not_finite(he, rows, width, dtype, wtype):
    """An infinity and a NaN in dy, and in the gradient that reaches s from elsewhere: their rows of dx and their columns of dw, and no others."""
    x, dy, ds, w = rand(1, rows, width, dtype=dtype), rand(2, rows, width, dtype=dtype), rand(3, rows, width, dtype=dtype), 1 + rand(4, width, dtype=wtype, scale=0.2)
    _, s, rstd = he.rms_norm(x, w)
    plain_dx, plain_dw = he.rms_norm_backward(dy, s, w, rstd, ds=ds)
    dy[1, 0], dy[2, -1], ds[5, width // 2] = INF, NAN, NAN
    dx, dw = he.rms_norm_backward(dy, s, w, rstd, ds=ds)
    good = [r for r in range(rows) if r not in (1, 2, 5)]
    assert torch.equal(dx[good], plain_dx[good])
    assert not torch.isfinite(dx[[1, 2]]).any()
    at = torch.arange(width, device="cuda") == width // 2
    assert torch.isnan(dx[5, at]).all() and torch.equal(dx[5, ~at], plain_dx[5, ~at])
    assert torch.isinf(dw[0]) and torch.isnan(dw[-1]) and torch.equal(dw[1:-1], plain_dw[1:-1])


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("width", WIDTHS)
def test_rows_of_zeros(he, width, dtype):
    """With eps: y = 0 and ds = dy w eps^-1/2; without: not finite, and no other row is touched."""
    x, dy, w = rand(1, 9, width, dtype=dtype), rand(2, 9, width, dtype=dtype), 1 + rand(4, width, scale=0.2)
    x[4] = 0
    y, s, rstd = he.rms_norm(x, w)
    want = ref.rms_norm(x, w, dy=dy)
    assert not y[4].any()
    for name, got in zip(("dx", "dw"), he.rms_norm_backward(dy, s, w, rstd)):
        eref.check(got, want[name], name)
    y, s, rstd = he.rms_norm(x, w, eps=0.0)
    good = [r for r in range(9) if r != 4]
    want = ref.rms_norm(x[good], w, eps=0.0)
    eref.check(y[good], want["y"], "y")
    assert torch.isinf(rstd[4]) and torch.isnan(y[4]).all()
