"""Root-mean-square norm, rows in 8 bits and their products without a GPU: what the C entry points and the binding refuse, and the reference that the GPU tests
compare with, against differences and torch's own formulas."""
import ctypes
import struct

import pytest
import torch

import paper_2210_02574_amd as pkg
import rows8_reference as ref
import workloads as wl
from paper_2210_02574_amd.embedding import SentenceEncoder

EINVAL, EWORKSPACE, ENODEV = -1, -4, -6
P = 1 << 20  # an address that is never read: every call here ends before a launch


@pytest.fixture(scope="module")
def he():
    return pkg.HE.from_params(wl.C1B)


rows_ = struct.Struct("@Pq").pack        # he_rows: d, stride
rows8 = struct.Struct("@PqP").pack       # he_rows8: d, stride, d_scale
norm_ = struct.Struct("@iiqid").pack     # he_norm: type, weight_type, rows, width, eps
product_ = struct.Struct("@iiqii").pack  # he_product8: type, bias_type, rows, width, channels


def _pack(f, t):
    return None if t is None else f(*t)


def _norm(he, n=norm_(2, 0, 5, 64, 1e-5), x=(P, 64), residual=None, w=P, y=(P, 64), sum_=None, rstd=P):
    return he.lib.he_rms_norm(he.ctx, n, _pack(rows_, x), _pack(rows_, residual), w, _pack(rows_, y), _pack(rows_, sum_), rstd, None)


def _norm8(he, n=norm_(2, 0, 5, 64, 1e-5), x=(P, 64), residual=None, w=P, y=(P, 64, P), sum_=None):
    return he.lib.he_rms_norm8(he.ctx, n, _pack(rows_, x), _pack(rows_, residual), w, _pack(rows8, y), _pack(rows_, sum_), None)


BAD_NORMS = [norm_(3, 0, 5, 64, 1e-5), norm_(-1, 0, 5, 64, 1e-5), norm_(2, 1, 5, 64, 1e-5), norm_(0, 2, 5, 64, 1e-5), norm_(2, 0, -1, 64, 1e-5), norm_(2, 0, 1 << 31, 64, 1e-5),
             norm_(2, 0, 5, 0, 1e-5), norm_(2, 0, 5, 16385, 1e-5)]
BAD_EPS = [norm_(2, 0, 5, 64, v) for v in (-1.0, float("nan"), float("inf"), 1e300)]


def test_rms_norm_refusals(he):
    for f in (_norm, _norm8):
        assert f(he) == ENODEV  # nothing wrong but the device
        for n in [None] + BAD_NORMS + BAD_EPS:
            assert f(he, n) == EINVAL
        for kw in ({"x": None}, {"x": (0, 64)}, {"x": (P, 63)}, {"x": (P + 1, 64)}, {"y": None}, {"w": None}, {"w": P + 2}, {"residual": (P, 64)}, {"residual": (P, 63), "sum_": (P, 64)},
                   {"residual": (P, 64), "sum_": (P, 63)}, {"residual": (P + 1, 64), "sum_": (P, 64)}, {"residual": (P, 64), "sum_": (P + 1, 64)}):
            assert f(he, **kw) == EINVAL, kw
        assert f(he, residual=(P, 64), sum_=(P, 64)) == ENODEV
        assert f(he, norm_(2, 2, 5, 64, 1e-5), w=P + 2) == ENODEV
        assert f(he, norm_(2, 0, 0, 64, 1e-5), x=None, y=None) == ENODEV  # no rows: buffers are not looked at
    for y in ((P, 63), (P + 1, 64), (0, 64)):
        assert _norm(he, y=y) == EINVAL
    for y in ((P, 63, P), (0, 64, P), (P, 64, 0), (P, 64, P + 2)):
        assert _norm8(he, y=y) == EINVAL
    assert _norm8(he, y=(P + 1, 65, P)) == ENODEV  # integers that are written may begin anywhere
    assert _norm(he, rstd=None) == EINVAL and _norm(he, rstd=P + 2) == EINVAL
    assert he.lib.he_rms_norm(None, *[None] * 8) == EINVAL and he.lib.he_rms_norm8(None, *[None] * 7) == EINVAL


def test_rms_norm_grad_refusals(he):
    def grad(n=norm_(2, 0, 500, 64, 0.0), dy=(P, 64), s=(P, 64), w=P, rstd=P, add=None, ds=(P, 64), dw=P, ws=P, size=1 << 40):
        return he.lib.he_rms_norm_grad(he.ctx, n, _pack(rows_, dy), _pack(rows_, s), w, rstd, _pack(rows_, add), _pack(rows_, ds), dw, ws, size, None)

    need = ctypes.c_size_t()  # (500 rows: 50 of this width are one work-group's, which needs no workspace)
    assert grad() == ENODEV and grad(add=(P, 64)) == ENODEV
    for n in [None] + BAD_NORMS:
        assert grad(n) == EINVAL and he.lib.he_rms_norm_workspace_bytes(he.ctx, n, ctypes.byref(need)) == EINVAL
    for kw in ({"dy": None}, {"dy": (P, 63)}, {"s": None}, {"s": (P + 1, 64)}, {"w": None}, {"w": P + 2}, {"rstd": None}, {"rstd": P + 2}, {"add": (P, 63)}, {"ds": None}, {"ds": (P, 63)},
               {"dw": None}, {"dw": P + 2}, {"ws": P + 2}):
        assert grad(**kw) == EINVAL, kw
    assert he.lib.he_rms_norm_workspace_bytes(he.ctx, norm_(2, 0, 500, 64, 0.0), ctypes.byref(need)) == 0 and need.value >= 64 * 4
    assert grad(ws=None) == EWORKSPACE and grad(size=need.value - 1) == EWORKSPACE and grad(size=need.value) == ENODEV
    assert he.lib.he_rms_norm_workspace_bytes(he.ctx, norm_(2, 0, 5, 64, 0.0), ctypes.byref(need)) == 0 and need.value == 0
    assert grad(norm_(2, 0, 5, 64, 0.0), ws=None, size=0) == ENODEV  # few rows
    assert he.lib.he_rms_norm_workspace_bytes(he.ctx, norm_(2, 0, 0, 64, 0.0), ctypes.byref(need)) == 0 and need.value == 0
    assert grad(norm_(2, 0, 0, 64, 0.0), dy=None, s=None, ds=None, rstd=None, ws=None, size=0) == ENODEV


def test_quantize_refusals(he):
    def quantize(type=2, rows=5, width=64, x=(P, 64), y=(P, 64, P)):
        return he.lib.he_quantize8(he.ctx, type, rows, width, 0, _pack(rows_, x), _pack(rows8, y), None)

    assert quantize() == ENODEV and quantize(rows=0, x=None, y=None) == ENODEV
    for kw in ({"type": 3}, {"type": -1}, {"rows": -1}, {"rows": 1 << 31}, {"width": 0}, {"width": 16385, "x": (P, 1 << 20), "y": (P, 1 << 20, P)}, {"x": None}, {"x": (P, 63)},
               {"x": (P + 1, 64)}, {"y": None}, {"y": (P, 63, P)}, {"y": (0, 64, P)}, {"y": (P, 64, 0)}, {"y": (P, 64, P + 1)}):
        assert quantize(**kw) == EINVAL, kw


def test_product_refusals(he):
    def product(type=2, bias_type=0, rows=5, width=64, channels=7, x=(P, 64, P), w=(P, 64, P), bias=P, o=(P, 7), p=True):
        return he.lib.he_linear8(he.ctx, product_(type, bias_type, rows, width, channels) if p else None, _pack(rows8, x), _pack(rows8, w), bias, _pack(rows_, o), None)

    assert product() == ENODEV and product(bias=None) == ENODEV and product(rows=0, x=None, o=None) == ENODEV
    assert product(bias_type=2, bias=P + 2) == ENODEV and product(o=(P + 2, 9)) == ENODEV  # results may begin anywhere
    big = (P, (1 << 23) - 16, P)
    assert product(width=65536, x=big, w=big) == ENODEV
    for kw in ({"p": False}, {"type": 3}, {"type": -1}, {"bias_type": 1}, {"type": 0, "bias_type": 2}, {"rows": -1}, {"rows": 1 << 31}, {"width": 0}, {"width": 65537, "x": big, "w": big},
               {"channels": 0}, {"channels": (1 << 24) + 1, "o": (P, 1 << 25)}, {"bias": P + 2}, {"o": None}, {"o": (P, 6)}, {"o": (P + 1, 7)},
               {"rows": 1 << 30, "channels": 1 << 24, "o": (P, 1 << 24)}):
        assert product(**kw) == EINVAL, kw
    for bad in (None, (0, 64, P), (P, 64, 0), (P, 64, P + 2), (P, 48, P), (P, 72, P), (P + 8, 64, P), (P, -64, P), (P, 1 << 23, P)):
        assert product(x=bad) == EINVAL and product(w=bad) == EINVAL, bad


def test_binding_refusals(he):
    x, w = torch.zeros(4, 16), torch.ones(16)
    i8, s = torch.zeros(4, 16, dtype=torch.int8), torch.ones(4)
    for f in (lambda: he.rms_norm(x, w), lambda: he.rms_norm8(x, w), lambda: he.rms_norm_backward(x, x, w, s), lambda: he.quantize8(x), lambda: he.linear8(i8, s, i8, s)):
        with pytest.raises(ValueError, match="device|want"):
            f()  # CPU tensors: there is no fallback
    for f in (lambda: he.rms_norm(x.long(), w), lambda: he.quantize8(i8), lambda: he.quantize8(x.double())):
        with pytest.raises(ValueError, match="float32, float16 or bfloat16"):
            f()
    with pytest.raises(ValueError, match="tensor"):
        he.linear8(i8, None, i8, s)


def test_encoder_refusals(he):
    w, one = SentenceEncoder.random_layer(16, 2, 24, 1, torch.float32, "cpu"), torch.ones(16)
    with pytest.raises(ValueError, match="norm:"):
        SentenceEncoder(he, [w], 2, norm="batch")
    for kw in ({"norm": "rms"}, {"last": one}):
        with pytest.raises(ValueError, match="last"):
            SentenceEncoder(he, [w], 2, **kw)
    rms = {k: v for k, v in w.items() if k not in ("norm1_bias", "norm2_bias")}
    SentenceEncoder(he, [rms], 2, norm="rms", last=one)
    with pytest.raises(ValueError, match="lacks norm1_bias, norm2_bias"):
        SentenceEncoder(he, [rms], 2)
    with pytest.raises(ValueError, match="lacks norm2"):
        SentenceEncoder(he, [{k: v for k, v in rms.items() if k != "norm2"}], 2, norm="rms", last=one)


# ---- the reference itself ----------------------------------------------------------------------------------------------


def test_reference_rms_norm_against_differences_and_torch():
    g = torch.Generator().manual_seed(4)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    x, w, dy = r(6, 9), r(9), r(6, 9)
    got = ref.rms_norm(x, w, dy=dy)
    torch_norm = lambda x, w: torch.nn.functional.rms_norm(x, (9,), w, 1e-5)  # noqa: E731
    assert (got["y"][0] - torch_norm(x, w)).abs().max() < 1e-12
    for name, t, key in (("x", x, "dx"), ("w", w, "dw")):
        for i in (0, t.numel() // 2, t.numel() - 1):
            a, b = t.clone(), t.clone()
            a.view(-1)[i] += 1e-6
            b.view(-1)[i] -= 1e-6
            f = lambda v: float((torch_norm(**{"x": x, "w": w, name: v}) * dy).sum())  # noqa: E731, B023
            assert abs((f(a) - f(b)) / 2e-6 - float(got[key][0].view(-1)[i])) < 1e-6


def test_reference_of_8_bits():
    f = torch.tensor([[1.0, -0.5, 0.25, 0.0], [0.0, 0.0, 0.0, 0.0]], dtype=torch.float64)
    q, t = ref.quotients(f)
    assert torch.equal(q[0], torch.tensor([127.0, -63.5, 31.75, 0.0], dtype=torch.float64)) and not q[1].any() and t.tolist() == [1.0, 0.0]
    x = torch.linspace(-6, 6, 25, dtype=torch.float64)
    assert (ref.gelu(x)[0] - torch.nn.functional.gelu(x)).abs().max() < 1e-12
    x8, w8 = torch.tensor([[1, -2]], dtype=torch.int8), torch.tensor([[3, 4], [5, -6], [0, 0]], dtype=torch.int8)
    o, _ = ref.linear8(x8, torch.tensor([0.5]), w8, torch.tensor([1.0, 2.0, 3.0]), torch.tensor([0.0, 1.0, 2.0]), torch.float32)
    assert o.tolist() == [[-2.5, 18.0, 2.0]]


def test_an_encoders_products_take_whole_weights_as_they_are():
    """A slice of all channels would cost a copy of their gradient."""
    from paper_2210_02574_amd.embedding import SentenceEncoder

    w = SentenceEncoder.random_layer(16, 2, 8, 1, torch.float32, "cpu")
    for t in w.values():
        t.requires_grad_(True)
    enc = SentenceEncoder(None, [w], 2)
    parts = lambda y: sorted(f.name() for f, _ in y.grad_fn.next_functions if f)  # noqa: E731
    x = torch.ones(3, 16)
    assert not any("Slice" in n for n in parts(enc._product(w, "qkv", x)))
    assert any("Slice" in n for n in parts(enc._product(w, "qkv", x, 16)))
