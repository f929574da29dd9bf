"""The operators on token states without a GPU: what the C entry points and the binding refuse, and the reference that the GPU tests compare with,
against differences and torch's own formulas."""
import ctypes
import struct

import numpy as np
import pytest
import torch

import paper_2210_02574_amd as pkg
import workloads as wl
from encoder_reference import attention, layer_norm, pool_mean
from paper_2210_02574_amd.embedding import SentenceEncoder, pack_embeddings

EINVAL, EWORKSPACE, ENODEV = -1, -4, -6
P = 1 << 20  # an address that is never read: every call here ends before a launch


@pytest.fixture(scope="module")
def he():
    return pkg.HE.from_params(wl.C1B)


class _C:
    """Descriptors as bytes, laid out as C does."""

    he_rows = struct.Struct("@Pq").pack                # d, stride
    he_heads = struct.Struct("@Pqq").pack              # d, row, head
    he_spans = struct.Struct("@PPiq").pack             # d_begin, d_end, count, rows
    he_norm = struct.Struct("@iiqid").pack             # type, weight_type, rows, width, eps
    he_attn = struct.Struct("@4iPPiqPPiqddPi4x").pack  # type, heads, kv_heads, dim, q, k, scale, cap, d_slopes, fill


def _ref(x):
    return ctypes.byref(x) if isinstance(x, ctypes.c_size_t) else x


def _norm(he, n=None, x=(P, 64), residual=None, w=P, b=P, y=(P, 64), sum_=None, mean=P, rstd=P):
    r = [None if t is None else _C.he_rows(*t) for t in (x, residual, y, sum_)]
    n = n or _C.he_norm(2, 0, 5, 64, 1e-5)
    return he.lib.he_layer_norm(he.ctx, _ref(n), _ref(r[0]), _ref(r[1]), w, b, _ref(r[2]), _ref(r[3]), mean, rstd, None)


def test_layer_norm_refusals(he):
    assert _norm(he) == ENODEV  # nothing wrong but the device
    for bad in (_C.he_norm(3, 0, 5, 64, 1e-5), _C.he_norm(-1, 0, 5, 64, 1e-5), _C.he_norm(2, 1, 5, 64, 1e-5), _C.he_norm(0, 2, 5, 64, 1e-5),
                _C.he_norm(2, 0, -1, 64, 1e-5), _C.he_norm(2, 0, 1 << 31, 64, 1e-5), _C.he_norm(2, 0, 5, 0, 1e-5),
                _C.he_norm(2, 0, 5, 16385, 1e-5), _C.he_norm(2, 0, 5, 64, -1.0), _C.he_norm(2, 0, 5, 64, float("nan")),
                _C.he_norm(2, 0, 5, 64, float("inf")), _C.he_norm(2, 0, 5, 64, 1e300)):
        assert _norm(he, bad) == EINVAL
    for kw in ({"x": None}, {"x": (0, 64)}, {"x": (P, 63)}, {"y": None}, {"y": (P, 63)}, {"w": None}, {"b": None}, {"mean": None},
               {"rstd": None}, {"residual": (P, 64)}, {"residual": (P, 63), "sum_": (P, 64)}, {"residual": (P, 64), "sum_": (P, 63)}):
        assert _norm(he, **kw) == EINVAL, kw
    assert he.lib.he_layer_norm(None, *[None] * 10) == EINVAL
    for kw in ({"x": (P + 1, 64)}, {"y": (P + 1, 64)}, {"w": P + 1}, {"b": P + 1}, {"mean": P + 2}, {"rstd": P + 2},
               {"residual": (P + 1, 64), "sum_": (P, 64)}, {"residual": (P, 64), "sum_": (P + 1, 64)}):  # not at a multiple of the element's size
        assert _norm(he, _C.he_norm(2, 2, 5, 64, 1e-5), **kw) == EINVAL, kw
    assert _norm(he, _C.he_norm(2, 0, 5, 64, 1e-5), w=P + 2) == EINVAL and _norm(he, _C.he_norm(2, 2, 5, 64, 1e-5), w=P + 2) == ENODEV
    assert _norm(he, _C.he_norm(2, 0, 0, 64, 1e-5), x=None, y=None) == ENODEV  # no rows: buffers are not looked at


def test_layer_norm_grad_refusals(he):
    need = ctypes.c_size_t()
    n = _C.he_norm(2, 0, 5, 64, 0.0)
    assert he.lib.he_layer_norm_workspace_bytes(he.ctx, _ref(n), _ref(need)) == 0 and need.value >= 2 * 64 * 4
    assert he.lib.he_layer_norm_workspace_bytes(he.ctx, _ref(_C.he_norm(2, 0, 5, 0, 0.0)), _ref(need)) == EINVAL
    assert he.lib.he_layer_norm_workspace_bytes(he.ctx, _ref(n), None) == EINVAL

    def call(dy=(P, 64), s=(P, 64), w=P, mean=P, rstd=P, add=None, ds=(P, 64), dw=P, db=P, ws=P, size=1 << 20, n=n):
        r = [None if t is None else _C.he_rows(*t) for t in (dy, s, add, ds)]
        return he.lib.he_layer_norm_grad(he.ctx, _ref(n), _ref(r[0]), _ref(r[1]), w, mean, rstd, _ref(r[2]), _ref(r[3]), dw, db, ws, size, None)

    assert call() == ENODEV
    for kw in ({"dy": None}, {"s": None}, {"s": (P, 8)}, {"w": None}, {"mean": None}, {"rstd": None}, {"add": (P, 63)}, {"add": (0, 64)},
               {"ds": None}, {"dw": None}, {"db": None}, {"ws": P + 2}):
        assert call(**kw) == EINVAL, kw
    for kw in ({"dy": (P + 1, 64)}, {"s": (P + 1, 64)}, {"add": (P + 1, 64)}, {"ds": (P + 1, 64)}, {"w": P + 1}, {"dw": P + 1}, {"db": P + 1},
               {"mean": P + 2}, {"rstd": P + 2}):
        assert call(**kw) == EINVAL, kw
    assert call(ws=None) == EWORKSPACE and call(size=need.value - 1) == EWORKSPACE


def _span(count=3, rows=40, begin=P, end=P):
    return begin or 0, end or 0, count, rows


def _spans(*args, **kw):
    return _C.he_spans(*_span(*args, **kw))


def test_pool_refusals(he):
    need = ctypes.c_size_t()
    long = _spans(1, 100000)
    assert he.lib.he_pool_workspace_bytes(he.ctx, _ref(long), 64, _ref(need)) == 0 and need.value >= 2 * 64 * 4
    x = _C.he_rows(P, 64)
    pool = lambda s, width=64, x=x, e=P, ws=P, size=1 << 30, type=0: he.lib.he_pool(  # noqa: E731
        he.ctx, type, _ref(s), width, _ref(x), e, ws, size, None)
    grad = lambda s, width=64, x=x, e=P, type=0: he.lib.he_pool_grad(he.ctx, type, _ref(s), width, e, _ref(x), 1, None)  # noqa: E731
    assert pool(_spans()) == ENODEV and grad(_spans()) == ENODEV
    assert pool(_spans(0, 40)) == ENODEV and grad(_spans(0, 40)) == ENODEV
    assert pool(_spans(1 << 23), size=1 << 40) == ENODEV and grad(_spans(1 << 23)) == ENODEV
    for s in (None, _spans(-1), _spans((1 << 23) + 1), _spans((1 << 24) + 1), _spans(begin=P + 2), _spans(end=P + 1), _spans(3, -1), _spans(3, 1 << 31), _spans(begin=None), _spans(end=None)):
        assert pool(s) == EINVAL and grad(s) == EINVAL
        assert he.lib.he_pool_workspace_bytes(he.ctx, _ref(s), 64, _ref(need)) == EINVAL
    for kw in ({"width": 0}, {"width": (1 << 20) + 1}, {"x": None}, {"x": _C.he_rows(P, 63)}, {"x": _C.he_rows(P + 2, 64)}, {"e": None}, {"e": P + 2},
               {"type": 3}):
        assert pool(_spans(), **kw) == EINVAL and grad(_spans(), **kw) == EINVAL, kw
    assert pool(long, ws=None) == EWORKSPACE and pool(long, size=64) == EWORKSPACE and pool(long, ws=P + 2) == EINVAL


def _attn(type=2, heads=4, kv=2, dim=64, q=None, k=None, scale=0.125, cap=0.0, slopes=0):
    return _C.he_attn(type, heads, kv, dim, *(q or _span()), *(k or _span()), scale, cap, slopes, 1)


def test_attention_refusals(he):
    h = _C.he_heads(P, 512, 64)

    def fwd(s, q=h, k=h, v=h, o=h, lse=P, ws=P, size=1 << 40):
        return he.lib.he_attention(he.ctx, _ref(s), _ref(q), _ref(k), _ref(v), _ref(o), lse, ws, size, None)

    def bwd(s, go=h, q=h, k=h, v=h, o=h, lse=P, dq=h, dk=h, dv=h, ws=P, size=1 << 40):
        return he.lib.he_attention_grad(he.ctx, _ref(s), *[_ref(t) for t in (go, q, k, v, o)], lse, _ref(dq), _ref(dk), _ref(dv), ws, size, None)

    assert fwd(_attn()) == ENODEV and bwd(_attn()) == ENODEV
    assert fwd(_attn(q=_span(0, 5), k=_span(0, 5))) == ENODEV and bwd(_attn(q=_span(0, 5), k=_span(0, 5))) == ENODEV
    need = ctypes.c_size_t()
    inf, nan = float("inf"), float("nan")
    for s in (None, _attn(type=3), _attn(heads=0), _attn(kv=0), _attn(heads=5), _attn(heads=65536, kv=1), _attn(dim=0), _attn(dim=12),
              _attn(dim=136), _attn(scale=0.0), _attn(scale=-1.0), _attn(scale=nan), _attn(scale=inf), _attn(scale=1e-60), _attn(scale=1e60), _attn(cap=-1.0),
              _attn(cap=nan), _attn(cap=inf), _attn(cap=1e-60), _attn(scale=1e30, cap=1e-30), _attn(q=_span(2)), _attn(q=_span(-1), k=_span(-1)), _attn(q=_span(3, -1)),
              _attn(q=_span(3, 1 << 31)), _attn(q=_span(begin=None)), _attn(k=_span(end=None))):
        assert fwd(s) == EINVAL and bwd(s) == EINVAL
        assert he.lib.he_attention_workspace_bytes(he.ctx, _ref(s), 0, _ref(need)) == EINVAL
    for bad in (None, _C.he_heads(0, 512, 64), _C.he_heads(P + 8, 512, 64), _C.he_heads(P, 508, 64), _C.he_heads(P, 512, 60), _C.he_heads(P, -512, 64)):
        for name in ("q", "k", "v", "o"):
            assert fwd(_attn(), **{name: bad}) == EINVAL, (name, bad)
        for name in ("go", "q", "k", "v", "o", "dq", "dk", "dv"):
            assert bwd(_attn(), **{name: bad}) == EINVAL, (name, bad)
    assert fwd(_attn(), lse=P + 2) == EINVAL and bwd(_attn(), lse=P + 2) == EINVAL
    assert fwd(_attn(slopes=P + 4)) == ENODEV and fwd(_attn(slopes=P + 2)) == EINVAL and bwd(_attn(slopes=P + 2)) == EINVAL
    assert fwd(_attn(), lse=None) == EINVAL and bwd(_attn(), lse=None) == EINVAL
    assert bwd(_attn(), ws=None) == EWORKSPACE and bwd(_attn(), size=40 * 4 * 4 - 1) == EWORKSPACE and bwd(_attn(), ws=P + 4) == EINVAL
    long = _attn(q=_span(1, 1), k=_span(1, 1 << 20))  # one query of many keys: cut along the keys
    assert he.lib.he_attention_workspace_bytes(he.ctx, _ref(long), 0, _ref(need)) == 0 and need.value >= 2 * 4 * 65 * 4
    assert fwd(long) == ENODEV and fwd(long, ws=None) == EWORKSPACE and fwd(long, size=need.value - 1) == EWORKSPACE and fwd(long, ws=P + 4) == EINVAL
    huge = _attn(heads=4096, kv=4096, q=_span(1, 1 << 30), k=_span(1, 1 << 30))  # more work-groups than a launch holds
    assert fwd(huge, size=1 << 62) == EINVAL and bwd(huge, size=1 << 62) == EINVAL
    for bad in (_C.he_heads(P, 32, 64), _C.he_heads(P, 512, 32), _C.he_heads(P, 0, 64), _C.he_heads(P, 512, 0), _C.he_heads(P, 64, 64), _C.he_heads(P, 72, 64),
                _C.he_heads(P, 128, 1024)):  # outputs that overlap themselves
        assert fwd(_attn(), o=bad) == EINVAL
        for name in ("dq", "dk", "dv"):
            assert bwd(_attn(), **{name: bad}) == EINVAL, name
        assert fwd(_attn(), q=bad, k=bad, v=bad) == ENODEV  # inputs may
    apart = _C.he_heads(P, 64, 40 * 64)  # one head after the other
    assert fwd(_attn(), o=apart) == ENODEV and bwd(_attn(), dq=apart, dk=apart, dv=apart) == ENODEV
    assert fwd(_attn(), q=_C.he_heads(P, 512, 1 << 46)) == EINVAL


def test_binding_refusals(he):
    x, w = torch.zeros(4, 8), torch.ones(8)
    off = torch.tensor([0, 4], dtype=torch.int32)
    for f in (lambda: he.layer_norm(x, w, w), lambda: he.layer_norm_backward(x, x, w, torch.zeros(4), torch.zeros(4)), lambda: he.pool_mean(x, off),
              lambda: he.pool_mean_backward(x, off, 4, torch.float32), lambda: he.attention(*[x.view(4, 1, 8)] * 3, off)):
        with pytest.raises(ValueError, match="device|want"):
            f()  # CPU tensors: there is no fallback
    for f in (lambda: he.layer_norm(x[0], w, w), lambda: he.layer_norm(x.t(), w, w), lambda: he.pool_mean(x.view(2, 2, 8), off), lambda: he.attention(x, x, x, off),
              lambda: he.layer_norm(x, None, w), lambda: he.layer_norm(x.to_sparse(), w, w),
              lambda: he.layer_norm(torch.complex(x, x).conj().imag, w, w), lambda: he.pool_mean_backward(x, off, 4, 5), lambda: he.pool_mean_backward(x, off, -1, torch.float32)):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: he.layer_norm(x.double(), w, w), lambda: he.pool_mean(x.long(), off), lambda: he.pool_mean_backward(x, off, 4, torch.float64)):
        with pytest.raises(ValueError, match="float32, float16 or bfloat16"):
            f()


def test_encoder_refusals(he):
    w = SentenceEncoder.random_layer(16, 2, 24, 1, torch.float32, "cpu")
    with pytest.raises(ValueError, match="pool"):
        SentenceEncoder(he, [w], 2, pool="max")
    with pytest.raises(ValueError, match="lacks norm2"):
        SentenceEncoder(he, [{k: v for k, v in w.items() if k != "norm2"}], 2)
    with pytest.raises(ValueError, match="constants"):
        SentenceEncoder(he, [w], 2, slopes=torch.ones(2, requires_grad=True))
    from paper_2210_02574_amd.embedding import attention as diff_attention

    with pytest.raises(ValueError, match="constants"):
        diff_attention(he, None, None, None, None, slopes=torch.ones(2, requires_grad=True))


def test_pack_embeddings_fills_the_last_ciphertext():
    e = torch.arange(3 * 768, dtype=torch.float32).view(3, 768)
    packed = pack_embeddings(e, 2048)  # two sentences to a ciphertext
    assert len(packed) == 2
    assert np.array_equal(packed[0][1024 + 4:1024 + 772], e[1].numpy()) and np.array_equal(packed[1][4:772], e[2].numpy())
    assert not packed[1][1024:].any() and not packed[0][772:1028].any()


# ---- the reference itself ----------------------------------------------------------------------------------------------


def _difference(f, x, i, step=1e-6):
    a, b = x.clone(), x.clone()
    a.view(-1)[i] += step
    b.view(-1)[i] -= step
    return (f(a) - f(b)) / (2 * step)


@pytest.mark.parametrize("cap,bias", [(0.0, False), (1.5, True)])
def test_reference_attention_gradients_against_differences(cap, bias):
    g = torch.Generator().manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    q, k, v, do = r(5, 4, 8), r(7, 2, 8), r(7, 2, 8), r(5, 4, 8)
    oq, ok = torch.tensor([0, 3, 3, 5]), torch.tensor([0, 4, 4, 7])
    sl = torch.tensor([0.5, 0.25, 0.125, 0.0]) if bias else None
    got = attention(q, k, v, oq, ok, cap=cap, slopes=sl, do=do)
    loss = lambda q=q, k=k, v=v: float((attention(q, k, v, oq, ok, cap=cap, slopes=sl)["o"][0] * do).sum())  # noqa: E731
    for name, x in (("q", q), ("k", k), ("v", v)):
        for i in (0, 9, x.numel() // 2, x.numel() - 1):
            assert abs(_difference(lambda t: loss(**{name: t}), x, i) - float(got["d" + name][0].view(-1)[i])) < 1e-7


def test_reference_layer_norm_and_mean_against_differences():
    g = torch.Generator().manual_seed(4)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    x, w, b, dy = r(6, 9), r(9), r(9), r(6, 9)
    s = torch.float64
    got = layer_norm(x, w, b, dy=dy)
    want = torch.nn.functional.layer_norm(x, (9,), w, b)
    assert (got["y"][0] - want).abs().max() < 1e-12
    loss = lambda x=x, w=w, b=b: float((torch.nn.functional.layer_norm(x, (9,), w, b) * dy).sum())  # noqa: E731
    for name, t, key in (("x", x, "dx"), ("w", w, "dw"), ("b", b, "db")):
        for i in (0, t.numel() - 1):
            assert abs(_difference(lambda v: loss(**{name: v}), t, i) - float(got[key][0].view(-1)[i])) < 1e-6
    e, _ = pool_mean(x, torch.tensor([0, 2, 2, 6]))
    assert torch.equal(e[1], torch.zeros(9, dtype=s)) and torch.allclose(e[2], x[2:].mean(0))
