"""The operators on token states on the GPU: against 64 bits with the bounds of encoder_reference, on other streams, in graphs, and together, from token
states to decrypted logits."""
import numpy as np
import pytest
import torch

import encoder_reference as ref
import paper_2210_02574_amd as pkg
import workloads as wl

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def he():
    assert torch.cuda.is_available(), "this test needs the MI355X"
    return pkg.HE.from_params(wl.C1B, device=0)


def rand(seed, *shape, dtype=F32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(*shape, generator=g)).to(dtype).cuda()


def i32(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def offsets_of(lengths):
    return i32(*np.concatenate([[0], np.cumsum(lengths)]).tolist())


# ---- layer norm ----------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype,wtype", [(F32, F32), (F16, F16), (F16, F32), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("rows,width", [(1, 1), (3, 7), (33, 16), (5, 250), (9, 256), (17, 257), (64, 768), (23, 1000), (7, 1021), (2050, 96), (6, 2048), (5, 2056),
                                        (3, 4096), (2, 5000), (3, 8192), (2, 10001), (2, 16384)])
def test_layer_norm(he, rows, width, dtype, wtype):
    x, r, dy, ds = (rand(i, rows, width, dtype=dtype) for i in (1, 2, 3, 4))
    x = x + 1  # a mean that has to be taken off
    w, b = 1 + rand(5, width, dtype=wtype, scale=0.2), rand(6, width, dtype=wtype, scale=0.2)
    for residual, extra in ((None, None), (r, ds)):
        want = ref.layer_norm(x, w, b, residual, dy=dy, ds=extra)
        y, s, mean, rstd = he.layer_norm(x, w, b, residual=residual)
        dx, dw, db = he.layer_norm_backward(dy, s, w, mean, rstd, ds=extra)
        assert dw.dtype == wtype and dx.dtype == dtype
        for name, got in (("y", y), ("s", s), ("mean", mean), ("rstd", rstd), ("dx", dx), ("dw", dw), ("db", db)):
            ref.check(got, want[name], f"{name}, residual {residual is not None}")


def test_layer_norm_of_strided_and_unaligned_rows(he):
    big = rand(1, 40, 3, 264, dtype=BF16)
    w, b = rand(2, 256), rand(3, 256)
    for x in (big[:, 1, :256], big[:, 2, 1:257], big[3:, 0, 3:259], big[::2, 1, 8:]):
        want = ref.layer_norm(x, w, b, dy=x)
        out = torch.full((x.shape[0], 2, 256), 7.0, dtype=BF16, device="cuda")
        y, s, mean, rstd = he.layer_norm(x, w, b, out=out[:, 1])
        ref.check(y, want["y"], "y")
        assert (out[:, 0] == 7).all() and s.data_ptr() == x.data_ptr()
        for name, got in zip(("dx", "dw", "db"), he.layer_norm_backward(x, s, w, mean, rstd)):
            ref.check(got, want[name], name)


def test_layer_norm_keeps_rows_apart(he):
    x, w, b = rand(1, 9, 768, dtype=BF16), rand(2, 768), rand(3, 768)
    y = he.layer_norm(x, w, b)[0]
    x[4, 100], x[6, 5] = float("nan"), float("inf")
    z = he.layer_norm(x, w, b)[0]
    rows = [i for i in range(9) if i not in (4, 6)]
    assert torch.equal(y[rows], z[rows]) and torch.isnan(z[4]).all() and torch.isnan(z[6]).all()


def test_layer_norm_of_no_rows(he):
    x, w = torch.zeros(0, 64, dtype=BF16, device="cuda"), rand(1, 64)
    y, s, mean, rstd = he.layer_norm(x, w, w)
    dx, dw, db = he.layer_norm_backward(x, s, w, mean, rstd)
    assert y.shape == dx.shape == (0, 64) and not dw.any() and not db.any()


def test_layer_norm_of_more_rows_than_a_launch_holds(he):
    """2^32 threads are too many, and 32 of them are a row's here.  Every row has the same numbers in another order of its two halves."""
    rows, row = (1 << 27) + 37, rand(1, 8, dtype=BF16)
    x = row.expand(rows, 8).contiguous()
    x[1::2] = row.roll(4)
    y, _, mean, rstd = he.layer_norm(x, torch.ones(8, device="cuda"), torch.zeros(8, device="cuda"))
    small = he.layer_norm(x[:2], torch.ones(8, device="cuda"), torch.zeros(8, device="cuda"))
    for k in range(2):
        assert (y[k::2] == small[0][k]).all() and (mean[k::2] == small[2][k]).all() and (rstd[k::2] == small[3][k]).all()


def test_layer_norm_weight_gradient_of_many_rows_repeats(he):
    x, dy = rand(1, 70001, 64, dtype=F16), rand(2, 70001, 64, dtype=F16)
    w = rand(3, 64)
    _, s, mean, rstd = he.layer_norm(x, w, w)
    a, b = he.layer_norm_backward(dy, s, w, mean, rstd), he.layer_norm_backward(dy, s, w, mean, rstd)
    want = ref.layer_norm(x, w, w, dy=dy)
    for name, u, v in zip(("dx", "dw", "db"), a, b):
        assert torch.equal(u, v)
        ref.check(u, want[name], name)


# ---- mean ----------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("lengths,width", [([1], 1), ([0, 1, 5], 7), ([3, 0, 0, 70], 768), ([1000], 24), ([2, 31, 33, 32, 1], 2056), ([7000, 1], 768), ([40] * 300, 33)])
def test_pool_mean(he, lengths, width, dtype):
    off = offsets_of(lengths)
    rows = sum(lengths)
    x, de = rand(1, rows, width, dtype=dtype), rand(2, len(lengths), width)
    ref.check(he.pool_mean(x, off), ref.pool_mean(x, off), "e")
    dx = he.pool_mean_backward(de, off, rows, dtype)
    n = torch.repeat_interleave(torch.arange(len(lengths)), torch.tensor(lengths))
    want = de.double().cpu()[n] / torch.tensor(lengths)[n][:, None]
    ref.check(dx, (want, (ref.half_step(dtype) + 2.0**-23) * want.abs() + (2.0**-24 if dtype == F16 else 0)), "dx")


def test_pool_mean_of_padded_rows(he):
    x = rand(1, 5 * 12 + 3, 40, dtype=BF16)
    begin, end = i32(2, 14, 26, 38, 50), i32(2, 26, 30, 49, 51)
    keep = torch.zeros(63, dtype=torch.bool)
    for b, e in zip(begin.tolist(), end.tolist()):
        keep[b:e] = True
    y = x.clone()
    y[~keep.cuda()] = float("nan")
    got = he.pool_mean(y, (begin, end))
    ref.check(got, ref.pool_mean(x, (begin, end)), "e")
    de = rand(2, 5, 40)
    dx = he.pool_mean_backward(de, (begin, end), 63, BF16)
    assert not dx[~keep.cuda()].any() and dx[keep.cuda()].abs().min() > 0
    out = torch.full_like(dx, 3.0)
    he.pool_mean_backward(de, (begin, end), 63, BF16, out=out)
    assert (out[~keep.cuda()] == 3).all() and torch.equal(out[keep.cuda()], dx[keep.cuda()])


def test_pool_mean_of_more_rows_and_sequences_than_a_launch_holds(he):
    rows = (1 << 29) + 40  # tiles of 32 rows would take 2^32 threads
    de = torch.full((1, 1), float(rows), device="cuda")
    dx = he.pool_mean_backward(de, i32(0, rows), rows, BF16)
    assert dx.shape == (rows, 1) and (dx == 1).all()
    # Tiles sum up to 2^18 ones exactly, and eighths of them to 2^26 or 2^26 + 40 (a multiple of 8).  Joining the eighths takes seven roundings above
    # 2^26, the length in 32 bits is one and the quotient one: 9 * 2^-24.
    assert (he.pool_mean(dx, i32(0, rows)).double() - 1).abs() <= 9 * 2.0**-24
    del dx
    count = (1 << 22) + 9  # work-groups of 1024 threads would take 2^32 of them
    off = torch.full((count + 1,), 5, dtype=torch.int32, device="cuda")
    off[:count - 3] = 0  # sequence count - 4 has all rows
    x = rand(1, 5, 8)
    e = he.pool_mean(x, off)
    assert not e[:count - 4].any() and not e[count - 3:].any()
    assert (e[count - 4].double() - x.double().mean(0)).abs().max() <= 5 * 2.0**-24 * x.abs().max()
    want = e[count - 4].double() / 5  # one rounding of the quotient
    assert ((he.pool_mean_backward(e, off, 5, F32) - want).abs() <= 2.0**-24 * want.abs()).all()


def test_pool_mean_of_no_sequences_and_no_rows(he):
    x = rand(1, 5, 8)
    assert he.pool_mean(x, i32(0)).shape == (0, 8)
    assert not he.pool_mean_backward(torch.zeros(0, 8, device="cuda"), i32(0), 5, F32).any()
    assert not he.pool_mean(x[:0], i32(0, 0, 0)).any()
    assert he.pool_mean_backward(torch.zeros(2, 8, device="cuda"), i32(0, 0, 0), 0, F32).shape == (0, 8)


# ---- attention -----------------------------------------------------------------------------------------------------------


def attend(he, q, k, v, off, do, **kw):
    o, lse = he.attention(q, k, v, off, **kw)
    return dict(zip(("o", "lse", "dq", "dk", "dv"), (o, lse, *he.attention_backward(do, q, k, v, o, lse, off, **kw))))


def compare(he, q, k, v, off, do, **kw):
    want, got = ref.attention(q, k, v, off, do=do, **kw), attend(he, q, k, v, off, do, **kw)
    for name in got:
        ref.check(got[name], want[name], name)
    return got


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("dim", [8, 32, 40, 64, 72, 96, 128])
@pytest.mark.parametrize("lengths", [[1], [2], [31, 1, 0, 33], [32], [64, 65], [127, 129, 5], [300]])
def test_attention(he, lengths, dim, dtype):
    off = offsets_of(lengths)
    q, k, v, do = (rand(i, sum(lengths), 2, dim, dtype=dtype) for i in (1, 2, 3, 4))
    compare(he, q, k, v, off, do)


@pytest.mark.parametrize("dtype,heads,kv,dim,cap", [(BF16, 96, 48, 64, 0.0), (F16, 100, 100, 40, 0.0), (BF16, 8, 4, 64, 15.0), (F32, 3, 1, 96, 0.0), (F16, 5, 5, 128, 0.0)])
def test_attention_of_long_sequences(he, dtype, heads, kv, dim, cap):
    """Tiles of 256 queries (the first two) and of 128 queries and keys."""
    off = offsets_of([1100, 2061])
    q, do = rand(1, 3161, heads, dim, dtype=dtype), rand(2, 3161, heads, dim, dtype=dtype)
    k, v = rand(3, 3161, kv, dim, dtype=dtype), rand(4, 3161, kv, dim, dtype=dtype)
    slopes = 0.01 * torch.arange(heads).float().cuda() if cap else None
    want, got = ref.attention(q, k, v, off, do=do, cap=cap, slopes=slopes, device="cuda"), attend(he, q, k, v, off, do, cap=cap, slopes=slopes)
    for name in got:
        ref.check(got[name], want[name], name)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("cap,bias", [(0.0, True), (2.0, False), (30.0, True)])
@pytest.mark.parametrize("heads,kv", [(4, 4), (6, 2), (5, 1)])
def test_attention_with_caps_biases_and_shared_heads(he, heads, kv, cap, bias, dtype):
    off = offsets_of([70, 0, 1, 140])
    qkv, do = rand(1, 211, heads + 2 * kv, 64, dtype=dtype), rand(2, 211, heads, 64, dtype=dtype)
    slopes = 2.0 ** -torch.arange(1, heads + 1).float().cuda() if bias else None
    compare(he, qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:], off, do, cap=cap, slopes=slopes, scale=0.2)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("queries,keys", [([1] * 5, [700, 1, 0, 64, 33]), ([3, 0, 40], [1500, 20, 0]), ([1], [4000]), ([200], [3]), ([0, 2], [9, 1030])])
def test_attention_of_other_keys_and_few_queries(he, queries, keys, dtype):
    oq, ok = offsets_of(queries), offsets_of(keys)
    q, do = rand(1, sum(queries), 4, 64, dtype=dtype), rand(2, sum(queries), 4, 64, dtype=dtype)
    k, v = rand(3, sum(keys), 2, 64, dtype=dtype), rand(4, sum(keys), 2, 64, dtype=dtype)
    slopes = torch.tensor([0.5, 0.1, 0.01, 0.0], device="cuda")
    for sl in (None, slopes):
        compare(he, q, k, v, oq, do, offsets_k=ok, slopes=sl)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("lengths,heads,kv,dim", [([150, 0, 120], 32, 1, 32), ([300, 261], 8, 2, 64), ([230, 1, 410], 12, 2, 40), ([90], 96, 8, 128)])
def test_attention_gradients_of_cut_queries(he, lengths, heads, kv, dim, dtype):
    """Short sequences whose key heads are shared by many: the queries of a tile of 32 or 64 keys are cut into parts."""
    import ctypes
    import struct

    rows = sum(lengths)
    need, span = ctypes.c_size_t(), (64, 64, len(lengths), rows + 5)
    s = struct.Struct("@4iPPiqPPiqddPi4x").pack({F32: 0, F16: 1, BF16: 2}[dtype], heads, kv, dim, *span, *span, 1.0, 0.0, 0, 1)
    assert he.lib.he_attention_workspace_bytes(he.ctx, s, 1, ctypes.byref(need)) == 0 and need.value > 2 * 2 * kv * rows * dim * 4
    q, do = (rand(i, rows + 5, heads, dim, dtype=dtype) for i in (1, 4))
    k, v = (rand(i, rows + 5, kv, dim, dtype=dtype) for i in (2, 3))
    compare(he, q, k, v, offsets_of(lengths), do, slopes=torch.linspace(0.0, 0.1, heads, device="cuda"))


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("heads,kv,queries,keys", [(6, 2, [1, 1, 0, 3], [200, 0, 50, 33]), (8, 1, [4, 1, 2], [1, 129, 300]), (32, 1, [1, 1], [5, 2100]),
                                                   (33, 1, [1, 1], [40, 70]), (12, 4, [10, 20, 3, 7], [40, 128, 1, 500]), (4, 2, [1], [3000])])
def test_attention_of_few_queries_and_shared_heads(he, heads, kv, queries, keys, dtype):
    """Query heads that share a key head lie in one tile, some of which reach over a tile's end; of rows of no sequence as well."""
    off, off_k = np.cumsum([2] + queries).tolist(), offsets_of(keys)
    rows, sl = off[-1] + 3, torch.linspace(0.0, 0.2, heads, device="cuda")
    q, do = (rand(i, rows, heads, 32, dtype=dtype) for i in (1, 4))
    k, v = (rand(i, sum(keys), kv, 32, dtype=dtype) for i in (2, 3))
    for cap, slopes in ((0.0, None), (9.0, sl)):
        compare(he, q, k, v, (i32(*off[:-1]), i32(*off[1:])), do, offsets_k=off_k, cap=cap, slopes=slopes)
    out = torch.full_like(q, 7.0)
    he.attention(q, k, v, (i32(*off[:-1]), i32(*off[1:])), offsets_k=off_k, out=out)
    assert (out[:2] == 7).all() and (out[-3:] == 7).all() and not (out[2:-3] == 7).all()


@pytest.mark.parametrize("seed", range(24))
def test_attention_of_drawn_shapes(he, seed):
    """Types, heads, sizes, gaps between sequences, lengths of queries and keys, caps and biases as they come."""
    r = np.random.default_rng(seed)
    dtype, kv, group, dim = [F32, F16, BF16][seed % 3], int(r.integers(1, 4)), int(r.choice([1, 2, 4, 7])), 8 * int(r.integers(1, 17))
    gap, longest = int(r.choice([0, 0, 5])), int(r.choice([1, 8, 40, 150, 700]))

    def spans(n):
        at = np.cumsum(np.r_[r.integers(0, gap + 1), n + r.integers(0, gap + 1, len(n))])
        return (i32(*at[:-1].tolist()), i32(*(at[:-1] + n).tolist())), int(at[-1]) + gap

    nq = r.integers(0, longest + 1, r.integers(1, 13))
    (off, rows), (off_k, rows_k) = spans(nq), spans(r.integers(0, r.choice([4, 60, 900]), len(nq)))
    if r.random() < 0.5:
        off_k, rows_k = off, rows
    q, do = (rand(i, rows, kv * group, dim, dtype=dtype) for i in (1, 4))
    k, v = (rand(i, rows_k, kv, dim, dtype=dtype) for i in (2, 3))
    slopes = None if r.random() < 0.5 else 0.3 * torch.rand(kv * group, device="cuda", generator=torch.Generator("cuda").manual_seed(seed))
    compare(he, q, k, v, off, do, offsets_k=off_k, cap=float(r.choice([0.0, 8.0])), slopes=slopes)


def test_attention_is_cut_where_it_should_be(he):
    """Sizes that test_attention_of_other_keys_and_few_queries (one query of many keys) and test_attention_of_long_sequences (few tiles of keys under many
    queries) run really are cut and joined."""
    import ctypes
    import struct

    need = ctypes.c_size_t()
    attn = struct.Struct("@4iPPiqPPiqddPi4x").pack  # he_attn
    sq, sk = (64, 64, 1, 1), (64, 64, 1, 4000)  # begin, end (only their count is looked at), count, rows
    s = attn(2, 4, 2, 64, *sq, *sk, 0.125, 0.0, 0, 1)
    assert he.lib.he_attention_workspace_bytes(he.ctx, s, 0, ctypes.byref(need)) == 0 and need.value > 0
    both = (64, 64, 2, 3161)
    s = attn(2, 8, 4, 64, *both, *both, 0.125, 15.0, 0, 1)
    assert he.lib.he_attention_workspace_bytes(he.ctx, s, 1, ctypes.byref(need)) == 0 and need.value > 2 * 2 * 4 * 3161 * 64 * 4


def test_attention_scores_far_from_zero(he):
    """Scores of +-200 and maxima that rise from tile to tile: the running maximum moves, and nothing overflows."""
    for dtype in (F16, BF16):
        q = rand(1, 260, 2, 64, dtype=dtype)
        k = q * torch.linspace(-8, 24, 260, device="cuda").view(-1, 1, 1).to(dtype)
        compare(he, q, k, rand(2, 260, 2, 64, dtype=dtype), i32(0, 260), rand(3, 260, 2, 64, dtype=dtype))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_of_a_padded_batch(he, dtype):
    """Rows of no sequence may hold anything: they reach no other row, and get zeros, or stay as they were in buffers of the caller's."""
    begin, end = i32(3, 53, 103, 153), i32(40, 53, 150, 154)
    rows, keep = 210, torch.zeros(210, dtype=torch.bool)
    for b, e in zip(begin.tolist(), end.tolist()):
        keep[b:e] = True
    gone = ~keep.cuda()
    q, k, v, do = (rand(i, rows, 4, 64, dtype=dtype) for i in (1, 2, 3, 4))
    want = ref.attention(q, k, v, (begin, end), do=do)
    for i, t in enumerate((q, k, v, do)):
        t[gone] = (float("nan"), float("inf"), float("nan"), float("-inf"))[i]
    got = attend(he, q, k, v, (begin, end), do)
    for name in got:
        ref.check(got[name], want[name], name)
        assert name == "lse" or not got[name][gone].any(), name
    out = torch.full((rows, 3, 4, 64), 5.0, dtype=dtype, device="cuda")
    o, lse = he.attention(q, k, v, (begin, end), out=out[:, 1])
    assert (out[gone] == 5).all() and torch.equal(o[~gone], got["o"][~gone]) and torch.equal(lse, got["lse"])
    grads = he.attention_backward(do, q, k, v, got["o"], lse, (begin, end), out=[out[:, i] for i in range(3)])
    assert (out[gone] == 5).all()
    for name, g in zip(("dq", "dk", "dv"), grads):
        assert torch.equal(g[~gone], got[name][~gone]), name


def test_attention_keeps_sequences_apart(he):
    """NaN and infinities of one sentence stay in it."""
    off = offsets_of([20, 44, 30, 128, 1])
    q, k, v, do = (rand(i, 223, 2, 64, dtype=BF16) for i in (1, 2, 3, 4))
    a = attend(he, q, k, v, off, do)
    k[25], v[30], q[40], do[50], v[100] = float("nan"), float("inf"), float("-inf"), float("nan"), float("nan")
    b = attend(he, q, k, v, off, do)
    mine = torch.zeros(223, dtype=torch.bool, device="cuda")
    mine[20:64] = mine[94:222] = True
    for name in a:
        u, w = (a[name].t(), b[name].t()) if name == "lse" else (a[name], b[name])
        assert torch.equal(u[~mine], w[~mine]), name


def test_attention_of_rows_behind_the_last_sequence(he):
    off = i32(4, 30, 50)  # rows before the first and behind the last sequence
    q, k, v, do = (rand(i, 400, 2, 32, dtype=F16) for i in (1, 2, 3, 4))
    compare(he, q, k, v, off, do)


def test_attention_of_no_sequences(he):
    q = rand(1, 6, 2, 32)
    o, lse = he.attention(q, q, q, i32(0))
    assert not o.any() and (lse == float("-inf")).all()
    assert not any(g.any() for g in he.attention_backward(q, q, q, q, o, lse, i32(0)))
    e = q[:0]
    o, lse = he.attention(e, e, e, i32(0, 0))
    assert o.shape == (0, 2, 32) and lse.shape == (2, 0)
    o, lse = he.attention(q, e, e, i32(0, 6), offsets_k=i32(0, 0))
    assert not o.any() and (lse == float("-inf")).all()
    dq, dk, dv = he.attention_backward(q, q, e, e, o, lse, i32(0, 6), offsets_k=i32(0, 0))
    assert not dq.any() and dk.shape == dv.shape == (0, 2, 32)


def test_attention_of_many_sequences(he):
    """More sequences than a wave has lanes, and than its square: the search of a tile's sequence takes several steps."""
    for count in (65, 5000):
        n = np.random.default_rng(count).integers(0, 4, count)
        n[0], n[7], n[-1] = 0, 40, 0
        off = offsets_of(n)
        q, k, v, do = (rand(i, int(n.sum()), 1, 16, dtype=F32) for i in (1, 2, 3, 4))
        compare(he, q, k, v, off, do)


def test_attention_offsets_that_break_the_rule_stay_in_the_buffers(he):
    q = rand(1, 64, 2, 32, dtype=BF16)
    for off in (i32(0, 500, 64), i32(-9, 30, 64), i32(0, 40, 10, 64), (i32(10, 0), i32(5, 100))):
        o, lse = he.attention(q, q, q, off)
        he.attention_backward(q, q, q, q, o, lse, off)
        he.pool_mean(q.view(64, 64), off)
        he.pool_mean_backward(torch.ones(len(off[0]) if isinstance(off, tuple) else len(off) - 1, 64, device="cuda"), off, 64, BF16)
    torch.cuda.synchronize()


def test_attention_far_into_a_long_buffer(he):
    """Row offsets in elements that pass 32 bits."""
    rows = (1 << 31) // (40 * 128) + 300
    buf = torch.zeros(rows, 40, 128, dtype=BF16, device="cuda")
    buf[-200:] = rand(1, 200, 40, 128, dtype=BF16)
    q, k, v = buf[:, 38:], buf[:, 36:38], buf[:, 34:36]
    off = (i32(0, rows - 150), i32(3, rows - 2))
    o, lse = he.attention(q, k, v, off)
    do = buf[:, 32:34]
    dq, dk, dv = he.attention_backward(do, q, k, v, o, lse, off)
    tail = slice(rows - 150, rows - 2)
    want = ref.attention(q[tail], k[tail], v[tail], i32(0, 148), do=do[tail])
    for name, got in (("o", o), ("dq", dq), ("dk", dk), ("dv", dv)):
        ref.check(got[tail], want[name], name)
        assert not got[rows - 2:].any()


def test_attention_repeats_bit_for_bit(he):
    off = offsets_of([500, 300, 77])
    q, k, v, do = (rand(i, 877, 6, 64, dtype=BF16) for i in (1, 2, 3, 4))
    a, b = attend(he, q, k, v, off, do), attend(he, q, k, v, off, do)
    assert all(torch.equal(a[n], b[n]) for n in a)


def test_refusals_on_the_device(he):
    x = rand(1, 8, 2, 32, dtype=BF16)
    off = i32(0, 8)
    for f in (lambda: he.attention(x, x, x[:, :, :24], off), lambda: he.attention(x, x[:4], x[:4], off), lambda: he.attention(x, x.half(), x, off),
              lambda: he.attention(x, x, x, off.long()), lambda: he.attention(x, x, x, off.cpu()), lambda: he.attention(x[:, :, 1:25], x, x, off),
              lambda: he.attention(x, x, x, off, offsets_k=i32(0, 4, 8)), lambda: he.attention(x, x, x, off, slopes=torch.ones(3, device="cuda")),
              lambda: he.attention(x, x, x, off, out=x.float()), lambda: he.attention(x.double(), x.double(), x.double(), off),
              lambda: he.attention_backward(x, x, x, x, x, torch.zeros(8, 2, device="cuda"), off),
              lambda: he.pool_mean(x[:, 0], off, out=torch.zeros(1, 31, device="cuda")), lambda: he.pool_mean_backward(x[:1, 0], off, 8, BF16),
              lambda: he.layer_norm(x[:, 0], rand(1, 31), rand(2, 31)), lambda: he.layer_norm(x[:, 0], rand(1, 32), rand(2, 32, dtype=BF16)),
              lambda: he.layer_norm(x[:, 0], rand(1, 32), rand(2, 32), residual=x[:4, 0])):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: he.attention(x, x, x, off, scale=0.0), lambda: he.attention(x, x, x, off, cap=-1.0), lambda: he.layer_norm(x[:, 0], rand(1, 32), rand(2, 32), eps=-1.0),
              lambda: he.layer_norm(x[:, 0], rand(1, 32, dtype=F16), rand(2, 32, dtype=F16)), lambda: he.attention(x, x, x, off, out=x[:1].expand(8, 2, 32))):
        with pytest.raises(pkg.HeError, match="EINVAL"):
            f()


# ---- streams, graphs, together -----------------------------------------------------------------------------------------------


def _everything(he, x, r, w, b, qkv, do, off, de):
    y, s, mean, rstd = he.layer_norm(x, w, b, residual=r)
    o, lse = he.attention(qkv[:, :4], qkv[:, 4:6], qkv[:, 6:], off, cap=20.0)
    one = he.attention(qkv[:1, :4], qkv[:, 4:6], qkv[:, 6:], off[:2], offsets_k=off[::4].contiguous())[0]  # a lone query of all keys: cut and joined
    e = he.pool_mean(y, off)
    return (y, s, o, lse, one, e, *he.layer_norm_backward(x, s, w, mean, rstd, ds=r),
            *he.attention_backward(do, qkv[:, :4], qkv[:, 4:6], qkv[:, 6:], o, lse, off, cap=20.0), he.pool_mean_backward(de, off, x.shape[0], x.dtype))


def _inputs(seed):
    off = offsets_of([1, 600, 0, 1400])
    return (rand(seed, 2001, 64, dtype=BF16), rand(seed + 1, 2001, 64, dtype=BF16), rand(seed + 2, 64), rand(seed + 3, 64), rand(seed + 4, 2001, 8, 64, dtype=BF16),
            rand(seed + 5, 2001, 4, 64, dtype=BF16), off, rand(seed + 6, 4, 64))


def test_two_streams_at_once(he):
    ins = [_inputs(10), _inputs(20)]
    want = [[t.clone() for t in _everything(he, *i)] for i in ins]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [None, None]
    for rep in range(3):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                got[k] = _everything(he, *ins[k])
        torch.cuda.synchronize()
        for k in range(2):
            assert all(torch.equal(a, b) for a, b in zip(got[k], want[k])), (rep, k)


def test_two_captured_graphs(he):
    """Two graphs captured on one stream and replayed on two at once: neither shares a workspace with the other; inputs change between replays."""
    ins = [_inputs(30), _inputs(40)]
    fresh = [_inputs(50), _inputs(60)]
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


def _plain_encoder(layers, x, off, heads, pool):
    """The encoder in 64 bits by torch's differentiable elementary operations."""
    x = x.double()
    norm = lambda t, w, b: (t - t.mean(1, keepdim=True)) * (t.var(1, unbiased=False, keepdim=True) + 1e-5).rsqrt() * w + b  # noqa: E731
    o = off.tolist()
    for w in layers:
        w = {k: v.double() if not v.requires_grad or v.dtype != torch.float64 else v for k, v in w.items()}
        d = x.shape[1] // heads
        qkv = (x @ w["qkv"].T + w["qkv_bias"]).view(-1, 3 * heads, d)
        rows = []
        for b, e in zip(o[:-1], o[1:]):
            q, k, v = (qkv[b:e, i * heads:(i + 1) * heads].transpose(0, 1) for i in range(3))
            rows.append((torch.softmax(q @ k.transpose(1, 2) * d**-0.5, -1) @ v).transpose(0, 1).flatten(1))
        x = norm(x + torch.cat(rows) @ w["out"].T + w["out_bias"], w["norm1"], w["norm1_bias"])
        f = torch.nn.functional.gelu(x @ w["up"].T + w["up_bias"]) @ w["down"].T + w["down_bias"]
        x = norm(x + f, w["norm2"], w["norm2_bias"])
    if pool == "mean":
        return torch.stack([x[b:e].mean(0) if e > b else x[:1].sum(0) * 0 for b, e in zip(o[:-1], o[1:])])
    return torch.stack([x[b] if e > b else x[:1].sum(0) * 0 for b, e in zip(o[:-1], o[1:])])


@pytest.mark.parametrize("pool", ["mean", "first"])
def test_encoder_and_its_gradients(he, pool):
    """All operators together in 32 bits.  Errors of single operations are near 2^-24 of their operands, a few hundred of them follow one another
    over two layers, norms multiply by at most rstd ~ 1: 2^-14 of the largest element is granted."""
    from paper_2210_02574_amd.embedding import SentenceEncoder

    layers = [SentenceEncoder.random_layer(64, 2, 96, 5 + i, F32, "cuda", std=0.1) for i in range(2)]
    states, off, de = rand(1, 60, 64), offsets_of([20, 0, 1, 39]), rand(2, 4, 64)
    leaves = [states] + [v for w in layers for v in w.values()]
    for t in leaves:
        t.requires_grad_(True)
    e = SentenceEncoder(he, layers, 2, pool=pool)(states, off)
    got = torch.autograd.grad(e, leaves, de, allow_unused=True)
    plain = _plain_encoder(layers, states, off, 2, pool)
    want = torch.autograd.grad(plain, leaves, de.double(), allow_unused=True)
    assert e.dtype == F32 and (e - plain).abs().max() <= 2.0**-14 * plain.abs().max()
    for g, w in zip(got, want):
        assert (g is None) == (w is None)
        if w is not None:
            assert (g - w).abs().max() <= 2.0**-14 * max(1.0, float(w.abs().max())), g.shape


def test_gradients_against_differences(he):
    """The differentiable functions in 32 bits along random directions: central differences with step h are off by h^2 and by 2^-24 |f| / h."""
    from paper_2210_02574_amd.embedding import attention, layer_norm, pool_mean

    off = offsets_of([9, 30])
    x = [rand(i, 39, 128) for i in (1, 2)] + [rand(3, 128), rand(4, 128)]
    c = rand(5, 2, 128).double()
    sl = torch.tensor([0.1, 0.02, 0.3, 0.0], device="cuda")

    def f(x, r, w, b):
        y, s = layer_norm(he, x, w, b, residual=r)
        o = attention(he, y.view(39, 4, 32), s.view(39, 4, 32)[:, :2], y.view(39, 4, 32)[:, 2:], off, cap=3.0, slopes=sl)
        return (pool_mean(he, o.flatten(1), off).double() * c).sum()

    leaves = [t.requires_grad_(True) for t in x]
    grads = torch.autograd.grad(f(*leaves), leaves)
    h = 2.0**-7
    for i in range(4):
        d = rand(10 + i, *x[i].shape)
        d = d / d.norm()
        with torch.no_grad():
            a = [t + h * d if j == i else t for j, t in enumerate(x)]
            b = [t - h * d if j == i else t for j, t in enumerate(x)]
            diff = float(f(*a) - f(*b)) / (2 * h)
        want = float((grads[i] * d).sum())
        assert abs(diff - want) < 2.0**-11 * (1 + float(grads[i].norm())), (i, diff, want)


def test_gradients_of_no_sentences_are_zeros(he):
    from paper_2210_02574_amd.embedding import SentenceEncoder

    layer, x = SentenceEncoder.random_layer(64, 2, 96, 5, F32, "cuda"), rand(1, 6, 64).requires_grad_(True)
    torch.full((6 * 384,), float("nan"), device="cuda")  # what memory that is not written may hold
    layer["qkv"].requires_grad_(True)
    e = SentenceEncoder(he, [layer], 2)(x, i32(0))
    assert e.shape == (0, 64)
    e.sum().backward()
    assert not x.grad.any() and not layer["qkv"].grad.any()
    d = [torch.full((6, 2, 32), float("nan"), device="cuda") for _ in range(3)]
    q = rand(2, 6, 2, 32)
    o, lse = he.attention(q, q, q, i32(0))
    he.attention_backward(q, q, q, q, o, lse, i32(0), out=d, fill=True)
    assert not any(t.any() for t in d)


def test_refusals_of_the_differentiable_functions(he):
    """A second derivative, and offsets that are written between the two passes."""
    from paper_2210_02574_amd.embedding import attention, layer_norm, pool_mean

    w = torch.ones(64, device="cuda")
    fns = (lambda x, o: layer_norm(he, x, w, w)[0], lambda x, o: attention(he, *[x.view(6, 2, 32)] * 3, o), lambda x, o: pool_mean(he, x, o),
           lambda x, o: attention(he, *[x.view(6, 2, 32)] * 3, (o[:1], o[1:]), offsets_k=(o[:1], o[1:])))
    for k, f in enumerate(fns):
        off, x = i32(0, 6), rand(1, 6, 64).requires_grad_(True)
        g, = torch.autograd.grad(f(x, off).square().sum(), x, create_graph=True)
        with pytest.raises(RuntimeError, match="once_differentiable"):
            g.sum().backward()
        y = f(x, off).square().sum()
        off[0] = 1
        if k:
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                y.backward()


def test_sentences_to_encrypted_logits(he):
    """The whole path: token states -> embeddings -> packed, encrypted -> encrypted classifier -> logits, against the same in the clear."""
    from paper_2210_02574_amd.classifier import EncryptedInference, logits_from_slots
    from paper_2210_02574_amd.embedding import SentenceEncoder

    layers = [SentenceEncoder.random_layer(768, 12, 1024, 7 + i, BF16, "cuda") for i in range(2)]
    enc = SentenceEncoder(he, layers, 12)
    lengths = [17, 1, 64]  # three sentences: two to a ciphertext of this ring, and one filled up
    states, off = rand(9, sum(lengths), 768, dtype=BF16), offsets_of(lengths)
    W = wl.weights(11)
    level, scale = 3, 2.0**30
    inf = EncryptedInference(he, level)
    sk = he.keygen_secret(12)
    keys = inf.make_keys(sk, 13)
    cts = inf.encrypt_sentences(sk, enc, states, off, scale, 14)
    assert len(cts) == 2
    e = enc(states, off).double().cpu().numpy()
    pts = inf.encode_weights(W)
    got = np.concatenate([logits_from_slots(he.decrypt(sk, he.to_host(inf.run(ct, pts, keys)), scale)) for ct in cts])
    assert np.abs(got[:3] - e @ W.T).max() < 2.0**-8  # scale 2^30 on the smallest ring
    assert np.abs(got[3]).max() < 2.0**-8
