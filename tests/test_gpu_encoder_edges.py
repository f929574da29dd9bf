"""The operators on token states on the GPU at the edge of what is documented: first calls of several threads, large caps, weights and gradients at
the ends of a type's range, buffers that autograd holds."""
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


def test_a_context_knows_its_stream_before_it_says_that_it_is_ready():
    """A second thread that finds the extension in place calls at once: its kernels belong on its own current stream then."""
    streams = []

    class Watched(pkg.HE):
        def __setattr__(self, name, value):
            if name == "_tensors" and value is not None:
                streams.append(self._raw_stream(0))
            super().__setattr__(name, value)

    he, side, x = Watched.from_params(wl.C1B, device=0), torch.cuda.Stream(), rand(1, 3, 8)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        he.pool_mean(x, i32(0, 3))
    torch.cuda.synchronize()
    assert streams == [side.cuda_stream]


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("cap", [1e3, 1e5, 1e8, 1e30])
@pytest.mark.parametrize("lengths,heads,kv,bias", [([40, 0, 130], 4, 2, True), ([1100], 16, 8, False), ([700, 460], 12, 12, True)])
def test_attention_under_caps_that_scores_never_reach(he, lengths, heads, kv, bias, cap, dtype):
    """A cap far above the scores changes nothing, so what is granted is what is granted without one."""
    off, rows = offsets_of(lengths), sum(lengths)
    q, do = rand(1, rows, heads, 64, dtype=dtype, scale=2.0), rand(4, rows, heads, 64, dtype=dtype)
    k, v = (rand(i, rows, kv, 64, dtype=dtype) for i in (2, 3))
    slopes = torch.linspace(0.0, 0.1, heads, device="cuda") if bias else None
    free = ref.attention(q, k, v, off, do=do, slopes=slopes, device="cuda")
    want = ref.attention(q, k, v, off, do=do, slopes=slopes, cap=cap, device="cuda")
    o, lse = he.attention(q, k, v, off, cap=cap, slopes=slopes)
    grads = he.attention_backward(do, q, k, v, o, lse, off, cap=cap, slopes=slopes)
    for name, got in zip(("o", "lse", "dq", "dk", "dv"), (o, lse, *grads)):
        ref.check(got, (want[name][0], free[name][1]), name)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("cap", [63.0, 64.0, 65.0, 200.0])
def test_attention_under_caps_on_both_sides_of_the_rule(he, cap, dtype):
    """Scores that reach the cap, on both sides of 64, where the tanh is made in another way."""
    off = offsets_of([90, 1, 300])
    q, do = rand(1, 391, 4, 64, dtype=dtype, scale=60.0), rand(4, 391, 4, 64, dtype=dtype)
    k, v = (rand(i, 391, 2, 64, dtype=dtype) for i in (2, 3))
    want = ref.attention(q, k, v, off, do=do, cap=cap, device="cuda")
    o, lse = he.attention(q, k, v, off, cap=cap)
    for name, got in zip(("o", "lse", "dq", "dk", "dv"), (o, lse, *he.attention_backward(do, q, k, v, o, lse, off, cap=cap))):
        ref.check(got, want[name], name)


@pytest.mark.parametrize("seqs,queries,keys", [(1, 1100, 60000), (20, 20, 3000)])
def test_fp16_weights_far_below_the_largest(he, seqs, queries, keys):
    """One key's weight is 2^25.2 times each of the others', which alone carry a value.  A weight is held down to 2^-31 of the largest, so it is off by 2^-32 of
    that at most."""
    u, heads = 2.0**-11, 16
    k, v = torch.zeros(seqs * keys, 1, 8, dtype=F16, device="cuda"), torch.ones(seqs * keys, 1, 8, dtype=F16, device="cuda")
    k[..., 0] = -17.46875
    k[::keys] = 0
    v[::keys] = 0
    q = torch.zeros(seqs * queries, heads, 8, dtype=F16, device="cuda")
    q[..., 0] = 1
    at = torch.arange(seqs + 1, dtype=torch.int32, device="cuda")
    o, _ = he.attention(q, k.expand(-1, heads, 8), v.expand(-1, heads, 8), at * queries, offsets_k=at * keys, scale=1.0)
    w = (keys - 1) * np.exp(-17.46875)
    p = w / (1 + w)
    e = 16 * ref.F32 * 17.5 + 4 * ref.F32 * 17.5 + 2.0**-22
    assert (o.double() - p).abs().max() <= (u + 2 * e + 2.0**-14) * p + keys * 2.0**-32 + u * p


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("seqs,queries,keys", [(1, 1100, 60000), (20, 20, 3000)])
def test_sums_of_many_small_weights(he, seqs, queries, keys, dtype):
    """The same weights: each is too small to change a sum in 32 bits of which the largest is a part.  A lane's sum takes eight at a time and meets half of the
    keys or fewer, so it is off by half a step, 2^-24 below 2, keys / 16 times.  2^-20: two steps of a logarithm below 8, fp16's lift."""
    k = torch.zeros(seqs * keys, 1, 8, dtype=dtype, device="cuda")
    k[..., 0] = -17.5
    k[::keys] = 0
    q = torch.zeros(seqs * queries, 16, 8, dtype=dtype, device="cuda")
    q[..., 0] = 1
    at = torch.arange(seqs + 1, dtype=torch.int32, device="cuda")
    lse = he.attention(q, k.expand(-1, 16, 8), k.expand(-1, 16, 8), at * queries, offsets_k=at * keys, scale=1.0)[1]
    e = 16 * ref.F32 * 17.5 + 4 * ref.F32 * 17.5 + 2.0**-22
    w = (keys - 1) * np.exp(-17.5)
    assert (lse.double() - np.log1p(w)).abs().max() <= 2 * e * w + 2.0**-20 + keys / 16 * 2.0**-24


def _gradients(q, k, v, do, scale):
    """{name: (value, bound)} of dq, dk and dv of one sequence with one head, [rows][dim] each, in 64 bits on the device.  As encoder_reference has them, but
    for what a factor of small size is off by: with G and V the largest norms of a row of do and of v, ds is at most G V / 2, and is lifted by a power of
    two that brings this to 2^14 or more; p is lifted by 2^12.  So half a step of fp16, 2^-25, is 2^-40 G V of a ds and 2^-37 of a p.  A result's own
    half step is 2^-25."""
    u, f = 2.0**-11, ref.F32
    q, k, v, do = (t.double() for t in (q, k, v, do))
    d = q.shape[1]
    t, t_abs = scale * q @ k.T, scale * q.abs() @ k.abs().T
    e = ((d + 8) * f * t_abs + 4 * f * t.abs()).amax(1, keepdim=True) + 2.0**-22
    p = torch.softmax(t, 1)
    del t, t_abs
    rel = u + 2 * e + 2.0**-14
    o, dp = p @ v, do @ v.T
    ob = (rel * p) @ v.abs() + u * o.abs()
    size = do.abs() @ v.abs().T + (do * o).abs().sum(1, keepdim=True)
    db = (do.abs() * ob).sum(1, keepdim=True) + (d + 8) * f * size
    dt = p * (dp - (do * o).sum(1, keepdim=True)) * scale
    most = float(do.norm(dim=1).max() * v.norm(dim=1).max())
    te = rel * dt.abs() + p * db * scale + 2.0**-40 * most * scale
    out = {"dq": (dt @ k, te @ k.abs()), "dk": (dt.T @ q, te.T @ q.abs()), "dv": (p.T @ do, (rel * p + 2.0**-37).T @ do.abs())}
    return {n: (a.cpu(), (b + u * a.abs() + 2.0**-25).cpu()) for n, (a, b) in out.items()}


def _check_gradients(he, q, k, v, do, scale, cap=0.0):
    q, k, v, do = (t.to(F16).contiguous() for t in (q, k, v, do))
    args = [t[:, None] for t in (q, k, v)]
    extra = {"offsets_k": i32(0, len(k)), "scale": scale, "cap": cap}
    o, lse = he.attention(*args, i32(0, len(q)), **extra)
    got = he.attention_backward(do[:, None], *args, o, lse, i32(0, len(q)), **extra)
    want = _gradients(q, k, v, do, scale)
    for name, g in zip(("dq", "dk", "dv"), got):
        ref.check(g[:, 0], want[name], name)


def test_fp16_gradients_of_long_rows_with_equal_weights(he):
    """Weights of 1 / 166940: 100.5 of fp16's smallest steps, so that each of them rounds the same way by 2^-7.7 of itself."""
    n, ones = 166940, torch.ones(8, device="cuda")
    s = torch.ones(n, 1, device="cuda")
    s[1::2] = -1
    r = s[:512]
    _check_gradients(he, 0 * r * ones, s * 2.0**-12 * ones, s * ones, 0.125 * ones.expand(512, 8), 8**-0.5)  # dv and dq
    _check_gradients(he, 8 * r * ones, s * 2.0**-12 * ones, s * ones, 0.125 * r * ones, 8**-0.5)  # dk and dq


@pytest.mark.parametrize("size", [2.0**-12, 1.0, 2.0**10])
@pytest.mark.parametrize("cap", [0.0, 1e6])
def test_fp16_gradients_of_long_rows_and_of_any_size(he, size, cap):
    """Gradients whose terms are below fp16's smallest number, and large ones."""
    q, do = rand(1, 300, 64), rand(2, 300, 64, scale=size)
    k, v = rand(3, 20000, 64), rand(4, 20000, 64)
    _check_gradients(he, q, k, v, do, 0.125, cap)


@pytest.mark.parametrize("keys", [2, 40, 700])
def test_fp16_gradients_near_the_largest_number(he, keys):
    """ds passes 65504, dq, dk and dv do not."""
    s = torch.ones(keys, 1, device="cuda")
    s[1::2] = -1
    ones = torch.ones(64, device="cuda")
    r = torch.ones(30, 1, device="cuda")
    r[1::2] = -1
    q, do = 2.0**-9 * r * ones, 30000 * r * ones  # a dp of 1.9e6
    do[3] = 2.0**-10
    _check_gradients(he, q, s * 2.0**-4 * ones, s * ones, do, 0.125)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("cap,lengths,heads,kv,dim", [(0.0, [20, 333, 1, 200], 4, 2, 64), (25.0, [20, 333, 1, 200], 4, 2, 64), (1e4, [700], 3, 3, 32), (0.0, [1500, 90], 6, 2, 128)])
def test_biased_gradients_do_not_depend_on_how_o_was_rounded(he, cap, lengths, heads, kv, dim, dtype):
    """Values with a large part in common: dp - delta is small beside both.  o is rounded to 16 bits, delta must not be.  Bounds as in encoder_reference without
    that rounding; what takes its place is the sum p (dp - delta), off by 2 e + 2^-14 of its terms (weights and 4096 additions at most), and the
    mean that it is multiplied with, off by u of a correction of |do| |o| u."""
    u, f, off = ref.half_step(dtype), ref.F32, offsets_of(lengths)
    rows = sum(lengths)
    q, do = rand(1, rows, heads, dim, dtype=dtype), rand(2, rows, heads, dim, dtype=dtype)
    k, v = rand(3, rows, kv, dim, dtype=dtype), (16 + rand(4, rows, kv, dim)).to(dtype)
    slopes = 2.0 ** -torch.arange(1, heads + 1).float().cuda()
    o, lse = he.attention(q, k, v, off, cap=cap, slopes=slopes)
    dq, dk, _ = he.attention_backward(do, q, k, v, o, lse, off, cap=cap, slopes=slopes)
    scale, at = dim**-0.5, np.cumsum([0] + lengths)
    want_k, bound_k = (torch.zeros(rows, kv, dim, dtype=torch.float64, device="cuda") for _ in range(2))
    for b, e in zip(at[:-1], at[1:]):
        dist = (torch.arange(e - b, device="cuda")[:, None] - torch.arange(e - b, device="cuda")[None]).abs().double()
        for i in range(heads):
            c = i // (heads // kv)
            Q, K, V, G = (t.double() for t in (q[b:e, i], k[b:e, c], v[b:e, c], do[b:e, i]))
            t, err = scale * Q @ K.T, (dim + 8) * f * scale * Q.abs() @ K.abs().T
            th = torch.zeros_like(t)
            if cap:
                th = torch.tanh(t / cap)
                t, err = cap * th, err + 2 * 2.0**-23 * min(cap, 64)
            t = t - float(slopes[i]) * dist
            err = (err + 4 * f * t.abs()).amax(1, keepdim=True) + 2.0**-22
            p = torch.softmax(t, 1)
            slope = 1 - th**2
            dp, size = G @ V.T, G.abs() @ V.abs().T
            d = dp - (p * dp).sum(1, keepdim=True)
            rounded = u * u * (G.abs() * (p @ V).abs()).sum(1, keepdim=True)
            db = (dim + 8) * f * 2 * size + (2 * err + 2.0**-14) * (p * d.abs()).sum(1, keepdim=True) + 2 * rounded
            dt = p * d * slope * scale
            te = (u + 2 * err + 2.0**-14) * dt.abs() + p * db * slope * scale
            if cap:
                te = te + (p * d).abs() * scale * 2 * (2.0**-22 + err / cap)
            ref.check(dq[b:e, i], ((dt @ K).cpu(), (te @ K.abs() + u * (dt @ K).abs() + 2.0**-25).cpu()), f"dq of head {i}")
            want_k[b:e, c] += dt.T @ Q
            bound_k[b:e, c] += te.T @ Q.abs()
    ref.check(dk, (want_k.cpu(), (bound_k + u * want_k.abs() + 2.0**-25).cpu()), "dk")


def test_gradients_that_begin_between_two_vectors(he):
    """The gradient that reaches the operator is what the program behind it makes: here a part of a longer buffer, at no multiple of 16 bytes."""
    from paper_2210_02574_amd.embedding import _SelfAttention, attention

    off = i32(0, 9, 20)
    for dtype in (BF16, F32):
        x = rand(1, 20, 6, 32, dtype=dtype).requires_grad_(True)
        one, g = rand(2, 1, dtype=dtype), rand(3, 1 + 20 * 2 * 32, dtype=dtype)
        for f in (lambda: attention(he, x[:, :2], x[:, 2:4], x[:, 4:], off), lambda: _SelfAttention.apply(he, x, 2, off, 0.0, None)):
            got, = torch.autograd.grad(torch.cat([one, f().flatten()]), x, g)
            want, = torch.autograd.grad(f().flatten(), x, g[1:].clone())
            assert torch.equal(got, want)


def _written(he):
    """Every call that takes buffers to write to: (the call, what its buffers are like)."""
    off, x, w = i32(0, 3, 8), rand(1, 8, 2, 32), rand(2, 64)
    o, lse = he.attention(x, x, x, off)
    rows = x.view(8, 64)
    return [(lambda out: he.layer_norm(rows, w, w, out=out[0]), [rows]), (lambda out: he.pool_mean(rows, off, out=out[0]), [rows[:2]]),
            (lambda out: he.pool_mean_backward(rows[:2], off, 8, F32, out=out[0]), [rows]), (lambda out: he.attention(x, x, x, off, out=out[0]), [x]),
            (lambda out: he.attention_backward(x, x, x, x, o, lse, off, out=out), [x, x, x])]


@pytest.mark.parametrize("call", range(5))
def test_autograd_notices_buffers_that_are_written(he, call):
    f, like = _written(he)[call]
    for i in range(len(like)):
        out, x = [torch.ones_like(t) for t in like], torch.ones_like(like[i], requires_grad=True)
        y = (x * out[i]).sum()  # keeps out[i] for its gradient
        f(out)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()
    with torch.inference_mode():
        f([torch.ones_like(t) for t in like])  # tensors without a version


@pytest.mark.parametrize("call", range(5))
def test_buffers_that_autograd_tracks_are_refused(he, call):
    f, like = _written(he)[call]
    for i in range(len(like)):
        out = [torch.ones_like(t) for t in like]
        out[i].requires_grad_(True)
        with pytest.raises(ValueError, match="require gradients"):
            f(out)
        with torch.no_grad():
            f(out)  # as torch's own writing operations have it


def test_buffers_that_overlap_are_refused(he):
    off, buf = i32(0, 3, 8), rand(1, 4096)
    rows, w = buf[:512].view(8, 64), rand(2, 64)
    x = buf[:512].view(8, 2, 32)
    o, lse = he.attention(x, x, x, off)
    joint = rand(3, 8, 6, 32)
    cut = lambda *at: [joint[:, a:a + 2] for a in at]  # noqa: E731
    for f in (lambda: he.layer_norm(rows, w, w, out=rows), lambda: he.layer_norm(rows, w, w, out=buf[32:544].view(8, 64)),
              lambda: he.layer_norm(rows[:, :32], w[:32], w[:32], residual=rows[:, 32:], out=buf[16:528].view(8, 64)[:, :32]),
              lambda: he.layer_norm(rows, buf[1024:1088], w, out=buf[1000:1512].view(8, 64)), lambda: he.pool_mean(rows, off, out=buf[64:192].view(2, 64)),
              lambda: he.pool_mean_backward(buf[:128].view(2, 64), off, 8, F32, out=rows), lambda: he.attention(x, x, x, off, out=x),
              lambda: he.attention(x, x, x, off, out=buf[256:768].view(2, 8, 32).transpose(0, 1)), lambda: he.attention(x, joint[:, :2], joint[:, 2:4], off, out=joint[:, 1:3]),
              lambda: he.attention_backward(x, x, x, x, o, lse, off, out=cut(0, 1, 4)), lambda: he.attention_backward(x, x, x, x, o, lse, off, out=cut(0, 2, 3)),
              lambda: he.attention_backward(x, *cut(0, 2, 4), o, lse, off, out=[torch.ones_like(x), *cut(0, 2)]),
              lambda: he.attention_backward(x, x, x, x, o, lse, off, out=[torch.ones_like(x), o, torch.ones_like(x)]),
              lambda: he.attention_backward(x, x, x, x, o, lse, off, out=[torch.ones_like(x)] + [torch.ones_like(x)] * 2)):
        with pytest.raises(ValueError, match="overlap"):
            f()


def test_buffers_beside_one_another_are_taken(he):
    """Rows and heads that take turns in one buffer, and parts of one: none of them overlaps."""
    off, w, r = i32(0, 3, 8), rand(2, 64), rand(4, 8, 64)
    want = he.layer_norm(r, w, w)[0]
    both = torch.cat([r, torch.zeros_like(r)], 1)
    assert torch.equal(he.layer_norm(both[:, :64], w, w, out=both[:, 64:])[0], want) and torch.equal(both[:, :64], r)
    one = torch.cat([r, r, torch.zeros_like(r)])
    assert torch.equal(he.layer_norm(one[:8], w, w, residual=one[8:16], out=one[16:])[0], he.layer_norm(r, w, w, residual=r)[0])
    assert torch.equal(he.layer_norm(both[:1, :64], w, w, out=both[1:2, :64])[0], want[:1])  # rows of one, whose strides nothing asks for
    q, k, v = (rand(i, 8, 2, 32) for i in (5, 6, 7))
    o, lse = he.attention(q, k, v, off)
    joint = torch.cat([q, k, v, torch.zeros_like(q)], 1)
    assert torch.equal(he.attention(joint[:, :2], joint[:, 2:4], joint[:, 4:6], off, out=joint[:, 6:])[0], o) and torch.equal(joint[:, :2], q)
    heads = torch.stack([q, k, v, torch.zeros_like(q)]).transpose(1, 2).contiguous().transpose(1, 2)  # one head after the other
    assert torch.equal(he.attention(*heads[:3], off, out=heads[3])[0], o)
    mixed = torch.stack([q, k, v, torch.zeros_like(q)], 2)  # [rows][heads][4][dim]
    assert torch.equal(he.attention(*(mixed[:, :, i] for i in range(3)), off, out=mixed[:, :, 3])[0], o) and torch.equal(mixed[:, :, 0], q)
    grads = he.attention_backward(q, q, k, v, o, lse, off)
    d = torch.empty(8, 6, 32, device="cuda")
    he.attention_backward(q, q, k, v, o, lse, off, out=[d[:, i:i + 2] for i in (0, 2, 4)])
    assert all(torch.equal(d[:, 2 * i:2 * i + 2], g) for i, g in enumerate(grads))


def test_attention_of_one_row_or_one_head_whose_stride_nothing_takes(he):
    """The stride of a dimension of one element is no address: it may be any number."""
    k, v, off = rand(2, 7, 2, 32, dtype=BF16), rand(3, 7, 2, 32, dtype=BF16), (i32(0, 1), i32(0, 7))
    q = rand(1, 1, 2, 32, dtype=BF16)
    o, lse = he.attention(q, k, v, off[0], offsets_k=off[1])
    grads = he.attention_backward(q, q, k, v, o, lse, off[0], offsets_k=off[1])
    odd = torch.as_strided(q, (1, 2, 32), (101, 32, 1))
    far = torch.as_strided(q, (1, 2, 32), (1 << 24, 32, 1))
    for one in (odd, far):
        out = torch.as_strided(torch.empty_like(q), one.shape, one.stride())
        assert torch.equal(he.attention(one, k, v, off[0], offsets_k=off[1], out=out)[0], o) and torch.equal(he.attention(one, k, v, off[0], offsets_k=off[1])[0], o)
        assert all(torch.equal(a, b) for a, b in zip(he.attention_backward(one, one, k, v, o, lse, off[0], offsets_k=off[1]), grads))
    lone = torch.as_strided(k[:, :1].contiguous(), (7, 1, 32), (32, 5, 1))
    want = he.attention(q[:, :1], k[:, :1], k[:, :1], off[0], offsets_k=off[1])[0]
    assert torch.equal(he.attention(q[:, :1], lone, lone, off[0], offsets_k=off[1])[0], want)


def _fp16_inputs(seed, rows=223):
    return [rand(seed + i, rows, 2, 64, dtype=F16) for i in range(4)]


def test_fp16_gradients_keep_sequences_and_padding_apart(he):
    """The powers of two that lift ds come from the rows of a sequence alone: neither its neighbours' NaN and infinities nor those of rows of no
    sequence change a bit of it."""
    begin, end = i32(3, 53, 90, 103, 153), i32(40, 53, 100, 150, 154)
    keep = torch.zeros(223, dtype=torch.bool, device="cuda")
    for b, e in zip(begin.tolist(), end.tolist()):
        keep[b:e] = True
    q, k, v, do = _fp16_inputs(1)
    for sl in (None, torch.tensor([0.5, 0.01], device="cuda")):
        want = ref.attention(q, k, v, (begin, end), do=do, slopes=sl)
        o, lse = he.attention(q, k, v, (begin, end), slopes=sl)
        clean = he.attention_backward(do, q, k, v, o, lse, (begin, end), slopes=sl)
        for name, g in zip(("dq", "dk", "dv"), clean):
            ref.check(g, want[name], name)
        bad = [t.clone() for t in (q, k, v, do)]
        for t, x in zip(bad, ("nan", "inf", "nan", "-inf")):
            t[~keep] = float(x)
            t[95] = float(x)  # the third sequence
        o2, lse2 = he.attention(*bad[:3], (begin, end), slopes=sl)
        mine = keep.clone()
        mine[90:100] = False
        for g, c in zip(he.attention_backward(bad[3], *bad[:3], o2, lse2, (begin, end), slopes=sl), clean):
            assert torch.equal(g[mine], c[mine]) and not g[~keep].any()


def test_fp16_gradients_in_a_captured_graph(he):
    """The powers of two are found again in every replay."""
    off, sl = offsets_of([1, 60, 0, 162]), torch.tensor([0.5, 0.01], device="cuda")

    def run(q, k, v, do):
        o, lse = he.attention(q, k, v, off, slopes=sl)
        return (o, lse, *he.attention_backward(do, q, k, v, o, lse, off, slopes=sl), *he.attention_backward(do, q, k, v, *he.attention(q, k, v, off), off))

    ins, side, graph = _fp16_inputs(1), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(*ins)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        outs = run(*ins)
    for rep, size in enumerate((1.0, 2.0**-10, 2.0**9, 1.0)):
        for t, new in zip(ins, _fp16_inputs(10 * rep)):
            t.copy_(new)
        ins[3].mul_(size)
        want = [t.clone() for t in run(*ins)]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), rep


def test_fp16_gradients_of_offsets_that_break_the_rule_stay_in_the_buffers(he):
    q = rand(1, 64, 2, 32, dtype=F16)
    sl = torch.tensor([0.5, 0.01], device="cuda")
    for off in (i32(0, 500, 64), i32(-9, 30, 64), i32(0, 40, 10, 64), (i32(10, 0), i32(5, 100))):
        o, lse = he.attention(q, q, q, off)
        he.attention_backward(q, q, q, q, o, lse, off)
        he.attention_backward(q, q, q, q, o, lse, off, slopes=sl)
    torch.cuda.synchronize()


@pytest.mark.parametrize("lengths", [[9000], [30, 7000, 2, 900]])
def test_fp16_gradients_of_sequences_of_many_tiles(he, lengths):
    """More tiles than a wave has lanes: their sizes take several trips."""
    rows, off = sum(lengths), offsets_of(lengths)
    q, k, v, do = _fp16_inputs(5, rows)
    v[-3:] *= 100  # the largest in the last tile
    want = ref.attention(q, k, v, off, do=do, device="cuda")
    o, lse = he.attention(q, k, v, off)
    for name, g in zip(("dq", "dk", "dv"), he.attention_backward(do, q, k, v, o, lse, off)):
        ref.check(g, want[name], name)


def test_fp16_gradients_of_keys_without_much_weight(he):
    """Large do and v, and scores that leave some keys with next to nothing: their part of dk is small, and still right to fp16's smallest steps."""
    q, do = rand(1, 1, 112, scale=8.0), rand(2, 1, 112, scale=64.0)  # one query: no errors that cancel
    _check_gradients(he, q, rand(3, 500, 112), rand(4, 500, 112, scale=8.0), do, 112**-0.5)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("cap", [8.0, 50.0, 64.0, 1e5])
@pytest.mark.parametrize("queries", [7, 1400])
def test_capped_scores_of_few_keys(he, queries, cap, dtype):
    """lse of up to 32 keys in 32 bits.  Products have one term each, so a score is off by a few roundings (four of 2^-24 are granted, the library's tanh among them), and
    lse by that, by two steps of a logarithm below 8 (fp16's lift: 2^-20) and by its own rounding."""
    keys = [1, 2, 3, 17, 32, 33, 40]
    per = queries // 7
    q, k = torch.zeros(queries, 16, 32, dtype=dtype, device="cuda"), torch.zeros(sum(keys), 16, 32, dtype=dtype, device="cuda")
    q[..., 0], k[..., 0] = rand(1, queries, 16, dtype=dtype, scale=2.0), rand(2, sum(keys), 16, dtype=dtype, scale=2.0)
    lse = he.attention(q, k, k, offsets_of([per] * 7), offsets_k=offsets_of(keys), scale=0.5, cap=cap)[1].double()
    at = 0
    for i, n in enumerate(keys):
        t = 0.5 * q[i * per:(i + 1) * per, :, 0].double()[:, :, None] * k[at:at + n, :, 0].double().t()[None]
        t, at = cap * torch.tanh(t / cap), at + n
        want = torch.logsumexp(t, -1)
        # above 32 keys tanh is off by 2^-22 of the cap where that is at most 64
        bound = 4 * ref.F32 * t.abs().amax(-1) + 2.0**-20 + ref.F32 * want.abs() + (2.0**-22 * cap if n > 32 and cap <= 64 else 0.0)
        got = lse[:, i * per:(i + 1) * per].t()
        assert ((got - want).abs() <= bound).all(), (n, float((got - want).abs().max()))
