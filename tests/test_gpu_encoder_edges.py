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
