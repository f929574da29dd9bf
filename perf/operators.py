"""The operators between token states and the embedding that is encrypted: attention inside each sequence of a batch, layer norm, the mean
over a sequence; forward, and with their gradients.

`own` false: the plain forms, in elementary torch operations; true: the calls that a program makes of the framework.  Sequences are rows
[begin, end) of the token axis, packed back to back or padded to one length; their lengths belong to the case, their contents to the seed.
"""
import functools
import math
import random

import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-5


@functools.lru_cache(maxsize=None)
def _he():
    from paper_2210_02574_amd import HE

    q = [2**40 - d for d in (147455, 237567, 368639)]
    return HE(12, q, [2**50 - 16383], 3, device=0)


# ---- the cases ----------------------------------------------------------------------------------------------------


def _attention(name, seqs, longest, heads, dtype, kv_heads=None, dim=64, cap=0.0, slopes=False, padded=False, one_query=False, train=False):
    return {"name": name, "op": "attention", "seqs": seqs, "longest": longest, "heads": heads, "kv_heads": kv_heads or heads, "dim": dim,
            "dtype": dtype, "cap": cap, "slopes": slopes, "padded": padded, "one_query": one_query, "train": train}


def _norm(name, rows, width, dtype, weight_dtype="f32", residual=False, train=False):
    return {"name": name, "op": "norm", "rows": rows, "width": width, "dtype": dtype, "weight_dtype": weight_dtype, "residual": residual, "train": train}


def _mean(name, seqs, longest, width, dtype, padded=False, train=False):
    return {"name": name, "op": "mean", "seqs": seqs, "longest": longest, "width": width, "dtype": dtype, "padded": padded, "train": train}


def listed():
    return [
        # one short sentence in 32 bits, as a client embeds what it asks about: the call itself is what costs
        _attention("attention_one_f32", 1, 23, 12, "f32"),
        # the sentences of one ciphertext, padded to the longest
        _attention("attention_32_bf16", 32, 128, 12, "bf16", padded=True),
        # the last layer of an encoder, which needs one row of each document alone
        _attention("attention_last_bf16", 16, 2048, 12, "bf16", one_query=True),
        # one long document, heads of 128, shared key heads
        _attention("attention_long_bf16", 1, 16384, 12, "bf16", kv_heads=4, dim=128),
        # a step of fitting the encoder: many sentences of mixed lengths, packed
        _attention("attention_train_bf16", 64, 512, 12, "bf16", train=True),
        # a step on long documents with capped scores, a distance bias and shared key heads
        _attention("attention_train_f16", 3, 4000, 16, "f16", kv_heads=8, cap=30.0, slopes=True, train=True),
        # the rows of one short sentence
        _norm("norm_one_bf16", 23, 768, "bf16"),
        # a large batch behind its residual sum
        _norm("norm_large_bf16", 65536, 768, "bf16", residual=True),
        # a training step behind a residual sum
        _norm("norm_train_bf16", 16384, 768, "bf16", residual=True, train=True),
        # a training step in 32 bits on a width that no vector divides
        _norm("norm_train_f32", 4999, 1021, "f32", train=True),
        # the embeddings of one ciphertext's sentences
        _mean("mean_32_bf16", 32, 128, 768, "bf16", padded=True),
        # a training step over many packed documents
        _mean("mean_train_bf16", 256, 1024, 768, "bf16", train=True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(["attention", "attention", "norm", "mean"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    train = rng.random() < 0.5
    if op == "norm":
        width = _log_int(rng, 16, 8192)
        c = _norm("", _log_int(rng, 1, min(65536, (48 << 20) // width)), width, dtype, rng.choice(["f32", dtype]), rng.random() < 0.5, train)
    elif op == "mean":
        seqs, width = _log_int(rng, 1, 512), _log_int(rng, 16, 2048)
        c = _mean("", seqs, _log_int(rng, 1, max(1, min(8192, (64 << 20) // (width * seqs)))), width, dtype, rng.random() < 0.5, train)
    else:
        kv = rng.choice([2, 4, 8])
        heads = kv * rng.choice([1, 2, 3])
        seqs, one = _log_int(rng, 1, 256), rng.random() < 0.2
        # scores of a step in 32 bits, or of a step with gradients, cost more than others; stay below the largest listed case
        most = (12 << 28) // (8 * heads * seqs * (4 if train else 1) * (8 if dtype == "f32" else 1))
        top = min(8192, (1 << 17) // seqs, math.isqrt(most))
        c = _attention("", seqs, _log_int(rng, 1, max(1, top)), heads, dtype, kv, rng.choice([32, 64, 64, 96, 128]), rng.choice([0.0, 0.0, 20.0, 50.0]),
                       rng.random() < 0.4, rng.random() < 0.4, one, train and not one)
    del c["name"]
    return c


def _lengths(case):
    """Lengths from an eighth of the longest up to it, the longest among them; in batches of eight or more one is empty and one a single row."""
    seqs, longest = case["seqs"], case["longest"]
    r = random.Random(1000 * seqs + longest)
    n = [r.randint(max(1, longest // 8), longest) for _ in range(seqs)]
    n[r.randrange(seqs)] = longest
    if seqs >= 8:
        i = n.index(longest)
        n[(i + 1) % seqs], n[(i + 2) % seqs] = 0, 1
    return n


def _spans(case):
    """(begin, end) of every sequence, and the rows in all."""
    n = _lengths(case)
    if case["padded"]:
        return [case["longest"] * i for i in range(len(n))], [case["longest"] * i + v for i, v in enumerate(n)], case["longest"] * len(n)
    begin = [sum(n[:i]) for i in range(len(n))]
    return begin, [b + v for b, v in zip(begin, n)], sum(n)


# ---- inputs --------------------------------------------------------------------------------------------------------


def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _normal(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device=DEVICE).to(dtype)


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


def prepare(case, seed):
    g, dtype = _generator(seed), DTYPES[case["dtype"]]
    s = dict(case)
    if case["op"] == "norm":
        rows, width, wt = case["rows"], case["width"], DTYPES[case["weight_dtype"]]
        s["x"] = _normal(g, rows, width, dtype=dtype)
        s["r"] = _normal(g, rows, width, dtype=dtype) if case["residual"] else None
        s["w"] = (1 + 0.1 * _normal(g, width)).to(wt)
        s["b"] = (0.1 * _normal(g, width)).to(wt)
        if case["train"]:
            s["dy"] = _normal(g, rows, width, dtype=dtype)
        return s
    begin, end, rows = _spans(case)
    s["begin"], s["end"], s["rows"] = _i32(begin), _i32(end), rows
    s["offsets"] = (s["begin"], s["end"]) if case["padded"] else _i32(begin + end[-1:])
    if case["op"] == "mean":
        s["x"] = _normal(g, rows, case["width"], dtype=dtype)
        if case["train"]:
            s["de"] = _normal(g, case["seqs"], case["width"])
        return s
    heads, kv, dim = case["heads"], case["kv_heads"], case["dim"]
    qkv = _normal(g, rows, heads + 2 * kv, dim, dtype=dtype)  # as one projection gives them
    s["q"], s["k"], s["v"] = qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:]
    s["q_begin"], s["q_end"], s["q_offsets"] = s["begin"], s["end"], s["offsets"]
    s["q_longest"] = case["longest"]
    if case["one_query"]:
        first = list(range(case["seqs"] + 1))
        s["q"] = _normal(g, case["seqs"], heads, dim, dtype=dtype)
        s["q_begin"], s["q_end"], s["q_offsets"] = _i32(first[:-1]), _i32(first[1:]), _i32(first)
        s["q_longest"] = 1
    s["slope"] = 2.0 ** -(8.0 * torch.arange(1, heads + 1, device=DEVICE) / heads) if case["slopes"] else None
    if case["train"]:
        s["do"] = _normal(g, rows, heads, dim, dtype=dtype)
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------


def _rows_of(begin, end, longest):
    """[seqs][longest] row numbers, and which of them are rows of the sequence."""
    at = begin.long()[:, None] + torch.arange(longest, device=begin.device)
    ok = at < end.long()[:, None]
    return torch.where(ok, at, torch.zeros_like(at)), ok


def _padded(x, at, ok):
    """[rows][heads][dim] -> [seqs][heads][longest][dim] in 32 bits, zeros behind a sequence."""
    return torch.where(ok[:, :, None, None], x[at].float(), 0.0).transpose(1, 2)


def _packed(x, at, ok, rows, fill=0.0):
    """[seqs][heads][longest][...] -> [rows][heads][...]"""
    x = x.transpose(1, 2)
    out = torch.full((rows,) + x.shape[2:], fill, device=x.device)
    out[at[ok]] = x[ok]
    return out


def _scores(s, q, k, ok_k, n_q, n_k):
    """Scores [seqs][kv][group][queries][keys], and the tanh of the capped ones."""
    t = torch.matmul(q, k.transpose(-1, -2).unsqueeze(2)) / math.sqrt(s["dim"])
    th = None
    if s["cap"]:
        th = torch.tanh(t / s["cap"])
        t = s["cap"] * th
    if s["slopes"]:
        i = torch.arange(q.shape[-2], device=q.device)[None, :, None] + (n_k - n_q)[:, None, None]
        far = (i - torch.arange(k.shape[-2], device=q.device)[None, None, :]).abs().float()
        t = t - s["slope"].view(1, s["kv_heads"], -1, 1, 1) * far[:, None, None]
    return t.masked_fill(~ok_k[:, None, None, None, :], -math.inf), th


def _attention_plain(s):
    kv, group = s["kv_heads"], s["heads"] // s["kv_heads"]
    at_q, ok_q = _rows_of(s["q_begin"], s["q_end"], s["q_longest"])
    at_k, ok_k = _rows_of(s["begin"], s["end"], s["longest"])
    q, k, v = _padded(s["q"], at_q, ok_q), _padded(s["k"], at_k, ok_k), _padded(s["v"], at_k, ok_k)
    shape = q.shape
    q = q.reshape(shape[0], kv, group, shape[2], shape[3])
    t, th = _scores(s, q, k, ok_k, s["q_end"] - s["q_begin"], s["end"] - s["begin"])
    top = t.amax(-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, 0.0)
    p = torch.exp(t - top)
    del t
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total > 0, total, 1.0)
    o = torch.matmul(p, v.unsqueeze(2))
    rows = s["q"].shape[0]
    out = _packed(o.reshape(shape), at_q, ok_q, rows).to(s["q"].dtype)
    if not s["train"]:
        lse = (top + torch.log(total)).reshape(shape[:3])
        return out, _packed(lse, at_q, ok_q, rows, -math.inf).transpose(0, 1).contiguous()
    do = _padded(s["do"], at_q, ok_q).reshape(q.shape)
    dt = p * (torch.matmul(do, v.transpose(-1, -2).unsqueeze(2)) - (do * o).sum(-1, keepdim=True))
    if s["cap"]:
        dt = dt * (1 - th * th)
    dt = dt / math.sqrt(s["dim"])
    dq = torch.matmul(dt, k.unsqueeze(2)).reshape(shape)
    dk = torch.matmul(dt.transpose(-1, -2), q).sum(2)
    dv = torch.matmul(p.transpose(-1, -2), do).sum(2)
    t = s["q"].dtype
    return out, _packed(dq, at_q, ok_q, rows).to(t), _packed(dk, at_k, ok_k, rows).to(t), _packed(dv, at_k, ok_k, rows).to(t)


def _norm_plain(s):
    x = s["x"] if s["r"] is None else (s["x"].float() + s["r"].float()).to(s["x"].dtype)  # the sum is kept, and normalised as it is kept
    f = x.float()
    mean = f.mean(-1, keepdim=True)
    rstd = torch.rsqrt(((f - mean) ** 2).mean(-1, keepdim=True) + EPS)
    xh, w = (f - mean) * rstd, s["w"].float()
    y = (xh * w + s["b"].float()).to(x.dtype)
    kept = () if s["r"] is None else (x,)
    if not s["train"]:
        return (y,) + kept
    dy = s["dy"].float()
    g = dy * w
    dx = rstd * (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True))
    return (y,) + kept + (dx.to(x.dtype), (dy * xh).sum(0).to(s["w"].dtype), dy.sum(0).to(s["w"].dtype))


def _mean_plain(s):
    at, ok = _rows_of(s["begin"], s["end"], s["longest"])
    n = (s["end"] - s["begin"]).clamp(min=1).float()[:, None]
    e = torch.where(ok[:, :, None], s["x"][at].float(), 0.0).sum(1) / n
    if not s["train"]:
        return e
    dx = torch.zeros(s["x"].shape, dtype=s["x"].dtype, device=e.device)
    dx[at[ok]] = (s["de"] / n).to(dx.dtype)[:, None].expand(-1, s["longest"], -1)[ok]
    return e, dx


def run(s):
    if not own:
        return {"attention": _attention_plain, "norm": _norm_plain, "mean": _mean_plain}[s["op"]](s)
    he = _he()
    if s["op"] == "norm":
        y, kept, mean, rstd = he.layer_norm(s["x"], s["w"], s["b"], residual=s["r"], eps=EPS)
        out = (y,) if s["r"] is None else (y, kept)
        return out + he.layer_norm_backward(s["dy"], kept, s["w"], mean, rstd) if s["train"] else out
    if s["op"] == "mean":
        e = he.pool_mean(s["x"], s["offsets"])
        return (e, he.pool_mean_backward(s["de"], s["offsets"], s["x"].shape[0], s["x"].dtype)) if s["train"] else e
    extra = {"offsets_k": s["offsets"], "cap": s["cap"], "slopes": s["slope"]}
    o, lse = he.attention(s["q"], s["k"], s["v"], s["q_offsets"], **extra)
    if not s["train"]:
        return o, lse
    return (o,) + he.attention_backward(s["do"], s["q"], s["k"], s["v"], o, lse, s["q_offsets"], **extra)


# ---- what a pass cannot do without, and its result in 64 bits ------------------------------------------------------------


def work(case):
    size = 4.0 if case["dtype"] == "f32" else 2.0
    if case["op"] == "norm":
        n, w = float(case["rows"] * case["width"]), 4.0 if case["weight_dtype"] == "f32" else 2.0
        b = n * size * (4 if case["residual"] else 2) + 2 * w * case["width"]
        if case["train"]:
            b += 2 * n * size + 2 * w * case["width"]
        return {"bytes": b, "flops": n * (8 + (14 if case["train"] else 0))}
    n = _lengths(case)
    if case["op"] == "mean":
        b = sum(n) * case["width"] * size + 4.0 * case["seqs"] * case["width"]
        return {"bytes": b * (2 if case["train"] else 1), "flops": float(sum(n) * case["width"])}
    m = [1] * len(n) if case["one_query"] else n
    h, kv, d = case["heads"], case["kv_heads"], case["dim"]
    queries, keys, pairs = float(sum(m)), float(sum(n)), float(sum(a * b for a, b in zip(m, n)))
    if case["train"]:
        return {"bytes": size * d * (4 * queries * h + 4 * keys * kv), "flops": 14.0 * d * h * pairs}
    return {"bytes": size * d * (2 * queries * h + 2 * keys * kv) + 4 * queries * h, "flops": 4.0 * d * h * pairs}


def _exact_attention(case, s):
    h, kv, d = case["heads"], case["kv_heads"], case["dim"]
    t_q, t_k = s["q"].shape[0], s["k"].shape[0]
    f64 = {"dtype": torch.float64, "device": DEVICE}
    o, lse = torch.zeros(t_q, h, d, **f64), torch.full((h, t_q), -math.inf, **f64)
    dq, dk, dv = torch.zeros(t_q, h, d, **f64), torch.zeros(t_k, kv, d, **f64), torch.zeros(t_k, kv, d, **f64)
    spans = zip(*(s[x].tolist() for x in ("q_begin", "q_end", "begin", "end")))
    for qb, qe, kb, ke in spans:
        if qe == qb or ke == kb:
            continue
        back = torch.arange(qe - qb, **f64)[:, None] + float((ke - kb) - (qe - qb)) - torch.arange(ke - kb, **f64)[None, :]
        for i in range(h):
            c = i // (h // kv)
            q, k, v = s["q"][qb:qe, i].double(), s["k"][kb:ke, c].double(), s["v"][kb:ke, c].double()
            a = q @ k.t() * d**-0.5
            slope = 1.0
            if case["cap"]:
                a = a / case["cap"]
                a.tanh_()
                slope = 1 - a**2
                a = a * case["cap"]
            if case["slopes"]:
                a -= float(s["slope"][i]) * back.abs()
            z = torch.logsumexp(a, 1)
            a = torch.exp(a - z[:, None])
            lse[i, qb:qe] = z
            o[qb:qe, i] = a @ v
            if case["train"]:
                do = s["do"][qb:qe, i].double()
                dv[kb:ke, c] += a.t() @ do
                a = a * (do @ v.t() - (do * o[qb:qe, i]).sum(1)[:, None]) * slope * d**-0.5
                dq[qb:qe, i] = a @ k
                dk[kb:ke, c] += a.t() @ q
    return (o, dq, dk, dv) if case["train"] else (o, lse)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "attention":
        return _exact_attention(case, s)
    if case["op"] == "mean":
        x = s["x"].double()
        e = torch.zeros(case["seqs"], case["width"], dtype=torch.float64, device=DEVICE)
        dx = torch.zeros_like(x)
        for i, (b, f) in enumerate(zip(s["begin"].tolist(), s["end"].tolist())):
            if f > b:
                e[i] = x[b:f].sum(0) / (f - b)
                if case["train"]:
                    dx[b:f] = s["de"][i].double() / (f - b)
        return (e, dx) if case["train"] else e
    x, w = s["x"].double(), s["w"].double()
    if case["residual"]:
        x = (x + s["r"].double()).to(s["x"].dtype).double()
    var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
    sd = torch.sqrt(var + EPS)
    xh = (x - mean) / sd
    out = (xh * w + s["b"].double(),) + ((x,) if case["residual"] else ())
    if case["train"]:
        dy = s["dy"].double()
        a = dy * w / sd
        out += (a - a.mean(1, keepdim=True) - xh * (a * xh).mean(1, keepdim=True), (dy * xh).sum(0), dy.sum(0))
    return out
