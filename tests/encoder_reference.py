"""The operators on token states in 64 bits on the CPU, from their definitions, with bounds for the kernels' roundings.

Bounds, with u = half the type's step (finfo.eps / 2) and f = 2^-24:
  a score is a sum of dim products in 32 bits and a few operations on it, so it is off by at most e_i = (dim + 8) f scale max|q_i| . |k_j| (as a sum of
  absolute products), plus 4 f |score| and, under a cap, 2 * 2^-23 cap for the tanh; an exponential of it by that much relatively, twice, with lse;
  p and dt are rounded to the type as factors (u each), sums of n terms in 32 bits are off by n f of their absolute terms, at most 2^-12 of them
  here (n <= 4096), and typically far less: 2^-14 is granted; the result is rounded once more (u).
  fp16 has steps of 2^-24 below 2^-14, so there a factor is off by half of one, 2^-25, at least: z = 2^-25 is added to the error of each p and dt.
"""
import math

import torch

F32 = 2.0**-24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def spans(offsets):
    if isinstance(offsets, (tuple, list)):
        return list(zip(offsets[0].tolist(), offsets[1].tolist()))
    o = offsets.tolist()
    return list(zip(o[:-1], o[1:]))


def attention(q, k, v, offsets, offsets_k=None, scale=None, cap=0.0, slopes=None, do=None, device="cpu"):
    """{name: (value, bound)} for o, lse and, with do, dq, dk, dv.  device: where the 64-bit arithmetic runs."""
    u = half_step(q.dtype)
    zero = 2.0**-25 if q.dtype == torch.float16 else 0.0
    q, k, v = (t.double().to(device) for t in (q, k, v))
    (tq, h, d), (tk, kv, _) = q.shape, k.shape
    scale = d**-0.5 if scale is None else scale
    z = lambda *s: torch.zeros(*s, dtype=torch.float64, device=device)  # noqa: E731
    out = {n: [z(*s), z(*s)] for n, s in (("o", q.shape), ("lse", (h, tq)), ("dq", q.shape), ("dk", k.shape), ("dv", k.shape))}
    out["lse"][0] -= math.inf
    if do is not None:
        do = do.double().to(device)
    for (qb, qe), (kb, ke) in zip(spans(offsets), spans(offsets if offsets_k is None else offsets_k)):
        if qe <= qb or ke <= kb:
            continue
        at = torch.arange(max(qe - qb, ke - kb), device=device)
        dist = (at[:qe - qb, None] + (ke - kb) - (qe - qb) - at[None, :ke - kb]).abs().double()
        for i in range(h):
            c = i // (h // kv)
            Q, K, V = q[qb:qe, i], k[kb:ke, c], v[kb:ke, c]
            t = scale * Q @ K.T
            e = (d + 8) * F32 * scale * (Q.abs() @ K.abs().T)
            th = torch.zeros_like(t)
            if cap:
                th = torch.tanh(t / cap)
                t = cap * th
                e = e + 2 * 2.0**-23 * cap
            if slopes is not None:
                t = t - float(slopes[i]) * dist
            e = (e + 4 * F32 * t.abs()).amax(1, keepdim=True) + 2.0**-22  # of a row's scores
            lse = torch.logsumexp(t, 1, keepdim=True)
            p = torch.exp(t - lse)
            o = p @ V
            rel = u + 2 * e + 2.0**-14
            out["o"][0][qb:qe, i], out["lse"][0][i, qb:qe] = o, lse[:, 0]
            ob = (rel * p + zero) @ V.abs() + u * o.abs()
            out["o"][1][qb:qe, i], out["lse"][1][i, qb:qe] = ob, (e + 4 * F32 * (lse.abs() + 32))[:, 0]
            if do is None:
                continue
            G = do[qb:qe, i]
            dp = G @ V.T
            delta = (G * o).sum(1, keepdim=True)
            slope = 1 - th**2
            ds = p * (dp - delta)
            dt = ds * slope * scale
            # delta is taken from o as rounded; dp and delta are sums of dim products
            db = (G.abs() * ob).sum(1, keepdim=True) + (d + 8) * F32 * (G.abs() @ V.abs().T + (G * o).abs().sum(1, keepdim=True))
            te = zero + (u + 2 * e + 2.0**-14) * dt.abs() + p * db * slope * scale
            if cap:  # 1 - th^2, th off by its own error and by the score's
                te = te + ds.abs() * scale * 2 * (2.0**-22 + e / cap)
            out["dq"][0][qb:qe, i] += dt @ K
            out["dq"][1][qb:qe, i] += te @ K.abs()
            out["dk"][0][kb:ke, c] += dt.T @ Q
            out["dk"][1][kb:ke, c] += te.T @ Q.abs()
            out["dv"][0][kb:ke, c] += p.T @ G
            out["dv"][1][kb:ke, c] += (rel * p + zero).T @ G.abs()
    for n in ("dq", "dk", "dv"):
        out[n][1] = out[n][1] + u * out[n][0].abs()
    return {n: (a.cpu(), (b + 1e-30 + (2.0**-24 if u == 2.0**-11 else 0.0)).cpu()) for n, (a, b) in out.items()}  # fp16: its smallest step


def layer_norm(x, w, b, r=None, eps=1e-5, dy=None, ds=None):
    """{name: (value, bound)} for y, s, mean, rstd and, with dy, dx, dw, db.  A row's mean is off by m_e = 2^-17 mean|s| (sums of at most 128 terms in a
    row, and a tree), so xh by x_e = rstd (m_e + 2^-17 |s - m|) or so, and the means of g and g xh likewise."""
    u, uw = half_step(x.dtype), half_step(w.dtype)
    s = x.cpu() if r is None else (x.cpu().float() + r.cpu().float()).to(x.dtype)
    S, W, B = s.double(), w.double().cpu(), b.double().cpu()
    m = S.mean(1, keepdim=True)
    rstd = ((S - m).pow(2).mean(1, keepdim=True) + eps).rsqrt()
    xh = (S - m) * rstd
    me = 2.0**-17 * S.abs().mean(1, keepdim=True)
    xe = rstd * me + 2.0**-16 * xh.abs()
    y = xh * W + B
    out = {"y": (y, u * y.abs() + xe * W.abs() + 2.0**-22 * (xh * W).abs() + 2.0**-22 * B.abs()), "s": (S, torch.zeros_like(S)),
           "mean": (m[:, 0], me[:, 0]), "rstd": (rstd[:, 0], 2.0**-16 * rstd[:, 0])}
    if dy is not None:
        G = dy.double().cpu()
        g = G * W
        c2 = (g * xh).mean(1, keepdim=True)
        dx = rstd * (g - g.mean(1, keepdim=True) - xh * c2)
        size = rstd * (g.abs() + g.abs().mean(1, keepdim=True) + xh.abs() * (g * xh).abs().mean(1, keepdim=True))
        bound = 2.0**-15 * size + rstd * (xe * c2.abs() + xh.abs() * (g.abs() * xe).mean(1, keepdim=True))
        if ds is not None:
            dx = dx + ds.double().cpu()
            bound = bound + 2.0**-22 * dx.abs()
        n = 2.0**-15  # the sum over rows in 32 bits: partial sums of few rows, joined
        dw, db = (G * xh).sum(0), G.sum(0)
        out["dx"] = dx, bound + u * dx.abs()
        out["dw"] = dw, uw * dw.abs() + n * (G * xh).abs().sum(0) + (G.abs() * xe).sum(0)
        out["db"] = db, uw * db.abs() + n * G.abs().sum(0)
    tiny = 2.0**-24 if u == 2.0**-11 else 0.0
    return {k: (a, e + 1e-30 + tiny) for k, (a, e) in out.items()}


def pool_mean(x, offsets):
    x = x.double().cpu()
    e = torch.stack([x[b:f].mean(0) if f > b else torch.zeros(x.shape[1], dtype=torch.float64) for b, f in spans(offsets)])
    size = torch.stack([x[b:f].abs().mean(0) if f > b else torch.zeros(x.shape[1], dtype=torch.float64) for b, f in spans(offsets)])
    return e, 2.0**-14 * size + 1e-30  # sums of at most 1024 terms in a row, 2^-24 each


def check(got, want, what):
    """Every element within its bound; infinities and NaN where the reference has them."""
    value, bound = want
    got = got.detach().double().cpu()
    assert got.shape == value.shape, (what, got.shape, value.shape)
    fine = torch.isfinite(value)
    assert torch.equal(torch.isfinite(got), fine), f"{what}: finite values elsewhere"
    assert torch.equal(got[~fine], value[~fine]) or bool(torch.isnan(value[~fine]).any()), f"{what}: other infinities"
    over = ((got - value).abs() - bound)[fine]
    if over.numel():
        worst = int(over.argmax())
        assert float(over.max()) <= 0, f"{what}: off by {float((got - value).abs()[fine][worst]):.3g}, granted {float(bound[fine][worst]):.3g}"
