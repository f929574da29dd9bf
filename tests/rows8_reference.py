"""Root-mean-square norm, rows in 8 bits and their products in 64 bits, from their definitions, with bounds for the kernels' roundings.

Bounds, with u = half the type's step (finfo.eps / 2): a sum of a row's squares has at most 64 roundings in a chain (32 of a thread's, a tree, 16 shares), all of one sign, so it is within 2^-18
of itself, rstd within 2^-18 with its own rounding, y = s rstd w within u + 2^-17.  A sum of products of both signs is off by 2^-18 of its absolute terms, and by the 2^-18 of rstd.
127 f / t is off by 127 times 3 2^-24 (f, t and the product with 127 / t rounded) where f is not a number of 32 bits, less than 2^-15; where it is, the integers are exact.
A product's sum is exact; four roundings to 32 bits follow and one to the type.
"""
import torch

from encoder_reference import half_step


def rms_norm(x, w, r=None, eps=1e-5, dy=None, ds=None):
    """{name: (value, bound)} for y, s, rstd and, with dy, dx, dw."""
    u, uw = half_step(x.dtype), half_step(w.dtype)
    s = x.cpu() if r is None else (x.cpu().float() + r.cpu().float()).to(x.dtype)
    S, W = s.double(), w.double().cpu()
    rstd = (S.pow(2).mean(1, keepdim=True) + eps).rsqrt()
    xh = S * rstd
    y = xh * W
    out = {"y": (y, (u + 2.0**-17) * y.abs()), "s": (S, torch.zeros_like(S)), "rstd": (rstd[:, 0], 2.0**-18 * rstd[:, 0])}
    if dy is not None:
        G = dy.double().cpu()
        g = G * W
        dx = rstd * (g - xh * (g * xh).mean(1, keepdim=True))
        bound = 2.0**-16 * rstd * (g.abs() + xh.abs() * (g * xh).abs().mean(1, keepdim=True))
        if ds is not None:
            dx = dx + ds.double().cpu()
            bound = bound + 2.0**-22 * dx.abs()
        dw = (G * xh).sum(0)
        out["dx"] = dx, bound + u * dx.abs()
        out["dw"] = dw, uw * dw.abs() + 2.0**-16 * (G * xh).abs().sum(0)
    tiny = 2.0**-24 if u == 2.0**-11 else 0.0
    return {k: (a, e + 1e-30 + tiny) for k, (a, e) in out.items()}


def quotients(f):
    """127 f / t of rows f in 64 bits, and t."""
    t = f.abs().amax(1, keepdim=True)
    return 127 * f / torch.where(t > 0, t, 1.0), t[:, 0]


def gelu(x):
    """(value, relative error granted) of x Phi(x)."""
    x = x.double().cpu()
    return x * torch.special.ndtr(x), 2.0**-20 * (1 + x * x / 8)


def linear8(x8, scale, w8, w_scale, bias, dtype):
    """(value, bound), where the operands are."""
    v = (x8.double() @ w8.double().t()) * scale.double()[:, None] * w_scale.double()
    o = v if bias is None else v + bias.double()
    u = half_step(dtype)
    return o, u * o.abs() + 2.0**-22 * (v.abs() + o.abs()) + (2.0**-24 if dtype == torch.float16 else 1e-30)
