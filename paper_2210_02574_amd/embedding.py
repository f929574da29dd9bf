"""From the states of a sentence's tokens to the embedding that is encrypted: the data owner's half of the paper's pipeline (Section 2.1,
x -> F_emb(x), then encryption), with gradients, so that an encoder can be fitted in the clear before its embeddings are.

The operators are the library's (HE.attention, HE.layer_norm, HE.rms_norm, HE.pool_mean); the functions here make them differentiable, and SentenceEncoder puts them
together.  Matrix products with weights are plain library products there; SentenceEncoder8, for inference, has them in 8 bits (HE.rms_norm8, HE.quantize8,
HE.linear8).  Sentences are packed back to back or padded, as HE's offsets say.
Gradients are of the first order: a backward pass that is to be differentiated again is refused.  One that is captured in a HIP graph needs leaves that no living eager
graph has: torch would have the capture wait for that graph's stream.
"""
from __future__ import annotations

import math
from typing import Dict, List, Sequence

import numpy as np
import torch
from torch.autograd.function import once_differentiable
from torch.nn import functional as F

from .classifier import BLOCK, pack_samples


def _kept(offsets):
    """Offsets as tensors to save for a backward pass, which then notices if they have been written since, and as what HE takes from those."""
    if isinstance(offsets, (tuple, list)):
        return tuple(offsets), tuple
    return (offsets,), lambda t: t[0]


def _dense(grad):
    """A gradient as HE.attention_backward takes it, dense and at a multiple of 16 bytes: it may be any part of what the program behind made."""
    grad = grad.contiguous()
    return grad.clone() if grad.data_ptr() % 16 else grad


class _Norm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, he, x, weight, bias, residual, eps):
        y, s, mean, rstd = he.layer_norm(x, weight, bias, residual=residual, eps=eps)
        ctx.he, ctx.residual = he, residual is not None
        ctx.save_for_backward(s, weight, mean, rstd)
        ctx.set_materialize_grads(False)
        return (y, s) if ctx.residual else (y, None)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, ds):
        s, weight, mean, rstd = ctx.saved_tensors
        if dy is None:  # only the sum was used
            return None, ds, None, None, ds if ctx.residual else None, None
        dx, dw, db = ctx.he.layer_norm_backward(dy.contiguous(), s, weight, mean, rstd, ds=None if ds is None else ds.contiguous())
        return None, dx, dw, db, dx if ctx.residual else None, None


def layer_norm(he, x, weight, bias, residual=None, eps: float = 1e-5):
    """(y, s): layer norm of s = x + residual, and s itself (x without a residual).  Differentiable in x, residual, weight and bias."""
    y, s = _Norm.apply(he, x, weight, bias, residual, eps)
    return y, x if s is None else s


class _Rms(torch.autograd.Function):
    @staticmethod
    def forward(ctx, he, x, weight, residual, eps):
        y, s, rstd = he.rms_norm(x, weight, residual=residual, eps=eps)
        ctx.he, ctx.residual = he, residual is not None
        ctx.save_for_backward(s, weight, rstd)
        ctx.set_materialize_grads(False)
        return (y, s) if ctx.residual else (y, None)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, ds):
        s, weight, rstd = ctx.saved_tensors
        if dy is None:  # only the sum was used
            return None, ds, None, ds if ctx.residual else None, None
        dx, dw = ctx.he.rms_norm_backward(dy.contiguous(), s, weight, rstd, ds=None if ds is None else ds.contiguous())
        return None, dx, dw, dx if ctx.residual else None, None


def rms_norm(he, x, weight, residual=None, eps: float = 1e-5):
    """(y, s): root-mean-square norm of s = x + residual, and s itself (x without a residual).  Differentiable in x, residual and weight."""
    y, s = _Rms.apply(he, x, weight, residual, eps)
    return y, x if s is None else s


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, he, q, k, v, offsets, offsets_k, scale, cap, slopes):
        o, lse = he.attention(q, k, v, offsets, offsets_k=offsets_k, scale=scale, cap=cap, slopes=slopes)
        (a, join), (b, join_k) = _kept(offsets), ((None,), lambda t: None) if offsets_k is None else _kept(offsets_k)
        ctx.he, ctx.args = he, (len(a), join, join_k, scale, cap)
        ctx.save_for_backward(q, k, v, o, lse, slopes, *a, *b)
        return o

    @staticmethod
    @once_differentiable
    def backward(ctx, do):
        n, join, join_k, scale, cap = ctx.args
        q, k, v, o, lse, slopes, *off = ctx.saved_tensors
        grads = ctx.he.attention_backward(_dense(do), q, k, v, o, lse, join(off[:n]), offsets_k=join_k(off[n:]), scale=scale, cap=cap, slopes=slopes)
        return (None, *grads, None, None, None, None, None)


def attention(he, q, k, v, offsets, offsets_k=None, scale=None, cap: float = 0.0, slopes=None):
    """HE.attention's o, differentiable in q, k and v."""
    if slopes is not None and slopes.requires_grad:
        raise ValueError("slopes are constants: they have no gradient")
    return _Attention.apply(he, q, k, v, offsets, offsets_k, scale, cap, slopes)


class _SelfAttention(torch.autograd.Function):
    """The same on one joint projection [rows][heads + 2 kv_heads][dim], whose gradient is written in one piece."""

    @staticmethod
    def forward(ctx, he, qkv, kv_heads, offsets, cap, slopes):
        h = qkv.shape[1] - 2 * kv_heads
        o, lse = he.attention(qkv[:, :h], qkv[:, h:h + kv_heads], qkv[:, h + kv_heads:], offsets, cap=cap, slopes=slopes)
        off, join = _kept(offsets)
        ctx.he, ctx.args = he, (kv_heads, join, cap)
        ctx.save_for_backward(qkv, o, lse, slopes, *off)
        return o

    @staticmethod
    @once_differentiable
    def backward(ctx, do):
        kv, join, cap = ctx.args
        qkv, o, lse, slopes, *off = ctx.saved_tensors
        h = qkv.shape[1] - 2 * kv
        d = torch.empty_like(qkv)
        cut = lambda t: (t[:, :h], t[:, h:h + kv], t[:, h + kv:])  # noqa: E731
        ctx.he.attention_backward(_dense(do), *cut(qkv), o, lse, join(off), cap=cap, slopes=slopes, out=cut(d), fill=True)
        return None, d, None, None, None, None


class _Pool(torch.autograd.Function):
    @staticmethod
    def forward(ctx, he, x, offsets):
        off, join = _kept(offsets)
        ctx.he, ctx.args = he, (join, x.shape[0], x.dtype)
        ctx.save_for_backward(*off)
        return he.pool_mean(x, offsets)

    @staticmethod
    @once_differentiable
    def backward(ctx, de):
        join, rows, dtype = ctx.args
        return None, ctx.he.pool_mean_backward(de.contiguous(), join(ctx.saved_tensors), rows, dtype), None


def pool_mean(he, x, offsets):
    """Mean of each sentence's rows in 32 bits, differentiable in x."""
    return _Pool.apply(he, x, offsets)


class SentenceEncoder:
    """Transformer layers over packed sentences, and the embedding of each sentence.

    layers: per layer a dict of weights: qkv [(heads + 2 kv_heads) dim][width] and qkv_bias, out [width][heads dim] and out_bias, up and up_bias,
    down and down_bias (the products of the feed-forward part, with a Gaussian error unit between), and its norms' weights.
    norm: "layer", a layer norm behind each residual sum (norm1, norm1_bias, norm2, norm2_bias), or "rms", a root-mean-square norm ahead of each half of a layer (norm1,
    norm2) and one behind the last layer (last: its weight [width]).
    pool: "mean" of a sentence's rows, or its "first" row; the last layer then computes that row of each sentence alone.
    cap, slopes: as HE.attention takes them, the same in every layer; no slopes with pool "first"."""

    PRODUCTS = ("qkv", "out", "up", "down")
    NORMS = {"layer": ("norm1", "norm1_bias", "norm2", "norm2_bias"), "rms": ("norm1", "norm2")}
    NAMES = ("qkv", "qkv_bias", "out", "out_bias", "up", "up_bias", "down", "down_bias") + NORMS["layer"]

    def __init__(self, he, layers: Sequence[Dict[str, torch.Tensor]], heads: int, kv_heads: int = 0, pool: str = "mean", cap: float = 0.0,
                 slopes=None, eps: float = 1e-5, norm: str = "layer", last=None):
        if pool not in ("mean", "first"):
            raise ValueError(f"pool: {pool!r}, want 'mean' or 'first'")
        if norm not in self.NORMS:
            raise ValueError(f"norm: {norm!r}, want 'layer' or 'rms'")
        if (last is None) == (norm == "rms"):
            raise ValueError("last: the weight of the norm behind the last layer, with norm='rms' alone")
        if slopes is not None and slopes.requires_grad:
            raise ValueError("slopes are constants: they have no gradient")
        if slopes is not None and pool == "first":
            raise ValueError("pool='first' with a distance bias: a lone query stands at its sentence's last position, not its first")
        for i, w in enumerate(layers):
            missing = [n for n in self.NAMES[:8] + self.NORMS[norm] if n not in w]
            if missing:
                raise ValueError(f"layer {i} lacks {', '.join(missing)}")
        self.he, self.layers, self.heads, self.kv_heads = he, list(layers), heads, kv_heads or heads
        self.pool, self.cap, self.slopes, self.eps, self.norm, self.last = pool, cap, slopes, eps, norm, last

    @classmethod
    def random_layer(cls, width: int, heads: int, inner: int, seed: int, dtype, device, kv_heads: int = 0, std: float = 0.02):
        """Weights of one layer: N(0, std^2), norms at one, biases at zero."""
        g = torch.Generator(device="cpu")
        g.manual_seed(seed)
        kv, dim = kv_heads or heads, width // heads
        shapes = {"qkv": ((heads + 2 * kv) * dim, width), "out": (width, heads * dim), "up": (inner, width), "down": (width, inner)}
        w = {n: (std * torch.randn(s, generator=g)).to(device, dtype) for n, s in shapes.items()}
        w |= {n + "_bias": torch.zeros(s[0], dtype=dtype, device=device) for n, s in shapes.items()}
        for n in ("norm1", "norm2"):
            w[n], w[n + "_bias"] = torch.ones(width, dtype=dtype, device=device), torch.zeros(width, dtype=dtype, device=device)
        return w

    def in_8_bits(self) -> "SentenceEncoder8":
        """This encoder with its products in 8 bits, for inference; later changes of its weights do not reach the result."""
        return SentenceEncoder8(self)

    # What a product reads, of rows, of their Gaussian error units, and of the norm of the sum f + x (x alone without f), which comes back as well.
    def _rows(self, x):
        return x

    def _units(self, x):
        return F.gelu(x)

    def _rms(self, f, x, weight):
        return rms_norm(self.he, x, weight, eps=self.eps) if f is None else rms_norm(self.he, f, weight, residual=x, eps=self.eps)

    def _take(self, a, begin):
        return a[begin]

    def _product(self, w, name, a, lo=None, hi=None):
        """Rows of a times weights w[name], or their channels lo .. hi."""
        part = self._all if lo is None and hi is None else lambda t: t[lo:hi]
        return F.linear(a, part(w[name]), part(w[name + "_bias"]))

    @staticmethod
    def _all(t):  # (a slice of all would be a copy of the gradient)
        return t

    def _head(self, w, f, x):
        """What a layer's first product reads, and the layer's input."""
        return (self._rows(x), x) if self.norm == "layer" else self._rms(f, x, w["norm1"])

    def _rest(self, w, o, x):
        """The layer behind its attention: o [rows][heads][dim], x the layer's input on those rows.  (f, x): the layer's result is x, or x + f where f is not None."""
        f = self._product(w, "out", self._rows(o.flatten(1)))
        if self.norm == "rms":
            a, x = self._rms(f, x, w["norm2"])
            return self._product(w, "down", self._units(self._product(w, "up", a))), x
        x, _ = layer_norm(self.he, f, w["norm1"], w["norm1_bias"], residual=x, eps=self.eps)
        f = self._product(w, "down", self._units(self._product(w, "up", self._rows(x))))
        return None, layer_norm(self.he, f, w["norm2"], w["norm2_bias"], residual=x, eps=self.eps)[0]

    def _end(self, f, x):
        """The states behind the last layer."""
        if self.norm == "layer":
            return x
        return rms_norm(self.he, x, self.last, eps=self.eps)[0] if f is None else rms_norm(self.he, f, self.last, residual=x, eps=self.eps)[0]

    def __call__(self, states, offsets):
        """states [rows][width], offsets as HE's operators take them -> embeddings [sentences][width] in 32 bits."""
        f, x, kv = None, states, self.kv_heads
        if not x.shape[0]:
            return pool_mean(self.he, x, offsets)  # sentences without rows
        for i, w in enumerate(self.layers):
            a, x = self._head(w, f, x)
            if self.pool == "first" and i == len(self.layers) - 1:
                return self._last_first(w, a, x, offsets)
            qkv = self._product(w, "qkv", a).unflatten(1, (self.heads + 2 * kv, -1))
            f, x = self._rest(w, _SelfAttention.apply(self.he, qkv, kv, offsets, self.cap, self.slopes), x)
        x = self._end(f, x)
        if self.pool == "mean":
            return pool_mean(self.he, x, offsets)
        begin, some = self._first(x, offsets)
        return torch.where(some[:, None], x[begin], 0.0).float()

    @staticmethod
    def _first(x, offsets):
        """First rows of the sentences, and which sentences have one."""
        begin, end = offsets if isinstance(offsets, (tuple, list)) else (offsets[:-1], offsets[1:])
        return begin.clamp(0, max(x.shape[0] - 1, 0)).long(), end > begin

    def _last_first(self, w, a, x, offsets):
        """The last layer on the first row of each sentence: one query to a sentence's keys."""
        begin, some = self._first(x, offsets)
        rows = x[begin]
        dim = w["qkv_bias"].shape[0] // (self.heads + 2 * self.kv_heads)
        cut = self.heads * dim
        q = self._product(w, "qkv", rows if a is x else self._take(a, begin), None, cut).unflatten(1, (self.heads, dim))
        kvs = self._product(w, "qkv", a, cut).unflatten(1, (2 * self.kv_heads, dim))
        one = torch.arange(len(begin) + 1, dtype=torch.int32, device=x.device)
        o = attention(self.he, q, kvs[:, :self.kv_heads], kvs[:, self.kv_heads:], one, offsets_k=offsets, cap=self.cap)
        return torch.where(some[:, None], self._end(*self._rest(w, o, rows)), 0.0).float()


class SentenceEncoder8(SentenceEncoder):
    """An encoder whose products with weights are in 8 bits, with a scale for each row and channel: weights are laid out once, all others copied, rows where they come out of a norm, attention
    or the Gaussian error units.  Norms, attention and residual sums stay as they are.  No gradients pass through 8-bit rows.
    The rows of a product's weights are at most MAX_WIDTH wide."""

    MAX_WIDTH = 16384  # of rows that HE.quantize8 and HE.rms_norm8 make

    def __init__(self, encoder: SentenceEncoder):
        for i, w in enumerate(encoder.layers):
            for n in self.PRODUCTS:
                if w[n].shape[1] > self.MAX_WIDTH:
                    raise ValueError(f"layer {i}: {n} has rows of {w[n].shape[1]}, rows in 8 bits are at most {self.MAX_WIDTH} wide")
        he = encoder.he

        def eight(t):
            rows, scale = he.quantize8(t.detach().contiguous())  # (weights may be views of any strides)
            return rows, scale.clone()  # (apart from the integers' storage: torch.save takes no two types of one)

        copy = lambda t: None if t is None else t.detach().clone()  # noqa: E731 (a step of an optimizer writes to the source's tensors)
        layers = [{n: eight(w[n]) if n in self.PRODUCTS else copy(w[n]) for n in self.NAMES[:8] + self.NORMS[encoder.norm]} for w in encoder.layers]
        super().__init__(he, layers, encoder.heads, encoder.kv_heads, encoder.pool, encoder.cap, copy(encoder.slopes), encoder.eps, encoder.norm, copy(encoder.last))
        self.dtype = encoder.layers[0]["qkv"].dtype if layers else None  # of the states between the products

    def in_8_bits(self):
        return self

    def _rows(self, x):
        return self.he.quantize8(x)

    def _units(self, x):
        return self.he.quantize8(x, gelu=True)

    def _rms(self, f, x, weight):
        x8, scale, s = self.he.rms_norm8(x, weight, eps=self.eps) if f is None else self.he.rms_norm8(f, weight, residual=x, eps=self.eps)
        return (x8, scale), s

    def _take(self, a, begin):
        x8, scale = a  # with what stands behind each row: rows begin at multiples of 64 bytes
        return x8.as_strided((x8.shape[0], x8.stride(0)), (x8.stride(0), 1))[begin][:, :x8.shape[1]], scale[begin]

    def _product(self, w, name, a, lo=None, hi=None):
        part = self._all if lo is None and hi is None else lambda t: t[lo:hi]
        w8, scale = w[name]
        return self.he.linear8(*a, part(w8), part(scale), bias=part(w[name + "_bias"]), dtype=self.dtype)

    def __call__(self, states, offsets):
        if states.requires_grad and torch.is_grad_enabled():
            raise ValueError("states: an encoder in 8 bits has no gradients")
        return super().__call__(states, offsets)


def pack_embeddings(e, n_slots: int) -> List[np.ndarray]:
    """Embeddings [sentences][768] as the slot vectors of ciphertexts, n_slots / 1024 sentences to each, the last one filled up with zeros."""
    e = e.detach().cpu().numpy().astype(np.float64) if torch.is_tensor(e) else np.asarray(e, dtype=np.float64)
    nb = n_slots // BLOCK
    full = np.zeros((max(1, math.ceil(e.shape[0] / nb)) * nb, e.shape[1]))
    full[:e.shape[0]] = e
    return [pack_samples(full[i:i + nb], n_slots) for i in range(0, full.shape[0], nb)]
