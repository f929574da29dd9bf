"""ctypes binding of the C ABI declared in include/he.h.

Argument marshalling only: every computation runs inside the shared library.  Device buffers
are torch int64 tensors on the GPU (their bits are the uint64 residues); host buffers are
numpy arrays.  The library is loaded from the package directory and a missing build is an
error, never a fallback.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import List, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libhe_gfx950.so")

HE_OK = 0
HE_EWORKSPACE = -4
ERRORS = {
    -1: "HE_EINVAL", -2: "HE_ELEVEL", -3: "HE_ENOKEY", -4: "HE_EWORKSPACE",
    -5: "HE_EHIP", -6: "HE_ENODEV", -7: "HE_ENOMEM", -8: "HE_ESCRATCH",
}

# every symbol include/he.h declares
SYMBOLS = [
    "he_ctx_create", "he_ctx_destroy", "he_strerror", "he_last_hip_error", "he_ctx_modulus",
    "he_galois_element", "he_gauss_cdt", "he_workspace_bytes", "he_ctx_set_conversion",
    "he_keygen_secret", "he_sk_destroy", "he_sk_coeffs", "he_keygen_relin", "he_keygen_rot",
    "he_keygen_conj", "he_keygen_public", "he_encrypt_public_coeffs", "he_keygen_secret_sparse", "he_modraise", "he_pmult_sum",
    "he_evk_from_host", "he_evk_to_host", "he_evk_destroy",
    "he_encode", "he_decode", "he_plain_to_ntt", "he_encrypt_coeffs", "he_decrypt_coeffs", "he_decrypt",
    "he_ntt", "he_intt", "he_add", "he_sub", "he_pmult", "he_cmult", "he_add_const", "he_moddrop",
    "he_hmult_relin", "he_hmult_relin_rescale", "he_rescale", "he_hrot", "he_hrot_many", "he_rotate_sum",
    "he_add_batch", "he_sub_batch", "he_pmult_batch", "he_cmult_batch", "he_add_const_batch", "he_moddrop_batch",
    "he_hmult_relin_batch", "he_hmult_relin_rescale_batch", "he_rescale_batch", "he_hrot_batch", "he_hrot_batch_keys", "he_hrot_batch_levels", "he_rotate_sum_batch",
    "he_hrot_noalloc",
    "he_layer_norm", "he_layer_norm_workspace_bytes", "he_layer_norm_grad", "he_pool", "he_pool_workspace_bytes", "he_pool_grad",
    "he_attention", "he_attention_workspace_bytes", "he_attention_grad",
    "he_profile_start", "he_profile_stop",
]


class HeError(RuntimeError):
    def __init__(self, code: int, where: str, detail: str = ""):
        self.code = code
        super().__init__(f"{where}: {ERRORS.get(code, code)}" + (f" ({detail})" if detail else ""))


class he_kernel_stat(ctypes.Structure):
    _fields_ = [
        ("name", ctypes.c_char * 48), ("launches", ctypes.c_int64), ("total_ms", ctypes.c_double),
        ("bytes", ctypes.c_double),
    ]


# descriptors of the operators on token states, laid out as C does
_ROWS = struct.Struct("@Pq")               # he_rows: d, stride
_HEADS = struct.Struct("@Pqq")             # he_heads: d, row, head
_SPANS = struct.Struct("@PPiq")            # he_spans: d_begin, d_end, count, rows
_NORM = struct.Struct("@iiqid")            # he_norm: type, weight_type, rows, width, eps
_ATTN = struct.Struct("@4iPPiqPPiqddPi4x") # he_attn: type, heads, kv_heads, dim, q, k, scale, cap, d_slopes, fill


class he_params(ctypes.Structure):
    _fields_ = [
        ("logN", ctypes.c_int32), ("L", ctypes.c_int32), ("K", ctypes.c_int32), ("dnum", ctypes.c_int32),
        ("q", ctypes.POINTER(ctypes.c_uint64)), ("p", ctypes.POINTER(ctypes.c_uint64)),
    ]


_lib = None


def load_library() -> ctypes.CDLL:
    """Loads the in-tree HIP library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2210_02574_amd.build` "
                "(hipcc --offload-arch=gfx950); there is no fallback path"
            )
        from .build import is_stale

        if is_stale() and not os.environ.get("HE_ALLOW_STALE_LIB"):
            raise ImportError(
                f"{LIB_PATH} was built from other sources than the present ones: rebuild it with "
                "`python -m paper_2210_02574_amd.build` (or set HE_ALLOW_STALE_LIB=1 to load it anyway)"
            )
        # torch first: it brings its own HIP runtime, and a process must not end up with the system's runtime
        # initialised by this library and torch's by torch (the second one then finds no GPU)
        import torch  # noqa: F401

        lib = ctypes.CDLL(LIB_PATH)
        vp, i32, u64, sz, dbl = ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint64, ctypes.c_size_t, ctypes.c_double
        ds = ctypes.c_char_p
        sig = {
            "he_ctx_create": [ctypes.POINTER(he_params), i32, ctypes.POINTER(vp)],
            "he_ctx_destroy": [vp],
            "he_strerror": [i32],
            "he_last_hip_error": [vp],
            "he_ctx_modulus": [vp, i32, ctypes.POINTER(u64), ctypes.POINTER(u64)],
            "he_ctx_set_conversion": [vp, i32],
            "he_galois_element": [vp, i32, ctypes.POINTER(u64)],
            "he_gauss_cdt": [vp],
            "he_workspace_bytes": [vp, i32, i32, ctypes.POINTER(sz)],
            "he_keygen_secret": [vp, u64, ctypes.POINTER(vp)],
            "he_sk_destroy": [vp],
            "he_sk_coeffs": [vp, vp],
            "he_keygen_relin": [vp, vp, u64, ctypes.POINTER(vp)],
            "he_keygen_rot": [vp, vp, i32, u64, ctypes.POINTER(vp)],
            "he_keygen_conj": [vp, vp, u64, ctypes.POINTER(vp)],
            "he_keygen_secret_sparse": [vp, u64, i32, ctypes.POINTER(vp)],
            "he_modraise": [vp, vp, vp, i32, vp, sz, vp],
            "he_pmult_sum": [vp, vp, vp, i32, vp, i32, vp],
            "he_keygen_public": [vp, vp, u64, vp],
            "he_encrypt_public_coeffs": [vp, vp, vp, i32, u64, vp],
            "he_evk_from_host": [vp, vp, u64, ctypes.POINTER(vp)],
            "he_evk_to_host": [vp, vp],
            "he_evk_destroy": [vp],
            "he_encode": [vp, vp, vp, i32, dbl, vp],
            "he_decode": [vp, vp, dbl, vp, vp],
            "he_plain_to_ntt": [vp, vp, i32, vp],
            "he_encrypt_coeffs": [vp, vp, vp, i32, u64, vp],
            "he_decrypt_coeffs": [vp, vp, vp, i32, vp],
            "he_decrypt": [vp, vp, vp, i32, dbl, vp, vp],
            "he_ntt": [vp, vp, vp, i32, vp],
            "he_intt": [vp, vp, vp, i32, vp],
            "he_add": [vp, vp, vp, vp, i32, vp],
            "he_sub": [vp, vp, vp, vp, i32, vp],
            "he_pmult": [vp, vp, vp, vp, i32, vp],
            "he_cmult": [vp, vp, vp, vp, i32, vp],
            "he_add_const": [vp, vp, vp, vp, i32, vp],
            "he_moddrop": [vp, vp, i32, vp, i32, vp],
            "he_hmult_relin": [vp, vp, vp, vp, vp, i32, vp, sz, vp],
            "he_hmult_relin_rescale": [vp, vp, vp, vp, vp, i32, vp, sz, vp],
            "he_rescale": [vp, vp, vp, i32, vp, sz, vp],
            "he_hrot": [vp, vp, vp, vp, i32, vp, sz, vp],
            "he_hrot_noalloc": [vp, vp, vp, vp, i32, vp],
            "he_hrot_many": [vp, vp, i32, vp, vp, i32, vp, sz, vp],
            "he_rotate_sum": [vp, vp, i32, vp, i32, vp, sz, vp],
            "he_add_batch": [vp, vp, vp, vp, i32, i32, vp],
            "he_sub_batch": [vp, vp, vp, vp, i32, i32, vp],
            "he_pmult_batch": [vp, vp, vp, vp, i32, i32, vp],
            "he_cmult_batch": [vp, vp, vp, vp, i32, i32, vp],
            "he_add_const_batch": [vp, vp, vp, vp, i32, i32, vp],
            "he_moddrop_batch": [vp, vp, i32, vp, i32, i32, vp],
            "he_hmult_relin_batch": [vp, vp, vp, vp, vp, i32, i32, vp, sz, vp],
            "he_hmult_relin_rescale_batch": [vp, vp, vp, vp, vp, i32, i32, vp, sz, vp],
            "he_rescale_batch": [vp, vp, vp, i32, i32, vp, sz, vp],
            "he_hrot_batch": [vp, vp, vp, vp, i32, i32, vp, sz, vp],
            "he_hrot_batch_keys": [vp, vp, vp, vp, i32, i32, vp, sz, vp],
            "he_hrot_batch_levels": [vp, vp, vp, vp, vp, i32, vp, sz, vp],
            "he_rotate_sum_batch": [vp, vp, i32, vp, i32, i32, vp, sz, vp],
            # descriptors go as bytes (ds)
            "he_layer_norm": [vp, ds, ds, ds, vp, vp, ds, ds, vp, vp, vp],
            "he_layer_norm_workspace_bytes": [vp, ds, ctypes.POINTER(sz)],
            "he_layer_norm_grad": [vp, ds, ds, ds, vp, vp, vp, ds, ds, vp, vp, vp, sz, vp],
            "he_pool": [vp, i32, ds, i32, ds, vp, vp, sz, vp],
            "he_pool_workspace_bytes": [vp, ds, i32, ctypes.POINTER(sz)],
            "he_pool_grad": [vp, i32, ds, i32, vp, ds, i32, vp],
            "he_attention": [vp, ds, ds, ds, ds, ds, vp, vp, sz, vp],
            "he_attention_workspace_bytes": [vp, ds, i32, ctypes.POINTER(sz)],
            "he_attention_grad": [vp, ds, ds, ds, ds, ds, ds, vp, ds, ds, ds, vp, sz, vp],
            "he_profile_start": [vp],
            "he_profile_stop": [vp, vp, i32, ctypes.POINTER(i32)],
        }
        for name in SYMBOLS:
            fn = getattr(lib, name)
            fn.argtypes = sig[name]
            fn.restype = i32
        lib.he_strerror.restype = ctypes.c_char_p
        lib.he_last_hip_error.restype = ctypes.c_char_p
        for name in ("he_ctx_destroy", "he_sk_destroy", "he_evk_destroy"):
            getattr(lib, name).restype = None
        _lib = lib
    return _lib


def _hp(a: np.ndarray):
    return ctypes.c_void_p(a.ctypes.data)


class SecretKey:
    def __init__(self, he, handle):
        self.he, self.handle = he, handle

    def coeffs(self) -> np.ndarray:
        out = np.empty(self.he.N, dtype=np.int8)
        self.he._chk(self.he.lib.he_sk_coeffs(self.handle, _hp(out)), "he_sk_coeffs")
        return out

    def __del__(self):
        try:
            self.he.lib.he_sk_destroy(self.handle)
        except Exception:
            pass


class EvalKey:
    def __init__(self, he, handle):
        self.he, self.handle = he, handle

    def to_host(self) -> np.ndarray:
        he = self.he
        out = np.empty((he.dnum, 2, he.M, he.N), dtype=np.uint64)
        he._chk(he.lib.he_evk_to_host(self.handle, _hp(out)), "he_evk_to_host")
        return out

    def __del__(self):
        try:
            self.he.lib.he_evk_destroy(self.handle)
        except Exception:
            pass


class HE:
    """One library context.  device = -1: host functions only; device >= 0: that GPU."""

    def __init__(self, logN: int, q: Sequence[int], p: Sequence[int], dnum: int, device: int = -1):
        self.lib = load_library()
        self.logN, self.N, self.n = logN, 1 << logN, 1 << (logN - 1)
        self.q, self.p = [int(v) for v in q], [int(v) for v in p]
        self.L, self.K, self.M, self.dnum = len(self.q), len(self.p), len(self.q) + len(self.p), dnum
        self.alpha = -(-self.L // dnum)
        self.device = device
        self._qa = (ctypes.c_uint64 * self.L)(*self.q)
        self._pa = (ctypes.c_uint64 * self.K)(*self.p)
        prm = he_params(logN, self.L, self.K, dnum, self._qa, self._pa)
        h = ctypes.c_void_p()
        if device >= 0:
            import torch

            torch.cuda.init()  # torch owns device memory and streams: its runtime comes up before the library's
        rc = self.lib.he_ctx_create(ctypes.byref(prm), device, ctypes.byref(h))
        if rc != HE_OK:
            raise HeError(rc, "he_ctx_create")
        self.ctx = h
        self._ws = None
        self._type_of = None

    @classmethod
    def from_params(cls, params, device: int = -1):
        return cls(params.logN, params.q, params.p, params.dnum, device)

    def __del__(self):
        try:
            self._ws = None
            self.lib.he_ctx_destroy(self.ctx)
        except Exception:
            pass

    def _chk(self, rc: int, where: str):
        if rc != HE_OK:
            detail = self.lib.he_last_hip_error(self.ctx).decode() if rc == -5 else ""
            raise HeError(rc, where, detail)

    # ---- context queries --------------------------------------------------------------------
    def modulus(self, i: int):
        m, psi = ctypes.c_uint64(), ctypes.c_uint64()
        self._chk(self.lib.he_ctx_modulus(self.ctx, i, ctypes.byref(m), ctypes.byref(psi)), "he_ctx_modulus")
        return int(m.value), int(psi.value)

    def set_exact_conversion(self, exact: bool):
        """Selects the corrected base conversions (True) or the fast ones (False, the default) for later calls."""
        self._chk(self.lib.he_ctx_set_conversion(self.ctx, 1 if exact else 0), "he_ctx_set_conversion")

    def galois_element(self, r: int) -> int:
        g = ctypes.c_uint64()
        self._chk(self.lib.he_galois_element(self.ctx, r, ctypes.byref(g)), "he_galois_element")
        return int(g.value)

    def gauss_cdt(self) -> List[int]:
        out = np.empty(38, dtype=np.uint64)
        self._chk(self.lib.he_gauss_cdt(_hp(out)), "he_gauss_cdt")
        return [int(v) for v in out]

    def workspace_bytes(self, level: int, count: int = 1) -> int:
        out = ctypes.c_size_t()
        self._chk(self.lib.he_workspace_bytes(self.ctx, level, count, ctypes.byref(out)), "he_workspace_bytes")
        return int(out.value)

    # ---- host: keys ----------------------------------------------------------------------------
    def keygen_secret(self, seed: int) -> SecretKey:
        h = ctypes.c_void_p()
        self._chk(self.lib.he_keygen_secret(self.ctx, seed, ctypes.byref(h)), "he_keygen_secret")
        return SecretKey(self, h)

    def keygen_secret_sparse(self, seed: int, h: int) -> SecretKey:
        """Secret with exactly h non-zero coefficients (bootstrapping)."""
        hd = ctypes.c_void_p()
        self._chk(self.lib.he_keygen_secret_sparse(self.ctx, seed, h, ctypes.byref(hd)), "he_keygen_secret_sparse")
        return SecretKey(self, hd)

    def keygen_relin(self, sk: SecretKey, seed: int) -> EvalKey:
        h = ctypes.c_void_p()
        self._chk(self.lib.he_keygen_relin(self.ctx, sk.handle, seed, ctypes.byref(h)), "he_keygen_relin")
        return EvalKey(self, h)

    def keygen_rot(self, sk: SecretKey, r: int, seed: int) -> EvalKey:
        h = ctypes.c_void_p()
        self._chk(self.lib.he_keygen_rot(self.ctx, sk.handle, r, seed, ctypes.byref(h)), "he_keygen_rot")
        return EvalKey(self, h)

    def keygen_conj(self, sk: SecretKey, seed: int) -> EvalKey:
        """Key of slot-wise complex conjugation; apply it with hrot / hconj."""
        h = ctypes.c_void_p()
        self._chk(self.lib.he_keygen_conj(self.ctx, sk.handle, seed, ctypes.byref(h)), "he_keygen_conj")
        return EvalKey(self, h)

    def keygen_public(self, sk: SecretKey, seed: int) -> np.ndarray:
        pk = np.empty((2, self.L, self.N), dtype=np.uint64)
        self._chk(self.lib.he_keygen_public(self.ctx, sk.handle, seed, _hp(pk)), "he_keygen_public")
        return pk

    def encrypt_public_coeffs(self, pk: np.ndarray, coeffs: np.ndarray, level: int, seed: int) -> np.ndarray:
        pk = np.ascontiguousarray(pk, dtype=np.uint64)
        assert pk.shape == (2, self.L, self.N)
        m = np.ascontiguousarray(coeffs, dtype=np.int64)
        assert m.shape == (self.N,)
        out = np.empty((2, level, self.N), dtype=np.uint64)
        self._chk(self.lib.he_encrypt_public_coeffs(self.ctx, _hp(pk), _hp(m), level, seed, _hp(out)),
                  "he_encrypt_public_coeffs")
        return out

    def evk_from_host(self, evk: np.ndarray, g: int = 1) -> EvalKey:
        evk = np.ascontiguousarray(evk, dtype=np.uint64)
        assert evk.shape == (self.dnum, 2, self.M, self.N)
        h = ctypes.c_void_p()
        self._chk(self.lib.he_evk_from_host(self.ctx, _hp(evk), g, ctypes.byref(h)), "he_evk_from_host")
        return EvalKey(self, h)

    # ---- host: encode / encrypt / decrypt -----------------------------------------------------------
    def encode(self, z, scale: float) -> np.ndarray:
        z = np.asarray(z)
        re = np.ascontiguousarray(z.real, dtype=np.float64)
        im = np.ascontiguousarray(z.imag, dtype=np.float64) if np.iscomplexobj(z) else None
        out = np.empty(self.N, dtype=np.int64)
        self._chk(
            self.lib.he_encode(self.ctx, _hp(re), _hp(im) if im is not None else None, re.shape[0], scale, _hp(out)),
            "he_encode",
        )
        return out

    def decode(self, coeffs, scale: float) -> np.ndarray:
        m = np.ascontiguousarray(coeffs, dtype=np.float64)
        re, im = np.empty(self.n), np.empty(self.n)
        self._chk(self.lib.he_decode(self.ctx, _hp(m), scale, _hp(re), _hp(im)), "he_decode")
        return re + 1j * im

    def plain_to_ntt(self, coeffs: np.ndarray, level: int) -> np.ndarray:
        m = np.ascontiguousarray(coeffs, dtype=np.int64)
        out = np.empty((level, self.N), dtype=np.uint64)
        self._chk(self.lib.he_plain_to_ntt(self.ctx, _hp(m), level, _hp(out)), "he_plain_to_ntt")
        return out

    def encrypt_coeffs(self, sk: SecretKey, coeffs: np.ndarray, level: int, seed: int) -> np.ndarray:
        m = np.ascontiguousarray(coeffs, dtype=np.int64)
        assert m.shape == (self.N,)
        out = np.empty((2, level, self.N), dtype=np.uint64)
        self._chk(self.lib.he_encrypt_coeffs(self.ctx, sk.handle, _hp(m), level, seed, _hp(out)), "he_encrypt_coeffs")
        return out

    def decrypt_coeffs(self, sk: SecretKey, ct: np.ndarray) -> np.ndarray:
        ct = np.ascontiguousarray(ct, dtype=np.uint64)
        level = ct.shape[1]
        out = np.empty(self.N, dtype=np.float64)
        self._chk(self.lib.he_decrypt_coeffs(self.ctx, sk.handle, _hp(ct), level, _hp(out)), "he_decrypt_coeffs")
        return out

    def decrypt(self, sk: SecretKey, ct: np.ndarray, scale: float) -> np.ndarray:
        ct = np.ascontiguousarray(ct, dtype=np.uint64)
        level = ct.shape[1]
        re, im = np.empty(self.n), np.empty(self.n)
        self._chk(self.lib.he_decrypt(self.ctx, sk.handle, _hp(ct), level, scale, _hp(re), _hp(im)), "he_decrypt")
        return re + 1j * im

    # ---- device plumbing (torch: memory and streams only) ----------------------------------------------
    def to_device(self, a: np.ndarray):
        import torch

        a = np.ascontiguousarray(a, dtype=np.uint64)
        return torch.from_numpy(a.view(np.int64)).to(f"cuda:{self.device}")

    @staticmethod
    def to_host(t) -> np.ndarray:
        return t.detach().cpu().contiguous().numpy().view(np.uint64)

    def empty_ct(self, level: int):
        import torch

        return torch.empty((2, level, self.N), dtype=torch.int64, device=f"cuda:{self.device}")

    def _stream(self):
        import torch

        return ctypes.c_void_p(torch.cuda.current_stream(self.device).cuda_stream)

    def _workspace(self, level: int, count: int = 1):
        """One workspace per stream: calls enqueued on different streams may run concurrently."""
        import torch

        need = self.workspace_bytes(level, count)
        key = torch.cuda.current_stream(self.device).cuda_stream
        if self._ws is None:
            self._ws = {}
        ws = self._ws.get(key)
        if ws is None or ws.numel() * 8 < need:
            self._ws[key] = None
            ws = self._ws[key] = torch.empty(need // 8, dtype=torch.int64, device=f"cuda:{self.device}")
        return ctypes.c_void_p(ws.data_ptr()), ws.numel() * 8

    @staticmethod
    def _dp(t):
        assert t.is_cuda and t.is_contiguous() and t.element_size() == 8
        return ctypes.c_void_p(t.data_ptr())

    # ---- device: polynomial arithmetic --------------------------------------------------------------------
    def ntt(self, limbs, mod_idx: Sequence[int]):
        mi = np.ascontiguousarray(mod_idx, dtype=np.int32)
        assert limbs.numel() == mi.shape[0] * self.N
        self._chk(self.lib.he_ntt(self.ctx, self._dp(limbs), _hp(mi), mi.shape[0], self._stream()), "he_ntt")
        return limbs

    def intt(self, limbs, mod_idx: Sequence[int]):
        mi = np.ascontiguousarray(mod_idx, dtype=np.int32)
        assert limbs.numel() == mi.shape[0] * self.N
        self._chk(self.lib.he_intt(self.ctx, self._dp(limbs), _hp(mi), mi.shape[0], self._stream()), "he_intt")
        return limbs

    def _level(self, ct) -> int:
        assert ct.dim() == 3 and ct.shape[0] == 2 and ct.shape[2] == self.N
        return int(ct.shape[1])

    def add(self, a, b, out=None):
        level = self._level(a)
        assert b.shape == a.shape
        out = self.empty_ct(level) if out is None else out
        self._chk(self.lib.he_add(self.ctx, self._dp(a), self._dp(b), self._dp(out), level, self._stream()), "he_add")
        return out

    def sub(self, a, b, out=None):
        level = self._level(a)
        assert b.shape == a.shape
        out = self.empty_ct(level) if out is None else out
        self._chk(self.lib.he_sub(self.ctx, self._dp(a), self._dp(b), self._dp(out), level, self._stream()), "he_sub")
        return out

    def pmult(self, ct, pt, out=None):
        level = self._level(ct)
        assert tuple(pt.shape) == (level, self.N)
        out = self.empty_ct(level) if out is None else out
        self._chk(
            self.lib.he_pmult(self.ctx, self._dp(ct), self._dp(pt), self._dp(out), level, self._stream()), "he_pmult"
        )
        return out

    def cmult(self, ct, scalars: Sequence[int], out=None):
        level = self._level(ct)
        sc = np.array([int(v) for v in scalars], dtype=np.uint64)
        assert sc.shape == (level,)
        out = self.empty_ct(level) if out is None else out
        self._chk(self.lib.he_cmult(self.ctx, self._dp(ct), _hp(sc), self._dp(out), level, self._stream()), "he_cmult")
        return out

    def add_const(self, ct, scalars: Sequence[int], out=None):
        level = self._level(ct)
        sc = np.array([int(v) for v in scalars], dtype=np.uint64)
        assert sc.shape == (level,)
        out = self.empty_ct(level) if out is None else out
        self._chk(
            self.lib.he_add_const(self.ctx, self._dp(ct), _hp(sc), self._dp(out), level, self._stream()), "he_add_const"
        )
        return out

    def moddrop(self, ct, level: int, out=None):
        in_level = self._level(ct)
        if level == in_level and out is None:
            return ct
        out = self.empty_ct(level) if out is None else out
        self._chk(
            self.lib.he_moddrop(self.ctx, self._dp(ct), in_level, self._dp(out), level, self._stream()), "he_moddrop"
        )
        return out

    # ---- device: hot path ----------------------------------------------------------------------------------------
    def hmult_relin(self, relin: EvalKey, a, b, out=None):
        level = self._level(a)
        assert b.shape == a.shape
        out = self.empty_ct(level) if out is None else out
        ws, wsb = self._workspace(level)
        self._chk(
            self.lib.he_hmult_relin(
                self.ctx, relin.handle, self._dp(a), self._dp(b), self._dp(out), level, ws, wsb, self._stream()
            ),
            "he_hmult_relin",
        )
        return out

    def hmult_relin_rescale(self, relin: EvalKey, a, b, out=None):
        """rescale(hmult_relin(a, b)) in one call (same residues)."""
        level = self._level(a)
        assert b.shape == a.shape
        out = self.empty_ct(level - 1) if out is None else out
        ws, wsb = self._workspace(level)
        self._chk(
            self.lib.he_hmult_relin_rescale(
                self.ctx, relin.handle, self._dp(a), self._dp(b), self._dp(out), level, ws, wsb, self._stream()
            ),
            "he_hmult_relin_rescale",
        )
        return out

    def rescale(self, ct, out=None):
        level = self._level(ct)
        out = self.empty_ct(level - 1) if out is None else out
        ws, wsb = self._workspace(level)
        self._chk(
            self.lib.he_rescale(self.ctx, self._dp(ct), self._dp(out), level, ws, wsb, self._stream()), "he_rescale"
        )
        return out

    def pmult_sum(self, cts, pts, out=None):
        """sum_k cts[k] * pts[k] in one pass (at most 64 terms per call; longer lists are chunked and added)."""
        assert len(cts) == len(pts) and len(cts) >= 1
        level = self._level(cts[0])
        out = self.empty_ct(level) if out is None else out
        acc = None
        for lo in range(0, len(cts), 64):
            c, p = cts[lo:lo + 64], pts[lo:lo + 64]
            ca = (ctypes.c_void_p * len(c))(*[t.data_ptr() for t in c])
            pa = (ctypes.c_void_p * len(p))(*[t.data_ptr() for t in p])
            dst = out if acc is None else self.empty_ct(level)
            self._chk(self.lib.he_pmult_sum(self.ctx, ca, pa, len(c), self._dp(dst), level, self._stream()),
                      "he_pmult_sum")
            acc = dst if acc is None else self.add(acc, dst, out=acc)
        return out

    def modraise(self, ct, level_out: int, out=None):
        """Level-1 ciphertext -> level_out limbs of the same centred coefficients (first step of bootstrapping)."""
        assert self._level(ct) == 1
        out = self.empty_ct(level_out) if out is None else out
        ws, wsb = self._workspace(level_out)
        self._chk(self.lib.he_modraise(self.ctx, self._dp(ct), self._dp(out), level_out, ws, wsb, self._stream()),
                  "he_modraise")
        return out

    def hconj(self, conj: EvalKey, ct, out=None):
        """Complex conjugation of every slot (key from keygen_conj)."""
        return self.hrot(conj, ct, out=out)

    def hrot(self, rot: EvalKey, ct, out=None):
        level = self._level(ct)
        out = self.empty_ct(level) if out is None else out
        ws, wsb = self._workspace(level)
        self._chk(
            self.lib.he_hrot(self.ctx, rot.handle, self._dp(ct), self._dp(out), level, ws, wsb, self._stream()),
            "he_hrot",
        )
        return out

    def hrot_noalloc(self, rot: EvalKey, ct, out):
        """hrot on the library's static scratch array: no workspace, no allocation (the caller passes `out`)."""
        level = self._level(ct)
        assert tuple(out.shape) == tuple(ct.shape)
        self._chk(
            self.lib.he_hrot_noalloc(self.ctx, rot.handle, self._dp(ct), self._dp(out), level, self._stream()),
            "he_hrot_noalloc",
        )
        return out

    def hrot_many(self, rots: Sequence[EvalKey], ct, outs=None):
        level = self._level(ct)
        n = len(rots)
        outs = [self.empty_ct(level) for _ in range(n)] if outs is None else outs
        keys = (ctypes.c_void_p * n)(*[k.handle for k in rots])
        ptrs = (ctypes.c_void_p * n)(*[o.data_ptr() for o in outs])
        ws, wsb = self._workspace(level, min(n, 32))  # room for all rotations: they then share every launch
        self._chk(
            self.lib.he_hrot_many(self.ctx, keys, n, self._dp(ct), ptrs, level, ws, wsb, self._stream()),
            "he_hrot_many",
        )
        return outs

    def rotate_sum(self, rots: Sequence[EvalKey], ct):
        level = self._level(ct)
        n = len(rots)
        keys = (ctypes.c_void_p * n)(*[k.handle for k in rots])
        ws, wsb = self._workspace(level)
        self._chk(
            self.lib.he_rotate_sum(self.ctx, keys, n, self._dp(ct), level, ws, wsb, self._stream()), "he_rotate_sum"
        )
        return ct

    # ---- device: batches [count][2][level][N] ---------------------------------------------------------------------
    def _blevel(self, cts):
        assert cts.dim() == 4 and cts.shape[1] == 2 and cts.shape[3] == self.N and cts.is_contiguous()
        return int(cts.shape[2]), int(cts.shape[0])

    def empty_batch(self, count: int, level: int):
        import torch

        return torch.empty((count, 2, level, self.N), dtype=torch.int64, device=f"cuda:{self.device}")

    def add_batch(self, a, b, out=None):
        level, count = self._blevel(a)
        assert b.shape == a.shape
        out = self.empty_batch(count, level) if out is None else out
        self._chk(self.lib.he_add_batch(self.ctx, self._dp(a), self._dp(b), self._dp(out), level, count, self._stream()),
                  "he_add_batch")
        return out

    def sub_batch(self, a, b, out=None):
        level, count = self._blevel(a)
        assert b.shape == a.shape
        out = self.empty_batch(count, level) if out is None else out
        self._chk(self.lib.he_sub_batch(self.ctx, self._dp(a), self._dp(b), self._dp(out), level, count, self._stream()),
                  "he_sub_batch")
        return out

    def pmult_batch(self, cts, pt, out=None):
        level, count = self._blevel(cts)
        assert tuple(pt.shape) == (level, self.N)
        out = self.empty_batch(count, level) if out is None else out
        self._chk(self.lib.he_pmult_batch(self.ctx, self._dp(cts), self._dp(pt), self._dp(out), level, count,
                                          self._stream()), "he_pmult_batch")
        return out

    def cmult_batch(self, cts, scalars: Sequence[int], out=None):
        level, count = self._blevel(cts)
        sc = np.array([int(v) for v in scalars], dtype=np.uint64)
        assert sc.shape == (level,)
        out = self.empty_batch(count, level) if out is None else out
        self._chk(self.lib.he_cmult_batch(self.ctx, self._dp(cts), _hp(sc), self._dp(out), level, count, self._stream()),
                  "he_cmult_batch")
        return out

    def add_const_batch(self, cts, scalars: Sequence[int], out=None):
        level, count = self._blevel(cts)
        sc = np.array([int(v) for v in scalars], dtype=np.uint64)
        assert sc.shape == (level,)
        out = self.empty_batch(count, level) if out is None else out
        self._chk(self.lib.he_add_const_batch(self.ctx, self._dp(cts), _hp(sc), self._dp(out), level, count,
                                              self._stream()), "he_add_const_batch")
        return out

    def moddrop_batch(self, cts, level: int, out=None):
        in_level, count = self._blevel(cts)
        if level == in_level and out is None:
            return cts
        out = self.empty_batch(count, level) if out is None else out
        self._chk(self.lib.he_moddrop_batch(self.ctx, self._dp(cts), in_level, self._dp(out), level, count,
                                            self._stream()), "he_moddrop_batch")
        return out

    def hmult_relin_batch(self, relin: EvalKey, a, b, out=None):
        level, count = self._blevel(a)
        assert b.shape == a.shape
        out = self.empty_batch(count, level) if out is None else out
        ws, wsb = self._workspace(level, count)
        self._chk(self.lib.he_hmult_relin_batch(self.ctx, relin.handle, self._dp(a), self._dp(b), self._dp(out), level,
                                                count, ws, wsb, self._stream()), "he_hmult_relin_batch")
        return out

    def hmult_relin_rescale_batch(self, relin: EvalKey, a, b, out=None):
        level, count = self._blevel(a)
        assert b.shape == a.shape
        out = self.empty_batch(count, level - 1) if out is None else out
        ws, wsb = self._workspace(level, count)
        self._chk(self.lib.he_hmult_relin_rescale_batch(self.ctx, relin.handle, self._dp(a), self._dp(b), self._dp(out),
                                                        level, count, ws, wsb, self._stream()),
                  "he_hmult_relin_rescale_batch")
        return out

    def rescale_batch(self, cts, out=None):
        level, count = self._blevel(cts)
        out = self.empty_batch(count, level - 1) if out is None else out
        ws, wsb = self._workspace(level, count)
        self._chk(self.lib.he_rescale_batch(self.ctx, self._dp(cts), self._dp(out), level, count, ws, wsb,
                                            self._stream()), "he_rescale_batch")
        return out

    def hrot_batch(self, rot: EvalKey, cts, out=None):
        level, count = self._blevel(cts)
        out = self.empty_batch(count, level) if out is None else out
        ws, wsb = self._workspace(level, count)
        self._chk(self.lib.he_hrot_batch(self.ctx, rot.handle, self._dp(cts), self._dp(out), level, count, ws, wsb,
                                         self._stream()), "he_hrot_batch")
        return out

    def hrot_batch_keys(self, rots: Sequence[EvalKey], cts, out=None):
        """Rotate ciphertext o of the batch with key rots[o]."""
        level, count = self._blevel(cts)
        if len(rots) != count:
            raise ValueError("one key per ciphertext")
        out = self.empty_batch(count, level) if out is None else out
        keys = (ctypes.c_void_p * count)(*[k.handle for k in rots])
        ws, wsb = self._workspace(level, min(count, 32))
        self._chk(self.lib.he_hrot_batch_keys(self.ctx, keys, self._dp(cts), self._dp(out), level, count, ws, wsb,
                                              self._stream()), "he_hrot_batch_keys")
        return out

    def hrot_batch_levels(self, rots: Sequence[EvalKey], levels: Sequence[int], packed, out=None):
        """Rotate ciphertexts of mixed levels packed back to back (`packed`: flat [sum 2 level_o][N] tensor),
        operation o with key rots[o]; returns the results packed the same way."""
        import torch

        lv = np.ascontiguousarray(levels, dtype=np.int32)
        count = lv.shape[0]
        if len(rots) != count:
            raise ValueError("one key per ciphertext")
        assert packed.dim() == 2 and packed.shape[1] == self.N and int(packed.shape[0]) == 2 * int(lv.sum())
        out = torch.empty_like(packed) if out is None else out
        keys = (ctypes.c_void_p * count)(*[k.handle for k in rots])
        ws, wsb = self._workspace(int(lv.max()), min(count, 32))
        self._chk(self.lib.he_hrot_batch_levels(self.ctx, keys, _hp(lv), self._dp(packed), self._dp(out), count, ws, wsb,
                                                self._stream()), "he_hrot_batch_levels")
        return out

    def rotate_sum_batch(self, rots: Sequence[EvalKey], cts):
        level, count = self._blevel(cts)
        n = len(rots)
        keys = (ctypes.c_void_p * n)(*[k.handle for k in rots])
        ws, wsb = self._workspace(level, count)
        self._chk(self.lib.he_rotate_sum_batch(self.ctx, keys, n, self._dp(cts), level, count, ws, wsb, self._stream()),
                  "he_rotate_sum_batch")
        return cts

    # ---- device: from token states to embeddings ------------------------------------------------------------------
    # Floating-point rows on this context's device.  Sequences: an int32 tensor [count + 1] of offsets (sequence i is the rows
    # offsets[i] .. offsets[i + 1]), or a pair (begin, end) of int32 tensors [count] where rows between them belong to none (a
    # padded batch).  An `out` that is given keeps its rows of no sequence; one that is made here has zeros there.
    # Calls on short sentences last as long as this code does, so descriptors are packed as bytes (a ctypes structure takes
    # several times as long to fill) and tensors are asked for each number once.
    def _types(self):
        import torch

        self._t32, self._i32 = torch.float32, torch.int32
        self._empty_like, self._dense = torch.empty_like, torch.contiguous_format
        self._type_of = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}  # HE_F32, HE_F16, HE_BF16
        self._raw_stream = torch._C._cuda_getCurrentRawStream  # of torch.cuda.current_stream, without an object around it
        return self._type_of

    def _type(self, dtype) -> int:
        code = (self._type_of or self._types()).get(dtype)
        if code is None:
            raise ValueError(f"{dtype}: rows are float32, float16 or bfloat16")
        return code

    def _placed(self, t, what: str, dtype=None):
        if t.get_device() != self.device or self.device < 0:
            raise ValueError(f"{what}: on {t.device}, the context is on device {self.device}")
        if dtype is not None and t.dtype != dtype:
            raise ValueError(f"{what}: {t.dtype}, want {dtype}")

    def _rows(self, t, what: str, shape, dtype=None) -> bytes:
        """[rows][width], dense along the width: he_rows."""
        if t.shape != shape or len(shape) != 2:
            raise ValueError(f"{what}: {tuple(t.shape)}, want [rows][width]" + (f" = {tuple(shape)}" if shape != t.shape else ""))
        rows, width = shape
        stride, dense = t.stride()
        if dense != 1 and width > 1:
            raise ValueError(f"{what}: want rows that are dense along the width")
        if t.get_device() != self.device or self.device < 0 or (dtype is not None and t.dtype is not dtype):
            self._placed(t, what, dtype)
        return _ROWS.pack(t.data_ptr(), stride if rows > 1 else width)

    def _vector(self, t, what: str, n: int, dtype) -> int:
        shape = t.shape
        if len(shape) != 1 or shape[0] != n or not t.is_contiguous():
            raise ValueError(f"{what}: want a dense vector of {n}")
        if t.get_device() != self.device or self.device < 0 or (dtype is not None and t.dtype is not dtype):
            self._placed(t, what, dtype)
        return t.data_ptr()

    def _spans(self, offsets, rows: int, what: str = "offsets"):
        """The fields of he_spans."""
        if self._type_of is None:
            self._types()
        if isinstance(offsets, (tuple, list)):
            begin, end = offsets
            if begin.dim() != 1 or end.shape != begin.shape:
                raise ValueError(f"{what}: begin and end are vectors of one length")
            count = begin.shape[0]
            return self._vector(begin, what, count, self._i32), self._vector(end, what, count, self._i32), count, rows
        shape = offsets.shape
        if len(shape) != 1 or shape[0] < 1:
            raise ValueError(f"{what}: want a vector of count + 1 offsets, or a pair of vectors (begin, end)")
        n = shape[0]
        p = self._vector(offsets, what, n, self._i32)
        return p, p + 4, n - 1, rows

    def _scratch(self, like, need: int):
        """A workspace of this call's own, from torch's allocator: calls on other streams and captured graphs have theirs."""
        return like.new_empty((need + 3) // 4, dtype=self._t32) if need else None

    def layer_norm(self, x, weight, bias, residual=None, eps: float = 1e-5, out=None):
        """(x - mean) rstd weight + bias over the last dimension of x [rows][width], of s = x + residual with one (rounded to the type).
        Returns (y, s, mean, rstd); s is x itself without a residual.  Keep s, mean and rstd for layer_norm_backward."""
        dtype, shape = x.dtype, x.shape
        code = self._type(dtype)
        xr = self._rows(x, "x", shape)
        rows, width = shape
        wd = weight.dtype
        w, b = self._vector(weight, "weight", width, None), self._vector(bias, "bias", width, wd)
        rr = sr = None
        s = x
        if residual is not None:
            rr = self._rows(residual, "residual", shape, dtype)
            s = self._empty_like(x, memory_format=self._dense)
            sr = _ROWS.pack(s.data_ptr(), width)
        if out is None:
            y = self._empty_like(x, memory_format=self._dense)
            yr = _ROWS.pack(y.data_ptr(), width)
        else:
            y, yr = out, self._rows(out, "out", shape, dtype)
        mean, rstd = x.new_empty((2, rows), dtype=self._t32).unbind(0)
        rc = self.lib.he_layer_norm(self.ctx, _NORM.pack(code, self._type(wd), rows, width, eps), xr, rr, w, b, yr, sr, mean.data_ptr(), rstd.data_ptr(),
                                    self._raw_stream(self.device))
        if rc:
            self._chk(rc, "he_layer_norm")
        return y, s, mean, rstd

    def layer_norm_backward(self, dy, s, weight, mean, rstd, ds=None):
        """(dx, dweight, dbias) from the gradient of y; ds: a gradient that reaches s from elsewhere, added to dx.  dx is the gradient of x and
        of the residual both."""
        dtype, shape = s.dtype, s.shape
        code = self._type(dtype)
        sr = self._rows(s, "s", shape)
        rows, width = shape
        dyr, ar = self._rows(dy, "dy", shape, dtype), None if ds is None else self._rows(ds, "ds", shape, dtype)
        w, m, r = self._vector(weight, "weight", width, None), self._vector(mean, "mean", rows, self._t32), self._vector(rstd, "rstd", rows, self._t32)
        n = _NORM.pack(code, self._type(weight.dtype), rows, width, 0.0)
        need = ctypes.c_size_t()
        rc = self.lib.he_layer_norm_workspace_bytes(self.ctx, n, need)
        if rc:
            self._chk(rc, "he_layer_norm_workspace_bytes")
        dx = self._empty_like(s, memory_format=self._dense)
        dw, db = weight.new_empty((2, width)).unbind(0)
        ws = self._scratch(s, need.value)
        rc = self.lib.he_layer_norm_grad(self.ctx, n, dyr, sr, w, m, r, ar, _ROWS.pack(dx.data_ptr(), width), dw.data_ptr(), db.data_ptr(),
                                         ws.data_ptr() if ws is not None else None, need.value, self._raw_stream(self.device))
        if rc:
            self._chk(rc, "he_layer_norm_grad")
        return dx, dw, db

    def pool_mean(self, x, offsets, out=None):
        """Mean of the rows of each sequence of x [rows][width]: [count][width] in 32 bits, zeros for an empty sequence."""
        code, shape = self._type(x.dtype), x.shape
        xr = self._rows(x, "x", shape)
        rows, width = shape
        span = self._spans(offsets, rows)
        count, sp = span[2], _SPANS.pack(*span)
        if out is None:
            e = x.new_empty((count, width), dtype=self._t32)
        else:
            e = out
            if e.shape != (count, width) or not e.is_contiguous():
                raise ValueError(f"out: want a dense [{count}][{width}]")
            self._placed(e, "out", self._t32)

        def sizes():
            need = ctypes.c_size_t()
            self._chk(self.lib.he_pool_workspace_bytes(self.ctx, sp, width, need), "he_pool_workspace_bytes")
            return need.value

        self._with_scratch(self.lib.he_pool, sizes, "he_pool", x, code, sp, width, xr, e.data_ptr())
        return e

    def pool_mean_backward(self, de, offsets, rows: int, dtype, out=None):
        """Gradient of pool_mean's x [rows][width], of type dtype, from de [count][width]."""
        code, span = self._type(dtype), self._spans(offsets, rows)
        count = span[2]
        if de.dim() != 2 or de.shape[0] != count or not de.is_contiguous():
            raise ValueError(f"de: want a dense [{count}][width]")
        width = de.shape[1]
        self._placed(de, "de", self._t32)
        if out is None:
            dx = de.new_empty((rows, width), dtype=dtype) if count else de.new_zeros((rows, width), dtype=dtype)
            xr = _ROWS.pack(dx.data_ptr(), width)
        else:
            dx = out
            if tuple(dx.shape) != (rows, width):
                raise ValueError(f"out: want [{rows}][{width}]")
            xr = self._rows(dx, "out", dx.shape, dtype)
        rc = self.lib.he_pool_grad(self.ctx, code, _SPANS.pack(*span), width, de.data_ptr(), xr, out is None, self._raw_stream(self.device))
        if rc:
            self._chk(rc, "he_pool_grad")
        return dx

    def _heads(self, t, what: str, shape, dtype=None) -> bytes:
        """[rows][heads][dim] with a dense last dimension: he_heads."""
        if t.shape != shape or len(shape) != 3:
            raise ValueError(f"{what}: {tuple(t.shape)}, want [rows][heads][dim]" + (f" = {tuple(shape)}" if shape != t.shape else ""))
        row, head, dense = t.stride()
        p = t.data_ptr()
        if t.get_device() != self.device or self.device < 0 or (dtype is not None and t.dtype is not dtype):
            self._placed(t, what, dtype)
        if dense != 1 and shape[2] > 1:
            raise ValueError(f"{what}: the last dimension is not dense")
        if (p | (row | head) * t.element_size()) & 15 and t.numel():
            raise ValueError(f"{what}: address {p:#x} or strides {t.stride()} not in multiples of 16 bytes")
        return _HEADS.pack(p, row, head)

    def _attn(self, q, k, v, offsets, offsets_k, scale, cap, slopes, fill):
        """(he_attn, count of sequences, he_heads of q, k, v)"""
        dtype, shape, kshape = q.dtype, q.shape, k.shape
        code, qh = self._type(dtype), self._heads(q, "q", shape)
        rows, heads, dim = shape
        if len(kshape) != 3 or kshape[2] != dim:
            raise ValueError(f"k: {tuple(kshape)}, want [rows][heads][{dim}]")
        rows_k, kv, _ = kshape
        kh, vh = self._heads(k, "k", kshape, dtype), self._heads(v, "v", kshape, dtype)
        if kv == 0 or heads % kv:
            raise ValueError(f"{heads} query heads on {kv} key heads")
        sq = sk = self._spans(offsets, rows)
        if offsets_k is not None and (offsets_k is not offsets or rows_k != rows):
            sk = self._spans(offsets_k, rows_k, "offsets_k")
            if sk[2] != sq[2]:
                raise ValueError("offsets and offsets_k: another number of sequences")
        elif rows_k != rows:
            raise ValueError("keys of another length than the queries need offsets_k")
        sl = 0 if slopes is None else self._vector(slopes, "slopes", heads, self._t32)
        return _ATTN.pack(code, heads, kv, dim, *sq, *sk, dim**-0.5 if scale is None else scale, cap, sl, fill), sq[2], qh, kh, vh

    def _with_scratch(self, fn, sizes, where: str, like, *args):
        """fn(ctx, *args, workspace, bytes, stream), first without a workspace: most calls take none, and one that does says so before it enqueues
        anything.  sizes() gives the bytes then."""
        rc = fn(self.ctx, *args, None, 0, self._raw_stream(self.device))
        if rc == HE_EWORKSPACE:
            need = sizes()
            ws = self._scratch(like, need)
            rc = fn(self.ctx, *args, ws.data_ptr(), need, self._raw_stream(self.device))
        if rc:
            self._chk(rc, where)

    def _attn_bytes(self, s, backward: bool) -> int:
        need = ctypes.c_size_t()
        rc = self.lib.he_attention_workspace_bytes(self.ctx, s, backward, need)
        if rc:
            self._chk(rc, "he_attention_workspace_bytes")
        return need.value

    def attention(self, q, k, v, offsets, offsets_k=None, scale=None, cap: float = 0.0, slopes=None, out=None):
        """Attention inside each sequence: q [rows][heads][dim], k and v [rows_k][kv_heads][dim] (strided views of a joint projection are fine;
        query head h reads key head h // (heads / kv_heads)).  offsets_k: the sequences of the keys, where they are not the queries'.
        scale: of the products, 1 / sqrt(dim) by default; cap > 0: cap tanh(score / cap); slopes [heads] float32: minus slope times distance.
        Returns (o, lse): o like q, lse [heads][rows] float32."""
        s, count, qh, kh, vh = self._attn(q, k, v, offsets, offsets_k, scale, cap, slopes, out is None)
        shape = q.shape
        lse = q.new_empty((shape[1], shape[0]), dtype=self._t32)
        if out is None:
            o = self._empty_like(q, memory_format=self._dense) if count else q.new_zeros(shape)
            oh = _HEADS.pack(o.data_ptr(), shape[1] * shape[2], shape[2])
        else:
            o, oh = out, self._heads(out, "out", shape, q.dtype)
        if out is not None or not count:
            lse.fill_(float("-inf"))
        self._with_scratch(self.lib.he_attention, lambda: self._attn_bytes(s, False), "he_attention", q, s, qh, kh, vh, oh, lse.data_ptr())
        return o, lse

    def attention_backward(self, do, q, k, v, o, lse, offsets, offsets_k=None, scale=None, cap: float = 0.0, slopes=None, out=None,
                           fill=None):
        """(dq, dk, dv) from the gradient of o, with o and lse of the forward call and its other arguments.  out: three tensors (strided views are
        fine) to write them to; fill: whether their rows of no sequence become zeros (by default where they are made here).  Slopes are constants:
        they have no gradient."""
        s, count, qh, kh, vh = self._attn(q, k, v, offsets, offsets_k, scale, cap, slopes, out is None if fill is None else bool(fill))
        dtype, shape = q.dtype, q.shape
        gh, oh = self._heads(do, "do", shape, dtype), self._heads(o, "o", shape, dtype)
        if lse.shape != (shape[1], shape[0]) or not lse.is_contiguous():
            raise ValueError("lse: want a dense [heads][rows]")
        self._placed(lse, "lse", self._t32)
        if out is None:
            dq, dk, dv = [self._empty_like(t, memory_format=self._dense) if count else t.new_zeros(t.shape) for t in (q, k, v)]
            kv = k.shape[1] * shape[2]
            gq, gk, gv = (_HEADS.pack(t.data_ptr(), n, shape[2]) for t, n in ((dq, shape[1] * shape[2]), (dk, kv), (dv, kv)))
        else:
            dq, dk, dv = out
            if not count and fill:  # the library writes nothing without sequences
                for t in out:
                    t.zero_()
            gq, gk, gv = self._heads(dq, "dq", shape, dtype), self._heads(dk, "dk", k.shape, dtype), self._heads(dv, "dv", k.shape, dtype)
        n = self._attn_bytes(s, True)
        ws = self._scratch(q, n)
        rc = self.lib.he_attention_grad(self.ctx, s, gh, qh, kh, vh, oh, lse.data_ptr(), gq, gk, gv, ws.data_ptr() if ws is not None else None, n,
                                        self._raw_stream(self.device))
        if rc:
            self._chk(rc, "he_attention_grad")
        return dq, dk, dv

    # ---- measurement -------------------------------------------------------------------------------------------------
    def profile_start(self):
        self._chk(self.lib.he_profile_start(self.ctx), "he_profile_start")

    def profile_stop(self):
        """Per-kernel {name: (launches, total_ms, bytes)} since profile_start."""
        buf = (he_kernel_stat * 64)()
        n = ctypes.c_int32()
        self._chk(self.lib.he_profile_stop(self.ctx, buf, 64, ctypes.byref(n)), "he_profile_stop")
        return {buf[i].name.decode(): (int(buf[i].launches), float(buf[i].total_ms), float(buf[i].bytes))
                for i in range(n.value)}
