"""Thin ctypes binding over libmhclite.so (argument marshalling only).

Every method of :class:`MhcLite` has the name of the C entry point it calls
(``include/mhclite.h``) and passes the tensors' device pointers straight through;
no step of the path runs in Python or on the CPU.  PyTorch supplies device memory
and the CUDA stream.  Without the compiled library or without a CUDA device the
calls raise.  The calls around the stack, made once a token when a model decodes, are
marshalled by a small extension module (``csrc/marshal.cpp``), loaded with the first of
them, the others by ctypes.
"""
from __future__ import annotations

import ctypes as C
import importlib
import math
import os
import threading

_LIB = None
_MARSHAL = None
_PKG_DIR = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG_DIR, "libmhclite.so")

OK, ERR_BAD_ARG, ERR_CUDA, ERR_WORKSPACE, ERR_TIMEOUT, ERR_INDEX = 0, -1, -2, -3, -4, -5


class MhcLiteError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str = ""):
        self.status = status
        super().__init__(f"{where}: status {status} ({status_string(status)}) {detail}".rstrip())


_p, _i, _i64, _f, _d, _sz = C.c_void_p, C.c_int, C.c_int64, C.c_float, C.c_double, C.c_size_t

# name -> (restype, argtypes); mirrors include/mhclite.h
SIGNATURES = {
    "mhclite_create": (_i, [C.POINTER(_p), _i, _i, _i]),
    "mhclite_destroy": (_i, [_p]),
    "mhclite_status_string": (C.c_char_p, [_i]),
    "mhclite_last_error": (C.c_char_p, [_p]),
    "mhclite_perm_table": (_i, [_i, _p]),
    "mhclite_perm_table_device": (_i, [_p, _p]),
    "mhclite_workspace_bytes": (_sz, [_i, _i, _i64, _i]),
    "mhclite_set_workspace": (_i, [_p, _p, _sz]),
    "mhclite_set_perm_subset": (_i, [_p, _i, _p]),
    "mhclite_workspace_bytes_subset": (_sz, [_i, _i, _i64, _i]),
    "mhclite_coeffs_fwd": (_i, [_p, _i64, _p, _p, _p, _p, _p, _f, _p, _p, _p, _p, _p, _p, _p]),
    "mhclite_premix_fwd": (_i, [_p, _i64, _p, _p, _p, _p]),
    "mhclite_postres_fwd": (_i, [_p, _i64, _p, _p, _p, _p, _p, _p]),
    "mhclite_pre_fwd_fused": (_i, [_p, _i64, _p, _p, _p, _p, _p, _f, _p, _p, _p, _p, _p, _p, _p, _p]),
    "mhclite_pre_fwd_fused_ustat": (_i, [_p, _i64, _p, _p, _p, _p, _p, _f, _p, _p, _p, _p, _p, _p, _p, _p, _f, _p]),
    "mhclite_postres_fwd_next_proj": (_i, [_p, _i64, _p, _p, _p, _p, _p, _p, _p, _p]),
    "mhclite_pre_fwd_resume": (_i, [_p, _i64, _p, _p, _p, _f, _p, _p, _p, _p, _p, _p, _p, _p]),
    "mhclite_postres_bwd": (_i, [_p, _i64, _p, _p, _p, _p, _p, _p, _p, _p, _p, _i, _p]),
    "mhclite_premix_bwd": (_i, [_p, _i64, _p, _p, _p, _p, _p, _i, _p]),
    "mhclite_coeffs_bwd": (_i, [_p, _i64, _p, _p, _p, _p, _f, _p, _p, _p, _p, _p, _p, _p, _p, _p, _i,
                                _p, _p, _p, _p, _i, _p]),
    "mhclite_static_scratch_bytes": (_sz, []),
    "mhclite_coeffs_bwd_static": (_i, [_p, _i64, _p, _p, _p, _p, _f, _p, _p, _p, _p, _p, _p, _p, _p, _p, _i,
                                       _p, _p, _p, _p, _i, _p]),
    "mhclite_tail_bwd_fused": (_i, [_p, _i64, _p, _p, _p, _p, _f, _p, _p, _p, _p, _p, _p, _p, _p, _p, _p,
                                    _p, _p, _p, _p, _p, _i, _p]),
    "mhc_sk20_coeffs_fwd": (_i, [_p, _i64, _p, _p, _p, _p, _p, _f, _i, _p, _p, _p, _p, _p, _p]),
    "mhc_sk20_pre_fwd_fused": (_i, [_p, _i64, _p, _p, _p, _p, _p, _f, _i, _p, _p, _p, _p, _p, _p, _p]),
    "mhc_sk20_coeffs_bwd": (_i, [_p, _i64, _p, _p, _p, _p, _p, _f, _i, _p, _p, _p, _p, _p, _p, _p, _p, _i,
                                 _p, _p, _p, _p, _i, _p]),
    "mhc_sk20_tail_bwd_fused": (_i, [_p, _i64, _p, _p, _p, _p, _p, _f, _i, _p, _p, _p, _p, _p, _p, _p, _p, _p,
                                     _p, _p, _p, _p, _p, _i, _p]),
    "mhclite_ds_gap": (_i, [_p, _i64, _p, _p, _p, _p]),
    "mhclite_ds_gap_stats": (_i, [_p, _i64, _p, _p, _p]),
    "mhclite_log_inv_nu_histogram": (_i, [_p, _i64, _p, _i, _f, _f, _p, _p]),
    "mhclite_depth_product": (_i, [_p, _i64, _p, _p, _i, _p]),
    "mhclite_relative_range": (_i, [_p, _i64, _p, _p, _p]),
    "mhclite_step_host_bytes": (_sz, [_i, _i, _i64]),
    "mhclite_step_host": (_i, [_p, _i64, _p, _p, _p, _p, _p, _p, _p, _p, _f, _p, _p, _p, _p, _p, _p, _p, _p, _i,
                               _p, _sz, _p]),
    "mhclite_kernel_launches": (_i64, [_p]),
    "mhclite_device_status": (_i, [_p]),
    "mhclite_set_kernel_timing": (_i, [_p, _i]),
    "mhclite_kernel_time_ms": (_i, [_p, _i, C.POINTER(_f)]),
    "mhclite_set_status_words": (_i, [_p, _p]),
    "mhclite_embed_fwd": (_i, [_p, _i64, _i64, _p, _p, _i, _f, _p, _p]),
    "mhclite_embed_scratch_bytes": (_sz, [_i, _i64, _i64]),
    "mhclite_embed_bwd": (_i, [_p, _i64, _i64, _p, _p, _f, _p, _i, _p, _sz, _p]),
    "mhclite_block_in_fwd": (_i, [_p, _i64, _p, _p, _f, _p, _p, _p]),
    "mhclite_block_scratch_bytes": (_sz, [_i, _i64]),
    "mhclite_block_in_bwd": (_i, [_p, _i64, _p, _p, _p, _p, _p, _p, _i, _p, _sz, _p]),
    "mhclite_block_out_fwd": (_i, [_p, _i64, _p, _p, _p, _p, _f, _f, _p, _p, _p, _p]),
    "mhclite_block_out_bwd": (_i, [_p, _i64, _p, _p, _p, _p, _p, _f, _p, _p, _p, _p, _p, _p, _i, _p, _sz, _p]),
    "mhclite_dropout": (_i, [_p, _i64, _p, _f, _p, _p, _p]),
    "mhclite_linear_ce_scratch_bytes": (_sz, [_i, _i64, _i64, _i]),
    "mhclite_linear_ce_fwd": (_i, [_p, _i64, _i64, _p, _p, _p, _f, _p, _p, _p, _sz, _p]),
    "mhclite_linear_ce_bwd": (_i, [_p, _i64, _i64, _p, _p, _p, _f, _p, _p, _p, _p, _p, _sz, _p]),
    "mhclite_linear_distill_scratch_bytes": (_sz, [_i, _i64, _i64, _i, _i]),
    "mhclite_linear_distill_fwd": (_i, [_p, _i64, _i64, _i, _p, _p, _p, _p, _i, _f, _f, _p, _p, _p, _p, _sz, _p]),
    "mhclite_linear_distill_bwd": (_i, [_p, _i64, _i64, _i, _p, _p, _p, _p, _i, _f, _f, _p, _p, _p, _p, _p, _p, _sz, _p]),
    "mhclite_policy_scratch_bytes": (_sz, [_i64, _i64]),
    "mhclite_policy_loss": (_i, [_p, _i64, _i64, _p, _p, _p, _p, _p, _p, _i, _d, _d, _d, _i, _p, _p, _p, _p, _p, _sz, _p]),
    "mhclite_preference_scratch_bytes": (_sz, [_i64, _i64]),
    "mhclite_preference_loss": (_i, [_p, _i64, _i64, _p, _p, _p, _p, _d, _d, _d, _i, _p, _p, _p, _p, _p, _sz, _p]),
}


def load(path: str | None = None):
    """Loads libmhclite.so (building it with nvcc if it is absent). Raises if that fails."""
    global _LIB
    if _LIB is not None and path is None:
        return _LIB
    path = path or LIB_PATH
    if not os.path.exists(path):
        from . import build as _build
        _build.build()
    lib = C.CDLL(path)
    for name, (res, args) in SIGNATURES.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args
    _LIB = lib
    return lib


def load_marshal():
    """The extension module that marshals the calls around the stack, bound to the loaded library's entry points."""
    global _MARSHAL
    if _MARSHAL is None:
        import torch  # noqa: F401  (its libraries have to be loaded before the extension's)
        lib = load()
        try:
            from . import _marshal
        except ImportError:
            from . import build as _build
            _build.build_marshal()
            importlib.invalidate_caches()
            from . import _marshal
        _marshal.bind({name: C.cast(getattr(lib, name), _p).value for name in SIGNATURES})
        _MARSHAL = _marshal
    return _MARSHAL


def status_string(status: int) -> str:
    return load().mhclite_status_string(int(status)).decode()


def perm_table(n: int):
    """sigma[k, i] of the lexicographically ordered permutations, from the library's host generator."""
    import numpy as np
    buf = np.zeros((math.factorial(n), n), dtype=np.uint8)
    rc = load().mhclite_perm_table(n, buf.ctypes.data)
    if rc:
        raise MhcLiteError(rc, "mhclite_perm_table")
    return buf


def workspace_bytes(n: int, Cc: int, T: int, kind: int = 0) -> int:
    return int(load().mhclite_workspace_bytes(n, Cc, T, kind))


# Status words (8 int32 a context) that kernels report into when a token index or a wait goes wrong.  A captured graph, or work
# queued on any stream, can still report after its context is gone, so the memory is never given back: 32 bytes a context.
_status_slabs: dict = {}                # device -> (tensors [_STATUS_SLAB, 8], rows of the last one in use)
_status_lock = threading.Lock()
_STATUS_SLAB = 128


def _status_words(torch, device: int):
    with _status_lock:
        slabs, used = _status_slabs.get(device, ([], _STATUS_SLAB))
        if used == _STATUS_SLAB:
            slabs, used = slabs + [torch.empty(_STATUS_SLAB, 8, dtype=torch.int32, device=f"cuda:{device}")], 0
        _status_slabs[device] = (slabs, used + 1)
        return slabs[-1][used]


class MhcLite:
    """One library context: n residual streams of C channels on one CUDA device."""

    def __init__(self, n: int, C_: int, device: int = 0):
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("mHC-lite needs a CUDA device; there is no CPU path")
        self._torch = torch
        # the handle itself where torch hands it out: building a Stream object costs a microsecond a call
        self._raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda d: torch.cuda.current_stream(d).cuda_stream)
        self.lib = load()
        self.n, self.C, self.device = n, C_, device
        self.nfact = math.factorial(n)          # residual weights per token (K once a subset is attached)
        self._table = None
        h = _p()
        rc = self.lib.mhclite_create(C.byref(h), n, C_, device)
        if rc:
            raise MhcLiteError(rc, "mhclite_create")
        self._h = h
        self._ws = None
        # status words of the calls around the stack (lookup, loss): part of device_status()
        self._status = _status_words(torch, device)
        self.clear_device_status()

    def __getattr__(self, name):
        # the extension module and its view of the context, with the first call around the stack: the mixing step does
        # without them, and they cost an attribute of the object from then on
        if name not in ("_m", "_c"):
            raise AttributeError(f"{type(self).__name__!r} object has no attribute {name!r}")
        self._m = load_marshal()
        if "_c" not in self.__dict__:
            self._c = self._m.make(self._h.value, self.device, self.n, self.C)
        return self.__dict__[name]

    def close(self):
        if getattr(self, "_h", None):
            self.lib.mhclite_destroy(self._h)
            self._h = self._c = None

    __del__ = close

    # -- helpers ---------------------------------------------------------------------------------
    def _check(self, rc: int, where: str):
        if rc:
            raise MhcLiteError(rc, where, self.lib.mhclite_last_error(self._h).decode())

    def _ptr(self, t, dtype=None):
        if t is None:
            return None
        torch = self._torch
        if not t.is_cuda or t.device.index != self.device or not t.is_contiguous():
            raise ValueError("expected a contiguous tensor on cuda:%d" % self.device)
        if dtype is not None and t.dtype != dtype:
            raise ValueError(f"expected dtype {dtype}, got {t.dtype}")
        return t.data_ptr()

    def _stream(self):
        return self._raw_stream(self.device)

    def n_cols(self, kind: int = 0) -> int:
        return (self.nfact if kind == 0 else self.n * self.n) + 2 * self.n

    def set_perm_subset(self, table):
        """Attaches a table [K, n] (uint8 tensor on the device, or None) of K distinct permutations:
        Eq. (5) then runs over those K matrices only (paper Section 5)."""
        if table is None:
            self._check(self.lib.mhclite_set_perm_subset(self._h, 0, None), "mhclite_set_perm_subset")
            self._table, self.nfact = None, math.factorial(self.n)
            return
        if table.dtype != self._torch.uint8 or table.dim() != 2 or table.shape[1] != self.n:
            raise ValueError("expected a uint8 tensor of shape [K, n]")
        self._check(self.lib.mhclite_set_perm_subset(self._h, table.shape[0], self._ptr(table)), "mhclite_set_perm_subset")
        self._table, self.nfact = table, int(table.shape[0])

    def ensure_workspace(self, T: int, kind: int = 0):
        """Allocates (with torch) and attaches scratch large enough for T tokens."""
        lite = (workspace_bytes(self.n, self.C, T, 0) if self._table is None else
                int(self.lib.mhclite_workspace_bytes_subset(self.n, self.C, T, self.nfact)))
        need = max(lite, workspace_bytes(self.n, self.C, T, kind) if kind else 0)
        if self._ws is None or self._ws.numel() < need:
            self._ws = self._torch.empty(need + 256, dtype=self._torch.uint8, device=f"cuda:{self.device}")
            base = self._ws.data_ptr()
            self._ws_off = (-base) % 256
            self._check(self.lib.mhclite_set_workspace(self._h, base + self._ws_off, need), "mhclite_set_workspace")
        return need

    def perm_table_device(self):
        import numpy as np
        buf = np.zeros((self.nfact, self.n), dtype=np.uint8)
        self._check(self.lib.mhclite_perm_table_device(self._h, buf.ctypes.data), "mhclite_perm_table_device")
        return buf

    # -- forward ---------------------------------------------------------------------------------
    def coeffs_fwd(self, x, W, b, alpha, gain, eps, H_res, H_pre, H_post, a_saved, p_saved, rstd):
        t, f, h = self._torch, self._torch.float32, self._torch.bfloat16
        self.ensure_workspace(x.shape[0], 0)
        self._check(self.lib.mhclite_coeffs_fwd(
            self._h, x.shape[0], self._ptr(x, h), self._ptr(W, f), self._ptr(b, f), self._ptr(alpha, f),
            self._ptr(gain, f), float(eps), self._ptr(H_res, f), self._ptr(H_pre, f), self._ptr(H_post, f),
            self._ptr(a_saved, f), self._ptr(p_saved, f), self._ptr(rstd, f), self._stream()), "mhclite_coeffs_fwd")

    def premix_fwd(self, x, H_pre, u):
        f, h = self._torch.float32, self._torch.bfloat16
        self._check(self.lib.mhclite_premix_fwd(self._h, x.shape[0], self._ptr(x, h), self._ptr(H_pre, f),
                                                self._ptr(u, h), self._stream()), "mhclite_premix_fwd")

    def postres_fwd(self, x, y, H_res, H_post, x_next):
        f, h = self._torch.float32, self._torch.bfloat16
        self._check(self.lib.mhclite_postres_fwd(self._h, x.shape[0], self._ptr(x, h), self._ptr(y, h),
                                                 self._ptr(H_res, f), self._ptr(H_post, f), self._ptr(x_next, h),
                                                 self._stream()), "mhclite_postres_fwd")

    def pre_fwd_fused(self, x, W, b, alpha, gain, eps, H_res, H_pre, H_post, a_saved, p_saved, rstd, u):
        f, h = self._torch.float32, self._torch.bfloat16
        self._check(self.lib.mhclite_pre_fwd_fused(
            self._h, x.shape[0], self._ptr(x, h), self._ptr(W, f), self._ptr(b, f), self._ptr(alpha, f),
            self._ptr(gain, f), float(eps), self._ptr(H_res, f), self._ptr(H_pre, f), self._ptr(H_post, f),
            self._ptr(a_saved, f), self._ptr(p_saved, f), self._ptr(rstd, f), self._ptr(u, h), self._stream()),
            "mhclite_pre_fwd_fused")

    def pre_fwd_fused_ustat(self, x, W, b, alpha, gain, eps, H_res, H_pre, H_post, a_saved, p_saved, rstd, u, u_rstd,
                            eps_u):
        f, h = self._torch.float32, self._torch.bfloat16
        self._check(self.lib.mhclite_pre_fwd_fused_ustat(
            self._h, x.shape[0], self._ptr(x, h), self._ptr(W, f), self._ptr(b, f), self._ptr(alpha, f),
            self._ptr(gain, f), float(eps), self._ptr(H_res, f), self._ptr(H_pre, f), self._ptr(H_post, f),
            self._ptr(a_saved, f), self._ptr(p_saved, f), self._ptr(rstd, f), self._ptr(u, h), self._ptr(u_rstd, f),
            float(eps_u), self._stream()), "mhclite_pre_fwd_fused_ustat")

    def postres_fwd_next_proj(self, x, y, H_res, H_post, x_next, W_next, gain_next):
        f, h = self._torch.float32, self._torch.bfloat16
        self.ensure_workspace(x.shape[0], 0)
        self._check(self.lib.mhclite_postres_fwd_next_proj(
            self._h, x.shape[0], self._ptr(x, h), self._ptr(y, h), self._ptr(H_res, f), self._ptr(H_post, f),
            self._ptr(x_next, h), self._ptr(W_next, f), self._ptr(gain_next, f), self._stream()),
            "mhclite_postres_fwd_next_proj")

    def pre_fwd_resume(self, x, b, alpha, eps, H_res, H_pre, H_post, a_saved, p_saved, rstd, u):
        f, h = self._torch.float32, self._torch.bfloat16
        self._check(self.lib.mhclite_pre_fwd_resume(
            self._h, x.shape[0], self._ptr(x, h), self._ptr(b, f), self._ptr(alpha, f), float(eps),
            self._ptr(H_res, f), self._ptr(H_pre, f), self._ptr(H_post, f), self._ptr(a_saved, f), self._ptr(p_saved, f),
            self._ptr(rstd, f), self._ptr(u, h), self._stream()), "mhclite_pre_fwd_resume")

    # -- backward --------------------------------------------------------------------------------
    def postres_bwd(self, x, y, H_res, H_post, g, dy, dH_res, dH_post, dx=None, accumulate_dx=False):
        f, h = self._torch.float32, self._torch.bfloat16
        self._check(self.lib.mhclite_postres_bwd(
            self._h, x.shape[0], self._ptr(x, h), self._ptr(y, h), self._ptr(H_res, f), self._ptr(H_post, f),
            self._ptr(g, h), self._ptr(dy, h), self._ptr(dH_res, f), self._ptr(dH_post, f), self._ptr(dx, h),
            int(accumulate_dx), self._stream()), "mhclite_postres_bwd")

    def premix_bwd(self, x, H_pre, du, dH_pre, dx=None, accumulate_dx=False):
        f, h = self._torch.float32, self._torch.bfloat16
        self._check(self.lib.mhclite_premix_bwd(
            self._h, x.shape[0], self._ptr(x, h), self._ptr(H_pre, f), self._ptr(du, h), self._ptr(dH_pre, f),
            self._ptr(dx, h), int(accumulate_dx), self._stream()), "mhclite_premix_bwd")

    def coeffs_bwd(self, x, W, alpha, gain, eps, a_saved, p_saved, rstd, H_pre, H_post, dH_res, dH_pre, dH_post,
                   dx, accumulate_dx, dW, db, dalpha, dgain, accumulate_params=False):
        f, h = self._torch.float32, self._torch.bfloat16
        self.ensure_workspace(x.shape[0], 0)
        self._check(self.lib.mhclite_coeffs_bwd(
            self._h, x.shape[0], self._ptr(x, h), self._ptr(W, f), self._ptr(alpha, f), self._ptr(gain, f), float(eps),
            self._ptr(a_saved, f), self._ptr(p_saved, f), self._ptr(rstd, f), self._ptr(H_pre, f), self._ptr(H_post, f),
            self._ptr(dH_res, f), self._ptr(dH_pre, f), self._ptr(dH_post, f), self._ptr(dx, h), int(accumulate_dx),
            self._ptr(dW, f), self._ptr(db, f), self._ptr(dalpha, f), self._ptr(dgain, f), int(accumulate_params),
            self._stream()), "mhclite_coeffs_bwd")

    def coeffs_bwd_static(self, x, W, alpha, gain, eps, a_saved, p_saved, rstd, H_pre, H_post, dH_res, dH_pre,
                          dH_post, dx, accumulate_dx, dW, db, dalpha, dgain, accumulate_params=False):
        """coeffs_bwd for callers that cannot allocate: scratch is the library's built-in device array
        (no workspace is attached or touched; sizes beyond the array raise)."""
        f, h = self._torch.float32, self._torch.bfloat16
        self._check(self.lib.mhclite_coeffs_bwd_static(
            self._h, x.shape[0], self._ptr(x, h), self._ptr(W, f), self._ptr(alpha, f), self._ptr(gain, f), float(eps),
            self._ptr(a_saved, f), self._ptr(p_saved, f), self._ptr(rstd, f), self._ptr(H_pre, f), self._ptr(H_post, f),
            self._ptr(dH_res, f), self._ptr(dH_pre, f), self._ptr(dH_post, f), self._ptr(dx, h), int(accumulate_dx),
            self._ptr(dW, f), self._ptr(db, f), self._ptr(dalpha, f), self._ptr(dgain, f), int(accumulate_params),
            self._stream()), "mhclite_coeffs_bwd_static")

    def tail_bwd_fused(self, x, W, alpha, gain, eps, a_saved, p_saved, rstd, H_res, H_pre, H_post, g, du,
                       dH_res, dH_post, dx, dW, db, dalpha, dgain, accumulate_params=False):
        f, h = self._torch.float32, self._torch.bfloat16
        self.ensure_workspace(x.shape[0], 0)
        self._check(self.lib.mhclite_tail_bwd_fused(
            self._h, x.shape[0], self._ptr(x, h), self._ptr(W, f), self._ptr(alpha, f), self._ptr(gain, f), float(eps),
            self._ptr(a_saved, f), self._ptr(p_saved, f), self._ptr(rstd, f), self._ptr(H_res, f), self._ptr(H_pre, f),
            self._ptr(H_post, f), self._ptr(g, h), self._ptr(du, h), self._ptr(dH_res, f), self._ptr(dH_post, f),
            self._ptr(dx, h), self._ptr(dW, f), self._ptr(db, f), self._ptr(dalpha, f), self._ptr(dgain, f),
            int(accumulate_params), self._stream()), "mhclite_tail_bwd_fused")

    # -- SK comparison path ----------------------------------------------------------------------
    def sk20_coeffs_fwd(self, x, W_sk, b_sk, alpha, gain, eps, iters, H_res, H_pre, H_post, p_saved, rstd):
        f, h = self._torch.float32, self._torch.bfloat16
        self._check(self.lib.mhc_sk20_coeffs_fwd(
            self._h, x.shape[0], self._ptr(x, h), self._ptr(W_sk, f), self._ptr(b_sk, f), self._ptr(alpha, f),
            self._ptr(gain, f), float(eps), int(iters), self._ptr(H_res, f), self._ptr(H_pre, f), self._ptr(H_post, f),
            self._ptr(p_saved, f), self._ptr(rstd, f), self._stream()), "mhc_sk20_coeffs_fwd")

    def sk20_pre_fwd_fused(self, x, W_sk, b_sk, alpha, gain, eps, iters, H_res, H_pre, H_post, p_saved, rstd, u):
        f, h = self._torch.float32, self._torch.bfloat16
        self.ensure_workspace(x.shape[0], 1)
        self._check(self.lib.mhc_sk20_pre_fwd_fused(
            self._h, x.shape[0], self._ptr(x, h), self._ptr(W_sk, f), self._ptr(b_sk, f), self._ptr(alpha, f),
            self._ptr(gain, f), float(eps), int(iters), self._ptr(H_res, f), self._ptr(H_pre, f), self._ptr(H_post, f),
            self._ptr(p_saved, f), self._ptr(rstd, f), self._ptr(u, h), self._stream()), "mhc_sk20_pre_fwd_fused")

    def sk20_coeffs_bwd(self, x, W_sk, b_sk, alpha, gain, eps, iters, p_saved, rstd, H_pre, H_post, dH_res, dH_pre,
                        dH_post, dx, accumulate_dx, dW, db, dalpha, dgain, accumulate_params=False):
        f, h = self._torch.float32, self._torch.bfloat16
        self.ensure_workspace(x.shape[0], 1)
        self._check(self.lib.mhc_sk20_coeffs_bwd(
            self._h, x.shape[0], self._ptr(x, h), self._ptr(W_sk, f), self._ptr(b_sk, f), self._ptr(alpha, f),
            self._ptr(gain, f), float(eps), int(iters), self._ptr(p_saved, f), self._ptr(rstd, f), self._ptr(H_pre, f),
            self._ptr(H_post, f), self._ptr(dH_res, f), self._ptr(dH_pre, f), self._ptr(dH_post, f), self._ptr(dx, h),
            int(accumulate_dx), self._ptr(dW, f), self._ptr(db, f), self._ptr(dalpha, f), self._ptr(dgain, f),
            int(accumulate_params), self._stream()), "mhc_sk20_coeffs_bwd")

    def sk20_tail_bwd_fused(self, x, W_sk, b_sk, alpha, gain, eps, iters, p_saved, rstd, H_res, H_pre, H_post, g, du,
                            dH_res, dH_post, dx, dW, db, dalpha, dgain, accumulate_params=False):
        f, h = self._torch.float32, self._torch.bfloat16
        self.ensure_workspace(x.shape[0], 1)
        self._check(self.lib.mhc_sk20_tail_bwd_fused(
            self._h, x.shape[0], self._ptr(x, h), self._ptr(W_sk, f), self._ptr(b_sk, f), self._ptr(alpha, f),
            self._ptr(gain, f), float(eps), int(iters), self._ptr(p_saved, f), self._ptr(rstd, f), self._ptr(H_res, f),
            self._ptr(H_pre, f), self._ptr(H_post, f), self._ptr(g, h), self._ptr(du, h), self._ptr(dH_res, f),
            self._ptr(dH_post, f), self._ptr(dx, h), self._ptr(dW, f), self._ptr(db, f), self._ptr(dalpha, f),
            self._ptr(dgain, f), int(accumulate_params), self._stream()), "mhc_sk20_tail_bwd_fused")

    KERNELS = ("proj_fwd", "act_premix", "postres_fwd", "postres_bwd", "tail_pre", "tail_dx")

    def set_kernel_timing(self, on: bool):
        self._check(self.lib.mhclite_set_kernel_timing(self._h, int(on)), "mhclite_set_kernel_timing")

    def kernel_time_ms(self, kernel: int) -> float:
        ms = _f()
        self._check(self.lib.mhclite_kernel_time_ms(self._h, kernel, C.byref(ms)), "mhclite_kernel_time_ms")
        return float(ms.value)

    def device_status(self):
        """Raises if a kernel recorded a timed-out wait or a token index outside its table (synchronises the device)."""
        self._check(self.lib.mhclite_device_status(self._h), "mhclite_device_status")

    def clear_device_status(self):
        """Forgets what device_status reports, so that later reports are seen: waits for all work queued on the device, then
        attaches the status words anew."""
        self._check(self.lib.mhclite_set_status_words(self._h, self._status.data_ptr()), "mhclite_set_status_words")

    def kernel_launches(self) -> int:
        return int(self.lib.mhclite_kernel_launches(self._h))

    def step_host(self, x_host, y_host, g_host, du_host, W, b, alpha, gain, eps, u_host, x_next_host, dy_host,
                  dx_host, dW, db, dalpha, dgain, accumulate_params=False):
        """One fwd+bwd pass from (pinned) HOST activation tensors; device staging is kept on the context."""
        torch, f = self._torch, self._torch.float32
        T = x_host.shape[0]
        for t in (x_host, y_host, g_host, du_host, u_host, x_next_host, dy_host, dx_host):
            if t.is_cuda or t.dtype != torch.bfloat16 or not t.is_contiguous():
                raise ValueError("expected contiguous bf16 host tensors")
        self.ensure_workspace(T, 0)
        need = int(self.lib.mhclite_step_host_bytes(self.n, self.C, T))
        if getattr(self, "_staging", None) is None or self._staging.numel() < need + 256:
            self._staging = torch.empty(need + 256, dtype=torch.uint8, device=f"cuda:{self.device}")
        base = self._staging.data_ptr()
        base += (-base) % 256
        self._check(self.lib.mhclite_step_host(
            self._h, T, x_host.data_ptr(), y_host.data_ptr(), g_host.data_ptr(), du_host.data_ptr(),
            self._ptr(W, f), self._ptr(b, f), self._ptr(alpha, f), self._ptr(gain, f), float(eps),
            u_host.data_ptr(), x_next_host.data_ptr(), dy_host.data_ptr(), dx_host.data_ptr(),
            self._ptr(dW, f), self._ptr(db, f), self._ptr(dalpha, f), self._ptr(dgain, f), int(accumulate_params),
            base, need, self._stream()), "mhclite_step_host")

    def ds_gap_stats(self, H_res, stats):
        """stats [4] f32 <- (max l1, sum l1, max column deviation, sum column deviation) over the tokens."""
        f = self._torch.float32
        self._check(self.lib.mhclite_ds_gap_stats(self._h, H_res.shape[0], self._ptr(H_res, f), self._ptr(stats, f),
                                                  self._stream()), "mhclite_ds_gap_stats")

    def log_inv_nu_histogram(self, X, bins, lo, hi, hist):
        """hist [bins + 1] int64 <- histogram of log10(1/nu) of the matrices X[t]; hist[bins] counts nu == 0."""
        self._check(self.lib.mhclite_log_inv_nu_histogram(self._h, X.shape[0], self._ptr(X, self._torch.float32), int(bins),
                                                          float(lo), float(hi), self._ptr(hist, self._torch.int64),
                                                          self._stream()), "mhclite_log_inv_nu_histogram")

    def depth_product(self, H_res, P, first=False):
        """P[t] <- H_res[t] P[t] in place (P[t] <- H_res[t] when first)."""
        f = self._torch.float32
        self._check(self.lib.mhclite_depth_product(self._h, H_res.shape[0], self._ptr(H_res, f), self._ptr(P, f),
                                                   int(first), self._stream()), "mhclite_depth_product")

    def relative_range(self, X, nu):
        f = self._torch.float32
        self._check(self.lib.mhclite_relative_range(self._h, X.shape[0], self._ptr(X, f), self._ptr(nu, f),
                                                    self._stream()), "mhclite_relative_range")

    def ds_gap(self, H_res, l1_err=None, colsum_dev=None):
        f = self._torch.float32
        self._check(self.lib.mhclite_ds_gap(self._h, H_res.shape[0], self._ptr(H_res, f), self._ptr(l1_err, f),
                                            self._ptr(colsum_dev, f), self._stream()), "mhclite_ds_gap")

    # -- around the stack: lookup, block norms, dropout, loss ------------------------------------------
    # Every tensor is contiguous, on the context's device, and of exactly the stated type and shape (ValueError otherwise).
    # Scratch is allocated a call with torch on the current stream, which takes it back in stream order (and keeps it to a
    # captured graph): calls on several streams and several graphs do not share any.
    def embed_fwd(self, ids, E, scale, x0):
        """x0[t,j,:] = bf16(scale * E[ids[t],:]) for the n streams j; ids [T] int64, E fp32 or bf16 [V,C], x0 [T,n,C] bf16."""
        rc = self._m.embed_fwd(self._c, ids, E, scale, x0)
        if rc:
            self._check(rc, "mhclite_embed_fwd")

    def embed_bwd(self, ids, g, scale, dE, accumulate=False):
        """dE[v,:] (+)= scale * sum of g[t,j,:] over the streams j and the tokens t with ids[t] = v; g [T,n,C] bf16,
        dE [V,C] fp32."""
        rc = self._m.embed_bwd(self._c, ids, g, scale, dE, accumulate)
        if rc:
            self._check(rc, "mhclite_embed_bwd")

    def block_in_fwd(self, u, w, eps, v, rstd):
        """v = u rstd w with rstd = (mean u^2 + eps)^-1/2: the norm that opens a sublayer.  u, v [T,C] bf16; w [C], rstd [T]
        fp32."""
        rc = self._m.block_in_fwd(self._c, u, w, eps, v, rstd)
        if rc:
            self._check(rc, "mhclite_block_in_fwd")

    def block_in_bwd(self, u, w, rstd, dv, du, dw, accumulate_params=False):
        """Gradient of block_in_fwd: du [T,C] bf16, dw [C] fp32 from dv [T,C] bf16."""
        rc = self._m.block_in_bwd(self._c, u, w, rstd, dv, du, dw, accumulate_params)
        if rc:
            self._check(rc, "mhclite_block_in_bwd")

    def block_out_fwd(self, o, gate, w, scale, eps, p_drop, rng, y, rstd):
        """y = scale * dropout(sigmoid(gate) o rstd w): what closes a sublayer before the merge.  gate (bf16 [T,C]) and
        scale (fp32 [1]) may be None; rng is an int64 tensor (seed, offset) on the device, None where p_drop is 0."""
        rc = self._m.block_out_fwd(self._c, o, gate, w, scale, eps, p_drop, rng, y, rstd)
        if rc:
            self._check(rc, "mhclite_block_out_fwd")

    def block_out_bwd(self, o, gate, w, scale, rstd, p_drop, rng, dy, d_o, dgate, dw, dscale, accumulate_params=False):
        """Gradient of block_out_fwd with the same rng values; dgate is given exactly where gate is, dscale may be None."""
        rc = self._m.block_out_bwd(self._c, o, gate, w, scale, rstd, p_drop, rng, dy, d_o, dgate, dw, dscale, accumulate_params)
        if rc:
            self._check(rc, "mhclite_block_out_bwd")

    def dropout(self, x, p, rng, y):
        """y = x / (1 - p) where an element stays, 0 where not; the same call on a gradient is the backward.  x, y: bf16
        of one shape; the mask is a function of rng = (seed, offset), int64 on the device, and is not stored."""
        rc = self._m.dropout(self._c, x, p, rng, y)
        if rc:
            self._check(rc, "mhclite_dropout")

    def linear_ce_fwd(self, h, W, target, logit_scale, loss, lse):
        """loss[t] = lse[t] - l[t, target[t]] and lse[t] = log sum exp l[t,:] of l = logit_scale h W^T, which is not stored;
        h [T,C], W [V,C] bf16, target [T] int64 (negative: no target, loss and lse 0), loss and lse [T] fp32."""
        rc = self._m.linear_ce_fwd(self._c, h, W, target, logit_scale, loss, lse)
        if rc:
            self._check(rc, "mhclite_linear_ce_fwd")

    def linear_ce_bwd(self, h, W, target, logit_scale, lse, dloss, dh, dW):
        """dh [T,C], dW [V,C] bf16 from dloss [T] fp32 and the forward's lse."""
        rc = self._m.linear_ce_bwd(self._c, h, W, target, logit_scale, lse, dloss, dh, dW)
        if rc:
            self._check(rc, "mhclite_linear_ce_bwd")

    def linear_distill_fwd(self, h, W, ids, teacher, logit_scale, temperature, loss, lse, logp):
        """Divergence of a teacher's top entries from the student: with x = logit_scale / temperature h W^T, which is not
        stored, lse[t] = log sum exp x[t,:], logp[t,k] = x[t, ids[t,k]] - lse[t] and p = softmax(teacher / temperature) over a
        row's present entries, loss[t] = sum_k p (log p - logp).  h [T,C], W [V,C] bf16; ids [T,K] int64 (negative: absent,
        logp 0), teacher [T,K] fp32 or bf16; loss, lse [T], logp [T,K] fp32 (0 in rows without a teacher)."""
        rc = self._m.linear_distill_fwd(self._c, h, W, ids, teacher, logit_scale, temperature, loss, lse, logp)
        if rc:
            self._check(rc, "mhclite_linear_distill_fwd")

    def linear_distill_bwd(self, h, W, ids, teacher, logit_scale, temperature, lse, logp, dloss, dh, dW):
        """dh [T,C], dW [V,C] bf16 from dloss [T] fp32 and the forward's lse and logp."""
        rc = self._m.linear_distill_bwd(self._c, h, W, ids, teacher, logit_scale, temperature, lse, logp, dloss, dh, dW)
        if rc:
            self._check(rc, "mhclite_linear_distill_bwd")

    def policy_loss(self, nll, nll_old, nll_ref, target, starts, adv, token_adv, clip_low, clip_high, kl_weight, mean, loss, stats,
                    dloss=None, dnll=None):
        """Clipped policy loss of S sequences with a KL term, and with dloss its gradient: r = exp(nll_old - nll),
        d = nll - nll_ref, loss[s] = sum (mean: mean) over a sequence's tokens with target >= 0 of
        max(-A r, -A clip(r, 1 - clip_low, 1 + clip_high)) + kl_weight (exp(d) - d - 1).  nll, nll_old, nll_ref (or None),
        dnll [T] fp32, target [T] int64, all as linear_ce_fwd takes and leaves them; starts [S+1] int64: sequence s holds the
        tokens starts[s] .. starts[s+1] - 1; adv [S] fp32, or [T] with token_adv; loss, dloss [S], stats [S,3] fp32 (tokens
        that count, clipped ones, sum or mean of the divergence).  dnll is what linear_ce_bwd takes as dloss."""
        rc = self._m.policy_loss(self._c, nll, nll_old, nll_ref, target, starts, adv, token_adv, clip_low, clip_high, kl_weight, mean,
                                 loss, stats, dloss, dnll)
        if rc:
            self._check(rc, "mhclite_policy_loss")

    def preference_loss(self, nll, nll_ref, target, starts, beta, margin, smoothing, mean, loss, reward, dloss=None, dnll=None):
        """Preference loss of P pairs of sequences (2 p chosen, 2 p + 1 rejected; starts [2P+1]), and with dloss its gradient:
        R = sum (mean: mean) of nll_ref - nll over a sequence's tokens with target >= 0, x = beta (R_chosen - R_rejected) -
        margin, loss[p] = -(1 - smoothing) log sigmoid(x) - smoothing log sigmoid(-x), reward[p] = beta R of both.  Without
        nll_ref (None) R is of -nll.  loss, dloss [P], reward [P,2]; the others as in policy_loss."""
        rc = self._m.preference_loss(self._c, nll, nll_ref, target, starts, beta, margin, smoothing, mean, loss, reward, dloss, dnll)
        if rc:
            self._check(rc, "mhclite_preference_loss")
