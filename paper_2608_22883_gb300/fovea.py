"""Thin ctypes binding of libfovea (include/fovea.h).

Argument marshalling only: every step of the path runs in the library's CUDA
kernels.  PyTorch provides device memory (tensors, workspaces) and streams.
If the library has not been built this module raises at first use: there is
no CPU fallback.
"""

from __future__ import annotations

import ctypes
import functools
import os
from typing import Dict, Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "_lib", "libfovea.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_CUDA, ERR_OOM, ERR_TIMEOUT = range(6)
STATUS_NAMES = {0: "OK", 1: "INVALID_ARG", 2: "UNSUPPORTED", 3: "CUDA", 4: "OOM", 5: "TIMEOUT"}
BF16, FP32, E4M3 = 0, 1, 2
MAX_D, MAX_H, MAX_K, MAX_ENTRIES, MAX_SEQ = 8192, 4096, 1024, 32768, 512

# Field order of fovea_params after the scalar header (C struct order).
PARAM_NAMES = (
    "ln_v_gamma", "ln_v_beta", "W_K", "W_U",
    "ln_h_gamma", "ln_h_beta", "E_dep", "W_Q",
    "W_f1", "b_f1", "W_f2", "b_f2",
    "W_g1", "b_g1", "w_g2", "b_g2",
    "rms_gamma",
)

EXPORTS = (
    "fovea_build_memory", "fovea_memory_destroy", "fovea_memory_info", "fovea_memory_tensors",
    "fovea_workspace_size", "fovea_workspace_init", "fovea_retrieve_fuse", "fovea_sync_errors",
    "fovea_last_error", "fovea_timing_enable", "fovea_timing_read", "fovea_version",
    "fovea_retrieve_fuse_noalloc", "fovea_noalloc_sync_errors", "fovea_memory_folded_keys",
    "fovea_lm_head_topk", "fovea_debug_wait_limit", "fovea_lm_head_workspace_size",
    "fovea_add_rms_norm", "fovea_quantize_w4", "fovea_linear_w4", "fovea_token_logprobs",
    "fovea_token_logprobs_grad", "fovea_linear_w4_workspace_size",
)
NOALLOC_WORKSPACE_BYTES = 32 << 20


class FoveaError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


class CParams(ctypes.Structure):
    _fields_ = [("d_model", ctypes.c_int), ("mlp_hidden", ctypes.c_int),
                ("max_depth", ctypes.c_int), ("dtype", ctypes.c_int),
                ("ln_eps", ctypes.c_float), ("rms_eps", ctypes.c_float)] + \
               [(n, ctypes.c_void_p) for n in PARAM_NAMES]


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build(); "
                               "the FOVEA path has no CPU fallback")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32p = ctypes.c_void_p, ctypes.POINTER(ctypes.c_int32)
        L.fovea_build_memory.argtypes = [ctypes.POINTER(CParams), vp, vp, ctypes.c_int, ctypes.c_int,
                                         vp, ctypes.POINTER(vp)]
        L.fovea_memory_destroy.argtypes = [vp]
        L.fovea_memory_destroy.restype = None
        L.fovea_memory_info.argtypes = [vp, ctypes.POINTER(ctypes.c_int), ctypes.POINTER(ctypes.c_int), i32p]
        L.fovea_memory_tensors.argtypes = [vp, ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(vp),
                                           ctypes.POINTER(ctypes.c_int64)]
        L.fovea_memory_folded_keys.argtypes = [vp, vp, ctypes.POINTER(vp)]
        L.fovea_lm_head_topk.argtypes = [vp, ctypes.c_int, ctypes.c_int, ctypes.c_int, vp,
                                         ctypes.c_int, ctypes.c_int, vp, vp, vp, vp,
                                         ctypes.c_size_t, vp]
        L.fovea_workspace_size.argtypes = [ctypes.POINTER(CParams), vp, i32p, ctypes.c_int,
                                           ctypes.POINTER(ctypes.c_size_t)]
        L.fovea_workspace_init.argtypes = [vp, ctypes.c_size_t, vp]
        L.fovea_retrieve_fuse.argtypes = [ctypes.POINTER(CParams), vp, vp, vp, i32p, vp,
                                          ctypes.c_float, ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                          vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        L.fovea_retrieve_fuse_noalloc.argtypes = [ctypes.POINTER(CParams), vp, vp, vp, i32p, vp,
                                                  ctypes.c_float, ctypes.c_int, ctypes.c_int,
                                                  ctypes.c_int, vp, vp, vp, vp, vp, vp]
        L.fovea_retrieve_fuse_noalloc.restype = ctypes.c_int
        L.fovea_lm_head_workspace_size.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                                    ctypes.c_int, ctypes.POINTER(ctypes.c_size_t)]
        L.fovea_lm_head_workspace_size.restype = ctypes.c_int
        L.fovea_noalloc_sync_errors.argtypes = [vp]
        L.fovea_noalloc_sync_errors.restype = ctypes.c_int
        L.fovea_debug_wait_limit.argtypes = [ctypes.c_ulonglong]
        L.fovea_debug_wait_limit.restype = ctypes.c_int
        L.fovea_sync_errors.argtypes = [vp, vp]
        L.fovea_last_error.restype = ctypes.c_char_p
        L.fovea_last_error.argtypes = []
        L.fovea_timing_enable.argtypes = [ctypes.c_int]
        L.fovea_timing_read.argtypes = [ctypes.POINTER(ctypes.c_char_p), ctypes.POINTER(ctypes.c_double),
                                        ctypes.POINTER(ctypes.c_int), ctypes.c_int]
        L.fovea_timing_read.restype = ctypes.c_int
        L.fovea_version.restype = ctypes.c_int
        i, i64, f32 = ctypes.c_int, ctypes.c_int64, ctypes.c_float
        L.fovea_add_rms_norm.argtypes = [vp, i64, vp, i64, vp, i, i, i, f32, vp, vp, vp, vp, i, vp]
        L.fovea_quantize_w4.argtypes = [vp, i64, i, i, i, i, vp, vp, vp, vp]
        L.fovea_linear_w4.argtypes = [vp, i64, i, vp, i, i, vp, vp, vp, vp, i, i, i, vp, i, vp,
                                      ctypes.c_size_t, vp]
        L.fovea_linear_w4_workspace_size.argtypes = [i, i, i, i, i, ctypes.POINTER(ctypes.c_size_t)]
        L.fovea_token_logprobs.argtypes = [vp, i64, i, i, i, vp, vp, i64, vp, i, i, vp, vp, vp, vp,
                                           vp, vp, vp]
        L.fovea_token_logprobs_grad.argtypes = [vp, i64, i, i, i, vp, vp, i64, vp, vp, vp, vp, i,
                                                vp, vp, i, vp, vp, vp, vp]
        for name in ("fovea_build_memory", "fovea_memory_info", "fovea_memory_tensors",
                     "fovea_memory_folded_keys", "fovea_lm_head_topk",
                     "fovea_workspace_size", "fovea_workspace_init", "fovea_retrieve_fuse",
                     "fovea_sync_errors", "fovea_timing_enable", "fovea_add_rms_norm",
                     "fovea_quantize_w4", "fovea_linear_w4", "fovea_token_logprobs",
                     "fovea_token_logprobs_grad", "fovea_linear_w4_workspace_size"):
            getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


def _check(status: int):
    if status != OK:
        raise FoveaError(status, lib().fovea_last_error().decode())


def last_error() -> str:
    return lib().fovea_last_error().decode()


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensors passed to libfovea must be contiguous")
    return t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else stream


def torch_dtype(dtype: int) -> torch.dtype:
    return torch.bfloat16 if dtype == BF16 else torch.float32


class Params:
    """fovea_params over a dict of device tensors named as in PARAM_NAMES."""

    def __init__(self, weights: Dict[str, torch.Tensor], *, d_model: int, mlp_hidden: int = 512,
                 max_depth: int = 6, dtype: int = BF16, ln_eps: float = 1e-5,
                 rms_eps: float = 1e-6):
        self.weights = weights          # keeps the tensors alive
        c = CParams()
        c.d_model, c.mlp_hidden, c.max_depth, c.dtype = d_model, mlp_hidden, max_depth, dtype
        c.ln_eps, c.rms_eps = ln_eps, rms_eps
        for n in PARAM_NAMES:
            t = weights.get(n)
            setattr(c, n, None if t is None else _ptr(t))
        self.c = c
        self.d_model, self.mlp_hidden, self.max_depth, self.dtype = d_model, mlp_hidden, max_depth, dtype

    @property
    def ref(self):
        return ctypes.byref(self.c)


class _CudaView:
    """__cuda_array_interface__ over library-owned device memory (no copy)."""

    def __init__(self, ptr: int, shape, typestr: str):
        self.__cuda_array_interface__ = {"shape": tuple(shape), "typestr": typestr,
                                         "data": (ptr, False), "version": 3, "strides": None}


class Memory:
    """A fovea_memory handle (library-owned device buffers)."""

    def __init__(self, handle: ctypes.c_void_p, params: Params):
        self.handle = handle
        self.d = params.d_model
        self.dtype = params.dtype
        B, total = ctypes.c_int(), ctypes.c_int()
        _check(lib().fovea_memory_info(handle, ctypes.byref(B), ctypes.byref(total), None))
        self.B, self.total = B.value, total.value
        counts = (ctypes.c_int32 * self.B)()
        _check(lib().fovea_memory_info(handle, None, None, counts))
        self.valid_counts = list(counts)

    def views(self):
        """(keys [total, d], values [total, d], index [total], offsets list) as
        torch views of the handle's device memory (valid while it lives)."""
        k, u, idx = ctypes.c_void_p(), ctypes.c_void_p(), ctypes.c_void_p()
        offs = (ctypes.c_int64 * (self.B + 1))()
        _check(lib().fovea_memory_tensors(self.handle, ctypes.byref(k), ctypes.byref(u),
                                          ctypes.byref(idx), offs))
        if self.total == 0:
            e = torch.empty((0, self.d), dtype=torch_dtype(self.dtype), device="cuda")
            return e, e, torch.empty(0, dtype=torch.int32, device="cuda"), list(offs)
        ts = "<i2" if self.dtype == BF16 else "<f4"

        def view(ptr):
            t = torch.as_tensor(_CudaView(ptr, (self.total, self.d), ts), device="cuda")
            return t.view(torch.bfloat16) if self.dtype == BF16 else t
        index = torch.as_tensor(_CudaView(idx.value, (self.total,), "<i4"), device="cuda")
        return view(k.value), view(u.value), index, list(offs)

    def folded_keys(self, params: Params) -> Optional[torch.Tensor]:
        """The folded keys kappa = W_Q^T k as [total, 2d] bf16 (row i: kappa_hi
        then kappa_lo; a view of the handle's memory) when the memory holds
        them for params' W_Q, else None; a step with these params then scores
        against them."""
        f = ctypes.c_void_p()
        _check(lib().fovea_memory_folded_keys(self.handle, params.c.W_Q, ctypes.byref(f)))
        if not f.value:
            return None
        if self.total == 0:
            return torch.empty((0, 2 * self.d), dtype=torch.bfloat16, device="cuda")
        return torch.as_tensor(_CudaView(f.value, (self.total, 2 * self.d), "<i2"),
                               device="cuda").view(torch.bfloat16)

    def destroy(self):
        if self.handle:
            lib().fovea_memory_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def build_memory(params: Params, v: torch.Tensor, mask: Optional[torch.Tensor] = None,
                 stream=None) -> Memory:
    """fovea_build_memory: v [B, M_max, d] (params dtype), mask [B, M_max] uint8 or None."""
    B, M_max = v.shape[0], v.shape[1]
    out = ctypes.c_void_p()
    _check(lib().fovea_build_memory(params.ref, _ptr(v), _ptr(mask), B, M_max, _stream(stream),
                                    ctypes.byref(out)))
    return Memory(out, params)


def _offsets(row_offsets) -> ctypes.Array:
    vals = [int(x) for x in row_offsets]
    return (ctypes.c_int32 * len(vals))(*vals)


def workspace_size(params: Params, memory: Memory, row_offsets, k_max: int) -> int:
    n = ctypes.c_size_t()
    _check(lib().fovea_workspace_size(params.ref, memory.handle, _offsets(row_offsets), k_max,
                                      ctypes.byref(n)))
    return n.value


def new_workspace(params: Params, memory: Memory, row_offsets, k_max: int, stream=None) -> torch.Tensor:
    """Allocate (torch) and initialise a workspace for these shapes."""
    n = workspace_size(params, memory, row_offsets, k_max)
    ws = torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")
    _check(lib().fovea_workspace_init(_ptr(ws), ws.numel(), _stream(stream)))
    return ws


def _l_max(params: Params, l_max: Optional[int]) -> int:
    return params.max_depth if l_max is None else int(l_max)


def retrieve_fuse(params: Params, memory: Memory, h: torch.Tensor, depth: torch.Tensor,
                  row_offsets, row_scale: Optional[torch.Tensor], rho: float, k_min: int,
                  k_max: int, h_out: torch.Tensor, workspace: torch.Tensor, *,
                  counts: Optional[torch.Tensor] = None, indices: Optional[torch.Tensor] = None,
                  readout: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                  l_max: Optional[int] = None, stream=None, offsets_c=None) -> None:
    """fovea_retrieve_fuse into caller-allocated outputs (asynchronous).
    l_max: depth gate (None: every row is corrected)."""
    offs = offsets_c if offsets_c is not None else _offsets(row_offsets)
    _check(lib().fovea_retrieve_fuse(params.ref, memory.handle, _ptr(h), _ptr(depth), offs,
                                     _ptr(row_scale), float(rho), int(k_min), int(k_max),
                                     _l_max(params, l_max), _ptr(h_out), _ptr(counts),
                                     _ptr(indices), _ptr(readout), _ptr(gate), _ptr(workspace),
                                     workspace.numel(), _stream(stream)))


def step(params: Params, memory: Memory, h: torch.Tensor, depth: torch.Tensor, row_offsets,
         row_scale: Optional[torch.Tensor], rho: float, k_min: int, k_max: int, *,
         workspace: Optional[torch.Tensor] = None, want_readout: bool = True,
         l_max: Optional[int] = None, stream=None) -> Dict[str, torch.Tensor]:
    """Allocate outputs with torch and run one draft step; returns them."""
    N = h.shape[0]
    dev = h.device
    if workspace is None:
        workspace = new_workspace(params, memory, row_offsets, k_max, stream)
    out = dict(
        h_out=torch.empty_like(h),
        counts=torch.empty(N, dtype=torch.int32, device=dev),
        indices=torch.empty((N, k_max), dtype=torch.int32, device=dev),
        readout=torch.empty((N, params.d_model), dtype=torch.float32, device=dev) if want_readout else None,
        gate=torch.empty(N, dtype=torch.float32, device=dev),
    )
    retrieve_fuse(params, memory, h, depth, row_offsets, row_scale, rho, k_min, k_max,
                  out["h_out"], workspace, counts=out["counts"], indices=out["indices"],
                  readout=out["readout"], gate=out["gate"], l_max=l_max, stream=stream)
    out["workspace"] = workspace
    return out


def retrieve_fuse_noalloc(params: Params, memory: Memory, h: torch.Tensor, depth: torch.Tensor,
                          row_offsets, row_scale: Optional[torch.Tensor], rho: float, k_min: int,
                          k_max: int, h_out: torch.Tensor, *,
                          counts: Optional[torch.Tensor] = None,
                          indices: Optional[torch.Tensor] = None,
                          readout: Optional[torch.Tensor] = None,
                          gate: Optional[torch.Tensor] = None, l_max: Optional[int] = None,
                          stream=None) -> None:
    """fovea_retrieve_fuse_noalloc: the draft step with the library's static
    scratch instead of a workspace (for callers that cannot allocate)."""
    _check(lib().fovea_retrieve_fuse_noalloc(params.ref, memory.handle, _ptr(h), _ptr(depth),
                                             _offsets(row_offsets), _ptr(row_scale), float(rho),
                                             int(k_min), int(k_max), _l_max(params, l_max),
                                             _ptr(h_out), _ptr(counts), _ptr(indices),
                                             _ptr(readout), _ptr(gate), _stream(stream)))


def noalloc_sync_errors(stream=None) -> None:
    """fovea_noalloc_sync_errors: read and clear the static array's error word."""
    _check(lib().fovea_noalloc_sync_errors(_stream(stream)))


def workspace_init(workspace: torch.Tensor, stream=None) -> None:
    """fovea_workspace_init: write the header of a workspace."""
    _check(lib().fovea_workspace_init(_ptr(workspace), workspace.numel(), _stream(stream)))


def sync_errors(workspace: torch.Tensor, stream=None) -> None:
    _check(lib().fovea_sync_errors(_ptr(workspace), _stream(stream)))


def debug_wait_limit(limit_ns: int) -> None:
    """fovea_debug_wait_limit: limit of the bounded device waits of later
    launches (0: the default of about 2 s).  For tests of the timeout path."""
    _check(lib().fovea_debug_wait_limit(int(limit_ns)))


def lm_head_workspace(vocab: int, d_model: int, N: int, k_c: int, stream=None) -> torch.Tensor:
    """An initialised workspace for fovea_lm_head_topk of this shape."""
    n = ctypes.c_size_t()
    _check(lib().fovea_lm_head_workspace_size(vocab, d_model, N, k_c, ctypes.byref(n)))
    ws = torch.empty(n.value, dtype=torch.uint8, device="cuda")
    _check(lib().fovea_workspace_init(_ptr(ws), ws.numel(), _stream(stream)))
    return ws


def lm_head_topk(W_LM: torch.Tensor, h_hat: torch.Tensor, k_c: int, workspace: torch.Tensor,
                 logits: Optional[torch.Tensor] = None, stream=None, write_logits: bool = True):
    """fovea_lm_head_topk: z = h_hat W_LM^T [N, V] (fp32) and the k_c largest
    logits per row (token indices, values), descending, smaller index first
    on ties.  Returns (top_idx [N, k_c] int32, top_val [N, k_c], logits);
    with write_logits=False the logits are not written (NULL) and None is
    returned in their place."""
    V, d = W_LM.shape
    N = h_hat.shape[0]
    dt = BF16 if W_LM.dtype == torch.bfloat16 else FP32
    if not write_logits:
        logits = None
    elif logits is None:
        logits = torch.empty((N, V), dtype=torch.float32, device=h_hat.device)
    idx = torch.empty((N, k_c), dtype=torch.int32, device=h_hat.device)
    val = torch.empty((N, k_c), dtype=torch.float32, device=h_hat.device)
    _check(lib().fovea_lm_head_topk(_ptr(W_LM), V, d, dt, _ptr(h_hat), N, k_c,
                                    _ptr(logits) if logits is not None else None,
                                    _ptr(idx), _ptr(val), _ptr(workspace), workspace.numel(),
                                    _stream(stream)))
    return idx, val, logits


# ---------------------------------------------------------------------------
# Operators of the drafter's exit.  All tensors of a call are on the current device.
# ---------------------------------------------------------------------------

_DTYPES = {torch.bfloat16: BF16, torch.float32: FP32, torch.float8_e4m3fn: E4M3}
_ROW_TYPES = (torch.bfloat16, torch.float32)
_X_TYPES = (torch.bfloat16, torch.float32, torch.float8_e4m3fn)


def _refuse(name: str, t, shape, dtypes, dense: bool, device: Optional[int] = None) -> None:
    """The error of a tensor that is not on the GPU (on this one), not of one of these
    types, not of this shape (None: any size), or not contiguous (along its rows)."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if device is not None and t.get_device() != device:
        raise ValueError(f"{name} is on cuda:{t.get_device()}; the others are on cuda:{device}")
    if t.dtype not in dtypes:
        raise ValueError(f"{name} has type {t.dtype}; expected {' or '.join(map(str, dtypes))}")
    have = tuple(t.shape)
    if len(have) != len(shape) or any(w is not None and h != w for h, w in zip(have, shape)):
        raise ValueError(f"{name} has shape {list(have)}; expected {list(shape)} (None: any)")
    if dense and not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if len(have) == 2 and have[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{name} must be contiguous along its rows")


# The checks below cost a call about a third of a microsecond each; _refuse
# finds the words when one fails.

def _need_rows(name: str, t, dtypes, device: Optional[int] = None):
    """t is a CUDA matrix of one of these types with contiguous rows, on this device
    (None: any): its (rows, columns, row stride)."""
    if not isinstance(t, torch.Tensor) or t.dtype not in dtypes or t.dim() != 2 \
            or (not t.is_cuda if device is None else t.get_device() != device):
        _refuse(name, t, (None, None), dtypes, False, device)
    n, m = t.shape
    ld, inner = t.stride()
    if inner != 1 and m > 1:
        _refuse(name, t, (None, None), dtypes, False)
    return n, m, ld if n > 1 else m


def _need(name: str, t, shape, dtype, device: int) -> int:
    """t is a contiguous tensor of this type and shape on this device: its address."""
    if not isinstance(t, torch.Tensor) or t.get_device() != device or t.dtype is not dtype \
            or t.shape != shape or not t.is_contiguous():
        _refuse(name, t, shape, (dtype,), True, device)
    return t.data_ptr()


def _device_of(name: str, t: torch.Tensor) -> int:
    """The device of a call's first tensor: the current one, where the kernels launch."""
    device = t.get_device()
    if device != torch.cuda.current_device():
        raise ValueError(f"{name} is on cuda:{device}, which is not the current device "
                         f"(cuda:{torch.cuda.current_device()})")
    return device


def _side_stream(stream, device, raw, inputs):
    """A call on another stream than the current one: (its handle, an allocator
    from its pool).  The inputs are recorded as used there, so that neither memory
    is reused too early; ordering the streams themselves stays with the caller."""
    side = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
    if side == raw:
        return raw, torch.empty
    s = stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(side, device)
    for t in inputs:
        if t is not None:
            t.record_stream(s)

    def empty(shape, **kw):
        with torch.cuda.stream(s):
            return torch.empty(shape, **kw)
    return side, empty


def _on(stream, device, *inputs):
    """(stream handle, allocator of outputs) of a call; stream None: the current one."""
    raw = torch._C._cuda_getCurrentRawStream(device.index)
    return (raw, torch.empty) if stream is None else _side_stream(stream, device, raw, inputs)


def add_rms_norm(x: torch.Tensor, gamma: torch.Tensor, residual: Optional[torch.Tensor] = None, *,
                 eps: float = 1e-6, want_out: bool = True, q8_group: Optional[int] = None,
                 stream=None) -> Dict[str, Optional[torch.Tensor]]:
    """fovea_add_rms_norm: s = x + residual and y = RMSNorm(s) * gamma for rows
    x [N, d] (bf16 or fp32; rows may be strided).  Returns a dict of
      sum       s in x's type (None without a residual)
      out       y in x's type (None with want_out=False)
      q8        y in 8 bits, float8_e4m3fn, and
      q8_scale  its scales, fp32: [N] for q8_group = 0 (a scale per row), else
                [N, ceil(d / q8_group)] for q8_group of 32, 64 or 128 columns
                (both only when q8_group is given)."""
    N, d, ld = _need_rows("x", x, _ROW_TYPES)
    dt, dev, at = x.dtype, x.device, _device_of("x", x)
    gamma_at = _need("gamma", gamma, (d,), dt, at)
    residual_at, residual_ld = None, 0
    if residual is not None:
        n, m, residual_ld = _need_rows("residual", residual, (dt,), at)
        if n != N or m != d:
            _refuse("residual", residual, (N, d), (dt,), False)
        residual_at = residual.data_ptr()
    elif not want_out and q8_group is None:
        raise ValueError("nothing to compute: no residual, want_out=False and no q8_group")
    if q8_group not in (None, 0, 32, 64, 128):
        raise ValueError(f"q8_group {q8_group} is not None, 0, 32, 64 or 128")
    raw, empty = _on(stream, dev, x, gamma, residual)
    s = out = q8 = scale = None
    s_at = out_at = q8_at = scale_at = None
    if residual is not None:
        s = empty((N, d), dtype=dt, device=dev)
        s_at = s.data_ptr()
    if want_out:
        out = empty((N, d), dtype=dt, device=dev)
        out_at = out.data_ptr()
    r = {"sum": s, "out": out}
    if q8_group is not None:
        r["q8"] = q8 = empty((N, d), dtype=torch.float8_e4m3fn, device=dev)
        r["q8_scale"] = scale = empty((N, -(-d // q8_group)) if q8_group else (N,),
                                      dtype=torch.float32, device=dev)
        q8_at, scale_at = q8.data_ptr(), scale.data_ptr()
    st = lib().fovea_add_rms_norm(x.data_ptr(), ld, residual_at, residual_ld, gamma_at, N, d,
                                  _DTYPES[dt], eps, s_at, out_at, q8_at, scale_at, q8_group or 0, raw)
    if st:
        _check(st)
    return r


def quantize_w4(W: torch.Tensor, group: int = 128, *, symmetric: bool = True,
                stream=None) -> Dict[str, Optional[torch.Tensor]]:
    """fovea_quantize_w4: W [out, in] (bf16 or fp32; in a multiple of 32) in 4
    bits with a scale per `group` (32, 64 or 128) columns.  Returns a dict of
    codes [out, in / 2] uint8 (the even column in the low four bits), scales
    [out, ceil(in / group)] bf16 and zeros (uint8, like scales; None: symmetric,
    8 everywhere), as linear_w4 takes them."""
    out_f, in_f, ld = _need_rows("W", W, _ROW_TYPES)
    if group not in (32, 64, 128):
        raise ValueError(f"group {group} is not 32, 64 or 128")
    dev = W.device
    _device_of("W", W)
    raw, empty = _on(stream, dev, W)
    groups = -(-in_f // group)
    codes = empty((out_f, in_f // 2), dtype=torch.uint8, device=dev)
    scales = empty((out_f, groups), dtype=torch.bfloat16, device=dev)
    zeros = None if symmetric else empty((out_f, groups), dtype=torch.uint8, device=dev)
    st = lib().fovea_quantize_w4(W.data_ptr(), ld, out_f, in_f, _DTYPES[W.dtype], group,
                                 codes.data_ptr(), scales.data_ptr(),
                                 None if symmetric else zeros.data_ptr(), raw)
    if st:
        _check(st)
    return {"codes": codes, "scales": scales, "zeros": zeros}


@functools.lru_cache(maxsize=512)       # a function of its arguments alone
def linear_w4_workspace_size(N: int, in_features: int, group: int = 128,
                             dtype: torch.dtype = torch.bfloat16, x_group: int = 0) -> int:
    """fovea_linear_w4_workspace_size: bytes linear_w4 needs for N rows of x (0:
    none; x_group: group when x_scale has a scale per group)."""
    n = ctypes.c_size_t()
    _check(lib().fovea_linear_w4_workspace_size(N, in_features, group, _DTYPES[dtype], x_group,
                                                ctypes.byref(n)))
    return n.value


def linear_w4(x: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor,
              zeros: Optional[torch.Tensor] = None, *, group: int = 128,
              x_scale: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
              out_dtype: torch.dtype = torch.float32, workspace: Optional[torch.Tensor] = None,
              stream=None) -> torch.Tensor:
    """fovea_linear_w4: y [N, out] = x W^T (+ bias) with W in 4 bits (codes,
    scales, zeros and group as quantize_w4 gives them; a zero point may be up to
    127, the low seven bits of its byte).  x [N, in] is bf16, fp32,
    or float8_e4m3fn with x_scale [N] or [N, ceil(in / group)] fp32 (add_rms_norm's
    q8 and q8_scale); bias [out] fp32; y is fp32 or bf16 (out_dtype).
    workspace: a uint8 tensor of linear_w4_workspace_size bytes (None: allocated
    for the call when one is needed; it needs no workspace_init); sync_errors(workspace)
    tells whether a bounded device wait gave up in a call since the last one, which
    also leaves NaN in y."""
    N, in_f, ld = _need_rows("x", x, _X_TYPES)
    dt, dev, at = x.dtype, x.device, _device_of("x", x)
    if group not in (32, 64, 128):
        raise ValueError(f"group {group} is not 32, 64 or 128")
    out_f = codes.shape[0] if isinstance(codes, torch.Tensor) and codes.dim() == 2 else 0
    codes_at = _need("codes", codes, (out_f, in_f // 2), torch.uint8, at)
    groups = -(-in_f // group)
    scales_at = _need("scales", scales, (out_f, groups), torch.bfloat16, at)
    zeros_at = x_scale_at = bias_at = None
    if zeros is not None:
        zeros_at = _need("zeros", zeros, (out_f, groups), torch.uint8, at)
    x_group = 0
    if (dt is torch.float8_e4m3fn) != (x_scale is not None):
        raise ValueError("x_scale goes with float8_e4m3fn rows, and only with them")
    if x_scale is not None:
        x_group = group if x_scale.dim() == 2 else 0
        x_scale_at = _need("x_scale", x_scale, (N, groups) if x_group else (N,), torch.float32, at)
    if bias is not None:
        bias_at = _need("bias", bias, (out_f,), torch.float32, at)
    if out_dtype not in _ROW_TYPES:
        raise ValueError(f"out_dtype {out_dtype} is neither bf16 nor fp32")
    raw, empty = _on(stream, dev, x, codes, scales, zeros, x_scale, bias, workspace)
    ws_at, ws_bytes = None, 0
    if workspace is not None:
        ws_bytes = workspace.numel()
        ws_at = _need("workspace", workspace, (ws_bytes,), torch.uint8, at)
    else:
        ws_bytes = linear_w4_workspace_size(N, in_f, group, dt, x_group)
        if ws_bytes:
            workspace = empty((ws_bytes,), dtype=torch.uint8, device=dev)
            ws_at = workspace.data_ptr()
    y = empty((N, out_f), dtype=out_dtype, device=dev)
    st = lib().fovea_linear_w4(x.data_ptr(), ld, _DTYPES[dt], x_scale_at, x_group, N, codes_at,
                               scales_at, zeros_at, bias_at, out_f, in_f, group, y.data_ptr(),
                               _DTYPES[out_dtype], ws_at, ws_bytes, raw)
    if st:
        _check(st)
    return y


def _need_scores(logits, tokens, row_scale, allowed):
    """Checks what both score calls take; returns (device, N, vocab, logits' row
    stride, n_tokens, and the addresses of tokens, row_scale and allowed, allowed's
    row stride)."""
    N, V, ld = _need_rows("logits", logits, _ROW_TYPES)
    at = _device_of("logits", logits)
    T, tokens_at, scale_at, allowed_at, allowed_ld = 0, None, None, None, 0
    if tokens is not None:
        T = tokens.shape[1] if isinstance(tokens, torch.Tensor) and tokens.dim() == 2 else 0
        tokens_at = _need("tokens", tokens, (N, T), torch.int32, at)
    if row_scale is not None:
        scale_at = _need("row_scale", row_scale, (N,), torch.float32, at)
    if allowed is not None:
        rows, words, allowed_ld = _need_rows("allowed", allowed, (torch.int32,), at)
        if words != (V + 31) // 32 or rows not in (1, N):
            raise ValueError(f"allowed has shape {list(allowed.shape)}; expected "
                             f"[{N} or 1, {(V + 31) // 32}]")
        allowed_at = allowed.data_ptr()
        if rows == 1:
            allowed_ld = 0
    return at, N, V, ld, T, tokens_at, scale_at, allowed_at, allowed_ld


def token_logprobs(logits: torch.Tensor, tokens: Optional[torch.Tensor] = None, top_k: int = 0, *,
                   row_scale: Optional[torch.Tensor] = None, allowed: Optional[torch.Tensor] = None,
                   stream=None) -> Dict[str, torch.Tensor]:
    """fovea_token_logprobs: under the softmax of z = logits * row_scale over each
    row's allowed tokens (logits [N, vocab] bf16 or fp32, rows may be strided;
    row_scale [N] fp32 inverse temperatures; allowed [N or 1, ceil(vocab / 32)]
    int32 words, bit i % 32 of word i / 32 for token i), a dict of
      logprobs      [N, T] of tokens [N, T] int32 (-1: none, 0; when given)
      lse, entropy  [N]; stats [N, 2]: the largest z and log sum e^(z - it)
      top_idx       [N, top_k] int32, the largest logits' tokens, descending, the
                    smaller token first on ties, -1 past the tokens that have any
                    probability; top_logprobs [N, top_k] (when top_k > 0)."""
    at, N, V, ld, T, tokens_at, scale_at, allowed_at, allowed_ld = _need_scores(logits, tokens, row_scale,
                                                                                allowed)
    dev = logits.device
    raw, empty = _on(stream, dev, logits, tokens, row_scale, allowed)
    f32 = torch.float32
    lse, entropy = empty((N,), dtype=f32, device=dev), empty((N,), dtype=f32, device=dev)
    stats = empty((N, 2), dtype=f32, device=dev)
    r = {"lse": lse, "entropy": entropy, "stats": stats}
    lp_at = idx_at = top_at = None
    if tokens is not None:
        r["logprobs"] = lp = empty((N, T), dtype=f32, device=dev)
        lp_at = lp.data_ptr()
    if top_k > 0:
        r["top_idx"] = idx = empty((N, top_k), dtype=torch.int32, device=dev)
        r["top_logprobs"] = top = empty((N, top_k), dtype=f32, device=dev)
        idx_at, top_at = idx.data_ptr(), top.data_ptr()
    st = lib().fovea_token_logprobs(logits.data_ptr(), ld, N, V, _DTYPES[logits.dtype], scale_at,
                                    allowed_at, allowed_ld, tokens_at, T, top_k, lp_at,
                                    lse.data_ptr(), entropy.data_ptr(), stats.data_ptr(), idx_at,
                                    top_at, raw)
    if st:
        _check(st)
    return r


def token_logprobs_grad(logits: torch.Tensor, stats: torch.Tensor, entropy: torch.Tensor, *,
                        tokens: Optional[torch.Tensor] = None,
                        grad_logprobs: Optional[torch.Tensor] = None,
                        top_idx: Optional[torch.Tensor] = None,
                        grad_top: Optional[torch.Tensor] = None,
                        grad_entropy: Optional[torch.Tensor] = None,
                        grad_lse: Optional[torch.Tensor] = None,
                        row_scale: Optional[torch.Tensor] = None,
                        allowed: Optional[torch.Tensor] = None,
                        out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """fovea_token_logprobs_grad: the gradient [N, vocab] (logits' type) with
    respect to logits of token_logprobs(logits, tokens, top_k, row_scale=...,
    allowed=...), from the stats, entropy and top_idx that call returned and the
    fp32 gradients of its outputs (each may be left out: 0).  `out` takes the
    result when given; it may be logits itself, when dense."""
    if (tokens is None) != (grad_logprobs is None) or (top_idx is None) != (grad_top is None):
        raise ValueError("tokens and grad_logprobs, top_idx and grad_top, go together")
    at, N, V, ld, T, tokens_at, scale_at, allowed_at, allowed_ld = _need_scores(logits, tokens, row_scale,
                                                                                allowed)
    f32 = torch.float32
    stats_at = _need("stats", stats, (N, 2), f32, at)
    entropy_at = _need("entropy", entropy, (N,), f32, at)
    k, glp_at, idx_at, gtop_at, gH_at, glse_at = 0, None, None, None, None, None
    if tokens is not None:
        glp_at = _need("grad_logprobs", grad_logprobs, (N, T), f32, at)
    if top_idx is not None:
        k = top_idx.shape[1] if isinstance(top_idx, torch.Tensor) and top_idx.dim() == 2 else 0
        idx_at = _need("top_idx", top_idx, (N, k), torch.int32, at)
        gtop_at = _need("grad_top", grad_top, (N, k), f32, at)
    if grad_entropy is not None:
        gH_at = _need("grad_entropy", grad_entropy, (N,), f32, at)
    if grad_lse is not None:
        glse_at = _need("grad_lse", grad_lse, (N,), f32, at)
    dt, dev = logits.dtype, logits.device
    raw, empty = _on(stream, dev, logits, stats, entropy, tokens, grad_logprobs, top_idx, grad_top,
                     grad_entropy, grad_lse, row_scale, allowed, out)
    if out is None:
        out = empty((N, V), dtype=dt, device=dev)
    else:
        _need("out", out, (N, V), dt, at)
    st = lib().fovea_token_logprobs_grad(logits.data_ptr(), ld, N, V, _DTYPES[dt], scale_at, allowed_at,
                                         allowed_ld, stats_at, entropy_at, tokens_at, glp_at, T, idx_at,
                                         gtop_at, k, gH_at, glse_at, out.data_ptr(), raw)
    if st:
        _check(st)
    return out


def timing_enable(on: bool = True) -> None:
    _check(lib().fovea_timing_enable(1 if on else 0))


def timing_read() -> Dict[str, tuple]:
    """{kernel name: (total ms, launches)} of launches recorded since enabling."""
    cap = 64
    names = (ctypes.c_char_p * cap)()
    ms = (ctypes.c_double * cap)()
    cnt = (ctypes.c_int * cap)()
    n = lib().fovea_timing_read(names, ms, cnt, cap)
    return {names[i].decode(): (ms[i], cnt[i]) for i in range(min(n, cap))}


def version() -> int:
    return lib().fovea_version()
