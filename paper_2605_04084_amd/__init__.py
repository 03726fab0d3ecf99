"""Python binding for libfasq, the MI355X product-quantized matmul library.

The binding marshals arguments only: every computation runs in the HIP
kernels of ``libfasq.so``.  Torch is used for device buffers and streams.
If the library is not built, every call raises :class:`LibraryNotBuilt`;
there is no fallback.

Operation (FASQ, Sec. 3.1.2, Eq. lut-accumulate): ``y = x . W_hat^T`` where
``W_hat[n, s*d + i] = codebook[u(n, s), i]`` and ``u(n, s)`` are packed ids
(8, 12 or 16 bits, one least-significant-bit-first stream per output row).
The encoder (Sec. 3.1.1, Alg. 1) produces the codebook and the ids from dense
weights by k-means.
"""

from __future__ import annotations

import array
import ctypes
import math
import os
import threading
from typing import Optional

__all__ = [
    "FasqError",
    "LibraryNotBuilt",
    "LIB_PATH",
    "lib",
    "library_loaded",
    "abi_version",
    "idx_row_bytes",
    "plan",
    "status_string",
    "last_error",
    "pq_gemv",
    "pq_gemm",
    "pq_reconstruct",
    "pq_gemv_batched",
    "pq_encode",
    "pq_gemv_ex",
    "pq_gemm_lut",
    "gemm_lut_raw",
    "gemv_ex_raw",
    "gemv_ex_workspace_bytes",
    "pq_gemm_ex",
    "gemm_ex_raw",
    "gemm_ex_workspace_bytes",
    "encode_raw",
    "encode_workspace_bytes",
    "gemv_raw",
    "gemv_batched_raw",
    "gemm_raw",
    "reconstruct_raw",
    "FASQ_OK",
    "FASQ_ERR_INVALID_ARG",
    "FASQ_ERR_UNSUPPORTED",
    "FASQ_ERR_HIP",
    "FASQ_ERR_HOST_MEMORY",
    "LaunchList",
    "rope_frequencies",
    "rope_table",
    "rope_append",
    "paged_attention",
    "paged_attention_workspace_bytes",
    "draft_tree",
    "process_logits",
    "process_logits_workspace_bytes",
    "residual_norm",
    "lora_batched",
    "lora_workspace_bytes",
    "EXPORTED_SYMBOLS",
    "ABI_VERSION",
]

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libfasq.so")

ABI_VERSION = 8  # FASQ_ABI_VERSION of include/fasq.h

FASQ_OK = 0
FASQ_ERR_INVALID_ARG = 1
FASQ_ERR_UNSUPPORTED = 2
FASQ_ERR_HIP = 3
FASQ_ERR_HOST_MEMORY = 4

EXPORTED_SYMBOLS = (
    "fasq_pq_gemv",
    "fasq_pq_gemm",
    "fasq_pq_gemv_batched",
    "fasq_pq_reconstruct",
    "fasq_idx_row_bytes",
    "fasq_status_string",
    "fasq_last_error",
    "fasq_abi_version",
    "fasq_pq_plan",
    "fasq_pq_encode",
    "fasq_pq_encode_workspace_bytes",
    "fasq_pq_gemv_ex",
    "fasq_pq_gemv_ex_workspace_bytes",
    "fasq_pq_gemm_lut",
    "fasq_pq_gemm_ex",
    "fasq_pq_gemm_ex_workspace_bytes",
    "fasq_pq_gemv_ex_noalloc",
    "fasq_noalloc_scratch_bytes",
    "fasq_launch_list_create",
    "fasq_launch_list_begin",
    "fasq_launch_list_end",
    "fasq_launch_list_run",
    "fasq_launch_list_size",
    "fasq_launch_list_destroy",
    "fasq_rope_table",
    "fasq_rope_append",
    "fasq_paged_attention",
    "fasq_paged_attention_ex",
    "fasq_paged_attention_workspace_bytes",
    "fasq_process_logits",
    "fasq_process_logits_workspace_bytes",
    "fasq_residual_norm",
    "fasq_lora_batched",
    "fasq_lora_workspace_bytes",
)


class LibraryNotBuilt(ImportError):
    pass


class FasqError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{message} (status {status})")
        self.status = status


_lock = threading.Lock()
_lib: Optional[ctypes.CDLL] = None

_c_i64 = ctypes.c_int64
_c_int = ctypes.c_int
_c_vp = ctypes.c_void_p


class KvCache(ctypes.Structure):
    """``fasq_kv_cache``: the pages of keys and values and their strides (in elements)."""

    _fields_ = [("k", _c_vp), ("v", _c_vp), ("num_pages", _c_i64), ("page_size", _c_i64), ("page_stride", _c_i64),
                ("slot_stride", _c_i64), ("head_stride", _c_i64)]


class AttentionScores(ctypes.Structure):
    """``fasq_attention_scores``: caps, biases and masks of an attention call."""

    _fields_ = [("softcap", ctypes.c_float), ("slopes", _c_vp), ("spans", _c_vp), ("tree", _c_vp), ("tree_stride", _c_i64),
                ("tree_words", _c_i64)]


class TokenRules(ctypes.Structure):
    """``fasq_token_rules``: what stands between logits and tokens."""

    _fields_ = [("requests", _c_vp), ("S", _c_i64), ("tokens", _c_vp), ("token_stride", _c_i64), ("max_tokens", _c_i64),
                ("token_count", _c_vp), ("prompt_len", _c_vp), ("repetition", _c_vp), ("presence", _c_vp),
                ("frequency", _c_vp), ("bias_ids", _c_vp), ("bias_values", _c_vp), ("max_bias", _c_i64),
                ("temperature", _c_vp), ("allowed", _c_vp), ("allowed_stride", _c_i64), ("draft_tokens", _c_vp),
                ("q_start", _c_vp), ("tree", _c_vp), ("tree_stride", _c_i64), ("tree_words", _c_i64)]


def lib() -> ctypes.CDLL:
    """Load ``libfasq.so`` (once) and declare its signatures."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is not None:
            return _lib
        if not os.path.exists(LIB_PATH):
            raise LibraryNotBuilt(f"{LIB_PATH} is missing; build it with __graft_entry__.build()")
        L = ctypes.CDLL(LIB_PATH)
        mm = [_c_vp, _c_i64, _c_i64, _c_i64, _c_vp, _c_int, _c_int, _c_vp, _c_i64, _c_vp, _c_vp]
        for name in ("fasq_pq_gemv", "fasq_pq_gemm", "fasq_pq_gemm_lut"):
            f = getattr(L, name)
            f.argtypes = mm
            f.restype = _c_int
        _pp = ctypes.POINTER(_c_vp)
        _pi64 = ctypes.POINTER(_c_i64)
        L.fasq_pq_gemv_batched.argtypes = [_c_vp, _c_i64, _c_i64, _c_int, _pp, _pi64, _pp, _pi64, _pp, _c_int,
                                           _c_int, _c_vp]
        L.fasq_pq_gemv_batched.restype = _c_int
        L.fasq_pq_reconstruct.argtypes = [_c_vp, _c_i64, _c_i64, _c_int, _c_int, _c_vp, _c_i64, _c_vp, _c_vp]
        L.fasq_pq_reconstruct.restype = _c_int
        L.fasq_idx_row_bytes.argtypes = [_c_i64, _c_int, _c_int]
        L.fasq_idx_row_bytes.restype = _c_i64
        L.fasq_status_string.argtypes = [_c_int]
        L.fasq_status_string.restype = ctypes.c_char_p
        L.fasq_last_error.argtypes = []
        L.fasq_last_error.restype = ctypes.c_char_p
        L.fasq_abi_version.argtypes = []
        L.fasq_abi_version.restype = _c_int
        L.fasq_pq_plan.argtypes = [_c_int, _c_i64, _c_i64, _c_i64, _c_int, _c_int, _c_i64]
        L.fasq_pq_plan.restype = ctypes.c_char_p
        L.fasq_pq_encode.argtypes = [_c_vp, _c_i64, _c_i64, _c_int, _c_i64, _c_int, _c_vp, _c_int, _c_vp, _c_vp,
                                     _c_vp, _c_i64, _c_vp]
        L.fasq_pq_encode.restype = _c_int
        L.fasq_pq_encode_workspace_bytes.argtypes = [_c_i64, _c_i64, _c_int, _c_i64]
        L.fasq_pq_encode_workspace_bytes.restype = _c_i64
        L.fasq_pq_gemv_ex.argtypes = [_c_vp, _c_i64, _c_i64, _c_i64, _c_vp, _c_int, _c_int, _c_vp, _c_i64, _c_i64,
                                      _c_vp, _c_vp, _c_i64, _c_vp]
        L.fasq_pq_gemv_ex.restype = _c_int
        L.fasq_pq_gemv_ex_workspace_bytes.argtypes = [_c_i64, _c_i64, _c_i64, _c_int, _c_int, _c_i64, _c_i64]
        L.fasq_pq_gemv_ex_workspace_bytes.restype = _c_i64
        L.fasq_pq_gemm_ex.argtypes = [_c_vp, _c_i64, _c_i64, _c_i64, _c_vp, _c_int, _c_int, _c_vp, _c_i64, _c_vp,
                                      _c_vp, _c_i64, _c_vp]
        L.fasq_pq_gemm_ex.restype = _c_int
        L.fasq_pq_gemm_ex_workspace_bytes.argtypes = [_c_i64, _c_i64, _c_i64, _c_int, _c_int, _c_i64]
        L.fasq_pq_gemm_ex_workspace_bytes.restype = _c_i64
        L.fasq_pq_gemv_ex_noalloc.argtypes = [_c_vp, _c_i64, _c_i64, _c_i64, _c_vp, _c_int, _c_int, _c_vp, _c_i64,
                                              _c_i64, _c_vp, _c_vp]
        L.fasq_pq_gemv_ex_noalloc.restype = _c_int
        L.fasq_noalloc_scratch_bytes.argtypes = []
        L.fasq_noalloc_scratch_bytes.restype = _c_i64
        L.fasq_launch_list_create.argtypes = [ctypes.POINTER(_c_vp)]
        L.fasq_launch_list_create.restype = _c_int
        for name in ("fasq_launch_list_begin", "fasq_launch_list_end"):
            getattr(L, name).argtypes = [_c_vp]
            getattr(L, name).restype = _c_int
        L.fasq_launch_list_run.argtypes = [_c_vp, _c_vp]
        L.fasq_launch_list_run.restype = _c_int
        L.fasq_launch_list_size.argtypes = [_c_vp]
        L.fasq_launch_list_size.restype = _c_i64
        L.fasq_launch_list_destroy.argtypes = [_c_vp]
        L.fasq_launch_list_destroy.restype = None
        L.fasq_rope_table.argtypes = [ctypes.POINTER(ctypes.c_double), _c_int, _c_i64, ctypes.c_double, _c_vp, _c_vp]
        L.fasq_rope_append.argtypes = [_c_vp, _c_i64, _c_i64, _c_int, _c_vp, _c_i64, _c_i64, _c_vp, _c_i64, _c_i64,
                                       _c_vp, _c_i64, _c_i64, _c_int, _c_i64, _c_int, _c_vp, _c_i64, _c_int, _c_int,
                                       _c_vp, _c_vp, _c_vp, _c_vp, ctypes.c_float, ctypes.POINTER(KvCache), _c_vp]
        L.fasq_paged_attention.argtypes = [_c_vp, _c_i64, _c_i64, _c_i64, _c_int, ctypes.POINTER(KvCache), _c_int,
                                           _c_int, _c_vp, _c_i64, _c_i64, _c_vp, _c_vp, _c_i64, ctypes.c_float, _c_int,
                                           _c_i64, _c_vp, _c_i64, _c_i64, _c_vp, _c_vp, _c_i64, _c_vp]
        L.fasq_paged_attention_ex.argtypes = [_c_vp, _c_i64, _c_i64, _c_i64, _c_int, ctypes.POINTER(KvCache), _c_int,
                                              _c_int, _c_vp, _c_i64, _c_i64, _c_vp, _c_vp, _c_i64, ctypes.c_float,
                                              _c_int, _c_i64, ctypes.POINTER(AttentionScores), _c_vp, _c_i64, _c_i64,
                                              _c_vp, _c_vp, _c_i64, _c_vp]
        L.fasq_process_logits.argtypes = [_c_vp, _c_int, _c_i64, _c_i64, _c_i64, _c_vp, _c_vp, _c_int,
                                          _c_i64, _c_vp, _c_vp, _c_vp, _c_i64, _c_vp]
        L.fasq_process_logits_workspace_bytes.argtypes = [_c_i64, _c_i64]
        L.fasq_paged_attention_workspace_bytes.argtypes = [_c_i64, _c_i64, _c_int, _c_int, _c_int]
        L.fasq_residual_norm.argtypes = [_c_vp, _c_vp, _c_i64, _c_i64, _c_vp, _c_vp, _c_i64, ctypes.c_float, _c_vp,
                                         ctypes.c_float, _c_vp, _c_vp, _c_vp]
        L.fasq_lora_batched.argtypes = [_c_vp, _c_i64, _c_i64, _c_vp, _c_i64, _c_int, _c_vp, _c_int, _c_vp, _c_vp,
                                        _c_vp, _c_vp, _c_vp, _c_vp, _c_i64, _c_vp]
        L.fasq_lora_workspace_bytes.argtypes = [_c_i64, _c_i64, _c_int, _c_int]
        for name in ("fasq_rope_table", "fasq_rope_append", "fasq_paged_attention", "fasq_paged_attention_ex",
                     "fasq_process_logits", "fasq_residual_norm", "fasq_lora_batched"):
            getattr(L, name).restype = _c_int
        for name in ("fasq_paged_attention_workspace_bytes", "fasq_process_logits_workspace_bytes",
                     "fasq_lora_workspace_bytes"):
            getattr(L, name).restype = _c_i64
        _lib = L
        return L


def library_loaded() -> bool:
    return _lib is not None


def abi_version() -> int:
    return lib().fasq_abi_version()


def idx_row_bytes(K: int, d: int, idx_bits: int) -> int:
    return lib().fasq_idx_row_bytes(K, d, idx_bits)


def plan(regime: str, M: int, K: int, N: int, idx_bits: int, d: int, C: int) -> str:
    """Kernel instantiation a call would launch: regime "gemv", "gemm", or
    "gemv_batched" (a grouped decode launch over several matrices of these
    sizes)."""
    code = {"gemv": 0, "gemm": 1, "gemv_batched": 2}[regime]
    return lib().fasq_pq_plan(code, M, K, N, idx_bits, d, C).decode()


def status_string(status: int) -> str:
    return lib().fasq_status_string(status).decode()


def last_error() -> str:
    return lib().fasq_last_error().decode()


def _check(status: int) -> None:
    if status != FASQ_OK:
        raise FasqError(status, f"{status_string(status)}: {last_error()}")


# ---------------------------------------------------------------------------
# Raw-pointer entry points (integers are device addresses; stream 0 = null)
# ---------------------------------------------------------------------------

def gemv_raw(x, M, K, N, idx, idx_bits, d, codebook, C, y, stream=0) -> int:
    return lib().fasq_pq_gemv(x, M, K, N, idx, idx_bits, d, codebook, C, y, stream)


def gemm_raw(x, M, K, N, idx, idx_bits, d, codebook, C, y, stream=0) -> int:
    return lib().fasq_pq_gemm(x, M, K, N, idx, idx_bits, d, codebook, C, y, stream)


def gemv_batched_raw(x, M, K, idx, N, codebook, C, y, idx_bits, d, stream=0) -> int:
    """``idx``, ``N``, ``codebook``, ``C`` and ``y`` are equal-length sequences of
    integers (device addresses, sizes); they are marshalled into host arrays."""
    n = len(idx)
    if not (len(N) == len(codebook) == len(C) == len(y) == n):
        raise ValueError("the matrix sequences must have equal lengths")
    arr_p = _c_vp * max(n, 1)
    arr_i = _c_i64 * max(n, 1)
    return lib().fasq_pq_gemv_batched(x, M, K, n, arr_p(*idx), arr_i(*N), arr_p(*codebook), arr_i(*C),
                                      arr_p(*y), idx_bits, d, stream)


def reconstruct_raw(idx, N, K, idx_bits, d, codebook, C, w, stream=0) -> int:
    return lib().fasq_pq_reconstruct(idx, N, K, idx_bits, d, codebook, C, w, stream)


# ---------------------------------------------------------------------------
# Torch-tensor entry points
# ---------------------------------------------------------------------------

# A call's host time is most of what a small layer costs (4096 x 1024, one
# token: 3.7 us on the GPU, 11 us a call in the binding with torch's stream object,
# its device context and an import per call, 7.5 us without), so the tensor
# entry points below ask torch for plain integers: the raw stream handle of
# the tensor's device, and a device switch only when another device is current.
_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch

        _torch_module = torch
    return _torch_module


def _stream_of(device: int) -> int:
    """The handle of torch's current stream on the device of that index."""
    return _torch()._C._cuda_getCurrentRawStream(device)


def _on_device(device: int, fn, *args) -> int:
    """``fn(*args, stream)`` with that device current."""
    torch = _torch()
    if torch._C._cuda_getDevice() == device:  # there is a tensor on it, so torch's runtime is up
        return fn(*args, torch._C._cuda_getCurrentRawStream(device))
    with torch.cuda.device(device):
        return fn(*args, _stream_of(device))


def _row_bytes(K: int, d: int, idx_bits: int) -> int:
    """``fasq_idx_row_bytes`` of sizes taken from tensors (-1 when invalid)."""
    if K < 1 or d < 1 or K % d or idx_bits not in (8, 12, 16):
        return -1
    return (K // d * idx_bits + 7) // 8


def _require(t, name, dtype, ndim):
    torch = _torch()
    if isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is dtype and t.dim() == ndim and t.is_contiguous():
        return
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.dim() != ndim:
        raise ValueError(f"{name} must be {ndim}-D")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _matmul(fn, x, idx, idx_bits, d, codebook, out=None):
    torch = _torch()
    _require(x, "x", torch.float16, 2)
    _require(idx, "idx", torch.uint8, 2)
    _require(codebook, "codebook", torch.float16, 2)
    M, K = x.shape
    N, R = idx.shape
    C, dd = codebook.shape
    if dd != d:
        raise ValueError(f"codebook is [C x {dd}] but d = {d}")
    want = _row_bytes(K, d, idx_bits)
    if want < 0:
        raise ValueError("invalid (K, d, idx_bits)")
    if R != want:
        raise ValueError(f"idx rows are {R} bytes, expected {want}")
    if out is None:
        out = x.new_empty((M, N))
    else:
        _require(out, "out", torch.float16, 2)
        if tuple(out.shape) != (M, N):
            raise ValueError("out must be [M x N]")
    device = x.get_device()
    if idx.get_device() != device or codebook.get_device() != device or out.get_device() != device:
        raise ValueError("all tensors must be on one device")
    _check(_on_device(device, fn, x.data_ptr(), M, K, N, idx.data_ptr(), idx_bits, d, codebook.data_ptr(), C,
                      out.data_ptr()))
    return out


def pq_gemv(x, idx, idx_bits: int, d: int, codebook, out=None):
    """Decode-regime ``y = x . W_hat^T`` (fp16 [M x N]); see ``fasq_pq_gemv``."""
    return _matmul(lib().fasq_pq_gemv, x, idx, idx_bits, d, codebook, out)


def pq_gemm(x, idx, idx_bits: int, d: int, codebook, out=None):
    """Prefill-regime ``y = x . W_hat^T`` (MFMA path); see ``fasq_pq_gemm``."""
    return _matmul(lib().fasq_pq_gemm, x, idx, idx_bits, d, codebook, out)


def pq_gemm_lut(x, idx, idx_bits: int, d: int, codebook, out=None):
    """``y = x . W_hat^T`` with the paper's lookup-table GEMM design (for
    comparison); see ``fasq_pq_gemm_lut``."""
    return _matmul(lib().fasq_pq_gemm_lut, x, idx, idx_bits, d, codebook, out)


def gemm_lut_raw(x, M, K, N, idx, idx_bits, d, codebook, C, y, stream=0) -> int:
    return lib().fasq_pq_gemm_lut(x, M, K, N, idx, idx_bits, d, codebook, C, y, stream)


def pq_gemv_batched(x, idxs, idx_bits: int, d: int, codebooks, outs=None):
    """Decode-regime ``y_i = x . W_hat_i^T`` for several matrices sharing x;
    see ``fasq_pq_gemv_batched``.  Returns the list of outputs."""
    torch = _torch()
    _require(x, "x", torch.float16, 2)
    M, K = x.shape
    if len(idxs) != len(codebooks) or (outs is not None and len(outs) != len(idxs)):
        raise ValueError("idxs, codebooks and outs must have equal lengths")
    want = _row_bytes(K, d, idx_bits)
    if want < 0:
        raise ValueError("invalid (K, d, idx_bits)")
    device = x.get_device()
    ys = []
    for i, (idx, cb) in enumerate(zip(idxs, codebooks)):
        _require(idx, f"idx[{i}]", torch.uint8, 2)
        _require(cb, f"codebook[{i}]", torch.float16, 2)
        if cb.shape[1] != d:
            raise ValueError(f"codebook[{i}] is [C x {cb.shape[1]}] but d = {d}")
        if idx.shape[1] != want:
            raise ValueError(f"idx[{i}] rows are {idx.shape[1]} bytes, expected {want}")
        if outs is None:
            y = x.new_empty((M, idx.shape[0]))
        else:
            y = outs[i]
            _require(y, f"out[{i}]", torch.float16, 2)
            if tuple(y.shape) != (M, idx.shape[0]):
                raise ValueError(f"out[{i}] must be [M x N]")
        for t in (idx, cb, y):
            if t.get_device() != device:
                raise ValueError("all tensors must be on one device")
        ys.append(y)
    _check(_on_device(device, gemv_batched_raw, x.data_ptr(), M, K, [t.data_ptr() for t in idxs],
                      [t.shape[0] for t in idxs], [t.data_ptr() for t in codebooks], [t.shape[0] for t in codebooks],
                      [t.data_ptr() for t in ys], idx_bits, d))
    return ys


def pq_reconstruct(idx, K: int, idx_bits: int, d: int, codebook, out=None):
    """Explicit ``W_hat`` (fp16 [N x K]), bit copies of codebook entries."""
    torch = _torch()
    _require(idx, "idx", torch.uint8, 2)
    _require(codebook, "codebook", torch.float16, 2)
    N, R = idx.shape
    C, dd = codebook.shape
    if dd != d:
        raise ValueError(f"codebook is [C x {dd}] but d = {d}")
    want = idx_row_bytes(K, d, idx_bits)
    if want < 0 or R != want:
        raise ValueError(f"idx rows are {R} bytes, expected {want}")
    if out is None:
        out = torch.empty((N, K), dtype=torch.float16, device=idx.device)
    else:
        _require(out, "out", torch.float16, 2)
        if tuple(out.shape) != (N, K):
            raise ValueError("out must be [N x K]")
    _check(_on_device(idx.get_device(), lib().fasq_pq_reconstruct, idx.data_ptr(), N, K, idx_bits, d,
                      codebook.data_ptr(), C, out.data_ptr()))
    return out


def encode_workspace_bytes(N: int, K: int, d: int, C: int) -> int:
    return lib().fasq_pq_encode_workspace_bytes(N, K, d, C)


def encode_raw(w, N, K, d, C, idx_bits, init_codebook, iters, codebook, idx, workspace, workspace_bytes,
               stream=0) -> int:
    return lib().fasq_pq_encode(w, N, K, d, C, idx_bits, init_codebook, iters, codebook, idx, workspace,
                                workspace_bytes, stream)


def pq_encode(w, d: int, idx_bits: int, init_codebook, iters: int, workspace=None):
    """k-means PQ encoding of dense fp16 weights ``w`` [N x K] with the
    starting codebook ``init_codebook`` (fp16 [C x d]); see ``fasq_pq_encode``.
    Returns ``(codebook, idx)``: fp16 [C x d] and uint8 [N x R] device tensors."""
    torch = _torch()
    _require(w, "w", torch.float16, 2)
    _require(init_codebook, "init_codebook", torch.float16, 2)
    N, K = w.shape
    C, dd = init_codebook.shape
    if dd != d:
        raise ValueError(f"init_codebook is [C x {dd}] but d = {d}")
    R = idx_row_bytes(K, d, idx_bits)
    if R < 0:
        raise ValueError("invalid (K, d, idx_bits)")
    need = encode_workspace_bytes(N, K, d, C)
    if need < 0:
        raise ValueError("invalid encoder sizes")
    if workspace is None:
        workspace, _ = _workspace(None, need, w.get_device(), w)
    elif not (workspace.is_cuda and workspace.is_contiguous() and workspace.numel() * workspace.element_size() >= need):
        raise ValueError(f"workspace must be a contiguous device tensor of at least {need} bytes")
    if init_codebook.device != w.device or workspace.device != w.device:
        raise ValueError("all tensors must be on one device")
    codebook = torch.empty((C, d), dtype=torch.float16, device=w.device)
    idx = torch.empty((N, R), dtype=torch.uint8, device=w.device)
    _check(_on_device(w.get_device(), encode_raw, w.data_ptr(), N, K, d, C, idx_bits, init_codebook.data_ptr(), iters,
                      codebook.data_ptr(), idx.data_ptr(), workspace.data_ptr(),
                      workspace.numel() * workspace.element_size()))
    return codebook, idx


def gemv_ex_workspace_bytes(M: int, K: int, N: int, idx_bits: int, d: int, C: int, cb_stride: int) -> int:
    return lib().fasq_pq_gemv_ex_workspace_bytes(M, K, N, idx_bits, d, C, cb_stride)


def gemv_ex_raw(x, M, K, N, idx, idx_bits, d, codebook, C, cb_stride, y, workspace, workspace_bytes, stream=0) -> int:
    return lib().fasq_pq_gemv_ex(x, M, K, N, idx, idx_bits, d, codebook, C, cb_stride, y, workspace,
                                 workspace_bytes, stream)


def gemv_ex_noalloc_raw(x, M, K, N, idx, idx_bits, d, codebook, C, cb_stride, y, stream=0) -> int:
    return lib().fasq_pq_gemv_ex_noalloc(x, M, K, N, idx, idx_bits, d, codebook, C, cb_stride, y, stream)


def noalloc_scratch_bytes() -> int:
    return lib().fasq_noalloc_scratch_bytes()


def pq_gemv_ex(x, idx, idx_bits: int, d: int, codebook, out=None, workspace=None):
    """Decode-regime ``y = x . W_hat^T`` with per-subspace codebooks
    (``codebook`` fp16 [S x C x d]) or one shared codebook ([C x d]); see
    ``fasq_pq_gemv_ex``."""
    torch = _torch()
    _require(x, "x", torch.float16, 2)
    _require(idx, "idx", torch.uint8, 2)
    if not isinstance(codebook, torch.Tensor) or codebook.dim() not in (2, 3):
        raise ValueError("codebook must be [C x d] or [S x C x d]")
    _require(codebook, "codebook", torch.float16, codebook.dim())
    M, K = x.shape
    N, R = idx.shape
    if codebook.shape[-1] != d:
        raise ValueError(f"codebook entries have {codebook.shape[-1]} values but d = {d}")
    C = codebook.shape[-2]
    if codebook.dim() == 3:
        if codebook.shape[0] != K // d:
            raise ValueError(f"per-subspace codebook has {codebook.shape[0]} books, expected K / d = {K // d}")
        stride = C * d
    else:
        stride = 0
    want = _row_bytes(K, d, idx_bits)
    if want < 0 or R != want:
        raise ValueError(f"idx rows are {R} bytes, expected {want}")
    if out is None:
        out = x.new_empty((M, N))
    else:
        _require(out, "out", torch.float16, 2)
        if tuple(out.shape) != (M, N):
            raise ValueError("out must be [M x N]")
    need = gemv_ex_workspace_bytes(M, K, N, idx_bits, d, C, stride)
    if need < 0:
        raise ValueError("invalid sizes")
    if workspace is None:
        workspace, ws_bytes = _workspace(None, need, x.get_device(), x)
    else:
        ws_bytes = workspace.numel() * workspace.element_size()
    ws_ptr = workspace.data_ptr() if workspace is not None else 0
    device = x.get_device()
    if idx.get_device() != device or codebook.get_device() != device or out.get_device() != device:
        raise ValueError("all tensors must be on one device")
    _check(_on_device(device, gemv_ex_raw, x.data_ptr(), M, K, N, idx.data_ptr(), idx_bits, d, codebook.data_ptr(), C,
                      stride, out.data_ptr(), ws_ptr, ws_bytes))
    return out


def gemm_ex_workspace_bytes(M: int, K: int, N: int, idx_bits: int, d: int, C: int) -> int:
    return lib().fasq_pq_gemm_ex_workspace_bytes(M, K, N, idx_bits, d, C)


def gemm_ex_raw(x, M, K, N, idx, idx_bits, d, codebook, C, y, workspace, workspace_bytes, stream=0) -> int:
    return lib().fasq_pq_gemm_ex(x, M, K, N, idx, idx_bits, d, codebook, C, y, workspace, workspace_bytes, stream)


def pq_gemm_ex(x, idx, idx_bits: int, d: int, codebook, out=None, workspace=None):
    """Prefill-regime ``y = x . W_hat^T`` that may also split K over
    workgroups, with a workspace for the partial sums (allocated here when
    not given); see ``fasq_pq_gemm_ex``."""
    torch = _torch()
    _require(x, "x", torch.float16, 2)
    M, K = x.shape
    N = idx.shape[0] if isinstance(idx, torch.Tensor) and idx.dim() == 2 else 0
    C = codebook.shape[0] if isinstance(codebook, torch.Tensor) and codebook.dim() == 2 else 0
    need = gemm_ex_workspace_bytes(M, K, N, idx_bits, d, C) if N and C else 0
    if need < 0:
        raise ValueError("invalid sizes")
    if workspace is None:
        workspace, ws_bytes = _workspace(None, need, x.get_device(), x)
    else:
        ws_bytes = workspace.numel() * workspace.element_size()
    ws_ptr = workspace.data_ptr() if workspace is not None else 0

    def call(xp, M_, K_, N_, ip, bits, dd, cp, C_, yp, stream):
        return lib().fasq_pq_gemm_ex(xp, M_, K_, N_, ip, bits, dd, cp, C_, yp, ws_ptr, ws_bytes, stream)

    return _matmul(call, x, idx, idx_bits, d, codebook, out)


# ---------------------------------------------------------------------------
# Between the projections: rotary positions, attention, norms, adapters
# ---------------------------------------------------------------------------

# As above, most of what a small call costs is its host side (a norm of one row:
# 2.5 us on the GPU), so a tensor is looked at in one expression, and the
# functions that name what is wrong run only where it fails.

def _require_rows(t, name, dtype, ndim):
    """As ``_require``, but only the last dimension has to be contiguous."""
    torch = _torch()
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.dim() != ndim:
        raise ValueError(f"{name} must be {ndim}-D")
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"the last dimension of {name} must be contiguous")


def _same_device(device, *tensors):
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise ValueError("all tensors must be on one device")


def _check_tensor(t, name, dtype, shape, device):
    """A contiguous tensor of that type and shape on that device."""
    if not (isinstance(t, _torch().Tensor) and t.dtype is dtype and t.shape == shape and t.get_device() == device
            and t.is_contiguous()):
        _require(t, name, dtype, len(shape))
        if t.shape != shape:
            raise ValueError(f"{name} must be [{' x '.join(map(str, shape))}], got {list(t.shape)}")
        _same_device(device, t)


def _check_rows(t, name, dtype, shape, device):
    """The same, with any strides but the last."""
    if not (isinstance(t, _torch().Tensor) and t.dtype is dtype and t.shape == shape and t.get_device() == device
            and (t.stride(-1) == 1 or shape[-1] == 1)):
        _require_rows(t, name, dtype, len(shape))
        if t.shape != shape:
            raise ValueError(f"{name} must be [{' x '.join(map(str, shape))}], got {list(t.shape)}")
        _same_device(device, t)


def _ptr(t):
    return 0 if t is None else t.data_ptr()


def _kv_cache(k_cache, v_cache, device, Hkv=None, D=None):
    """The structure of two caches [pages x page_size x heads x D] (any strides but the last)."""
    torch = _torch()
    _require_rows(k_cache, "k_cache", torch.float16, 4)
    shape, strides = k_cache.shape, k_cache.stride()
    pages, page_size, heads, d = shape
    if (Hkv is not None and heads != Hkv) or (D is not None and d != D):
        raise ValueError("the caches must be [pages x page_size x Hkv x D]")
    if not (isinstance(v_cache, torch.Tensor) and v_cache.dtype is torch.float16 and v_cache.shape == shape
            and v_cache.stride() == strides and v_cache.get_device() == device):
        _require_rows(v_cache, "v_cache", torch.float16, 4)
        if v_cache.shape != shape or any(n > 1 and a != b for n, a, b in zip(shape, v_cache.stride(), strides)):
            raise ValueError("k_cache and v_cache must have the same shape and strides")
        _same_device(device, v_cache)
    if k_cache.get_device() != device:
        _same_device(device, k_cache)
    if pages == 1 or page_size == 1 or heads == 1:  # these strides are never taken, and may be anything
        strides = [s if n > 1 else 0 for n, s in zip(shape, strides)]
    return KvCache(k_cache.data_ptr(), v_cache.data_ptr(), pages, page_size, strides[0], strides[1], strides[2])


_needs = {}  # workspace bytes by entry point, device and sizes


def _workspace_need(name, device, *sizes):
    """``name(*sizes)`` on the current device (``device``): asked once for sizes that
    come again with every step (0.6 us of a call)."""
    key = (name, device, sizes)
    need = _needs.get(key)
    if need is None:
        need = getattr(lib(), name)(*sizes)
        if need >= 0 and len(_needs) < 4096:
            _needs[key] = need
    return need


def _workspace(workspace, need, device, like):
    """The workspace to use and its bytes: the caller's, or a new one on the tensor ``like``'s device."""
    if workspace is None:
        if need <= 0:
            return None, 0
        kept = getattr(_recording, "kept", None)
        if kept and kept[-1].numel() >= need and kept[-1].get_device() == device:
            return kept[-1], need  # the launches of a list follow each other
        workspace = like.new_empty(need, dtype=_torch().uint8)
        if kept is not None:  # the recorded launches name it after this call has returned
            kept.append(workspace)
        return workspace, need
    if not (workspace.is_cuda and workspace.is_contiguous()):
        raise ValueError("workspace must be a contiguous device tensor")
    _same_device(device, workspace)
    return workspace, workspace.numel() * workspace.element_size()


def rope_frequencies(rot: int, base: float = 10000.0, scaling: Optional[str] = None, factor: float = 1.0,
                     original: int = 0, low: float = 1.0, high: Optional[float] = None):
    """The rotary frequencies ``w_i`` (``rot / 2`` Python floats) and the scale of
    the table, for :func:`rope_table`.

    ``w_i = base ** (-2 i / rot)``, and for contexts ``factor`` times the
    ``original`` one:

    * ``"linear"``: ``w / factor`` (positions interpolated);
    * ``"ntk"``: the base raised to ``base * factor ** (rot / (rot - 2))``, which
      leaves the fastest pair alone and slows the slowest by ``factor``;
    * ``"wavelength"``: pairs that turn more than ``high`` times over the original
      context are left, those that turn less than ``low`` times are slowed by
      ``factor``, between them both are mixed by the number of turns (the
      scaling of Llama-3's long-context models: low 1, high 4, the defaults);
    * ``"yarn"`` (arXiv 2309.00071): the mix is linear in the pair's index between
      the pairs that turn ``high`` (32, as in the paper, unless given) and ``low`` times, and the
      table's scale is ``0.1 ln(factor) + 1``.
    """
    if rot < 2 or rot % 2 or rot > 256:
        raise ValueError("rot must be even and lie in [2, 256]")
    if not base > 0 or not factor > 0:
        raise ValueError("base and factor must be positive")
    half, scale = rot // 2, 1.0
    if scaling == "ntk":
        if rot < 4:
            raise ValueError("ntk needs rot >= 4")
        base = base * factor ** (rot / (rot - 2))
    w = [base ** (-2.0 * i / rot) for i in range(half)]
    if scaling is None or scaling == "ntk":
        return w, scale
    if scaling == "linear":
        return [v / factor for v in w], scale
    if scaling not in ("wavelength", "yarn"):
        raise ValueError("scaling must be None, 'linear', 'ntk', 'wavelength' or 'yarn'")
    if high is None:
        high = 32.0 if scaling == "yarn" else 4.0
    if original < 1 or not 0 < low < high:
        raise ValueError(f"{scaling} needs original >= 1 and 0 < low < high")
    turns = [original * v / (2 * math.pi) for v in w]
    if scaling == "wavelength":
        keep = [min(max((t - low) / (high - low), 0.0), 1.0) for t in turns]
    else:
        def pair_of(n):  # the (fractional) pair that turns n times over the original context
            return rot * math.log(original / (2 * math.pi * n)) / (2 * math.log(base))

        first = max(math.floor(pair_of(high)), 0)
        last = min(math.ceil(pair_of(low)), rot - 1)
        span = max(last - first, 1e-3)
        keep = [1.0 - min(max((i - first) / span, 0.0), 1.0) for i in range(half)]
        scale = 0.1 * math.log(factor) + 1.0 if factor > 1 else 1.0
    return [v * k + v / factor * (1 - k) for v, k in zip(w, keep)], scale


def rope_table(inv_freq, positions: int, scale: float = 1.0, device="cuda"):
    """fp32 ``[positions x rot / 2 x 2]``: cosine and sine of every position and
    pair, times ``scale``; made once and kept.  See ``fasq_rope_table``."""
    torch = _torch()
    half = len(inv_freq)
    if positions < 1:
        raise ValueError("positions must be >= 1")
    table = torch.empty((positions, half, 2), dtype=torch.float32, device=device)
    if not table.is_cuda:
        raise ValueError("the table must be on a device")
    w = (ctypes.c_double * max(half, 1))(*[float(v) for v in inv_freq])
    _check(_on_device(table.get_device(), lib().fasq_rope_table, w, half, positions, float(scale), table.data_ptr()))
    return table


def rope_append(q, k, v, table, positions, slots, k_cache, v_cache, interleaved: bool = False, q_norm=None,
                k_norm=None, eps: float = 1e-6, out=None):
    """Rotary positions (and, with ``q_norm`` / ``k_norm``, the norm of each head
    before them) of new tokens ``q`` [T x Hq x D], ``k`` and ``v`` [T x Hkv x D];
    ``k`` and ``v`` go to the slots ``slots`` of the paged caches
    [pages x page_size x Hkv x D], the turned queries are returned (``out`` may
    be ``q``).  ``q`` may be None (returns None), or ``k`` and ``v`` (with
    ``slots`` and the caches).  ``table`` None: no rotation.  See
    ``fasq_rope_append``."""
    torch = _torch()
    f16, i32 = torch.float16, torch.int32
    some = q if q is not None else k
    if some is None:
        raise ValueError("q or k must be given")
    if (k is None) != (v is None):
        raise ValueError("k and v are given together or not at all")
    _require_rows(some, "q" if q is not None else "k", f16, 3)
    T, Hq, D = some.shape
    device = some.get_device()
    Hkv = rot = rows = kp = vp = sp = 0
    qs = qos = ks = vs = (0, 0)
    cache = None
    if q is not None:
        if out is None:
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
        else:
            _check_rows(out, "out", f16, q.shape, device)
        qs, qos = q.stride(), out.stride()
    else:
        Hq = 0
        if out is not None:
            raise ValueError("out needs q")
    if k is not None:
        _require_rows(k, "k", f16, 3)
        Hkv = k.shape[1]
        _check_rows(k, "k", f16, (T, Hkv, D), device)
        _check_rows(v, "v", f16, (T, Hkv, D), device)
        cache = _kv_cache(k_cache, v_cache, device, Hkv, D)
        _check_tensor(slots, "slots", i32, (T,), device)
        ks, vs, kp, vp, sp = k.stride(), v.stride(), k.data_ptr(), v.data_ptr(), slots.data_ptr()
    if table is not None:
        _require(table, "table", torch.float32, 3)
        rows, half, two = table.shape
        rot = 2 * half
        if two != 2 or rot > D:
            raise ValueError("table must be [positions x rot / 2 x 2] with rot <= D")
        if table.get_device() != device:
            _same_device(device, table)
        _check_tensor(positions, "positions", i32, (T,), device)
    if q_norm is not None:
        _check_tensor(q_norm, "q_norm", f16, (D,), device)
    if k_norm is not None:
        _check_tensor(k_norm, "k_norm", f16, (D,), device)
    _check(_on_device(device, lib().fasq_rope_append, _ptr(q), qs[0], qs[1], Hq, _ptr(out), qos[0], qos[1], kp, ks[0],
                      ks[1], vp, vs[0], vs[1], Hkv, T, D, _ptr(table), rows, rot, interleaved,
                      positions.data_ptr() if table is not None else 0, sp, _ptr(q_norm), _ptr(k_norm), eps, cache))
    return out


def paged_attention_workspace_bytes(T: int, B: int, Hq: int, Hkv: int, D: int) -> int:
    return lib().fasq_paged_attention_workspace_bytes(T, B, Hq, Hkv, D)


def paged_attention(q, k_cache, v_cache, pages, q_start, kv_len, scale: Optional[float] = None, causal: bool = True,
                    window: int = 0, out=None, return_lse: bool = False, workspace=None, softcap: float = 0.0,
                    slopes=None, spans=None, tree=None):
    """Attention of the new tokens ``q`` [T x Hq x D] of B requests over the paged
    caches [pages x page_size x Hkv x D]: request b has the tokens
    ``q_start[b] : q_start[b + 1]`` and the first ``kv_len[b]`` slots of the
    pages ``pages[b]`` (all int32).  Returns the output [T x Hq x D] (tokens of
    no request are not written), and with ``return_lse`` also the fp32 logarithms
    of the softmax sums [T x Hq].  ``scale`` is ``D ** -0.5`` unless given;
    ``window`` 0 sees everything.  See ``fasq_paged_attention``.

    ``softcap`` c > 0 takes ``c * tanh(score / c)`` for a score; ``slopes`` (fp32
    [Hq]) take ``slopes[h] * |position - key|`` off it before that.  ``spans``
    (int32 [T x 2]) give each token its run of keys in place of ``causal`` and
    ``window``; ``tree`` (int32 [T x words]) says bit by bit which of the
    request's new tokens a token sees (:func:`draft_tree`).  See ``fasq_attention_scores``."""
    torch = _torch()
    i32 = torch.int32
    _require_rows(q, "q", torch.float16, 3)
    T, Hq, D = q.shape
    device = q.get_device()
    cache = _kv_cache(k_cache, v_cache, device, None, D)
    Hkv = k_cache.shape[2]
    if Hkv < 1 or Hq % Hkv:
        raise ValueError("the caches must be [pages x page_size x Hkv x D], Hq a multiple of Hkv")
    _require(kv_len, "kv_len", i32, 1)
    B = kv_len.shape[0]
    _check_tensor(q_start, "q_start", i32, (B + 1,), device)
    _require_rows(pages, "pages", i32, 2)
    if pages.shape[0] != B:
        raise ValueError("pages must be [B x max_pages], q_start [B + 1] and kv_len [B]")
    if kv_len.get_device() != device or pages.get_device() != device:
        _same_device(device, kv_len, pages)
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    else:
        _check_rows(out, "out", torch.float16, q.shape, device)
    lse = q.new_empty((T, Hq), dtype=torch.float32) if return_lse else None
    qs, os_ = q.stride(), out.stride()
    L = lib()
    scores = None
    if softcap or slopes is not None or spans is not None or tree is not None:
        scores = AttentionScores(softcap or 0.0)
        if slopes is not None:
            _check_tensor(slopes, "slopes", torch.float32, (Hq,), device)
            scores.slopes = slopes.data_ptr()
        if spans is not None:
            _check_tensor(spans, "spans", i32, (T, 2), device)
            scores.spans = spans.data_ptr()
        if tree is not None:
            scores.tree, scores.tree_stride, scores.tree_words = _tree(tree, T, device)

    def call(stream):
        need = _workspace_need("fasq_paged_attention_workspace_bytes", device, T, B, Hq, Hkv, D) if workspace is None else 0
        ws, ws_bytes = _workspace(workspace, need, device, q)
        if scores is not None:
            return L.fasq_paged_attention_ex(q.data_ptr(), qs[0], qs[1], T, Hq, cache, Hkv, D, pages.data_ptr(),
                                             pages.stride(0), pages.shape[1], q_start.data_ptr(), kv_len.data_ptr(), B,
                                             D ** -0.5 if scale is None else scale, causal, window, scores,
                                             out.data_ptr(), os_[0], os_[1], _ptr(lse), _ptr(ws), ws_bytes, stream)
        return L.fasq_paged_attention(q.data_ptr(), qs[0], qs[1], T, Hq, cache, Hkv, D, pages.data_ptr(),
                                      pages.stride(0), pages.shape[1], q_start.data_ptr(), kv_len.data_ptr(), B,
                                      D ** -0.5 if scale is None else scale, causal, window, out.data_ptr(), os_[0],
                                      os_[1], _ptr(lse), _ptr(ws), ws_bytes, stream)

    _check(_on_device(device, call))
    return (out, lse) if return_lse else out


def _tree(tree, rows, device):
    """Address, row stride and words of a tree's rows."""
    _require_rows(tree, "tree", _torch().int32, 2)
    if tree.shape[0] != rows or tree.shape[1] < 1:
        raise ValueError(f"tree must be [{rows} x words], got {list(tree.shape)}")
    _same_device(device, tree)
    words = tree.shape[1]
    return tree.data_ptr(), tree.stride(0) if rows > 1 else words, words


def draft_tree(parents, device="cuda"):
    """What :func:`paged_attention` and :func:`process_logits` take of trees of
    drafted tokens: ``parents[b][i]`` is the node that request b's i-th new token
    follows (an earlier one; -1: none, it follows what is cached).  Returns
    ``(tree, depth)``: int32 [T x words], bit j of a node's row set for itself and
    the nodes it follows, and int32 [T], how many those are before itself.  Both
    are on ``device``; made once where all steps draft alike."""
    torch = _torch()
    words = max([1] + [-(-len(p) // 32) for p in parents])
    rows, depth = [], []
    for nodes in parents:
        ways = []
        for i, p in enumerate(nodes):
            if not -1 <= p < i:
                raise ValueError("a node follows an earlier one, or -1")
            ways.append((ways[p] if p >= 0 else 0) | 1 << i)
            depth.append(bin(ways[i]).count("1") - 1)
        rows += [[w >> 32 * k & 0xFFFFFFFF for k in range(words)] for w in ways]
    rows = torch.tensor(rows, dtype=torch.int64).reshape(-1, words)
    tree = torch.where(rows >= 1 << 31, rows - (1 << 32), rows).to(torch.int32)
    return tree.to(device), torch.tensor(depth, dtype=torch.int32).to(device)


def process_logits_workspace_bytes(R: int, V: int) -> int:
    return lib().fasq_process_logits_workspace_bytes(R, V)


def process_logits(logits, requests=None, *, tokens=None, token_count=None, prompt_len=None, repetition=None, presence=None,
                   frequency=None, bias_ids=None, bias_values=None, temperature=None, allowed=None, draft_tokens=None,
                   q_start=None, tree=None, requests_count: Optional[int] = None, out=None, write: bool = True,
                   choose: bool = False, choice=None, lse=None, workspace=None):
    """Rows of logits [R x V] (fp16 or fp32) under the rules of their requests,
    row r of request ``requests[r]`` (int32 [R]; None: row r of request r; a row
    whose request does not exist is left alone).

    ``tokens`` (int32 [S x L], the first ``token_count[s]`` of each row, of them
    ``prompt_len[s]`` the prompt) take the penalties ``repetition``, ``presence``
    and ``frequency`` (fp32 [S]); with drafted trees (``draft_tokens`` [R],
    ``q_start`` [S + 1], ``tree`` [R x words]) a node's own and its ancestors'
    tokens are counted too.  ``bias_ids`` and ``bias_values`` [S x E] add to single
    logits, ``temperature`` [S] divides all, and ``allowed`` (int32 [R x
    ceil(V / 32)]) leaves the tokens whose bit is set.  S is taken from these, or
    from ``requests_count`` where none is given.

    Returns the rows (``out``, fp16 or fp32, may be ``logits``; None with ``write``
    False), or with ``choose`` ``(rows, choice, lse)``: the likeliest tokens (int32
    [R], the lowest of equal ones; -1: none is allowed) and the logarithms of the
    softmax sums (fp32 [R]), in ``choice`` and ``lse`` where they are given.  See
    ``fasq_process_logits``."""
    torch = _torch()
    i32, f32 = torch.int32, torch.float32
    if not isinstance(logits, torch.Tensor):
        raise TypeError("logits must be a torch.Tensor")
    wide = logits.dtype is f32
    _require_rows(logits, "logits", f32 if wide else torch.float16, 2)
    R, V = logits.shape
    device = logits.get_device()
    if (tokens is None) != (token_count is None) or (bias_ids is None) != (bias_values is None):
        raise ValueError("tokens come with token_count, bias_ids with bias_values")
    S = requests_count if requests_count is not None else R if requests is None else None
    if S is None:
        for t in (token_count, temperature, repetition, presence, frequency, prompt_len, bias_ids):
            if isinstance(t, torch.Tensor) and t.dim() > 0:
                S = t.shape[0]
                break
        else:
            if q_start is not None:
                _require(q_start, "q_start", i32, 1)
            S = (1 << 24) if q_start is None else q_start.shape[0] - 1
    of_request, of_row = (S,), (R,)

    def vector(t, name, dtype, shape):
        if t is None:
            return 0
        # what _check_tensor asks: this is most of what a small call costs
        if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape and t.get_device() == device
                and t.is_contiguous()):
            _check_tensor(t, name, dtype, shape, device)
        return t.data_ptr()

    token_at = token_stride = max_tokens = bias_at = max_bias = value_at = allowed_at = allowed_stride = 0
    tree_at = tree_stride = words = 0
    if tokens is not None:
        _require_rows(tokens, "tokens", i32, 2)
        max_tokens = tokens.shape[1]
        _check_rows(tokens, "tokens", i32, (S, max_tokens), device)
        token_at, token_stride = tokens.data_ptr(), tokens.stride(0)
    if bias_ids is not None:
        _require(bias_ids, "bias_ids", i32, 2)
        max_bias = bias_ids.shape[1]
        bias_at = vector(bias_ids, "bias_ids", i32, (S, max_bias))
        value_at = vector(bias_values, "bias_values", f32, (S, max_bias))
    if allowed is not None:
        _check_rows(allowed, "allowed", i32, (R, (V + 31) // 32), device)
        allowed_at, allowed_stride = allowed.data_ptr(), allowed.stride(0)
    if tree is not None:
        tree_at, tree_stride, words = _tree(tree, R, device)
    # the fields of fasq_token_rules, eight bytes each
    rules = array.array("q", (
        vector(requests, "requests", i32, of_row), S, token_at, token_stride, max_tokens,
        vector(token_count, "token_count", i32, of_request), vector(prompt_len, "prompt_len", i32, of_request),
        vector(repetition, "repetition", f32, of_request), vector(presence, "presence", f32, of_request),
        vector(frequency, "frequency", f32, of_request), bias_at, value_at, max_bias,
        vector(temperature, "temperature", f32, of_request), allowed_at, allowed_stride,
        vector(draft_tokens, "draft_tokens", i32, of_row), vector(q_start, "q_start", i32, (S + 1,)), tree_at, tree_stride,
        words))
    out_wide, out_at, out_stride = False, 0, 0
    if write:
        if out is None:
            out = torch.empty_like(logits, memory_format=torch.contiguous_format)
            out_wide = wide
        else:
            out_wide = isinstance(out, torch.Tensor) and out.dtype is f32
            _check_rows(out, "out", f32 if out_wide else torch.float16, logits.shape, device)
        out_at, out_stride = out.data_ptr(), out.stride(0)
    elif out is not None:
        raise ValueError("out is given, but write is False")
    if choose:
        if choice is None:
            choice = logits.new_empty(of_row, dtype=i32)
        else:
            vector(choice, "choice", i32, of_row)
        if lse is None:
            lse = logits.new_empty(of_row, dtype=f32)
        else:
            vector(lse, "lse", f32, of_row)
    elif choice is not None or lse is not None:
        raise ValueError("choice and lse need choose")
    L = lib()

    def call(stream):
        need = _workspace_need("fasq_process_logits_workspace_bytes", device, R, V) if choose and workspace is None else 0
        ws, ws_bytes = _workspace(workspace, need, device, logits)
        return L.fasq_process_logits(logits.data_ptr(), wide, logits.stride(0), R, V, rules.buffer_info()[0], out_at, out_wide,
                                     out_stride, _ptr(choice), _ptr(lse), _ptr(ws), ws_bytes, stream)

    _check(_on_device(device, call))
    return (out, choice, lse) if choose else out


def residual_norm(x, y=None, weight=None, eps: float = 1e-5, post_weight=None, gate=None, scale: float = 1.0,
                  x_out=None, out=None):
    """The residual stream between two blocks, over rows of ``x`` [M x N]:
    ``x_new = x + scale * gate * u`` with ``u = y`` or, with ``post_weight``, its
    norm, and ``h`` = the norm of ``x_new`` with ``weight``.  ``gate`` is [N] or
    [M x N].  Returns ``(x_new, h)``; ``x_new`` is None without ``y`` (unless
    ``x_out`` is given), ``h`` is None without ``weight``.  See
    ``fasq_residual_norm``."""
    torch = _torch()
    f16 = torch.float16
    _require(x, "x", f16, 2)
    shape = x.shape
    M, N = shape
    device = x.get_device()
    stride = 0
    if y is not None:
        _check_tensor(y, "y", f16, shape, device)
        if x_out is None:
            x_out = torch.empty_like(x)
        else:
            _check_tensor(x_out, "x_out", f16, shape, device)
    elif x_out is not None:
        _check_tensor(x_out, "x_out", f16, shape, device)
    if weight is not None:
        _check_tensor(weight, "weight", f16, (N,), device)
        if out is None:
            out = torch.empty_like(x)
    if out is not None:
        _check_tensor(out, "out", f16, shape, device)
    if post_weight is not None:
        _check_tensor(post_weight, "post_weight", f16, (N,), device)
    if gate is not None:
        stride = N if getattr(gate, "ndim", 1) == 2 else 0
        _check_tensor(gate, "gate", f16, shape if stride else (N,), device)
    _check(_on_device(device, lib().fasq_residual_norm, x.data_ptr(), _ptr(y), M, N, _ptr(post_weight), _ptr(gate),
                      stride, scale, _ptr(weight), eps, _ptr(x_out), _ptr(out)))
    return x_out, out


def lora_workspace_bytes(M: int, K: int, r: int, count: int) -> int:
    return lib().fasq_lora_workspace_bytes(M, K, r, count)


def lora_batched(x, adapters, As, Bs, scales, bases, outs=None, workspace=None):
    """Low-rank adapters beside projections that read the same ``x`` [M x K]:
    ``y_i = base_i + scales[a] * B_i[a] (A_i[a] x)`` with ``a = adapters[m]`` for
    each token m (int32; outside the pool: no adapter).  ``As[i]`` is
    [L x r x K], ``Bs[i]`` [L x N_i x r], ``bases[i]`` [M x N_i] or None,
    ``scales`` fp32 [L].  ``outs[i]`` may be ``bases[i]``.  Returns the list of
    outputs; see ``fasq_lora_batched``."""
    torch = _torch()
    f16 = torch.float16
    _require(x, "x", f16, 2)
    _require(scales, "scales", torch.float32, 1)
    M, K = x.shape
    device = x.get_device()
    _check_tensor(adapters, "adapters", torch.int32, (M,), device)
    if scales.get_device() != device:
        _same_device(device, scales)
    L, n = scales.shape[0], len(As)
    if not (len(Bs) == len(bases) == n and (outs is None or len(outs) == n)) or n < 1:
        raise ValueError("As, Bs, bases and outs must have equal lengths, at least 1")
    Tensor = torch.Tensor
    r, ys, sizes, a_ptrs, b_ptrs, base_ptrs, y_ptrs = -1, [], [], [], [], [], []
    for i in range(n):
        A, B, base = As[i], Bs[i], bases[i]
        if r < 0:
            _require(A, "A[0]", f16, 3)
            r = A.shape[1]
        N = B.shape[1] if isinstance(B, Tensor) and B.dim() == 3 else -1
        # what _check_tensor asks, of both at once: this loop is most of a short call
        if not (N >= 0 and isinstance(A, Tensor) and A.dtype is f16 and B.dtype is f16 and A.shape == (L, r, K)
                and B.shape == (L, N, r) and A.get_device() == device and B.get_device() == device
                and A.is_contiguous() and B.is_contiguous()):
            _require(B, f"B[{i}]", f16, 3)
            _check_tensor(A, f"A[{i}]", f16, (L, r, K), device)
            _check_tensor(B, f"B[{i}]", f16, (L, N, r), device)
        if base is None:
            base_ptrs.append(0)
        else:
            _check_tensor(base, f"base[{i}]", f16, (M, N), device)
            base_ptrs.append(base.data_ptr())
        if outs is None:
            y = x.new_empty((M, N)) if base is None else torch.empty_like(base)
        else:
            y = outs[i]
            if y is not base:
                _check_tensor(y, f"out[{i}]", f16, (M, N), device)
        ys.append(y)
        sizes.append(N)
        a_ptrs.append(A.data_ptr())
        b_ptrs.append(B.data_ptr())
        y_ptrs.append(y.data_ptr())
    # sizes and addresses side by side in one host array
    host = array.array("q", sizes + a_ptrs + b_ptrs + base_ptrs + y_ptrs)
    at, step = host.buffer_info()[0], 8 * n
    c = lib()

    def call(stream):
        need = c.fasq_lora_workspace_bytes(M, K, r, n) if workspace is None else 0
        ws, ws_bytes = _workspace(workspace, need, device, x)
        return c.fasq_lora_batched(x.data_ptr(), M, K, adapters.data_ptr(), L, r, scales.data_ptr(), n, at, at + step,
                                   at + 2 * step, at + 3 * step, at + 4 * step, _ptr(ws), ws_bytes, stream)

    _check(_on_device(device, call))
    return ys


# ---------------------------------------------------------------------------
# Launch lists
# ---------------------------------------------------------------------------

_recording = threading.local()  # .kept: the workspaces of the list that this thread records


class LaunchList:
    """The kernel launches of a sequence of fasq calls, recorded once and
    queued again with :meth:`run` (``fasq_launch_list_*``).

    Calls made on this thread inside ``with lst:`` (or between :meth:`begin`
    and :meth:`end`) are checked and planned as usual but only recorded; the
    buffers they name must stay alive while the list may run.  The workspace of
    calls that are given none is the list's: one for all of them, kept until the
    list is closed and every run that was queued before is over.  So runs of one
    list follow each other, on one stream or on streams that wait for each
    other and for the one that was current while it recorded; a graph
    captured of a run needs the list open; a stream given as a handle outlives the list.
    """

    def __init__(self):
        h = _c_vp()
        _check(lib().fasq_launch_list_create(ctypes.byref(h)))
        self._h = h
        self._kept = []  # workspaces; the last is the largest, earlier launches may name the others
        self._streams = set()  # handles of the streams that they have been used on

    @property
    def handle(self) -> int:
        """The ``fasq_launch_list*`` (0 once closed)."""
        return (self._h.value or 0) if self._h is not None else 0

    def begin(self) -> None:
        _check(lib().fasq_launch_list_begin(self._live()))
        _recording.kept = self._kept
        self._streams.clear()

    def end(self) -> None:
        _check(lib().fasq_launch_list_end(self._live()))
        _recording.kept = None

    def __enter__(self) -> "LaunchList":
        self.begin()
        return self

    def __exit__(self, *exc) -> bool:
        self.end()
        return False

    def run(self, stream=None) -> None:
        """Queue the recorded launches on ``stream`` (an integer HIP stream
        handle, a torch stream, or None for torch's current stream)."""
        if stream is None:
            stream = _stream_of(_torch().cuda.current_device())
        elif not isinstance(stream, int):
            stream = stream.cuda_stream
        _check(lib().fasq_launch_list_run(self._live(), stream))
        if self._kept and stream not in self._streams:
            # torch's allocator waits for this stream before it hands the memory on
            cuda = _torch().cuda
            for w in self._kept:  # ExternalStream takes 0 for a new stream
                w.record_stream(cuda.ExternalStream(stream, device=w.device) if stream else cuda.default_stream(w.device))
            self._streams.add(stream)

    def __len__(self) -> int:
        return int(lib().fasq_launch_list_size(self._live()))

    def close(self) -> None:
        if self._h is not None and self._h.value:
            lib().fasq_launch_list_destroy(self._h)
            if getattr(_recording, "kept", None) is self._kept:
                _recording.kept = None
            self._kept = []
        self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _live(self):
        if self._h is None or not self._h.value:
            raise ValueError("the launch list is closed")
        return self._h
