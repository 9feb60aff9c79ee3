"""Binding of libapmm.so (C ABI in include/apmm.h): ctypes, and csrc/apmm_call.cpp for the plain cases of the calls made most often.

Argument marshalling only: every step of the path (pack, GEMM, recovery, epilogue) runs
in the library's HIP kernels.  PyTorch supplies device memory and the stream.  There is
no fallback: if the library is missing or a call fails, an exception is raised.
"""
import ctypes
import functools
import math
import os
import warnings

import torch  # imported before the library so that both share one HIP runtime (same soname)

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libapmm.so")

ALGO_AUTO, ALGO_VALU_POPCOUNT, ALGO_DECODE, ALGO_MFMA_FP4, ALGO_DECODE_VALU = 0, 1, 3, 4, 5
ALGO_PLANE_PAIRS_GLOBAL, ALGO_PLANES_REGISTERS, ALGO_MFMA_KSPLIT = 6, 7, 8

EXPORTS = [
    "apmm_packed_bytes", "apmm_packed_activation_bytes", "apmm_workspace_bytes", "apmm_pack_weights", "apmm_pack_activations",
    "apmm_quantize_pack_activations", "apmm_unpack", "apmm_unpack_activations", "apmm_gemm", "apmm_gemm_ex", "apmm_gemm_from_codes", "apmm_gemm_from_codes_noalloc", "apmm_gemm_grouped",
    "apmm_kv_write", "apmm_kv_read", "apmm_kv_attention", "apmm_kv_attention_workspace_bytes",
    "apmm_rotary", "apmm_kv_write_rotary", "apmm_kv_weights", "apmm_kv_weights_workspace_bytes", "apmm_kv_evict", "apmm_kv_evict_workspace_bytes", "apmm_w4_packed_bytes", "apmm_w4_workspace_bytes",
    "apmm_w4_pack", "apmm_w4_gemm",
    "apmm_time_next_gemm", "apmm_last_gemm_kernel", "apmm_status_string", "apmm_last_error", "apmm_version",
]



class ApmmProblem(ctypes.Structure):
    """struct apmm_problem of include/apmm.h"""
    _fields_ = [("M", ctypes.c_int64), ("N", ctypes.c_int64), ("K", ctypes.c_int64),
                ("a_packed", ctypes.c_void_p), ("w_packed", ctypes.c_void_p),
                ("c_i32", ctypes.c_void_p), ("c_f16", ctypes.c_void_p),
                ("w_scale", ctypes.c_void_p), ("a_scale", ctypes.c_void_p), ("a_codes", ctypes.c_void_p)]


class ApmmKvCache(ctypes.Structure):
    """struct apmm_kv_cache of include/apmm.h"""
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("pages", ctypes.c_int64), ("page_size", ctypes.c_int),
                ("kv_heads", ctypes.c_int), ("head_dim", ctypes.c_int), ("dtype", ctypes.c_int)]


class ApmmKvBatch(ctypes.Structure):
    """struct apmm_kv_batch of include/apmm.h"""
    _fields_ = [("sequences", ctypes.c_int), ("tokens", ctypes.c_int64), ("lengths", ctypes.c_void_p), ("starts", ctypes.c_void_p),
                ("page_table", ctypes.c_void_p), ("table_stride", ctypes.c_int64), ("table_width", ctypes.c_int64)]


class ApmmRotation(ctypes.Structure):
    """struct apmm_rotation of include/apmm.h"""
    _fields_ = [("frequencies", ctypes.c_void_p), ("pairs", ctypes.c_int64), ("interleaved", ctypes.c_int), ("magnitude", ctypes.c_float)]


_lib = None
try:  # the marshalling of the calls below in C++ (csrc/apmm_call.cpp); without it they go through ctypes, with the same results
    from . import _apmm_call as _call
except ImportError as _reason:  # not built, or built for another torch or Python
    _call = None
    warnings.warn("the calls' C++ marshalling is not used, each takes 2 to 3 us longer: %s" % _reason, RuntimeWarning)
_CALL_FUNCTIONS = ("apmm_packed_bytes", "apmm_packed_activation_bytes", "apmm_pack_weights", "apmm_pack_activations",
                   "apmm_quantize_pack_activations", "apmm_gemm_ex", "apmm_gemm_from_codes", "apmm_kv_write", "apmm_kv_read", "apmm_kv_attention",
                   "apmm_kv_attention_workspace_bytes", "apmm_rotary", "apmm_kv_write_rotary", "apmm_kv_weights", "apmm_kv_weights_workspace_bytes", "apmm_kv_evict",
                   "apmm_kv_evict_workspace_bytes", "apmm_w4_packed_bytes", "apmm_w4_workspace_bytes", "apmm_w4_gemm")


class ApmmError(RuntimeError):
    def __init__(self, status, text):
        super().__init__("apmm status %d: %s" % (status, text))
        self.status = status


def load():
    """Load the HIP library; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            "%s is missing: build it with `python -c 'import __graft_entry__ as g; g.build()'`" % LIB_PATH)
    lib = ctypes.CDLL(LIB_PATH)
    i64, vp, ci = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int
    lib.apmm_packed_bytes.restype = ctypes.c_size_t
    lib.apmm_packed_bytes.argtypes = [i64, i64, ci]
    lib.apmm_packed_activation_bytes.restype = ctypes.c_size_t
    lib.apmm_packed_activation_bytes.argtypes = [i64, i64, ci]
    lib.apmm_workspace_bytes.restype = ctypes.c_size_t
    lib.apmm_workspace_bytes.argtypes = [i64, i64, i64, ci, ci]
    for name in ("apmm_pack_weights", "apmm_pack_activations"):
        fn = getattr(lib, name)
        fn.restype = ci
        fn.argtypes = [vp, i64, i64, ci, vp, vp]
    lib.apmm_quantize_pack_activations.restype = ci
    lib.apmm_quantize_pack_activations.argtypes = [vp, i64, i64, ci, vp, vp, vp]
    for name in ("apmm_unpack", "apmm_unpack_activations"):
        fn = getattr(lib, name)
        fn.restype = ci
        fn.argtypes = [vp, i64, i64, ci, vp, vp]
    gemm_args = [i64, i64, i64, ci, ci, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.apmm_gemm.restype = ci
    lib.apmm_gemm.argtypes = gemm_args
    lib.apmm_gemm_ex.restype = ci
    lib.apmm_gemm_ex.argtypes = gemm_args + [ci]
    lib.apmm_gemm_from_codes.restype = ci
    lib.apmm_gemm_from_codes.argtypes = gemm_args
    lib.apmm_gemm_from_codes_noalloc.restype = ci
    lib.apmm_gemm_from_codes_noalloc.argtypes = [i64, i64, i64, ci, ci, vp, vp, vp, vp, vp, vp, vp]
    lib.apmm_gemm_grouped.restype = ci
    lib.apmm_gemm_grouped.argtypes = [ci, ctypes.POINTER(ApmmProblem), ci, ci, vp, ctypes.c_size_t, vp]
    cache, batch, rows = ctypes.POINTER(ApmmKvCache), ctypes.POINTER(ApmmKvBatch), [vp, i64, i64]
    for name in ("apmm_kv_write", "apmm_kv_read"):
        fn = getattr(lib, name)
        fn.restype = ci
        fn.argtypes = [cache, batch] + rows + rows + [vp]
    lib.apmm_kv_attention.restype = ci
    lib.apmm_kv_attention.argtypes = [cache, batch, ci] + rows + rows + [ctypes.c_float, i64, i64, vp, ctypes.c_size_t, vp]
    lib.apmm_kv_attention_workspace_bytes.restype = ctypes.c_size_t
    lib.apmm_kv_attention_workspace_bytes.argtypes = [cache, batch, ci]
    rotation = ctypes.POINTER(ApmmRotation)
    lib.apmm_rotary.restype = ci
    lib.apmm_rotary.argtypes = [i64, ci, ci, ci] + rows + [vp, rotation, ci] + rows + [vp]
    lib.apmm_kv_write_rotary.restype = ci
    lib.apmm_kv_write_rotary.argtypes = [cache, batch, ci, vp, rotation] + rows * 4 + [vp]
    lib.apmm_kv_weights.restype = ci
    lib.apmm_kv_weights.argtypes = [cache, batch, ci] + rows + [vp, i64, i64, i64, ctypes.c_float, ctypes.c_float, i64, i64, vp, ctypes.c_size_t, vp]
    lib.apmm_kv_weights_workspace_bytes.restype = ctypes.c_size_t
    lib.apmm_kv_weights_workspace_bytes.argtypes = [cache, batch, ci]
    lib.apmm_kv_evict.restype = ci
    lib.apmm_kv_evict.argtypes = [cache, ci, vp, vp, i64, i64, vp, i64, i64, i64, i64, i64, i64, vp, i64, i64, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.apmm_kv_evict_workspace_bytes.restype = ctypes.c_size_t
    lib.apmm_kv_evict_workspace_bytes.argtypes = [cache, ci, i64]
    lib.apmm_w4_packed_bytes.restype = ctypes.c_size_t
    lib.apmm_w4_packed_bytes.argtypes = [i64, i64, ci]
    lib.apmm_w4_pack.restype = ci
    lib.apmm_w4_pack.argtypes = [vp, vp, i64, i64, ci, ci, vp, vp]
    lib.apmm_w4_gemm.restype = ci
    lib.apmm_w4_gemm.argtypes = [i64, i64, i64, ci, ci, vp, i64, vp, vp, i64, vp, ctypes.c_size_t, vp]
    lib.apmm_w4_workspace_bytes.restype = ctypes.c_size_t
    lib.apmm_w4_workspace_bytes.argtypes = [i64, i64, i64, ci]
    lib.apmm_time_next_gemm.restype = ci
    lib.apmm_time_next_gemm.argtypes = [vp, vp]
    lib.apmm_last_gemm_kernel.restype = ctypes.c_char_p
    lib.apmm_last_gemm_kernel.argtypes = []
    lib.apmm_status_string.restype = ctypes.c_char_p
    lib.apmm_status_string.argtypes = [ci]
    lib.apmm_last_error.restype = ctypes.c_char_p
    lib.apmm_last_error.argtypes = []
    lib.apmm_version.restype = ci
    lib.apmm_version.argtypes = []
    _lib = lib
    if _call is not None:
        _call.set_library(tuple(ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in _CALL_FUNCTIONS), _check)
    return lib


def _check(status):
    if status != 0:
        lib = load()
        text = lib.apmm_last_error().decode() or lib.apmm_status_string(status).decode()
        raise ApmmError(status, text)


# A single small product is as long as its call from Python, so the plain cases of the calls that a decode step is made of (torch tensors on the GPU,
# integers and flags) are marshalled in C++ (csrc/apmm_call.cpp; the end of this file); what is not plain comes to the functions
# here.  They are kept short as well: addresses go to ctypes as plain integers (the argument types convert them), the stream handle
# is read without building a Stream object, packed sizes are computed once per shape.
def _stream():
    if not torch.cuda.is_initialized():
        torch.cuda.init()
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _ptr(t):
    return t.data_ptr() if t is not None else None


def _dev_u8(t, what):
    if t.dtype != torch.uint8 or not t.is_cuda or not t.is_contiguous() or t.dim() != 2:
        raise ValueError("%s must be a contiguous 2-D uint8 CUDA tensor" % what)


def _check_scale(s, n, what):
    if s.dtype != torch.float16 or s.numel() != n or not s.is_cuda or not s.is_contiguous():
        raise ValueError("%s must be a contiguous float16 CUDA vector of the right length" % what)


@functools.lru_cache(maxsize=1024, typed=True)
def apmm_packed_bytes(rows, K, bits):
    return int(load().apmm_packed_bytes(rows, K, bits))


@functools.lru_cache(maxsize=1024, typed=True)
def apmm_packed_activation_bytes(M, K, p):
    return int(load().apmm_packed_activation_bytes(M, K, p))


def apmm_workspace_bytes(M, N, K, p, q):
    return int(load().apmm_workspace_bytes(M, N, K, p, q))


def _pack(fn_name, codes, bits, out):
    _dev_u8(codes, "codes")
    rows, K = codes.shape
    nbytes = (apmm_packed_activation_bytes if fn_name == "apmm_pack_activations" else apmm_packed_bytes)(rows, K, bits)
    if out is None:
        out = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=codes.device)
    elif out.nbytes < nbytes:
        raise ValueError("packed buffer too small")
    _check(getattr(load(), fn_name)(_ptr(codes), rows, K, bits, _ptr(out), _stream()))
    return out


def apmm_pack_weights(w_codes, q, out=None):
    """N x K uint8 weight codes -> opaque packed buffer (uint8 tensor)."""
    return _pack("apmm_pack_weights", w_codes, q, out)


def apmm_pack_activations(a_codes, p, out=None):
    """M x K uint8 activation codes -> opaque packed buffer (uint8 tensor)."""
    return _pack("apmm_pack_activations", a_codes, p, out)


def apmm_quantize_pack_activations(x_f16, p, out=None, scale_out=None):
    """M x K float16 activations -> (opaque packed buffer, float16 per-token scales)."""
    if x_f16.dtype != torch.float16 or not x_f16.is_cuda or not x_f16.is_contiguous() or x_f16.dim() != 2:
        raise ValueError("x must be a contiguous 2-D float16 CUDA tensor")
    M, K = x_f16.shape
    nbytes = apmm_packed_activation_bytes(M, K, p)
    if out is None:
        out = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=x_f16.device)
    elif out.nbytes < nbytes:
        raise ValueError("packed buffer too small")
    if scale_out is None:
        scale_out = torch.empty(M, dtype=torch.float16, device=x_f16.device)
    elif scale_out.dtype != torch.float16 or scale_out.numel() < M:
        raise ValueError("scale_out must hold M float16 values")
    _check(load().apmm_quantize_pack_activations(_ptr(x_f16), M, K, p, _ptr(out), _ptr(scale_out), _stream()))
    return out, scale_out


def apmm_unpack(packed, rows, K, bits):
    """Packed weights -> N x K uint8 codes."""
    codes = torch.empty((rows, K), dtype=torch.uint8, device=packed.device)
    _check(load().apmm_unpack(_ptr(packed), rows, K, bits, _ptr(codes), _stream()))
    return codes


def apmm_unpack_activations(a_packed, M, K, p):
    """Packed activations -> M x K uint8 codes."""
    codes = torch.empty((M, K), dtype=torch.uint8, device=a_packed.device)
    _check(load().apmm_unpack_activations(_ptr(a_packed), M, K, p, _ptr(codes), _stream()))
    return codes


def apmm_gemm(M, N, K, p, q, a_packed, w_packed, want_i32=True, want_f16=False, w_scale=None, a_scale=None,
              c_i32=None, c_f16=None, workspace=None, algo=ALGO_AUTO):
    """C = A W^T on packed operands.  Returns (c_i32 or None, c_f16 or None).

    w_scale / a_scale are float16 CUDA vectors of length N / M (or None).  c_i32 / c_f16 may be
    preallocated outputs (int32 / float16, M x N).
    """
    dev = a_packed.device
    if want_i32 and c_i32 is None:
        c_i32 = torch.empty((M, N), dtype=torch.int32, device=dev)
    if want_f16 and c_f16 is None:
        c_f16 = torch.empty((M, N), dtype=torch.float16, device=dev)
    if w_scale is not None:
        _check_scale(w_scale, N, "w_scale")
    if a_scale is not None:
        _check_scale(a_scale, M, "a_scale")
    ws_bytes = 0 if workspace is None else workspace.nbytes
    _check(load().apmm_gemm_ex(M, N, K, p, q, _ptr(a_packed), _ptr(w_packed), _ptr(c_i32), _ptr(c_f16),
                               _ptr(w_scale), _ptr(a_scale), _ptr(workspace), ws_bytes, _stream(), algo))
    return c_i32, c_f16


def apmm_gemm_from_codes(a_codes, N, p, q, w_packed, want_i32=True, want_f16=False, w_scale=None, a_scale=None,
                         c_i32=None, c_f16=None, workspace=None):
    """C = A W^T straight from the M x K uint8 activation codes: one launch for a few tokens, else packing
    into `workspace` (uint8 tensor of apmm_packed_activation_bytes(M, K, p) bytes) followed by the GEMM."""
    _dev_u8(a_codes, "a_codes")
    M, K = a_codes.shape
    dev = a_codes.device
    if want_i32 and c_i32 is None:
        c_i32 = torch.empty((M, N), dtype=torch.int32, device=dev)
    if want_f16 and c_f16 is None:
        c_f16 = torch.empty((M, N), dtype=torch.float16, device=dev)
    ws_bytes = 0 if workspace is None else workspace.nbytes
    _check(load().apmm_gemm_from_codes(M, N, K, p, q, _ptr(a_codes), _ptr(w_packed), _ptr(c_i32), _ptr(c_f16),
                                       _ptr(w_scale), _ptr(a_scale), _ptr(workspace), ws_bytes, _stream()))
    return c_i32, c_f16


NOALLOC_MAX_PACKED_BYTES = 8 << 20  # APMM_NOALLOC_MAX_PACKED_BYTES of include/apmm.h


def apmm_gemm_from_codes_noalloc(a_codes, N, p, q, w_packed, c_i32=None, c_f16=None, w_scale=None, a_scale=None):
    """apmm_gemm_from_codes with the packed activations in the library's built-in buffer.  The call itself
    allocates nothing: the outputs are the caller's preallocated tensors."""
    _dev_u8(a_codes, "a_codes")
    M, K = a_codes.shape
    _check(load().apmm_gemm_from_codes_noalloc(M, N, K, p, q, _ptr(a_codes), _ptr(w_packed), _ptr(c_i32), _ptr(c_f16),
                                               _ptr(w_scale), _ptr(a_scale), _stream()))
    return c_i32, c_f16


def apmm_version():
    return int(load().apmm_version())


def apmm_gemm_grouped(problems, p, q):
    """Several GEMMs of equal p, q with as few launches as possible.

    problems: list of dicts with keys M, N, K, w_packed, a_packed or a_codes (unpacked uint8 codes, small-M
    shapes only) and optionally c_i32, c_f16 (output tensors), w_scale, a_scale.  Outputs must be preallocated
    by the caller.
    """
    arr = (ApmmProblem * max(len(problems), 1))()
    for i, pr in enumerate(problems):
        arr[i].M, arr[i].N, arr[i].K = pr["M"], pr["N"], pr["K"]
        for key in ("a_packed", "w_packed", "c_i32", "c_f16", "w_scale", "a_scale", "a_codes"):
            t = pr.get(key)
            setattr(arr[i], key, t.data_ptr() if t is not None else None)
    _check(load().apmm_gemm_grouped(len(problems), arr, p, q, None, 0, _stream()))


_KV_DTYPES = {torch.float16: 0, torch.bfloat16: 1}


def apmm_kv_cache(pages, page_size, kv_heads, head_dim, dtype=torch.float16, device="cuda"):
    """A four-bit key/value cache (layout: include/apmm.h) of zeros: (codes, scales)."""
    return (torch.zeros((pages, kv_heads, 2, page_size * head_dim // 2), dtype=torch.uint8, device=device),
            torch.zeros((pages, kv_heads, 2, page_size), dtype=dtype, device=device))


def _kv_cache(codes, scales):
    if codes.dtype != torch.uint8 or scales.dtype not in _KV_DTYPES or codes.dim() != 4 or scales.dim() != 4 or codes.shape[:3] != scales.shape[:3] or \
            codes.shape[2] != 2 or not codes.is_contiguous() or not scales.is_contiguous() or not codes.is_cuda or scales.device != codes.device:
        raise ValueError("codes and scales must be contiguous CUDA tensors, uint8 pages x heads x 2 x page_size * head_dim / 2 and float16 or bfloat16 pages x heads x 2 x page_size")
    if codes.get_device() != torch.cuda.current_device():
        raise ValueError("the cache must be on the current device, whose stream the call goes to")
    pages, heads, _, page_size = scales.shape
    if page_size < 1 or codes.shape[3] < 1 or codes.shape[3] * 2 % page_size:
        raise ValueError("codes must hold a whole number of channels a token, one at least")
    return ApmmKvCache(codes.data_ptr(), scales.data_ptr(), pages, page_size, heads, codes.shape[3] * 2 // page_size, _KV_DTYPES[scales.dtype])


def _kv_batch(codes, page_table, lengths, starts, tokens):
    for t, what, dim in ((page_table, "page_table", 2), (lengths, "lengths", 1), (starts, "starts", 1)):
        if t is None and what == "starts":
            continue
        if t.dtype != torch.int32 or t.dim() != dim or t.device != codes.device or (t.shape[-1] > 1 and t.stride(-1) != 1):
            raise ValueError("%s must be a %d-D int32 tensor on the cache's device, contiguous in its last dimension" % (what, dim))
    n = lengths.shape[0]
    if page_table.shape[0] != n or (starts is not None and starts.shape[0] != n + 1) or (starts is None and tokens != n):
        raise ValueError("page_table needs a row, starts (if given) one element more than there are lengths; without starts each sequence has one token")
    width = page_table.shape[1]
    return ApmmKvBatch(n, tokens, lengths.data_ptr(), _ptr(starts), page_table.data_ptr(), page_table.stride(0) if n > 1 else width, width)


def _kv_rows(t, codes, scales, heads, head_dim, tokens, what):
    if t.dtype != scales.dtype or t.device != codes.device or t.dim() != 3 or t.shape[1] != heads or t.shape[2] != head_dim or t.shape[0] != tokens or t.stride(2) != 1:
        raise ValueError("%s must be tokens x %d x %d of the scales' type on the cache's device, contiguous in its last dimension" % (what, heads, head_dim))
    return t.data_ptr(), t.stride(0), t.stride(1)


def apmm_kv_write(k, v, codes, scales, page_table, lengths, starts=None):
    """Quantise new keys and values (tokens x kv heads x head_dim) into the cache.

    lengths (int32, one a sequence) counts the new tokens; starts (int32, sequences + 1) says which rows of k and v are whose, None: one a
    sequence.  page_table: int32, sequences x pages.
    """
    cache = _kv_cache(codes, scales)
    batch = _kv_batch(codes, page_table, lengths, starts, k.shape[0])
    _check(load().apmm_kv_write(cache, batch, *_kv_rows(k, codes, scales, cache.kv_heads, cache.head_dim, batch.tokens, "k"),
                                *_kv_rows(v, codes, scales, cache.kv_heads, cache.head_dim, batch.tokens, "v"), _stream()))


def apmm_kv_read(codes, scales, page_table, lengths, tokens, starts=None, k_out=None, v_out=None):
    """Keys and values of the last starts[b + 1] - starts[b] tokens (None: of the last one) of each sequence, `tokens` in all: (k, v)."""
    cache = _kv_cache(codes, scales)
    batch = _kv_batch(codes, page_table, lengths, starts, tokens)
    if k_out is None:
        k_out = torch.empty((tokens, cache.kv_heads, cache.head_dim), dtype=scales.dtype, device=codes.device)
    if v_out is None:
        v_out = torch.empty((tokens, cache.kv_heads, cache.head_dim), dtype=scales.dtype, device=codes.device)
    _check(load().apmm_kv_read(cache, batch, *_kv_rows(k_out, codes, scales, cache.kv_heads, cache.head_dim, tokens, "k_out"),
                               *_kv_rows(v_out, codes, scales, cache.kv_heads, cache.head_dim, tokens, "v_out"), _stream()))
    return k_out, v_out


def apmm_kv_attention(q, codes, scales, page_table, lengths, starts=None, window=0, sinks=0, scale=None, out=None, workspace=None):
    """Causal attention of the new tokens' queries (tokens x query heads x head_dim) over the cache, which holds their keys and values already.

    window > 0: only the last `window` keys up to the query's own and the first `sinks` of the sequence are seen.  scale: 1 / sqrt(head_dim) if None.
    workspace: uint8 tensor of apmm_kv_attention_workspace_bytes(...) bytes; allocated if None.  A query that sees no key gets zeros.
    """
    cache = _kv_cache(codes, scales)
    if q.dim() != 3 or q.shape[2] != cache.head_dim:
        raise ValueError("q must be tokens x query heads x %d" % cache.head_dim)
    tokens, heads, head_dim = q.shape
    batch = _kv_batch(codes, page_table, lengths, starts, tokens)
    if out is None:
        out = torch.empty((tokens, heads, head_dim), dtype=q.dtype, device=q.device)
    rows = _kv_rows(q, codes, scales, heads, head_dim, tokens, "q") + _kv_rows(out, codes, scales, heads, head_dim, tokens, "out")
    lib = load()
    if workspace is None:
        need = lib.apmm_kv_attention_workspace_bytes(cache, batch, heads)
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
    elif workspace.device != codes.device or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on the cache's device")
    _check(lib.apmm_kv_attention(cache, batch, heads, *rows, head_dim ** -0.5 if scale is None else scale, window, sinks,
                                 _ptr(workspace), 0 if workspace is None else workspace.nbytes, _stream()))
    return out


def apmm_kv_attention_workspace_bytes(tokens, q_heads, codes, scales, page_table, lengths):
    """Bytes of workspace that apmm_kv_attention needs for `tokens` queries."""
    batch = _kv_batch(codes, page_table, lengths, None, lengths.shape[0])
    batch.tokens = tokens
    return int(load().apmm_kv_attention_workspace_bytes(_kv_cache(codes, scales), batch, q_heads))


# ---- rotary positions, the cache's budget, four-bit weights of groups
def apmm_rotary_frequencies(rotary_dim, base=10000.0, factor=1.0, original=None, fast=32.0, slow=1.0, device="cuda"):
    """Radians a position for the rotary_dim / 2 pairs, in 64 bits: base^(-2 i / rotary_dim), for contexts `factor` times longer than a model was trained for divided by factor.

    With `original`, the positions that the model was trained for, frequencies of at least `fast` turns in them stay as they are, those of at most `slow` are divided, and between
    the two a ramp over the turns mixes both.  (The magnitude that goes with it is 1 + 0.1 ln(factor) as a rule.)
    """
    if rotary_dim < 2 or rotary_dim % 2:
        raise ValueError("rotary_dim must be even and at least 2")
    f = base ** (torch.arange(0, rotary_dim, 2, dtype=torch.float64) / -rotary_dim)
    if original is None:
        return (f / factor).to(device)
    keep = ((f * (original / (2.0 * math.pi)) - slow) / (fast - slow)).clamp(0.0, 1.0)
    return (f * (keep + (1.0 - keep) / factor)).to(device)


def _rotation(frequencies, interleaved, magnitude, device, what):
    if frequencies.dtype != torch.float64 or frequencies.dim() != 1 or not frequencies.is_contiguous() or frequencies.device != device:
        raise ValueError("frequencies must be a contiguous float64 vector on %s device" % what)
    return ApmmRotation(frequencies.data_ptr(), frequencies.shape[0], bool(interleaved), magnitude)


def _positions(positions, tokens, device):
    if positions.dtype != torch.int32 or positions.dim() != 1 or positions.shape[0] != tokens or positions.device != device or (tokens > 1 and positions.stride(0) != 1):
        raise ValueError("positions must be a contiguous int32 vector of one a token, on the rows' device")
    return positions.data_ptr()


def apmm_rotary(x, positions, frequencies, interleaved=False, magnitude=1.0, inverse=False, out=None):
    """Turn the pairs of the first 2 * len(frequencies) channels of x (tokens x heads x head_dim, float16 or bfloat16) by position times frequency (float64, radians).

    Pairs are neighbours (interleaved) or len(frequencies) apart.  inverse: turned back, which is also the gradient.  out: x itself, or rows that do not overlap it.
    """
    if x.dtype not in _KV_DTYPES or not x.is_cuda or x.dim() != 3 or (x.shape[2] > 1 and x.stride(2) != 1):
        raise ValueError("x must be a float16 or bfloat16 CUDA tensor, tokens x heads x head_dim, contiguous in its last dimension")
    if x.get_device() != torch.cuda.current_device():
        raise ValueError("x must be on the current device, whose stream the call goes to")
    if out is None:
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    elif out.dtype != x.dtype or out.device != x.device or out.shape != x.shape or (x.shape[2] > 1 and out.stride(2) != 1):
        raise ValueError("out must be of x's shape, type and device, contiguous in its last dimension")
    tokens, heads, head_dim = x.shape
    _check(load().apmm_rotary(tokens, heads, head_dim, _KV_DTYPES[x.dtype], x.data_ptr(), x.stride(0), x.stride(1), _positions(positions, tokens, x.device),
                              _rotation(frequencies, interleaved, magnitude, x.device, "x's"), bool(inverse), out.data_ptr(), out.stride(0), out.stride(1), _stream()))
    return out


def apmm_kv_write_rotary(q, k, v, codes, scales, page_table, lengths, frequencies, starts=None, positions=None, interleaved=False, magnitude=1.0, q_out=None):
    """apmm_rotary of q and k and apmm_kv_write of these k and of v in one launch; the turned q (in q_out, which may be q).  positions: int32, one a new token, None: its place in its
    sequence.  q may be None."""
    cache = _kv_cache(codes, scales)
    batch = _kv_batch(codes, page_table, lengths, starts, k.shape[0])
    tokens, head_dim = batch.tokens, cache.head_dim
    heads, q_rows = 0, (None, 0, 0) * 2
    if q is not None:
        if q.dim() != 3:
            raise ValueError("q must be tokens x query heads x %d" % head_dim)
        heads = q.shape[1]
        if q_out is None:
            q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        q_rows = _kv_rows(q, codes, scales, heads, head_dim, tokens, "q") + _kv_rows(q_out, codes, scales, heads, head_dim, tokens, "q_out")
    elif q_out is not None:
        raise ValueError("q_out without q")
    rotation = _rotation(frequencies, interleaved, magnitude, codes.device, "the cache's")
    _check(load().apmm_kv_write_rotary(cache, batch, heads, None if positions is None else _positions(positions, tokens, codes.device), rotation, *q_rows,
                                       *_kv_rows(k, codes, scales, cache.kv_heads, head_dim, tokens, "k"), *_kv_rows(v, codes, scales, cache.kv_heads, head_dim, tokens, "v"), _stream()))
    return q_out


def _kv_weights_rows(weights, codes, sequences, kv_heads):
    if weights.dtype != torch.float32 or weights.device != codes.device or weights.dim() != 3 or weights.shape[0] != sequences or weights.shape[1] != kv_heads or \
            weights.shape[2] < 1 or (weights.shape[2] > 1 and weights.stride(2) != 1):
        raise ValueError("weights must be a float32 tensor on the cache's device, sequences x %d x capacity, contiguous in its last dimension" % kv_heads)
    return weights.data_ptr(), weights.stride(0), weights.stride(1), weights.shape[2]


def apmm_kv_weights(q, codes, scales, page_table, lengths, weights, starts=None, window=0, sinks=0, scale=None, decay=1.0, workspace=None):
    """What attention of the new tokens' queries gives each cached token, summed over the queries and the query heads of a key/value head, added to decay * weights (float32, sequences
    x kv heads x capacity, changed and returned).  Arguments and the keys that a query sees as in apmm_kv_attention; workspace: uint8 tensor of
    apmm_kv_weights_workspace_bytes(...) bytes, allocated if None.
    """
    cache = _kv_cache(codes, scales)
    if q.dim() != 3 or q.shape[2] != cache.head_dim:
        raise ValueError("q must be tokens x query heads x %d" % cache.head_dim)
    tokens, heads, head_dim = q.shape
    batch = _kv_batch(codes, page_table, lengths, starts, tokens)
    rows = _kv_rows(q, codes, scales, heads, head_dim, tokens, "q")
    to = _kv_weights_rows(weights, codes, batch.sequences, cache.kv_heads)
    lib = load()
    if workspace is None:
        need = lib.apmm_kv_weights_workspace_bytes(cache, batch, heads)
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
    elif workspace.device != codes.device or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on the cache's device")
    _check(lib.apmm_kv_weights(cache, batch, heads, *rows, *to, decay, head_dim ** -0.5 if scale is None else scale, window, sinks,
                               _ptr(workspace), 0 if workspace is None else workspace.nbytes, _stream()))
    return weights


def apmm_kv_weights_workspace_bytes(tokens, q_heads, codes, scales, page_table, lengths):
    """Bytes of workspace that apmm_kv_weights needs for `tokens` queries."""
    batch = _kv_batch(codes, page_table, lengths, None, lengths.shape[0])
    batch.tokens = tokens
    return int(load().apmm_kv_weights_workspace_bytes(_kv_cache(codes, scales), batch, q_heads))


def apmm_kv_evict(codes, scales, page_table, lengths, weights, budget, to_table, sinks=0, recent=0, kept=None, to_weights=None, to_lengths=None, workspace=None):
    """Keep of each sequence and head the first `sinks` tokens, the last `recent` and the heaviest others, `budget` in all: copied in their order to the pages of to_table (int32, sequences
    x pages, none of a sequence of the call).  (places they had, int32, sequences x kv heads x budget with -1 behind the last; their weights; the new lengths.)
    workspace: uint8 tensor of apmm_kv_evict_workspace_bytes(...) bytes, allocated if None.
    """
    cache = _kv_cache(codes, scales)
    batch = _kv_batch(codes, page_table, lengths, None, lengths.shape[0])
    _kv_batch(codes, to_table, lengths, None, lengths.shape[0])
    sequences, shape = batch.sequences, (batch.sequences, cache.kv_heads, budget)
    rows = _kv_weights_rows(weights, codes, sequences, cache.kv_heads)
    if kept is None:
        kept = torch.empty(shape, dtype=torch.int32, device=codes.device)
    if to_weights is None:
        to_weights = torch.empty(shape, dtype=torch.float32, device=codes.device)
    if to_lengths is None:
        to_lengths = torch.empty(sequences, dtype=torch.int32, device=codes.device)
    for t, what, dtype, of in ((kept, "kept", torch.int32, shape), (to_weights, "to_weights", torch.float32, shape), (to_lengths, "to_lengths", torch.int32, (sequences,))):
        if t.dtype != dtype or tuple(t.shape) != of or t.device != codes.device or not t.is_contiguous():
            raise ValueError("%s must be a contiguous tensor of %s on the cache's device, %s" % (what, dtype, " x ".join(map(str, of))))
    lib = load()
    if workspace is None:
        need = lib.apmm_kv_evict_workspace_bytes(cache, sequences, batch.table_width)
        workspace = torch.empty(need, dtype=torch.uint8, device=codes.device) if need else None
    elif workspace.device != codes.device or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on the cache's device")
    _check(lib.apmm_kv_evict(cache, sequences, batch.lengths, batch.page_table, batch.table_stride, batch.table_width, *rows, budget, sinks, recent,
                             to_table.data_ptr(), to_table.stride(0) if sequences > 1 else to_table.shape[1], to_table.shape[1], to_lengths.data_ptr(), kept.data_ptr(),
                             to_weights.data_ptr(), _ptr(workspace), 0 if workspace is None else workspace.nbytes, _stream()))
    return kept, to_weights, to_lengths


def apmm_kv_evict_workspace_bytes(codes, scales, page_table):
    """Bytes of workspace that apmm_kv_evict needs for sequences with this page table."""
    return int(load().apmm_kv_evict_workspace_bytes(_kv_cache(codes, scales), page_table.shape[0], page_table.shape[1]))


@functools.lru_cache(maxsize=1024, typed=True)
def apmm_w4_packed_bytes(N, K, group):
    return int(load().apmm_w4_packed_bytes(N, K, group))


def _on_current_device(t, what):
    if not t.is_cuda or t.get_device() != torch.cuda.current_device():
        raise ValueError("%s must be on the current CUDA device, whose stream the call goes to" % what)


def apmm_w4_pack(codes, scales, group, out=None):
    """N x K uint8 codes of four bits and their N x ceil(K / group) scales (float16 or bfloat16, the type of the activations) -> packed weights of apmm_w4_gemm (uint8 tensor)."""
    _dev_u8(codes, "codes")
    _on_current_device(codes, "codes")
    N, K = codes.shape
    if group < 1 or scales.dtype not in _KV_DTYPES or scales.device != codes.device or tuple(scales.shape) != (N, -(-K // group)) or not scales.is_contiguous():
        raise ValueError("scales must be a contiguous float16 or bfloat16 tensor on the codes' device, N x ceil(K / group)")
    nbytes = apmm_w4_packed_bytes(N, K, group)
    if out is None:
        out = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=codes.device)
    elif out.nbytes < nbytes or out.device != codes.device or not out.is_contiguous():
        raise ValueError("packed buffer too small, or not contiguous on the codes' device")
    _check(load().apmm_w4_pack(codes.data_ptr(), scales.data_ptr(), N, K, group, _KV_DTYPES[scales.dtype], out.data_ptr(), _stream()))
    return out


@functools.lru_cache(maxsize=1024, typed=True)
def apmm_w4_workspace_bytes(M, N, K, group):
    return int(load().apmm_w4_workspace_bytes(M, N, K, group))


def apmm_w4_gemm(x, packed, N, group, out=None, workspace=None):
    """x (M x K, float16 or bfloat16, rows at any distance) times packed weights of N channels: M x N of x's type.

    packed: apmm_w4_pack's, of scales of x's type and of the same group (a form for others that is as long is not told apart).

    workspace: uint8 tensor of apmm_w4_workspace_bytes(M, N, K, group) bytes; allocated if None.
    """
    if x.dtype not in _KV_DTYPES or x.dim() != 2 or (x.shape[1] > 1 and x.stride(1) != 1):
        raise ValueError("x must be a 2-D float16 or bfloat16 tensor, contiguous in its last dimension")
    _on_current_device(x, "x")
    M, K = x.shape
    if packed.dtype != torch.uint8 or packed.device != x.device or not packed.is_contiguous() or packed.nbytes < apmm_w4_packed_bytes(N, K, group):
        raise ValueError("packed must be what apmm_w4_pack gave for N channels, x's inputs and the group, on x's device")
    if out is None:
        out = torch.empty((M, N), dtype=x.dtype, device=x.device)
    elif out.dtype != x.dtype or tuple(out.shape) != (M, N) or out.device != x.device or (N > 1 and out.stride(1) != 1):
        raise ValueError("out must be M x N of x's type on x's device, contiguous in its last dimension")
    if workspace is None:
        need = apmm_w4_workspace_bytes(M, N, K, group)
        workspace = torch.empty(need, dtype=torch.uint8, device=x.device) if need else None
    elif workspace.device != x.device or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on x's device")
    _check(load().apmm_w4_gemm(M, N, K, group, _KV_DTYPES[x.dtype], x.data_ptr(), x.stride(0), packed.data_ptr(), out.data_ptr(), out.stride(0),
                               _ptr(workspace), 0 if workspace is None else workspace.nbytes, _stream()))
    return out


def apmm_last_gemm_kernel():
    """Name of the GEMM kernel the last GEMM call of this thread launched."""
    return load().apmm_last_gemm_kernel().decode()


def apmm_time_next_gemm(start_event, stop_event):
    """Attach two torch.cuda.Event (created with enable_timing=True and recorded once, so that their
    handles exist) to the kernel dispatch of the next large-tile MFMA GEMM call of this thread."""
    _check(load().apmm_time_next_gemm(ctypes.c_void_p(start_event.cuda_event), ctypes.c_void_p(stop_event.cuda_event)))


_general = {}  # the Python functions behind the C++ calls
if _call is not None:
    for _name in ("apmm_pack_weights", "apmm_pack_activations", "apmm_quantize_pack_activations", "apmm_gemm", "apmm_gemm_from_codes", "apmm_kv_write", "apmm_kv_read",
                  "apmm_kv_attention", "apmm_rotary", "apmm_kv_write_rotary", "apmm_kv_weights", "apmm_kv_evict", "apmm_w4_gemm"):
        _general[_name] = globals()[_name]
        _call.set_general(_name, _general[_name])
        globals()[_name] = getattr(_call, _name)
