"""Thin ctypes binding of ``libdecode_attn.so`` (the C ABI of
``include/decode_attn.h``) for torch tensors.

Argument marshalling only: every step of the decode runs in the HIP kernels
behind the C ABI.  There is no fallback: if the library is missing or a call
returns an error status, a Python exception is raised.

Tensors must be contiguous, on the current HIP device, float32 (int32 for
``len``).  Calls are asynchronous on torch's current stream (or ``stream``).
The ``paged_*`` and ``prompt_*`` calls and ``rotary_axes`` also take bfloat16 and
float16, and rows with a stride between tokens (views into a fused projection's
output).
"""
from __future__ import annotations

import ctypes
import os
import struct

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIBRARY_PATH = os.environ.get("DECODE_ATTN_LIB", os.path.join(_PKG, "libdecode_attn.so"))

STATUS = {
    0: "DA_OK", 1: "DA_ERR_NULL", 2: "DA_ERR_SHAPE", 3: "DA_ERR_UNSUPPORTED",
    4: "DA_ERR_ALIGN", 5: "DA_ERR_SCALE", 6: "DA_ERR_WORKSPACE", 7: "DA_ERR_HIP",
}

# Every symbol the header declares, with its ctypes signature.
_vp, _ci, _cf, _sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
_i64 = ctypes.c_int64
SIGNATURES = {
    "da_status_string": (ctypes.c_char_p, [_ci]),
    "da_decode_workspace_bytes": (_sz, [_ci] * 6),
    "da_decode_workspace_counter_bytes": (_sz, [_ci] * 6),
    "da_decode_workspace_reset": (_ci, [_vp, _sz] + [_ci] * 6 + [_vp]),
    "da_decode_attn": (_ci, [_vp, _vp, _vp, _vp, _cf, _vp] + [_ci] * 6 + [_vp, _sz, _vp]),
    "da_decode_step": (_ci, [_vp] * 6 + [_cf, _vp] + [_ci] * 6 + [_vp, _sz, _vp]),
    "da_decode_partial": (_ci, [_vp] * 6 + [_cf] + [_ci] * 6 + [_vp, _sz, _vp]),
    "da_decode_merge": (_ci, [_vp, _vp] + [_ci] * 6 + [_vp, _sz, _vp]),
    "da_decode_multi": (_ci, [_vp, _vp, _vp, _vp, _cf, _vp] + [_ci] * 7 + [_vp, _sz, _vp]),
    "da_decode_multi_step": (_ci, [_vp] * 6 + [_cf, _vp] + [_ci] * 7 + [_vp, _sz, _vp]),
    "da_prompt_attn": (_ci, [ctypes.c_char_p] + [_vp, _i64] * 3
                       + [_cf, _vp, _vp, _vp, _sz, _vp]),
    "da_prompt_workspace_bytes": (_sz, [ctypes.c_char_p]),
    "da_prompt_attn_grad": (_ci, [ctypes.c_char_p] + [_vp, _i64] * 3
                            + [_vp, _vp, _vp, _i64, _cf] + [_vp, _i64] * 3 + [_vp, _sz, _vp]),
    "da_prompt_grad_workspace_bytes": (_sz, [ctypes.c_char_p]),
    "da_rotary_axes": (_ci, [ctypes.c_char_p] + [_vp, _i64, _ci, _vp, _i64] * 2 + [_vp]),
    "da_kv_append": (_ci, [_vp] * 5 + [_ci] * 5 + [_vp]),
    "da_kv_append_rows": (_ci, [_vp] * 5 + [_ci] * 6 + [_vp]),
    "da_decode_attn_noalloc": (_ci, [_vp, _vp, _vp, _vp, _cf, _vp] + [_ci] * 6 + [_vp]),
    "da_paged_page_bytes": (_sz, [_ci] * 4),
    "da_paged_append": (_ci, [_vp, _vp, _vp, _i64, _i64, _vp, _i64, _ci, _vp, _vp]
                        + [_ci] * 3 + [_vp]),
    "da_paged_gather": (_ci, [_vp] * 4),
    "da_paged_attn": (_ci, [_vp, _vp, _i64, _ci, _cf, _ci, _vp, _vp, _sz, _vp]),
    "da_paged_workspace_bytes": (_sz, [_ci] * 6),
    "da_paged_workspace_counter_bytes": (_sz, [_ci] * 6),
    # tuning and testing only (explicit segment size)
    "da_decode_chunk_rows": (_ci, [_ci] * 6),
    "da_decode_workspace_bytes_ex": (_sz, [_ci] * 7),
    "da_decode_multi_ex": (_ci, [_vp, _vp, _vp, _vp, _cf, _vp] + [_ci] * 8 + [_vp, _sz, _vp]),
    "da_decode_partial_ex": (_ci, [_vp] * 6 + [_cf] + [_ci] * 8 + [_vp, _sz, _vp]),
    "da_decode_merge_ex": (_ci, [_vp, _vp] + [_ci] * 8 + [_vp, _sz, _vp]),
}


class DecodeAttnError(RuntimeError):
    """A non-OK status from the library."""

    def __init__(self, fn: str, status: int):
        self.status = status
        super().__init__(f"{fn}: {_lib.da_status_string(status).decode()}")


def _load():
    if not os.path.exists(LIBRARY_PATH):
        raise ImportError(
            f"HIP library {LIBRARY_PATH} is not built; run __graft_entry__.build() "
            "(there is no CPU fallback)")
    lib = ctypes.CDLL(LIBRARY_PATH)
    for name, (res, args) in SIGNATURES.items():
        f = getattr(lib, name)
        f.restype = res
        f.argtypes = args
    return lib


_lib = _load()


def _check(fn: str, status: int) -> None:
    if status != 0:
        raise DecodeAttnError(fn, status)


def _dev(t: torch.Tensor, name: str, dtype) -> int:
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_cuda:
        raise TypeError(f"{name} must be on the GPU")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


# torch.cuda.current_stream() builds a Stream object: 2.7 us of a 9.3 us call,
# where the handle alone takes 0.2 us.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None:
        return _raw_stream(torch.cuda.current_device())
    return torch.cuda.current_stream().cuda_stream


def chunk_rows(B, h_q, h_kv, n_max, d_k, d_v) -> int:
    """Segment rows the library picks for these shapes (0: invalid); tuning only."""
    return int(_lib.da_decode_chunk_rows(B, h_q, h_kv, n_max, d_k, d_v))


def workspace_bytes(B, h_q, h_kv, n_max, d_k, d_v, chunk_rows: int = 0) -> int:
    """Workspace bytes a decode with these shapes needs (``chunk_rows`` != 0:
    for the tuning calls with that segment size)."""
    if chunk_rows:
        return int(_lib.da_decode_workspace_bytes_ex(B, h_q, h_kv, n_max, d_k, d_v,
                                                     chunk_rows))
    return int(_lib.da_decode_workspace_bytes(B, h_q, h_kv, n_max, d_k, d_v))


def workspace_counter_bytes(B, h_q, h_kv, n_max, d_k, d_v) -> int:
    """Leading workspace bytes that must be zero before first use."""
    return int(_lib.da_decode_workspace_counter_bytes(B, h_q, h_kv, n_max, d_k, d_v))


def workspace_reset(workspace, B, h_q, h_kv, n_max, d_k, d_v, stream=None) -> None:
    """Zero the counter region of ``workspace`` (h_q counts query rows, h_q*T
    for the T-row calls) with a kernel on the stream."""
    wp, wn = _ws(workspace)
    _check("da_decode_workspace_reset", _lib.da_decode_workspace_reset(
        wp, wn, B, h_q, h_kv, n_max, d_k, d_v, _stream(stream)))


def _shapes(q, K, V):
    if q.dim() != 3 or K.dim() != 4 or V.dim() != 4:
        raise ValueError("q must be [B,h_q,d_k], K [B,h_kv,n_max,d_k], V [B,h_kv,n_max,d_v]")
    B, h_q, d_k = q.shape
    Bk, h_kv, n_max, d_k2 = K.shape
    Bv, h_kv2, n_max2, d_v = V.shape
    if not (B == Bk == Bv and h_kv == h_kv2 and n_max == n_max2 and d_k == d_k2):
        raise ValueError("inconsistent q/K/V shapes")
    return B, h_q, h_kv, n_max, d_k, d_v


def alloc_workspace(q, K, V, chunk_rows: int = 0) -> torch.Tensor:
    """A zeroed workspace for decodes of these shapes (reusable across calls:
    every completed decode leaves its counter region zero again)."""
    B, h_q, h_kv, n_max, d_k, d_v = _shapes(q, K, V)
    n = workspace_bytes(B, h_q, h_kv, n_max, d_k, d_v, chunk_rows)
    if n == 0:
        _check("da_decode_workspace_bytes", 2)
    return torch.zeros(n, dtype=torch.uint8, device=q.device)


def _ws(ws):
    if ws.dtype != torch.uint8 or not ws.is_cuda or not ws.is_contiguous():
        raise TypeError("workspace must be a contiguous uint8 GPU tensor")
    return ws.data_ptr(), ws.numel()


def decode_attn(q, K, V, lens, scale: float, out=None, workspace=None,
                chunk_rows: int = 0, stream=None) -> torch.Tensor:
    """out[b,h,:] = softmax(scale * K[b,g] q[b,h]) V[b,g] over len[b] rows
    (``chunk_rows`` != 0: the tuning call with that segment size)."""
    B, h_q, h_kv, n_max, d_k, d_v = _shapes(q, K, V)
    if out is None:
        out = torch.empty((B, h_q, d_v), dtype=torch.float32, device=q.device)
    if workspace is None:
        workspace = alloc_workspace(q, K, V, chunk_rows)
    wp, wn = _ws(workspace)
    args = (_dev(q, "q", torch.float32), _dev(K, "K", torch.float32),
            _dev(V, "V", torch.float32), _dev(lens, "len", torch.int32),
            float(scale), _dev(out, "out", torch.float32), B, h_q, h_kv, n_max, d_k, d_v)
    if chunk_rows:
        _check("da_decode_multi_ex", _lib.da_decode_multi_ex(
            *args, 1, int(chunk_rows), wp, wn, _stream(stream)))
    else:
        _check("da_decode_attn", _lib.da_decode_attn(*args, wp, wn, _stream(stream)))
    return out


NOALLOC_MAX_WORKSPACE_BYTES = 64 << 20


def decode_attn_noalloc(q, K, V, lens, scale: float, out, stream=None) -> torch.Tensor:
    """decode_attn on the library's own static workspace (no allocation by
    the library; ``out`` is the caller's).  Calls on one GPU must not
    overlap in time."""
    B, h_q, h_kv, n_max, d_k, d_v = _shapes(q, K, V)
    _check("da_decode_attn_noalloc", _lib.da_decode_attn_noalloc(
        _dev(q, "q", torch.float32), _dev(K, "K", torch.float32),
        _dev(V, "V", torch.float32), _dev(lens, "len", torch.int32),
        float(scale), _dev(out, "out", torch.float32), B, h_q, h_kv, n_max, d_k, d_v,
        _stream(stream)))
    return out


def decode_step(q, K, V, k_new, v_new, lens, scale: float, out=None, workspace=None,
                chunk_rows: int = 0, stream=None) -> torch.Tensor:
    """kv_append(K, V, k_new, v_new, lens) then decode_attn(q, K, V, lens),
    fused into two kernel launches, or one where every slab is a single
    segment that is not split, with h_q / h_kv <= 16 and d_k + d_v <= 256
    (``chunk_rows`` != 0: always two, through the tuning calls)."""
    B, h_q, h_kv, n_max, d_k, d_v = _shapes(q, K, V)
    _new_rows(k_new, v_new, B, h_kv, d_k, d_v)
    if out is None:
        out = torch.empty((B, h_q, d_v), dtype=torch.float32, device=q.device)
    if workspace is None:
        workspace = alloc_workspace(q, K, V, chunk_rows)
    if chunk_rows:
        decode_partial(q, K, V, lens, scale, workspace, chunk_rows, k_new, v_new, stream)
        return decode_merge(out, workspace, B, h_q, h_kv, n_max, d_k, d_v, chunk_rows,
                            lens, stream)
    wp, wn = _ws(workspace)
    _check("da_decode_step", _lib.da_decode_step(
        _dev(q, "q", torch.float32), _dev(K, "K", torch.float32),
        _dev(V, "V", torch.float32), _dev(k_new, "k_new", torch.float32),
        _dev(v_new, "v_new", torch.float32), _dev(lens, "len", torch.int32),
        float(scale), _dev(out, "out", torch.float32), B, h_q, h_kv, n_max, d_k,
        d_v, wp, wn, _stream(stream)))
    return out


def _new_rows(k_new, v_new, B, h_kv, d_k, d_v):
    if tuple(k_new.shape) != (B, h_kv, d_k) or tuple(v_new.shape) != (B, h_kv, d_v):
        raise ValueError("k_new must be [B,h_kv,d_k] and v_new [B,h_kv,d_v]")


def decode_partial(q, K, V, lens, scale: float, workspace, chunk_rows: int = 0,
                   k_new=None, v_new=None, stream=None, T: int = 1) -> None:
    """Partials of the decode into ``workspace`` (follow with decode_merge).
    With ``k_new``/``v_new`` the partial also performs the fused append.
    ``T`` > 1 or ``chunk_rows`` != 0 go through the tuning call
    (q [B,h_q,T,d_k], k_new/v_new [B,h_kv,T,d] then)."""
    if T == 1 and q.dim() == 3:
        B, h_q, h_kv, n_max, d_k, d_v = _shapes(q, K, V)
    else:
        B, h_q, h_kv, n_max, d_k, d_v, T = _multi_shapes(q, K, V)
    wp, wn = _ws(workspace)
    kp = vp = None
    if k_new is not None or v_new is not None:
        if T == 1 and k_new.dim() == 3:
            _new_rows(k_new, v_new, B, h_kv, d_k, d_v)
        elif (tuple(k_new.shape) != (B, h_kv, T, d_k)
              or tuple(v_new.shape) != (B, h_kv, T, d_v)):
            raise ValueError("k_new must be [B,h_kv,T,d_k] and v_new [B,h_kv,T,d_v]")
        kp = _dev(k_new, "k_new", torch.float32)
        vp = _dev(v_new, "v_new", torch.float32)
    args = (_dev(q, "q", torch.float32), _dev(K, "K", torch.float32),
            _dev(V, "V", torch.float32), kp, vp, _dev(lens, "len", torch.int32),
            float(scale), B, h_q, h_kv, n_max, d_k, d_v)
    if T != 1 or chunk_rows:
        _check("da_decode_partial_ex", _lib.da_decode_partial_ex(
            *args, int(T), int(chunk_rows), wp, wn, _stream(stream)))
    else:
        _check("da_decode_partial", _lib.da_decode_partial(*args, wp, wn, _stream(stream)))


def decode_merge(out, workspace, B, h_q, h_kv, n_max, d_k, d_v,
                 chunk_rows: int = 0, lens=None, stream=None, T: int = 1) -> torch.Tensor:
    """Combine the partials in ``workspace`` into ``out`` (re-zeroes the
    workspace counters).  ``lens``: after a partial with a fused append, the
    lengths to advance.  ``T`` and ``chunk_rows``: those of the partial."""
    wp, wn = _ws(workspace)
    lp = None if lens is None else _dev(lens, "len", torch.int32)
    op = _dev(out, "out", torch.float32)
    if T != 1 or chunk_rows:
        _check("da_decode_merge_ex", _lib.da_decode_merge_ex(
            op, lp, B, h_q, h_kv, n_max, d_k, d_v, int(T), int(chunk_rows), wp, wn,
            _stream(stream)))
    else:
        _check("da_decode_merge", _lib.da_decode_merge(
            op, lp, B, h_q, h_kv, n_max, d_k, d_v, wp, wn, _stream(stream)))
    return out


def kv_append(K, V, k_new, v_new, lens, stream=None) -> None:
    """Write k_new/v_new at row len[b] of every KV head, then len[b] += 1."""
    if K.dim() != 4 or V.dim() != 4:
        raise ValueError("K and V must be [B,h_kv,n_max,d]")
    B, h_kv, n_max, d_k = K.shape
    d_v = V.shape[3]
    if tuple(V.shape[:3]) != (B, h_kv, n_max):
        raise ValueError("K and V disagree in [B,h_kv,n_max]")
    _new_rows(k_new, v_new, B, h_kv, d_k, d_v)
    _check("da_kv_append", _lib.da_kv_append(
        _dev(K, "K", torch.float32), _dev(V, "V", torch.float32),
        _dev(k_new, "k_new", torch.float32), _dev(v_new, "v_new", torch.float32),
        _dev(lens, "len", torch.int32), B, h_kv, n_max, d_k, d_v, _stream(stream)))


# --- several query rows per head (causal) -------------------------------------

def _multi_shapes(q, K, V):
    if q.dim() != 4 or K.dim() != 4 or V.dim() != 4:
        raise ValueError("q must be [B,h_q,T,d_k], K [B,h_kv,n_max,d_k], V [B,h_kv,n_max,d_v]")
    B, h_q, T, d_k = q.shape
    Bk, h_kv, n_max, d_k2 = K.shape
    Bv, h_kv2, n_max2, d_v = V.shape
    if not (B == Bk == Bv and h_kv == h_kv2 and n_max == n_max2 and d_k == d_k2):
        raise ValueError("inconsistent q/K/V shapes")
    return B, h_q, h_kv, n_max, d_k, d_v, T


def alloc_multi_workspace(q, K, V, chunk_rows: int = 0) -> torch.Tensor:
    """A zeroed workspace for multi-row decodes of these shapes (q [B,h_q,T,d_k])."""
    B, h_q, h_kv, n_max, d_k, d_v, T = _multi_shapes(q, K, V)
    n = workspace_bytes(B, h_q * T, h_kv, n_max, d_k, d_v, chunk_rows)
    if n == 0:
        _check("da_decode_workspace_bytes", 2)
    return torch.zeros(n, dtype=torch.uint8, device=q.device)


def decode_multi(q, K, V, lens, scale: float, out=None, workspace=None,
                 chunk_rows: int = 0, stream=None) -> torch.Tensor:
    """T query rows per head, causal: row r of sequence b attends cache rows
    0 .. len[b]-T+r.  q [B,h_q,T,d_k] -> out [B,h_q,T,d_v]."""
    B, h_q, h_kv, n_max, d_k, d_v, T = _multi_shapes(q, K, V)
    if out is None:
        out = torch.empty((B, h_q, T, d_v), dtype=torch.float32, device=q.device)
    if workspace is None:
        workspace = alloc_multi_workspace(q, K, V, chunk_rows)
    wp, wn = _ws(workspace)
    args = (_dev(q, "q", torch.float32), _dev(K, "K", torch.float32),
            _dev(V, "V", torch.float32), _dev(lens, "len", torch.int32),
            float(scale), _dev(out, "out", torch.float32), B, h_q, h_kv, n_max, d_k,
            d_v, T)
    if chunk_rows:
        _check("da_decode_multi_ex", _lib.da_decode_multi_ex(
            *args, int(chunk_rows), wp, wn, _stream(stream)))
    else:
        _check("da_decode_multi", _lib.da_decode_multi(*args, wp, wn, _stream(stream)))
    return out


def decode_multi_step(q, K, V, k_new, v_new, lens, scale: float, out=None,
                      workspace=None, chunk_rows: int = 0, stream=None) -> torch.Tensor:
    """T successive decode steps at once: append k_new/v_new [B,h_kv,T,d] at
    len[b].., then query row r attends rows 0 .. len[b]+r (len on entry)."""
    B, h_q, h_kv, n_max, d_k, d_v, T = _multi_shapes(q, K, V)
    if tuple(k_new.shape) != (B, h_kv, T, d_k) or tuple(v_new.shape) != (B, h_kv, T, d_v):
        raise ValueError("k_new must be [B,h_kv,T,d_k] and v_new [B,h_kv,T,d_v]")
    if out is None:
        out = torch.empty((B, h_q, T, d_v), dtype=torch.float32, device=q.device)
    if workspace is None:
        workspace = alloc_multi_workspace(q, K, V, chunk_rows)
    if chunk_rows:
        decode_partial(q, K, V, lens, scale, workspace, chunk_rows, k_new, v_new, stream, T)
        return decode_merge(out, workspace, B, h_q, h_kv, n_max, d_k, d_v, chunk_rows,
                            lens, stream, T)
    wp, wn = _ws(workspace)
    _check("da_decode_multi_step", _lib.da_decode_multi_step(
        _dev(q, "q", torch.float32), _dev(K, "K", torch.float32),
        _dev(V, "V", torch.float32), _dev(k_new, "k_new", torch.float32),
        _dev(v_new, "v_new", torch.float32), _dev(lens, "len", torch.int32),
        float(scale), _dev(out, "out", torch.float32), B, h_q, h_kv, n_max, d_k,
        d_v, T, wp, wn, _stream(stream)))
    return out


def kv_append_rows(K, V, k_new, v_new, lens, stream=None) -> None:
    """Append T rows per KV head (k_new [B,h_kv,T,d_k]) at len[b].., as many
    as fit; len[b] advances by the rows written."""
    if K.dim() != 4 or V.dim() != 4 or k_new.dim() != 4:
        raise ValueError("K, V must be [B,h_kv,n_max,d] and k_new/v_new [B,h_kv,T,d]")
    B, h_kv, n_max, d_k = K.shape
    d_v = V.shape[3]
    T = k_new.shape[2]
    if tuple(k_new.shape) != (B, h_kv, T, d_k) or tuple(v_new.shape) != (B, h_kv, T, d_v):
        raise ValueError("k_new must be [B,h_kv,T,d_k] and v_new [B,h_kv,T,d_v]")
    _check("da_kv_append_rows", _lib.da_kv_append_rows(
        _dev(K, "K", torch.float32), _dev(V, "V", torch.float32),
        _dev(k_new, "k_new", torch.float32), _dev(v_new, "v_new", torch.float32),
        _dev(lens, "len", torch.int32), B, h_kv, n_max, d_k, d_v, T, _stream(stream)))


# --- paged cache ----------------------------------------------------------------

# The arguments of the calls from here on, taken apart in C++.  It is made for one Python and one
# torch; where it cannot be imported, the calls below do the same work in Python
# (10 us more a call), and all others do not need it.
try:
    from . import paged_call as _call
    _call.use(*(ctypes.cast(getattr(_lib, f), _vp).value
                for f in ("da_paged_append", "da_paged_gather", "da_paged_attn",
                          "da_prompt_attn", "da_prompt_attn_grad", "da_rotary_axes")))
except ImportError as e:
    import warnings

    warnings.warn(f"paged_call cannot be imported ({e}); calls take their arguments apart "
                  "in Python. Run __graft_entry__.build() to build it.", RuntimeWarning)
    _call = None

# da_paged_kv: five pointers, ten ints.  Packed as bytes: filling a
# ctypes.Structure of 15 fields takes twice as long.
_pack_kv = struct.Struct("=5Q10i").pack

_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_DENSE, _MX4 = 0, 1
_i32, _u8, _f32 = torch.int32, torch.uint8, torch.float32


def paged_alloc(n_pages: int, page_rows: int, h_kv: int, d: int, dtype=torch.bfloat16,
                format: str = "dense", device="cuda"):
    """Zeroed K and V pools: [n_pages,h_kv,page_rows,d] of ``dtype``, or of 4 bits a
    value (format "mx4"): uint8 [n_pages,h_kv,page_rows,d/2 + d/32], where the last
    two dimensions are one run of bytes, in the layout of the C header."""
    if format not in ("dense", "mx4"):
        raise ValueError("format must be 'dense' or 'mx4'")
    if dtype not in _DTYPES:
        raise TypeError(f"dtype must be float32, bfloat16 or float16, got {dtype}")
    if _lib.da_paged_page_bytes(page_rows, d, _DTYPES[dtype], int(format == "mx4")) == 0:
        raise ValueError("page_rows must be a power of two from 16 to 32768 and d 64, 128 or 256")
    if format == "mx4":
        shape, dtype = (n_pages, h_kv, page_rows, d // 2 + d // 32), torch.uint8
    else:
        shape = (n_pages, h_kv, page_rows, d)
    return (torch.zeros(shape, dtype=dtype, device=device),
            torch.zeros(shape, dtype=dtype, device=device))


def rotary_table(n: int, rot_dim: int, base: float = 10000.0, device="cuda") -> torch.Tensor:
    """cos and sin of position * base^(-2i/rot_dim), i < rot_dim/2, for positions 0
    to n-1: float32 [n, rot_dim], the angles computed in 64 bits."""
    i = torch.arange(rot_dim // 2, dtype=torch.float64)
    a = torch.arange(n, dtype=torch.float64)[:, None] * base ** (-2.0 * i / rot_dim)
    return torch.cat((a.cos(), a.sin()), 1).to(device=device, dtype=torch.float32)


def _refuse(t, name, dtype, gpu):
    """The error of a tensor that a call cannot take."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_cuda:
        raise TypeError(f"{name} must be on the GPU")
    if t.get_device() != gpu:
        raise ValueError(f"{name} must be on the current device")
    raise ValueError(f"{name} must be contiguous")


def _here(t, name, dtype, gpu) -> int:
    """Address of a contiguous tensor of this type on the current device, gpu."""
    if (isinstance(t, torch.Tensor) and t.dtype is dtype and t.get_device() == gpu
            and t.is_contiguous()):
        return t.data_ptr()
    _refuse(t, name, dtype, gpu)


def _stride(t, name, shape) -> int:
    """Token stride (elements) of rows [rows, heads, d] that are not contiguous."""
    rows, heads, d = shape
    stride, head_stride, one = t.stride()
    if one != 1 or (head_stride != d and heads != 1):
        raise ValueError(f"{name}: a token's heads must be contiguous")
    return stride if rows > 1 else heads * d


def _need(condition, message):
    if not condition:
        raise ValueError(message)


def _paged(K, V, pages, past, rows, d, dtype, row_start, T):
    """(da_paged_kv as bytes, current device, h_kv, T) of a call.  The checks are
    written out: a tensor's attributes take 0.1 us each, and so does a call."""
    if not (isinstance(K, torch.Tensor) and isinstance(V, torch.Tensor)
            and isinstance(pages, torch.Tensor) and isinstance(past, torch.Tensor)):
        raise TypeError("K, V, pages and past must be torch.Tensors")
    code = _DTYPES.get(dtype)
    if code is None:
        raise TypeError(f"rows must be float32, bfloat16 or float16, got {dtype}")
    shape = K.shape
    if len(shape) != 4 or V.shape != shape:
        raise ValueError("K and V must be pools of one shape, [n_pages,h_kv,page_rows,..]")
    n_pages, h_kv, page_rows, width = shape
    mx4 = K.dtype is _u8
    pool = _u8 if mx4 else dtype
    if width != (d // 2 + d // 32 if mx4 else d):
        raise ValueError(f"pools of width {width} do not hold rows of d={d}")
    gpu = K.get_device()
    if not (gpu >= 0 and gpu == torch._C._cuda_getDevice() and K.dtype is pool
            and V.dtype is pool and pages.dtype is _i32 and past.dtype is _i32
            and V.get_device() == gpu and pages.get_device() == gpu and past.get_device() == gpu
            and K.is_contiguous() and V.is_contiguous() and pages.is_contiguous()
            and past.is_contiguous()):
        gpu = torch.cuda.current_device() if gpu >= 0 else 0
        for t, name, kind in ((K, "K", pool), (V, "V", pool), (pages, "pages", _i32),
                              (past, "past", _i32)):
            _here(t, name, kind, gpu)
    _need(pages.dim() == 2, "pages must be [B,max_pages]")
    B, max_pages = pages.shape
    _need(past.dim() == 1 and past.numel() == B, "past must be [B], as pages is [B,max_pages]")
    start = 0
    if row_start is not None:
        start = _here(row_start, "row_start", _i32, gpu)
        _need(row_start.dim() == 1 and row_start.numel() == B + 1, "row_start must be [B+1]")
        _need(T >= 1, "with row_start, T is the most rows of a sequence")
    else:
        if T == 0 and B:
            T = rows // B
        _need(rows == B * T, "without row_start every sequence has T rows: rows must be B*T")
    try:
        kv = _pack_kv(K.data_ptr(), V.data_ptr(), pages.data_ptr(), past.data_ptr(), start, B,
                      h_kv, d, n_pages, page_rows, max_pages, rows, T, code,
                      _MX4 if mx4 else _DENSE)
    except struct.error as e:
        raise ValueError(f"sizes and T must be integers of 32 bits: {e}") from None
    return kv, gpu, h_kv, T


def _paged_stream(stream, gpu) -> int:
    return _stream(stream) if stream is not None or _raw_stream is None else _raw_stream(gpu)


def _fast(K, stream):
    """(gpu, stream) of a call that paged_call may take: K on the current device."""
    if _call is not None and isinstance(K, torch.Tensor):
        gpu = K.get_device()
        if gpu >= 0 and gpu == torch._C._cuda_getDevice():
            return gpu, _paged_stream(stream, gpu)
    return None


def _empty(t, name, stream):
    """A result like t, in memory of the stream that will write it."""
    shape = _rows(t, name)
    if stream is None:
        return torch.empty(shape, dtype=t.dtype, device=t.device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=t.dtype, device=t.device)


def _rows(t, name):
    if not isinstance(t, torch.Tensor) or t.dim() != 3:
        raise ValueError(f"{name} must be [rows, heads, d]")
    return t.shape


def paged_append(K, V, pages, past, k_new, v_new, q=None, rotary=None, interleaved: bool = False,
                 row_start=None, T: int = 0, q_out=None, stream=None):
    """Rows k_new, v_new [rows,h_kv,d] into the pages of positions past[b] + r, k_new
    turned by ``rotary`` [positions, rot_dim] on the way, and q [rows,h_q,d] turned
    into q_out (returned).  ``row_start`` [B+1]: each sequence's rows, at most ``T``;
    else T rows each.  past is not changed.  A ``q_out`` not given is allocated on
    ``stream``."""
    if q is not None and q_out is None:
        q_out = _empty(q, "q", stream)
    fast = _fast(K, stream)
    if fast is not None:
        status = _call.append(K, V, pages, past, k_new, v_new, q, rotary, interleaved, row_start,
                              T, q_out, *fast)
        if status == 0:
            return q_out
        if status > 0:
            _check("da_paged_append", status)
    shape = _rows(k_new, "k_new")
    rows, heads, d = shape
    dtype = k_new.dtype
    kv, gpu, h_kv, T = _paged(K, V, pages, past, rows, d, dtype, row_start, T)
    if heads != h_kv or _rows(v_new, "v_new") != shape:
        raise ValueError("k_new and v_new must be [rows,h_kv,d]")
    if not (v_new.dtype is dtype and k_new.get_device() == gpu and v_new.get_device() == gpu):
        _refuse(k_new if k_new.get_device() != gpu else v_new, "k_new and v_new", dtype, gpu)
    ks = vs = heads * d
    if not k_new.is_contiguous():
        ks = _stride(k_new, "k_new", shape)
    if not v_new.is_contiguous():
        vs = _stride(v_new, "v_new", shape)
    qp = qo = rp = None
    qs = h_q = n_rot = rot_dim = 0
    if q is not None:
        shape = _rows(q, "q")
        h_q = shape[1]
        _need(shape[0] == rows and shape[2] == d, "q must be [rows,h_q,d]")
        if not (q.dtype is dtype and q.get_device() == gpu):
            _refuse(q, "q", dtype, gpu)
        qs = h_q * d if q.is_contiguous() else _stride(q, "q", shape)
        qp = q.data_ptr()
        qo = _here(q_out, "q_out", dtype, gpu)
        _need(q_out.shape == shape, "q_out must have q's shape")
    if rotary is not None:
        rp = _here(rotary, "rotary", _f32, gpu)
        _need(rotary.dim() == 2, "rotary must be [positions, rot_dim]")
        n_rot, rot_dim = rotary.shape
    status = _lib.da_paged_append(kv, k_new.data_ptr(), v_new.data_ptr(), ks, vs, qp, qs, h_q, qo,
                                  rp, n_rot, rot_dim, 1 if interleaved else 0,
                                  _paged_stream(stream, gpu))
    if status:
        _check("da_paged_append", status)
    return q_out


def paged_gather(K, V, pages, past, k_out, v_out, row_start=None, T: int = 0, stream=None):
    """The rows at positions past[b] + r into k_out and v_out [rows,h_kv,d] (zeros
    where there is no page): the places that paged_append with the same
    ``past``, ``row_start`` and ``T`` writes."""
    fast = _fast(K, stream)
    if fast is not None:
        status = _call.gather(K, V, pages, past, k_out, v_out, row_start, T, *fast)
        if status == 0:
            return k_out, v_out
        if status > 0:
            _check("da_paged_gather", status)
    rows, heads, d = _rows(k_out, "k_out")
    dtype = k_out.dtype
    kv, gpu, h_kv, T = _paged(K, V, pages, past, rows, d, dtype, row_start, T)
    if heads != h_kv or _rows(v_out, "v_out") != k_out.shape:
        raise ValueError("k_out and v_out must be [rows,h_kv,d]")
    status = _lib.da_paged_gather(kv, _here(k_out, "k_out", dtype, gpu),
                                  _here(v_out, "v_out", dtype, gpu), _paged_stream(stream, gpu))
    if status:
        _check("da_paged_gather", status)
    return k_out, v_out


def paged_workspace_bytes(B, h_q, h_kv, d, T: int = 1, dtype=torch.bfloat16) -> int:
    """Workspace bytes of paged_attn for these sizes (0: invalid)."""
    return int(_lib.da_paged_workspace_bytes(B, h_q, h_kv, d, T, _DTYPES.get(dtype, -1)))


def paged_workspace_counter_bytes(B, h_q, h_kv, d, T: int = 1, dtype=torch.bfloat16) -> int:
    """Leading workspace bytes that must be zero before first use."""
    return int(_lib.da_paged_workspace_counter_bytes(B, h_q, h_kv, d, T,
                                                     _DTYPES.get(dtype, -1)))


def paged_workspace(q, K, pages, T: int = 0) -> torch.Tensor:
    """A workspace for paged_attn with q [rows,h_q,d] and these pools and sequences
    (T: most rows of a sequence; 0: rows / B), its counters zeroed: reusable call
    after call, by one call at a time."""
    B = pages.shape[0]
    sizes = (B, q.shape[1], K.shape[1], q.shape[2], T or q.shape[0] // max(B, 1), q.dtype)
    n = paged_workspace_bytes(*sizes)
    if n == 0:
        _check("da_paged_workspace_bytes", 2)
    ws = torch.empty(n, dtype=torch.uint8, device=q.device)
    ws[:paged_workspace_counter_bytes(*sizes)].zero_()
    return ws


def paged_attn(q, K, V, pages, past, scale: float, causal: bool = True, row_start=None,
               T: int = 0, out=None, workspace=None, stream=None) -> torch.Tensor:
    """out[n,h,:] = softmax(scale * q[n,h].K) V over the sequence's positions up to
    the row's own, past[b] + r (causal; append first), or over all past[b] of
    them.  q [rows,h_q,d], any stride between tokens.  An ``out`` or ``workspace`` not
    given is allocated on ``stream``."""
    if out is None:
        out = _empty(q, "q", stream)
    fast = _fast(K, stream) if workspace is not None else None
    if fast is not None:
        status = _call.attn(K, V, pages, past, q, scale, causal, row_start, T, out, workspace,
                            *fast)
        if status == 0:
            return out
        if status > 0:
            _check("da_paged_attn", status)
    shape = _rows(q, "q")
    rows, h_q, d = shape
    dtype = q.dtype
    kv, gpu, _, T = _paged(K, V, pages, past, rows, d, dtype, row_start, T)
    if q.get_device() != gpu:
        _refuse(q, "q", dtype, gpu)
    op = _here(out, "out", dtype, gpu)
    _need(out.shape == shape, "out must have q's shape")
    if workspace is None:
        with torch.cuda.stream(stream):        # (None: the current one)
            workspace = paged_workspace(q, K, pages, T)
    status = _lib.da_paged_attn(
        kv, q.data_ptr(), h_q * d if q.is_contiguous() else _stride(q, "q", shape), h_q, scale,
        1 if causal else 0, op, _here(workspace, "workspace", _u8, gpu), workspace.numel(),
        _paged_stream(stream, gpu))
    if status:
        _check("da_paged_attn", status)
    return out


# --- whole prompts ----------------------------------------------------------------

# da_prompt: two pointers, ten ints.  da_rotary: two pointers, twelve ints.
_pack_prompt = struct.Struct("=2Q10i").pack
_pack_rotary = struct.Struct("=2Q12i").pack


def _tokens(t, name, dtype, gpu, rows, heads, d):
    """(address, token stride) of rows [rows, heads, d] of a token-major array."""
    if not isinstance(t, torch.Tensor) or t.dim() != 3:
        raise ValueError(f"{name} must be [rows, heads, d]")
    if t.dtype is not dtype or t.get_device() != gpu or gpu < 0:
        _refuse(t, name, dtype, gpu)
    shape = t.shape
    if shape[0] != rows or shape[1] != heads or shape[2] != d:
        raise ValueError(f"{name} must be [{rows},{heads},{d}], got {list(shape)}")
    return t.data_ptr(), heads * d if t.is_contiguous() else _stride(t, name, shape)


def _prompt(q, k, row_start, T, key_start, N, causal):
    """(da_prompt as bytes, current device) of a call's batch."""
    rows, h_q, d = _rows(q, "q")
    keys, h_kv, _ = _rows(k, "k")
    code = _DTYPES.get(q.dtype)
    if code is None:
        raise TypeError(f"q must be float32, bfloat16 or float16, got {q.dtype}")
    gpu = q.get_device()
    if gpu < 0 or gpu != torch._C._cuda_getDevice():
        _refuse(q, "q", q.dtype, torch.cuda.current_device() if gpu >= 0 else 0)
    if key_start is None and N == 0 and row_start is not None and keys == rows:
        key_start, N = row_start, T
    rs = ks = 0
    B = None
    if row_start is not None:
        rs = _here(row_start, "row_start", _i32, gpu)
        _need(row_start.dim() == 1 and row_start.numel() >= 2, "row_start must be [B+1]")
        _need(T >= 1, "with row_start, T is the most rows of a sequence")
        B = row_start.numel() - 1
    if key_start is not None:
        ks = _here(key_start, "key_start", _i32, gpu)
        _need(key_start.dim() == 1 and key_start.numel() >= 2, "key_start must be [B+1]")
        _need(N >= 1, "with key_start, N is the most keys of a sequence")
        _need(B is None or B == key_start.numel() - 1, "row_start and key_start must be of one B")
        B = key_start.numel() - 1
    if row_start is None:
        if B is None:
            B = rows // T if T > 0 else 1
        T = T or rows // max(B, 1)
        _need(rows == B * T, "without row_start every sequence has T rows: rows must be B*T")
    if key_start is None:
        N = N or keys // max(B, 1)
        _need(keys == B * N, "without key_start every sequence has N keys: keys must be B*N")
    try:
        return _pack_prompt(rs, ks, B, h_q, h_kv, d, rows, keys, T, N, code,
                            1 if causal else 0), gpu
    except struct.error as e:
        raise ValueError(f"sizes, T and N must be integers of 32 bits: {e}") from None


def _bytes(n, stream, gpu):
    """n bytes in memory of the stream that will use them."""
    with torch.cuda.stream(stream):            # (None: the current one)
        return torch.empty(n, dtype=_u8, device=f"cuda:{gpu}")


def prompt_workspace_bytes(q, k, row_start=None, T: int = 0, key_start=None, N: int = 0,
                           grad: bool = False) -> int:
    """Workspace bytes of prompt_attn (grad: of prompt_attn_grad) for these arrays (0:
    invalid)."""
    p, _ = _prompt(q, k, row_start, T, key_start, N, True)
    return int((_lib.da_prompt_grad_workspace_bytes if grad
                else _lib.da_prompt_workspace_bytes)(p))


def prompt_workspace(q, k, row_start=None, T: int = 0, key_start=None, N: int = 0,
                     grad: bool = False) -> torch.Tensor:
    """A workspace for prompt_attn (grad: for prompt_attn_grad) with these arrays:
    reusable call after call, by one call at a time."""
    n = prompt_workspace_bytes(q, k, row_start, T, key_start, N, grad)
    if n == 0:
        _check("da_prompt_workspace_bytes", 2)
    return torch.empty(n, dtype=_u8, device=q.device)


def prompt_attn(q, k, v, scale: float, causal: bool = True, row_start=None, T: int = 0,
                key_start=None, N: int = 0, out=None, lse=None, workspace=None,
                stream=None) -> torch.Tensor:
    """out[n,h,:] = softmax(scale * q[n,h] k) v over packed sequences: rows
    row_start[b] .. row_start[b+1]-1 of q [rows,h_q,d], at most ``T``, attend to keys
    key_start[b] .. of k and v [keys,h_kv,d], at most ``N``, all of them or (causal) up
    to the row's own, the last row's being the last key.  Without ``row_start`` every
    sequence has T rows (0: one sequence), without ``key_start`` N keys; where neither
    is given and there are as many keys as rows, the keys are the rows' own.  ``lse``
    [rows,h_q] float32 is written where given: what prompt_attn_grad needs.  Any stride
    between tokens up to 4 MiB.  An ``out`` or ``workspace`` not given is allocated on ``stream``.

    Keys of other lengths than the rows' (cross attention) need ``key_start``, or ``N`` where
    all have as many: without both, as many keys as rows in all are taken for the rows' own.

    No call of this library is recorded by autograd: ``out`` does not require a gradient,
    whatever q, k and v do.  A program that uses autograd calls this in the forward of a
    torch.autograd.Function, with ``lse``, and prompt_attn_grad in its backward."""
    if out is None:
        out = _empty(q, "q", stream)
    fast = _fast(q, stream) if workspace is not None else None
    if fast is not None:
        status = _call.prompt(q, k, v, scale, causal, row_start, T, key_start, N, out, lse,
                              workspace, *fast)
        if status == 0:
            return out
        if status > 0:
            _check("da_prompt_attn", status)
    p, gpu = _prompt(q, k, row_start, T, key_start, N, causal)
    rows, h_q, d = q.shape
    keys, h_kv = k.shape[:2]
    dtype = q.dtype
    qp, qs = _tokens(q, "q", dtype, gpu, rows, h_q, d)
    kp, ks = _tokens(k, "k", dtype, gpu, keys, h_kv, d)
    vp, vs = _tokens(v, "v", dtype, gpu, keys, h_kv, d)
    op = _here(out, "out", dtype, gpu)
    _need(out.shape == q.shape, "out must have q's shape")
    lp = None
    if lse is not None:
        lp = _here(lse, "lse", _f32, gpu)
        _need(lse.shape == (rows, h_q), "lse must be [rows,h_q]")
    if workspace is None:
        n = _lib.da_prompt_workspace_bytes(p)
        workspace = _bytes(max(int(n), 16), stream, gpu)
    status = _lib.da_prompt_attn(p, qp, qs, kp, ks, vp, vs, scale, op, lp,
                                 _here(workspace, "workspace", _u8, gpu), workspace.numel(),
                                 _paged_stream(stream, gpu))
    if status:
        _check("da_prompt_attn", status)
    return out


def prompt_attn_grad(q, k, v, out, lse, d_out, scale: float, causal: bool = True, row_start=None,
                     T: int = 0, key_start=None, N: int = 0, dq=None, dk=None, dv=None,
                     workspace=None, stream=None):
    """(dq, dk, dv): the gradient of prompt_attn's ``out`` with respect to q, k and v
    for d_out [rows,h_q,d], out and lse being that call's.  dq, dk and dv may be given
    with any stride between tokens (views into a fused projection's gradient); those
    not given, and the workspace, are allocated on ``stream``."""
    if dq is None:
        dq = _empty(q, "q", stream)
    if dk is None:
        dk = _empty(k, "k", stream)
    if dv is None:
        dv = _empty(v, "v", stream)
    fast = _fast(q, stream) if workspace is not None else None
    if fast is not None:
        status = _call.prompt_grad(q, k, v, out, lse, d_out, scale, causal, row_start, T,
                                   key_start, N, dq, dk, dv, workspace, *fast)
        if status == 0:
            return dq, dk, dv
        if status > 0:
            _check("da_prompt_attn_grad", status)
    p, gpu = _prompt(q, k, row_start, T, key_start, N, causal)
    rows, h_q, d = q.shape
    keys, h_kv = k.shape[:2]
    dtype = q.dtype
    a = _tokens(q, "q", dtype, gpu, rows, h_q, d)
    b = _tokens(k, "k", dtype, gpu, keys, h_kv, d)
    c = _tokens(v, "v", dtype, gpu, keys, h_kv, d)
    op = _here(out, "out", dtype, gpu)
    _need(out.shape == q.shape, "out must have q's shape")
    lp = _here(lse, "lse", _f32, gpu)
    _need(lse.shape == (rows, h_q), "lse must be [rows,h_q]")
    g = _tokens(d_out, "d_out", dtype, gpu, rows, h_q, d)
    results = (*_tokens(dq, "dq", dtype, gpu, rows, h_q, d),
               *_tokens(dk, "dk", dtype, gpu, keys, h_kv, d),
               *_tokens(dv, "dv", dtype, gpu, keys, h_kv, d))
    if workspace is None:
        n = _lib.da_prompt_grad_workspace_bytes(p)
        workspace = _bytes(max(int(n), 16), stream, gpu)
    status = _lib.da_prompt_attn_grad(p, *a, *b, *c, op, lp, *g, scale, *results,
                                      _here(workspace, "workspace", _u8, gpu),
                                      workspace.numel(), _paged_stream(stream, gpu))
    if status:
        _check("da_prompt_attn_grad", status)
    return dq, dk, dv


def rotary_axes(q, positions, table, sections, k=None, interleaved: bool = False,
                inverse: bool = False, q_out=None, k_out=None, stream=None):
    """(q_out, k_out): q [rows,h_q,d] and, where given, k [rows,h_kv,d] turned by
    positions of several axes.  ``positions`` int32 [axes,rows]; ``table`` as of
    rotary_table, [positions,rot_dim]; ``sections``: how many of the rot_dim/2 pairs
    each axis turns.  ``inverse`` turns back, which is the gradient.  Any stride
    between tokens; results not given are allocated on ``stream``, and may be the
    inputs.  Not recorded by autograd: in a torch.autograd.Function, the backward is the
    call with ``inverse`` turned over."""
    if q_out is None:
        q_out = _empty(q, "q", stream)
    if k is not None and k_out is None:
        k_out = _empty(k, "k", stream)
    fast = _fast(q, stream)
    if fast is not None:
        status = _call.rotary(q, positions, table, sections, k, interleaved, inverse, q_out,
                              k_out, *fast)
        if status == 0:
            return q_out, k_out if k is not None else None
        if status > 0:
            _check("da_rotary_axes", status)
    rows, h_q, d = _rows(q, "q")
    dtype = q.dtype
    code = _DTYPES.get(dtype)
    if code is None:
        raise TypeError(f"q must be float32, bfloat16 or float16, got {dtype}")
    gpu = q.get_device()
    if gpu < 0 or gpu != torch._C._cuda_getDevice():
        _refuse(q, "q", dtype, torch.cuda.current_device() if gpu >= 0 else 0)
    pp = _here(positions, "positions", _i32, gpu)
    axes = len(sections)
    _need(1 <= axes <= 4, "there must be 1 to 4 sections")
    _need(positions.shape == (axes, rows), "positions must be [axes,rows]")
    tp = _here(table, "table", _f32, gpu)
    _need(table.dim() == 2, "table must be [positions, rot_dim]")
    n_table, rot_dim = table.shape
    qp, qs = _tokens(q, "q", dtype, gpu, rows, h_q, d)
    qo, qos = _tokens(q_out, "q_out", dtype, gpu, rows, h_q, d)
    h_kv = ks = kos = 0
    kp = ko = None
    if k is not None:
        h_kv = _rows(k, "k")[1]
        kp, ks = _tokens(k, "k", dtype, gpu, rows, h_kv, d)
        ko, kos = _tokens(k_out, "k_out", dtype, gpu, rows, h_kv, d)
    try:
        p = _pack_rotary(pp, tp, rows, d, code, n_table, rot_dim, axes,
                         *sections, *(0,) * (4 - axes), 1 if interleaved else 0,
                         1 if inverse else 0)
    except struct.error as e:
        raise ValueError(f"sizes and sections must be integers of 32 bits: {e}") from None
    status = _lib.da_rotary_axes(p, qp, qs, h_q, qo, qos, kp, ks, h_kv, ko, kos,
                                 _paged_stream(stream, gpu))
    if status:
        _check("da_rotary_axes", status)
    return q_out, k_out if k is not None else None
