"""Python binding of ``libavq.so``: argument marshalling only.

Every step of the forward pass runs in the HIP kernels behind the C ABI
declared in ``include/avq.h``; this module checks tensor shapes, dtypes and
devices, passes raw device pointers and the current HIP stream, and turns a
non-OK status into an exception. There is no fallback: if the library is not
built, every call raises.
"""
from __future__ import annotations

import ctypes
import functools
import os
from pathlib import Path
from typing import Optional

import torch

# AVQ_LIB names another build of the same library (a sanitizer build of the
# host code, for instance); by default the in-tree build is loaded
_LIB_PATH = Path(os.environ.get("AVQ_LIB") or Path(__file__).resolve().parent / "libavq.so")
_lib = None

AVQ_OK, AVQ_ERR_INVALID_ARG, AVQ_ERR_UNSUPPORTED, AVQ_ERR_DEVICE = 0, 1, 2, 3
AVQ_F32, AVQ_BF16 = 0, 1
_DTYPES = {torch.float32: AVQ_F32, torch.bfloat16: AVQ_BF16}
SYMBOLS = ("avq_version", "avq_last_error", "avq_packed_bytes", "avq_assign",
           "avq_aggregate", "avq_attention_fwd", "avq_attention_fwd_tiled",
           "avq_codebook_update", "avq_attention_fwd_ordered", "avq_gilbert_order",
           "avq_pack_aggregates", "avq_assign_aggregate", "avq_prompt_attention_fwd",
           "avq_prompt_attention_workspace",
           "avq_cache_page_bytes", "avq_cache_append", "avq_cache_gather",
           "avq_cache_attention_workspace", "avq_cache_attention_fwd",
           "avq_rotate_axes", "avq_cross_attention_workspace", "avq_cross_attention_fwd",
           "avq_cross_attention_bwd_workspace", "avq_cross_attention_bwd",
           "avq_cache_prefix_attention_workspace", "avq_cache_prefix_attention_fwd")
CACHE_UNDIVIDED = 512  # positions of cached sequences whose keys are not divided
IMPORTANCE_TILE = 64  # parents per codeword tile of attention_fwd(tiled_importance=True)


class AvqError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"status {status}: {message}")
        self.status = status


def library_path() -> Path:
    return _LIB_PATH


def lib():
    """The loaded C library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not _LIB_PATH.exists():
            raise RuntimeError(f"{_LIB_PATH} is missing: build it with "
                               "`python -m paper_2607_12789_amd.build`")
        L = ctypes.CDLL(str(_LIB_PATH))
        i32, vp = ctypes.c_int32, ctypes.c_void_p
        L.avq_version.restype = ctypes.c_int
        L.avq_last_error.restype = ctypes.c_char_p
        L.avq_packed_bytes.argtypes = [ctypes.c_int, i32, i32, i32]
        L.avq_packed_bytes.restype = ctypes.c_int64
        L.avq_assign.argtypes = [ctypes.c_int, i32, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp]
        L.avq_aggregate.argtypes = [ctypes.c_int, i32, i32, i32, i32, i32, i32,
                                    vp, vp, vp, vp, vp, vp]
        for name in ("avq_attention_fwd", "avq_attention_fwd_tiled"):
            getattr(L, name).argtypes = [ctypes.c_int, i32, i32, i32, i32, i32, i32, i32, i32,
                                         vp, vp, vp, vp, vp, vp, vp, vp]
        L.avq_attention_fwd_ordered.argtypes = [ctypes.c_int, i32, i32, i32, i32, i32, i32, i32,
                                                i32, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp]
        L.avq_gilbert_order.argtypes = [i32, i32, vp, vp]
        L.avq_codebook_update.argtypes = [ctypes.c_int, i32, i32, i32, i32, i32, ctypes.c_float,
                                          vp, vp, vp, vp, vp, vp, vp]
        L.avq_pack_aggregates.argtypes = [ctypes.c_int, i32, i32, i32, i32, i32, vp, vp, vp, vp]
        L.avq_assign_aggregate.argtypes = [ctypes.c_int, i32, i32, i32, i32, i32, i32,
                                           vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
        i64, ci, cf = ctypes.c_int64, ctypes.c_int, ctypes.c_float
        L.avq_prompt_attention_fwd.argtypes = [ci, i32, i32, i32, i32, i32, i32, cf, i32, vp, i64,
                                               vp, i64, vp, i64, vp, vp, vp, vp, vp, i64, vp]
        L.avq_prompt_attention_workspace.argtypes = [ci] + [i32] * 6
        L.avq_prompt_attention_workspace.restype = i64
        L.avq_cache_page_bytes.argtypes = [ci, ci, i32, i32]
        L.avq_cache_page_bytes.restype = i64
        L.avq_cache_append.argtypes = [ci, ci] + [i32] * 11 + [vp, i64, vp, i64, vp, i64] + [vp] * 9
        L.avq_cache_gather.argtypes = [ci, ci] + [i32] * 7 + [vp] * 7
        L.avq_cache_attention_workspace.argtypes = [i32] * 5
        L.avq_cache_attention_workspace.restype = i64
        L.avq_cache_attention_fwd.argtypes = [ci, ci] + [i32] * 8 + [cf, vp, i64, vp, vp, vp, vp,
                                                                     vp, vp, i64, vp]
        L.avq_rotate_axes.argtypes = ([ci] + [i32] * 6 + [ctypes.c_char_p] + [i32] * 3
                                      + [vp, i64, vp, i64] + [vp] * 6)
        L.avq_cross_attention_fwd.argtypes = ([ci] + [i32] * 6 + [cf] + [vp, i64] * 3 + [vp] * 6
                                              + [i64, vp])
        L.avq_cross_attention_bwd.argtypes = ([ci] + [i32] * 6 + [cf] + [vp, i64] * 4 + [vp] * 9
                                              + [i64, vp])
        L.avq_cache_prefix_attention_fwd.argtypes = [ci, ci] + [i32] * 9 + [cf, vp, i64] + [vp] * 8 + [
            i64, vp]
        for name in ("avq_cross_attention_workspace", "avq_cross_attention_bwd_workspace"):
            getattr(L, name).argtypes = [ci] + [i32] * 6
            getattr(L, name).restype = i64
        L.avq_cache_prefix_attention_workspace.argtypes = [i32] * 6
        L.avq_cache_prefix_attention_workspace.restype = i64
        for name in ("avq_prompt_attention_fwd", "avq_cache_append", "avq_cache_gather",
                     "avq_cache_attention_fwd", "avq_rotate_axes", "avq_cross_attention_fwd",
                     "avq_cross_attention_bwd", "avq_cache_prefix_attention_fwd"):
            getattr(L, name).restype = ci
        for name in ("avq_assign", "avq_aggregate", "avq_attention_fwd", "avq_pack_aggregates",
                     "avq_assign_aggregate",
                     "avq_attention_fwd_tiled", "avq_codebook_update",
                     "avq_attention_fwd_ordered", "avq_gilbert_order"):
            getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


def _check(status: int) -> None:
    if status != AVQ_OK:
        raise AvqError(status, lib().avq_last_error().decode())


# Addresses are passed as integers: the argument types convert them, without
# a pointer object per argument.
def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _stream(stream) -> int:
    return (torch.cuda.current_stream() if stream is None else stream).cuda_stream


def _dev(t: torch.Tensor, name: str, dtype=None, shape=None):
    if (isinstance(t, torch.Tensor) and t.is_cuda and t.is_contiguous()
            and (dtype is None or t.dtype == dtype) and (shape is None or t.shape == shape)):
        return t
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a tensor on the GPU")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    return t


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype not in _DTYPES:
        raise ValueError(f"unsupported dtype {t.dtype}: use float32 or bfloat16")
    return _DTYPES[t.dtype]


def assign(K, Cp, Cc, parent_idx=None, code_idx=None, stream=None):
    """Tree assignment of the keys (``avq_assign``). Returns (parent_idx, code_idx)."""
    B, H, N, d = K.shape
    M0, Ch = Cc.shape[1], Cc.shape[2]
    _dev(K, "K")
    _dev(Cp, "Cp", K.dtype, (H, M0, d))
    _dev(Cc, "Cc", K.dtype, (H, M0, Ch, d))
    if parent_idx is None:
        parent_idx = torch.empty((B, H, N), dtype=torch.int32, device=K.device)
    if code_idx is None:
        code_idx = torch.empty((B, H, N), dtype=torch.int32, device=K.device)
    _dev(parent_idx, "parent_idx", torch.int32, (B, H, N))
    _dev(code_idx, "code_idx", torch.int32, (B, H, N))
    _check(lib().avq_assign(_dtype_code(K), B, H, N, d, M0, Ch, _ptr(K), _ptr(Cp), _ptr(Cc),
                            _ptr(parent_idx), _ptr(code_idx), _stream(stream)))
    return parent_idx, code_idx


def packed_bytes(dtype: torch.dtype, M0: int, Ch: int, d: int) -> int:
    """Bytes of the packed aggregates of one (batch, head)."""
    if dtype not in _DTYPES:
        raise ValueError(f"unsupported dtype {dtype}: use float32 or bfloat16")
    n = lib().avq_packed_bytes(_DTYPES[dtype], M0, Ch, d)
    if n < 0:
        raise ValueError(f"invalid sizes M0={M0} Ch={Ch} d={d}")
    return n


# The same for sizes that are a tensor's own (plain ints, so equal keys are
# equal sizes): 0.1 us where the library call takes 0.9.
_packed_bytes_of = functools.lru_cache(maxsize=256)(packed_bytes)


def aggregate(V, code_idx, M0: int, Ch: int, packed=None, counts=None, Vbar=None,
              sums: bool = False, stream=None):
    """Per-codeword counts, packed aggregates and optionally fp32 sums (``avq_aggregate``).

    Returns (packed, counts, Vbar); Vbar is None unless ``sums`` is set or a
    buffer is given. ``packed`` is a uint8 tensor [B, H, packed_bytes(...)]
    that ``attention_fwd`` takes.
    """
    B, H, N, d = V.shape
    Mtot = M0 * (1 + Ch)
    _dev(V, "V")
    _dev(code_idx, "code_idx", torch.int32, (B, H, N))
    E = packed_bytes(V.dtype, M0, Ch, d)
    if packed is None:
        packed = torch.empty((B, H, E), dtype=torch.uint8, device=V.device)
    if counts is None:
        counts = torch.empty((B, H, Mtot), dtype=torch.int32, device=V.device)
    if Vbar is None and sums:
        Vbar = torch.empty((B, H, Mtot, d), dtype=torch.float32, device=V.device)
    _dev(packed, "packed", torch.uint8, (B, H, E))
    _dev(counts, "counts", torch.int32, (B, H, Mtot))
    if Vbar is not None:
        _dev(Vbar, "Vbar", torch.float32, (B, H, Mtot, d))
    _check(lib().avq_aggregate(_dtype_code(V), B, H, N, d, M0, Ch, _ptr(V), _ptr(code_idx),
                               _ptr(Vbar), _ptr(counts), _ptr(packed), _stream(stream)))
    return packed, counts, Vbar


def assign_aggregate(K, V, Cp, Cc, parent_idx=None, code_idx=None, packed=None, counts=None,
                     Vbar=None, sums: bool = False, stream=None):
    """Alg. 1 as one precompute (``avq_assign_aggregate``): the codes of
    ``assign`` and the aggregates of ``aggregate``, with the child compare and
    the value sums in one pass. Returns (parent_idx, code_idx, packed, counts,
    Vbar); Vbar is None unless ``sums`` is set or a buffer is given."""
    B, H, N, d = K.shape
    M0, Ch = Cc.shape[1], Cc.shape[2]
    Mtot = M0 * (1 + Ch)
    _dev(K, "K")
    _dev(V, "V", K.dtype, (B, H, N, d))
    _dev(Cp, "Cp", K.dtype, (H, M0, d))
    _dev(Cc, "Cc", K.dtype, (H, M0, Ch, d))
    dev = K.device
    if parent_idx is None:
        parent_idx = torch.empty((B, H, N), dtype=torch.int32, device=dev)
    if code_idx is None:
        code_idx = torch.empty((B, H, N), dtype=torch.int32, device=dev)
    E = _packed_bytes_of(K.dtype, M0, Ch, d)
    if packed is None:
        packed = torch.empty((B, H, E), dtype=torch.uint8, device=dev)
    if counts is None:
        counts = torch.empty((B, H, Mtot), dtype=torch.int32, device=dev)
    if Vbar is None and sums:
        Vbar = torch.empty((B, H, Mtot, d), dtype=torch.float32, device=dev)
    _dev(parent_idx, "parent_idx", torch.int32, (B, H, N))
    _dev(code_idx, "code_idx", torch.int32, (B, H, N))
    _dev(packed, "packed", torch.uint8, (B, H, E))
    _dev(counts, "counts", torch.int32, (B, H, Mtot))
    if Vbar is not None:
        _dev(Vbar, "Vbar", torch.float32, (B, H, Mtot, d))
    _check(lib().avq_assign_aggregate(_dtype_code(K), B, H, N, d, M0, Ch, _ptr(K), _ptr(V),
                                      _ptr(Cp), _ptr(Cc), _ptr(parent_idx), _ptr(code_idx),
                                      _ptr(Vbar), _ptr(counts), _ptr(packed), _stream(stream)))
    return parent_idx, code_idx, packed, counts, Vbar


def pack_aggregates(Vbar, counts, M0: int, Ch: int, dtype, packed=None, stream=None):
    """The paper's aggregates (Vbar fp32 [B, H, Mtot, d], counts int32
    [B, H, Mtot]) in the operand layout ``attention_fwd`` reads
    (``avq_pack_aggregates``). Returns packed (uint8 [B, H, packed_bytes])."""
    B, H, Mtot, d = Vbar.shape
    if Mtot != M0 * (1 + Ch):
        raise ValueError(f"Vbar holds {Mtot} codes, expected M0 * (1 + Ch) = {M0 * (1 + Ch)}")
    _dev(Vbar, "Vbar", torch.float32)
    _dev(counts, "counts", torch.int32, (B, H, Mtot))
    E = packed_bytes(dtype, M0, Ch, d)
    if packed is None:
        packed = torch.empty((B, H, E), dtype=torch.uint8, device=Vbar.device)
    _dev(packed, "packed", torch.uint8, (B, H, E))
    _check(lib().avq_pack_aggregates(_DTYPES[dtype], B, H, d, M0, Ch, _ptr(Vbar), _ptr(counts),
                                     _ptr(packed), _stream(stream)))
    return packed


def attention_fwd(Q, Cp, Cc, packed, P: int, block_q: int, Y=None, topp_idx=None,
                  importance=None, debug: bool = False, tiled_importance: bool = False,
                  query_order=None, stream=None):
    """Refined-codebook attention (``avq_attention_fwd``, or
    ``avq_attention_fwd_tiled`` with ``tiled_importance``: the importance of
    App. B over tiles of IMPORTANCE_TILE parents).

    query_order (int32 [N] on the GPU): take the queries in this order
    (``avq_attention_fwd_ordered``); Y rows still land on their tokens.

    Returns Y, or (Y, topp_idx, importance) when ``debug`` is set (the two
    debug outputs are then allocated if not given).
    """
    B, H, N, d = Q.shape
    M0, Ch = Cc.shape[1], Cc.shape[2]
    T = (N + block_q - 1) // block_q if block_q > 0 else 0
    _dev(Q, "Q")
    _dev(Cp, "Cp", Q.dtype, (H, M0, d))
    _dev(Cc, "Cc", Q.dtype, (H, M0, Ch, d))
    _dev(packed, "packed", torch.uint8, (B, H, _packed_bytes_of(Q.dtype, M0, Ch, d)))
    if Y is None:
        Y = torch.empty_like(Q)
    _dev(Y, "Y", Q.dtype, Q.shape)
    if debug:
        if topp_idx is None:
            topp_idx = torch.empty((B, H, T, max(P, 0)), dtype=torch.int32, device=Q.device)
        if importance is None:
            importance = torch.empty((B, H, T, M0), dtype=torch.float32, device=Q.device)
    if topp_idx is not None:
        _dev(topp_idx, "topp_idx", torch.int32, (B, H, T, P))
    if importance is not None:
        _dev(importance, "importance", torch.float32, (B, H, T, M0))
    if query_order is not None:
        _dev(query_order, "query_order", torch.int32, (N,))
        _check(lib().avq_attention_fwd_ordered(
            _dtype_code(Q), B, H, N, d, M0, Ch, P, block_q, _ptr(query_order),
            int(bool(tiled_importance)), _ptr(Q), _ptr(Cp), _ptr(Cc), _ptr(packed), _ptr(Y),
            _ptr(topp_idx), _ptr(importance), _stream(stream)))
    else:
        fn = lib().avq_attention_fwd_tiled if tiled_importance else lib().avq_attention_fwd
        _check(fn(_dtype_code(Q), B, H, N, d, M0, Ch, P, block_q, _ptr(Q), _ptr(Cp), _ptr(Cc),
                  _ptr(packed), _ptr(Y), _ptr(topp_idx), _ptr(importance), _stream(stream)))
    if debug:
        return Y, topp_idx, importance
    return Y


def forward(Q, K, V, Cp, Cc, P: int, block_q: int, stream=None):
    """The whole forward pass: assign, aggregate, attention. Returns Y."""
    _, _, packed, _, _ = assign_aggregate(K, V, Cp, Cc, stream=stream)
    return attention_fwd(Q, Cp, Cc, packed, P, block_q, stream=stream)


def codebook_update(sums, counts, S, Nema, M0: int, Ch: int, lam: float, Cp_out=None,
                    Cc_out=None, dtype=None, stream=None):
    """EMA codebook step with the constrained child projection
    (``avq_codebook_update``). sums [B, H, Mtot, d] fp32 and counts
    [B, H, Mtot] int32 are the aggregates of the keys; S [H, Mtot, d] and
    Nema [H, Mtot] (fp32) are updated in place. Returns (Cp, Cc) in ``dtype``
    (default bfloat16 unless Cp_out is given)."""
    B, H, Mtot, d = sums.shape
    if Mtot != M0 * (1 + Ch):
        raise ValueError(f"sums hold {Mtot} codes, expected M0 * (1 + Ch) = {M0 * (1 + Ch)}")
    _dev(sums, "sums", torch.float32)
    _dev(counts, "counts", torch.int32, (B, H, Mtot))
    _dev(S, "S", torch.float32, (H, Mtot, d))
    _dev(Nema, "Nema", torch.float32, (H, Mtot))
    if dtype is None:
        dtype = Cp_out.dtype if Cp_out is not None else torch.bfloat16
    if Cp_out is None:
        Cp_out = torch.empty((H, M0, d), dtype=dtype, device=sums.device)
    if Cc_out is None:
        Cc_out = torch.empty((H, M0, Ch, d), dtype=dtype, device=sums.device)
    _dev(Cp_out, "Cp_out", dtype, (H, M0, d))
    _dev(Cc_out, "Cc_out", dtype, (H, M0, Ch, d))
    _check(lib().avq_codebook_update(_dtype_code(Cp_out), B, H, d, M0, Ch, float(lam), _ptr(sums),
                                     _ptr(counts), _ptr(S), _ptr(Nema), _ptr(Cp_out),
                                     _ptr(Cc_out), _stream(stream)))
    return Cp_out, Cc_out


def gilbert_order(width: int, height: int):
    """Tokens of a width x height grid (token y*width + x) in the order of a
    generalized Hilbert curve (``avq_gilbert_order``, host only). Returns
    (order, rank) as int32 CPU tensors, rank[order[k]] = k."""
    n = int(width) * int(height)
    order = torch.empty(max(n, 0), dtype=torch.int32)
    rank = torch.empty(max(n, 0), dtype=torch.int32)
    _check(lib().avq_gilbert_order(int(width), int(height), _ptr(order), _ptr(rank)))
    return order, rank


# ---- exact attention of packed prompts, and the paged cache ------------------


def _launch_stream(stream, device: torch.device) -> int:
    """The handle of the stream a call runs on, which must be one of the
    tensors' device: the library launches on the current device."""
    current = torch.cuda.current_device()
    if device.index != current or (stream is not None and stream.device != device):
        raise ValueError(f"tensors on {device}: the current device is cuda:{current}"
                         + (f", the stream's {stream.device}" if stream is not None else ""))
    if stream is None:
        # the current stream's handle without a Stream object (0.1 us instead of
        # 2.6) where this torch gives it out
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if raw is not None:
            return raw(current)
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


def _elsewhere(t: Optional[torch.Tensor], at: int) -> bool:
    return t is not None and t.get_device() != at


def _same_device(ref: torch.Tensor, **tensors) -> None:
    for name, t in tensors.items():
        if t is not None and t.device != ref.device:
            raise ValueError(f"{name} is on {t.device}, expected {ref.device}")


def _empty(stream, shape, dtype, device):
    """An output, allocated on the stream the call runs on: the allocator then
    reuses its memory only behind the call."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _like(t: torch.Tensor, stream):
    """A contiguous output of a tensor's sizes and type (0.5 us less than _empty where
    the tensor is contiguous too)."""
    if stream is None and t.is_contiguous():
        return torch.empty_like(t)
    return _empty(stream, t.shape, t.dtype, t.device)


def _rows(t: torch.Tensor, name: str, H=None, d=None, dtype=None) -> int:
    """Checks packed token rows [T, H, d] with contiguous heads; returns the
    elements from one token to the next."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a tensor on the GPU")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    shape = t.shape
    if len(shape) == 3 and (H is None or shape[1] == H) and (d is None or shape[2] == d):
        T, h, w = shape
        if t.is_contiguous():
            return h * w
        s = t.stride()
        if (w > 1 and s[2] != 1) or (h > 1 and s[1] != w):
            raise ValueError(f"{name}: the heads of a token must be contiguous")
        return s[0] if T > 1 else h * w
    raise ValueError(f"{name} must be [tokens, {'heads' if H is None else H}, "
                     f"{'d' if d is None else d}], got {tuple(shape)}")


def prompt_attention_workspace(dtype, S: int, Tq: int, Tk: int, Hq: int, d: int,
                               causal: bool = True) -> int:
    """Bytes of the workspace of ``prompt_attention_fwd`` (0: none needed)."""
    if dtype not in _DTYPES:
        raise ValueError(f"unsupported dtype {dtype}: use float32 or bfloat16")
    n = lib().avq_prompt_attention_workspace(_DTYPES[dtype], S, Tq, Tk, Hq, d, int(bool(causal)))
    if n < 0:
        raise ValueError(f"unsupported sizes S={S} Tq={Tq} Tk={Tk} Hq={Hq} d={d}")
    return n


# Sizes only; the call costs as much as the checks of two tensors.
_prompt_workspace_of = functools.lru_cache(maxsize=256)(prompt_attention_workspace)


def prompt_attention_fwd(Q, K, V, cu_q, cu_k, scale: float, causal: bool = True, Y=None,
                         with_lse: bool = False, lse=None, workspace=None, stream=None):
    """Exact attention of packed sequences (``avq_prompt_attention_fwd``).

    Q [Tq, Hq, d], K and V [Tk, Hkv, d]: packed token rows (a token's heads
    contiguous; slices of a fused projection are taken as they are). cu_q,
    cu_k: int32 [S + 1] on the GPU. With ``causal`` the queries are the last
    ones of their sequence's keys. Rows behind the last sequence are left as
    they were. workspace: a uint8 tensor of ``prompt_attention_workspace(...)``
    bytes (allocated if needed and not given). Returns Y [Tq, Hq, d], or
    (Y, lse) with ``with_lse`` (lse: fp32 [Tq, Hq]).
    """
    q_stride = _rows(Q, "Q")
    Tq, Hq, d = Q.shape
    k_stride = _rows(K, "K", d=d, dtype=Q.dtype)
    Tk, Hkv = K.shape[0], K.shape[1]
    v_stride = _rows(V, "V", Hkv, d, Q.dtype)
    if V.shape[0] != Tk:
        raise ValueError(f"V must have {Tk} tokens, got {V.shape[0]}")
    _dev(cu_q, "cu_q", torch.int32)
    _dev(cu_k, "cu_k", torch.int32, cu_q.shape)
    if cu_q.dim() != 1 or cu_q.shape[0] < 2:
        raise ValueError(f"cu_q must be [sequences + 1], got {tuple(cu_q.shape)}")
    s = _launch_stream(stream, Q.device)
    if Y is None:
        Y = _empty(stream, (Tq, Hq, d), Q.dtype, Q.device)
    else:
        _dev(Y, "Y", Q.dtype, (Tq, Hq, d))
    if lse is not None:
        _dev(lse, "lse", torch.float32, (Tq, Hq))
    elif with_lse:
        lse = _empty(stream, (Tq, Hq), torch.float32, Q.device)
    S = cu_q.shape[0] - 1
    if workspace is not None:
        _dev(workspace, "workspace", torch.uint8)
    else:
        n = _prompt_workspace_of(Q.dtype, S, Tq, Tk, Hq, d, bool(causal))
        if n:
            workspace = _empty(stream, (n,), torch.uint8, Q.device)
    at = Q.get_device()
    if (not K.get_device() == V.get_device() == cu_q.get_device() == cu_k.get_device()
            == Y.get_device() == at or _elsewhere(lse, at) or _elsewhere(workspace, at)):
        _same_device(Q, K=K, V=V, cu_q=cu_q, cu_k=cu_k, Y=Y, lse=lse, workspace=workspace)
    _check(lib().avq_prompt_attention_fwd(
        _dtype_code(Q), S, Tq, Tk, Hq, Hkv, d, float(scale), int(bool(causal)),
        Q.data_ptr(), q_stride, K.data_ptr(), k_stride, V.data_ptr(), v_stride, cu_q.data_ptr(),
        cu_k.data_ptr(), Y.data_ptr(), _ptr(lse), _ptr(workspace),
        0 if workspace is None else workspace.numel(), s))
    return (Y, lse) if with_lse else Y


def cache_page_bytes(dtype: torch.dtype, page_size: int, d: int, fp4: bool = False) -> int:
    """Bytes of one (page, key-value head) of a paged cache: the cache is a
    uint8 tensor [n_pages, Hkv, cache_page_bytes(...)]."""
    if dtype not in _DTYPES:
        raise ValueError(f"unsupported dtype {dtype}: use float32 or bfloat16")
    n = lib().avq_cache_page_bytes(_DTYPES[dtype], int(bool(fp4)), page_size, d)
    if n < 0:
        raise ValueError(f"unsupported page_size={page_size} d={d}")
    return n


_cache_page_bytes_of = functools.lru_cache(maxsize=256)(cache_page_bytes)


def _cache(cache, block_table, dtype, page_size, d, fp4, S=None):
    """Checks a cache and its block table; returns (n_pages, Hkv, S, max_pages)."""
    _dev(cache, "cache", torch.uint8)
    shape = cache.shape
    if len(shape) != 3:
        raise ValueError(f"cache must be [pages, heads, page bytes], got {tuple(shape)}")
    n_pages, Hkv, E = shape
    need = _cache_page_bytes_of(dtype, page_size, d, bool(fp4))
    if E != need:
        raise ValueError(f"cache holds {E} bytes per page and head, expected {need}")
    _dev(block_table, "block_table", torch.int32)
    table = block_table.shape
    if len(table) != 2 or (S is not None and table[0] != S):
        raise ValueError(f"block_table must be [{'sequences' if S is None else S}, pages], "
                         f"got {tuple(table)}")
    return n_pages, Hkv, table[0], table[1]


def cache_append(K, V, cache, block_table, start, page_size: int, cu=None, Q=None, cos=None,
                 sin=None, interleaved: bool = False, fp4: bool = False, Q_out=None,
                 with_K: bool = False, K_out=None, stream=None):
    """Appends keys (rotated to their positions) and values to a paged cache
    (``avq_cache_append``), and rotates the same tokens' queries.

    K, V [T, Hkv, d] and Q [T, Hq, d]: packed token rows as for
    ``prompt_attention_fwd``; cu int32 [S + 1], or None for one token per
    sequence (T = S); start int32 [S]: tokens cached before; cos, sin fp32
    [n_pos, rot / 2] (None: no rotation). The cache is written in place.
    Returns (Q_out, K_out): the rotated queries (None without Q) and, with
    ``with_K`` or a buffer, the rotated keys (otherwise None).
    """
    k_stride = _rows(K, "K")
    T, Hkv, d = K.shape
    v_stride = _rows(V, "V", Hkv, d, K.dtype)
    if V.shape[0] != T:
        raise ValueError(f"V must have {T} tokens, got {V.shape[0]}")
    _dev(start, "start", torch.int32)
    if start.dim() != 1:
        raise ValueError(f"start must be [sequences], got {tuple(start.shape)}")
    S = start.shape[0]
    n_pages, heads, _, max_pages = _cache(cache, block_table, K.dtype, page_size, d, fp4, S)
    if heads != Hkv:
        raise ValueError(f"cache holds {heads} heads, expected {Hkv}")
    if cu is not None:
        _dev(cu, "cu", torch.int32, (S + 1,))
    rot = n_pos = 0
    if (cos is None) != (sin is None):
        raise ValueError("cos and sin come together")
    if cos is not None:
        _dev(cos, "cos", torch.float32)
        _dev(sin, "sin", torch.float32, cos.shape)
        if cos.dim() != 2:
            raise ValueError(f"cos must be [positions, rot / 2], got {tuple(cos.shape)}")
        n_pos, rot = cos.shape[0], 2 * cos.shape[1]
        if rot == 0:
            raise ValueError("cos holds no angles: pass None for no rotation")
    s = _launch_stream(stream, K.device)
    Hq, q_stride = Hkv, 0
    if Q is not None:
        q_stride = _rows(Q, "Q", d=d, dtype=K.dtype)
        Hq = Q.shape[1]
        if Q.shape[0] != T:
            raise ValueError(f"Q must have {T} tokens, got {Q.shape[0]}")
        if Q_out is None:
            Q_out = _empty(stream, (T, Hq, d), Q.dtype, Q.device)
        else:
            _dev(Q_out, "Q_out", Q.dtype, (T, Hq, d))
    elif Q_out is not None:
        raise ValueError("Q_out without Q")
    if K_out is not None:
        _dev(K_out, "K_out", K.dtype, (T, Hkv, d))
    elif with_K:
        K_out = _empty(stream, (T, Hkv, d), K.dtype, K.device)
    at = K.get_device()
    if (not V.get_device() == cache.get_device() == block_table.get_device() == start.get_device()
            == at or _elsewhere(cu, at) or _elsewhere(Q, at) or _elsewhere(Q_out, at)
            or _elsewhere(cos, at) or _elsewhere(sin, at) or _elsewhere(K_out, at)):
        _same_device(K, V=V, cache=cache, block_table=block_table, start=start, cu=cu, Q=Q,
                     cos=cos, sin=sin, Q_out=Q_out, K_out=K_out)
    _check(lib().avq_cache_append(
        _dtype_code(K), int(bool(fp4)), S, T, Hq, Hkv, d, n_pages, page_size, max_pages, rot, n_pos,
        int(bool(interleaved)), _ptr(Q), q_stride, K.data_ptr(), k_stride, V.data_ptr(), v_stride,
        _ptr(cu), start.data_ptr(), block_table.data_ptr(), _ptr(cos), _ptr(sin),
        cache.data_ptr(), _ptr(Q_out), _ptr(K_out), s))
    return Q_out, K_out


def cache_gather(cache, block_table, start, cu, T: int, page_size: int, dtype, d: int,
                 fp4: bool = False, K=None, V=None, stream=None):
    """Cached positions start[s] + i as packed rows cu[s] + i
    (``avq_cache_gather``). Returns (K, V), [T, Hkv, d] in ``dtype``."""
    n_pages, Hkv, S, max_pages = _cache(cache, block_table, dtype, page_size, d, fp4)
    _dev(start, "start", torch.int32, (S,))
    _dev(cu, "cu", torch.int32, (S + 1,))
    s = _launch_stream(stream, cache.device)
    if K is None:
        K = _empty(stream, (T, Hkv, d), dtype, cache.device)
    else:
        _dev(K, "K", dtype, (T, Hkv, d))
    if V is None:
        V = _empty(stream, (T, Hkv, d), dtype, cache.device)
    else:
        _dev(V, "V", dtype, (T, Hkv, d))
    if not (block_table.get_device() == start.get_device() == cu.get_device() == K.get_device()
            == V.get_device() == cache.get_device()):
        _same_device(cache, block_table=block_table, start=start, cu=cu, K=K, V=V)
    _check(lib().avq_cache_gather(
        _DTYPES[dtype], int(bool(fp4)), S, T, Hkv, d, n_pages, page_size, max_pages,
        cache.data_ptr(), cu.data_ptr(), start.data_ptr(), block_table.data_ptr(), K.data_ptr(),
        V.data_ptr(), s))
    return K, V


def cache_attention_workspace(S: int, n_q: int, Hq: int, Hkv: int, d: int) -> int:
    """Bytes of the workspace of ``cache_attention_fwd``."""
    n = lib().avq_cache_attention_workspace(S, n_q, Hq, Hkv, d)
    if n < 0:
        raise ValueError(f"unsupported sizes S={S} n_q={n_q} Hq={Hq} Hkv={Hkv} d={d}")
    return n


_cache_workspace_of = functools.lru_cache(maxsize=256)(cache_attention_workspace)


def _newest(Q):
    """Checks the newest tokens' queries; returns their sizes and the elements from
    one token to the next."""
    if not isinstance(Q, torch.Tensor) or not Q.is_cuda:
        raise ValueError("Q must be a tensor on the GPU")
    if Q.dim() != 4:
        raise ValueError(f"Q must be [sequences, tokens, heads, d], got {tuple(Q.shape)}")
    S, n_q, Hq, d = Q.shape
    if Q.is_contiguous():
        return S, n_q, Hq, d, Hq * d
    if S > 1 and n_q > 1 and Q.stride(0) != n_q * Q.stride(1):
        raise ValueError("Q: the tokens must be evenly spaced")
    return S, n_q, Hq, d, _rows(Q.view(S * n_q, Hq, d), "Q")


def cache_attention_fwd(Q, cache, block_table, lens, page_size: int, scale: float,
                        fp4: bool = False, Y=None, with_lse: bool = False, lse=None,
                        workspace=None, stream=None):
    """Exact attention of each sequence's newest tokens over its paged cache
    (``avq_cache_attention_fwd``).

    Q [S, n_q, Hq, d]; lens int32 [S]: cached positions, the n_q tokens' own
    among them. workspace: a uint8 tensor of ``cache_attention_workspace(...)``
    bytes (allocated if needed and not given; a cache with room for at most
    ``CACHE_UNDIVIDED`` positions per sequence needs none). Returns Y
    [S, n_q, Hq, d], or (Y, lse) with ``with_lse`` (lse: fp32 [S, n_q, Hq]).
    """
    S, n_q, Hq, d, q_stride = _newest(Q)
    n_pages, Hkv, _, max_pages = _cache(cache, block_table, Q.dtype, page_size, d, fp4, S)
    _dev(lens, "lens", torch.int32, (S,))
    s = _launch_stream(stream, Q.device)
    if Y is None:
        Y = _empty(stream, (S, n_q, Hq, d), Q.dtype, Q.device)
    else:
        _dev(Y, "Y", Q.dtype, (S, n_q, Hq, d))
    if lse is not None:
        _dev(lse, "lse", torch.float32, (S, n_q, Hq))
    elif with_lse:
        lse = _empty(stream, (S, n_q, Hq), torch.float32, Q.device)
    if workspace is not None:
        _dev(workspace, "workspace", torch.uint8)
    else:
        n = _cache_workspace_of(S, n_q, Hq, Hkv, d)  # refuses unsupported sizes
        if max_pages * page_size > CACHE_UNDIVIDED:
            workspace = _empty(stream, (n,), torch.uint8, Q.device)
    at = Q.get_device()
    if (not cache.get_device() == block_table.get_device() == lens.get_device() == Y.get_device()
            == at or _elsewhere(workspace, at) or _elsewhere(lse, at)):
        _same_device(Q, cache=cache, block_table=block_table, lens=lens, Y=Y, lse=lse,
                     workspace=workspace)
    _check(lib().avq_cache_attention_fwd(
        _dtype_code(Q), int(bool(fp4)), S, n_q, Hq, Hkv, d, n_pages, page_size, max_pages,
        float(scale), Q.data_ptr(), q_stride, cache.data_ptr(), lens.data_ptr(),
        block_table.data_ptr(), Y.data_ptr(), _ptr(lse), _ptr(workspace),
        0 if workspace is None else workspace.numel(), s))
    return (Y, lse) if with_lse else Y


# ---- rotary positions with several axes, cross attention ----------------------


@functools.lru_cache(maxsize=256)
def _axis_bytes(axis: tuple) -> bytes:
    if not all(isinstance(a, int) and 0 <= a < 256 for a in axis):
        raise ValueError(f"axis must hold axis numbers, got {axis}")
    return bytes(axis)


def rotate_axes(Q, K, pos, cos, sin, axis, interleaved: bool = False, inverse: bool = False,
                Q_out=None, K_out=None, stream=None):
    """Rotates packed queries and keys by positions on several axes
    (``avq_rotate_axes``), or with ``inverse`` back: the gradients' way.

    Q [T, Hq, d], K [T, Hkv, d] or None: packed token rows as for
    ``prompt_attention_fwd``; pos int32 [T, n_axes] on the GPU; cos, sin fp32
    [n_pos, rot / 2]; axis: a tuple of rot / 2 axis numbers, one per pair. A token
    with a position outside the tables is not written. Returns (Q_out, K_out),
    which may be given and may be Q and K themselves; K_out is None without K.
    """
    q_stride = _rows(Q, "Q")
    T, Hq, d = Q.shape
    _dev(pos, "pos", torch.int32)
    if pos.dim() != 2 or pos.shape[0] != T:
        raise ValueError(f"pos must be [{T} tokens, axes], got {tuple(pos.shape)}")
    _dev(cos, "cos", torch.float32)
    _dev(sin, "sin", torch.float32, cos.shape)
    if cos.dim() != 2:
        raise ValueError(f"cos must be [positions, rot / 2], got {tuple(cos.shape)}")
    n_pos, half = cos.shape
    axes = _axis_bytes(axis if type(axis) is tuple else tuple(axis))
    if len(axes) != half:
        raise ValueError(f"axis must name the axes of {half} pairs, got {len(axes)}")
    Hkv, k_stride = Hq, 0
    if K is not None:
        k_stride = _rows(K, "K", d=d, dtype=Q.dtype)
        Hkv = K.shape[1]
        if K.shape[0] != T:
            raise ValueError(f"K must have {T} tokens, got {K.shape[0]}")
    elif K_out is not None:
        raise ValueError("K_out without K")
    s = _launch_stream(stream, Q.device)
    if Q_out is None:
        Q_out = _like(Q, stream)
    else:
        _dev(Q_out, "Q_out", Q.dtype, (T, Hq, d))
    if K_out is not None:
        _dev(K_out, "K_out", Q.dtype, (T, Hkv, d))
    elif K is not None:
        K_out = _like(K, stream)
    at = Q.get_device()
    if (not pos.get_device() == cos.get_device() == sin.get_device() == Q_out.get_device() == at
            or _elsewhere(K, at) or _elsewhere(K_out, at)):
        _same_device(Q, K=K, pos=pos, cos=cos, sin=sin, Q_out=Q_out, K_out=K_out)
    _check(lib().avq_rotate_axes(
        _dtype_code(Q), T, Hq, Hkv, d, 2 * half, pos.shape[1], axes, n_pos, int(bool(interleaved)),
        int(bool(inverse)), Q.data_ptr(), q_stride, _ptr(K), k_stride, pos.data_ptr(),
        cos.data_ptr(), sin.data_ptr(), Q_out.data_ptr(), _ptr(K_out), s))
    return Q_out, K_out


def cross_attention_workspace(dtype, S: int, Tq: int, Tk: int, Hq: int, Hkv: int, d: int,
                              backward: bool = False) -> int:
    """Bytes of the workspace of ``cross_attention_fwd`` (0: none needed) or
    ``cross_attention_bwd``."""
    if dtype not in _DTYPES:
        raise ValueError(f"unsupported dtype {dtype}: use float32 or bfloat16")
    L = lib()
    n = (L.avq_cross_attention_bwd_workspace if backward else L.avq_cross_attention_workspace)(
        _DTYPES[dtype], S, Tq, Tk, Hq, Hkv, d)
    if n < 0:
        raise ValueError(f"unsupported sizes S={S} Tq={Tq} Tk={Tk} Hq={Hq} Hkv={Hkv} d={d}")
    return n


_cross_workspace_of = functools.lru_cache(maxsize=256)(cross_attention_workspace)


def _cross(Q, K, V, cu_q, cu_k, mask):
    """Checks what the cross attention calls share; returns the strides."""
    q_stride = _rows(Q, "Q")
    d = Q.shape[2]
    k_stride = _rows(K, "K", d=d, dtype=Q.dtype)
    Tk = K.shape[0]
    v_stride = _rows(V, "V", K.shape[1], d, Q.dtype)
    if V.shape[0] != Tk:
        raise ValueError(f"V must have {Tk} tokens, got {V.shape[0]}")
    _dev(cu_q, "cu_q", torch.int32)
    _dev(cu_k, "cu_k", torch.int32, cu_q.shape)
    if cu_q.dim() != 1 or cu_q.shape[0] < 2:
        raise ValueError(f"cu_q must be [sources + 1], got {tuple(cu_q.shape)}")
    if mask is not None:
        if isinstance(mask, torch.Tensor) and mask.dtype not in (torch.bool, torch.uint8):
            raise ValueError(f"mask must be bool or uint8, got {mask.dtype}")
        _dev(mask, "mask", None, (Tk,))
    return q_stride, k_stride, v_stride


def cross_attention_fwd(Q, K, V, cu_q, cu_k, scale: float, mask=None, Y=None,
                        with_lse: bool = False, lse=None, workspace=None, stream=None):
    """Exact attention of packed queries over the states of their source
    (``avq_cross_attention_fwd``).

    Q [Tq, Hq, d], K and V [Tk, Hkv, d]: packed token rows as for
    ``prompt_attention_fwd``; cu_q, cu_k int32 [S + 1] on the GPU: the queries and
    the states of each source. mask: bool or uint8 [Tk], False for states that take
    no part. Rows behind the last source are left as they were. Returns Y
    [Tq, Hq, d], or (Y, lse) with ``with_lse`` (lse: fp32 [Tq, Hq], which
    ``cross_attention_bwd`` takes).
    """
    q_stride, k_stride, v_stride = _cross(Q, K, V, cu_q, cu_k, mask)
    Tq, Hq, d = Q.shape
    Tk, Hkv = K.shape[0], K.shape[1]
    s = _launch_stream(stream, Q.device)
    if Y is None:
        Y = _like(Q, stream)
    else:
        _dev(Y, "Y", Q.dtype, (Tq, Hq, d))
    if lse is not None:
        _dev(lse, "lse", torch.float32, (Tq, Hq))
    elif with_lse:
        lse = _empty(stream, (Tq, Hq), torch.float32, Q.device)
    S = cu_q.shape[0] - 1
    if workspace is not None:
        _dev(workspace, "workspace", torch.uint8)
    else:
        n = _cross_workspace_of(Q.dtype, S, Tq, Tk, Hq, Hkv, d)
        if n:
            workspace = _empty(stream, (n,), torch.uint8, Q.device)
    at = Q.get_device()
    if (not K.get_device() == V.get_device() == cu_q.get_device() == cu_k.get_device()
            == Y.get_device() == at or _elsewhere(mask, at) or _elsewhere(lse, at)
            or _elsewhere(workspace, at)):
        _same_device(Q, K=K, V=V, cu_q=cu_q, cu_k=cu_k, mask=mask, Y=Y, lse=lse,
                     workspace=workspace)
    _check(lib().avq_cross_attention_fwd(
        _dtype_code(Q), S, Tq, Tk, Hq, Hkv, d, float(scale), Q.data_ptr(), q_stride, K.data_ptr(),
        k_stride, V.data_ptr(), v_stride, cu_q.data_ptr(), cu_k.data_ptr(), _ptr(mask),
        Y.data_ptr(), _ptr(lse), _ptr(workspace), 0 if workspace is None else workspace.numel(), s))
    return (Y, lse) if with_lse else Y


def cross_attention_bwd(dY, Q, K, V, Y, lse, cu_q, cu_k, scale: float, mask=None, dQ=None, dK=None,
                        dV=None, workspace=None, stream=None):
    """Gradients of ``cross_attention_fwd`` (``avq_cross_attention_bwd``): dY
    [Tq, Hq, d] (packed rows; an expanded or otherwise overlapping gradient is
    refused), the forward call's inputs and its Y and lse. Rows that belong to no
    source are left as they were (pass dQ, dK, dV to set them). workspace: a uint8
    tensor of ``cross_attention_workspace(..., backward=True)`` bytes. Returns
    (dQ, dK, dV)."""
    q_stride, k_stride, v_stride = _cross(Q, K, V, cu_q, cu_k, mask)
    Tq, Hq, d = Q.shape
    Tk, Hkv = K.shape[0], K.shape[1]
    dy_stride = _rows(dY, "dY", Hq, d, Q.dtype)
    if dY.shape[0] != Tq:
        raise ValueError(f"dY must have {Tq} tokens, got {dY.shape[0]}")
    _dev(Y, "Y", Q.dtype, (Tq, Hq, d))
    _dev(lse, "lse", torch.float32, (Tq, Hq))
    s = _launch_stream(stream, Q.device)
    if dQ is None:
        dQ = _like(Q, stream)
    else:
        _dev(dQ, "dQ", Q.dtype, (Tq, Hq, d))
    if dK is None:
        dK = _like(K, stream)
    else:
        _dev(dK, "dK", Q.dtype, (Tk, Hkv, d))
    if dV is None:
        dV = _like(K, stream)
    else:
        _dev(dV, "dV", Q.dtype, (Tk, Hkv, d))
    S = cu_q.shape[0] - 1
    if workspace is not None:
        _dev(workspace, "workspace", torch.uint8)
    else:
        n = _cross_workspace_of(Q.dtype, S, Tq, Tk, Hq, Hkv, d, True)
        workspace = _empty(stream, (n,), torch.uint8, Q.device)
    at = Q.get_device()
    if (not dY.get_device() == K.get_device() == V.get_device() == Y.get_device()
            == lse.get_device() == cu_q.get_device() == cu_k.get_device() == dQ.get_device()
            == dK.get_device() == dV.get_device() == workspace.get_device() == at
            or _elsewhere(mask, at)):
        _same_device(Q, dY=dY, K=K, V=V, Y=Y, lse=lse, cu_q=cu_q, cu_k=cu_k, mask=mask, dQ=dQ,
                     dK=dK, dV=dV, workspace=workspace)
    _check(lib().avq_cross_attention_bwd(
        _dtype_code(Q), S, Tq, Tk, Hq, Hkv, d, float(scale), dY.data_ptr(), dy_stride,
        Q.data_ptr(), q_stride, K.data_ptr(), k_stride, V.data_ptr(), v_stride, Y.data_ptr(),
        lse.data_ptr(), cu_q.data_ptr(), cu_k.data_ptr(), _ptr(mask), dQ.data_ptr(), dK.data_ptr(),
        dV.data_ptr(), workspace.data_ptr(), workspace.numel(), s))
    return dQ, dK, dV


# ---- groups of sequences that share their first positions ----------------------


def cache_prefix_attention_workspace(S: int, n_groups: int, n_q: int, Hq: int, Hkv: int,
                                     d: int) -> int:
    """Bytes of the workspace of ``cache_prefix_attention_fwd``."""
    n = lib().avq_cache_prefix_attention_workspace(S, n_groups, n_q, Hq, Hkv, d)
    if n < 0:
        raise ValueError(f"unsupported sizes S={S} n_groups={n_groups} n_q={n_q} Hq={Hq} Hkv={Hkv} "
                         f"d={d}")
    return n


_prefix_workspace_of = functools.lru_cache(maxsize=256)(cache_prefix_attention_workspace)


def cache_prefix_attention_fwd(Q, cache, block_table, lens, cu_groups, shared, page_size: int,
                               scale: float, fp4: bool = False, Y=None, with_lse: bool = False,
                               lse=None, workspace=None, stream=None):
    """``cache_attention_fwd`` for groups of sequences that share their first
    positions, which are attended to once per group
    (``avq_cache_prefix_attention_fwd``).

    cu_groups int32 [groups + 1]: group g is the sequences cu_groups[g] ..
    cu_groups[g + 1] - 1; shared int32 [groups]: how many first positions they have in
    common (a sequence that holds fewer reads its own). Where groups are small or most
    positions are the sequences' own, ``cache_attention_fwd`` is faster. The other
    arguments, and what is returned, are those of ``cache_attention_fwd``; workspace: a
    uint8 tensor of ``cache_prefix_attention_workspace(...)`` bytes (allocated if needed
    and not given).
    """
    S, n_q, Hq, d, q_stride = _newest(Q)
    n_pages, Hkv, _, max_pages = _cache(cache, block_table, Q.dtype, page_size, d, fp4, S)
    _dev(lens, "lens", torch.int32, (S,))
    _dev(shared, "shared", torch.int32)
    if shared.dim() != 1:
        raise ValueError(f"shared must be [groups], got {tuple(shared.shape)}")
    n_groups = shared.shape[0]
    _dev(cu_groups, "cu_groups", torch.int32, (n_groups + 1,))
    s = _launch_stream(stream, Q.device)
    if Y is None:
        Y = _like(Q, stream)
    else:
        _dev(Y, "Y", Q.dtype, (S, n_q, Hq, d))
    if lse is not None:
        _dev(lse, "lse", torch.float32, (S, n_q, Hq))
    elif with_lse:
        lse = _empty(stream, (S, n_q, Hq), torch.float32, Q.device)
    if workspace is not None:
        _dev(workspace, "workspace", torch.uint8)
    else:
        n = _prefix_workspace_of(S, n_groups, n_q, Hq, Hkv, d)  # refuses unsupported sizes
        if max_pages * page_size > CACHE_UNDIVIDED:
            workspace = _empty(stream, (n,), torch.uint8, Q.device)
    at = Q.get_device()
    if (not cache.get_device() == block_table.get_device() == lens.get_device()
            == cu_groups.get_device() == shared.get_device() == Y.get_device() == at
            or _elsewhere(workspace, at) or _elsewhere(lse, at)):
        _same_device(Q, cache=cache, block_table=block_table, lens=lens, cu_groups=cu_groups,
                     shared=shared, Y=Y, lse=lse, workspace=workspace)
    _check(lib().avq_cache_prefix_attention_fwd(
        _dtype_code(Q), int(bool(fp4)), S, n_groups, n_q, Hq, Hkv, d, n_pages, page_size, max_pages,
        float(scale), Q.data_ptr(), q_stride, cache.data_ptr(), lens.data_ptr(),
        block_table.data_ptr(), cu_groups.data_ptr(), shared.data_ptr(), Y.data_ptr(), _ptr(lse),
        _ptr(workspace), 0 if workspace is None else workspace.numel(), s))
    return (Y, lse) if with_lse else Y
