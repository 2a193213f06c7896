"""Thin ctypes binding over libkvcrush.so: same names as the C ABI
(include/kvcrush.h), argument marshalling only.  torch is used for device
memory and the current HIP stream; every computation happens in the library's
kernels.  There is no fallback: if the library is missing or a call fails, an
exception is raised.
"""
from __future__ import annotations

import contextlib
import ctypes
import os

import torch
from torch.autograd import forward_ad

_PKG_DIR = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG_DIR, "libkvcrush.so")

F32, BF16, F16 = 0, 1, 2
E4M3, I8, I4 = 3, 4, 5     # kvcrush_format: cache rows in 8 or 4 bits
ANCHORS = {"random": 0, "mean": 1, "alternating": 2, "explicit": 3}
OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_HIP = range(5)

EXPORTS = (
    "kvcrush_scores_workspace", "kvcrush_scores", "kvcrush_row_lse_workspace", "kvcrush_row_lse",
    "kvcrush_pool_scores",
    "kvcrush_select_workspace", "kvcrush_select", "kvcrush_select_static", "kvcrush_compact", "kvcrush_scores_append_workspace",
    "kvcrush_scores_append", "kvcrush_decode_step", "kvcrush_compact_cache", "kvcrush_compact_block_table", "kvcrush_status_string",
    "kvcrush_cache_write", "kvcrush_cache_read", "kvcrush_attend_workspace", "kvcrush_attend", "kvcrush_block_bounds",
    "kvcrush_block_select_workspace", "kvcrush_block_select", "kvcrush_version",
)


class KVCrushError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {status_string(status)} (status {status})")


class Shape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "Hq", "Hkv", "S", "D", "dtype", "reduce_groups",
                                                 "obs_window")] + [("softmax_scale", ctypes.c_float),
                                                                   ("q_stride", ctypes.c_int64 * 3),
                                                                   ("k_stride", ctypes.c_int64 * 3)]


class SelectArgs(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "Hs", "S", "budget", "n_important", "bit_topk", "anchor",
                                                 "score_stride", "n_sink", "n_recent", "unit")] + [
        ("anchor_seed", ctypes.c_uint64), ("anchor_bits", ctypes.c_void_p)]


class Cache(ctypes.Structure):
    """kvcrush_cache; made by make_cache, which also keeps the tensors that it points to."""
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "Hkv", "S", "D", "capacity", "format", "block_size", "n_blocks")] + [
        (n, ctypes.c_void_p) for n in ("k", "v", "k_param", "v_param", "lengths", "block_table")]


class AttendArgs(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("Hq", "T", "dtype")] + [
        ("softmax_scale", ctypes.c_float), ("q_stride", ctypes.c_int64 * 3), ("out_stride", ctypes.c_int64 * 3),
        ("mask", ctypes.c_void_p), ("mask_stride", ctypes.c_int64), ("n_new", ctypes.c_void_p), ("blocks", ctypes.c_void_p),
        ("n_list", ctypes.c_int32), ("unit", ctypes.c_int32)]


_lib = None


def load() -> ctypes.CDLL:
    """Load the library built by `paper_2503_00022_amd.build` (never builds, never falls back)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2503_00022_amd.build` "
                "(or __graft_entry__.build()); there is no CPU fallback")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
        L.kvcrush_scores_workspace.argtypes = [ctypes.POINTER(Shape)]
        L.kvcrush_scores_workspace.restype = sz
        L.kvcrush_scores.argtypes = [ctypes.POINTER(Shape), vp, vp, vp, vp, vp, sz, vp]
        L.kvcrush_scores.restype = ctypes.c_int
        L.kvcrush_row_lse_workspace.argtypes = [ctypes.POINTER(Shape)]
        L.kvcrush_row_lse_workspace.restype = sz
        L.kvcrush_row_lse.argtypes = [ctypes.POINTER(Shape), vp, vp, vp, vp, sz, vp]
        L.kvcrush_row_lse.restype = ctypes.c_int
        L.kvcrush_pool_scores.argtypes = [i32, i32, i32, vp, vp, vp]
        L.kvcrush_pool_scores.restype = ctypes.c_int
        L.kvcrush_select_workspace.argtypes = [ctypes.POINTER(SelectArgs)]
        L.kvcrush_select_workspace.restype = sz
        L.kvcrush_select.argtypes = [ctypes.POINTER(SelectArgs), vp, vp, vp, vp, vp, sz, vp]
        L.kvcrush_select.restype = ctypes.c_int
        L.kvcrush_select_static.argtypes = [ctypes.POINTER(SelectArgs), vp, vp, vp, vp, vp]
        L.kvcrush_select_static.restype = ctypes.c_int
        L.kvcrush_compact.argtypes = [i32] * 6 + [vp, vp, vp, vp, i32, vp, vp, vp]
        L.kvcrush_compact.restype = ctypes.c_int
        L.kvcrush_scores_append_workspace.argtypes = [ctypes.POINTER(Shape), i32]
        L.kvcrush_scores_append_workspace.restype = sz
        L.kvcrush_scores_append.argtypes = [ctypes.POINTER(Shape), i32, vp, vp, vp, vp, i32, vp, vp, sz, vp]
        L.kvcrush_scores_append.restype = ctypes.c_int
        L.kvcrush_decode_step.argtypes = [ctypes.POINTER(Shape), i32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.kvcrush_decode_step.restype = ctypes.c_int
        L.kvcrush_compact_cache.argtypes = [i32] * 8 + [vp] * 8
        L.kvcrush_compact_cache.restype = ctypes.c_int
        L.kvcrush_compact_block_table.argtypes = [i32] * 4 + [vp] * 4
        L.kvcrush_compact_block_table.restype = ctypes.c_int
        cache, attend, strides = ctypes.POINTER(Cache), ctypes.POINTER(AttendArgs), ctypes.POINTER(ctypes.c_int64)
        L.kvcrush_cache_write.argtypes = [cache, i32, i32, vp, vp, strides, strides, vp, vp]
        L.kvcrush_cache_write.restype = ctypes.c_int
        L.kvcrush_cache_read.argtypes = [cache, i32, vp, i32, vp, vp, vp]
        L.kvcrush_cache_read.restype = ctypes.c_int
        L.kvcrush_attend_workspace.argtypes = [cache, attend]
        L.kvcrush_attend_workspace.restype = sz
        L.kvcrush_attend.argtypes = [cache, attend, vp, vp, vp, vp, sz, vp]
        L.kvcrush_attend.restype = ctypes.c_int
        L.kvcrush_block_bounds.argtypes = [cache, i32, i32, vp, vp, vp, vp]
        L.kvcrush_block_bounds.restype = ctypes.c_int
        L.kvcrush_block_select_workspace.argtypes = [cache, attend, i32, i32]
        L.kvcrush_block_select_workspace.restype = sz
        L.kvcrush_block_select.argtypes = [cache, attend, i32, i32, i32, i32, vp, vp, vp, vp, vp, sz, vp]
        L.kvcrush_block_select.restype = ctypes.c_int
        L.kvcrush_status_string.argtypes = [ctypes.c_int]
        L.kvcrush_status_string.restype = ctypes.c_char_p
        L.kvcrush_version.restype = i32
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return load().kvcrush_status_string(status).decode()


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float16:
        return F16
    raise TypeError(f"kvcrush handles float32, bfloat16 and float16, got {t.dtype}")


def _dev(t: torch.Tensor, name: str) -> torch.Tensor:
    if t.device.type != "cuda":
        raise ValueError(f"{name} must live in GPU memory")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


def _dev_rows(t: torch.Tensor, name: str) -> torch.Tensor:
    """A [B,H,S,D] tensor or view on the GPU whose D values are contiguous (any other strides)."""
    if t.device.type != "cuda":
        raise ValueError(f"{name} must live in GPU memory")
    if t.dim() != 4 or (t.shape[3] > 1 and t.stride(3) != 1):
        raise ValueError(f"{name} must be [B,H,S,D] with the D values contiguous")
    return t


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


# The current stream's handle without the Stream object around it (0.1 us instead of 2.7, of the 15 that a whole
# decoding step has); read on every call.
_current_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda device: torch.cuda.current_stream(device).cuda_stream)


def _stream(stream=None):
    return ctypes.c_void_p(_current_raw_stream(torch.cuda.current_device()) if stream is None else stream.cuda_stream)


_no_context = contextlib.nullcontext()


def _memory_of(stream):
    """In this context a call with stream= allocates what it makes: in that stream's memory.  Of the current stream's, a block
    may come back that work still pending there reads or writes."""
    return _no_context if stream is None else torch.cuda.stream(stream)


def _hand_over(stream, *results):
    """Results made in `stream`'s memory go to the caller, who uses them under the current stream."""
    if stream is not None:
        for t in results:
            if t is not None:
                t.record_stream(torch.cuda.current_stream(t.device))


def _check(status: int, what: str):
    if status != OK:
        raise KVCrushError(status, what)


def make_shape(q: torch.Tensor, k: torch.Tensor, reduce_groups: bool, window: int = 0, scale: float = 0.0) -> Shape:
    B, Hq, S, D = q.shape
    shape = Shape(B, Hq, k.shape[1], S, D, _dtype_code(q), int(bool(reduce_groups)), int(window), float(scale))
    for t, field in ((q, shape.q_stride), (k, shape.k_stride)):
        if not t.is_contiguous():                     # views (a transposed projection output, a slice of a
            field[:] = list(t.stride()[:3])           # padded buffer) are read in place, never copied
    return shape


def kvcrush_scores_workspace(shape: Shape) -> int:
    return int(load().kvcrush_scores_workspace(ctypes.byref(shape)))


def kvcrush_scores(q, k, reduce_groups: bool, lse=None, scores=None, workspace=None, stream=None, window=0,
                   scale=0.0):
    """q [B,Hq,S,D], k [B,Hkv,S,D] on the GPU -> scores [B,Hs,S] fp32.
    window = W > 0 restricts the contributing queries to the last min(W, S).
    scale: factor on Q.K before the softmax (0: 1/sqrt(D)).
    Returns (scores, workspace); the workspace's first B*Hq*S floats hold the
    row log-sum-exps when `lse` was not supplied.
    q and k may be views with any sequence, head and token strides (D contiguous)."""
    q, k = _dev_rows(q, "q"), _dev_rows(k, "k")
    if q.dtype != k.dtype or q.dim() != 4 or k.dim() != 4 or q.shape[0] != k.shape[0] \
            or q.shape[2:] != k.shape[2:]:
        raise ValueError("q and k must be [B,H,S,D] tensors of one dtype with matching B, S, D")
    shape = make_shape(q, k, reduce_groups, window, scale)
    Hs = shape.Hkv if reduce_groups else shape.Hq
    need = kvcrush_scores_workspace(shape)
    made_scores = made_ws = None
    with _memory_of(stream):
        if scores is None:
            scores = made_scores = torch.empty(shape.B, Hs, shape.S, dtype=torch.float32, device=q.device)
        if workspace is None:
            workspace = made_ws = torch.empty(max(need, 16), dtype=torch.uint8, device=q.device)
    if lse is not None:
        lse = _dev(lse, "lse")
        if lse.dtype != torch.float32 or tuple(lse.shape) != (shape.B, shape.Hq, shape.S):
            raise ValueError("lse must be fp32 [B,Hq,S]")
    st = load().kvcrush_scores(ctypes.byref(shape), _ptr(q), _ptr(k), _ptr(lse), _ptr(_dev(scores, "scores")),
                               _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream(stream))
    _hand_over(stream, made_scores, made_ws)
    _check(st, "kvcrush_scores")
    return scores, workspace


def kvcrush_row_lse_workspace(shape: Shape) -> int:
    return int(load().kvcrush_row_lse_workspace(ctypes.byref(shape)))


def kvcrush_row_lse(q, k, lse_out=None, stream=None, window=0, workspace="auto", scale=0.0):
    """q [B,Hq,S,D], k [B,Hkv,S,D] on the GPU -> natural-log row normalisers fp32 [B,Hq,S]
    (with window = W > 0 only the rows of the last min(W, S) queries are defined).
    workspace: a uint8 tensor, None (run without scratch memory) or "auto" (allocate what
    kvcrush_row_lse_workspace asks for)."""
    q, k = _dev_rows(q, "q"), _dev_rows(k, "k")
    shape = make_shape(q, k, False, window, scale)
    made = None
    with _memory_of(stream):
        if lse_out is None:
            lse_out = made = torch.empty(shape.B, shape.Hq, shape.S, dtype=torch.float32, device=q.device)
        if isinstance(workspace, str):
            workspace = torch.empty(max(kvcrush_row_lse_workspace(shape), 16), dtype=torch.uint8, device=q.device)
    st = load().kvcrush_row_lse(ctypes.byref(shape), _ptr(q), _ptr(k), _ptr(_dev(lse_out, "lse_out")),
                                _ptr(workspace), 0 if workspace is None else workspace.numel(),
                                _stream(stream))
    _hand_over(stream, made)
    _check(st, "kvcrush_row_lse")
    return lse_out


def kvcrush_pool_scores(scores, kernel: int, out=None, stream=None):
    """Centred sliding maximum of width `kernel` (odd) along the last axis of fp32 scores."""
    scores = _dev(scores, "scores")
    if scores.dtype != torch.float32:
        raise ValueError("scores must be fp32")
    made = None
    if out is None:
        with _memory_of(stream):
            out = made = torch.empty_like(scores)
    S = scores.shape[-1]
    st = load().kvcrush_pool_scores(scores.numel() // S, S, kernel, _ptr(scores), _ptr(_dev(out, "out")),
                                    _stream(stream))
    _hand_over(stream, made)
    _check(st, "kvcrush_pool_scores")
    return out


def lse_from_workspace(workspace: torch.Tensor, B: int, Hq: int, S: int) -> torch.Tensor:
    return workspace[: B * Hq * S * 4].view(torch.float32).view(B, Hq, S)


def make_select_args(B, Hs, S, budget, n_important, bit_topk=0, anchor="alternating", anchor_seed=0,
                     anchor_bits=None, n_sink=0, n_recent=0, score_stride=0, unit=0) -> SelectArgs:
    return SelectArgs(B, Hs, S, budget, n_important, bit_topk, ANCHORS[anchor] if isinstance(anchor, str) else anchor,
                      score_stride, n_sink, n_recent, unit, anchor_seed & (2**64 - 1),
                      None if anchor_bits is None else anchor_bits.data_ptr())


def kvcrush_select_workspace(args: SelectArgs) -> int:
    return int(load().kvcrush_select_workspace(ctypes.byref(args)))


def kvcrush_select(scores, budget, n_important, bit_topk=0, anchor="alternating", anchor_seed=0,
                   anchor_bits=None, want_kind=True, want_bits=False, idx=None, workspace=None, stream=None,
                   n_sink=0, n_recent=0, valid_len=None, unit=0):
    """scores [B,Hs,S] fp32 on the GPU -> (idx int32 [B,budget], kind uint8 | None, bits int64 [B,S,W] | None).
    n_sink / n_recent tokens at the two ends are always kept; the rest of the budget goes to the middle.
    valid_len: scores is a capacity-strided cache [B,Hs,capacity] of which the first valid_len tokens count."""
    scores = _dev(scores, "scores")
    if scores.dtype != torch.float32 or scores.dim() != 3:
        raise ValueError("scores must be fp32 [B,Hs,S]")
    B, Hs, S = scores.shape
    stride = 0
    if valid_len is not None:
        stride, S = S, int(valid_len)
    if anchor_bits is not None:
        anchor_bits = _dev(anchor_bits, "anchor_bits")
    args = make_select_args(B, Hs, S, budget, n_important, bit_topk, anchor, anchor_seed, anchor_bits,
                            n_sink, n_recent, stride, unit)
    dev = scores.device
    made = None
    if unit > 1:   # one vector of Hs * unit bits per unit of the middle
        bits_shape = (B, max(S - n_sink - n_recent, 0) // unit, (Hs * unit + 63) // 64)
    else:
        bits_shape = (B, S, (Hs + 63) // 64)
    with _memory_of(stream):
        if idx is None:
            idx = made = torch.empty(B, budget, dtype=torch.int32, device=dev)
        kind = torch.empty(B, budget, dtype=torch.uint8, device=dev) if want_kind else None
        bits = torch.empty(bits_shape, dtype=torch.int64, device=dev) if want_bits else None
        if workspace is None:
            workspace = torch.empty(max(kvcrush_select_workspace(args), 16), dtype=torch.uint8, device=dev)
    st = load().kvcrush_select(ctypes.byref(args), _ptr(scores), _ptr(idx), _ptr(kind), _ptr(bits),
                               _ptr(workspace), workspace.numel(), _stream(stream))
    _hand_over(stream, made, kind, bits)
    _check(st, "kvcrush_select")
    return idx, kind, bits


SELECT_STATIC_MAX_BYTES = 4 << 20   # KVCRUSH_SELECT_STATIC_MAX_BYTES


def kvcrush_select_static(args: SelectArgs, scores, idx, kind=None, bits=None, stream=None):
    """kvcrush_select on the library's own fixed scratch array: every buffer is the caller's, nothing
    is allocated here or in the library.  args from make_select_args; idx int32 [B,budget], kind uint8
    [B,budget] or None, bits int64 or None, all preallocated on the GPU."""
    st = load().kvcrush_select_static(ctypes.byref(args), _ptr(_dev(scores, "scores")), _ptr(_dev(idx, "idx")),
                                      _ptr(kind), _ptr(bits), _stream(stream))
    _check(st, "kvcrush_select_static")
    return idx, kind, bits


def kvcrush_compact(k, v, idx, block_table=None, block_size=16, dense_shape=None, k_out=None, v_out=None,
                    stream=None, validate=True):
    """Dense k, v [B,Hkv,S,D]; or paged pools [n_blocks,block_size,Hkv,D] with block_table
    [B,S/block_size] int32 and dense_shape=(B,Hkv,S,D).  Returns (k_out, v_out) [B,Hkv,budget,D]."""
    k, v, idx = _dev(k, "k"), _dev(v, "v"), _dev(idx, "idx")
    if idx.dtype != torch.int32 or k.dtype != v.dtype or k.shape != v.shape:
        raise ValueError("idx must be int32; k and v must match")
    if block_table is None:
        B, Hkv, S, D = k.shape
    else:
        B, Hkv, S, D = dense_shape
        block_table = _dev(block_table, "block_table")
        if block_table.dtype != torch.int32 or tuple(block_table.shape) != (B, S // block_size):
            raise ValueError("block_table must be int32 [B, S/block_size]")
        if tuple(k.shape[1:]) != (block_size, Hkv, D):
            raise ValueError("paged pools must be [n_blocks, block_size, Hkv, D]")
    budget = idx.shape[1]
    if idx.shape[0] != B:
        raise ValueError("idx must be [B,budget]")
    if validate:  # host-side bounds checks of the gather's index operands (synchronises)
        if budget and (int(idx.min()) < 0 or int(idx.max()) >= S):
            raise ValueError("idx out of range")
        if block_table is not None and (int(block_table.min()) < 0 or int(block_table.max()) >= k.shape[0]):
            raise ValueError("block_table names a block outside the pool")
    made_k = made_v = None
    with _memory_of(stream):
        if k_out is None:
            k_out = made_k = torch.empty(B, Hkv, budget, D, dtype=k.dtype, device=k.device)
        if v_out is None:
            v_out = made_v = torch.empty(B, Hkv, budget, D, dtype=v.dtype, device=v.device)
    st = load().kvcrush_compact(B, Hkv, S, D, _dtype_code(k), budget, _ptr(k), _ptr(v), _ptr(idx),
                                _ptr(block_table), block_size, _ptr(_dev(k_out, "k_out")),
                                _ptr(_dev(v_out, "v_out")), _stream(stream))
    _hand_over(stream, made_k, made_v)
    _check(st, "kvcrush_compact")
    return k_out, v_out


def kvcrush_scores_append_workspace(shape: Shape, capacity: int) -> int:
    return int(load().kvcrush_scores_append_workspace(ctypes.byref(shape), capacity))


def kvcrush_scores_append(q_new, k_cache, scores_cache, S: int, reduce_groups: bool, workspace=None, stream=None,
                          lengths=None, block_table=None, block_size=16, scale=0.0):
    """One decoding step, in place on scores_cache [B,Hs,capacity] fp32: the new token's queries
    q_new [B,Hq,D] attend to the first S tokens of k_cache [B,Hkv,capacity,D] (the new key included).
    lengths: optional int32 [B] on the GPU with each sequence's own valid length (S is then their bound).
    block_table: k_cache is then a paged pool [n_blocks,block_size,Hkv,D], block_table int32
    [B,capacity/block_size]."""
    q_new, k_cache, scores_cache = _dev(q_new, "q_new"), _dev(k_cache, "k_cache"), _dev(scores_cache, "scores_cache")
    if q_new.dim() != 3 or k_cache.dim() != 4 or q_new.dtype != k_cache.dtype or scores_cache.dtype != torch.float32:
        raise ValueError("q_new [B,Hq,D] and k_cache [B,Hkv,capacity,D] of one dtype, scores_cache fp32")
    B, Hq, D = q_new.shape
    if block_table is None:
        Hkv, cap = k_cache.shape[1], k_cache.shape[2]
        if k_cache.shape[0] != B or k_cache.shape[3] != D:
            raise ValueError("q_new and k_cache disagree on B or D")
    else:
        block_table = _dev(block_table, "block_table")
        Hkv, cap = k_cache.shape[2], block_table.shape[1] * block_size
        if block_table.dtype != torch.int32 or block_table.shape[0] != B or k_cache.shape[1] != block_size \
                or k_cache.shape[3] != D:
            raise ValueError("paged k_cache must be [n_blocks,block_size,Hkv,D] with block_table int32 [B,n]")
    if tuple(scores_cache.shape) != (B, Hkv if reduce_groups else Hq, cap):
        raise ValueError("scores_cache must be [B,Hs,capacity]")
    shape = Shape(B, Hq, Hkv, int(S), D, _dtype_code(q_new), int(bool(reduce_groups)), 0, float(scale))
    if workspace is None:
        with _memory_of(stream):
            workspace = torch.empty(max(kvcrush_scores_append_workspace(shape, cap), 16), dtype=torch.uint8,
                                    device=q_new.device)
    if lengths is not None:
        lengths = _dev(lengths, "lengths")
        if lengths.dtype != torch.int32 or tuple(lengths.shape) != (B,):
            raise ValueError("lengths must be int32 [B]")
    st = load().kvcrush_scores_append(ctypes.byref(shape), cap, _ptr(lengths), _ptr(q_new), _ptr(k_cache),
                                      _ptr(block_table), block_size, _ptr(scores_cache), _ptr(workspace),
                                      workspace.numel(), _stream(stream))
    _check(st, "kvcrush_scores_append")
    return scores_cache


def _decode_step(shape, capacity, q_new, k_new, v_new, k, v, scores, workspace, stream=None):
    """The call itself, on addresses that the caller has checked."""
    st = load().kvcrush_decode_step(ctypes.byref(shape), capacity, q_new, k_new, v_new, k, v, scores, workspace.data_ptr(),
                                    workspace.numel(), _stream(stream))
    _check(st, "kvcrush_decode_step")


def kvcrush_decode_step(q_new, k_new, v_new, k_cache, v_cache, scores_cache, S: int, reduce_groups: bool, workspace,
                        stream=None, scale=0.0):
    """kvcrush_scores_append on dense caches whose row S - 1 the call itself fills with k_new and v_new [B,Hkv,D]."""
    for name, t in (("q_new", q_new), ("k_new", k_new), ("v_new", v_new), ("k_cache", k_cache), ("v_cache", v_cache),
                    ("scores_cache", scores_cache), ("workspace", workspace)):
        _dev(t, name)
    if q_new.dim() != 3 or k_cache.dim() != 4 or scores_cache.dtype != torch.float32 \
            or any(t.dtype != k_cache.dtype for t in (q_new, k_new, v_new, v_cache)):
        raise ValueError("q_new [B,Hq,D] and k_cache [B,Hkv,capacity,D] of one dtype, scores_cache fp32")
    B, Hq, D = q_new.shape
    Hkv, cap = k_cache.shape[1], k_cache.shape[2]
    if tuple(k_cache.shape) != (B, Hkv, cap, D) or v_cache.shape != k_cache.shape \
            or tuple(k_new.shape) != (B, Hkv, D) or v_new.shape != k_new.shape:
        raise ValueError("q_new, k_new, v_new and the caches disagree on B, Hkv or D")
    if tuple(scores_cache.shape) != (B, Hkv if reduce_groups else Hq, cap):
        raise ValueError("scores_cache must be [B,Hs,capacity]")
    shape = Shape(B, Hq, Hkv, int(S), D, _dtype_code(q_new), int(bool(reduce_groups)), 0, float(scale))
    _decode_step(shape, cap, q_new.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(),
                 scores_cache.data_ptr(), workspace, stream)
    return scores_cache


def kvcrush_compact_cache(k, v, scores, idx, k_out, v_out, scores_out, stream=None):
    """Eviction on capacity-strided caches: the tokens idx [B,budget] of k, v [B,Hkv,cap_src,D] and of
    scores [B,Hs,cap_src] move to the front of k_out, v_out [B,Hkv,cap_dst,D], scores_out [B,Hs,cap_dst]."""
    for name, t in (("k", k), ("v", v), ("scores", scores), ("idx", idx), ("k_out", k_out), ("v_out", v_out),
                    ("scores_out", scores_out)):
        _dev(t, name)
    if idx.dtype != torch.int32 or k.dtype != v.dtype or k.shape != v.shape or k_out.shape != v_out.shape \
            or k_out.dtype != k.dtype or scores.dtype != torch.float32 or scores_out.dtype != torch.float32:
        raise ValueError("idx int32; k, v, k_out, v_out of one dtype; scores fp32")
    B, Hkv, cap_src, D = k.shape
    cap_dst, Hs = k_out.shape[2], scores.shape[1]
    if tuple(scores.shape) != (B, Hs, cap_src) or tuple(scores_out.shape) != (B, Hs, cap_dst) \
            or tuple(k_out.shape) != (B, Hkv, cap_dst, D) or idx.shape[0] != B:
        raise ValueError("shapes of the source and destination caches do not match")
    st = load().kvcrush_compact_cache(B, Hkv, Hs, D, _dtype_code(k), cap_src, cap_dst, idx.shape[1], _ptr(k),
                                      _ptr(v), _ptr(scores), _ptr(idx), _ptr(k_out), _ptr(v_out),
                                      _ptr(scores_out), _stream(stream))
    _check(st, "kvcrush_compact_cache")
    return k_out, v_out, scores_out


def kvcrush_compact_block_table(idx, block_table, block_size: int, out=None, stream=None):
    """Page-level eviction on a paged pool: idx [B,budget] (whole blocks, from kvcrush_select with
    unit == block_size) and block_table [B,S/block_size] -> the kept blocks [B,budget/block_size]."""
    idx, block_table = _dev(idx, "idx"), _dev(block_table, "block_table")
    if idx.dtype != torch.int32 or block_table.dtype != torch.int32 or idx.shape[0] != block_table.shape[0]:
        raise ValueError("idx and block_table must be int32 with the same batch size")
    B, budget = idx.shape
    made = None
    if out is None:
        with _memory_of(stream):
            out = made = torch.empty(B, budget // block_size, dtype=torch.int32, device=idx.device)
    st = load().kvcrush_compact_block_table(B, block_table.shape[1] * block_size, budget, block_size, _ptr(idx),
                                            _ptr(block_table), _ptr(_dev(out, "out")), _stream(stream))
    _hand_over(stream, made)
    _check(st, "kvcrush_compact_block_table")
    return out


# ------------------------------------------------------------------------------------------- using the cache
_FORMATS = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16, torch.float8_e4m3fn: E4M3, torch.int8: I8,
            torch.uint8: I4}
_VALUES = (torch.float32, torch.bfloat16, torch.float16)
CODES = {"e4m3": torch.float8_e4m3fn, "i8": torch.int8, "i4": torch.uint8}   # element types of quantised caches


def make_cache(k, v, S: int, k_param=None, v_param=None, lengths=None, block_table=None) -> Cache:
    """Describes a layer's KV cache: k, v dense [B,Hkv,capacity,D], or with block_table int32 [B,n] pools
    [n_blocks,block_size,Hkv,D].  Their element type is the format: float32, bfloat16, float16 (no parameters), or
    float8_e4m3fn, int8 and uint8 (4-bit pairs, D / 2 bytes a row) with k_param, v_param: float32, one number a row
    ([B,Hkv,capacity] or [n_blocks,block_size,Hkv]; 4 bits: two, [..,2]).
    S: valid tokens of every sequence; with lengths, int32 [B] on the GPU, their upper bound.
    The tensors are kept alive by the result; `cache.S` may be assigned as the cache grows."""
    for name, t in (("k", k), ("v", v)):
        _dev(t, name)
    if k.dim() != 4 or v.shape != k.shape or v.dtype != k.dtype or k.dtype not in _FORMATS:
        raise ValueError("k and v must be 4-dimensional tensors of one shape and one of the cache's element types")
    fmt = _FORMATS[k.dtype]
    D = k.shape[3] * (2 if fmt == I4 else 1)
    rows = tuple(k.shape[:3])
    if fmt in (E4M3, I8, I4):
        for name, t in (("k_param", k_param), ("v_param", v_param)):
            if t is None or t.dtype != torch.float32 or tuple(_dev(t, name).shape) != (rows + (2,) if fmt == I4 else rows):
                raise ValueError(f"{name} must be float32 {list(rows + (2,) if fmt == I4 else rows)}")
    elif k_param is not None or v_param is not None:
        raise ValueError("only quantised caches have parameters")
    if block_table is None:
        B, Hkv, capacity, block_size, n_blocks = *rows, 0, 0
    else:
        n_blocks, block_size, Hkv = rows
        if block_table.dtype != torch.int32 or _dev(block_table, "block_table").dim() != 2:
            raise ValueError("block_table must be int32 [B,n]")
        B, capacity = block_table.shape[0], block_table.shape[1] * block_size
    if lengths is not None and (lengths.dtype != torch.int32 or tuple(_dev(lengths, "lengths").shape) != (B,)):
        raise ValueError("lengths must be int32 [B]")
    tensors = (k, v, k_param, v_param, lengths, block_table)
    if any(t is not None and t.device != k.device for t in tensors):
        raise ValueError("the cache's tensors must live on one device")
    if any(t is not None and t.requires_grad for t in tensors):
        raise ValueError("the cache's tensors must not require gradients: the calls on it have none")
    for name, t in zip(("k", "v", "k_param", "v_param"), tensors):
        if t is not None:
            _untracked(t, name)
    cache = Cache(B, Hkv, int(S), D, capacity, fmt, block_size, n_blocks, *(None if t is None else t.data_ptr() for t in tensors))
    cache.tensors, cache.device, cache.index = tensors, k.device, k.get_device()
    cache.value_dtype = torch.bfloat16 if k.dtype in CODES.values() else k.dtype
    cache.per_sequence, cache.values = (B,), (k_param, v_param) if fmt in (E4M3, I8, I4) else (k, v)
    return cache


def _untracked(t, name: str):
    """Autograd does not follow t, in neither direction: the calls on a cache would cut it off without a word."""
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name} requires a gradient, and the calls on a cache have none: use torch.no_grad() or detach()")
    if forward_ad._current_level >= 0 and forward_ad.unpack_dual(t).tangent is not None:
        raise ValueError(f"{name} has a forward-mode tangent, and the calls on a cache carry none on: use its primal part")


def _untracked_cache(cache):
    """Its tensors may have come to be followed since make_cache, by what was copied into them."""
    a, b = cache.values  # (set by make_cache)
    if a.requires_grad or b.requires_grad or forward_ad._current_level >= 0:
        for t in (a, b):
            if t.grad_fn is not None or not t.requires_grad:
                _untracked(t, "the cache")


def _here(t, name: str, index: int):
    if t.get_device() != index:
        raise ValueError(f"{name} must live on the cache's device" if t.is_cuda else f"{name} must live in GPU memory")


def _packed(t, name: str, index: int, dtype, shape):
    """A contiguous tensor on the cache's device, of this type and shape."""
    _here(t, name, index)
    if t.dtype != dtype or t.shape != shape:
        raise ValueError(f"{name} must be {dtype} {list(shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.requires_grad or forward_ad._current_level >= 0:
        _untracked(t, name)
    return t.data_ptr()


def _scratch(t, index: int):
    _here(t, "workspace", index)
    if not t.is_contiguous():   # (its nbytes are what the library may write from its first one on)
        raise ValueError("workspace must be contiguous")


def _rows(t, name: str, index: int):
    """[B,H,T,D] on the cache's device with the D values contiguous (any other strides)."""
    _here(t, name, index)
    if t.dim() != 4 or (t.shape[3] > 1 and t.stride(3) != 1):
        raise ValueError(f"{name} must be [B,H,T,D] with the D values contiguous")
    if t.requires_grad or forward_ad._current_level >= 0:
        _untracked(t, name)


def _strides(t):
    """Element strides of [B,H,T,D] (sequence, head, token), None if packed; an axis of one element has any stride, so its
    packed one is given.  Three zeros are the library's sign for packed: refused."""
    if t.is_contiguous():
        return None
    B, H, T, D = t.shape
    st = t.stride()
    st = st[0] if B > 1 else H * T * D, st[1] if H > 1 else T * D, st[2] if T > 1 else D
    if st == (0, 0, 0):
        raise ValueError("one row expanded to all sequences, heads and tokens: pass its contiguous() copy")
    return st


def _stride_array(t):
    st = _strides(t)
    return None if st is None else (ctypes.c_int64 * 3)(*st)


def _counts(n_new, cache):
    return None if n_new is None else _packed(n_new, "n_new", cache.index, torch.int32, cache.per_sequence)


# The small calls' kernels take a few us, about as long as Python takes for a dozen attribute reads and calls: what a call
# needs is read once, and the current device changes only where it has to.
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


class _Device:
    """The cache's device as the current one, if it is not."""

    def __init__(self, index):
        self.index, self.back = index, _current_device()

    def __enter__(self):
        if self.back != self.index:
            torch.cuda.set_device(self.index)

    def __exit__(self, *_):
        if self.back != self.index:
            torch.cuda.set_device(self.back)


def _stream_of(cache, stream):
    return _current_raw_stream(cache.index) if stream is None else stream.cuda_stream


def kvcrush_cache_write(cache: Cache, k_new, v_new, n_new=None, stream=None):
    """k_new, v_new [B,Hkv,T,D] (any strides but three zeros, D contiguous) become the last T tokens of their sequences: the cache's
    lengths count them already.  n_new int32 [B]: only the first n_new[b] of sequence b's are real.  Quantised caches
    take float32, bfloat16 and float16, the others their own type."""
    index, shape = cache.index, k_new.shape
    _rows(k_new, "k_new", index), _rows(v_new, "v_new", index)
    _untracked_cache(cache)
    if v_new.shape != shape or v_new.dtype != k_new.dtype or shape[0] != cache.B or shape[1] != cache.Hkv or shape[3] != cache.D:
        raise ValueError("k_new and v_new must be [B,Hkv,T,D] tensors of one type that fit the cache")
    with _Device(index):
        st = load().kvcrush_cache_write(cache, shape[2], _dtype_code(k_new), k_new.data_ptr(), v_new.data_ptr(),
                                        _stride_array(k_new), _stride_array(v_new), _counts(n_new, cache),
                                        _stream_of(cache, stream))
    _check(st, "kvcrush_cache_write")


def kvcrush_cache_read(cache: Cache, idx=None, n=None, dtype=None, k_out=None, v_out=None, stream=None):
    """The cache's rows as values: of the positions idx int32 [B,n], or of the first n (default: cache.S) tokens.
    -> (k, v) [B,Hkv,n,D] of `dtype` (default: k_out's; the cache's own type; bfloat16 of quantised ones).  Rows that a
    sequence does not have stay as they are in k_out and v_out; in tensors made here they are zero."""
    index, at = cache.index, None
    if idx is not None:
        n = idx.shape[-1]
        at = _packed(idx, "idx", index, torch.int32, (cache.B, n))
    elif n is None:
        n = cache.S
    _untracked_cache(cache)
    shape = (cache.B, cache.Hkv, n, cache.D)
    if dtype is None:
        dtype = k_out.dtype if k_out is not None else v_out.dtype if v_out is not None else cache.value_dtype
    made_k = made_v = None
    if k_out is None or v_out is None:
        # (some rows may stay unwritten: those of sequences shorter than n, of empty ones)
        new = torch.zeros if cache.lengths or (cache.S < n if idx is None else cache.S == 0) else torch.empty
        with _memory_of(stream):
            if k_out is None:
                k_out = made_k = new(shape, dtype=dtype, device=cache.device)
            if v_out is None:
                v_out = made_v = new(shape, dtype=dtype, device=cache.device)
    k_at, v_at = _packed(k_out, "k_out", index, dtype, shape), _packed(v_out, "v_out", index, dtype, shape)
    with _Device(index):
        st = load().kvcrush_cache_read(cache, n, at, _dtype_code(k_out), k_at, v_at, _stream_of(cache, stream))
    _hand_over(stream, made_k, made_v)
    _check(st, "kvcrush_cache_read")
    return k_out, v_out


def kvcrush_attend_workspace(cache: Cache, Hq: int, T: int, dtype, n_list=0, unit=0) -> int:
    """Bytes of scratch memory that kvcrush_attend needs for queries [B,Hq,T,D] of `dtype` (with lists: of n_list blocks
    of `unit` tokens) on this cache, its S and capacity being what they are now; a larger S needs no less."""
    args = AttendArgs(Hq, T, _FORMATS[dtype], blocks=16 if n_list else None, n_list=n_list, unit=unit)
    return int(load().kvcrush_attend_workspace(cache, args))


def _queries(cache, q):
    _rows(q, "q", cache.index)
    _untracked_cache(cache)
    B, Hq, T, D = q.shape
    dtype = q.dtype
    if B != cache.B or D != cache.D or dtype not in _VALUES:
        raise ValueError("q must be a float32, bfloat16 or float16 [B,Hq,T,D] that fits the cache")
    args = AttendArgs(Hq, T, _FORMATS[dtype])
    st = _strides(q)
    if st is not None:
        args.q_stride = st
    return args


def kvcrush_attend(cache: Cache, q, mask=None, n_new=None, blocks=None, unit=0, scale=0.0, out=None, lse=None, workspace=None,
                   stream=None):
    """The newest T tokens, whose rows are in the cache, attend to it: q [B,Hq,T,D] (any strides but three zeros, D contiguous) ->
    (out like q, lse float32 [B,Hq,T], the rows' natural log-sum-exps).
    mask: int64 words [B,T,ceil(T/64)], or [T,ceil(T/64)] for all sequences: bit j % 64 of word j / 64 of row t lets new
    token t see new token j; without it, those up to itself.  All tokens before the new ones are seen.
    n_new int32 [B]: only the first n_new[b] of the T tokens are real.
    blocks int32 [B,Hkv,T,n] (kvcrush_block_select): query t sees only these blocks of `unit` tokens."""
    args, index, shape = _queries(cache, q), cache.index, q.shape
    B, Hq, T, _ = shape
    args.softmax_scale = scale
    if mask is not None:
        words = (T + 63) // 64
        args.mask = _packed(mask, "mask", index, torch.int64, (B, T, words) if mask.dim() == 3 else (T, words))
        args.mask_stride = T * words if mask.dim() == 3 else 0
    if blocks is not None:
        if blocks.shape[-1] < 1:   # (no entries have no address, which is the library's sign for all tokens)
            raise ValueError("blocks must have one entry a list at least")
        args.blocks = _packed(blocks, "blocks", index, torch.int32, (B, cache.Hkv, T, blocks.shape[-1]))
        args.n_list, args.unit = blocks.shape[-1], unit
    if n_new is not None:
        args.n_new = _counts(n_new, cache)
    made_out = made_lse = None
    if out is not None:
        _rows(out, "out", index)
        if out.shape != shape or out.dtype != q.dtype:
            raise ValueError("out must have q's shape and type")
        st = _strides(out)
        if st is not None:
            args.out_stride = st
    if lse is not None:
        _packed(lse, "lse", index, torch.float32, shape[:3])
    if workspace is not None:
        _scratch(workspace, index)
    L = load()
    with _memory_of(stream):
        if out is None:
            out = made_out = torch.empty(shape, dtype=q.dtype, device=cache.device)
        if lse is None:
            lse = made_lse = torch.empty(shape[:3], dtype=torch.float32, device=cache.device)
        if workspace is None:
            workspace = torch.empty(max(L.kvcrush_attend_workspace(cache, args), 16), dtype=torch.uint8, device=cache.device)
    with _Device(index):
        st = L.kvcrush_attend(cache, args, q.data_ptr(), out.data_ptr(), lse.data_ptr(), workspace.data_ptr(), workspace.nbytes,
                              _stream_of(cache, stream))
    _hand_over(stream, made_out, made_lse)
    _check(st, "kvcrush_attend")
    return out, lse


def _block_shapes(cache, unit):
    if unit < 1:
        raise ValueError("unit must be positive")
    nb = (cache.capacity + unit - 1) // unit
    return (cache.B, cache.Hkv, nb, 2, cache.D), (cache.B, cache.Hkv, nb)


def kvcrush_block_bounds(cache: Cache, unit: int, bounds=None, scales=None, T=0, n_new=None, stream=None):
    """8-bit bounds of the keys of every block of `unit` tokens: (bounds int8 [B,Hkv,Nb,2,D], scales float32 [B,Hkv,Nb]),
    Nb = ceil(capacity / unit).  T > 0 refreshes, in bounds and scales given, the blocks of the last T tokens (of the
    n_new[b] real ones) only."""
    index = cache.index
    of_bounds, of_scales = _block_shapes(cache, unit)
    if (bounds is None) != (scales is None) or (bounds is None and T):
        raise ValueError("bounds and scales come together, and are needed to refresh blocks of them")
    _untracked_cache(cache)
    made = (None, None)
    if bounds is None:
        with _memory_of(stream):
            made = bounds, scales = (torch.zeros(of_bounds, dtype=torch.int8, device=cache.device),
                                     torch.zeros(of_scales, dtype=torch.float32, device=cache.device))
    bounds_at = _packed(bounds, "bounds", index, torch.int8, of_bounds)
    scales_at = _packed(scales, "scales", index, torch.float32, of_scales)
    with _Device(index):
        st = load().kvcrush_block_bounds(cache, unit, T, _counts(n_new, cache), bounds_at, scales_at, _stream_of(cache, stream))
    _hand_over(stream, *made)
    _check(st, "kvcrush_block_bounds")
    return bounds, scales


def kvcrush_block_select_workspace(cache: Cache, Hq: int, T: int, dtype, unit: int, n_select: int) -> int:
    return int(load().kvcrush_block_select_workspace(cache, AttendArgs(Hq, T, _FORMATS[dtype]), unit, n_select))


def kvcrush_block_select(cache: Cache, q, bounds, scales, unit: int, n_select: int, n_sink=1, n_recent=1, n_new=None, blocks=None,
                         workspace=None, stream=None):
    """For each query of q [B,Hq,T,D] and each KV head the n_select blocks to attend to: int32 [B,Hkv,T,n_select],
    ascending, -1 behind the last.  The first n_sink and last n_recent blocks of the sequence are among them, the others
    are those of the largest scores by kvcrush_block_bounds' bounds and scales."""
    args, index = _queries(cache, q), cache.index
    of_bounds, of_scales = _block_shapes(cache, unit)
    bounds_at = _packed(bounds, "bounds", index, torch.int8, of_bounds)
    scales_at = _packed(scales, "scales", index, torch.float32, of_scales)
    if n_new is not None:
        args.n_new = _counts(n_new, cache)
    L, made = load(), None
    shape = (cache.B, cache.Hkv, q.shape[2], n_select)
    if blocks is not None:
        _packed(blocks, "blocks", index, torch.int32, shape)
    if workspace is not None:
        _scratch(workspace, index)
    with _memory_of(stream):
        if blocks is None:
            blocks = made = torch.empty(shape if n_select > 0 else 0, dtype=torch.int32, device=cache.device)
        if workspace is None:
            need = L.kvcrush_block_select_workspace(cache, args, unit, n_select)
            workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=cache.device)
    with _Device(index):
        st = L.kvcrush_block_select(cache, args, unit, n_select, n_sink, n_recent, q.data_ptr(), bounds_at, scales_at,
                                    blocks.data_ptr(), workspace.data_ptr(), workspace.nbytes, _stream_of(cache, stream))
    _hand_over(stream, made)
    _check(st, "kvcrush_block_select")
    return blocks


def kvcrush_version() -> int:
    return int(load().kvcrush_version())
