"""Forcing-KV hot path on AMD MI355X: Python binding of libfkv.

Thin ctypes layer over the C ABI declared in ``include/fkv.h``; every
function has the C entry point's name and only marshals arguments (torch
tensors supply device memory, ``torch.cuda.current_stream()`` the stream).
All compute runs in the HIP kernels of ``libfkv.so``; there is no CPU
fallback.  If the library has not been built, calls raise
:class:`FkvLibraryMissing`.

Entry points (see ``include/fkv.h`` for the full contract):

* :func:`fkv_compress_static`  -- static structural pruning (Sec. 4.2, Eq. 2)
* :func:`fkv_score_segments`   -- segment similarity (Sec. 4.3, Eq. 3)
* :func:`fkv_select_compact`   -- BottomK + compaction (Sec. 4.3, Eq. 3)
* :func:`fkv_chunk_attention`  -- chunk attention (Eq. 2 / Eq. 4)
* :func:`fkv_chunk_attention_heads` -- the same for a subset of heads
* :func:`fkv_chunk_attention_static` -- the static heads' attention read in
  place from the cache (no compressed copy)
* :func:`fkv_append_frames`    -- rolling-cache write of a finished chunk
* :func:`fkv_fp8_pack`, :func:`fkv_fp8_pack_paged`, :func:`fkv_chunk_attention_fp8`
  -- the FP8 variant of the chunk attention (App. F)
* :func:`fkv_attention_mass`, :func:`fkv_classify_heads` -- offline head
  profiling (Sec. 4.1, Eq. 1)
* :func:`fkv_rotate_chunk`, :func:`fkv_append_frames_rotated` -- position
  rotation of a chunk's queries and keys, and the cache write with it
* :func:`fkv_append_frames_q8`, :func:`fkv_score_select_q8`,
  :func:`fkv_chunk_attention_q8` -- a rolling cache held in 8 bits
  (:class:`Cache8`): its write, its scoring and selection, and attention of any
  number of query tokens over it
* :func:`fkv_append_paged`, :func:`fkv_paged_attention` -- the paged cache of many
  sequences (:class:`PagedBatch`): its write, and attention of every sequence's
  new tokens over its pages
* :func:`fkv_latent_attention` -- the same over a paged cache of latent rows
* :func:`fkv_score_pooled`, :func:`fkv_select_compact_pooled` -- the
  first-block proxy of Sec. 4.3: one similarity row pooled over all heads,
  shared by the dynamic heads of every layer
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfkv.so")

FKV_OK, FKV_ERR_ARG, FKV_ERR_SHAPE, FKV_ERR_CAPACITY, FKV_ERR_DEVICE = range(5)
FKV_BF16, FKV_F32 = 0, 1
FKV_STATIC, FKV_DYNAMIC = 0, 1
FKV_SCOPE_FRAME, FKV_SCOPE_GLOBAL = 0, 1
FKV_PAIR_ADJACENT, FKV_PAIR_HALVES = 0, 1
FKV_MAX_HEADS, FKV_MAX_FRAMES, FKV_MAX_SEGMENTS = 64, 256, 4096
FKV_MAX_POSITION = 1 << 24
FKV_LATENT_AUTO, FKV_LATENT_ABSORBED, FKV_LATENT_EXPANDED = 0, 1, 2
FKV_LATENT_ROT, FKV_LATENT_FEW, FKV_MAX_SEQS = 64, 64, 1024

EXPORTED = ("fkv_num_segments", "fkv_kept_tokens_max", "fkv_compress_static",
            "fkv_score_workspace_size", "fkv_score_segments", "fkv_select_compact",
            "fkv_append_frames", "fkv_score_pooled_workspace_size", "fkv_score_pooled",
            "fkv_select_compact_pooled", "fkv_select", "fkv_score_select", "fkv_score_select_noalloc",
            "fkv_score_stats_size", "fkv_score_history",
            "fkv_score_segments_cached",
            "fkv_attention_workspace_size", "fkv_chunk_attention", "fkv_chunk_attention_heads",
            "fkv_chunk_attention_static", "fkv_chunk_attention_paged",
            "fkv_fp8_sizes", "fkv_fp8_pack", "fkv_fp8_pack_paged",
            "fkv_chunk_attention_fp8", "fkv_attention_mass_workspace_size", "fkv_attention_mass",
            "fkv_classify_heads", "fkv_rotate_chunk", "fkv_append_frames_rotated", "fkv_append_frames_q8",
            "fkv_score_select_q8", "fkv_chunk_attention_q8_workspace_size", "fkv_chunk_attention_q8",
            "fkv_append_paged", "fkv_paged_attention_workspace_size", "fkv_paged_attention",
            "fkv_latent_attention_workspace_size", "fkv_latent_attention", "fkv_last_error")


class FkvLibraryMissing(RuntimeError):
    pass


class FkvError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"fkv status {status}: {message}")
        self.status = status
        self.message = message


class fkv_shape(ctypes.Structure):
    _fields_ = [("n_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("frame_tokens", ctypes.c_int32), ("hist_frames", ctypes.c_int32),
                ("cap_frames", ctypes.c_int32), ("chunk_frames", ctypes.c_int32),
                ("seg_tokens", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class fkv_head(ctypes.Structure):
    _fields_ = [("type", ctypes.c_int32), ("sink_frames", ctypes.c_int32),
                ("recent_frames", ctypes.c_int32), ("keep_k", ctypes.c_int32),
                ("scope", ctypes.c_int32)]


class fkv_rope(ctypes.Structure):
    _fields_ = [("frame_pairs", ctypes.c_int32), ("row_pairs", ctypes.c_int32), ("col_pairs", ctypes.c_int32),
                ("row_tokens", ctypes.c_int32), ("token_step", ctypes.c_int32), ("pairing", ctypes.c_int32),
                ("theta", ctypes.c_double)]


class fkv_rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("head_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64)]


class fkv_cache8(ctypes.Structure):
    _fields_ = [("K8", ctypes.c_void_p), ("V8", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("block_tokens", ctypes.c_int32)]


class fkv_batch(ctypes.Structure):
    _fields_ = [("n_seqs", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("page_tokens", ctypes.c_int32),
                ("n_pages", ctypes.c_int32), ("n_tokens", ctypes.c_int32), ("max_new", ctypes.c_int32),
                ("sum_len", ctypes.c_int64), ("page_table", ctypes.c_void_p), ("seq_len", ctypes.c_void_p),
                ("q_start", ctypes.c_void_p)]


class fkv_span(ctypes.Structure):
    _fields_ = [("sink_tokens", ctypes.c_int32), ("recent_tokens", ctypes.c_int32)]


_lib = None


def lib():
    """Load libfkv.so (raises FkvLibraryMissing if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FkvLibraryMissing(
                f"{LIB_PATH} is missing: build it with `python -m paper_2605_09681_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        P, I32, I64, SZ, F = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float
        S, Hd = ctypes.POINTER(fkv_shape), ctypes.POINTER(fkv_head)
        L.fkv_num_segments.argtypes = [S]
        L.fkv_num_segments.restype = I32
        L.fkv_kept_tokens_max.argtypes = [S, Hd, I32, ctypes.POINTER(I64)]
        L.fkv_kept_tokens_max.restype = ctypes.c_int
        L.fkv_compress_static.argtypes = [S, Hd, P, P, P, P, P, I32, P, P]
        L.fkv_compress_static.restype = ctypes.c_int
        L.fkv_score_workspace_size.argtypes = [S, Hd, ctypes.POINTER(SZ)]
        L.fkv_score_workspace_size.restype = ctypes.c_int
        L.fkv_score_segments.argtypes = [S, Hd, P, P, P, P, P, SZ, P]
        L.fkv_score_segments.restype = ctypes.c_int
        L.fkv_select_compact.argtypes = [S, Hd, P, P, P, P, P, P, P, I32, P, P]
        L.fkv_select_compact.restype = ctypes.c_int
        L.fkv_append_frames.argtypes = [S, P, P, I32, P, P, P, P]
        L.fkv_append_frames.restype = ctypes.c_int
        L.fkv_score_pooled_workspace_size.argtypes = [S, ctypes.POINTER(SZ)]
        L.fkv_score_pooled_workspace_size.restype = ctypes.c_int
        L.fkv_score_pooled.argtypes = [S, P, P, P, P, P, SZ, P]
        L.fkv_score_pooled.restype = ctypes.c_int
        L.fkv_select_compact_pooled.argtypes = [S, Hd, P, P, P, P, P, P, P, I32, P, P]
        L.fkv_select_compact_pooled.restype = ctypes.c_int
        L.fkv_select.argtypes = [S, Hd, P, I32, P, P, P]
        L.fkv_select.restype = ctypes.c_int
        L.fkv_score_select.argtypes = [S, Hd, P, P, P, P, P, P, P, SZ, P]
        L.fkv_score_select.restype = ctypes.c_int
        L.fkv_score_select_noalloc.argtypes = [S, Hd, P, P, P, P, P, P, P]
        L.fkv_score_select_noalloc.restype = ctypes.c_int
        L.fkv_attention_workspace_size.argtypes = [S, ctypes.POINTER(SZ)]
        L.fkv_attention_workspace_size.restype = ctypes.c_int
        L.fkv_chunk_attention.argtypes = [S, P, P, P, I32, P, P, P, F, P, P, P, SZ, P]
        L.fkv_chunk_attention.restype = ctypes.c_int
        L.fkv_score_stats_size.argtypes = [S, Hd, I32, ctypes.POINTER(SZ)]
        L.fkv_score_stats_size.restype = ctypes.c_int
        L.fkv_score_history.argtypes = [S, Hd, I32, P, P, P, SZ, P, SZ, P]
        L.fkv_score_history.restype = ctypes.c_int
        L.fkv_score_segments_cached.argtypes = [S, Hd, I32, P, P, P, P, SZ, P, P, SZ, P]
        L.fkv_score_segments_cached.restype = ctypes.c_int
        L.fkv_chunk_attention_heads.argtypes = [S, P, I32, P, P, P, I32, P, P, P, F, P, P, P, SZ, P]
        L.fkv_chunk_attention_heads.restype = ctypes.c_int
        L.fkv_chunk_attention_static.argtypes = [S, Hd, P, P, P, P, P, P, F, P, P, P, SZ, P]
        L.fkv_chunk_attention_static.restype = ctypes.c_int
        L.fkv_chunk_attention_paged.argtypes = [S, Hd, P, I32, P, P, P, P, P, P, P, P, F, P, P, P, SZ, P]
        L.fkv_chunk_attention_paged.restype = ctypes.c_int
        L.fkv_fp8_sizes.argtypes = [S, I32] + [ctypes.POINTER(SZ)] * 4
        L.fkv_fp8_sizes.restype = ctypes.c_int
        L.fkv_fp8_pack.argtypes = [S, P, P, P, I32, P, P, P, P, P, P, P, P, SZ, P]
        L.fkv_fp8_pack.restype = ctypes.c_int
        L.fkv_fp8_pack_paged.argtypes = [S, Hd, P, P, ctypes.POINTER(I32), P, P, P, P, P, I32, P, P, P, P, P,
                                         SZ, P]
        L.fkv_fp8_pack_paged.restype = ctypes.c_int
        L.fkv_chunk_attention_fp8.argtypes = [S, P, P, P, I32, P, P, F, P, P, P, SZ, P]
        L.fkv_chunk_attention_fp8.restype = ctypes.c_int
        L.fkv_attention_mass_workspace_size.argtypes = [S, I32, ctypes.POINTER(SZ)]
        L.fkv_attention_mass_workspace_size.restype = ctypes.c_int
        L.fkv_attention_mass.argtypes = [S, P, P, I32, P, P, P, F, I32, P, I32, P, SZ, P]
        L.fkv_attention_mass.restype = ctypes.c_int
        L.fkv_classify_heads.argtypes = [P, I32, I32, I32, I32, I32, F, P]
        L.fkv_classify_heads.restype = ctypes.c_int
        Rp, Rw, C8 = ctypes.POINTER(fkv_rope), ctypes.POINTER(fkv_rows), ctypes.POINTER(fkv_cache8)
        L.fkv_rotate_chunk.argtypes = [S, Rp, P, Rw, Rw, Rw, P, P, P, P]
        L.fkv_rotate_chunk.restype = ctypes.c_int
        L.fkv_append_frames_rotated.argtypes = [S, Rp, P, Rw, Rw, I32, P, P, P, P]
        L.fkv_append_frames_rotated.restype = ctypes.c_int
        L.fkv_append_frames_q8.argtypes = [S, Rp, P, Rw, Rw, I32, P, C8, P]
        L.fkv_append_frames_q8.restype = ctypes.c_int
        L.fkv_score_select_q8.argtypes = [S, Hd, C8, P, P, P, P, P, P, SZ, P]
        L.fkv_score_select_q8.restype = ctypes.c_int
        L.fkv_chunk_attention_q8_workspace_size.argtypes = [S, Hd, I32, I32, ctypes.POINTER(SZ)]
        L.fkv_chunk_attention_q8_workspace_size.restype = ctypes.c_int
        L.fkv_chunk_attention_q8.argtypes = [S, Hd, C8, P, P, P, P, I32, P, P, I32, F, P, P, P, SZ, P]
        L.fkv_chunk_attention_q8.restype = ctypes.c_int
        B, Sp = ctypes.POINTER(fkv_batch), ctypes.POINTER(fkv_span)
        L.fkv_append_paged.argtypes = [B, I32, I32, I32, Rw, Rw, P, P, P]
        L.fkv_append_paged.restype = ctypes.c_int
        L.fkv_paged_attention_workspace_size.argtypes = [B, I32, I32, I32, ctypes.POINTER(SZ)]
        L.fkv_paged_attention_workspace_size.restype = ctypes.c_int
        L.fkv_paged_attention.argtypes = [B, I32, I32, I32, Rw, P, P, I32, Sp, F, Rw, P, P, SZ, P]
        L.fkv_paged_attention.restype = ctypes.c_int
        L.fkv_latent_attention_workspace_size.argtypes = [B, I32, I32, I32, I32, ctypes.POINTER(SZ)]
        L.fkv_latent_attention_workspace_size.restype = ctypes.c_int
        L.fkv_latent_attention.argtypes = [B, I32, I32, I32, Rw, P, P, P, I32, Sp, F, Rw, I32, P, SZ, P]
        L.fkv_latent_attention.restype = ctypes.c_int
        L.fkv_last_error.argtypes = []
        L.fkv_last_error.restype = ctypes.c_char_p
        _lib = L
    return _lib


# ---------------------------------------------------------------------------
# argument marshalling
# ---------------------------------------------------------------------------
def _i32(v, name: str) -> int:
    """v as a whole number of 32 bits (ctypes would cut others down to one)."""
    i = int(v)
    if i != v or not -1 << 31 <= i < 1 << 31:
        raise ValueError(f"{name}: {v} is not a whole number of 32 bits")
    return i


def make_shape(n_heads, head_dim, frame_tokens, hist_frames, cap_frames, chunk_frames,
               seg_tokens, dtype) -> fkv_shape:
    dt = {"bf16": FKV_BF16, "f32": FKV_F32, FKV_BF16: FKV_BF16, FKV_F32: FKV_F32}[dtype]
    sizes = (n_heads, head_dim, frame_tokens, hist_frames, cap_frames, chunk_frames, seg_tokens)
    return fkv_shape(*(_i32(v, "shape") for v in sizes), dt)


def make_heads(budgets: Sequence) -> ctypes.Array:
    """Per-head budgets: objects with type/sink_frames/recent_frames/keep_k/scope
    attributes, or 5-tuples in that order."""
    arr = (fkv_head * len(budgets))()
    for i, b in enumerate(budgets):
        vals = (b.type, b.sink_frames, b.recent_frames, b.keep_k, b.scope) if hasattr(b, "type") else tuple(b)
        arr[i] = fkv_head(*(_i32(v, f"budget of head {i}") for v in vals))
    return arr


def _torch_dtype(shape: fkv_shape):
    return torch.bfloat16 if shape.dtype == FKV_BF16 else torch.float32


def _check(t: torch.Tensor, name: str, dtype, size=None):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.device.type != "cuda":
        raise ValueError(f"{name} must be a GPU tensor (got {t.device})")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype} (got {t.dtype})")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if size is not None and tuple(t.shape) != tuple(size):
        raise ValueError(f"{name} must have shape {tuple(size)} (got {tuple(t.shape)})")
    return ctypes.c_void_p(t.data_ptr())


def _slots(frame_slot, H):
    if frame_slot is None:
        import numpy as np
        frame_slot = np.arange(H, dtype="int32")
    return _ints(frame_slot, H, "frame_slot")


def _heads(shape: fkv_shape, heads, allow_none: bool = False):
    """The host fkv_head array of a call: the C entry points read exactly
    shape.n_heads entries, so a shorter or longer array is rejected here."""
    if heads is None:
        if allow_none:
            return None
        raise ValueError("heads is None")
    if not isinstance(heads, ctypes.Array) or heads._type_ is not fkv_head:
        raise TypeError("heads must be an fkv_head array (see make_heads)")
    if len(heads) != shape.n_heads:
        raise ValueError(f"heads has {len(heads)} entries, the shape has {shape.n_heads} heads")
    return heads


def _stream(stream) -> ctypes.c_void_p:
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _raise(status: int):
    if status != FKV_OK:
        raise FkvError(status, lib().fkv_last_error().decode())


def _lq(shape):
    return shape.chunk_frames * shape.frame_tokens


# ---------------------------------------------------------------------------
# entry points
# ---------------------------------------------------------------------------
def fkv_num_segments(shape: fkv_shape) -> int:
    return int(lib().fkv_num_segments(ctypes.byref(shape)))


def fkv_kept_tokens_max(shape: fkv_shape, heads, head: int) -> int:
    out = ctypes.c_int64(0)
    _raise(lib().fkv_kept_tokens_max(ctypes.byref(shape), _heads(shape, heads), _i32(head, "head"), ctypes.byref(out)))
    return int(out.value)


def slab_tokens(shape: fkv_shape, heads) -> int:
    """Smallest slab (tokens per head of Kc/Vc) that fits every head's budget."""
    return max([fkv_kept_tokens_max(shape, heads, h) for h in range(shape.n_heads)] + [0])


def fkv_score_workspace_size(shape: fkv_shape, heads) -> int:
    out = ctypes.c_size_t(0)
    _raise(lib().fkv_score_workspace_size(ctypes.byref(shape), _heads(shape, heads), ctypes.byref(out)))
    return int(out.value)


def fkv_compress_static(shape: fkv_shape, heads, K_hist, V_hist, frame_slot, Kc, Vc, kv_len,
                        stream=None):
    dt = _torch_dtype(shape)
    hist = (shape.n_heads, shape.cap_frames, shape.frame_tokens, shape.head_dim)
    slab = Kc.shape[1] if Kc.dim() == 3 else -1
    comp = (shape.n_heads, slab, shape.head_dim)
    args = [_check(K_hist, "K_hist", dt, hist), _check(V_hist, "V_hist", dt, hist)]
    sl = _slots(frame_slot, shape.hist_frames)
    args += [_check(Kc, "Kc", dt, comp), _check(Vc, "Vc", dt, comp)]
    kl = _check(kv_len, "kv_len", torch.int32, (shape.n_heads,))
    _raise(lib().fkv_compress_static(ctypes.byref(shape), _heads(shape, heads), args[0], args[1], sl, args[2],
                                     args[3], int(slab), kl, _stream(stream)))


def fkv_score_segments(shape: fkv_shape, heads, K_hist, frame_slot, K_cur, scores,
                       workspace: Optional[torch.Tensor] = None, stream=None):
    """If ``workspace`` is None a torch uint8 tensor of the required size is
    allocated on the current device (through torch's caching allocator)."""
    dt = _torch_dtype(shape)
    hist = (shape.n_heads, shape.cap_frames, shape.frame_tokens, shape.head_dim)
    n_seg = fkv_num_segments(shape)
    kh = _check(K_hist, "K_hist", dt, hist)
    sl = _slots(frame_slot, shape.hist_frames)
    kc = _check(K_cur, "K_cur", dt, (shape.n_heads, _lq(shape), shape.head_dim))
    sc = _check(scores, "scores", torch.float32, (shape.n_heads, n_seg))
    need = fkv_score_workspace_size(shape, heads)
    if workspace is None:   # zero-filled: the scoring workspace starts with arrival counters
        workspace = torch.zeros(max(need, 1), dtype=torch.uint8, device=K_hist.device)
    ws = _check(workspace, "workspace", torch.uint8)
    _raise(lib().fkv_score_segments(ctypes.byref(shape), _heads(shape, heads), kh, sl, kc, sc, ws,
                                    workspace.numel(), _stream(stream)))
    return workspace


def fkv_score_stats_size(shape: fkv_shape, heads, pooled: bool = False) -> int:
    """Bytes of the per-frame statistics buffer of incremental rescoring."""
    out = ctypes.c_size_t(0)
    _raise(lib().fkv_score_stats_size(ctypes.byref(shape), _heads(shape, heads, allow_none=bool(pooled)), int(pooled), ctypes.byref(out)))
    return int(out.value)


def fkv_score_history(shape: fkv_shape, heads, K_hist, frame_slot, stats, workspace, pooled: bool = False,
                      stream=None):
    """Per-frame statistics of the history into ``stats`` (float64 device
    tensor of fkv_score_stats_size bytes), once per chunk."""
    dt = _torch_dtype(shape)
    hist = (shape.n_heads, shape.cap_frames, shape.frame_tokens, shape.head_dim)
    kh = _check(K_hist, "K_hist", dt, hist)
    st = _check(stats, "stats", torch.float64)
    ws = _check(workspace, "workspace", torch.uint8)
    _raise(lib().fkv_score_history(ctypes.byref(shape), _heads(shape, heads, allow_none=bool(pooled)), int(pooled), kh, _slots(frame_slot, shape.hist_frames),
                                   st, stats.numel() * 8, ws, workspace.numel(), _stream(stream)))


def fkv_score_segments_cached(shape: fkv_shape, heads, K_hist, frame_slot, K_cur, stats, scores, workspace,
                              pooled: bool = False, stream=None):
    """Scores of one AR step from the history statistics plus the pair
    (frame H-1, first frame of K_cur): the result of fkv_score_segments
    (or fkv_score_pooled when pooled) with two frames read per head."""
    dt = _torch_dtype(shape)
    hist = (shape.n_heads, shape.cap_frames, shape.frame_tokens, shape.head_dim)
    n_seg = fkv_num_segments(shape)
    kh = _check(K_hist, "K_hist", dt, hist)
    kc = _check(K_cur, "K_cur", dt, (shape.n_heads, _lq(shape), shape.head_dim))
    sc = _check(scores, "scores", torch.float32, (n_seg,) if pooled else (shape.n_heads, n_seg))
    st = _check(stats, "stats", torch.float64)
    ws = _check(workspace, "workspace", torch.uint8)
    _raise(lib().fkv_score_segments_cached(ctypes.byref(shape), _heads(shape, heads, allow_none=bool(pooled)), int(pooled), kh,
                                           _slots(frame_slot, shape.hist_frames), kc, st, stats.numel() * 8, sc,
                                           ws, workspace.numel(), _stream(stream)))


def fkv_append_frames(shape: fkv_shape, K_new, V_new, dst_slot, K_hist, V_hist, stream=None):
    """Writes the frames of K_new / V_new ([n_heads][n*F][d]) into the cache
    slots dst_slot (host ints, one per frame)."""
    dt = _torch_dtype(shape)
    hist = (shape.n_heads, shape.cap_frames, shape.frame_tokens, shape.head_dim)
    dst_slot = list(dst_slot)
    n = len(dst_slot)
    slots = _ints(dst_slot, n, "dst_slot")
    new = (shape.n_heads, n * shape.frame_tokens, shape.head_dim)
    kn, vn = _check(K_new, "K_new", dt, new), _check(V_new, "V_new", dt, new)
    kh, vh = _check(K_hist, "K_hist", dt, hist), _check(V_hist, "V_hist", dt, hist)
    _raise(lib().fkv_append_frames(ctypes.byref(shape), kn, vn, n, slots, kh, vh, _stream(stream)))


def fkv_score_pooled_workspace_size(shape: fkv_shape) -> int:
    out = ctypes.c_size_t(0)
    _raise(lib().fkv_score_pooled_workspace_size(ctypes.byref(shape), ctypes.byref(out)))
    return int(out.value)


def fkv_score_pooled(shape: fkv_shape, K_hist, frame_slot, K_cur, scores,
                     workspace: Optional[torch.Tensor] = None, stream=None):
    """One similarity row [n_seg] pooled over all heads (the first-block proxy).
    If ``workspace`` is None a torch uint8 tensor of the required size is
    allocated on the current device."""
    dt = _torch_dtype(shape)
    hist = (shape.n_heads, shape.cap_frames, shape.frame_tokens, shape.head_dim)
    n_seg = fkv_num_segments(shape)
    kh = _check(K_hist, "K_hist", dt, hist)
    sl = _slots(frame_slot, shape.hist_frames)
    kc = _check(K_cur, "K_cur", dt, (shape.n_heads, _lq(shape), shape.head_dim))
    sc = _check(scores, "scores", torch.float32, (n_seg,))
    need = fkv_score_pooled_workspace_size(shape)
    if workspace is None:   # zero-filled: the scoring workspace starts with arrival counters
        workspace = torch.zeros(max(need, 1), dtype=torch.uint8, device=K_hist.device)
    ws = _check(workspace, "workspace", torch.uint8)
    _raise(lib().fkv_score_pooled(ctypes.byref(shape), kh, sl, kc, sc, ws, workspace.numel(),
                                  _stream(stream)))
    return workspace


def fkv_select_compact_pooled(shape: fkv_shape, heads, scores, K_hist, V_hist, frame_slot,
                              kept_seg, Kc, Vc, kv_len, stream=None):
    """fkv_select_compact with one shared score row [n_seg]."""
    _select_compact(shape, heads, scores, K_hist, V_hist, frame_slot, kept_seg, Kc, Vc, kv_len,
                    stream, pooled=True)


def fkv_select(shape: fkv_shape, heads, scores, kept_seg, kv_len, shared_row: bool = False, stream=None):
    """BottomK only: kept_seg and kv_len of the dynamic heads, no copy.
    scores is [n_heads][n_seg], or [n_seg] with shared_row (the pooled proxy)."""
    n_seg = fkv_num_segments(shape)
    sc = _check(scores, "scores", torch.float32, (n_seg,) if shared_row else (shape.n_heads, n_seg))
    ks = _check(kept_seg, "kept_seg", torch.int32, (shape.n_heads, n_seg))
    kl = _check(kv_len, "kv_len", torch.int32, (shape.n_heads,))
    _raise(lib().fkv_select(ctypes.byref(shape), _heads(shape, heads), sc, int(bool(shared_row)), ks, kl,
                            _stream(stream)))


def fkv_score_select(shape: fkv_shape, heads, K_hist, frame_slot, K_cur, scores, kept_seg, kv_len,
                     workspace: Optional[torch.Tensor] = None, stream=None):
    """fkv_score_segments + fkv_select in one launch.  If ``workspace`` is None
    a zero-filled one is allocated (through torch's caching allocator)."""
    dt = _torch_dtype(shape)
    hist = (shape.n_heads, shape.cap_frames, shape.frame_tokens, shape.head_dim)
    n_seg = fkv_num_segments(shape)
    kh = _check(K_hist, "K_hist", dt, hist)
    sl = _slots(frame_slot, shape.hist_frames)
    kc = _check(K_cur, "K_cur", dt, (shape.n_heads, _lq(shape), shape.head_dim))
    sc = _check(scores, "scores", torch.float32, (shape.n_heads, n_seg))
    ks = _check(kept_seg, "kept_seg", torch.int32, (shape.n_heads, n_seg))
    kl = _check(kv_len, "kv_len", torch.int32, (shape.n_heads,))
    need = fkv_score_workspace_size(shape, heads)
    if workspace is None:
        workspace = torch.zeros(max(need, 1), dtype=torch.uint8, device=K_hist.device)
    ws = _check(workspace, "workspace", torch.uint8)
    _raise(lib().fkv_score_select(ctypes.byref(shape), _heads(shape, heads), kh, sl, kc, sc, ks, kl, ws,
                                  workspace.numel(), _stream(stream)))
    return workspace


def fkv_score_select_noalloc(shape: fkv_shape, heads, K_hist, frame_slot, K_cur, scores, kept_seg, kv_len,
                             stream=None):
    """fkv_score_select with the library's own per-GPU scratch as workspace:
    nothing is allocated.  Calls that overlap on one GPU race."""
    dt = _torch_dtype(shape)
    hist = (shape.n_heads, shape.cap_frames, shape.frame_tokens, shape.head_dim)
    n_seg = fkv_num_segments(shape)
    kh = _check(K_hist, "K_hist", dt, hist)
    sl = _slots(frame_slot, shape.hist_frames)
    kc = _check(K_cur, "K_cur", dt, (shape.n_heads, _lq(shape), shape.head_dim))
    sc = _check(scores, "scores", torch.float32, (shape.n_heads, n_seg))
    ks = _check(kept_seg, "kept_seg", torch.int32, (shape.n_heads, n_seg))
    kl = _check(kv_len, "kv_len", torch.int32, (shape.n_heads,))
    _raise(lib().fkv_score_select_noalloc(ctypes.byref(shape), _heads(shape, heads), kh, sl, kc, sc, ks, kl,
                                          _stream(stream)))


def fkv_select_compact(shape: fkv_shape, heads, scores, K_hist, V_hist, frame_slot, kept_seg,
                       Kc, Vc, kv_len, stream=None):
    _select_compact(shape, heads, scores, K_hist, V_hist, frame_slot, kept_seg, Kc, Vc, kv_len,
                    stream, pooled=False)


def _select_compact(shape, heads, scores, K_hist, V_hist, frame_slot, kept_seg, Kc, Vc, kv_len,
                    stream, pooled):
    dt = _torch_dtype(shape)
    hist = (shape.n_heads, shape.cap_frames, shape.frame_tokens, shape.head_dim)
    n_seg = fkv_num_segments(shape)
    sc = _check(scores, "scores", torch.float32, (n_seg,) if pooled else (shape.n_heads, n_seg))
    kh, vh = _check(K_hist, "K_hist", dt, hist), _check(V_hist, "V_hist", dt, hist)
    sl = _slots(frame_slot, shape.hist_frames)
    ks = _check(kept_seg, "kept_seg", torch.int32, (shape.n_heads, n_seg))
    slab = Kc.shape[1] if Kc.dim() == 3 else -1
    comp = (shape.n_heads, slab, shape.head_dim)
    kc, vc = _check(Kc, "Kc", dt, comp), _check(Vc, "Vc", dt, comp)
    kl = _check(kv_len, "kv_len", torch.int32, (shape.n_heads,))
    fn = lib().fkv_select_compact_pooled if pooled else lib().fkv_select_compact
    _raise(fn(ctypes.byref(shape), _heads(shape, heads), sc, kh, vh, sl, ks, kc, vc, int(slab), kl, _stream(stream)))


def fkv_attention_workspace_size(shape: fkv_shape) -> int:
    """Bytes of the balanced-schedule workspace on the current device."""
    out = ctypes.c_size_t(0)
    _raise(lib().fkv_attention_workspace_size(ctypes.byref(shape), ctypes.byref(out)))
    return int(out.value)


def _attention_args(shape: fkv_shape, Q, Kc, Vc, kv_len, K_cur, V_cur, O, lse, workspace):
    dt = _torch_dtype(shape)
    chunk = (shape.n_heads, _lq(shape), shape.head_dim)
    slab = Kc.shape[1] if Kc.dim() == 3 else -1
    comp = (shape.n_heads, slab, shape.head_dim)
    q = _check(Q, "Q", dt, chunk)
    kc, vc = _check(Kc, "Kc", dt, comp), _check(Vc, "Vc", dt, comp)
    kl = _check(kv_len, "kv_len", torch.int32, (shape.n_heads,))
    kq, vq = _check(K_cur, "K_cur", dt, chunk), _check(V_cur, "V_cur", dt, chunk)
    o = _check(O, "O", dt, chunk)
    ls = None if lse is None else _check(lse, "lse", torch.float32, (shape.n_heads, _lq(shape)))
    ws, nws = None, 0
    if workspace is not None:
        ws, nws = _check(workspace, "workspace", torch.uint8), workspace.numel()
    return q, kc, vc, int(slab), kl, kq, vq, o, ls, ws, nws


def fkv_chunk_attention(shape: fkv_shape, Q, Kc, Vc, kv_len, K_cur, V_cur, scale: float, O,
                        lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                        stream=None):
    """``workspace`` (uint8 device tensor of fkv_attention_workspace_size bytes,
    zero-filled before its first use, e.g. torch.zeros) selects the balanced
    schedule; None runs one workgroup per query tile."""
    q, kc, vc, slab, kl, kq, vq, o, ls, ws, nws = _attention_args(shape, Q, Kc, Vc, kv_len, K_cur, V_cur, O,
                                                                  lse, workspace)
    _raise(lib().fkv_chunk_attention(ctypes.byref(shape), q, kc, vc, slab, kl, kq, vq,
                                     ctypes.c_float(scale), o, ls, ws, nws, _stream(stream)))


def fkv_chunk_attention_heads(shape: fkv_shape, heads: Sequence[int], Q, Kc, Vc, kv_len, K_cur, V_cur,
                              scale: float, O, lse: Optional[torch.Tensor] = None,
                              workspace: Optional[torch.Tensor] = None, stream=None):
    """fkv_chunk_attention for the listed heads only (host ints); the other
    heads' rows of O and lse are left untouched."""
    q, kc, vc, slab, kl, kq, vq, o, ls, ws, nws = _attention_args(shape, Q, Kc, Vc, kv_len, K_cur, V_cur, O,
                                                                  lse, workspace)
    ids = list(heads)
    arr = _ints(ids, len(ids), "heads")
    _raise(lib().fkv_chunk_attention_heads(ctypes.byref(shape), arr, len(ids), q, kc, vc, slab, kl, kq, vq,
                                           ctypes.c_float(scale), o, ls, ws, nws, _stream(stream)))


def fkv_chunk_attention_static(shape: fkv_shape, heads, K_hist, V_hist, frame_slot, Q, K_cur, V_cur,
                               scale: float, O, lse: Optional[torch.Tensor] = None,
                               workspace: Optional[torch.Tensor] = None, stream=None):
    """Attention of the static heads over their kept frames read in place
    from K_hist / V_hist; only the static heads' rows of O and lse are
    written."""
    dt = _torch_dtype(shape)
    hist = (shape.n_heads, shape.cap_frames, shape.frame_tokens, shape.head_dim)
    chunk = (shape.n_heads, _lq(shape), shape.head_dim)
    kh, vh = _check(K_hist, "K_hist", dt, hist), _check(V_hist, "V_hist", dt, hist)
    sl = _slots(frame_slot, shape.hist_frames)
    q = _check(Q, "Q", dt, chunk)
    kq, vq = _check(K_cur, "K_cur", dt, chunk), _check(V_cur, "V_cur", dt, chunk)
    o = _check(O, "O", dt, chunk)
    ls = None if lse is None else _check(lse, "lse", torch.float32, (shape.n_heads, _lq(shape)))
    ws, nws = None, 0
    if workspace is not None:
        ws, nws = _check(workspace, "workspace", torch.uint8), workspace.numel()
    _raise(lib().fkv_chunk_attention_static(ctypes.byref(shape), _heads(shape, heads), kh, vh, sl, q, kq, vq,
                                            ctypes.c_float(scale), o, ls, ws, nws, _stream(stream)))


def fkv_chunk_attention_paged(shape: fkv_shape, heads, K_hist, V_hist, frame_slot, kept_seg, kv_len, Q, K_cur,
                              V_cur, scale: float, O, lse: Optional[torch.Tensor] = None,
                              workspace: Optional[torch.Tensor] = None, head_list: Optional[Sequence[int]] = None,
                              stream=None):
    """Attention of the listed heads (all by default) with every head's kept
    history read in place from K_hist / V_hist: the Eq. 2 frames of static
    heads, the kept segments (kept_seg, kv_len from fkv_select) of dynamic
    heads.  Only the listed heads' rows of O and lse are written."""
    dt = _torch_dtype(shape)
    hist = (shape.n_heads, shape.cap_frames, shape.frame_tokens, shape.head_dim)
    chunk = (shape.n_heads, _lq(shape), shape.head_dim)
    n_seg = fkv_num_segments(shape)
    kh, vh = _check(K_hist, "K_hist", dt, hist), _check(V_hist, "V_hist", dt, hist)
    sl = _slots(frame_slot, shape.hist_frames)
    ks = None if kept_seg is None else _check(kept_seg, "kept_seg", torch.int32, (shape.n_heads, n_seg))
    kl = None if kv_len is None else _check(kv_len, "kv_len", torch.int32, (shape.n_heads,))
    q = _check(Q, "Q", dt, chunk)
    kq, vq = _check(K_cur, "K_cur", dt, chunk), _check(V_cur, "V_cur", dt, chunk)
    o = _check(O, "O", dt, chunk)
    ls = None if lse is None else _check(lse, "lse", torch.float32, (shape.n_heads, _lq(shape)))
    ws, nws = None, 0
    if workspace is not None:
        ws, nws = _check(workspace, "workspace", torch.uint8), workspace.numel()
    arr, n = None, 0
    if head_list is not None:
        ids = list(head_list)
        arr, n = _ints(ids, len(ids), "head_list"), len(ids)
    _raise(lib().fkv_chunk_attention_paged(ctypes.byref(shape), _heads(shape, heads), arr, n, kh, vh, sl, ks, kl,
                                           q, kq, vq, ctypes.c_float(scale), o, ls, ws, nws, _stream(stream)))


def fkv_fp8_sizes(shape: fkv_shape, slab: int):
    """(q_bytes, kv_bytes, scale_bytes, workspace_bytes) of the FP8 buffers."""
    out = [ctypes.c_size_t(0) for _ in range(4)]
    _raise(lib().fkv_fp8_sizes(ctypes.byref(shape), int(slab), *[ctypes.byref(o) for o in out]))
    return tuple(int(o.value) for o in out)


def fkv_fp8_pack(shape: fkv_shape, Q, Kc, Vc, kv_len, K_cur, V_cur, Q8, K8, V8T, scales,
                 workspace, stream=None):
    dt = _torch_dtype(shape)
    chunk = (shape.n_heads, _lq(shape), shape.head_dim)
    slab = Kc.shape[1] if Kc.dim() == 3 else -1
    comp = (shape.n_heads, slab, shape.head_dim)
    qb, kvb, sb, wb = fkv_fp8_sizes(shape, slab)
    args = [_check(Q, "Q", dt, chunk), _check(Kc, "Kc", dt, comp), _check(Vc, "Vc", dt, comp), int(slab),
            _check(kv_len, "kv_len", torch.int32, (shape.n_heads,)), _check(K_cur, "K_cur", dt, chunk),
            _check(V_cur, "V_cur", dt, chunk)]
    for t, name, nb in ((Q8, "Q8", qb), (K8, "K8", kvb), (V8T, "V8T", kvb)):
        args.append(_check(t, name, torch.uint8))
        if t.numel() != nb:
            raise ValueError(f"{name} holds {t.numel()} bytes, {nb} expected")
    args.append(_check(scales, "scales", torch.float32))
    if scales.numel() * 4 != sb:
        raise ValueError(f"scales holds {scales.numel() * 4} bytes, {sb} expected")
    args += [_check(workspace, "workspace", torch.uint8), workspace.numel(), _stream(stream)]
    _raise(lib().fkv_fp8_pack(ctypes.byref(shape), *args))


def fkv_fp8_pack_paged(shape: fkv_shape, heads, K_hist, V_hist, frame_slot, kept_seg, kv_len, Q, K_cur, V_cur,
                       slab: int, Q8, K8, V8T, scales, workspace, stream=None):
    """fkv_fp8_pack with every head's retained history read in place from
    K_hist / V_hist (kept frames of static heads, kept segments of dynamic
    heads); writes the static heads' kv_len."""
    dt = _torch_dtype(shape)
    hist = (shape.n_heads, shape.cap_frames, shape.frame_tokens, shape.head_dim)
    chunk = (shape.n_heads, _lq(shape), shape.head_dim)
    n_seg = fkv_num_segments(shape)
    qb, kvb, sb, wb = fkv_fp8_sizes(shape, slab)
    args = [_heads(shape, heads), _check(K_hist, "K_hist", dt, hist), _check(V_hist, "V_hist", dt, hist),
            _slots(frame_slot, shape.hist_frames),
            None if kept_seg is None else _check(kept_seg, "kept_seg", torch.int32, (shape.n_heads, n_seg)),
            _check(kv_len, "kv_len", torch.int32, (shape.n_heads,)), _check(Q, "Q", dt, chunk),
            _check(K_cur, "K_cur", dt, chunk), _check(V_cur, "V_cur", dt, chunk), int(slab)]
    for t, name, nb in ((Q8, "Q8", qb), (K8, "K8", kvb), (V8T, "V8T", kvb)):
        args.append(_check(t, name, torch.uint8))
        if t.numel() != nb:
            raise ValueError(f"{name} holds {t.numel()} bytes, {nb} expected")
    args.append(_check(scales, "scales", torch.float32))
    if scales.numel() * 4 != sb:
        raise ValueError(f"scales holds {scales.numel() * 4} bytes, {sb} expected")
    args += [_check(workspace, "workspace", torch.uint8), workspace.numel(), _stream(stream)]
    _raise(lib().fkv_fp8_pack_paged(ctypes.byref(shape), *args))


def fkv_chunk_attention_fp8(shape: fkv_shape, Q8, K8, V8T, slab: int, kv_len, scales, scale: float, O,
                            lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                            stream=None):
    chunk = (shape.n_heads, _lq(shape), shape.head_dim)
    qb, kvb, sb, _ = fkv_fp8_sizes(shape, slab)
    for t, name, nb in ((Q8, "Q8", qb), (K8, "K8", kvb), (V8T, "V8T", kvb)):
        _check(t, name, torch.uint8)
        if t.numel() != nb:
            raise ValueError(f"{name} holds {t.numel()} bytes, {nb} expected")
    ls = None if lse is None else _check(lse, "lse", torch.float32, (shape.n_heads, _lq(shape)))
    ws, nws = None, 0
    if workspace is not None:
        ws, nws = _check(workspace, "workspace", torch.uint8), workspace.numel()
    _raise(lib().fkv_chunk_attention_fp8(
        ctypes.byref(shape), _check(Q8, "Q8", torch.uint8), _check(K8, "K8", torch.uint8),
        _check(V8T, "V8T", torch.uint8), int(slab), _check(kv_len, "kv_len", torch.int32, (shape.n_heads,)),
        _check(scales, "scales", torch.float32), ctypes.c_float(scale), _check(O, "O", torch.bfloat16, chunk),
        ls, ws, nws, _stream(stream)))


def fkv_attention_mass_workspace_size(shape: fkv_shape, n_bins: int) -> int:
    out = ctypes.c_size_t(0)
    _raise(lib().fkv_attention_mass_workspace_size(ctypes.byref(shape), _i32(n_bins, "n_bins"), ctypes.byref(out)))
    return int(out.value)


def fkv_attention_mass(shape: fkv_shape, Q, Kc, kv_len, K_cur, lse, scale: float, mass,
                       accumulate: bool = False, workspace: Optional[torch.Tensor] = None, stream=None):
    """Head-profiling attention mass per key block of F keys (see fkv.h)."""
    dt = _torch_dtype(shape)
    chunk = (shape.n_heads, _lq(shape), shape.head_dim)
    slab = Kc.shape[1] if Kc.dim() == 3 else -1
    m = _check(mass, "mass", torch.float32)
    if mass.dim() != 2 or mass.shape[0] != shape.n_heads:
        raise ValueError("mass must be [n_heads][n_bins]")
    n_bins = mass.shape[1]
    need = fkv_attention_mass_workspace_size(shape, n_bins)
    if workspace is None:
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=Q.device)
    _raise(lib().fkv_attention_mass(
        ctypes.byref(shape), _check(Q, "Q", dt, chunk), _check(Kc, "Kc", dt, (shape.n_heads, slab, shape.head_dim)),
        int(slab), _check(kv_len, "kv_len", torch.int32, (shape.n_heads,)), _check(K_cur, "K_cur", dt, chunk),
        _check(lse, "lse", torch.float32, (shape.n_heads, _lq(shape))), ctypes.c_float(scale), int(n_bins), m,
        1 if accumulate else 0, _check(workspace, "workspace", torch.uint8), workspace.numel(), _stream(stream)))
    return workspace


def fkv_classify_heads(mass, hist_frames: int, sink_frames: int = 1, transition_frames: int = 1,
                       alpha: float = 0.8):
    """Eq. 1 on a host mass table [n_heads][n_bins] (numpy float32 or a CPU
    tensor); returns a list of FKV_STATIC / FKV_DYNAMIC."""
    import numpy as np
    m = np.ascontiguousarray(mass.cpu().numpy() if isinstance(mass, torch.Tensor) else mass, dtype=np.float32)
    n_heads, n_bins = m.shape
    out = (ctypes.c_int32 * n_heads)()
    _raise(lib().fkv_classify_heads(m.ctypes.data_as(ctypes.c_void_p), n_heads, n_bins,
                                    *(_i32(v, "frames") for v in (hist_frames, sink_frames, transition_frames)), ctypes.c_float(alpha), out))
    return list(out)


# ---------------------------------------------------------------------------
# position rotation and the 8-bit rolling cache
# ---------------------------------------------------------------------------
def make_rope(frame_pairs: int, row_pairs: int = 0, col_pairs: int = 0, row_tokens: int = 1, token_step: int = 0,
              theta: float = 10000.0, pairing: int = FKV_PAIR_ADJACENT) -> fkv_rope:
    """How channel pairs turn with position: the first ``frame_pairs`` by the
    frame position, then ``row_pairs`` by the token's row and ``col_pairs`` by its
    column in rows of ``row_tokens`` tokens (see fkv.h)."""
    counts = (frame_pairs, row_pairs, col_pairs, row_tokens, token_step, pairing)
    return fkv_rope(*(_i32(v, "rope") for v in counts), float(theta))


class Cache8:
    """A rolling cache held in 8 bits: ``K``, ``V`` float8_e4m3fn
    [n_heads][cap_frames][F][d] and ``k_scale``, ``v_scale`` float32
    [n_heads][cap_frames][ceil(F / block_tokens)], powers of two."""

    def __init__(self, K, V, k_scale, v_scale, block_tokens: int):
        self.K, self.V, self.k_scale, self.v_scale, self.block_tokens = K, V, k_scale, v_scale, int(block_tokens)

    @classmethod
    def zeros(cls, shape: fkv_shape, block_tokens: int = 64, device="cuda"):
        """An empty cache of the shape's slots (codes 0, scales 1)."""
        size = (shape.n_heads, shape.cap_frames, shape.frame_tokens, shape.head_dim)
        nb = -(-shape.frame_tokens // int(block_tokens))
        code = lambda: torch.zeros(size, dtype=torch.uint8, device=device).view(torch.float8_e4m3fn)  # noqa: E731
        scale = lambda: torch.ones(size[:2] + (nb,), dtype=torch.float32, device=device)  # noqa: E731
        return cls(code(), code(), scale(), scale(), block_tokens)


def _ptr(t: torch.Tensor, name: str, dtype, size, device: int) -> int:
    """_check with the size given and the device already known (its index)."""
    if isinstance(t, torch.Tensor) and t.dtype is dtype and t.get_device() == device and t.shape == size and t.is_contiguous():
        return t.data_ptr()
    _check(t, name, dtype, size)
    raise ValueError(f"{name} is on {t.device}, other tensors of the call on cuda:{device}")


def _device_of(t: torch.Tensor, name: str) -> int:
    """Index of the GPU that a call runs on, whichever is current: that of its tensor t."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor (got {t.device})")
    return t.get_device()


def _cache8(shape: fkv_shape, c: Cache8, device: int):
    if not isinstance(c, Cache8):
        raise TypeError("cache must be a Cache8")
    if c.block_tokens not in (16, 32, 64, 128):
        raise ValueError(f"block_tokens {c.block_tokens} is not 16, 32, 64 or 128")
    size = (shape.n_heads, shape.cap_frames, shape.frame_tokens, shape.head_dim)
    nb = size[:2] + (-(-size[2] // c.block_tokens),)
    f8, f32 = torch.float8_e4m3fn, torch.float32
    return fkv_cache8(_ptr(c.K, "cache.K", f8, size, device), _ptr(c.V, "cache.V", f8, size, device),
                      _ptr(c.k_scale, "cache.k_scale", f32, nb, device), _ptr(c.v_scale, "cache.v_scale", f32, nb, device),
                      c.block_tokens)


def _rows(t: torch.Tensor, name: str, dtype, size, device: int):
    """Rows [n_heads][n][d] of any head and token stride, the channels adjacent."""
    if isinstance(t, torch.Tensor) and t.dtype is dtype and t.get_device() == device and t.shape == size:
        head, token, channel = t.stride()
        if channel != 1:
            raise ValueError(f"{name}: the channels of a row must be adjacent")
        # (a dimension of one element may report any stride)
        return fkv_rows(t.data_ptr(), head if size[0] > 1 else 0, token if size[1] > 1 else 0)
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype} (got {t.dtype})")
    if t.get_device() != device:
        raise ValueError(f"{name} must be on cuda:{device} (got {t.device})")
    raise ValueError(f"{name} must have shape {size} (got {tuple(t.shape)})")


def _ints(values, n: int, name: str):
    """A host int32 array of n entries from a sequence, numpy array or tensor of
    whole numbers (ctypes would cut others down to 32 bits)."""
    vals = values.tolist() if hasattr(values, "tolist") else list(values)
    if len(vals) != n:
        raise ValueError(f"{name} needs {n} entries (got {len(vals)})")
    ints = list(map(int, vals))
    if ints != vals or (n and not (-1 << 31 <= min(ints) and max(ints) < 1 << 31)):
        raise ValueError(f"{name}: {vals} are not whole numbers of 32 bits")
    return (ctypes.c_int32 * (n or 1))(*ints)


def _frames(shape: fkv_shape, frame_slot):
    H = shape.hist_frames
    return _ints(range(H) if frame_slot is None else frame_slot, H, "frame_slot")


def _positions(frame_pos, n: int):
    vals = frame_pos.tolist() if hasattr(frame_pos, "tolist") else frame_pos
    if len(vals) and not (-FKV_MAX_POSITION <= min(vals) and max(vals) <= FKV_MAX_POSITION):
        raise ValueError(f"frame_pos outside +-{FKV_MAX_POSITION}")
    return _ints(vals, n, "frame_pos")


def _n_seg(shape: fkv_shape) -> int:
    """fkv_num_segments of a shape that the call itself checks."""
    L = shape.seg_tokens
    return -(-shape.hist_frames * shape.frame_tokens // L) if L > 0 else 0


def _run(device: int, fn, args, stream):
    """fn(*args, stream) on ``device``, by default on its current stream."""
    if device == torch._C._cuda_getDevice():
        # (the stream's handle alone: a Stream object costs more than a small call's launch)
        return _raise(fn(*args, torch._C._cuda_getCurrentRawStream(device) if stream is None else stream.cuda_stream))
    with torch.cuda.device(device):
        _raise(fn(*args, torch._C._cuda_getCurrentRawStream(device) if stream is None else stream.cuda_stream))


def fkv_rotate_chunk(shape: fkv_shape, rope: fkv_rope, frame_pos, Q, K, V, Qr, Kr, Vr, stream=None):
    """Q and K of the chunk rotated into Qr and Kr, V copied into Vr
    ([n_heads][C*F][d] contiguous).  Q, K, V may be any strided views of that
    shape with adjacent channels (a projection's [tokens][3][n_heads][d], say).
    A pair of Nones is left out."""
    dt = _torch_dtype(shape)
    size = (shape.n_heads, _lq(shape), shape.head_dim)
    dev, src, dst = None, [], []
    for t, o, name in ((Q, Qr, "Q"), (K, Kr, "K"), (V, Vr, "V")):
        if (t is None) != (o is None):
            raise ValueError(f"{name} and its output must both be given or both be None")
        if t is None:
            src.append(None)
            dst.append(None)
            continue
        if dev is None:
            dev = _device_of(t, name)
        src.append(ctypes.byref(_rows(t, name, dt, size, dev)))
        dst.append(_ptr(o, name + "r", dt, size, dev))
    if dev is None:
        raise ValueError("nothing to rotate")
    pos = _positions(frame_pos, shape.chunk_frames)
    _run(dev, lib().fkv_rotate_chunk, (ctypes.byref(shape), ctypes.byref(rope), pos, *src, *dst), stream)


def _new_rows(shape, K_new, V_new, n, dev):
    size = (shape.n_heads, n * shape.frame_tokens, shape.head_dim)
    dt = _torch_dtype(shape)
    return ctypes.byref(_rows(K_new, "K_new", dt, size, dev)), ctypes.byref(_rows(V_new, "V_new", dt, size, dev))


def fkv_append_frames_rotated(shape: fkv_shape, rope: fkv_rope, frame_pos, K_new, V_new, dst_slot, K_hist, V_hist,
                              stream=None):
    """fkv_append_frames with the keys of frame f rotated at frame_pos[f] on the
    way.  K_new, V_new: strided views [n_heads][n*F][d] with adjacent channels."""
    dt = _torch_dtype(shape)
    hist = (shape.n_heads, shape.cap_frames, shape.frame_tokens, shape.head_dim)
    n = len(dst_slot)
    dev = _device_of(K_new, "K_new")
    kn, vn = _new_rows(shape, K_new, V_new, n, dev)
    kh, vh = _ptr(K_hist, "K_hist", dt, hist, dev), _ptr(V_hist, "V_hist", dt, hist, dev)
    _run(dev, lib().fkv_append_frames_rotated,
         (ctypes.byref(shape), ctypes.byref(rope), _positions(frame_pos, n), kn, vn, n, _ints(dst_slot, n, "dst_slot"), kh,
          vh), stream)


def fkv_append_frames_q8(shape: fkv_shape, rope: Optional[fkv_rope], frame_pos, K_new, V_new, dst_slot, cache: Cache8,
                         stream=None):
    """fkv_append_frames into an 8-bit cache, the keys rotated on the way (rope
    and frame_pos None: as they are).  K_new, V_new as in
    fkv_append_frames_rotated; the shape's dtype is theirs."""
    n = len(dst_slot)
    dev = _device_of(K_new, "K_new")
    kn, vn = _new_rows(shape, K_new, V_new, n, dev)
    c = _cache8(shape, cache, dev)
    rp, pos = (None, None) if rope is None else (ctypes.byref(rope), _positions(frame_pos, n))
    _run(dev, lib().fkv_append_frames_q8,
         (ctypes.byref(shape), rp, pos, kn, vn, n, _ints(dst_slot, n, "dst_slot"), ctypes.byref(c)), stream)


def fkv_score_select_q8(shape: fkv_shape, heads, cache: Cache8, frame_slot, K_cur, scores, kept_seg, kv_len,
                        workspace: Optional[torch.Tensor] = None, stream=None):
    """fkv_score_select over the keys of an 8-bit cache.  If ``workspace`` is
    None a zero-filled one is allocated (through torch's caching allocator)."""
    n, n_seg, i32 = shape.n_heads, _n_seg(shape), torch.int32
    dev = _device_of(K_cur, "K_cur")
    c = _cache8(shape, cache, dev)
    kc = _ptr(K_cur, "K_cur", _torch_dtype(shape), (n, _lq(shape), shape.head_dim), dev)
    sc = _ptr(scores, "scores", torch.float32, (n, n_seg), dev)
    ks, kl = _ptr(kept_seg, "kept_seg", i32, (n, n_seg), dev), _ptr(kv_len, "kv_len", i32, (n,), dev)
    if workspace is None:
        need = fkv_score_workspace_size(shape, heads)
        with torch.cuda.stream(stream):               # (filled on the stream that uses it)
            workspace = torch.zeros(max(need, 1), dtype=torch.uint8, device=K_cur.device)
    ws = _ptr(workspace, "workspace", torch.uint8, getattr(workspace, "shape", None), dev)
    _run(dev, lib().fkv_score_select_q8,
         (ctypes.byref(shape), _heads(shape, heads), ctypes.byref(c), _frames(shape, frame_slot),
          kc, sc, ks, kl, ws, workspace.numel()), stream)
    return workspace


def fkv_chunk_attention_q8_workspace_size(shape: fkv_shape, heads, n_q: int, n_cur: int) -> int:
    """Bytes of the workspace of fkv_chunk_attention_q8 on the current device."""
    out = ctypes.c_size_t(0)
    _raise(lib().fkv_chunk_attention_q8_workspace_size(ctypes.byref(shape), _heads(shape, heads), _i32(n_q, "n_q"),
                                                       _i32(n_cur, "n_cur"), ctypes.byref(out)))
    return int(out.value)


def fkv_chunk_attention_q8(shape: fkv_shape, heads, cache: Cache8, frame_slot, kept_seg, kv_len, Q, K_cur, V_cur,
                           scale: float, O, lse: Optional[torch.Tensor] = None,
                           workspace: Optional[torch.Tensor] = None, stream=None):
    """Attention of the query tokens Q [n_heads][n_q][d] over every head's kept
    history in the 8-bit cache and the current tokens K_cur, V_cur
    [n_heads][n_cur][d] (None, or n_cur = 0: none).  ``workspace``: uint8 device
    tensor of fkv_chunk_attention_q8_workspace_size bytes (no initialisation);
    None runs one workgroup per query tile."""
    bf, i32 = torch.bfloat16, torch.int32
    n, d = shape.n_heads, shape.head_dim
    dev = _device_of(Q, "Q")
    n_q = Q.shape[1] if Q.dim() == 3 else -1
    qs = (n, n_q, d)
    q, o = _ptr(Q, "Q", bf, qs, dev), _ptr(O, "O", bf, qs, dev)
    c = _cache8(shape, cache, dev)
    ks = kl = kq = vq = ls = ws = None
    n_cur = nws = 0
    if kept_seg is not None:
        ks = _ptr(kept_seg, "kept_seg", i32, (n, _n_seg(shape)), dev)
    if kv_len is not None:
        kl = _ptr(kv_len, "kv_len", i32, (n,), dev)
    if (K_cur is None) != (V_cur is None):
        raise ValueError("K_cur and V_cur must both be given or both be None")
    if K_cur is not None:
        n_cur = K_cur.shape[1] if K_cur.dim() == 3 else -1
        kq, vq = _ptr(K_cur, "K_cur", bf, (n, n_cur, d), dev), _ptr(V_cur, "V_cur", bf, (n, n_cur, d), dev)
    if lse is not None:
        ls = _ptr(lse, "lse", torch.float32, (n, n_q), dev)
    if workspace is not None:
        ws, nws = _ptr(workspace, "workspace", torch.uint8, getattr(workspace, "shape", None), dev), workspace.numel()
    _run(dev, lib().fkv_chunk_attention_q8,
         (ctypes.byref(shape), _heads(shape, heads), ctypes.byref(c), _frames(shape, frame_slot),
          ks, kl, q, n_q, kq, vq, n_cur, scale, o, ls, ws, nws), stream)


class PagedBatch:
    """The sequences of a call over paged caches (see fkv_batch in include/fkv.h).

    ``page_table`` int32 [n_seqs][max_pages], ``seq_len`` int32 [n_seqs] (new
    tokens included) and ``q_start`` int32 [n_seqs + 1] (rows of each sequence's
    new tokens) lie on the GPU and may be written between calls.  ``n_tokens``
    rows have the batch's tensors; ``max_new`` is at least every sequence's new
    tokens, ``sum_len`` at least the sum of ``seq_len`` (the expanded latent form
    needs it; elsewhere 0 for unknown, with which form "auto" stays absorbed)."""

    def __init__(self, page_table, seq_len, q_start, page_tokens: int, n_tokens: int, max_new: int, sum_len: int = 0):
        self.device = _device_of(page_table, "page_table")
        n = page_table.shape[0] if page_table.dim() == 2 else -1
        table = _ptr(page_table, "page_table", torch.int32, (n, page_table.shape[-1]), self.device)
        lens = _ptr(seq_len, "seq_len", torch.int32, (n,), self.device)
        starts = _ptr(q_start, "q_start", torch.int32, (n + 1,), self.device)
        total = int(sum_len)
        if total != sum_len or not 0 <= total < 1 << 62:
            raise ValueError(f"sum_len: {sum_len} is not a whole number of tokens")
        self.page_table, self.seq_len, self.q_start = page_table, seq_len, q_start
        self.n_seqs, self.page_tokens, self.n_tokens = n, _i32(page_tokens, "page_tokens"), _i32(n_tokens, "n_tokens")
        self.max_new, self.sum_len = _i32(max_new, "max_new"), total
        self._c = fkv_batch(n, page_table.shape[1], self.page_tokens, 1, self.n_tokens, self.max_new, total, table, lens, starts)

    def _arg(self, n_pages: int):
        """The C batch of a call over n_pages pages (one of its own: calls of other threads have theirs)."""
        c = fkv_batch.from_buffer_copy(self._c)
        c.n_pages = n_pages
        return ctypes.byref(c)


def _batch(batch) -> "PagedBatch":
    if not isinstance(batch, PagedBatch):
        raise TypeError("batch must be a PagedBatch")
    return batch


def _pages(t, name: str, dtype, page_tokens: int, device: int):
    """Pages [n_pages][n_heads][page_tokens][width], contiguous."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dim() != 4:
        raise ValueError(f"{name} must have 4 dimensions (got shape {tuple(t.shape)})")
    return _ptr(t, name, dtype, (t.shape[0], t.shape[1], page_tokens, t.shape[3]), device)


def _spans(spans, n: int):
    """A host fkv_span array from (sink_tokens, recent_tokens) pairs, recent_tokens -1 or None for all."""
    if spans is None:
        return None
    if len(spans) != n:
        raise ValueError(f"spans has {len(spans)} entries for {n} key heads")
    arr = (fkv_span * n)()
    for y, (sink, recent) in enumerate(spans):
        arr[y] = fkv_span(_i32(sink, "sink_tokens"), -1 if recent is None else _i32(recent, "recent_tokens"))
    return arr


def fkv_append_paged(batch: PagedBatch, K_new, V_new, K_pages, V_pages, stream=None):
    """The batch's new keys and values into their pages.  K_new, V_new: bf16 or
    fp32 views [n_heads][n_tokens][d] with adjacent channels; K_pages, V_pages
    [n_pages][n_heads][page_tokens][d].  V_new and V_pages None: keys (or latent
    rows, one head) alone."""
    b = _batch(batch)
    if not isinstance(K_pages, torch.Tensor) or K_pages.dtype not in (torch.bfloat16, torch.float32):
        raise TypeError("K_pages must be a bfloat16 or float32 tensor")
    if (V_new is None) != (V_pages is None):
        raise ValueError("V_new and V_pages must both be given or both be None")
    dt = K_pages.dtype
    kp = _pages(K_pages, "K_pages", dt, b.page_tokens, b.device)
    n_pages, heads, _, d = K_pages.shape
    size = (heads, b.n_tokens, d)
    vp = vn = None
    if V_pages is not None:
        vp = _ptr(V_pages, "V_pages", dt, K_pages.shape, b.device)
        vn = ctypes.byref(_rows(V_new, "V_new", dt, size, b.device))
    _run(b.device, lib().fkv_append_paged,
         (b._arg(n_pages), heads, d, FKV_BF16 if dt is torch.bfloat16 else FKV_F32,
          ctypes.byref(_rows(K_new, "K_new", dt, size, b.device)), vn, kp, vp), stream)


def fkv_paged_attention_workspace_size(batch: PagedBatch, n_heads: int, n_kv_heads: int, head_dim: int) -> int:
    """Bytes of the workspace of fkv_paged_attention on the batch's device."""
    out = ctypes.c_size_t(0)
    b = _batch(batch)
    with torch.cuda.device(b.device):
        _raise(lib().fkv_paged_attention_workspace_size(b._arg(1), _i32(n_heads, "n_heads"), _i32(n_kv_heads, "n_kv_heads"),
                                                        _i32(head_dim, "head_dim"), ctypes.byref(out)))
    return int(out.value)


def fkv_paged_attention(batch: PagedBatch, Q, K_pages, V_pages, scale: float, O, causal: bool = True, spans=None,
                        lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None):
    """Attention of every sequence's new tokens over its pages.  Q, O: bf16
    views [n_heads][n_tokens][d] with adjacent channels; K_pages, V_pages
    [n_pages][n_kv_heads][page_tokens][d]; spans: per key head (sink_tokens,
    recent_tokens), recent_tokens -1 for all, or None; lse float32
    [n_heads][n_tokens].  ``workspace``: uint8 device tensor of
    fkv_paged_attention_workspace_size bytes (no initialisation); None splits
    nothing."""
    b, bf = _batch(batch), torch.bfloat16
    kp = _pages(K_pages, "K_pages", bf, b.page_tokens, b.device)
    n_pages, kv, _, d = K_pages.shape
    vp = _ptr(V_pages, "V_pages", bf, K_pages.shape, b.device)
    n_heads = Q.shape[0] if isinstance(Q, torch.Tensor) and Q.dim() == 3 else -1
    size = (n_heads, b.n_tokens, d)
    q, o = _rows(Q, "Q", bf, size, b.device), _rows(O, "O", bf, size, b.device)
    ls = ws = None
    nws = 0
    if lse is not None:
        ls = _ptr(lse, "lse", torch.float32, size[:2], b.device)
    if workspace is not None:
        ws, nws = _ptr(workspace, "workspace", torch.uint8, getattr(workspace, "shape", None), b.device), workspace.numel()
    _run(b.device, lib().fkv_paged_attention,
         (b._arg(n_pages), n_heads, kv, d, ctypes.byref(q), kp, vp, int(bool(causal)), _spans(spans, kv), scale,
          ctypes.byref(o), ls, ws, nws), stream)


_FORMS = {"auto": FKV_LATENT_AUTO, "absorbed": FKV_LATENT_ABSORBED, "expanded": FKV_LATENT_EXPANDED}


def _form(form) -> int:
    if form not in _FORMS:
        raise ValueError(f"form {form!r} is not one of {sorted(_FORMS)}")
    return _FORMS[form]


def fkv_latent_attention_workspace_size(batch: PagedBatch, n_heads: int, head_dim: int, latent_dim: int,
                                        form: str = "auto") -> int:
    """Bytes of the workspace of fkv_latent_attention on the batch's device."""
    out = ctypes.c_size_t(0)
    b = _batch(batch)
    with torch.cuda.device(b.device):
        _raise(lib().fkv_latent_attention_workspace_size(b._arg(1), _i32(n_heads, "n_heads"), _i32(head_dim, "head_dim"),
                                                         _i32(latent_dim, "latent_dim"), _form(form), ctypes.byref(out)))
    return int(out.value)


def fkv_latent_attention(batch: PagedBatch, Q, pages, W_k, W_v, scale: float, O, causal: bool = True, span=None,
                         form: str = "auto", workspace: Optional[torch.Tensor] = None, stream=None):
    """Attention over a paged latent cache.  Q: bf16 view [n_heads][n_tokens][d +
    64]; pages [n_pages][1][page_tokens][latent_dim + 64]; W_k, W_v
    [n_heads][d][latent_dim]; O: bf16 view [n_heads][n_tokens][d]; span:
    (sink_tokens, recent_tokens) or None.  form: "auto", "absorbed" or "expanded".
    ``workspace``: uint8 device tensor of fkv_latent_attention_workspace_size
    bytes (no initialisation); None allocates one (through torch's caching
    allocator)."""
    b, bf = _batch(batch), torch.bfloat16
    pp = _pages(pages, "pages", bf, b.page_tokens, b.device)
    n_pages, one, _, width = pages.shape
    if one != 1:
        raise ValueError(f"pages of a latent cache have one head (got {one})")
    R = width - FKV_LATENT_ROT
    n_heads, d = (W_k.shape[0], W_k.shape[1]) if isinstance(W_k, torch.Tensor) and W_k.dim() == 3 else (-1, -1)
    wk, wv = _ptr(W_k, "W_k", bf, (n_heads, d, R), b.device), _ptr(W_v, "W_v", bf, (n_heads, d, R), b.device)
    q = _rows(Q, "Q", bf, (n_heads, b.n_tokens, d + FKV_LATENT_ROT), b.device)
    o = _rows(O, "O", bf, (n_heads, b.n_tokens, d), b.device)
    if workspace is None:
        need = fkv_latent_attention_workspace_size(b, n_heads, d, R, form)
        with torch.cuda.stream(stream):                # (used on that stream)
            workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=pages.device)
    ws = _ptr(workspace, "workspace", torch.uint8, getattr(workspace, "shape", None), b.device)
    _run(b.device, lib().fkv_latent_attention,
         (b._arg(n_pages), n_heads, d, R, ctypes.byref(q), pp, wk, wv, int(bool(causal)),
          None if span is None else _spans([span], 1), scale, ctypes.byref(o), _form(form), ws, workspace.numel()), stream)


def fkv_last_error() -> str:
    return lib().fkv_last_error().decode()
