"""MI355X (gfx950) hot path of training-free revisit consistency
(arXiv 2607.21848, Sec. 4.2 and Sec. 4.3).

Python binding of librevisit: argument marshalling only. Every stage runs
in the library's HIP kernels; torch tensors supply device memory and the
current HIP stream. The entry points mirror include/revisit.h:

* ``retrieve_chunks``          -- pose retrieval (Sec. 4.2, Eq. retrieval)
* ``reproject_correspondence`` -- depth/pose reprojection and visibility
                                  (Sec. 4.3, Eq. reprojection, Eq. visibility)
* ``reproject_rotation``       -- its fixed-centre case, the rotation / zoom
                                  homography without depth (Sec. 4.3)
* ``biased_chunk_attention``   -- attention with the Gaussian correspondence
                                  bias (Sec. 4.3, Eq. bias)
* ``rotary_embed``             -- rotary positions of q and k (time, row, column)
* ``attention_key_weight``     -- the weight of every cached key in the attention
* ``select_kept``              -- which units of the cache to keep, by weight
* ``compact_kv``               -- move of the kept units into a smaller cache
* ``append_paged_kv``          -- new keys and values of many streams into the
                                  pages of their cache, keys turned to their positions
* ``paged_chunk_attention``    -- the attention over those pages, in the queries' type or 8 bits

Each accepts optional preallocated outputs (``out=``) and, where a kernel
needs scratch memory, a preallocated ``workspace=`` (a uint8 GPU tensor of at
least ``attention_workspace_size(...)`` / ``retrieve_workspace_size(...)`` /
``key_weight_workspace_size(...)`` / ``select_workspace_size(...)`` /
``paged_attention_workspace_size(...)`` bytes), so a caller can run the path without allocating; without one the binding
allocates the workspace with torch on the current stream.
"""

from __future__ import annotations

import ctypes
from typing import Optional, Sequence

import torch

from . import _lib
from ._lib import BF16, F32, FP8_KV, FP8_QK, MAX_K, RevisitError, last_error, lib, status_string  # noqa: F401

__all__ = ["retrieve_chunks", "reproject_correspondence", "reproject_rotation", "biased_chunk_attention", "pack_retrieved_kv",
           "pool_token_depth", "rotary_embed", "attention_key_weight", "select_kept", "compact_kv", "append_paged_kv", "paged_chunk_attention",
           "StreamDriver",
           "attention_workspace_size", "retrieve_workspace_size", "key_weight_workspace_size", "select_workspace_size",
           "paged_attention_workspace_size", "RevisitError", "lib"]


# The small calls are as long as their marshalling (a launch itself is 4 us):
# the handle of the current stream without a Stream object (0.1 against 1.9 us),
# pointers as plain integers, and one expression for a tensor that is in order
# took a retrieval from 17.2 to 14.2 us of host time and an attention call from
# 16.6 to 11.9.
def _ptr(t: Optional[torch.Tensor]):
    return t.data_ptr() if t is not None else None


# not public names: without them the slower public ones
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _stream(device: torch.device):
    return _raw_stream(device.index)


def _need(t: torch.Tensor, name: str, dtype: torch.dtype, shape: Optional[Sequence[int]] = None, device=None):
    if (isinstance(t, torch.Tensor) and t.dtype == dtype and t.is_contiguous() and (shape is None or t.shape == shape)
            and (t.is_cuda if device is None else t.get_device() == device.index)):  # -1 and None on the CPU
        return t
    return _unfit(t, name, dtype, shape, device)


def _unfit(t, name: str, dtype: torch.dtype, shape=None, device=None, contiguous: bool = True):
    """What is wrong with a tensor; the tensor where nothing is."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.device.type != "cuda":
        raise ValueError(f"{name} must be a GPU tensor (got {t.device}); there is no CPU path")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype} (got {t.dtype})")
    if contiguous and not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    return t


def _workspace(nbytes: int, workspace: Optional[torch.Tensor], dev: torch.device, name: str):
    """The caller's workspace (checked) or a fresh one of nbytes; None when nothing is needed."""
    if workspace is not None:
        _need(workspace, name, torch.uint8, None, dev)
        return workspace
    if nbytes == 0:
        return None
    return torch.empty(nbytes, dtype=torch.uint8, device=dev)


def retrieve_workspace_size(n_bank: int, n_query: int, k: int) -> int:
    """Bytes of workspace retrieve_chunks needs (0 for banks of at most 8192 entries)."""
    n = ctypes.c_size_t(0)
    _lib.check("rc_retrieve_workspace_size", lib().rc_retrieve_workspace_size(int(n_bank), int(n_query), int(k),
                                                                              ctypes.byref(n)))
    return int(n.value)


def attention_workspace_size(dtype: torch.dtype, Lq: int, Lk: int, H: int, D: int, key_parts: int = 0) -> int:
    """Bytes of workspace biased_chunk_attention needs on the current device
    (dtype: torch.bfloat16, torch.float32 or torch.float8_e4m3fn for q)."""
    n = ctypes.c_size_t(0)
    _lib.check("rc_attention_workspace_size",
               lib().rc_attention_workspace_size(_attn_dtype(dtype), int(Lq), int(Lk), int(H), int(D), int(key_parts),
                                                 ctypes.byref(n)))
    return int(n.value)


def _attn_dtype_of(t: torch.Tensor, name: str) -> int:
    try:
        return _attn_dtype(t.dtype)
    except TypeError:
        raise TypeError(f"{name} must be bfloat16, float32 or float8_e4m3fn (got {t.dtype})") from None


def _attn_dtype(dtype: torch.dtype) -> int:
    if dtype == torch.bfloat16:
        return BF16
    if dtype == torch.float32:
        return F32
    if dtype == torch.float8_e4m3fn:
        return FP8_QK
    raise TypeError(f"q must be bfloat16, float32 or float8_e4m3fn (got {dtype})")


def retrieve_chunks(bank_c2w: torch.Tensor, query_c2w: torch.Tensor, query_chunk: torch.Tensor, *,
                    E: float, w_v: float, tau_c: float, tau_v: float, delta: int, first_candidate: int, k: int,
                    frames_per_chunk: Optional[int] = None, out=None, workspace: Optional[torch.Tensor] = None):
    """Top-k pose retrieval. bank_c2w [N,4,4] f32, query_c2w [Q,4,4] f32,
    query_chunk [Q] i32. Returns (idx [Q,k] i32, score [Q,k] f32,
    count [Q] i32, frame_sel [Q,k*F] i32 or None)."""
    dev = query_c2w.device
    N, Q = bank_c2w.shape[0], query_c2w.shape[0]
    _need(bank_c2w, "bank_c2w", torch.float32, (N, 4, 4), dev)
    _need(query_c2w, "query_c2w", torch.float32, (Q, 4, 4), dev)
    _need(query_chunk, "query_chunk", torch.int32, (Q,), dev)
    if out is None:
        idx = torch.empty((Q, k), dtype=torch.int32, device=dev)
        score = torch.empty((Q, k), dtype=torch.float32, device=dev)
        count = torch.empty((Q,), dtype=torch.int32, device=dev)
        sel = (torch.empty((Q, k * frames_per_chunk), dtype=torch.int32, device=dev)
               if frames_per_chunk is not None else None)
    else:
        idx, score, count, sel = out
        _need(idx, "out idx", torch.int32, (Q, k), dev)
        _need(score, "out score", torch.float32, (Q, k), dev)
        _need(count, "out count", torch.int32, (Q,), dev)
        if (sel is None) != (frames_per_chunk is None):
            raise ValueError("out frame_sel must be given exactly when frames_per_chunk is")
        if sel is not None:
            _need(sel, "out frame_sel", torch.int32, (Q, k * frames_per_chunk), dev)
    ws = _workspace(retrieve_workspace_size(N, Q, k), workspace, dev, "workspace")
    st = lib().retrieve_chunks(_ptr(bank_c2w), N, _ptr(query_c2w), _ptr(query_chunk), Q, E, w_v, tau_c, tau_v,
                               delta, first_candidate, k, _ptr(idx), _ptr(score), _ptr(count),
                               frames_per_chunk or 0, _ptr(sel), _ptr(ws), ws.numel() if ws is not None else 0,
                               _stream(dev))
    _lib.check("retrieve_chunks", st)
    return idx, score, count, sel


def reproject_correspondence(tgt_depth: torch.Tensor, tgt_c2w: torch.Tensor, tgt_K: torch.Tensor,
                             src_depth: torch.Tensor, src_c2w: torch.Tensor, src_K: torch.Tensor, *,
                             p: int, eps: float, src_sel: Optional[torch.Tensor] = None, out=None):
    """Correspondence of every target token into every source frame.

    Batched: tgt_depth [B,Tq,h*p,w*p], tgt_c2w [B,Tq,4,4], tgt_K [B,Tq,4];
    sources [B,S,...] or, with src_sel [B,S] i32, a frame bank [n_src,...].
    Unbatched inputs (no leading B) give unbatched outputs.
    Returns (uv [B,S,Tq*h*w,2] f32, idx [B,S,Tq*h*w] i32)."""
    batched = tgt_depth.dim() == 4
    if not batched:
        tgt_depth, tgt_c2w, tgt_K = tgt_depth[None], tgt_c2w[None], tgt_K[None]
        if src_sel is None:
            src_depth, src_c2w, src_K = src_depth[None], src_c2w[None], src_K[None]
        else:
            src_sel = src_sel[None]
    dev = tgt_depth.device
    B, Tq, Hd, Wd = tgt_depth.shape
    if Hd % p or Wd % p:
        raise ValueError(f"depth map {Hd}x{Wd} is not a whole number of {p}x{p} tokens")
    h, w = Hd // p, Wd // p
    _need(tgt_depth, "tgt_depth", torch.float32, None, dev)
    _need(tgt_c2w, "tgt_c2w", torch.float32, (B, Tq, 4, 4), dev)
    _need(tgt_K, "tgt_K", torch.float32, (B, Tq, 4), dev)
    if src_sel is None:
        S = src_depth.shape[1]
        _need(src_depth, "src_depth", torch.float32, (B, S, Hd, Wd), dev)
        _need(src_c2w, "src_c2w", torch.float32, (B, S, 4, 4), dev)
        _need(src_K, "src_K", torch.float32, (B, S, 4), dev)
        n_src = 0
    else:
        S = src_sel.shape[1]
        n_src = src_depth.shape[0]
        _need(src_sel, "src_sel", torch.int32, (B, S), dev)
        _need(src_depth, "src_depth", torch.float32, (n_src, Hd, Wd), dev)
        _need(src_c2w, "src_c2w", torch.float32, (n_src, 4, 4), dev)
        _need(src_K, "src_K", torch.float32, (n_src, 4), dev)
    Lq = Tq * h * w
    if out is None:
        uv = torch.empty((B, S, Lq, 2), dtype=torch.float32, device=dev)
        idx = torch.empty((B, S, Lq), dtype=torch.int32, device=dev)
    else:
        uv, idx = out
        _need(uv, "out uv", torch.float32, (B, S, Lq, 2), dev)
        _need(idx, "out idx", torch.int32, (B, S, Lq), dev)
    st = lib().reproject_correspondence(_ptr(tgt_depth), _ptr(tgt_c2w), _ptr(tgt_K), _ptr(src_depth),
                                        _ptr(src_c2w), _ptr(src_K), _ptr(src_sel), n_src, B, Tq, S, h, w, p,
                                        eps, _ptr(uv), _ptr(idx), _stream(dev))
    _lib.check("reproject_correspondence", st)
    if not batched:
        return uv[0], idx[0]
    return uv, idx


def reproject_rotation(tgt_c2w: torch.Tensor, tgt_K: torch.Tensor, src_c2w: torch.Tensor, src_K: torch.Tensor, *,
                       h: int, w: int, p: int, src_sel: Optional[torch.Tensor] = None, out=None):
    """Rotation-only correspondence (sources sharing the target's centre): the
    homography u^ = pi(K_s R_s^T R_t K_t^-1 u~), no depth, no visibility test.

    Batched: tgt_c2w [B,Tq,4,4], tgt_K [B,Tq,4]; sources [B,S,...] or, with
    src_sel [B,S] i32, a frame bank [n_src,...]; h, w the token grid, p the
    latent pixels per token side (K is in depth-map pixels). Unbatched inputs
    give unbatched outputs. Returns (uv [B,S,Tq*h*w,2] f32, idx [B,S,Tq*h*w]
    i32), idx = REVISIT_CENTRE_MOVED (-6) for a pair whose centres differ."""
    batched = tgt_c2w.dim() == 4
    if not batched:
        tgt_c2w, tgt_K = tgt_c2w[None], tgt_K[None]
        if src_sel is None:
            src_c2w, src_K = src_c2w[None], src_K[None]
        else:
            src_sel = src_sel[None]
    dev = tgt_c2w.device
    if tgt_c2w.dim() != 4:
        raise ValueError(f"tgt_c2w must be [B,Tq,4,4] or [Tq,4,4] (got {tuple(tgt_c2w.shape)})")
    B, Tq = tgt_c2w.shape[:2]
    _need(tgt_c2w, "tgt_c2w", torch.float32, (B, Tq, 4, 4), dev)
    _need(tgt_K, "tgt_K", torch.float32, (B, Tq, 4), dev)
    if src_sel is None:
        S = src_c2w.shape[1]
        _need(src_c2w, "src_c2w", torch.float32, (B, S, 4, 4), dev)
        _need(src_K, "src_K", torch.float32, (B, S, 4), dev)
        n_src = 0
    else:
        S = src_sel.shape[1]
        n_src = src_c2w.shape[0]
        _need(src_sel, "src_sel", torch.int32, (B, S), dev)
        _need(src_c2w, "src_c2w", torch.float32, (n_src, 4, 4), dev)
        _need(src_K, "src_K", torch.float32, (n_src, 4), dev)
    Lq = Tq * h * w
    if out is None:
        uv = torch.empty((B, S, Lq, 2), dtype=torch.float32, device=dev)
        idx = torch.empty((B, S, Lq), dtype=torch.int32, device=dev)
    else:
        uv, idx = out
        _need(uv, "out uv", torch.float32, (B, S, Lq, 2), dev)
        _need(idx, "out idx", torch.int32, (B, S, Lq), dev)
    st = lib().reproject_rotation(_ptr(tgt_c2w), _ptr(tgt_K), _ptr(src_c2w), _ptr(src_K), _ptr(src_sel), n_src,
                                  B, Tq, S, h, w, p, _ptr(uv), _ptr(idx), _stream(dev))
    _lib.check("reproject_rotation", st)
    if not batched:
        return uv[0], idx[0]
    return uv, idx


def biased_chunk_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, kv_frame_slot: torch.Tensor,
                           corr_uv: Optional[torch.Tensor], corr_idx: Optional[torch.Tensor], *,
                           h: int, w: int, softmax_scale: float, lam: float, sigma: float,
                           return_lse: bool = True, out=None, key_parts: int = 0,
                           workspace: Optional[torch.Tensor] = None, noalloc: bool = False):
    """Attention with the Gaussian correspondence bias on retrieved-frame keys.

    q [Lq,H,D], k, v [Lk,H,D] (bf16 with D=128, or fp32 with D in {64,128}, or
    q, k float8_e4m3fn with v bf16 and D=128: fp8 logits, o bf16);
    kv_frame_slot [Lk/(h*w)] i32; corr_uv [S,Lq,2] f32 and corr_idx [S,Lq] i32
    (None = no bias). key_parts: 0 = automatic key split, else a fixed
    number of parts (1..64). noalloc=True calls
    biased_chunk_attention_noalloc (the library's per-device scratch array
    instead of a workspace; with out= given nothing is allocated). Returns
    (o [Lq,H,D], lse [H,Lq] f32 or None)."""
    dev = q.device
    Lq, H, D = q.shape
    Lk = k.shape[0]
    dt = _attn_dtype(q.dtype)
    vdt = torch.bfloat16 if dt == FP8_QK else q.dtype  # fp8 q, k come with bf16 v, o
    _need(q, "q", q.dtype, None, dev)
    _need(k, "k", q.dtype, (Lk, H, D), dev)
    _need(v, "v", vdt, (Lk, H, D), dev)
    if Lk % (h * w):
        raise ValueError(f"Lk={Lk} is not a whole number of {h}x{w} frames")
    _need(kv_frame_slot, "kv_frame_slot", torch.int32, (Lk // (h * w),), dev)
    S = 0
    if corr_uv is not None:
        S = corr_uv.shape[0]
        _need(corr_uv, "corr_uv", torch.float32, (S, Lq, 2), dev)
        _need(corr_idx, "corr_idx", torch.int32, (S, Lq), dev)
    if out is None:
        o = torch.empty((Lq, H, D), dtype=vdt, device=dev)
        lse = torch.empty((H, Lq), dtype=torch.float32, device=dev) if return_lse else None
    else:
        o, lse = out
        _need(o, "o", vdt, (Lq, H, D), dev)
        if lse is not None:
            _need(lse, "lse", torch.float32, (H, Lq), dev)
    if noalloc:
        if workspace is not None:
            raise ValueError("noalloc=True takes no workspace (it uses the library's scratch array)")
        st = lib().biased_chunk_attention_noalloc(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), dt, Lq, Lk, H, D, h,
                                                  w, _ptr(kv_frame_slot), _ptr(corr_uv), _ptr(corr_idx), S,
                                                  softmax_scale, lam, sigma, int(key_parts), _stream(dev))
        _lib.check("biased_chunk_attention_noalloc", st)
        return o, lse
    if _current_device() == dev.index:
        nbytes = attention_workspace_size(q.dtype, Lq, Lk, H, D, key_parts)
    else:
        with torch.cuda.device(dev):
            nbytes = attention_workspace_size(q.dtype, Lq, Lk, H, D, key_parts)
    ws = _workspace(nbytes, workspace, dev, "workspace")
    st = lib().biased_chunk_attention(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), dt, Lq, Lk, H, D, h, w,
                                      _ptr(kv_frame_slot), _ptr(corr_uv), _ptr(corr_idx), S,
                                      softmax_scale, lam, sigma, int(key_parts), _ptr(ws),
                                      ws.numel() if ws is not None else 0, _stream(dev))
    _lib.check("biased_chunk_attention", st)
    return o, lse


def pack_retrieved_kv(store_k: torch.Tensor, store_v: torch.Tensor, sel: torch.Tensor,
                      cache_k: torch.Tensor, cache_v: torch.Tensor, *, F: int, h: int, w: int,
                      dst_pos: int, dst_row0: int, rope_t_pairs: int, rope_theta: float,
                      store_pos: Optional[torch.Tensor] = None) -> None:
    """Copy the selected chunks' keys and values into the cache slots, in place.

    store_k, store_v [L, n_store, F*h*w, H, D]; cache_k, cache_v [L, rows, H, D]
    (bf16 or fp32, D a multiple of 8); sel [n_sel] i32 (entries outside
    [0, n_store) leave their slot untouched); store_pos None or [n_store] i32.
    Slot s goes to cache rows dst_row0 + s*F*h*w and frame position
    dst_pos + s*F; the first rope_t_pairs pairs of each key are re-rotated."""
    dev = cache_k.device
    if store_k.dim() != 5 or cache_k.dim() != 4:
        raise ValueError("store_k must be [L, n_store, T, H, D] and cache_k [L, rows, H, D]")
    L, n_store, T, H, D = store_k.shape
    rows = cache_k.shape[1]
    if cache_k.dtype == torch.bfloat16:
        dt = BF16
    elif cache_k.dtype == torch.float32:
        dt = F32
    else:
        raise TypeError(f"cache_k must be bfloat16 or float32 (got {cache_k.dtype})")
    if T != F * h * w:
        raise ValueError(f"store rows per chunk {T} != F*h*w = {F * h * w}")
    _need(store_k, "store_k", cache_k.dtype, (L, n_store, T, H, D), dev)
    _need(store_v, "store_v", cache_k.dtype, (L, n_store, T, H, D), dev)
    _need(cache_k, "cache_k", cache_k.dtype, (L, rows, H, D), dev)
    _need(cache_v, "cache_v", cache_k.dtype, (L, rows, H, D), dev)
    _need(sel, "sel", torch.int32, None, dev)
    if store_pos is not None:
        _need(store_pos, "store_pos", torch.int32, (n_store,), dev)
    st = lib().pack_retrieved_kv(_ptr(store_k), _ptr(store_v), _ptr(store_pos), n_store, _ptr(sel), sel.numel(),
                                 int(dst_pos), _ptr(cache_k), _ptr(cache_v), int(dst_row0), rows, L, dt, F, h, w, H,
                                 D, int(rope_t_pairs), float(rope_theta), _stream(dev))
    _lib.check("pack_retrieved_kv", st)


def pool_token_depth(depth: torch.Tensor, p: int, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Token depth [n, h, w] f32 from depth maps [n, h*p, w*p] f32 (p x p means, fp32)."""
    dev = depth.device
    if depth.dim() != 3 or depth.shape[1] % p or depth.shape[2] % p:
        raise ValueError("depth must be [n, h*p, w*p]")
    n, Hd, Wd = depth.shape
    h, w = Hd // p, Wd // p
    _need(depth, "depth", torch.float32, (n, Hd, Wd), dev)
    if out is None:
        out = torch.empty((n, h, w), dtype=torch.float32, device=dev)
    _need(out, "out", torch.float32, (n, h, w), dev)
    _lib.check("pool_token_depth", lib().pool_token_depth(_ptr(depth), n, h, w, p, _ptr(out), _stream(dev)))
    return out


def _call(index: int, name: str, *args):
    """lib().<name>(*args, stream) on device `index` and its current stream, whichever device is current."""
    if _current_device() == index:
        st = getattr(_lib._LIB or lib(), name)(*args, _raw_stream(index))
    else:
        with torch.cuda.device(index):
            st = getattr(lib(), name)(*args, _raw_stream(index))
    if st:
        _lib.check(name.removesuffix("_strided"), st)


def _rows(t: torch.Tensor, name: str, dtype: torch.dtype, n: int, D: int, index: int):
    """A [n, H, D] tensor of whole rows (heads and elements contiguous, rows any distance apart); its H and row stride."""
    if isinstance(t, torch.Tensor) and t.dtype == dtype and t.get_device() == index:
        shape = t.shape
        if len(shape) == 3 and shape[0] == n and shape[2] == D:
            H = shape[1]
            if t.is_contiguous():
                return H, H * D
            row, head, one = t.stride()
            if (one == 1 or D == 1) and (head == D or H == 1):
                return H, row if n > 1 else H * D
            raise ValueError(f"{name}: a token's heads must be contiguous (strides {t.stride()})")
        raise ValueError(f"{name} has shape {tuple(shape)}, expected ({n}, heads, {D})")
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.get_device() != index:
        raise ValueError(f"{name} is on {t.device}, expected cuda:{index}")
    raise TypeError(f"{name} must be {dtype} (got {t.dtype})")


# types of rotary_embed by those of its input and output
_ROTARY_DTYPES = {(torch.bfloat16, torch.bfloat16): BF16, (torch.float32, torch.float32): F32,
                  (torch.bfloat16, torch.float8_e4m3fn): FP8_QK}


def rotary_embed(q: torch.Tensor, k: Optional[torch.Tensor] = None, *, pairs: Sequence[int], theta: float, h: int = 0,
                 w: int = 0, t0: int = 0, pos: Optional[torch.Tensor] = None, inverse: bool = False,
                 out_dtype: Optional[torch.dtype] = None, fp8_scale: Sequence[float] = (1.0, 1.0), out=None):
    """Rotary position embedding of q and k over time, row and column.

    q [n, Hq, D], k None or [n, Hk, D] (bf16 or fp32; rows may lie apart, as views
    of a packed projection do). pairs = (time, row, column) pairs of the bands.
    Token r stands at (t0 + r // (h*w), r // w % h, r % w), or at pos[r] with pos
    [n, 3] i32. inverse=True turns back, which is also the gradient with respect
    to q and k: no autograd graph is recorded. out_dtype: q's, or float8_e4m3fn for
    bf16 (values times fp8_scale = (q's, k's)). out = (q_out, k_out), which may be
    q and k themselves where the type stays; else no output may overlap an input
    or the other output. Returns (q_out, k_out); k_out is None without k."""
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise ValueError("q must be a tensor [n, heads, D]")
    dtype, index = q.dtype, q.get_device()
    n, _, D = q.shape
    q_out = k_out = None
    if out is not None:
        q_out, k_out = out
        if (k is None) != (k_out is None):
            raise ValueError("out k must be given exactly when k is")
    odt = out_dtype or (q_out.dtype if q_out is not None else dtype)
    dt = _ROTARY_DTYPES.get((dtype, odt))
    if dt is None:
        raise TypeError(f"q must be bfloat16 or float32 with outputs of the same type, or bfloat16 with float8_e4m3fn "
                        f"(got {dtype} and {odt})")
    if index < 0:
        raise ValueError(f"q must be a GPU tensor (got {q.device}); there is no CPU path")
    Hq, q_row = _rows(q, "q", dtype, n, D, index)
    if q_out is None:
        q_out = torch.empty((n, Hq, D), dtype=odt, device=q.device)
    Ho, qo_row = _rows(q_out, "out q", odt, n, D, index)
    if Ho != Hq:
        raise ValueError(f"out q has {Ho} heads, expected {Hq}")
    Hk = k_row = ko_row = 0
    if k is not None:
        Hk, k_row = _rows(k, "k", dtype, n, D, index)
        if k_out is None:
            k_out = torch.empty((n, Hk, D), dtype=odt, device=q.device)
        Ho, ko_row = _rows(k_out, "out k", odt, n, D, index)
        if Ho != Hk:
            raise ValueError(f"out k has {Ho} heads, expected {Hk}")
    if pos is not None:
        _need(pos, "pos", torch.int32, (n, 3), q.device)
    nt, ny, nx = pairs
    qs, ks = fp8_scale
    _call(index, "rotary_embed", q.data_ptr(), q_row, _ptr(k), k_row, q_out.data_ptr(), qo_row, _ptr(k_out), ko_row, dt, n, Hq, Hk, D,
          _ptr(pos), t0, h, w, nt, ny, nx, theta, 1 if inverse else 0, qs, ks)
    return q_out, k_out


def key_weight_workspace_size(dtype: torch.dtype, Lq: int, Lk: int, H: int, D: int, h: int, w: int, S: int = 0,
                              query_parts: int = 0) -> int:
    """Bytes of workspace attention_key_weight needs on the current device (S = 0 where lam is 0)."""
    n = ctypes.c_size_t(0)
    _lib.check("rc_key_weight_workspace_size",
               lib().rc_key_weight_workspace_size(_attn_dtype(dtype), Lq, Lk, H, D, h, w, S, query_parts, ctypes.byref(n)))
    return int(n.value)


def attention_key_weight(q: torch.Tensor, k: torch.Tensor, lse: torch.Tensor, kv_frame_slot: Optional[torch.Tensor],
                         corr_uv: Optional[torch.Tensor], corr_idx: Optional[torch.Tensor], *, h: int, w: int,
                         softmax_scale: float, lam: float, sigma: float, prev: Optional[torch.Tensor] = None,
                         decay: float = 1.0, query_parts: int = 0, out: Optional[torch.Tensor] = None,
                         workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Weight of every key in the attention: decay * prev + the sum over the
    queries of exp(logit - lse), with the logits of biased_chunk_attention.

    q [Lq,H,D], k [Lk,H,D], the slot table and correspondences as for
    biased_chunk_attention, lse [H,Lq] f32 as it returns; prev None or [H,Lk]
    f32. Queries whose lse is not finite add nothing. out may be prev. Returns
    the weights [H,Lk] f32."""
    dev = q.device
    Lq, H, D = q.shape
    Lk = k.shape[0]
    dt = _attn_dtype(q.dtype)
    _need(q, "q", q.dtype, None, dev)
    _need(k, "k", q.dtype, (Lk, H, D), dev)
    _need(lse, "lse", torch.float32, (H, Lq), dev)
    if h < 1 or w < 1 or Lk % (h * w):
        raise ValueError(f"Lk={Lk} is not a whole number of {h}x{w} frames")
    S = 0
    if corr_uv is not None:
        S = corr_uv.shape[0]
        _need(corr_uv, "corr_uv", torch.float32, (S, Lq, 2), dev)
        _need(corr_idx, "corr_idx", torch.int32, (S, Lq), dev)
        _need(kv_frame_slot, "kv_frame_slot", torch.int32, (Lk // (h * w),), dev)
    if prev is not None:
        _need(prev, "prev", torch.float32, (H, Lk), dev)
    if out is None:
        out = torch.empty((H, Lk), dtype=torch.float32, device=dev)
    else:
        _need(out, "out", torch.float32, (H, Lk), dev)
    if workspace is not None:
        _need(workspace, "workspace", torch.uint8, None, dev)
    elif query_parts > 1 or Lq >= 256:  # below, the automatic choice is one part, which needs none
        size = (q.dtype, Lq, Lk, H, D, h, w, S if lam != 0 else 0, query_parts)
        if _current_device() == dev.index:
            nbytes = key_weight_workspace_size(*size)
        else:
            with torch.cuda.device(dev):
                nbytes = key_weight_workspace_size(*size)
        if nbytes:
            workspace = torch.empty(nbytes, dtype=torch.uint8, device=dev)
    _call(dev.index, "attention_key_weight", _ptr(q), _ptr(k), _ptr(lse), dt, Lq, Lk, H, D, h, w, _ptr(kv_frame_slot), _ptr(corr_uv),
          _ptr(corr_idx), S, softmax_scale, lam, sigma, _ptr(prev), decay, _ptr(out), query_parts,
          _ptr(workspace), workspace.numel() if workspace is not None else 0)
    return out


def select_workspace_size(sets: int, heads: int, n_units: int, unit: int) -> int:
    """Bytes of workspace select_kept needs."""
    n = ctypes.c_size_t(0)
    _lib.check("rc_select_workspace_size", lib().rc_select_workspace_size(sets, heads, n_units, unit, ctypes.byref(n)))
    return int(n.value)


def select_kept(weight: torch.Tensor, *, unit: int, keep: int, first: int = 0, last: int = 0, return_score: bool = True,
                out=None, workspace: Optional[torch.Tensor] = None):
    """Which units of a cache stay, by accumulated weight.

    weight [sets, heads, n_units * unit] f32 (one set per choice: a layer with its
    heads, or a layer's head); the first `first` and last `last` units stay in
    any case, of the others those of largest summed weight, `keep` in all.
    Returns (idx [sets, keep] i32 ascending, score [sets, keep] f32 or None)."""
    if not isinstance(weight, torch.Tensor) or weight.dim() != 3:
        raise ValueError("weight must be a tensor [sets, heads, n_units * unit]")
    dev = weight.device
    sets, heads, cols = weight.shape
    _need(weight, "weight", torch.float32, None, dev)
    if unit < 1 or cols % unit:
        raise ValueError(f"{cols} weights are not a whole number of units of {unit}")
    if keep < 0:
        raise ValueError(f"keep={keep}")
    n_units = cols // unit
    if out is None:
        idx = torch.empty((sets, keep), dtype=torch.int32, device=dev)
        score = torch.empty((sets, keep), dtype=torch.float32, device=dev) if return_score else None
    else:
        idx, score = out
        _need(idx, "out idx", torch.int32, (sets, keep), dev)
        if score is not None:
            _need(score, "out score", torch.float32, (sets, keep), dev)
    if workspace is not None:
        _need(workspace, "workspace", torch.uint8, None, dev)
    elif heads > 1 or unit > 1 or cols > 1 << 10:  # few scores that are the weights themselves need none
        nbytes = select_workspace_size(sets, heads, n_units, unit)
        if nbytes:
            workspace = torch.empty(nbytes, dtype=torch.uint8, device=dev)
    _call(dev.index, "select_kept", weight.data_ptr(), sets, heads, n_units, unit, keep, first, last, idx.data_ptr(), _ptr(score),
          _ptr(workspace), workspace.numel() if workspace is not None else 0)
    return idx, score


def compact_kv(src_k: torch.Tensor, src_v: torch.Tensor, sel: torch.Tensor, dst_k: torch.Tensor, dst_v: torch.Tensor, *,
               unit: int, dst_row0: int = 0, weight: Optional[torch.Tensor] = None, out_weight: Optional[torch.Tensor] = None,
               src_pos: Optional[torch.Tensor] = None, dst_pos: int = 0, frames_per_unit: int = 0, rope_t_pairs: int = 0,
               rope_theta: float = 0.0) -> None:
    """Move the kept units of a cache into a smaller one, in place of dst's rows.

    src_k, src_v [L, rows, H, D], dst_k, dst_v [L, dst_rows, H, D] (bf16 or fp32,
    or fp8 keys with bf16 values); sel [L, 1 or H, keep] i32 units of `unit` rows
    (entries outside the source leave their rows as they are), going to rows
    dst_row0 + i*unit. No destination may overlap a source or another destination. weight [L, H, >= rows of the units] and out_weight [L, H, >=
    dst_row0 + keep*unit] f32 move alike. With rope_t_pairs > 0 keys are turned from
    their unit's frame position (src_pos [units] i32, else u*frames_per_unit) to
    dst_pos + i*frames_per_unit."""
    for t, name in ((src_k, "src_k"), (dst_k, "dst_k")):
        if not isinstance(t, torch.Tensor) or t.dim() != 4:
            raise ValueError(f"{name} must be a tensor [layers, rows, heads, D]")
    dev = dst_k.device
    L, rows, H, D = src_k.shape
    dst_rows = dst_k.shape[1]
    dt = _attn_dtype_of(src_k, "src_k")
    vdt = torch.bfloat16 if dt == FP8_QK else src_k.dtype
    _need(src_k, "src_k", src_k.dtype, None, dev)
    _need(src_v, "src_v", vdt, (L, rows, H, D), dev)
    _need(dst_k, "dst_k", src_k.dtype, (L, dst_rows, H, D), dev)
    _need(dst_v, "dst_v", vdt, (L, dst_rows, H, D), dev)
    _need(sel, "sel", torch.int32, None, dev)
    if sel.dim() != 3 or sel.shape[0] != L or sel.shape[1] not in (1, H):
        raise ValueError(f"sel has shape {tuple(sel.shape)}, expected ({L}, 1 or {H}, keep)")
    if unit < 1:
        raise ValueError(f"unit={unit}")
    n_units = rows // unit
    if src_pos is not None:
        _need(src_pos, "src_pos", torch.int32, None, dev)
        if src_pos.dim() != 1 or src_pos.shape[0] > n_units:
            raise ValueError(f"src_pos has shape {tuple(src_pos.shape)}, expected (units,), at most {n_units}")
        n_units = src_pos.shape[0]
    cols = dst_cols = 0
    if weight is not None or out_weight is not None:
        for t, name in ((weight, "weight"), (out_weight, "out_weight")):
            if t is None:
                raise ValueError("weight and out_weight are given together or not at all")
            _need(t, name, torch.float32, None, dev)
            if t.dim() != 3 or t.shape[0] != L or t.shape[1] != H:
                raise ValueError(f"{name} has shape {tuple(t.shape)}, expected ({L}, {H}, tokens)")
        cols, dst_cols = weight.shape[2], out_weight.shape[2]
        n_units = min(n_units, cols // unit)
    _call(dev.index, "compact_kv", _ptr(src_k), _ptr(src_v), rows, _ptr(sel), sel.shape[1], sel.shape[2], unit, n_units, _ptr(dst_k),
          _ptr(dst_v), dst_rows, dst_row0, _ptr(weight), cols, _ptr(out_weight), dst_cols, L, dt, H, D, _ptr(src_pos), dst_pos,
          frames_per_unit, rope_t_pairs, rope_theta)


# type of a paged cache by that of its pages, and the type of q, k, v and o beside it
_PAGED_DTYPES = {torch.bfloat16: (BF16, torch.bfloat16), torch.float32: (F32, torch.float32), torch.float8_e4m3fn: (FP8_KV, torch.bfloat16)}


def _pool(t, name, dtype, shape, dev):
    """Checks a pool of pages (or its scales), whose pages, heads and positions may be any distances apart; whether they lie
    one behind the other."""
    if not (isinstance(t, torch.Tensor) and t.dtype == dtype and t.shape == shape and t.get_device() == dev.index):
        _unfit(t, name, dtype, shape, dev, contiguous=False)
    if t.is_contiguous():
        return True
    if len(shape) == 4 and t.stride(3) != 1:
        raise ValueError(f"{name}: a position's elements must be contiguous (strides {t.stride()})")
    return False


def _pages(cache_k, cache_v, scale_k, scale_v, page_table, kv_len, cu, n, dev):
    """Checks a paged cache's tensors; (type, type of q, k, v and o, n_pages, H, page, D, B, max_pages, layout or None)."""
    if not isinstance(cache_k, torch.Tensor) or cache_k.dim() != 4:
        raise ValueError("cache_k must be a tensor [pages, heads, page, D]")
    dt, idt = _PAGED_DTYPES.get(cache_k.dtype, (None, None))
    if dt is None:
        raise TypeError(f"cache_k must be bfloat16, float32 or float8_e4m3fn (got {cache_k.dtype})")
    if not cache_k.is_cuda:
        raise ValueError(f"cache_k must be a GPU tensor (got {cache_k.device}); there is no CPU path")
    n_pages, H, page, D = shape = cache_k.shape
    whole = _pool(cache_k, "cache_k", cache_k.dtype, shape, dev)
    whole = _pool(cache_v, "cache_v", cache_k.dtype, shape, dev) and whole
    if dt == FP8_KV:
        shape = (n_pages, H, page // 32)
        whole = _pool(scale_k, "scale_k", torch.float8_e8m0fnu, shape, dev) and whole
        whole = _pool(scale_v, "scale_v", torch.float8_e8m0fnu, shape, dev) and whole
    elif scale_k is not None or scale_v is not None:
        raise ValueError("scale_k and scale_v belong to float8_e4m3fn pages")
    _need(page_table, "page_table", torch.int32, None, dev)
    if page_table.dim() != 2:
        raise ValueError(f"page_table has shape {tuple(page_table.shape)}, expected (streams, pages of a stream)")
    B, max_pages = page_table.shape
    _need(kv_len, "kv_len", torch.int32, (B,), dev)
    if cu is not None:
        _need(cu, "cu", torch.int32, (B + 1,), dev)
    elif n % B if B else n:
        raise ValueError(f"{n} tokens are not shared evenly by {B} streams: give cu")
    layout = None
    if not whole:
        layout = _lib.PoolLayout(*cache_k.stride()[:3], *cache_v.stride()[:3], *(scale_k.stride() + scale_v.stride() if dt == FP8_KV else ()))
    return dt, idt, n_pages, H, page, D, B, max_pages, layout


def append_paged_kv(k: torch.Tensor, v: torch.Tensor, cache_k: torch.Tensor, cache_v: torch.Tensor, page_table: torch.Tensor,
                    kv_len: torch.Tensor, *, pairs: Sequence[int], theta: float, cu: Optional[torch.Tensor] = None,
                    scale_k: Optional[torch.Tensor] = None, scale_v: Optional[torch.Tensor] = None, h: int = 0, w: int = 0, t0: int = 0,
                    pos: Optional[torch.Tensor] = None, out_len: Optional[torch.Tensor] = None) -> torch.Tensor:
    """New keys and values of many streams into the pages of their cache, in place.

    k, v [n, H, D] (rows may lie apart, as views of a packed projection do); cache_k,
    cache_v [pages, H, page, D] in the type of k and v (bf16, fp32), or
    float8_e4m3fn for bf16 k and v, with scale_k, scale_v [pages, H, page // 32]
    float8_e8m0fnu: a power of two for each 32 positions of a head. Pools and
    scales may be views (of [pages, page, H, D], of one tensor for keys and values):
    a position's D elements lie together, rows start on 16 bytes, and no two
    positions share memory. page_table [B, pages of a stream] i32, kv_len [B] i32 the positions that the streams hold.
    Stream s has tokens cu[s] .. cu[s+1]-1 of the n (cu [B+1] i32; None: n // B
    each); they go to its positions kv_len[s] on. Keys get the rotary position of
    rotary_embed (pairs, theta): position c stands at (t0 + c // (h*w), c // w % h,
    c % w), or a token at pos[i] with pos [n, 3] i32; pairs (0, 0, 0): keys as they are. Returns the new lengths [B]
    i32 (out_len, which must not be kv_len). No output may overlap an input; no
    autograd graph is recorded."""
    if not isinstance(k, torch.Tensor) or k.dim() != 3:
        raise ValueError("k must be a tensor [n, heads, D]")
    n = k.shape[0]
    dev = k.device
    dt, idt, n_pages, H, page, D, B, max_pages, layout = _pages(cache_k, cache_v, scale_k, scale_v, page_table, kv_len, cu, n, dev)
    Hk, k_row = _rows(k, "k", idt, n, D, dev.index)
    Hv, v_row = _rows(v, "v", idt, n, D, dev.index)
    if Hk != H or Hv != H:
        raise ValueError(f"k and v have {Hk} and {Hv} heads, expected {H}")
    if pos is not None:
        _need(pos, "pos", torch.int32, (n, 3), dev)
    if out_len is None:
        out_len = kv_len.new_empty((B,))
    else:
        _need(out_len, "out_len", torch.int32, (B,), dev)
    nt, ny, nx = pairs
    _call(dev.index, "append_paged_kv_strided", k.data_ptr(), k_row, v.data_ptr(), v_row, dt, n, _ptr(cu), B, kv_len.data_ptr(),
          out_len.data_ptr(), cache_k.data_ptr(), cache_v.data_ptr(), _ptr(scale_k), _ptr(scale_v), page_table.data_ptr(), n_pages, page,
          max_pages, H, D, _ptr(pos), t0, h, w, nt, ny, nx, theta, layout)
    return out_len


def paged_attention_workspace_size(dtype: torch.dtype, n: int, ragged: bool, B: int, Hq: int, Hk: int, D: int, page: int, max_pages: int,
                                   max_keys: int = 0, key_parts: int = 0) -> int:
    """Bytes of workspace paged_chunk_attention needs on the current device (dtype: of the pages; ragged: with cu)."""
    dt = _PAGED_DTYPES.get(dtype, (None,))[0]
    if dt is None:
        raise TypeError(f"pages must be bfloat16, float32 or float8_e4m3fn (got {dtype})")
    size = ctypes.c_size_t(0)
    st = (_lib._LIB or lib()).rc_paged_attention_workspace_size(dt, n, 1 if ragged else 0, B, Hq, Hk, D, page, max_pages, max_keys, key_parts,
                                                               ctypes.byref(size))
    if st:
        _lib.check("rc_paged_attention_workspace_size", st)
    return size.value


def paged_chunk_attention(q: torch.Tensor, cache_k: torch.Tensor, cache_v: torch.Tensor, page_table: torch.Tensor, kv_len: torch.Tensor, *,
                          softmax_scale: float, cu: Optional[torch.Tensor] = None, scale_k: Optional[torch.Tensor] = None,
                          scale_v: Optional[torch.Tensor] = None, visible: Optional[torch.Tensor] = None,
                          kv_frame_slot: Optional[torch.Tensor] = None, corr_uv: Optional[torch.Tensor] = None,
                          corr_idx: Optional[torch.Tensor] = None, h: int = 0, w: int = 0, lam: float = 0.0, sigma: float = 1.0,
                          max_keys: int = 0, key_parts: int = 0, return_lse: bool = True, out=None,
                          workspace: Optional[torch.Tensor] = None):
    """biased_chunk_attention over the pages of a cache, for the queries of many streams.

    q [n, Hq, D] (rows may lie apart), the pages, page_table, kv_len, cu and scales
    as for append_paged_kv; Hq is a multiple of the pages' heads. kv_len counts all
    keys of a stream, those appended for these queries included. visible None or
    [n] i32: the first keys of its stream that a query sees (causal: its own
    position + 1); a query without a key has o = 0 and lse = -inf. The bias, where
    corr_uv [S, n, 2] f32 and corr_idx [S, n] i32 are given: kv_frame_slot [B, frames]
    i32, position j of a stream being token j % (h*w) of its frame j // (h*w).
    max_keys: the longest stream's length if it is known, for the choice of the key
    split only. Returns (o [n, Hq, D], lse [Hq, n] f32 or None); rows behind the last
    stream's tokens are not written. Outputs must not overlap inputs; no autograd
    graph is recorded."""
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise ValueError("q must be a tensor [n, heads, D]")
    n, _, D = q.shape
    dev = q.device
    dt, idt, n_pages, Hk, page, Dk, B, max_pages, layout = _pages(cache_k, cache_v, scale_k, scale_v, page_table, kv_len, cu, n, dev)
    Hq, q_row = _rows(q, "q", idt, n, Dk, dev.index)
    if not Hk or Hq % Hk:
        raise ValueError(f"{Hq} query heads are not a multiple of {Hk} key heads")
    if visible is not None:
        _need(visible, "visible", torch.int32, (n,), dev)
    S = frames = 0
    if corr_uv is not None:
        S = corr_uv.shape[0] if isinstance(corr_uv, torch.Tensor) and corr_uv.dim() else -1
        _need(corr_uv, "corr_uv", torch.float32, (S, n, 2), dev)
        _need(corr_idx, "corr_idx", torch.int32, (S, n), dev)
        _need(kv_frame_slot, "kv_frame_slot", torch.int32, None, dev)
        if kv_frame_slot.dim() != 2 or kv_frame_slot.shape[0] != B:
            raise ValueError(f"kv_frame_slot has shape {tuple(kv_frame_slot.shape)}, expected ({B}, frames)")
        frames = kv_frame_slot.shape[1]
    elif corr_idx is not None or kv_frame_slot is not None:
        raise ValueError("corr_idx and kv_frame_slot belong to corr_uv")
    if out is None:
        o = q.new_empty((n, Hq, D))
        lse = q.new_empty((Hq, n), dtype=torch.float32) if return_lse else None
    else:
        o, lse = out
        _need(o, "o", idt, (n, Hq, D), dev)
        if lse is not None:
            _need(lse, "lse", torch.float32, (Hq, n), dev)
    if workspace is not None:
        _need(workspace, "workspace", torch.uint8, None, dev)
    else:
        size = (cache_k.dtype, n, cu is not None, B, Hq, Hk, D, page, max_pages, max_keys, key_parts)
        if _current_device() == dev.index:
            nbytes = paged_attention_workspace_size(*size)
        else:
            with torch.cuda.device(dev):
                nbytes = paged_attention_workspace_size(*size)
        if nbytes:
            workspace = q.new_empty(nbytes, dtype=torch.uint8)
    _call(dev.index, "paged_chunk_attention_strided", q.data_ptr(), q_row, cache_k.data_ptr(), cache_v.data_ptr(), _ptr(scale_k),
          _ptr(scale_v), o.data_ptr(), _ptr(lse), dt, n, _ptr(cu), B, kv_len.data_ptr(), _ptr(visible), page_table.data_ptr(), n_pages, page,
          max_pages, Hq, Hk, D, h, w, _ptr(kv_frame_slot), frames, _ptr(corr_uv), _ptr(corr_idx), S, softmax_scale, lam, sigma, max_keys,
          key_parts, _ptr(workspace), workspace.numel() if workspace is not None else 0, layout)
    return o, lse


class StreamDriver:
    """The paper's cache layout run chunk by chunk on the device (rc_stream_*).

    Owns a stream object: history ring of ``capacity`` chunks, pose bank of
    ``max_chunks``, packed cache. ``step`` runs the next chunk: depth
    [F, h*p, w*p] f32, c2w [F, 4, 4] f32, K [F, 4] f32, q, k, v
    [layers, F*h*w, H, D] (bf16 or f32, k embedded at positions 4F + f);
    returns o [layers, F*h*w, H, D] and lse [layers, H, F*h*w]."""

    def __init__(self, *, F: int, h: int, w: int, p: int, H: int, D: int, layers: int, dtype: torch.dtype,
                 capacity: int, max_chunks: int, E: float, w_v: float, tau_c: float, tau_v: float, delta: int,
                 eps: float, lam: float, sigma: float, softmax_scale: float, rope_t_pairs: int, rope_theta: float):
        if dtype == torch.bfloat16:
            dt = BF16
        elif dtype == torch.float32:
            dt = F32
        else:
            raise TypeError(f"dtype must be bfloat16 or float32 (got {dtype})")
        self.dtype = dtype
        self.F, self.h, self.w, self.p, self.H, self.D, self.layers = F, h, w, p, H, D, layers
        cfg = _lib.StreamConfig(F=F, h=h, w=w, p=p, H=H, D=D, layers=layers, dtype=dt, capacity=capacity,
                                max_chunks=max_chunks, E=E, w_v=w_v, tau_c=tau_c, tau_v=tau_v, delta=delta, eps=eps,
                                lam=lam, sigma=sigma, softmax_scale=softmax_scale, rope_t_pairs=rope_t_pairs,
                                rope_theta=rope_theta)
        handle = ctypes.c_void_p(0)
        _lib.check("rc_stream_create", lib().rc_stream_create(ctypes.byref(cfg), ctypes.byref(handle)))
        self._h = handle

    def step(self, depth, c2w, K, q, k, v, out=None):
        if not self._h:
            raise RuntimeError("stream already closed")
        dev = q.device
        T = self.F * self.h * self.w
        _need(depth, "depth", torch.float32, (self.F, self.h * self.p, self.w * self.p), dev)
        _need(c2w, "c2w", torch.float32, (self.F, 4, 4), dev)
        _need(K, "K", torch.float32, (self.F, 4), dev)
        shape = (self.layers, T, self.H, self.D)
        for t, name in ((q, "q"), (k, "k"), (v, "v")):
            _need(t, name, self.dtype, shape, dev)
        if out is None:
            o = torch.empty(shape, dtype=self.dtype, device=dev)
            lse = torch.empty((self.layers, self.H, T), dtype=torch.float32, device=dev)
        else:
            o, lse = out
            _need(o, "o", self.dtype, shape, dev)
            if lse is not None:
                _need(lse, "lse", torch.float32, (self.layers, self.H, T), dev)
        st = lib().rc_stream_step(self._h, _ptr(depth), _ptr(c2w), _ptr(K), _ptr(q), _ptr(k), _ptr(v), _ptr(o),
                                  _ptr(lse), _stream(dev))
        _lib.check("rc_stream_step", st)
        return o, lse

    def state(self):
        """The last step's layout sizes and device pointers (rc_stream_state)."""
        stt = _lib.StreamState()
        _lib.check("rc_stream_view", lib().rc_stream_view(self._h, ctypes.byref(stt)))
        return stt

    def close(self):
        if self._h:
            lib().rc_stream_destroy(self._h)
            self._h = ctypes.c_void_p(0)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
