"""AViTS resolution-transition hot path for GB300 (sm_103a).

A thin ctypes binding over ``libavits.so`` (include/avits.h).  Each function
has the name of its C entry point and only marshals arguments: torch tensors
become device pointers, the current torch stream becomes the cudaStream_t, a
non-OK status becomes an ``AvitsError``.  Every step of the path runs in the
library's CUDA kernels; there is no CPU fallback, and importing the functions
fails loudly when the library has not been built (``build()``).

Calls:
  avits_score_spatial       Eq. 3-5  text attention mass per image token
                            (text_mask=: interleaved text keys)
  avits_score_spatial_lse   Eq. 5  from the model attention's logsumexp over
                            all keys and the text keys only
  avits_score_temporal      Sec. 3.3.2  relative step change per token
  avits_score_spatiotemporal  both scores in one call
  avits_score_temporal_var  Eq. 6-7  step variance over N_T snapshots
  avits_fuse_select         Eq. 8-9  min-max fuse + deterministic top-k
                            (perturb=: caller's tie-break noise)
  avits_selective_upsample  Sec. 3.2 Stage 2  packed mixed-resolution sequence
  avits_select_upsample     selection + upsample in one launch
  avits_merge_final         Sec. 3.2 Stage 3  dense full-resolution latent
  avits_cache_append        new tokens into a paged key-value cache (KVCache)
  avits_cache_attention     one new token per sequence over its cached tokens,
                            with the weight each of them got
  avits_cache_evict         the cached tokens of the largest accumulated weights
  avits_device_status       device-side error word (read and cleared)
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Optional, Sequence

from . import _build

__all__ = [
    "AvitsError", "build", "lib", "library_path",
    "avits_score_spatial", "avits_score_spatial_workspace", "avits_score_spatial_lse",
    "avits_score_temporal",
    "avits_score_spatiotemporal",
    "avits_score_spatial_noalloc", "avits_score_spatial_noalloc_limit",
    "avits_score_temporal_var", "avits_fuse_select",
    "avits_selective_upsample", "avits_select_upsample",
    "avits_merge_final", "avits_merge_final_workspace", "avits_device_status",
    "KVCache", "avits_cache_append", "avits_cache_attention", "avits_cache_attention_workspace",
    "avits_cache_evict",
    "avits_selftest_bounded_wait", "avits_status_string", "avits_version", "SpatialWorkspace",
]

F32, BF16 = 0, 1
NEAREST, BILINEAR = 0, 1
STATUS = {0: "ok", 1: "invalid argument", 2: "unsupported", 3: "CUDA error",
          4: "device wait timed out", 5: "NaN in fused score", 6: "coverage",
          7: "cache length or page number out of range"}

_lib = None


class AvitsError(RuntimeError):
    def __init__(self, fn: str, code: int, detail: str = ""):
        self.code = code
        super().__init__("%s failed: %s%s" % (fn, STATUS.get(code, code),
                                               (" (" + detail + ")") if detail else ""))


def library_path() -> str:
    return _build.LIB


def build(force: bool = False) -> str:
    """Compile libavits.so for sm_103a (in-tree)."""
    return _build.build(force=force)


def lib():
    """Load libavits.so; raise if it is missing (no fallback path exists)."""
    global _lib
    if _lib is not None:
        return _lib
    path = _build.LIB
    if not os.path.exists(path):
        raise RuntimeError("libavits.so is not built (%s); run paper_2608_17995_gb300.build()" % path)
    L = ctypes.CDLL(path)
    vp, i32, i64, f32, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
    sig = {
        "avits_score_spatial": [vp, vp, i32, i32, i32, i32, i32, i32, i32, i64, i64, i64, i64, i64,
                                i64, f32, f32, i32, vp, vp, vp, sz, vp],
        "avits_score_spatial_workspace": [i32, i32, i32, i32, i32, i32],
        "avits_score_spatial_keymask": [vp, vp, i32, i32, i32, i32, i32, i32, i64, i64, i64, i64,
                                        i64, i64, vp, f32, f32, i32, vp, vp, vp, sz, vp],
        "avits_score_spatial_lse": [vp, vp, i32, i32, i32, i32, i32, i32, i64, i64, i64, i64,
                                    i64, i64, vp, f32, f32, i32, vp, vp, vp, sz, vp],
        "avits_score_temporal": [vp, vp, i32, i32, i32, i32, f32, vp, vp],
        "avits_attention_forward": [vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, vp, vp, vp, vp,
                                    f32, vp, vp, f32, i32, vp, vp, sz, vp],
        "avits_attention_forward_workspace": [i32, i32, i32],
        "avits_score_spatiotemporal": [vp, vp, i32, i32, i32, i32, i32, i32, i32, i64, i64, i64,
                                       i64, i64, i64, f32, f32, i32, vp, vp, vp, sz, vp, vp, i32,
                                       f32, vp, vp],
        "avits_score_temporal_var": [vp, i32, i32, i32, i32, i32, vp, vp],
        "avits_fuse_select": [vp, vp, i32, i32, f32, f32, i32, vp, vp, vp, vp, vp],
        "avits_fuse_select_perturbed": [vp, vp, vp, i32, i32, f32, f32, i32, vp, vp, vp, vp, vp],
        "avits_selective_upsample": [vp, i32, i32, i32, i32, i32, i32, i32, vp, vp, vp, vp, i32,
                                     i32, vp, vp, vp, vp, vp, vp, sz, vp],
        "avits_selective_upsample_workspace": [i32, i32, i32, i32],
        "avits_select_upsample": [vp, vp, vp, i32, i32, f32, f32, i32, vp, vp, vp, vp, vp, i32,
                                  i32, i32, i32, i32, vp, vp, i32, vp, vp, vp, vp, vp, vp, sz,
                                  vp],
        "avits_merge_final": [vp, i32, i32, i32, vp, vp, i32, i32, i32, i32, i32, vp, vp, sz, vp],
        "avits_merge_final_workspace": [i32, i32, i32, i32],
        "avits_score_spatial_noalloc": [vp, vp, i32, i32, i32, i32, i32, i32, i32, i64, i64, i64,
                                        i64, i64, i64, f32, f32, i32, vp, vp, vp],
        "avits_score_spatial_noalloc_limit": [],
        "avits_score_spatial_noalloc_error": [],
        "avits_cache_append": [vp, vp, vp, i32, vp, i64, i64, i64, i64, vp],
        "avits_cache_attention": [vp, vp, i32, i64, i64, f32, vp, i64, i64, vp, i32, f32, vp, sz,
                                  vp],
        "avits_cache_attention_workspace": [vp, i32, i32],
        "avits_cache_evict": [vp, vp, i32, i32, i32, vp, vp],
        "avits_device_status": [vp],
        "avits_selftest_bounded_wait": [ctypes.c_ulonglong, vp, vp],
        "avits_status_string": [i32],
        "avits_last_error_string": [],
        "avits_version": [],
    }
    for name, args in sig.items():
        fn = getattr(L, name)
        fn.argtypes = args
        fn.restype = ctypes.c_int
    for name in ("avits_score_spatial_workspace", "avits_merge_final_workspace",
                 "avits_score_spatial_noalloc_limit", "avits_attention_forward_workspace",
                 "avits_selective_upsample_workspace", "avits_cache_attention_workspace"):
        getattr(L, name).restype = ctypes.c_size_t
    for name in ("avits_status_string", "avits_last_error_string", "avits_version",
                 "avits_score_spatial_noalloc_error"):
        getattr(L, name).restype = ctypes.c_char_p
    _lib = L
    return L


# ------------------------------------------------------------- marshalling --
# A call's host time is mostly here, so the helpers stay lean: a lookup of the
# current stream as an object took 2.9 us (its raw handle 0.2), a size query
# through ctypes 1.0, and an attention call 20.8 us in all, 4.5 of them in the
# library.
_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


_Int64x3 = ctypes.c_int64 * 3


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if not t.is_cuda:
        raise ValueError("device tensor expected, got a %s tensor" % t.device)
    return t.data_ptr()


def _stream(stream) -> Optional[int]:
    """The stream's handle; None: the current stream of the current device."""
    if stream is None:
        torch = _torch()
        if not torch.cuda.is_initialized():
            return torch.cuda.current_stream().cuda_stream
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _dtype_code(t) -> int:
    torch = _torch()
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    raise TypeError("bfloat16 or float32 expected, got %s" % t.dtype)


def _check(fn: str, rc: int):
    if rc != 0:
        detail = lib().avits_last_error_string().decode() if rc == 3 else ""
        raise AvitsError(fn, rc, detail)


def avits_version() -> str:
    return lib().avits_version().decode()


def avits_status_string(code: int) -> str:
    return lib().avits_status_string(code).decode()


def avits_device_status(stream=None) -> int:
    """Synchronise the stream; return and clear the device error code (0 = ok)."""
    return lib().avits_device_status(_stream(stream))


def avits_selftest_bounded_wait(limit_ns: int, result, stream=None):
    """Run the bounded-wait failure path on barriers nothing arrives at (a
    test hook): result (cuda int64[5]) receives completion flags and wait
    times of the timing-out warp and of the warp the abort flag releases."""
    _check("avits_selftest_bounded_wait",
           lib().avits_selftest_bounded_wait(int(limit_ns), _ptr(result), _stream(stream)))


def avits_score_spatial_workspace(dtype, B, H, M, Nk, d) -> int:
    code = dtype if isinstance(dtype, int) else _dtype_code(_torch().empty(0, dtype=dtype))
    return int(lib().avits_score_spatial_workspace(code, B, H, M, Nk, d))


@functools.lru_cache(maxsize=256)
def _spatial_need(device: int, code: int, B: int, H: int, M: int, Nk: int, d: int) -> int:
    """The same by sizes and device (the query depends on nothing else)."""
    return int(lib().avits_score_spatial_workspace(code, B, H, M, Nk, d))


def _spatial_ws(code, q_img, B, H, M, Nk, d, workspace, stream):
    """Buffer and bytes for a spatial score on the current device."""
    need = _spatial_need(_torch().cuda.current_device(), code, B, H, M, Nk, d)
    if workspace is None:
        key = (q_img.device.index, stream)
        workspace = _default_ws.get(key)
        if workspace is None:
            workspace = _default_ws.setdefault(key, SpatialWorkspace(q_img.device))
    return workspace.get(need)


class SpatialWorkspace:
    """Device scratch for avits_score_spatial, grown on demand (reused by
    calls on one stream).  Allocated zero-filled: the counters at its start
    must be zero before a call, and every completed call leaves them zero;
    after a call that reported a device timeout, call reset()."""

    def __init__(self, device=None):
        self.buf = None
        self.device = device

    def get(self, nbytes: int):
        torch = _torch()
        if nbytes == 0:
            return None, 0
        if self.buf is None or self.buf.numel() < nbytes:
            self.buf = torch.zeros(nbytes, dtype=torch.uint8, device=self.device or "cuda")
        return self.buf, self.buf.numel()

    def reset(self):
        if self.buf is not None:
            self.buf.zero_()


_default_ws = {}


def avits_score_spatial(q_img, k_all, L: int, softmax_scale: float, A, weight: float = 1.0,
                        accumulate: bool = False, lse=None, workspace: Optional[SpatialWorkspace] = None,
                        stream=None, text_mask=None):
    """Eq. 3-5.  q_img [B,H,M,d] (any strides, d contiguous), k_all [B,H,Nk,d]
    with the L text keys first; A [B,M] fp32 written (or accumulated).  With
    ``text_mask`` ([B,Nk] uint8 / bool on the device, nonzero = text key) the
    text keys are the masked ones instead (avits_score_spatial_keymask; L is
    ignored)."""
    B, H, M, d = q_img.shape
    Nk = k_all.shape[2]
    if k_all.shape[0] != B or k_all.shape[1] != H or k_all.shape[3] != d:
        raise ValueError("q_img / k_all shapes disagree")
    qs, ks = q_img.stride(), k_all.stride()
    if qs[3] != 1 or ks[3] != 1:
        raise ValueError("the head-dim axis must be contiguous")
    dt = _dtype_code(q_img)
    if _dtype_code(k_all) != dt:
        raise TypeError("q_img and k_all dtypes differ")
    stream = _stream(stream)
    wbuf, wbytes = _spatial_ws(dt, q_img, B, H, M, Nk, d, workspace, stream)
    if text_mask is not None:
        if tuple(text_mask.shape) != (B, Nk) or text_mask.element_size() != 1 or \
                not text_mask.is_contiguous():
            raise ValueError("text_mask must be a contiguous [B,Nk] byte tensor")
        rc = lib().avits_score_spatial_keymask(
            _ptr(q_img), _ptr(k_all), dt, B, H, M, Nk, d, qs[0], qs[1], qs[2], ks[0], ks[1],
            ks[2], _ptr(text_mask), float(softmax_scale), float(weight), 1 if accumulate else 0,
            _ptr(A), _ptr(lse), _ptr(wbuf), wbytes, stream)
        _check("avits_score_spatial_keymask", rc)
        return A
    rc = lib().avits_score_spatial(
        _ptr(q_img), _ptr(k_all), dt, B, H, M, Nk, L, d, qs[0], qs[1], qs[2], ks[0], ks[1], ks[2],
        float(softmax_scale), float(weight), 1 if accumulate else 0,
        _ptr(A), _ptr(lse), _ptr(wbuf), wbytes, stream)
    _check("avits_score_spatial", rc)
    return A


def avits_score_spatial_lse(q_img, k_txt, lse_all, softmax_scale: float, A, weight: float = 1.0,
                            accumulate: bool = False, lse=None,
                            workspace: Optional[SpatialWorkspace] = None, stream=None):
    """Eq. 5 from the caller's logsumexp over all keys: q_img [B,H,M,d],
    k_txt [B,H,L,d] (the text keys only, any strides with d contiguous),
    lse_all [B,H,M] fp32 contiguous (natural log, e.g. from the model's
    attention forward); A [B,M] written (or accumulated)."""
    B, H, M, d = q_img.shape
    L = k_txt.shape[2]
    if k_txt.shape[0] != B or k_txt.shape[1] != H or k_txt.shape[3] != d:
        raise ValueError("q_img / k_txt shapes disagree")
    qs, ks = q_img.stride(), k_txt.stride()
    if qs[3] != 1 or ks[3] != 1:
        raise ValueError("the head-dim axis must be contiguous")
    if tuple(lse_all.shape) != (B, H, M) or not lse_all.is_contiguous():
        raise ValueError("lse_all must be a contiguous [B,H,M] tensor")
    dt = _dtype_code(q_img)
    if _dtype_code(k_txt) != dt:
        raise TypeError("q_img and k_txt dtypes differ")
    stream = _stream(stream)
    wbuf, wbytes = _spatial_ws(dt, q_img, B, H, M, L, d, workspace, stream)
    rc = lib().avits_score_spatial_lse(
        _ptr(q_img), _ptr(k_txt), dt, B, H, M, L, d, qs[0], qs[1], qs[2], ks[0], ks[1], ks[2],
        _ptr(lse_all), float(softmax_scale), float(weight), 1 if accumulate else 0,
        _ptr(A), _ptr(lse), _ptr(wbuf), wbytes, stream)
    _check("avits_score_spatial_lse", rc)
    return A


def avits_score_spatiotemporal(q_img, k_all, L: int, softmax_scale: float, A, h_t, h_prev, V,
                               weight: float = 1.0, accumulate: bool = False, lse=None,
                               eps: float = 1e-6, workspace: Optional[SpatialWorkspace] = None,
                               stream=None):
    """avits_score_spatial + avits_score_temporal in one call (the temporal
    kernel overlaps the spatial one on the tensor-core path)."""
    B, H, M, d = q_img.shape
    Nk = k_all.shape[2]
    D = h_t.shape[2]
    qs, ks = q_img.stride(), k_all.stride()
    if qs[3] != 1 or ks[3] != 1:
        raise ValueError("the head-dim axis must be contiguous")
    if not (h_t.is_contiguous() and h_prev.is_contiguous()) or tuple(h_t.shape[:2]) != (B, M):
        raise ValueError("h_t / h_prev must be contiguous [B, M, D]")
    dt = _dtype_code(q_img)
    stream = _stream(stream)
    wbuf, wbytes = _spatial_ws(dt, q_img, B, H, M, Nk, d, workspace, stream)
    rc = lib().avits_score_spatiotemporal(
        _ptr(q_img), _ptr(k_all), dt, B, H, M, Nk, L, d, qs[0], qs[1], qs[2], ks[0], ks[1], ks[2],
        float(softmax_scale), float(weight), 1 if accumulate else 0,
        _ptr(A), _ptr(lse), _ptr(wbuf), wbytes, _ptr(h_t), _ptr(h_prev), D, float(eps), _ptr(V),
        stream)
    _check("avits_score_spatiotemporal", rc)
    return A, V


def avits_attention_forward_workspace(B: int, H: int, Mq: int) -> int:
    return int(lib().avits_attention_forward_workspace(B, H, Mq))


@functools.lru_cache(maxsize=256)
def _attention_need(B: int, H: int, Mq: int) -> int:
    return avits_attention_forward_workspace(B, H, Mq)


def avits_attention_forward(q, k, v, L: int, softmax_scale: float, o, lse=None, A=None,
                            weight: float = 1.0, accumulate: bool = False,
                            workspace: Optional[SpatialWorkspace] = None, stream=None):
    """Eq. 4-5 + Eq. 3: the joint-attention forward O = softmax(scale Q K^T) V
    of a double-stream block (q [B,H,Mq,d], k / v [B,H,Nk,d], bf16, any
    strides with d contiguous, the L text keys first) into o [B,H,Mq,d]
    bf16, with lse [B,H,Mq,2] (all keys, text keys) and the spatial score A
    [B,Mq] (written or accumulated) when given."""
    B, H, Mq, d = q.shape
    Nk = k.shape[2]
    if tuple(k.shape) != (B, H, Nk, d) or tuple(v.shape) != (B, H, Nk, d) or \
            tuple(o.shape) != (B, H, Mq, d):
        raise ValueError("q / k / v / o shapes disagree")
    strides = (q.stride(), k.stride(), v.stride(), o.stride())
    for t in strides:
        if t[3] != 1:
            raise ValueError("the head-dim axis must be contiguous")
    dt = _dtype_code(q)
    if _dtype_code(k) != dt or _dtype_code(v) != dt or _dtype_code(o) != dt:
        raise TypeError("q, k, v and o dtypes differ")
    wbuf, wbytes = None, 0
    stream = _stream(stream)
    if A is not None:
        if workspace is None:
            key = ("attn", q.device.index, stream)
            workspace = _default_ws.setdefault(key, SpatialWorkspace(q.device))
        wbuf, wbytes = workspace.get(_attention_need(B, H, Mq))
    qs, ks, vs, os_ = (_Int64x3(t[0], t[1], t[2]) for t in strides)
    rc = lib().avits_attention_forward(
        _ptr(q), _ptr(k), _ptr(v), dt, B, H, Mq, Nk, L, d, qs, ks, vs, os_,
        float(softmax_scale), _ptr(o), _ptr(lse), float(weight), 1 if accumulate else 0,
        _ptr(A), _ptr(wbuf), wbytes, stream)
    _check("avits_attention_forward", rc)
    return o


def avits_score_temporal(h_t, h_prev, V, eps: float = 1e-6, stream=None):
    B, N, D = h_t.shape
    if not (h_t.is_contiguous() and h_prev.is_contiguous()):
        raise ValueError("h_t and h_prev must be contiguous")
    rc = lib().avits_score_temporal(_ptr(h_t), _ptr(h_prev), _dtype_code(h_t), B, N, D,
                                    float(eps), _ptr(V), _stream(stream))
    _check("avits_score_temporal", rc)
    return V


def avits_score_temporal_var(snaps: Sequence, V, stream=None):
    B, N, D = snaps[0].shape
    arr = (ctypes.c_void_p * len(snaps))(*[_ptr(s) for s in snaps])
    rc = lib().avits_score_temporal_var(arr, len(snaps), _dtype_code(snaps[0]), B, N, D, _ptr(V),
                                        _stream(stream))
    _check("avits_score_temporal_var", rc)
    return V


def avits_fuse_select(A, V, alpha: float, k: int, sel_idx, tok_offset, S=None, sel_mask=None,
                      eps_norm: float = 1e-6, stream=None, perturb=None):
    """Eq. 8-9; ``perturb`` ([B,M] fp32, optional): the caller's tie-breaking
    noise, added to S before the selection (avits_fuse_select_perturbed)."""
    B, M = A.shape
    if perturb is None:
        rc = lib().avits_fuse_select(_ptr(A), _ptr(V), B, M, float(alpha), float(eps_norm),
                                     int(k), _ptr(S), _ptr(sel_idx), _ptr(sel_mask),
                                     _ptr(tok_offset), _stream(stream))
        _check("avits_fuse_select", rc)
    else:
        if tuple(perturb.shape) != (B, M):
            raise ValueError("perturb must be [B,M]")
        rc = lib().avits_fuse_select_perturbed(_ptr(A), _ptr(V), _ptr(perturb), B, M,
                                               float(alpha), float(eps_norm), int(k), _ptr(S),
                                               _ptr(sel_idx), _ptr(sel_mask), _ptr(tok_offset),
                                               _stream(stream))
        _check("avits_fuse_select_perturbed", rc)
    return sel_idx


def avits_selective_upsample_workspace(mode: int, B: int, grid_h: int, grid_w: int) -> int:
    return int(lib().avits_selective_upsample_workspace(int(mode), B, grid_h, grid_w))


def _upsample_ws(mode, pos_in, B, grid_h, grid_w, workspace, device):
    """The cell-map workspace a mixed bilinear upsample needs (else none)."""
    if mode != BILINEAR or pos_in is None:
        return None, 0
    need = avits_selective_upsample_workspace(mode, B, grid_h, grid_w)
    if workspace is None:
        workspace = _torch().empty(need, dtype=_torch().uint8, device=device)
    return workspace, workspace.numel() * workspace.element_size()


def avits_select_upsample(A, V, alpha: float, k: int, sel_idx, tok_offset, sel_mask, latent,
                          grid_h: int, grid_w: int, out_latent, out_pos, out_span, out_src_tok,
                          out_src_sub, S=None, perturb=None, mode: int = NEAREST, pos_in=None,
                          span_in=None, eps_norm: float = 1e-6, workspace=None, stream=None):
    """avits_fuse_select(_perturbed) + avits_selective_upsample in one launch;
    the same outputs as the two calls."""
    B, M = A.shape
    T = latent.shape[2]
    ws, wb = _upsample_ws(mode, pos_in, B, grid_h, grid_w, workspace, latent.device)
    rc = lib().avits_select_upsample(
        _ptr(A), _ptr(V), _ptr(perturb), B, M, float(alpha), float(eps_norm), int(k), _ptr(S),
        _ptr(sel_idx), _ptr(sel_mask), _ptr(tok_offset), _ptr(latent), _dtype_code(latent),
        grid_h, grid_w, T // 4, 2, _ptr(pos_in), _ptr(span_in), int(mode), _ptr(out_latent),
        _ptr(out_pos), _ptr(out_span), _ptr(out_src_tok), _ptr(out_src_sub), _ptr(ws), wb,
        _stream(stream))
    _check("avits_select_upsample", rc)
    return sel_idx


def avits_selective_upsample(latent, grid_h: int, grid_w: int, sel_mask, tok_offset, k: int,
                             out_latent, out_pos, out_span, out_src_tok, out_src_sub,
                             mode: int = NEAREST, pos_in=None, span_in=None, workspace=None,
                             stream=None):
    """Sec. 3.2 Stage 2.  A mixed bilinear input (pos_in given) needs
    avits_selective_upsample_workspace() bytes of scratch (allocated here when
    ``workspace`` is None)."""
    B, M, T = latent.shape
    ws, wb = _upsample_ws(mode, pos_in, B, grid_h, grid_w, workspace, latent.device)
    rc = lib().avits_selective_upsample(
        _ptr(latent), _dtype_code(latent), B, M, grid_h, grid_w, T // 4, 2, _ptr(pos_in),
        _ptr(span_in), _ptr(sel_mask), _ptr(tok_offset), int(k), int(mode), _ptr(out_latent),
        _ptr(out_pos), _ptr(out_span), _ptr(out_src_tok), _ptr(out_src_sub), _ptr(ws), wb,
        _stream(stream))
    _check("avits_selective_upsample", rc)
    return out_latent


def avits_merge_final_workspace(mode: int, B: int, full_h: int, full_w: int) -> int:
    return int(lib().avits_merge_final_workspace(int(mode), B, full_h, full_w))


def avits_merge_final(mixed, pos, span, full_h: int, full_w: int, out_full, mode: int = NEAREST,
                      workspace=None, stream=None):
    B, N, T = mixed.shape
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib().avits_merge_final(_ptr(mixed), _dtype_code(mixed), B, N, _ptr(pos), _ptr(span),
                                 full_h, full_w, T // 4, 2, int(mode), _ptr(out_full),
                                 _ptr(workspace), ws_bytes, _stream(stream))
    _check("avits_merge_final", rc)
    return out_full


def avits_score_spatial_noalloc(q_img, k_all, L: int, softmax_scale: float, A, weight: float = 1.0,
                                accumulate: bool = False, lse=None, stream=None):
    """avits_score_spatial without a workspace: the library's fixed device
    scratch is used instead (for callers that cannot allocate where they call
    this, e.g. inside an engine plugin's enqueue).  Same arguments otherwise;
    bf16 tensor-core shapes only.  Calls on one device must not overlap."""
    L_ = lib()
    fn = L_.avits_score_spatial_noalloc
    B, H, M, d = q_img.shape
    Nk = k_all.shape[2]
    rc = fn(_ptr(q_img), _ptr(k_all), _dtype_code(q_img), B, H, M, Nk, L, d,
            q_img.stride(0), q_img.stride(1), q_img.stride(2),
            k_all.stride(0), k_all.stride(1), k_all.stride(2),
            float(softmax_scale), float(weight), 1 if accumulate else 0,
            _ptr(A), _ptr(lse), _stream(stream))
    if rc != 0:
        err = L_.avits_score_spatial_noalloc_error()
        raise AvitsError("avits_score_spatial_noalloc", rc,
                         err.decode() if isinstance(err, bytes) else "")
    return A


def avits_score_spatial_noalloc_limit() -> int:
    """Bytes of the fixed scratch array behind avits_score_spatial_noalloc."""
    return int(lib().avits_score_spatial_noalloc_limit())


# ------------------------------------------------- paged key-value cache --
_INT_MAX = 2 ** 31 - 1       # ctypes passes the low 32 bits of what is larger


class _CacheStruct(ctypes.Structure):
    _fields_ = [("k_pages", ctypes.c_void_p), ("v_pages", ctypes.c_void_p),
                ("block_table", ctypes.c_void_p), ("lens", ctypes.c_void_p),
                ("acc", ctypes.c_void_p)] + \
               [(n, ctypes.c_int64) for n in ("k_sp", "k_st", "k_sh", "v_sp", "v_st", "v_sh",
                                              "table_sb", "acc_sb", "acc_sh")] + \
               [(n, ctypes.c_int32) for n in ("dt", "B", "Hkv", "d", "num_pages", "page_size",
                                              "max_len")]


class KVCache:
    """The buffers of a paged key-value cache, described to the library once
    and used by any number of calls (which read the tensors' current contents).

    k_pages, v_pages  [num_pages, page_size, Hkv, d] bf16 or fp32, any strides
                      with d contiguous (pages may lie in memory head by head,
                      or keys and values side by side: pass the view)
    block_table       [B, columns] int32, a sequence's pages in order
    lens              [B] int32, its cached tokens
    acc               [B, Hkv, >= max_len] fp32, optional: accumulated weights
    max_len           an upper bound of lens known here (default: all that the
                      table can hold); a smaller one costs less workspace and,
                      where weights are wanted or tokens evicted, less time

    The description is fixed: other tensors are another KVCache.
    """
    __slots__ = ("k_pages", "v_pages", "block_table", "lens", "acc", "B", "Hkv", "d", "dtype",
                 "page_size", "max_len", "device", "int32", "float32", "_index", "_struct", "_ref",
                 "_need", "_alloc", "_free", "_append", "_attend", "_evict")

    def __init__(self, k_pages, v_pages, block_table, lens, acc=None, max_len: Optional[int] = None):
        torch = _torch()
        if k_pages.dim() != 4 or tuple(v_pages.shape) != tuple(k_pages.shape):
            raise ValueError("k_pages and v_pages must be [num_pages, page_size, Hkv, d]")
        num_pages, page_size, Hkv, d = k_pages.shape
        dt = _dtype_code(k_pages)
        if _dtype_code(v_pages) != dt:
            raise TypeError("k_pages and v_pages dtypes differ")
        if k_pages.stride(3) != 1 or v_pages.stride(3) != 1:
            raise ValueError("the head-dim axis must be contiguous")
        if block_table.dim() != 2 or block_table.dtype != torch.int32 or \
                (block_table.shape[1] > 1 and block_table.stride(1) != 1):
            raise ValueError("block_table must be an int32 [B, columns] tensor, rows contiguous")
        B, cols = block_table.shape
        if max_len is None:
            max_len = cols * page_size
        if not 0 < max_len <= cols * page_size:
            raise ValueError("max_len must be positive and fit the block table")
        if max_len > _INT_MAX:
            raise ValueError("the block table holds %d tokens: give a max_len that fits 32 bits"
                             % max_len)
        if max(num_pages, page_size, B, Hkv, d) > _INT_MAX:
            raise ValueError("sizes of more than 32 bits")
        if tuple(lens.shape) != (B,) or lens.dtype != torch.int32 or not lens.is_contiguous():
            raise ValueError("lens must be a contiguous int32 [B] tensor")
        if acc is not None and (acc.dim() != 3 or tuple(acc.shape[:2]) != (B, Hkv) or
                                acc.shape[2] < max_len or acc.dtype != torch.float32 or
                                (acc.shape[2] > 1 and acc.stride(2) != 1)):
            raise ValueError("acc must be a float32 [B, Hkv, >= max_len] tensor, rows contiguous")
        for t in (v_pages, block_table, lens, acc):
            if t is not None and t.device != k_pages.device:
                raise ValueError("the cache's tensors must be on one device")
        self.k_pages, self.v_pages, self.block_table = k_pages, v_pages, block_table
        self.lens, self.acc = lens, acc
        self.B, self.Hkv, self.d, self.dtype = B, Hkv, d, k_pages.dtype
        self.page_size, self.max_len, self.device = page_size, int(max_len), k_pages.device
        self._index = k_pages.get_device()
        ks, vs = k_pages.stride(), v_pages.stride()
        sa = acc.stride() if acc is not None else (0, 0, 0)
        self._struct = _CacheStruct(_ptr(k_pages), _ptr(v_pages), _ptr(block_table), _ptr(lens),
                                    _ptr(acc), ks[0], ks[1], ks[2], vs[0], vs[1], vs[2],
                                    block_table.stride(0), sa[0], sa[1], dt, B, Hkv, d, num_pages,
                                    page_size, self.max_len)
        self._ref = ctypes.addressof(self._struct)
        self._need = {}   # (H, weights) -> workspace bytes
        # looked up once: the calls' host time is most of a small call's
        self.int32, self.float32 = torch.int32, torch.float32
        # what torch.cuda.caching_allocator_alloc and _delete call
        self._alloc = torch._C._cuda_cudaCachingAllocator_raw_alloc
        self._free = torch._C._cuda_cudaCachingAllocator_raw_delete
        L = lib()
        self._append, self._attend = L.avits_cache_append, L.avits_cache_attention
        self._evict = L.avits_cache_evict

    def __setattr__(self, name, value):
        if hasattr(self, "_evict"):       # set last
            raise AttributeError("a KVCache's description is fixed: make another one")
        object.__setattr__(self, name, value)


def _call_stream(cache: KVCache, stream):
    """The stream's handle.  The calls launch on the current device: the cache
    has to be there."""
    C = _torch()._C
    if C._cuda_getDevice() != cache._index:
        raise ValueError("the cache is on %s, which is not the current device" % cache.device)
    return C._cuda_getCurrentRawStream(cache._index) if stream is None else _stream(stream)


def _elsewhere(cache: KVCache, *tensors):
    for t in tensors:
        if t is not None and t.get_device() != cache._index:
            raise ValueError("tensor on %s, the cache is on %s" % (t.device, cache.device))


# These calls are made once per token and layer, so their checks are plain
# comparisons: of a small call's time most is spent here and in the launch.
def avits_cache_append(cache: KVCache, k_new, v_new, cu_new, stream=None):
    """New tokens into the cache: k_new, v_new [T,Hkv,d] (any 16-byte aligned
    strides, d contiguous), sequence b's being rows cu_new[b] .. cu_new[b+1]-1
    (int32 [B+1]).  cache.lens already counts them; they go to the last places.
    With cache.acc their accumulated weights are set to zero."""
    T, Hkv, d = shape = k_new.shape
    if Hkv != cache.Hkv or d != cache.d or v_new.shape != shape:
        raise ValueError("k_new / v_new must be [T, Hkv, d] of the cache")
    if T > _INT_MAX:
        raise ValueError("more new tokens than 32 bits count")
    if k_new.dtype != cache.dtype or v_new.dtype != cache.dtype:
        raise TypeError("k_new / v_new and cache dtypes differ")
    k_st, k_sh, k_sd = k_new.stride()
    v_st, v_sh, v_sd = v_new.stride()
    if k_sd != 1 or v_sd != 1:
        raise ValueError("the head-dim axis must be contiguous")
    if cu_new.shape != (cache.B + 1,) or cu_new.dtype != cache.int32 or \
            not cu_new.is_contiguous():
        raise ValueError("cu_new must be a contiguous int32 [B+1] tensor")
    index = cache._index
    if k_new.get_device() != index or v_new.get_device() != index or cu_new.get_device() != index:
        _elsewhere(cache, k_new, v_new, cu_new)
    rc = cache._append(cache._ref, k_new.data_ptr(), v_new.data_ptr(), T, cu_new.data_ptr(), k_st,
                       k_sh, v_st, v_sh, _call_stream(cache, stream))
    if rc != 0:
        _check("avits_cache_append", rc)


def avits_cache_attention_workspace(cache: KVCache, H: int, weights: bool) -> int:
    if not 0 < H <= _INT_MAX:
        return 0
    return int(lib().avits_cache_attention_workspace(cache._ref, H, 2 if weights else 0))


def avits_cache_attention(cache: KVCache, q, softmax_scale: float, o, lse=None,
                          weight: Optional[float] = None, accumulate: bool = True,
                          workspace=None, stream=None):
    """One new token per sequence over its cached tokens: q [B,H,d] into o
    [B,H,d] (the cache's type, any strides, d contiguous; query heads hk*G ..
    hk*G+G-1 share KV head hk, G = H / Hkv) and lse [B,H] fp32.  With ``weight``
    cache.acc gets weight times the mean over a KV head's query heads of the
    softmax weight of each cached token, added (or written).  ``workspace``: a
    device byte tensor of avits_cache_attention_workspace() bytes, of the
    caller's own where calls may overlap; by default one from PyTorch's allocator
    for this call, given back to it (a capture that PyTorch did not begin keeps no
    such memory: pass one there)."""
    B, H, d = shape = q.shape
    if B != cache.B or d != cache.d or o.shape != shape:
        raise ValueError("q and o must be [B, H, d] of the cache")
    if H > _INT_MAX:
        raise ValueError("more heads than 32 bits count")
    if q.dtype != cache.dtype or o.dtype != cache.dtype:
        raise TypeError("q, o and cache dtypes differ")
    q_sb, q_sh, q_sd = q.stride()
    o_sb, o_sh, o_sd = o.stride()
    if q_sd != 1 or o_sd != 1:
        raise ValueError("the head-dim axis must be contiguous")
    index = cache._index
    if q.get_device() != index or o.get_device() != index:
        _elsewhere(cache, q, o)
    lse_at = None
    if lse is not None:
        if lse.shape != (B, H) or lse.dtype != cache.float32 or not lse.is_contiguous():
            raise ValueError("lse must be a contiguous float32 [B,H] tensor")
        if lse.get_device() != index:
            _elsewhere(cache, lse)
        lse_at = lse.data_ptr()
    if weight is None:
        mode, weight = 0, 0.0
    else:
        mode = 2 if accumulate else 1
        if cache.acc is None:
            raise ValueError("weights are wanted of a cache without acc")
    handle = _call_stream(cache, stream)
    ws_at, ws_bytes, own = None, 0, None
    if workspace is not None:
        if not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous")
        _elsewhere(cache, workspace)
        ws_at, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    else:
        need = cache._need.get((H, mode))
        if need is None:
            need = cache._need[(H, mode)] = \
                int(lib().avits_cache_attention_workspace(cache._ref, H, mode))
        if need:
            # of this call and its stream: the allocator hands it on in the stream's order,
            # also to calls of other threads, and in a capture it is the graph's own memory
            # (0.6 us for the two calls, a tensor 1.5)
            ws_at = own = cache._alloc(need, handle)
            ws_bytes = need
    try:
        rc = cache._attend(cache._ref, q.data_ptr(), H, q_sb, q_sh, softmax_scale, o.data_ptr(),
                           o_sb, o_sh, lse_at, mode, weight, ws_at, ws_bytes, handle)
    finally:
        if own is not None:
            cache._free(own)
    if rc != 0:
        _check("avits_cache_attention", rc)
    return o


def avits_cache_evict(src: KVCache, dst: KVCache, keep: int, sinks: int, recent: int, keep_idx,
                      stream=None):
    """Per sequence and KV head: all cached tokens if there are at most
    ``keep``, else the first ``sinks``, the last ``recent`` and those of the
    largest src.acc between them (ties: the lower place), in order, copied with
    their weights to the places 0 .. of dst (pages that src does not read), whose
    lens are written.  keep_idx [B,Hkv,keep] int32: their places in src, -1 past
    the kept ones."""
    if keep_idx.shape != (src.B, src.Hkv, keep) or keep_idx.dtype != src.int32 or \
            not keep_idx.is_contiguous():
        raise ValueError("keep_idx must be a contiguous int32 [B, Hkv, keep] tensor")
    if not (-_INT_MAX <= sinks <= _INT_MAX and -_INT_MAX <= recent <= _INT_MAX):
        raise ValueError("sinks and recent must fit 32 bits")
    if src.dtype != dst.dtype or src.B != dst.B or src.Hkv != dst.Hkv or src.d != dst.d:
        raise ValueError("the two caches' types or sizes differ")
    if src.acc is None or dst.acc is None:
        raise ValueError("eviction goes by accumulated weights: both caches need acc")
    if dst._index != src._index or keep_idx.get_device() != src._index:
        _elsewhere(src, dst.k_pages, keep_idx)
    rc = src._evict(src._ref, dst._ref, keep, sinks, recent, keep_idx.data_ptr(),
                    _call_stream(src, stream))
    if rc != 0:
        _check("avits_cache_evict", rc)
    return keep_idx
