"""Thin ctypes binding of libpt.so (include/pt.h).  Argument marshalling only: every step of the
forward pass runs in the library's HIP kernels.  torch is used for device memory and streams.

The module fails loudly when the library is missing; there is no CPU fallback.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional

import numpy as np

from .inputs import PT_BF16, PT_F32, PTConfig

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpt.so")

PT_LOGITS_NONE, PT_LOGITS_LAST, PT_LOGITS_ALL = 0, 1, 2
PT_FAMILY_GENERIC, PT_FAMILY_COUNT = 0, 4
PT_TUNE_GEMM_TILE_CONFIG, PT_TUNE_SKINNY_PLAN, PT_TUNE_FOLD_RMSNORM, PT_TUNE_ATTN_PREFILL = 0, 1, 2, 3
PT_PATH_AUTO, PT_PATH_GENERIC = 0, 1
PT_ROPE_HALF, PT_ROPE_INTERLEAVED = 0, 1
PT_ROPE_UNSCALED, PT_ROPE_LINEAR, PT_ROPE_BY_PARTS = 0, 1, 2
PT_W_EMBED, PT_W_HEAD, PT_W_Q, PT_W_K, PT_W_V, PT_W_O, PT_W_G, PT_W_U, PT_W_D, PT_W_G1, PT_W_G2, PT_W_GF, PT_W_ROUTER = range(1, 14)
WEIGHT_IDS = {"embed": PT_W_EMBED, "head": PT_W_HEAD, "wq": PT_W_Q, "wk": PT_W_K, "wv": PT_W_V,
              "wo": PT_W_O, "wg": PT_W_G, "wu": PT_W_U, "wd": PT_W_D, "g1": PT_W_G1, "g2": PT_W_G2,
              "gf": PT_W_GF, "wr": PT_W_ROUTER}


def pt_expert_layer(layer: int, expert: int) -> int:
    """PT_EXPERT_LAYER of include/pt.h: the `layer` argument that addresses expert `expert`'s WG / WU / WD."""
    return layer | ((expert + 1) << 12)

PT_OK = 0
PT_ERR_INVALID_CONFIG, PT_ERR_NULL_POINTER, PT_ERR_ARENA_TOO_SMALL, PT_ERR_CAPACITY = -1, -2, -3, -4
PT_ERR_BAD_STATE, PT_ERR_HIP, PT_ERR_INVALID_ARGUMENT = -5, -6, -7

EXPORTS = [
    "pt_query_bytes", "pt_create", "pt_destroy", "pt_init_weights", "pt_set_weight", "pt_get_weight",
    "pt_prefill", "pt_decode_step", "pt_track_merge", "pt_set_taps", "pt_set_kernel_path", "pt_reset",
    "pt_merge_count", "pt_seq_len", "pt_last_error", "pt_profile_enable", "pt_profile_read",
    "pt_profile_reset", "pt_profile_paths", "pt_sync_status", "pt_set_tuning", "pt_argmax", "pt_decode_step_static", "pt_prefill_ragged", "pt_seq_lens",
    "pt_set_moe_routes", "pt_rope_init", "pt_paged_append", "pt_paged_attention_bytes", "pt_paged_attention",
    "pt_page_copy", "pt_sample_bytes", "pt_sample",
]

KERNEL_CLASSES = ["embed", "rmsnorm", "gemm_qkv", "attn_prefill", "attn_decode", "gemm_out",
                  "gemm_gateup", "gemm_down", "merge", "gemm_head", "other", "gemm_router", "moe"]


class pt_config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in (
        "n_tracks", "n_layers", "block_depth", "d_model", "n_heads", "n_kv_heads", "head_dim",
        "d_ffn", "vocab", "max_batch", "max_seq", "dtype")] + [
        (n, C.c_float) for n in ("merge_scale", "rms_eps", "rope_theta", "init_std")] + [
        (n, C.c_int32) for n in ("n_experts", "top_k")]


class pt_paged_cache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p)] + [(n, C.c_int32) for n in (
        "dtype", "n_layers", "n_pages", "page_size", "n_kv_heads", "head_dim")] + [(n, C.c_int64) for n in (
            "layer_stride", "page_stride", "head_stride", "token_stride")]


class pt_paged_batch(C.Structure):
    _fields_ = [("row_start", C.c_void_p), ("kv_len", C.c_void_p), ("pages", C.c_void_p), ("pages_stride", C.c_int64)] + [
        (n, C.c_int32) for n in ("n_seqs", "total_rows", "max_q_len", "max_kv_len")] + [("status", C.c_void_p)]


class pt_head_rows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("row_stride", C.c_int64), ("head_stride", C.c_int64)]


class pt_rope(C.Structure):
    _fields_ = [("layout", C.c_int32), ("rotary_dim", C.c_int32), ("magnitude", C.c_double), ("turns", C.c_double * 128)]


class PTError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__("libpt error %d: %s" % (code, msg))
        self.code = code


_lib = None


def lib() -> C.CDLL:
    """Loads libpt.so (built by ``python -m paper_2602_07306_amd.build``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError("%s is missing: build it with `python -m paper_2602_07306_amd.build` "
                          "(there is no fallback path)" % LIB_PATH)
    L = C.CDLL(LIB_PATH)
    vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    cfgp = C.POINTER(pt_config)
    L.pt_query_bytes.argtypes = [cfgp, C.POINTER(sz), C.POINTER(sz), C.POINTER(sz)]
    L.pt_create.argtypes = [cfgp, vp, sz, vp, sz, vp, sz, vp, C.POINTER(vp)]
    L.pt_destroy.argtypes = [vp]
    L.pt_init_weights.argtypes = [vp, C.c_uint64]
    L.pt_set_weight.argtypes = [vp, i32, i32, i32, vp]
    L.pt_get_weight.argtypes = [vp, i32, i32, i32, vp]
    L.pt_prefill.argtypes = [vp, vp, vp, i32, i32, i32, i32, vp, vp]
    L.pt_decode_step.argtypes = [vp, vp, vp, i32, i32, vp, vp, vp]
    L.pt_decode_step_static.argtypes = [vp, vp, vp, i32, i32, vp, vp, vp]
    L.pt_prefill_ragged.argtypes = [vp, vp, vp, i32, i32, C.POINTER(i32), i32, vp, vp]
    L.pt_seq_lens.argtypes = [vp, C.POINTER(i32)]
    L.pt_track_merge.argtypes = [C.POINTER(vp), i32, i64, i32, i32, C.c_float, vp, vp]
    L.pt_set_taps.argtypes = [vp, vp, vp]
    L.pt_set_moe_routes.argtypes = [vp, vp, vp]
    L.pt_set_kernel_path.argtypes = [vp, i32]
    L.pt_reset.argtypes = [vp]
    L.pt_merge_count.argtypes = [vp]
    L.pt_merge_count.restype = i64
    L.pt_seq_len.argtypes = [vp]
    L.pt_seq_len.restype = i32
    L.pt_profile_enable.argtypes = [vp, C.c_uint32]
    L.pt_profile_read.argtypes = [vp, i32, C.POINTER(C.c_double), C.POINTER(i64)]
    L.pt_profile_reset.argtypes = [vp]
    L.pt_profile_paths.argtypes = [vp, i32, C.POINTER(i64)]
    L.pt_sync_status.argtypes = [vp]
    L.pt_set_tuning.argtypes = [i32, i32]
    L.pt_argmax.argtypes = [vp, i32, i32, vp, vp]
    cachep, batchp, rowsp, ropep = C.POINTER(pt_paged_cache), C.POINTER(pt_paged_batch), C.POINTER(pt_head_rows), C.POINTER(pt_rope)
    f64 = C.c_double
    L.pt_rope_init.argtypes = [ropep, i32, i32, f64, i32, f64, f64, f64, i32, f64]
    L.pt_paged_append.argtypes = [cachep, i32, batchp, ropep, rowsp, rowsp, i32, rowsp, rowsp, vp]
    L.pt_paged_attention_bytes.argtypes = [cachep, batchp, i32, C.POINTER(sz)]
    L.pt_paged_attention.argtypes = [cachep, i32, batchp, rowsp, rowsp, i32, C.c_float, i32, vp, sz, vp]
    L.pt_page_copy.argtypes = [cachep, vp, i32, vp]
    L.pt_sample_bytes.argtypes = [i32, i32, C.POINTER(sz)]
    L.pt_sample.argtypes = [vp, i64, i32, i32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.pt_last_error.argtypes = []
    L.pt_last_error.restype = C.c_char_p
    for name in EXPORTS:
        if name not in ("pt_merge_count", "pt_seq_len", "pt_last_error"):
            getattr(L, name).restype = C.c_int
    _lib = L
    return L


def _check(rc: int) -> None:
    if rc != 0:
        raise PTError(rc, lib().pt_last_error().decode())


def to_c_config(cfg: PTConfig) -> pt_config:
    return pt_config(cfg.n_tracks, cfg.n_layers, cfg.block_depth, cfg.d_model, cfg.n_heads,
                     cfg.n_kv_heads, cfg.head_dim, cfg.d_ffn, cfg.vocab, cfg.max_batch, cfg.max_seq,
                     cfg.dtype, cfg.merge_scale, cfg.rms_eps, cfg.rope_theta, cfg.init_std, cfg.n_experts,
                     cfg.top_k)


def pt_last_error() -> str:
    return lib().pt_last_error().decode()


def pt_set_tuning(knob: int, value: int) -> None:
    _check(lib().pt_set_tuning(knob, value))


def pt_query_bytes(cfg: PTConfig):
    """(weight_bytes, kv_bytes, workspace_bytes); host only."""
    w, kv, ws = C.c_size_t(), C.c_size_t(), C.c_size_t()
    c = to_c_config(cfg)
    _check(lib().pt_query_bytes(C.byref(c), C.byref(w), C.byref(kv), C.byref(ws)))
    return w.value, kv.value, ws.value


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def pt_track_merge(tracks, scale: float, out=None, stream=None):
    """out = scale * sum(tracks) through the library's merge kernel.  tracks: list of device
    tensors [tokens, d], all float32 or all bfloat16."""
    import torch
    t0 = tracks[0]
    dtype = PT_F32 if t0.dtype == torch.float32 else PT_BF16
    assert all(t.dtype == t0.dtype and t.shape == t0.shape and t.is_contiguous() for t in tracks)
    if out is None:
        out = torch.empty_like(t0)
    arr = (C.c_void_p * len(tracks))(*[t.data_ptr() for t in tracks])
    st = torch.cuda.current_stream().cuda_stream if stream is None else stream
    tokens, d = (t0.shape[0], t0.shape[1]) if t0.dim() == 2 else (t0.numel() // t0.shape[-1], t0.shape[-1])
    _check(lib().pt_track_merge(arr, len(tracks), tokens, d, dtype, float(scale), out.data_ptr(), st))
    return out


def pt_argmax(logits, out=None, stream=None):
    """out[r] = argmax of logits[r, :] (float32 device tensor [rows, vocab]), lowest id on ties."""
    import torch
    assert logits.dtype == torch.float32 and logits.is_contiguous() and logits.dim() == 2
    if out is None:
        out = torch.empty((logits.shape[0],), dtype=torch.int32, device=logits.device)
    st = torch.cuda.current_stream().cuda_stream if stream is None else getattr(stream, "cuda_stream", stream)
    _check(lib().pt_argmax(logits.data_ptr(), logits.shape[0], logits.shape[1], out.data_ptr(), st))
    return out


# -- serving over a paged cache ------------------------------------------------------------------
# A decode step makes these calls once per layer, and the GPU is done with a small one in a few microseconds: descriptors
# are built once, tensors are looked at once per call.

def _need(ok: bool, what: str) -> None:
    if not ok:
        raise PTError(PT_ERR_INVALID_ARGUMENT, what)


_current = None   # torch's (current stream of a device as a handle, current device, guard)


def _launch(index: int, stream, fn, *args) -> None:
    """fn(*args, stream) on GPU `index`, on its current stream if none is given."""
    global _current
    if index < 0:
        raise PTError(PT_ERR_INVALID_ARGUMENT, "the tensors must be on a GPU")
    if _current is None:
        import torch
        _current = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice, torch.cuda.device
    raw_stream, device, guard = _current
    st = raw_stream(index) if stream is None else getattr(stream, "cuda_stream", stream)
    if device() == index:
        rc = fn(*args, st)
    else:
        with guard(index):
            rc = fn(*args, st)
    if rc:
        _check(rc)


def _empty(shape, dtype, device, stream):
    """A tensor for a call on `stream`, allocated on that stream, so that neither earlier nor later owners of its memory
    overlap the call."""
    import torch
    _need(device.type == "cuda", "the tensors must be on a GPU")
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(stream, device=device)):
        return torch.empty(shape, dtype=dtype, device=device)


def _scratch(given, nbytes, device, stream):
    """(workspace, its address, its bytes): the caller's, or one of nbytes() for this call."""
    if given is None:
        import torch
        n = nbytes()
        if n == 0:
            return None, None, 0
        given = _empty(n, torch.uint8, device, stream)
        return given, given.data_ptr(), n
    _need(given.device == device and given.is_contiguous(), "workspace must be contiguous and on the operands' device")
    return given, given.data_ptr(), given.numel() * given.element_size()


class PTRope:
    """Rotary positions (pt_rope_init): layout PT_ROPE_HALF or PT_ROPE_INTERLEAVED of a head's first rotary_dim elements, base
    theta; scaling PT_ROPE_LINEAR by `factor`, or PT_ROPE_BY_PARTS by `factor` for pairs that turn less than `low` times
    over original_len positions, none above `high` turns and blended in between; rotated vectors are multiplied with
    `magnitude`."""

    def __init__(self, layout: int, rotary_dim: int, theta: float = 10000.0, scaling: int = PT_ROPE_UNSCALED, factor: float = 1.0,
                 low: float = 1.0, high: float = 32.0, original_len: int = 1, magnitude: float = 1.0):
        self.c = pt_rope()
        _check(lib().pt_rope_init(C.byref(self.c), layout, rotary_dim, theta, scaling, factor, low, high, original_len, magnitude))


class PTPagedCache:
    """A pool of pages: k and v of one shape [layers, pages, kv heads, page size, head width], float32 or bfloat16, the same
    strides, the last dimension contiguous (other orders as permuted views)."""

    def __init__(self, k, v):
        import torch
        _need(k.dim() == 5 and k.shape == v.shape, "k and v must be [layers, pages, kv heads, page size, head width]")
        _need(k.dtype == v.dtype and k.dtype in (torch.float32, torch.bfloat16), "k and v must both be float32 or both bfloat16")
        _need(k.device == v.device, "k and v must be on one device")
        # the stride of a dimension of one entry says nothing
        st = [0 if n == 1 else s for n, s in zip(k.shape, k.stride())]
        _need(st == [0 if n == 1 else s for n, s in zip(v.shape, v.stride())] and (st[4] == 1 or k.shape[4] == 1),
              "k and v must have the same strides and a contiguous last dimension")
        if k.shape[3] == 1:
            st[3] = k.shape[4]
        self.k, self.v, self.dtype, self.index = k, v, k.dtype, k.get_device()
        self.kv_heads, self.page_size, self.width = k.shape[2:]
        self.c = pt_paged_cache(k.data_ptr(), v.data_ptr(), PT_F32 if k.dtype == torch.float32 else PT_BF16, k.shape[0], k.shape[1],
                                k.shape[3], k.shape[2], k.shape[4], st[0], st[1], st[2], st[3])


class PTPagedBatch:
    """The rows of one step (pt_paged_batch): int32 device tensors row_start [n + 1], kv_len [n] and pages [n, width].  Their
    contents may change between calls (a captured graph reads them when it is replayed); the bounds hold for all of them.
    status: int32 device tensor of one element that collects the kernels' complaints, or None."""

    def __init__(self, row_start, kv_len, pages, total_rows: int, max_q_len: int = 0, max_kv_len: int = 0, status=None):
        import torch
        for t in (row_start, kv_len, pages) + (() if status is None else (status,)):
            _need(t.dtype == torch.int32 and t.device == pages.device, "row_start, kv_len, pages and status must be int32 on one device")
        _need(row_start.dim() == 1 and kv_len.dim() == 1 and pages.dim() == 2, "row_start and kv_len have one dimension, pages two")
        n = kv_len.shape[0]
        _need(row_start.shape[0] == n + 1 and pages.shape[0] == n, "row_start needs one entry more than kv_len, pages as many rows")
        _need(row_start.is_contiguous() and kv_len.is_contiguous(), "row_start and kv_len must be contiguous")
        _need(pages.shape[1] <= 1 or pages.stride(1) == 1, "the rows of pages must be contiguous")
        _need(status is None or status.numel() >= 1, "status needs one element")
        # with one sequence the stride between rows says nothing; rows further apart than their width hold no more entries
        self.width = pages.shape[1]
        _need(n <= 1 or pages.stride(0) >= self.width, "the rows of pages overlap")
        self.row_start, self.kv_len, self.pages, self.status = row_start, kv_len, pages, status
        self.total_rows, self.index = total_rows, pages.get_device()
        self.c = pt_paged_batch(row_start.data_ptr(), kv_len.data_ptr(), pages.data_ptr(), self.width if n <= 1 else pages.stride(0), n,
                                total_rows, max_q_len, max_kv_len, _ptr(status))
        self._bound = {}   # page size: the C descriptor with its max_kv_len

    def bound(self, cache):
        """The C descriptor for calls with `cache`: max_kv_len comes from the table's width where it was not given."""
        _need(self.index == cache.index, "batch and cache must be on one device")
        c = self._bound.get(cache.page_size)
        if c is None:
            room = min(self.width * cache.page_size, 0x7fffffff)
            _need(self.c.max_kv_len <= room, "max_kv_len exceeds the page table")
            c = pt_paged_batch.from_buffer_copy(self.c)
            c.max_kv_len = c.max_kv_len or room
            self._bound[cache.page_size] = c
        return c


def _rows(t, name: str, cache, batch, heads: int = 0):
    """(pt_head_rows, heads) of a device tensor [rows, heads, head width]."""
    shape, st = t.shape, t.stride()
    if not (len(shape) == 3 and t.dtype is cache.dtype and t.get_device() == cache.index):
        raise PTError(PT_ERR_INVALID_ARGUMENT, "%s must be [rows, heads, width] of the cache's type and device" % name)
    n, h, w = shape
    if not (n >= batch.total_rows and w == cache.width and (heads == 0 or h == heads) and st[2] == 1):
        raise PTError(PT_ERR_INVALID_ARGUMENT, "%s has shape %s and strides %s: need %d rows of %s heads of %d contiguous elements"
                      % (name, tuple(shape), st, batch.total_rows, heads or "any", cache.width))
    # the stride of a dimension of one entry says nothing
    return pt_head_rows(t.data_ptr(), st[0] if n > 1 else 0, st[1] if h > 1 else 0), h


def pt_paged_append(cache: PTPagedCache, layer: int, batch: PTPagedBatch, k, v, q=None, q_out=None, rope: Optional[PTRope] = None, stream=None):
    """Stores the batch's keys and values [rows, kv heads, width] in their pages, queries and keys rotated on the way.
    q [rows, heads, width] goes to q_out (made if not given; may be q).  Returns q_out."""
    cb = batch.bound(cache)
    ck, cv = _rows(k, "k", cache, batch, cache.kv_heads)[0], _rows(v, "v", cache, batch, cache.kv_heads)[0]
    cq = co = None
    heads = 0
    if q is not None:
        cq, heads = _rows(q, "q", cache, batch)
        if q_out is None:
            q_out = _empty(q.shape, q.dtype, q.device, stream)
        co = _rows(q_out, "q_out", cache, batch, heads)[0]
    else:
        _need(q_out is None, "q_out without q")
    _launch(cache.index, stream, lib().pt_paged_append, cache.c, layer, cb, None if rope is None else rope.c, cq, co, heads, ck, cv)
    return q_out


def pt_paged_attention_bytes(cache: PTPagedCache, batch: PTPagedBatch, n_heads: int) -> int:
    """Workspace bytes of pt_paged_attention."""
    n = C.c_size_t()
    _check(lib().pt_paged_attention_bytes(cache.c, batch.bound(cache), n_heads, C.byref(n)))
    return n.value


def pt_paged_attention(cache: PTPagedCache, layer: int, batch: PTPagedBatch, q, out=None, scale: Optional[float] = None, causal: bool = True,
                       workspace=None, stream=None):
    """Attention of the batch's queries [rows, heads, width] over their sequences' pages.  scale: 1 / sqrt(width) if not
    given.  workspace: uint8 device tensor of pt_paged_attention_bytes (made per call if not given).  Returns out."""
    cb = batch.bound(cache)
    cq, heads = _rows(q, "q", cache, batch)
    if out is None:
        out = _empty(q.shape, q.dtype, q.device, stream)
    co = _rows(out, "out", cache, batch, heads)[0]
    ws, at, size = _scratch(workspace, lambda: pt_paged_attention_bytes(cache, batch, heads), q.device, stream)
    _launch(cache.index, stream, lib().pt_paged_attention, cache.c, layer, cb, cq, co, heads, cache.width ** -0.5 if scale is None else scale,
            int(causal), at, size)
    return out


def pt_page_copy(cache: PTPagedCache, pairs, stream=None) -> None:
    """Copies pages inside the cache, every layer, K and V.  pairs: host array or list of (from, to)."""
    p = np.asarray(pairs)
    if p.size == 0:
        return
    _need(p.ndim == 2 and p.shape[1] == 2 and p.dtype.kind in "iu", "pairs must be whole numbers [n, 2]")
    if p.dtype != np.int32:
        _need(int(p.min()) >= 0 and int(p.max()) < 2 ** 31, "a page out of range")
    p = np.ascontiguousarray(p, dtype=np.int32)
    _launch(cache.index, stream, lib().pt_page_copy, cache.c, p.ctypes.data, p.shape[0])


def pt_sample_bytes(rows: int, vocab: int) -> int:
    """Workspace bytes of pt_sample."""
    n = C.c_size_t()
    _check(lib().pt_sample_bytes(rows, vocab, C.byref(n)))
    return n.value


def _row_params(t, dtype, rows: int, index: int, name: str):
    """Address of a parameter with one entry per row, or None."""
    if t is None:
        return None
    if not (t.dtype is dtype and t.shape == (rows,) and t.get_device() == index and (rows <= 1 or t.stride(0) == 1)):
        raise PTError(PT_ERR_INVALID_ARGUMENT, "%s must be contiguous %s [rows] on the logits' device" % (name, str(dtype)[6:]))
    return t.data_ptr()


def pt_sample(logits, uniform, temperature=None, top_k=None, top_p=None, min_p=None, out=None, workspace=None, stream=None):
    """One token per row of logits (float32 device tensor [rows, vocab], rows contiguous) by the given uniform numbers [rows]
    in [0, 1).  temperature, top_p, min_p: float32 [rows], top_k: int32 [rows], or None.  Returns int32 [rows]."""
    import torch
    f32, i32 = torch.float32, torch.int32
    _need(logits.dim() == 2 and logits.dtype is f32, "logits must be float32 [rows, vocab]")
    (rows, vocab), st, index = logits.shape, logits.stride(), logits.get_device()
    _need(st[1] == 1 or vocab == 1, "the rows of logits must be contiguous")
    _need(uniform is not None, "uniform is missing")
    params = (_row_params(uniform, f32, rows, index, "uniform"), _row_params(temperature, f32, rows, index, "temperature"),
              _row_params(top_k, i32, rows, index, "top_k"), _row_params(top_p, f32, rows, index, "top_p"), _row_params(min_p, f32, rows, index, "min_p"))
    if out is None:
        out = _empty((rows,), i32, logits.device, stream)
    to = _row_params(out, i32, rows, index, "out")
    ws, at, size = _scratch(workspace, lambda: pt_sample_bytes(rows, vocab), logits.device, stream)
    _launch(index, stream, lib().pt_sample, logits.data_ptr(), st[0] if rows > 1 else vocab, rows, vocab, *params, to, at, size)
    return out


class PTModel:
    """A pt_handle plus the torch tensors that back its three arenas."""

    def __init__(self, cfg: PTConfig, device: str = "cuda:0", stream=None):
        import torch
        self.torch = torch
        self.cfg = cfg
        self.device = torch.device(device)
        wb, kb, sb = pt_query_bytes(cfg)
        self.bytes = (wb, kb, sb)
        self._w = torch.empty(wb, dtype=torch.uint8, device=self.device)
        self._kv = torch.empty(kb, dtype=torch.uint8, device=self.device)
        self._ws = torch.empty(sb, dtype=torch.uint8, device=self.device)
        self.stream = torch.cuda.current_stream(self.device) if stream is None else stream
        h = C.c_void_p()
        c = to_c_config(cfg)
        _check(lib().pt_create(C.byref(c), self._w.data_ptr(), wb, self._kv.data_ptr(), kb,
                               self._ws.data_ptr(), sb, self.stream.cuda_stream, C.byref(h)))
        self.h = h
        self._taps = None

    def close(self):
        if self.h:
            lib().pt_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- weights -------------------------------------------------------------------------------
    def pt_init_weights(self, seed: int):
        _check(lib().pt_init_weights(self.h, seed))

    def pt_set_weight(self, name: str, track: int, layer: int, array):
        t = self.torch.as_tensor(np.ascontiguousarray(array, dtype=np.float32)).to(self.device)
        _check(lib().pt_set_weight(self.h, WEIGHT_IDS[name], track, layer, t.data_ptr()))
        self.torch.cuda.synchronize(self.device)

    def pt_get_weight(self, name: str, track: int, layer: int, shape):
        t = self.torch.empty(shape, dtype=self.torch.float32, device=self.device)
        _check(lib().pt_get_weight(self.h, WEIGHT_IDS[name], track, layer, t.data_ptr()))
        self.torch.cuda.synchronize(self.device)
        return t.cpu().numpy()

    def load_weights(self, W):
        """Uploads a dict of logical weights (layouts of inputs.make_weights)."""
        cfg = self.cfg
        E = cfg.n_experts
        for name in ("wq", "wk", "wv", "wo", "wg", "wu", "wd", "g1", "g2") + (("wr",) if E > 0 else ()):
            for i in range(cfg.n_tracks):
                for l in range(cfg.n_layers):
                    if E > 0 and name in ("wg", "wu", "wd"):
                        for e in range(E):
                            self.pt_set_weight(name, i, pt_expert_layer(l, e), W[name][i, l, e])
                    else:
                        self.pt_set_weight(name, i, l, W[name][i, l])
        self.pt_set_weight("gf", 0, 0, W["gf"])
        if cfg.vocab > 0:
            self.pt_set_weight("embed", 0, 0, W["embed"])
            self.pt_set_weight("head", 0, 0, W["head"])

    # -- forward -------------------------------------------------------------------------------
    def pt_set_taps(self, rows: int, track_taps: bool = False):
        cfg, torch = self.cfg, self.torch
        taps = torch.zeros((cfg.n_merges, rows, cfg.d_model), dtype=torch.float32, device=self.device)
        tt = (torch.zeros((cfg.n_merges, cfg.n_tracks, rows, cfg.d_model), dtype=torch.float32,
                          device=self.device) if track_taps else None)
        _check(lib().pt_set_taps(self.h, taps.data_ptr(), _ptr(tt)))
        self._taps = (taps, tt)
        return taps, tt

    def pt_clear_taps(self):
        _check(lib().pt_set_taps(self.h, None, None))
        self._taps = None

    def pt_set_moe_routes(self, rows: int, forced=None, observe: bool = True):
        """PT-MoE: observe and / or prescribe the expert selection of later forward calls over `rows` rows.
        forced: int array [n_layers, n_tracks, rows, top_k].  Returns the int32 device tensor that receives the
        selection (or None)."""
        cfg, torch = self.cfg, self.torch
        shape = (cfg.n_layers, cfg.n_tracks, rows, cfg.top_k)
        out = torch.full(shape, -1, dtype=torch.int32, device=self.device) if observe else None
        fin = None
        if forced is not None:
            fin = torch.as_tensor(np.ascontiguousarray(forced, dtype=np.int32)).to(self.device)
            assert tuple(fin.shape) == shape
        _check(lib().pt_set_moe_routes(self.h, _ptr(out), _ptr(fin)))
        self._routes = (out, fin)
        return out

    def pt_clear_moe_routes(self):
        _check(lib().pt_set_moe_routes(self.h, None, None))
        self._routes = None

    def pt_set_kernel_path(self, path: int):
        _check(lib().pt_set_kernel_path(self.h, path))

    def pt_prefill(self, tokens=None, hidden_in=None, logits_mode: int = PT_LOGITS_LAST,
                   want_hidden: bool = False, logits_out=None):
        """tokens: int32 device tensor [B, S]; hidden_in: float32 device tensor [B, S, d] or
        [T, B, S, d].  Returns (logits or None, hidden or None) as device tensors."""
        cfg, torch = self.cfg, self.torch
        if tokens is not None:
            B, S = tokens.shape
            ht = 1
        else:
            ht = 1 if hidden_in.dim() == 3 else hidden_in.shape[0]
            B, S = hidden_in.shape[-3], hidden_in.shape[-2]
        logits = logits_out
        if logits_mode != PT_LOGITS_NONE and logits is None:
            rows = B if logits_mode == PT_LOGITS_LAST else B * S
            logits = torch.empty((rows, cfg.vocab), dtype=torch.float32, device=self.device)
        hidden = torch.empty((B, S, cfg.d_model), dtype=torch.float32, device=self.device) if want_hidden else None
        _check(lib().pt_prefill(self.h, _ptr(tokens), _ptr(hidden_in), ht, B, S, logits_mode,
                                _ptr(logits), _ptr(hidden)))
        return logits, hidden

    def pt_prefill_ragged(self, lens, tokens=None, hidden_in=None, logits_mode: int = PT_LOGITS_LAST,
                          want_hidden: bool = False, logits_out=None):
        """Prefill of sequences of different lengths.  lens: host list of B lengths; tokens: int32 device tensor
        [sum(lens)] (packed); hidden_in: float32 device tensor [sum(lens), d] or [T, sum(lens), d].  Returns
        (logits or None, hidden or None) as device tensors, packed the same way."""
        cfg, torch = self.cfg, self.torch
        B, n = len(lens), int(sum(lens))
        ht = 1
        if tokens is None:
            ht = 1 if hidden_in.dim() == 2 else hidden_in.shape[0]
            assert hidden_in.shape[-2] == n
        else:
            assert tokens.numel() == n
        logits = logits_out
        if logits_mode != PT_LOGITS_NONE and logits is None:
            logits = torch.empty((B if logits_mode == PT_LOGITS_LAST else n, cfg.vocab), dtype=torch.float32, device=self.device)
        hidden = torch.empty((n, cfg.d_model), dtype=torch.float32, device=self.device) if want_hidden else None
        arr = (C.c_int32 * B)(*[int(x) for x in lens])
        _check(lib().pt_prefill_ragged(self.h, _ptr(tokens), _ptr(hidden_in), ht, B, arr, logits_mode, _ptr(logits), _ptr(hidden)))
        return logits, hidden

    def pt_seq_lens(self):
        B = 0
        arr = (C.c_int32 * max(self.cfg.max_batch, 1))()
        _check(lib().pt_seq_lens(self.h, arr))
        return list(arr)

    def pt_decode_step(self, tokens=None, hidden_in=None, want_logits: bool = True,
                       want_hidden: bool = False, want_argmax: bool = False, logits_out=None,
                       argmax_out=None, hidden_out=None, static_scratch: bool = False):
        """One decode step.  static_scratch=True calls pt_decode_step_static (temporaries in the library's
        static device array instead of the workspace arena); the output tensors are still the caller's."""
        cfg, torch = self.cfg, self.torch
        if tokens is not None:
            B, ht = tokens.shape[0], 1
        else:
            ht = 1 if hidden_in.dim() == 2 else hidden_in.shape[0]
            B = hidden_in.shape[-2]
        logits = logits_out
        if logits is None and (want_logits or want_argmax) and cfg.vocab > 0:
            logits = torch.empty((B, cfg.vocab), dtype=torch.float32, device=self.device)
        hidden = hidden_out
        if hidden is None and want_hidden:
            hidden = torch.empty((B, cfg.d_model), dtype=torch.float32, device=self.device)
        amax = argmax_out
        if amax is None and want_argmax:
            amax = torch.empty((B,), dtype=torch.int32, device=self.device)
        fn = lib().pt_decode_step_static if static_scratch else lib().pt_decode_step
        _check(fn(self.h, _ptr(tokens), _ptr(hidden_in), ht, B, _ptr(logits), _ptr(hidden), _ptr(amax)))
        return logits, hidden, amax

    def pt_profile_enable(self, classes):
        """classes: iterable of kernel-class names (KERNEL_CLASSES) to time; empty = off."""
        mask = 0
        for c in classes:
            mask |= 1 << KERNEL_CLASSES.index(c)
        _check(lib().pt_profile_enable(self.h, mask))

    def pt_profile_read(self, cls: str):
        """(total milliseconds, launches) of one kernel class since the last reset."""
        ms, n = C.c_double(), C.c_int64()
        _check(lib().pt_profile_read(self.h, KERNEL_CLASSES.index(cls), C.byref(ms), C.byref(n)))
        return ms.value, n.value

    def pt_profile_reset(self):
        _check(lib().pt_profile_reset(self.h))

    def pt_profile_paths(self, cls: str):
        """Launches of one kernel class per kernel family since the last pt_profile_reset
        (index 0: the shape-generic kernel; see include/pt.h)."""
        counts = (C.c_int64 * PT_FAMILY_COUNT)()
        _check(lib().pt_profile_paths(self.h, KERNEL_CLASSES.index(cls), counts))
        return list(counts)

    def pt_sync_status(self):
        """Synchronises the stream; raises PTError if a forward call met an out-of-range token id."""
        _check(lib().pt_sync_status(self.h))

    def pt_reset(self):
        _check(lib().pt_reset(self.h))

    def pt_merge_count(self) -> int:
        return lib().pt_merge_count(self.h)

    def pt_seq_len(self) -> int:
        return lib().pt_seq_len(self.h)
