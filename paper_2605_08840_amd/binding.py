"""ctypes binding of librestkv.so: argument marshalling only.

Function names and arguments mirror ``include/restkv.h``.  Tensors are torch
tensors on the GPU; torch is used for device memory and the current stream,
nothing else -- every step of the path runs in the library's HIP kernels.
There is no CPU fallback: a missing library raises.
"""
from __future__ import annotations

import ctypes
import math
import os
from dataclasses import dataclass, field
from typing import Optional

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
# RESTKV_LIB names another build of the same library (the host-sanitized one of the CPU tests)
LIB_PATH = os.environ.get("RESTKV_LIB") or os.path.join(_PKG, "librestkv.so")

RESTKV_F32 = 0
RESTKV_BF16 = 1
RESTKV_Q4 = 4
# ablation variants (restkv_params.variant, see include/restkv.h)
RESTKV_IND_ATTENTION = 1
RESTKV_IND_VALUE_NORM = 2
RESTKV_GROUP_MAX = 1 << 2
RESTKV_TEMPORAL_MEAN = 1 << 4
RESTKV_TEMPORAL_INV_EMA = 2 << 4
RESTKV_POOL_MAX = 1 << 6


class RestkvParams(ctypes.Structure):
    _fields_ = [
        ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
        ("seq_len", ctypes.c_int32), ("window", ctypes.c_int32), ("budget", ctypes.c_int32),
        ("dtype", ctypes.c_int32), ("causal", ctypes.c_int32), ("scale", ctypes.c_float),
        ("ema_alpha", ctypes.c_float), ("base_window", ctypes.c_int32), ("adaptive", ctypes.c_int32),
        ("beta", ctypes.c_float), ("variant", ctypes.c_int32),
        ("q_stride_h", ctypes.c_int64), ("q_stride_t", ctypes.c_int64),
        ("kv_stride_h", ctypes.c_int64), ("kv_stride_t", ctypes.c_int64), ("ld_score", ctypes.c_int64),
    ]


class RestkvCache(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "n_seqs", "n_q_heads", "n_kv_heads", "head_dim", "dtype", "format", "page_size", "n_pages", "max_pages", "max_len",
        "max_new", "n_tokens", "causal", "rotary_dim", "rotary_pairs", "n_positions", "out_dtype")] + [
        ("scale", ctypes.c_float)] + [(n, ctypes.c_int64) for n in (
            "page_stride", "head_stride", "token_stride", "table_stride_s", "table_stride_h", "lens_stride_s", "lens_stride_h",
            "q_stride_t", "q_stride_h", "kv_stride_t", "kv_stride_h", "out_stride_t", "out_stride_h", "lse_stride_t",
            "lse_stride_h")]

    def __setattr__(self, name, value):
        self.__dict__.pop("told", None)      # what the binding has worked out from the fields
        super().__setattr__(name, value)


class RestkvBeams(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_groups", "n_beams", "n_vocab", "n_out", "dtype", "end_token")] + [
        ("logit_stride", ctypes.c_int64)]

    def __setattr__(self, name, value):
        self.__dict__.pop("told", None)      # what the binding has worked out from the fields
        super().__setattr__(name, value)


class RestkvLayerPages(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k_pages", "v_pages", "k_scale", "v_scale")]


class RestkvError(RuntimeError):
    def __init__(self, code: int, what: str):
        self.code = code
        super().__init__(f"{what}: {strerror(code)} (code {code})")


_lib = None


def lib() -> ctypes.CDLL:
    """Loads the HIP library; fails loudly when it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: run `python -c 'import __graft_entry__ as g; g.build()'`"
                              " (there is no CPU fallback)")
        L = ctypes.CDLL(LIB_PATH)
        P = ctypes.POINTER(RestkvParams)
        vp, sz, i64 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int64
        L.restkv_workspace_bytes.restype = sz
        L.restkv_workspace_bytes.argtypes = [P]
        L.restkv_prepare_wo.argtypes = [P, vp, i64, vp, vp]
        L.restkv_score.argtypes = [P, vp, vp, vp, vp, vp, vp, sz, vp]
        L.restkv_score_from_attention.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.restkv_score_from_attention.restype = ctypes.c_int
        L.restkv_smooth.argtypes = [P, vp, vp, vp, vp, vp, vp, sz, vp]
        L.restkv_score_smooth.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.restkv_select.argtypes = [P, vp, vp, vp, sz, vp]
        L.restkv_smooth_b.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.restkv_select_b.argtypes = [P, vp, vp, vp, vp, sz, vp]
        L.restkv_select_static.argtypes = [P, vp, vp, vp]
        L.restkv_select_static.restype = ctypes.c_int
        L.restkv_select_static_capacity.restype = sz
        L.restkv_select_static_capacity.argtypes = []
        L.restkv_compact.argtypes = [P, vp, vp, vp, vp, vp, vp]
        L.restkv_evict.argtypes = [P] + [vp] * 13 + [sz, vp]
        L.restkv_evict.restype = ctypes.c_int
        C, i32 = ctypes.POINTER(RestkvCache), ctypes.c_int32
        L.restkv_append.argtypes = [C] + [vp] * 15
        L.restkv_append.restype = ctypes.c_int
        L.restkv_attend_workspace_bytes.argtypes = [C]
        L.restkv_attend_workspace_bytes.restype = sz
        L.restkv_attend.argtypes = [C] + [vp] * 11 + [sz, vp]
        L.restkv_attend.restype = ctypes.c_int
        L.restkv_fetch.argtypes = [C] + [vp] * 7 + [i32, i32, vp, vp, vp]
        L.restkv_fetch.restype = ctypes.c_int
        b = ctypes.POINTER(RestkvBeams)
        L.restkv_beam_workspace_bytes.argtypes = [b]
        L.restkv_beam_workspace_bytes.restype = sz
        L.restkv_beam_select.argtypes = [b] + [vp] * 8 + [sz, vp]
        L.restkv_beam_select.restype = ctypes.c_int
        L.restkv_beam_reorder.argtypes = [C, i32, vp, i64, vp, vp, vp, vp, i32, vp]
        L.restkv_beam_reorder.restype = ctypes.c_int
        L.restkv_attend_beams_workspace_bytes.argtypes = [C, i32]
        L.restkv_attend_beams_workspace_bytes.restype = sz
        L.restkv_debug_force_shared.argtypes = [ctypes.c_int]
        L.restkv_debug_force_shared.restype = ctypes.c_int
        L.restkv_debug_beams_list.argtypes = [C, i32, vp, vp]
        L.restkv_debug_beams_list.restype = ctypes.c_int
        L.restkv_attend_beams.argtypes = [C, i32] + [vp] * 12 + [sz, vp]
        L.restkv_attend_beams.restype = ctypes.c_int
        L.restkv_strerror.restype = ctypes.c_char_p
        L.restkv_strerror.argtypes = [ctypes.c_int]
        L.restkv_timing_read.argtypes = [vp, vp, ctypes.c_int]
        L.restkv_timing_enable.argtypes = [ctypes.c_int]
        L.restkv_stage_name.restype = ctypes.c_char_p
        L.restkv_stage_name.argtypes = [ctypes.c_int]
        L.restkv_debug_force_fp32.argtypes = [ctypes.c_int]
        L.restkv_debug_force_fp32.restype = ctypes.c_int
        L.restkv_debug_score_plan.argtypes = [P, vp]
        L.restkv_debug_score_plan.restype = ctypes.c_int
        L.restkv_debug_fp32_plan.argtypes = [P, vp]
        L.restkv_debug_fp32_plan.restype = ctypes.c_int
        L.restkv_stream_reference.argtypes = [vp, sz, vp, sz, vp]
        L.restkv_stream_reference.restype = ctypes.c_int
        for f in ("restkv_timing_enable", "restkv_timing_read", "restkv_prepare_wo", "restkv_score", "restkv_smooth", "restkv_select",
                  "restkv_compact", "restkv_version", "restkv_score_smooth", "restkv_smooth_b", "restkv_select_b"):
            getattr(L, f).restype = ctypes.c_int
        _lib = L
    return _lib


def strerror(code: int) -> str:
    return lib().restkv_strerror(int(code)).decode()


def make_params(*, n_q_heads, n_kv_heads, head_dim, seq_len, window, budget, dtype,
                causal=True, scale=0.0, ema_alpha=0.3, base_window=5, adaptive=True, beta=2000.0,
                q_stride_h=0, q_stride_t=0, kv_stride_h=0, kv_stride_t=0, ld_score=0, variant=0) -> RestkvParams:
    dt = {torch.float32: RESTKV_F32, torch.bfloat16: RESTKV_BF16, "f32": RESTKV_F32,
          "bf16": RESTKV_BF16}.get(dtype, dtype)
    return RestkvParams(n_q_heads, n_kv_heads, head_dim, seq_len, window, budget, int(dt),
                        int(bool(causal)), float(scale), float(ema_alpha), int(base_window),
                        int(bool(adaptive)), float(beta), int(variant), q_stride_h, q_stride_t, kv_stride_h,
                        kv_stride_t, ld_score)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream=None):
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _chk(rc: int, what: str):
    if rc != 0:
        raise RestkvError(rc, what)


def restkv_workspace_bytes(p: RestkvParams) -> int:
    return int(lib().restkv_workspace_bytes(ctypes.byref(p)))


def alloc_workspace(p: RestkvParams, device="cuda") -> torch.Tensor:
    n = restkv_workspace_bytes(p)
    if n == 0:
        raise RestkvError(-1, "restkv_workspace_bytes")
    return torch.empty(n + 256, dtype=torch.uint8, device=device)


def _ws(ws: Optional[torch.Tensor]):
    if ws is None:
        return None, 0
    off = (-ws.data_ptr()) % 256
    return ctypes.c_void_p(ws.data_ptr() + off), ws.numel() - off


def restkv_prepare_wo(p, w_o: torch.Tensor, gram: torch.Tensor, stream=None):
    _chk(lib().restkv_prepare_wo(ctypes.byref(p), _ptr(w_o), w_o.shape[1], _ptr(gram), _stream(stream)),
         "restkv_prepare_wo")


def restkv_score(p, q, k, v, gram, score, workspace, stream=None):
    wp, wn = _ws(workspace)
    _chk(lib().restkv_score(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(gram), _ptr(score),
                            wp, wn, _stream(stream)), "restkv_score")


def restkv_score_from_attention(p, q, k, v, gram, attn_out, lse, score, workspace, stream=None):
    wp, wn = _ws(workspace)
    _chk(lib().restkv_score_from_attention(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(gram), _ptr(attn_out),
                                           _ptr(lse), _ptr(score), wp, wn, _stream(stream)),
         "restkv_score_from_attention")


def restkv_smooth(p, score, ema, final, aws_info, aws_d, workspace, stream=None):
    wp, wn = _ws(workspace)
    _chk(lib().restkv_smooth(ctypes.byref(p), _ptr(score), _ptr(ema), _ptr(final), _ptr(aws_info),
                             _ptr(aws_d), wp, wn, _stream(stream)), "restkv_smooth")


def restkv_score_smooth(p, q, k, v, gram, score, ema, final, aws_info, aws_d, workspace, stream=None):
    wp, wn = _ws(workspace)
    _chk(lib().restkv_score_smooth(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(gram), _ptr(score),
                                   _ptr(ema), _ptr(final), _ptr(aws_info), _ptr(aws_d), wp, wn,
                                   _stream(stream)), "restkv_score_smooth")


def restkv_smooth_b(p, score, head_budget, ema, final, aws_info, aws_d, workspace, stream=None):
    wp, wn = _ws(workspace)
    _chk(lib().restkv_smooth_b(ctypes.byref(p), _ptr(score), _ptr(head_budget), _ptr(ema), _ptr(final),
                               _ptr(aws_info), _ptr(aws_d), wp, wn, _stream(stream)), "restkv_smooth_b")


def restkv_select_b(p, final, head_budget, idx, workspace, stream=None):
    wp, wn = _ws(workspace)
    _chk(lib().restkv_select_b(ctypes.byref(p), _ptr(final), _ptr(head_budget), _ptr(idx), wp, wn,
                               _stream(stream)), "restkv_select_b")


def restkv_select(p, final, idx, workspace, stream=None):
    wp, wn = _ws(workspace)
    _chk(lib().restkv_select(ctypes.byref(p), _ptr(final), _ptr(idx), wp, wn, _stream(stream)),
         "restkv_select")


def restkv_select_static(p, final, idx, stream=None):
    _chk(lib().restkv_select_static(ctypes.byref(p), _ptr(final), _ptr(idx), _stream(stream)),
         "restkv_select_static")


def restkv_select_static_capacity() -> int:
    return int(lib().restkv_select_static_capacity())


def restkv_compact(p, k, v, idx, k_out, v_out, stream=None):
    _chk(lib().restkv_compact(ctypes.byref(p), _ptr(k), _ptr(v), _ptr(idx), _ptr(k_out), _ptr(v_out),
                              _stream(stream)), "restkv_compact")


N_STAGES = 10


def restkv_timing_enable(on):
    """True / False, or a collection of stage names to time only those (see restkv_timing_read)."""
    if isinstance(on, (bool, int)):
        mask = -1 if on else 0
    else:
        names = [lib().restkv_stage_name(s).decode() for s in range(N_STAGES)]
        mask = 0
        for name in on:
            mask |= 1 << names.index(name)
    _chk(lib().restkv_timing_enable(mask), "restkv_timing_enable")


def restkv_timing_read():
    """{stage name: (total ms, launches)} since the last read; waits for the recorded events."""
    ms = (ctypes.c_double * N_STAGES)()
    cnt = (ctypes.c_int64 * N_STAGES)()
    _chk(lib().restkv_timing_read(ms, cnt, N_STAGES), "restkv_timing_read")
    return {lib().restkv_stage_name(s).decode(): (ms[s], cnt[s]) for s in range(N_STAGES)}


def restkv_debug_force_fp32(on: bool):
    _chk(lib().restkv_debug_force_fp32(int(bool(on))), "restkv_debug_force_fp32")


def restkv_debug_score_plan(p):
    """(key splits, 64-key tiles of a split, side by side, heavy weights in two parts) of the attention pass on the bf16 matrix-core path."""
    plan = (ctypes.c_int32 * 4)()
    _chk(lib().restkv_debug_score_plan(ctypes.byref(p), plan), "restkv_debug_score_plan")
    return tuple(plan)


def restkv_debug_fp32_plan(p):
    """(key splits, value-Gram pass in the attention launch, wavefronts of a score workgroup, these divide the heads) of a float32 layer."""
    plan = (ctypes.c_int32 * 4)()
    _chk(lib().restkv_debug_fp32_plan(ctypes.byref(p), plan), "restkv_debug_fp32_plan")
    return tuple(plan)


def restkv_stream_reference(src: Optional[torch.Tensor], read_bytes: int, dst: Optional[torch.Tensor],
                            write_bytes: int, stream=None):
    """Plain streaming kernel with a given read / write byte mix (a measurement aid)."""
    _chk(lib().restkv_stream_reference(_ptr(src), int(read_bytes), _ptr(dst), int(write_bytes), _stream(stream)),
         "restkv_stream_reference")


def restkv_version() -> int:
    return int(lib().restkv_version())


@dataclass
class LayerBuffers:
    """Device buffers of one layer's pass (allocated once, reused across layers)."""
    score: torch.Tensor
    ema: torch.Tensor
    final: torch.Tensor
    aws_info: torch.Tensor
    aws_d: torch.Tensor
    idx: torch.Tensor
    k_out: torch.Tensor
    v_out: torch.Tensor
    workspace: torch.Tensor


def alloc_layer_buffers(p: RestkvParams, dtype: torch.dtype, device="cuda") -> LayerBuffers:
    Hkv, W, B, d = p.n_kv_heads, p.window, p.budget, p.head_dim
    ld = p.ld_score if p.ld_score else p.seq_len - p.window
    f32 = dict(dtype=torch.float32, device=device)
    return LayerBuffers(
        score=torch.empty((Hkv, W, ld), **f32), ema=torch.empty((Hkv, ld), **f32),
        final=torch.empty((Hkv, ld), **f32),
        aws_info=torch.empty((Hkv, 2), dtype=torch.int32, device=device),
        aws_d=torch.empty((Hkv, 2), dtype=torch.float64, device=device),
        idx=torch.empty((Hkv, B), dtype=torch.int32, device=device),
        k_out=torch.empty((Hkv, B, d), dtype=dtype, device=device),
        v_out=torch.empty((Hkv, B, d), dtype=dtype, device=device),
        workspace=alloc_workspace(p, device))


def evict_layer(p: RestkvParams, q, k, v, gram, buf: LayerBuffers, stream=None, fused=False):
    """The stages of one layer on one stream (no host synchronisation): one call, or with fused=True the fused call
    of score and smoothing (restkv_score_smooth), then selection and gather."""
    if fused:
        restkv_score_smooth(p, q, k, v, gram, buf.score, buf.ema, buf.final, buf.aws_info, buf.aws_d, buf.workspace, stream)
        restkv_select(p, buf.final, buf.idx, buf.workspace, stream)
        restkv_compact(p, k, v, buf.idx, buf.k_out, buf.v_out, stream)
        return
    wp, wn = _ws(buf.workspace)
    _chk(lib().restkv_evict(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(gram), _ptr(buf.score), _ptr(buf.ema),
                            _ptr(buf.final), _ptr(buf.aws_info), _ptr(buf.aws_d), _ptr(buf.idx), _ptr(buf.k_out),
                            _ptr(buf.v_out), wp, wn, _stream(stream)), "restkv_evict")


# ---- paged cache ------------------------------------------------------------------------------
# Unlike the calls above these check their tensors: what a description says of them is what the kernels go by.

_TYPES = {torch.float32: RESTKV_F32, torch.bfloat16: RESTKV_BF16, "f32": RESTKV_F32, "bf16": RESTKV_BF16, "q4": RESTKV_Q4}
_TORCH = {RESTKV_F32: torch.float32, RESTKV_BF16: torch.bfloat16, RESTKV_Q4: torch.uint8}


def make_cache(*, n_seqs, n_q_heads, n_kv_heads, head_dim, page_size, n_pages, max_pages, dtype, format=None, max_new=1,
               n_tokens=None, max_len=0, causal=True, scale=0.0, rotary_dim=0, interleaved=False, n_positions=0, out_dtype=None,
               token_major=False, head_lens=False, head_tables=False, out_head_major=False, page_strides=None) -> RestkvCache:
    """Description of a paged cache and of the calls on it (see restkv_cache in include/restkv.h).

    n_tokens: rows of the packed token tensors (default n_seqs * max_new).  token_major: pages [n_pages, page_size, Hkv, ..]
    in place of [n_pages, Hkv, page_size, ..].  head_lens: lens [n_seqs, Hkv] in place of [n_seqs].  head_tables: table
    [n_seqs, Hkv, max_pages] in place of [n_seqs, max_pages], and pages of one head.  page_strides: (page, head, position)
    in rows, of arrays that are not contiguous.  Strides of token tensors are taken from the tensors of each call.

    The calls refuse a table, lens, new_start, cos, sin [n_positions, rotary_dim / 2], positions [n_tokens] or idx of another shape
    (table, lens, new_start, cos and sin may have more rows); where strides are set by hand it has to be as long as is read."""
    dt = int(_TYPES.get(dtype, dtype))
    fmt = dt if format is None else int(_TYPES.get(format, format))
    heads = 1 if head_tables else n_kv_heads
    c = RestkvCache(n_seqs, n_q_heads, n_kv_heads, head_dim, dt, fmt, page_size, n_pages, max_pages, max_len, max_new,
                    n_seqs * max_new if n_tokens is None else n_tokens, int(bool(causal)), rotary_dim, int(bool(interleaved)),
                    n_positions, dt if out_dtype is None else int(_TYPES.get(out_dtype, out_dtype)), float(scale))
    c.page_stride, c.head_stride, c.token_stride = page_strides or (
        page_size * heads, 0 if head_tables else 1 if token_major else page_size, heads if token_major else 1)
    c.table_stride_s, c.table_stride_h = (n_kv_heads * max_pages, max_pages) if head_tables else (max_pages, 0)
    c.lens_stride_s, c.lens_stride_h = (n_kv_heads, 1) if head_lens else (1, 0)
    c.q_stride_t, c.q_stride_h, c.kv_stride_t, c.kv_stride_h = n_q_heads * head_dim, head_dim, n_kv_heads * head_dim, head_dim
    c.out_stride_t, c.out_stride_h, c.lse_stride_t, c.lse_stride_h = n_q_heads * head_dim, head_dim, n_q_heads, 1
    if out_head_major:
        n = max(c.n_tokens, 1)
        c.out_stride_t, c.out_stride_h, c.lse_stride_t, c.lse_stride_h = head_dim, n * head_dim, 1, n
    return c


@dataclass(frozen=True)
class CachePages:
    """The arrays of a paged cache: k, v [n_pages, Hkv, page_size, d] ([n_pages, page_size, Hkv, d] token-major) of the
    cache's type, or for 4 bits uint8 [..., d/2] with k_scale, v_scale bfloat16 [..., d/32, 2] ({step, zero})."""
    k: torch.Tensor
    v: torch.Tensor
    k_scale: Optional[torch.Tensor] = None
    v_scale: Optional[torch.Tensor] = None
    rows: tuple = field(init=False, repr=False)      # shape and strides in rows of all arrays, checked once

    def __post_init__(self):
        q4 = self.k.dtype == torch.uint8
        arrays = [self.k, self.v]
        if q4:
            arrays += [self.k_scale, self.v_scale]
        elif self.k_scale is not None or self.v_scale is not None:
            raise RestkvError(-1, "CachePages: scales go with codes (uint8)")
        seen = set()
        for n, x in enumerate(arrays):
            if x is None:
                raise RestkvError(-1, "CachePages: codes come with k_scale and v_scale")
            tail = x.shape[3:]
            size = tail.numel()
            if x.dim() != (5 if n > 1 else 4) or x.stride()[3:] != ((2, 1) if n > 1 else (1,)) or \
                    any(st % size for st in x.stride()[:3]):
                raise RestkvError(-1, "CachePages: rows that are contiguous, a whole number of rows apart")
            if x.dtype != (torch.bfloat16 if n > 1 else self.k.dtype) or x.device != self.k.device or \
                    (n > 1 and (tail[0] * 16 != self.k.shape[3] or tail[1] != 2)) or (n == 1 and tail != self.k.shape[3:]):
                raise RestkvError(-1, "CachePages: arrays of one cache on one device")
            seen.add((tuple(x.shape[:3]), tuple(st // size for st in x.stride()[:3])))
        if len(seen) != 1:
            raise RestkvError(-1, "CachePages: all arrays of one layout")
        object.__setattr__(self, "rows", seen.pop() + (self.k.dtype, self.k.shape[3] * (2 if q4 else 1), self.k.get_device()))


def alloc_cache_pages(c: RestkvCache, device="cuda") -> CachePages:
    """Pages of the described cache (contiguous), zeroed."""
    heads = 1 if c.head_stride == 0 else c.n_kv_heads
    token_major = heads > 1 and c.token_stride >= heads
    shape = (c.n_pages, c.page_size, heads) if token_major else (c.n_pages, heads, c.page_size)
    d = c.head_dim
    if c.format != RESTKV_Q4:
        return CachePages(*(torch.zeros(shape + (d,), dtype=_TORCH[c.format], device=device) for _ in range(2)))
    return CachePages(*(torch.zeros(shape + (d // 2,), dtype=torch.uint8, device=device) for _ in range(2)),
                      *(torch.zeros(shape + (d // 32, 2), dtype=torch.bfloat16, device=device) for _ in range(2)))


def restkv_attend_workspace_bytes(c: RestkvCache) -> int:
    return int(lib().restkv_attend_workspace_bytes(ctypes.byref(c)))


def alloc_attend_workspace(c: RestkvCache, device="cuda") -> Optional[torch.Tensor]:
    """Scratch of restkv_attend, or None where it needs none."""
    n = restkv_attend_workspace_bytes(c)
    return torch.empty(n + 256, dtype=torch.uint8, device=device) if n else None


class _Told:
    """What a description says of the tensors of a call, worked out once (a field that is set makes it new).  It hangs on the description, so
    nothing here refers to that, not by ctypes.byref either: the two would keep each other for ever."""

    def __init__(self, c: RestkvCache):
        self.dtype, self.out_dtype = _TORCH.get(c.dtype), _TORCH.get(c.out_dtype)
        self.kv, self.q, self.lse = ((c.n_tokens, c.n_kv_heads, c.head_dim), (c.n_tokens, c.n_q_heads, c.head_dim),
                                     (c.n_tokens, c.n_q_heads))
        self.kv_stride, self.q_stride, self.out_stride, self.lse_stride = (
            (c.kv_stride_t, c.kv_stride_h, 1), (c.q_stride_t, c.q_stride_h, 1), (c.out_stride_t, c.out_stride_h, 1),
            (c.lse_stride_t, c.lse_stride_h))
        # flat arrays, as _check_flat takes them; where strides set by hand say more than a shape does, by the entries from the first
        # to the last that is read (strides 0, 0: the library's own)
        span = lambda s, h, n, default: ((c.n_seqs - 1) * (s if s or h else default) + (c.n_kv_heads - 1) * h + n) * (c.n_seqs > 0)  # noqa: E731
        n_seqs, heads, width, i32 = c.n_seqs, c.n_kv_heads, c.max_pages, torch.int32
        self.n_table = span(c.table_stride_s, c.table_stride_h, width, width)
        self.n_lens = span(c.lens_stride_s, c.lens_stride_h, 1, 1)
        shape = {(0, 0): (n_seqs, width), (width, 0): (n_seqs, width), (heads * width, width): (n_seqs, heads, width)}
        self.table = (shape.get((c.table_stride_s, c.table_stride_h)), i32, "table", self.n_table)
        shape = {(0, 0): (n_seqs,), (1, 0): (n_seqs,), (heads, 1): (n_seqs, heads)}
        self.lens = (shape.get((c.lens_stride_s, c.lens_stride_h)), i32, "lens", self.n_lens)
        self.new = ((n_seqs + 1,), i32, "new_start", 0)
        self.cos, self.sin = (((c.n_positions, c.rotary_dim // 2), torch.float32, name, 0) for name in ("cos", "sin"))
        self.turns = c.n_positions * (c.rotary_dim // 2) != 0
        self.positions = ((c.n_tokens,), i32, "positions", None)
        self.grid = ((n_seqs, c.max_new), i32, "positions", None) if n_seqs * c.max_new == c.n_tokens else self.positions
        self.pages = None                    # the last layout of pages that was found to be the described one
        self.n_seqs, self.shared = n_seqs, {}            # shared pages of groups, by their beams


def _told(c: RestkvCache) -> _Told:
    t = c.__dict__.get("told")
    if t is None:
        t = c.__dict__["told"] = _Told(c)
    return t


def _check_pages(what: str, c: RestkvCache, told: _Told, pages: CachePages) -> int:
    """The GPU that the cache is on."""
    rows = pages.rows
    if rows == told.pages:
        return rows[4]
    shape, strides, dtype, d, dev = rows
    page, head, pos = c.page_stride, c.head_stride, c.token_stride
    if not pos:
        page, head, pos = c.page_size * c.n_kv_heads, c.page_size, 1
    heads = 1 if c.table_stride_h and not head else c.n_kv_heads
    # (a stride along one entry says nothing)
    as_told = [(shape[0] >= c.n_pages and a == heads and b == c.page_size and (strides[0] == page or c.n_pages == 1) and
                (sa == head or a == 1) and sb == pos)
               for a, b, sa, sb in ((shape[1], shape[2], strides[1], strides[2]), (shape[2], shape[1], strides[2], strides[1]))]
    if not any(as_told) or d != c.head_dim or dtype != _TORCH.get(c.format):
        raise RestkvError(-1, f"{what}: pages {shape} with strides {strides} in rows of {d} {dtype} are not the described ones")
    if dev < 0:
        raise RestkvError(-1, f"{what}: the pages are not on a GPU")
    told.pages = rows
    return dev


def _reads_as(t, shape, n) -> bool:
    """Whether a contiguous tensor holds the described values where the kernels look for them: the same but for dimensions of
    one, its rows one after the other, or (unless n is None) with rows behind the last that is read; without a shape n values."""
    if shape is None:
        return t.numel() >= n
    got, total = t.shape, math.prod(shape)
    if not total or (len(got) == 1 and got[0] == total):
        return True
    if n is not None and len(got) == len(shape) and got[1:] == shape[1:] and got[0] >= shape[0]:
        return True
    return [x for x in got if x != 1] == [x for x in shape if x != 1]


def _check_flat(what, dev, t, told):
    """Address of a contiguous tensor that is as told: (shape, type, name, n); see _reads_as."""
    shape, dtype, name, n = told
    if t is None or t.dtype is not dtype or t.get_device() != dev or not t.is_contiguous() or \
            (t.shape != shape and not _reads_as(t, shape, n)):
        raise RestkvError(-1, f"{what}: {name} has to be contiguous {dtype}, {shape or n} values on GPU {dev}")
    return t.data_ptr()


def _check_rows(what, dev, dtype, name, t, shape, strides):
    """Strides of a tensor [tokens, heads, d] or [tokens, heads], those given where it has them."""
    if t.dtype is not dtype or t.get_device() != dev or t.shape != shape:
        raise RestkvError(-1, f"{what}: {name} has to be {dtype} {tuple(shape)} on GPU {dev}")
    st = t.stride()
    if st == strides:
        return strides
    least = shape[2] if len(shape) == 3 else 1
    if len(shape) == 3 and st[2] != 1:
        raise RestkvError(-1, f"{what}: {name} has to be contiguous along its last dimension")
    # (a stride along one entry, or none, says nothing; the library asks for one that a contiguous tensor could have)
    along, across = st[0] if shape[0] > 1 else shape[1] * least, st[1] if shape[1] > 1 else least
    if along < least or across < least:
        raise RestkvError(-1, f"{what}: rows of {name} overlap")
    return (along, across) + strides[2:]


def _as_strided(c: RestkvCache, **strides) -> RestkvCache:
    """A copy of the description with these strides of token tensors."""
    c = RestkvCache.from_buffer_copy(c)
    for kind, st in strides.items():
        setattr(c, kind + "_stride_t", st[0])
        setattr(c, kind + "_stride_h", st[1])
    return c


def _on_gpu(dev: int, stream, what: str, f, *args):
    """The call on GPU `dev`, on the given stream or that GPU's current one."""
    # (torch's own lookup without the Stream object around it: 0.1 us of 1.1, of a call of 10)
    s = torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream
    if dev == torch.cuda.current_device():
        rc = f(*args, s)
    else:
        with torch.cuda.device(dev):
            rc = f(*args, s)
    if rc:
        raise RestkvError(rc, what)


def _addr(t):
    return None if t is None else t.data_ptr()


def restkv_append(c: RestkvCache, k, v, pages: CachePages, table, lens, *, new_start=None, positions=None, cos=None, sin=None,
                  q=None, q_out=None, stream=None):
    """New keys (rotated by their positions) and values [n_tokens, Hkv, d] into the pages, and new queries [n_tokens, Hq, d]
    rotated beside them; lens counts the new tokens already."""
    what, told = "restkv_append", _told(c)
    dev, dt, desc = _check_pages(what, c, told, pages), told.dtype, c
    tb, ln = _check_flat(what, dev, table, told.table), _check_flat(what, dev, lens, told.lens)
    ns = None if new_start is None else _check_flat(what, dev, new_start, told.new)
    kv = _check_rows(what, dev, dt, "k", k, told.kv, told.kv_stride)
    if _check_rows(what, dev, dt, "v", v, told.kv, kv) != kv:
        raise RestkvError(-1, f"{what}: k and v have to have the same strides")
    qs = told.q_stride
    if q is not None and q_out is not None:
        qs = _check_rows(what, dev, dt, "q", q, told.q, qs)
        if q_out is not q and _check_rows(what, dev, dt, "q_out", q_out, told.q, qs) != qs:
            raise RestkvError(-1, f"{what}: q and q_out have to have the same strides")
    cs = sn = None
    if told.turns:
        cs, sn = _check_flat(what, dev, cos, told.cos), _check_flat(what, dev, sin, told.sin)
    ps = None
    if positions is not None:        # (or a row for each sequence, where each has max_new tokens)
        by_row = ns is None and positions.shape == told.grid[0]
        ps = _check_flat(what, dev, positions, told.grid if by_row else told.positions)
    if kv is not told.kv_stride or qs is not told.q_stride:
        desc = _as_strided(c, kv=kv, q=qs)
    _on_gpu(dev, stream, what, lib().restkv_append, desc, k.data_ptr(), v.data_ptr(), pages.k.data_ptr(), pages.v.data_ptr(),
            _addr(pages.k_scale), _addr(pages.v_scale), tb, ln, ns, ps, cs, sn, _addr(q), _addr(q_out))


def restkv_attend(c: RestkvCache, q, pages: CachePages, table, lens, out, lse=None, workspace=None, *, new_start=None,
                  stream=None):
    """Attention of the newest tokens' queries q [n_tokens, Hq, d] over the pages: out [n_tokens, Hq, d], lse [n_tokens, Hq]."""
    what, told = "restkv_attend", _told(c)
    dev, desc = _check_pages(what, c, told, pages), c
    tb, ln = _check_flat(what, dev, table, told.table), _check_flat(what, dev, lens, told.lens)
    ns = None if new_start is None else _check_flat(what, dev, new_start, told.new)
    qs = _check_rows(what, dev, told.dtype, "q", q, told.q, told.q_stride)
    outs = _check_rows(what, dev, told.out_dtype, "out", out, told.q, told.out_stride)
    ls = told.lse_stride if lse is None else _check_rows(what, dev, torch.float32, "lse", lse, told.lse, told.lse_stride)
    if qs is not told.q_stride or outs is not told.out_stride or ls is not told.lse_stride:
        desc = _as_strided(c, q=qs, out=outs, lse=ls)
    wp, wn = None, 0
    if workspace is not None:
        if workspace.get_device() != dev or workspace.dtype is not torch.uint8 or not workspace.is_contiguous():
            raise RestkvError(-1, f"{what}: the workspace has to be contiguous uint8 on GPU {dev}")
        at = workspace.data_ptr()
        wp, wn = at + -at % 256, max(workspace.numel() - -at % 256, 0)
    _on_gpu(dev, stream, what, lib().restkv_attend, desc, q.data_ptr(), pages.k.data_ptr(), pages.v.data_ptr(), _addr(pages.k_scale),
            _addr(pages.v_scale), tb, ln, ns, out.data_ptr(), _addr(lse), wp, wn)


def restkv_fetch(c: RestkvCache, pages: CachePages, table, lens, k_out, v_out, *, idx=None, first=0, stream=None):
    """Rows of the pages as dense k_out, v_out [n_seqs, Hkv, n, d]: positions idx [n_seqs, Hkv, n], or first .. first + n - 1."""
    what, told = "restkv_fetch", _told(c)
    dev = _check_pages(what, c, told, pages)
    tb, ln = _check_flat(what, dev, table, told.table), _check_flat(what, dev, lens, told.lens)
    shape = k_out.shape
    if len(shape) != 4 or shape != (c.n_seqs, c.n_kv_heads, shape[2], c.head_dim) or v_out.shape != shape:
        raise RestkvError(-1, f"{what}: k_out and v_out have to be [n_seqs, Hkv, n, d]")
    kp, vp = _check_flat(what, dev, k_out, (shape, told.dtype, "k_out", None)), _check_flat(what, dev, v_out, (shape, told.dtype, "v_out", None))
    ix = None if idx is None else _check_flat(what, dev, idx, (shape[:3], torch.int32, "idx", None))
    _on_gpu(dev, stream, what, lib().restkv_fetch, c, pages.k.data_ptr(), pages.v.data_ptr(), _addr(pages.k_scale),
            _addr(pages.v_scale), tb, ln, ix, int(first), shape[2], kp, vp)


# ---- beams --------------------------------------------------------------------------------------


def make_beams(*, n_groups, n_beams, n_vocab, dtype, n_out=None, end_token=-1, logit_stride=0) -> RestkvBeams:
    """Description of a choice of continuations (see restkv_beams in include/restkv.h): n_out (default n_beams) of each request's
    n_beams; end_token ends a beam (default: none does).  logit_stride: elements from one row of logits to the next, 0: n_vocab."""
    return RestkvBeams(n_groups, n_beams, n_vocab, n_beams if n_out is None else n_out, int(_TYPES.get(dtype, dtype)), end_token,
                       logit_stride)


def restkv_beam_workspace_bytes(b: RestkvBeams) -> int:
    return int(lib().restkv_beam_workspace_bytes(ctypes.byref(b)))


def alloc_beam_workspace(b: RestkvBeams, device="cuda") -> torch.Tensor:
    """Scratch of restkv_beam_select."""
    return torch.empty(restkv_beam_workspace_bytes(b) + 256, dtype=torch.uint8, device=device)


class _BeamsTold:
    """What a description says of the tensors of restkv_beam_select, worked out once (a field that is set makes it new)."""

    def __init__(self, b: RestkvBeams):
        self.dtype = _TORCH.get(b.dtype)
        rows, stride = b.n_groups * b.n_beams, b.logit_stride or b.n_vocab
        self.flat, self.flat_strides = (rows, b.n_vocab), (stride, 1)
        self.grouped, self.stride, self.many = (b.n_groups, b.n_beams, b.n_vocab), stride, (b.n_groups > 1, b.n_beams > 1, b.n_vocab > 1)
        into, of = (b.n_groups, b.n_out), (b.n_groups, b.n_beams)
        self.scores, self.finished = (of, torch.float32, "scores", None), (of, torch.int32, "finished", None)
        self.new_scores, self.new_finished = (into, torch.float32, "new_scores", None), (into, torch.int32, "new_finished", None)
        self.parents, self.tokens = (into, torch.int32, "parents", None), (into, torch.int32, "tokens", None)

    def takes(self, shape, strides) -> bool:
        """Whether logits of this shape are rows at the described distance (a stride along one entry says nothing)."""
        groups, beams, vocab = self.many
        if strides[-1] != 1 and vocab:
            return False
        if shape == self.flat:
            return strides[0] == self.stride or shape[0] <= 1
        return shape == self.grouped and (strides[1] == self.stride or not beams) and \
            (strides[0] == self.grouped[1] * self.stride or not groups)


def _take_workspace(what, dev, workspace):
    """Address (aligned) and bytes of a workspace, or None and 0."""
    if workspace is None:
        return None, 0
    if workspace.get_device() != dev or workspace.dtype is not torch.uint8 or not workspace.is_contiguous():
        raise RestkvError(-1, f"{what}: the workspace has to be contiguous uint8 on GPU {dev}")
    at = workspace.data_ptr()
    return at + -at % 256, max(workspace.numel() - -at % 256, 0)


def restkv_beam_select(b: RestkvBeams, logits, scores, new_scores, parents, tokens, workspace, *, finished=None, new_finished=None,
                       stream=None):
    """The n_out best continuations of each request, best first: new_scores, parents (beams), tokens [n_groups, n_out] from logits
    [n_groups * n_beams, n_vocab] (or [n_groups, n_beams, n_vocab]) and scores [n_groups, n_beams]; finished and new_finished
    (int32, nonzero: ended) beside them.  new_scores may be scores and new_finished finished, where n_out = n_beams."""
    what, dev = "restkv_beam_select", logits.get_device()
    told = b.__dict__.get("told")
    if told is None:
        told = b.__dict__["told"] = _BeamsTold(b)
    if dev < 0 or logits.dtype is not told.dtype or \
            ((logits.shape != told.flat or logits.stride() != told.flat_strides) and not told.takes(logits.shape, logits.stride())):
        raise RestkvError(-1, f"{what}: logits have to be {told.dtype} {told.flat}, rows {told.stride} apart, on a GPU")
    sc, ns = _check_flat(what, dev, scores, told.scores), _check_flat(what, dev, new_scores, told.new_scores)
    ps, tk = _check_flat(what, dev, parents, told.parents), _check_flat(what, dev, tokens, told.tokens)
    fn = None if finished is None else _check_flat(what, dev, finished, told.finished)
    nf = None if new_finished is None else _check_flat(what, dev, new_finished, told.new_finished)
    wp, wn = _take_workspace(what, dev, workspace)
    _on_gpu(dev, stream, what, lib().restkv_beam_select, b, logits.data_ptr(), sc, fn, ns, ps, tk, nf, wp, wn)


class CacheLayers:
    """The pages of a model's layers, all of one layout on one GPU, as restkv_beam_reorder takes them (kept while in use)."""

    def __init__(self, layers):
        self.pages = tuple(layers)
        if len({x.rows for x in self.pages}) > 1:
            raise RestkvError(-1, "CacheLayers: pages of one layout on one GPU")
        self.array = (RestkvLayerPages * len(self.pages))(*((x.k.data_ptr(), x.v.data_ptr(), _addr(x.k_scale), _addr(x.v_scale))
                                                           for x in self.pages))


def restkv_beam_reorder(c: RestkvCache, n_beams, parents, table, lens, layers, table_out=None, *, stream=None):
    """Beam b of each group of n_beams sequences goes on from beam parents[group, b] (int32, rows may be a stride apart): table_out
    (default: in place) names the pages, and in all layers (CacheLayers, or CachePages of each) the rows of pages that are not full
    are copied."""
    what, told = "restkv_beam_reorder", _told(c)
    if not isinstance(layers, CacheLayers):
        layers = CacheLayers(layers)
    dev = _check_pages(what, c, told, layers.pages[0]) if layers.pages else table.get_device()
    n_groups = c.n_seqs // n_beams if n_beams > 0 else 0
    tb, ln = _check_flat(what, dev, table, told.table), _check_flat(what, dev, lens, told.lens)
    to = tb if table_out is None else _check_flat(what, dev, table_out, told.table)
    st = parents.stride()
    if parents.dtype is not torch.int32 or parents.get_device() != dev or dev < 0 or parents.shape != (n_groups, n_beams) or \
            (st[1] != 1 and n_beams > 1) or (n_groups > 1 and st[0] < n_beams):
        raise RestkvError(-1, f"{what}: parents have to be int32 [{n_groups}, {n_beams}] on GPU {dev}, rows that do not overlap")
    _on_gpu(dev, stream, what, lib().restkv_beam_reorder, c, n_beams, parents.data_ptr(), st[0] if n_groups > 1 else 0, ln, tb, to,
            layers.array, len(layers.pages))


def restkv_attend_beams_workspace_bytes(c: RestkvCache, n_beams) -> int:
    return int(lib().restkv_attend_beams_workspace_bytes(ctypes.byref(c), n_beams))


def alloc_attend_beams_workspace(c: RestkvCache, n_beams, device="cuda") -> Optional[torch.Tensor]:
    """Scratch of restkv_attend_beams, or None where it needs none."""
    n = restkv_attend_beams_workspace_bytes(c, n_beams)
    return torch.empty(n + 256, dtype=torch.uint8, device=device) if n else None


def restkv_debug_force_shared(on: bool):
    _chk(lib().restkv_debug_force_shared(int(bool(on))), "restkv_debug_force_shared")


def restkv_debug_beams_list(c: RestkvCache, n_beams, tiles):
    """(chunks of shared positions, room for them, chunks of what beams have behind them, room) for entries of so many tiles (a host list),
    where restkv_attend_beams works by a list of chunks."""
    tiles, chunks = (ctypes.c_int32 * len(tiles))(*tiles), (ctypes.c_int32 * 4)()
    entries = (c.n_seqs // n_beams + c.n_seqs) * (c.n_kv_heads if c.lens_stride_h else 1) if n_beams > 0 else 0
    if len(tiles) != entries:
        raise RestkvError(-1, f"restkv_debug_beams_list: tiles of {entries} entries")
    _chk(lib().restkv_debug_beams_list(ctypes.byref(c), n_beams, tiles, chunks), "restkv_debug_beams_list")
    return tuple(chunks)


def restkv_attend_beams(c: RestkvCache, n_beams, shared, q, pages: CachePages, table, lens, out, lse=None, workspace=None, *,
                        new_start=None, stream=None):
    """restkv_attend where the tables of each n_beams neighbouring sequences begin with the same shared[group] pages (int32), which
    are read once for all of them."""
    what, told = "restkv_attend_beams", _told(c)
    dev, desc = _check_pages(what, c, told, pages), c
    of = told.shared.get(n_beams)
    if of is None:
        of = told.shared[n_beams] = ((told.n_seqs // max(n_beams, 1),), torch.int32, "shared", None)
    sh, tb, ln = _check_flat(what, dev, shared, of), _check_flat(what, dev, table, told.table), _check_flat(what, dev, lens, told.lens)
    ns = None if new_start is None else _check_flat(what, dev, new_start, told.new)
    qs = _check_rows(what, dev, told.dtype, "q", q, told.q, told.q_stride)
    outs = _check_rows(what, dev, told.out_dtype, "out", out, told.q, told.out_stride)
    ls = told.lse_stride if lse is None else _check_rows(what, dev, torch.float32, "lse", lse, told.lse, told.lse_stride)
    if qs is not told.q_stride or outs is not told.out_stride or ls is not told.lse_stride:
        desc = _as_strided(c, q=qs, out=outs, lse=ls)
    wp, wn = _take_workspace(what, dev, workspace)
    _on_gpu(dev, stream, what, lib().restkv_attend_beams, desc, n_beams, sh, q.data_ptr(), pages.k.data_ptr(), pages.v.data_ptr(),
            _addr(pages.k_scale), _addr(pages.v_scale), tb, ln, ns, out.data_ptr(), _addr(lse), wp, wn)
