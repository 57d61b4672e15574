"""ctypes binding of libgrowpage.so (include/growpage.h).

Argument marshalling only: tensors become device pointers, the current torch
stream becomes the HIP stream, and a non-zero status becomes GrowPageError.
Every step of the computation runs in the library's HIP kernels.  If the
library has not been built, importing a function raises instead of falling
back to anything else.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libgrowpage.so")

GP_F32, GP_BF16 = 0, 1
GP_OP_DECODE, GP_OP_SCORE, GP_OP_APPLY, GP_OP_SELECT = 0, 1, 2, 3
GP_COMPRESS, GP_GROW, GP_FALLBACK, GP_PREEMPT, GP_NOT_BOUNDARY = 0, 1, 2, 3, 4
GP_SHRINK = 5
GP_POLICY_GROWPAGE, GP_POLICY_FIXED, GP_POLICY_RANDOM, GP_POLICY_INVERSE, GP_POLICY_SHRINK = 0, 1, 2, 3, 4
GP_METRIC_TOP_P, GP_METRIC_ENTROPY = 0, 1
GP_DECODE_CHUNKS, GP_DECODE_MERGE, GP_DECODE_PREFIX = 1, 2, 4
GP_LAYOUT_SHIFT, GP_LAYOUT_FILL = 0, 1
GP_SCORE_WEIGHTS, GP_SCORE_COUNTS = 1, 2
PAGE_SIZE = 16
GP_ERR_SCRATCH = 5

EXPORTS = ("gp_update_summaries", "gp_decode_attention", "gp_decode_attention_noalloc", "gp_decode_attention_shared",
           "gp_decode_attention_stages", "gp_decode_step", "gp_boundary_score", "gp_boundary_score_stages",
           "gp_boundary_apply", "gp_boundary_select", "gp_boundary_decide", "gp_boundary_compact",
           "gp_release_held", "gp_append_step", "gp_append_rope", "gp_append_rope_q8", "gp_decode_attention_q8",
           "gp_page_bounds", "gp_page_bounds_q8", "gp_select_pages", "gp_decode_attention_pages",
           "gp_decode_attention_pages_q8", "gp_workspace_bytes", "gp_status_string", "gp_stream_read")


class GrowPageError(RuntimeError):
    def __init__(self, status: int, where: str):
        super().__init__(f"{where}: status {status} ({status_string(status)})")
        self.status = status


class _KVLayer(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("pool_pages", ctypes.c_int32),
                ("num_kv_heads", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int)]


class _KV8Layer(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("pool_pages", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("head_dim", ctypes.c_int32)]


class _PageState(ctypes.Structure):
    _fields_ = [("page_table", ctypes.c_void_p), ("num_pages", ctypes.c_void_p),
                ("seq_lens", ctypes.c_void_p), ("refcount", ctypes.c_void_p),
                ("free_list", ctypes.c_void_p), ("free_count", ctypes.c_void_p),
                ("num_reqs", ctypes.c_int32), ("max_pages", ctypes.c_int32),
                ("pool_pages", ctypes.c_int32)]


class _PrefixGroup(ctypes.Structure):
    _fields_ = [("first_req", ctypes.c_int32), ("num_reqs", ctypes.c_int32), ("prefix_pages", ctypes.c_int32)]


class _Params(ctypes.Structure):
    _fields_ = [("beta_s", ctypes.c_float), ("beta_l", ctypes.c_float), ("p", ctypes.c_float),
                ("tau", ctypes.c_float), ("scale", ctypes.c_float), ("rope_theta", ctypes.c_float),
                ("k_loc", ctypes.c_int32), ("reserve_pages", ctypes.c_int32),
                ("policy", ctypes.c_int32), ("metric", ctypes.c_int32), ("fixed_pages", ctypes.c_int32),
                ("min_capacity_pages", ctypes.c_int32), ("compress_prob", ctypes.c_float),
                ("shrink_threshold", ctypes.c_float), ("draws", ctypes.c_void_p), ("layout", ctypes.c_int32),
                ("select_skip_grows", ctypes.c_int32)]


_lib = None


def load() -> ctypes.CDLL:
    """Load the built library (raises if it is missing)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run `python -m paper_2609_03494_amd.build`")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, f32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_float, ctypes.c_size_t
    lib.gp_status_string.restype = ctypes.c_char_p
    lib.gp_status_string.argtypes = [ctypes.c_int]
    lib.gp_workspace_bytes.restype = sz
    lib.gp_workspace_bytes.argtypes = [i32] * 8 + [ctypes.c_int, i32]
    lib.gp_stream_read.restype = ctypes.c_int
    lib.gp_stream_read.argtypes = [vp, sz, vp, vp]
    lib.gp_update_summaries.restype = ctypes.c_int
    lib.gp_update_summaries.argtypes = [vp, ctypes.c_int, i32, i32, i32, vp, vp, vp, i32, f32, f32, vp]
    lib.gp_decode_attention.restype = ctypes.c_int
    lib.gp_decode_attention.argtypes = [ctypes.POINTER(_KVLayer), ctypes.POINTER(_PageState), vp, i32,
                                        f32, vp, vp, sz, vp]
    lib.gp_decode_attention_noalloc.restype = ctypes.c_int
    lib.gp_decode_attention_noalloc.argtypes = [ctypes.POINTER(_KVLayer), ctypes.POINTER(_PageState), vp,
                                                i32, f32, vp, vp]
    lib.gp_decode_attention_shared.restype = ctypes.c_int
    lib.gp_decode_attention_shared.argtypes = [ctypes.POINTER(_KVLayer), ctypes.POINTER(_PageState), vp, i32,
                                               f32, vp, ctypes.POINTER(_PrefixGroup), i32, i32, vp, sz, vp]
    lib.gp_decode_attention_stages.restype = ctypes.c_int
    lib.gp_decode_attention_stages.argtypes = [ctypes.POINTER(_KVLayer), ctypes.POINTER(_PageState), vp, i32,
                                               f32, vp, i32, vp, sz, vp]
    lib.gp_decode_step.restype = ctypes.c_int
    lib.gp_decode_step.argtypes = [ctypes.POINTER(_KVLayer), ctypes.POINTER(_PageState), vp, vp, i32, f32,
                                   vp, vp, vp, vp, i32, f32, f32, vp, vp, vp, i32, vp, sz, vp]
    lib.gp_boundary_score.restype = ctypes.c_int
    lib.gp_boundary_score.argtypes = [ctypes.POINTER(_KVLayer), ctypes.POINTER(_PageState), vp, vp, i32,
                                      vp, vp, vp, i32, i32, ctypes.POINTER(_Params), vp, vp, i32, vp,
                                      sz, vp]
    lib.gp_boundary_score_stages.restype = ctypes.c_int
    lib.gp_boundary_score_stages.argtypes = lib.gp_boundary_score.argtypes + [i32]
    lib.gp_boundary_apply.restype = ctypes.c_int
    apply_args = [ctypes.POINTER(_KVLayer), i32, ctypes.POINTER(_PageState), vp, i32,
                  vp, vp, i32, ctypes.POINTER(_Params), vp, vp, vp, vp, sz, vp]
    for name in ("gp_boundary_apply", "gp_boundary_select", "gp_boundary_compact"):
        getattr(lib, name).restype = ctypes.c_int
        getattr(lib, name).argtypes = apply_args
    lib.gp_boundary_decide.restype = ctypes.c_int
    lib.gp_boundary_decide.argtypes = apply_args + [i32]
    lib.gp_release_held.restype = ctypes.c_int
    lib.gp_release_held.argtypes = [ctypes.POINTER(_PageState), vp]
    lib.gp_append_step.restype = ctypes.c_int
    lib.gp_append_step.argtypes = [ctypes.POINTER(_KVLayer), i32, ctypes.POINTER(_PageState), vp, vp, vp, vp,
                                   i32, vp, vp, vp, i32, f32, f32, vp]
    i64, ps_p, kv_p, kv8_p = ctypes.c_int64, ctypes.POINTER(_PageState), ctypes.POINTER(_KVLayer), ctypes.POINTER(_KV8Layer)
    rope_args = [ps_p, vp, vp, i32, vp, i64, vp, vp, i64, vp, i64, i32, f32, i32, vp]
    pages_args = [ps_p, vp, i32, vp, i32, f32, vp, vp, sz, vp]
    for name, layer, rest in (("gp_append_rope", kv_p, rope_args), ("gp_append_rope_q8", kv8_p, rope_args),
                              ("gp_decode_attention_q8", kv8_p, [ps_p, vp, i32, f32, vp, vp, sz, vp]),
                              ("gp_page_bounds", kv_p, [ps_p, vp, i32, vp, vp]),
                              ("gp_page_bounds_q8", kv8_p, [ps_p, vp, i32, vp, vp]),
                              ("gp_decode_attention_pages", kv_p, pages_args),
                              ("gp_decode_attention_pages_q8", kv8_p, pages_args)):
        getattr(lib, name).restype = ctypes.c_int
        getattr(lib, name).argtypes = [layer] + rest
    lib.gp_select_pages.restype = ctypes.c_int
    lib.gp_select_pages.argtypes = [vp, ctypes.c_int, ps_p, vp, i32, i32, i32, i32, i32, i32, vp, vp, sz, vp]
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load().gp_status_string(int(status)).decode()


def _check(status: int, where: str) -> None:
    if status != 0:
        raise GrowPageError(status, where)


def _ptr(t: torch.Tensor | None) -> int | None:
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensors passed to the library must be contiguous")
    return t.data_ptr()


def _stream(stream) -> int:
    # (the current stream's handle alone: torch.cuda.current_stream() makes an object
    # around it, 2.8 us of a call of 10-14)
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()) if stream is None else stream.cuda_stream


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return GP_F32
    if t.dtype == torch.bfloat16:
        return GP_BF16
    raise ValueError(f"unsupported dtype {t.dtype}")


@dataclass
class KVLayer:
    """K and V pools [pool_pages, num_kv_heads, 16, head_dim] (float32 or bfloat16)."""
    k: torch.Tensor
    v: torch.Tensor

    def c(self) -> _KVLayer:
        pool, hkv, b, d = self.k.shape
        return _KVLayer(_ptr(self.k), _ptr(self.v), pool, hkv, b, d, _dtype_code(self.k))


_CODES = (torch.float8_e4m3fn, torch.uint8)


@dataclass
class KV8Layer:
    """An 8-bit cache: K and V pools [pool_pages, num_kv_heads, 16, head_dim] of e4m3
    codes (float8_e4m3fn or uint8) and their scales [pool_pages, num_kv_heads] float32."""
    k: torch.Tensor
    v: torch.Tensor
    k_scale: torch.Tensor
    v_scale: torch.Tensor

    def c(self) -> _KV8Layer:
        k, v, ks, vs = self.k, self.v, self.k_scale, self.v_scale
        shape = k.shape
        if v.shape != shape or k.dtype not in _CODES or v.dtype not in _CODES:
            raise ValueError("8-bit pools: two tensors of one shape, float8_e4m3fn or uint8")
        pool, hkv, b, d = shape
        if ks.dtype != torch.float32 or vs.dtype != torch.float32 or ks.shape != (pool, hkv) or vs.shape != (pool, hkv):
            raise ValueError("scales of an 8-bit cache: float32 [pool_pages, num_kv_heads]")
        return _KV8Layer(_ptr(k), _ptr(v), _ptr(ks), _ptr(vs), pool, hkv, b, d)


@dataclass
class PageState:
    """Device page state (int32 tensors).  free_count is a one-element tensor."""
    page_table: torch.Tensor   # [R, max_pages]
    num_pages: torch.Tensor    # [R]
    seq_lens: torch.Tensor     # [R]
    refcount: torch.Tensor     # [pool_pages]
    free_list: torch.Tensor    # [pool_pages]
    free_count: torch.Tensor   # [1]

    def c(self) -> _PageState:
        R, maxp = self.page_table.shape
        return _PageState(_ptr(self.page_table), _ptr(self.num_pages), _ptr(self.seq_lens),
                          _ptr(self.refcount), _ptr(self.free_list), _ptr(self.free_count),
                          R, maxp, self.refcount.shape[0])


@dataclass
class Params:
    beta_s: float = 0.9
    beta_l: float = 0.999
    p: float = 0.99
    tau: float = 0.0
    scale: float = 1.0 / 128 ** 0.5
    rope_theta: float = 1.0e6
    k_loc: int = 4
    reserve_pages: int = 0
    policy: int = 0                 # GP_POLICY_*
    metric: int = 0                 # GP_METRIC_*
    fixed_pages: int = 256
    min_capacity_pages: int = 64
    compress_prob: float = 0.7
    shrink_threshold: float = -0.005
    draws: torch.Tensor | None = None   # [num_bnd] float32 on the device (RANDOM only)
    layout: int = 0                 # GP_LAYOUT_*
    select_skip_grows: int = 0      # gp_boundary_select: k_counts are final (see the header)

    def c(self) -> _Params:
        if self.draws is not None and (self.draws.dtype != torch.float32 or not self.draws.is_contiguous()):
            raise ValueError("draws must be a contiguous float32 tensor")
        return _Params(self.beta_s, self.beta_l, self.p, self.tau, self.scale, self.rope_theta,
                       self.k_loc, self.reserve_pages, self.policy, self.metric, self.fixed_pages,
                       self.min_capacity_pages, self.compress_prob, self.shrink_threshold,
                       _ptr(self.draws), self.layout, self.select_skip_grows)


def gp_workspace_bytes(op: int, num_reqs: int, num_bnd: int, num_q_heads: int, num_kv_heads: int,
                       head_dim: int, max_pages: int, dtype: torch.dtype, n_layers: int = 1) -> int:
    code = GP_F32 if dtype == torch.float32 else GP_BF16
    n = load().gp_workspace_bytes(op, num_reqs, num_bnd, num_q_heads, num_kv_heads, head_dim,
                                  max_pages, PAGE_SIZE, code, n_layers)
    if n == 0:
        raise GrowPageError(2, "gp_workspace_bytes")
    return int(n)


def workspace(op: int, num_reqs: int, num_bnd: int, num_q_heads: int, num_kv_heads: int,
              head_dim: int, max_pages: int, dtype: torch.dtype, n_layers: int = 1,
              device="cuda") -> torch.Tensor:
    """A zero-filled workspace of the size the library asks for."""
    n = gp_workspace_bytes(op, num_reqs, num_bnd, num_q_heads, num_kv_heads, head_dim, max_pages,
                           dtype, n_layers)
    return torch.zeros(n, dtype=torch.uint8, device=device)


def gp_update_summaries(q_pre: torch.Tensor, slot_ids: torch.Tensor, init: torch.Tensor,
                        qstate: torch.Tensor, beta_s: float, beta_l: float, stream=None) -> None:
    R, Hq, d = q_pre.shape
    st = load().gp_update_summaries(_ptr(q_pre), _dtype_code(q_pre), R, Hq, d, _ptr(slot_ids),
                                    _ptr(init), _ptr(qstate), qstate.shape[0], beta_s, beta_l,
                                    _stream(stream))
    _check(st, "gp_update_summaries")


def gp_decode_attention(kv: KVLayer, ps: PageState, q_post: torch.Tensor, scale: float,
                        out: torch.Tensor, ws: torch.Tensor, stream=None) -> None:
    c_kv, c_ps = kv.c(), ps.c()
    st = load().gp_decode_attention(ctypes.byref(c_kv), ctypes.byref(c_ps), _ptr(q_post),
                                    q_post.shape[1], scale, _ptr(out), _ptr(ws), ws.numel(),
                                    _stream(stream))
    _check(st, "gp_decode_attention")


def gp_stream_read(src: torch.Tensor, out: torch.Tensor, stream=None) -> None:
    """The streaming-read reference kernel over src's bytes (XOR into out[0],
    an int32 device tensor)."""
    st = load().gp_stream_read(_ptr(src), src.numel() * src.element_size(), _ptr(out), _stream(stream))
    _check(st, "gp_stream_read")


def gp_decode_attention_noalloc(kv: KVLayer, ps: PageState, q_post: torch.Tensor, scale: float,
                                out: torch.Tensor, stream=None) -> None:
    """gp_decode_attention with its partials in the library's static scratch
    (no workspace, nothing allocated)."""
    c_kv, c_ps = kv.c(), ps.c()
    st = load().gp_decode_attention_noalloc(ctypes.byref(c_kv), ctypes.byref(c_ps), _ptr(q_post),
                                            q_post.shape[1], scale, _ptr(out), _stream(stream))
    _check(st, "gp_decode_attention_noalloc")


def gp_decode_attention_shared(kv: KVLayer, ps: PageState, q_post: torch.Tensor, scale: float,
                               out: torch.Tensor, groups, ws: torch.Tensor,
                               stages: int = GP_DECODE_PREFIX | GP_DECODE_CHUNKS | GP_DECODE_MERGE,
                               stream=None) -> None:
    """Decode attention with shared-prefix groups: ``groups`` is a list of
    (first_req, num_reqs, prefix_pages); ``stages`` any of GP_DECODE_PREFIX,
    GP_DECODE_CHUNKS, GP_DECODE_MERGE."""
    arr = (_PrefixGroup * max(len(groups), 1))(*[_PrefixGroup(*map(int, g)) for g in groups])
    c_kv, c_ps = kv.c(), ps.c()
    st = load().gp_decode_attention_shared(ctypes.byref(c_kv), ctypes.byref(c_ps), _ptr(q_post),
                                           q_post.shape[1], scale, _ptr(out), arr, len(groups), int(stages),
                                           _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "gp_decode_attention_shared")


def gp_decode_attention_stages(kv: KVLayer, ps: PageState, q_post: torch.Tensor, scale: float,
                               out: torch.Tensor, stages: int, ws: torch.Tensor, stream=None) -> None:
    """Decode attention's chunk pass (GP_DECODE_CHUNKS) and/or merge (GP_DECODE_MERGE)."""
    c_kv, c_ps = kv.c(), ps.c()
    st = load().gp_decode_attention_stages(ctypes.byref(c_kv), ctypes.byref(c_ps), _ptr(q_post),
                                           q_post.shape[1], scale, _ptr(out), stages, _ptr(ws), ws.numel(),
                                           _stream(stream))
    _check(st, "gp_decode_attention_stages")


def gp_decode_step(kv: KVLayer, ps: PageState, q_post: torch.Tensor, q_pre: torch.Tensor, scale: float,
                   out: torch.Tensor, slot_ids: torch.Tensor, init: torch.Tensor, qstate: torch.Tensor,
                   beta_s: float, beta_l: float, ws: torch.Tensor, k_new: torch.Tensor | None = None,
                   v_new: torch.Tensor | None = None, positions: torch.Tensor | None = None,
                   advance: bool = True, stream=None) -> None:
    """The step's new token (k_new, v_new [R][Hkv][d], optional), the summary
    update and decode attention in one launch."""
    c_kv, c_ps = kv.c(), ps.c()
    st = load().gp_decode_step(ctypes.byref(c_kv), ctypes.byref(c_ps), _ptr(q_post), _ptr(q_pre),
                               q_post.shape[1], scale, _ptr(out), _ptr(slot_ids), _ptr(init),
                               _ptr(qstate), qstate.shape[0], beta_s, beta_l, _ptr(k_new), _ptr(v_new),
                               _ptr(positions), int(bool(advance)), _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "gp_decode_step")


def gp_boundary_score(kv: KVLayer, ps: PageState, q_pre: torch.Tensor, qstate: torch.Tensor,
                      slot_ids: torch.Tensor, positions: torch.Tensor, bnd: torch.Tensor,
                      params: Params, k_counts: torch.Tensor, scores: torch.Tensor,
                      ws: torch.Tensor, stream=None, stages=None) -> None:
    """stages None: gp_boundary_score; else gp_boundary_score_stages with that
    mask (GP_SCORE_WEIGHTS, GP_SCORE_COUNTS)."""
    c_kv, c_ps, c_p = kv.c(), ps.c(), params.c()
    args = (ctypes.byref(c_kv), ctypes.byref(c_ps), _ptr(q_pre), _ptr(qstate), qstate.shape[0], _ptr(slot_ids),
            _ptr(positions), _ptr(bnd), bnd.shape[0], q_pre.shape[1], ctypes.byref(c_p), _ptr(k_counts),
            _ptr(scores), scores.shape[-1], _ptr(ws), ws.numel(), _stream(stream))
    if stages is None:
        _check(load().gp_boundary_score(*args), "gp_boundary_score")
    else:
        _check(load().gp_boundary_score_stages(*args, stages), "gp_boundary_score_stages")


def _apply_like(name, layers, ps, bnd, k_counts, scores, params, decisions, delta, counters, ws, stream,
                *extra) -> None:
    arr = (_KVLayer * len(layers))(*[layer.c() for layer in layers])
    c_ps, c_p = ps.c(), params.c()
    st = getattr(load(), name)(arr, len(layers), ctypes.byref(c_ps), _ptr(bnd), bnd.shape[0],
                               _ptr(k_counts), _ptr(scores), scores.shape[-1], ctypes.byref(c_p),
                               _ptr(decisions), _ptr(delta), _ptr(counters), _ptr(ws),
                               ws.numel(), _stream(stream), *extra)
    _check(st, name)


def gp_boundary_apply(layers: list[KVLayer], ps: PageState, bnd: torch.Tensor,
                      k_counts: torch.Tensor, scores: torch.Tensor, params: Params,
                      decisions: torch.Tensor, delta: torch.Tensor, counters: torch.Tensor,
                      ws: torch.Tensor, stream=None) -> None:
    _apply_like("gp_boundary_apply", layers, ps, bnd, k_counts, scores, params, decisions, delta, counters,
                ws, stream)


def gp_boundary_select(layers, ps, bnd, k_counts, scores, params, decisions, delta, counters, ws,
                       stream=None) -> None:
    """First part of gp_boundary_apply: eviction lists and saved rows (workspace only)."""
    _apply_like("gp_boundary_select", layers, ps, bnd, k_counts, scores, params, decisions, delta, counters,
                ws, stream)


def gp_boundary_decide(layers, ps, bnd, k_counts, scores, params, decisions, delta, counters, ws,
                       hold: bool = False, stream=None) -> None:
    """Second part: decisions and page metadata; hold=True leaves compressing requests held."""
    _apply_like("gp_boundary_decide", layers, ps, bnd, k_counts, scores, params, decisions, delta, counters,
                ws, stream, int(bool(hold)))


def gp_boundary_compact(layers, ps, bnd, k_counts, scores, params, decisions, delta, counters, ws,
                        stream=None) -> None:
    """Third part: compaction and the release of freed pages."""
    _apply_like("gp_boundary_compact", layers, ps, bnd, k_counts, scores, params, decisions, delta, counters,
                ws, stream)


def gp_release_held(ps: PageState, stream=None) -> None:
    c_ps = ps.c()
    _check(load().gp_release_held(ctypes.byref(c_ps), _stream(stream)), "gp_release_held")


def gp_append_step(layers: list[KVLayer], ps: PageState, positions: torch.Tensor, k_new: torch.Tensor,
                   v_new: torch.Tensor, q_pre: torch.Tensor, slot_ids: torch.Tensor, init: torch.Tensor | None,
                   qstate: torch.Tensor, beta_s: float, beta_l: float, stream=None) -> None:
    """k_new, v_new [L][R][Hkv][d]; q_pre [L][R][Hq][d]; qstate [L][M][2][Hq][d]."""
    L = len(layers)
    if k_new.dim() != 4 or k_new.shape[0] != L or q_pre.dim() != 4 or qstate.dim() != 5:
        raise ValueError("gp_append_step: k_new/v_new [L,R,Hkv,d], q_pre [L,R,Hq,d], qstate [L,M,2,Hq,d]")
    arr = (_KVLayer * L)(*[layer.c() for layer in layers])
    c_ps = ps.c()
    st = load().gp_append_step(arr, L, ctypes.byref(c_ps), _ptr(positions), _ptr(k_new), _ptr(v_new),
                               _ptr(q_pre), q_pre.shape[2], _ptr(slot_ids), _ptr(init), _ptr(qstate),
                               qstate.shape[1], float(beta_s), float(beta_l), _stream(stream))
    _check(st, "gp_append_step")


def _on_device(name: str, kv: KVLayer | KV8Layer | None, ps: PageState, *tensors) -> None:
    """The calls below run on the current device; all tensors that their kernels read or write lie there."""
    dev = ps.page_table.get_device()
    layer = () if kv is None else (kv.k, kv.v, kv.k_scale, kv.v_scale) if isinstance(kv, KV8Layer) else (kv.k, kv.v)
    for t in (ps.num_pages, ps.seq_lens, *layer, *tensors):
        if t is not None and t.get_device() != dev:
            raise ValueError(f"{name}: tensors on different devices")
    if dev < 0 or dev != torch.cuda.current_device():
        raise ValueError(f"{name}: tensors that are not on the current device")


def _append_rope(name, kv, dtype, ps, positions, k_new, v_new, rope_theta, q, q_out, tok_start, advance, stream):
    c_kv, c_ps = kv.c(), ps.c()
    d, shape = c_kv.head_dim, k_new.shape
    T = shape[0]
    if shape != (T, c_kv.num_kv_heads, d) or v_new.shape != shape or k_new.dtype != dtype or v_new.dtype != dtype:
        raise ValueError(f"{name}: k_new and v_new [tokens, {c_kv.num_kv_heads}, {d}], {dtype}")
    Hq = q_ptr = qo_ptr = q_row = 0
    if q is not None:
        Hq = q.shape[1] if q.dim() == 3 else 0
        if q.shape != (T, Hq, d) or q.dtype != dtype or q_out is None or q_out.shape != q.shape or q_out.dtype != dtype:
            raise ValueError(f"{name}: q and q_out [tokens, heads, {d}], {dtype}")
        q_ptr, qo_ptr, q_row = q.data_ptr(), _ptr(q_out), _row(q.stride(), T, Hq, d, name)
    if tok_start is not None and (tok_start.dtype != torch.int32 or tok_start.numel() != c_ps.num_reqs + 1):
        raise ValueError(f"{name}: tok_start [num_reqs + 1] int32")
    if positions.dtype != torch.int32 or positions.numel() < c_ps.num_reqs:
        raise ValueError(f"{name}: positions [num_reqs] int32")
    _on_device(name, kv, ps, positions, k_new, v_new, q, q_out, tok_start)
    st = getattr(load(), name)(ctypes.byref(c_kv), ctypes.byref(c_ps), _ptr(positions), _ptr(tok_start), T, q_ptr, q_row,
                               qo_ptr, k_new.data_ptr(), _row(k_new.stride(), T, shape[1], d, name), v_new.data_ptr(),
                               _row(v_new.stride(), T, shape[1], d, name), Hq, rope_theta, bool(advance), _stream(stream))
    _check(st, name)


def _row(strides, T: int, heads: int, d: int, name: str) -> int:
    """The stride from token to token of [tokens, heads, head_dim]: any, a token's own elements side by side."""
    if strides[2] != 1 or (heads > 1 and strides[1] != d):
        raise ValueError(f"{name}: the heads of a token lie side by side")
    return strides[0] if T > 1 else heads * d


def gp_append_rope(kv: KVLayer, ps: PageState, positions: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor,
                   rope_theta: float, q: torch.Tensor | None = None, q_out: torch.Tensor | None = None,
                   tok_start: torch.Tensor | None = None, advance: bool = True, stream=None) -> None:
    """New tokens into the cache, keys and queries rotated: k_new, v_new [T, Hkv, d] and
    q [T, Hq, d] with any stride from token to token; tok_start [R + 1] int32, or None
    for one token per request; q_out [T, Hq, d] takes the rotated queries."""
    _append_rope("gp_append_rope", kv, kv.k.dtype, ps, positions, k_new, v_new, rope_theta, q, q_out, tok_start,
                 advance, stream)


def gp_append_rope_q8(kv: KV8Layer, ps: PageState, positions: torch.Tensor, k_new: torch.Tensor,
                      v_new: torch.Tensor, rope_theta: float, q: torch.Tensor | None = None,
                      q_out: torch.Tensor | None = None, tok_start: torch.Tensor | None = None,
                      advance: bool = True, stream=None) -> None:
    """gp_append_rope into an 8-bit cache (rows bfloat16)."""
    _append_rope("gp_append_rope_q8", kv, torch.bfloat16, ps, positions, k_new, v_new, rope_theta, q, q_out,
                 tok_start, advance, stream)


def _of(t: torch.Tensor, dtype, name: str) -> int:
    if t.dtype != dtype:
        raise ValueError(f"{name}: {dtype}, not {t.dtype}")
    return _ptr(t)


def _queries(name: str, q_post: torch.Tensor, out: torch.Tensor, R: int, d: int) -> None:
    shape = q_post.shape
    if len(shape) != 3 or shape[0] != R or shape[2] != d or out.shape != shape:
        raise ValueError(f"{name}: q_post and out [{R}, heads, {d}]")


def gp_decode_attention_q8(kv: KV8Layer, ps: PageState, q_post: torch.Tensor, scale: float, out: torch.Tensor,
                           ws: torch.Tensor, stream=None) -> None:
    """Decode attention over an 8-bit cache; q_post and out bfloat16."""
    c_kv, c_ps = kv.c(), ps.c()
    _queries("gp_decode_attention_q8", q_post, out, c_ps.num_reqs, c_kv.head_dim)
    _on_device("gp_decode_attention_q8", kv, ps, q_post, out, ws)
    st = load().gp_decode_attention_q8(ctypes.byref(c_kv), ctypes.byref(c_ps), _of(q_post, torch.bfloat16, "q_post"),
                                       q_post.shape[1], scale, _of(out, torch.bfloat16, "out"), _ptr(ws), ws.numel(),
                                       _stream(stream))
    _check(st, "gp_decode_attention_q8")


def _page_bounds(name, kv, dtype, ps, bounds, from_tokens, max_update, stream):
    c_kv, c_ps = kv.c(), ps.c()
    if bounds.dtype != dtype or bounds.shape != (c_kv.pool_pages, c_kv.num_kv_heads, 2, c_kv.head_dim):
        raise ValueError(f"{name}: bounds [pool_pages, num_kv_heads, 2, head_dim], {dtype}")
    if from_tokens is not None and (from_tokens.dtype != torch.int32 or from_tokens.numel() != c_ps.num_reqs):
        raise ValueError(f"{name}: from_tokens [num_reqs] int32")
    _on_device(name, kv, ps, bounds, from_tokens)
    _check(getattr(load(), name)(ctypes.byref(c_kv), ctypes.byref(c_ps), _ptr(from_tokens), max_update, _ptr(bounds),
                                 _stream(stream)), name)


def gp_page_bounds(kv: KVLayer, ps: PageState, bounds: torch.Tensor, from_tokens: torch.Tensor | None = None,
                   max_update: int = 0, stream=None) -> None:
    """Least and greatest key values of each page, KV head and dim into bounds [pool, Hkv, 2, d]."""
    _page_bounds("gp_page_bounds", kv, kv.k.dtype, ps, bounds, from_tokens, max_update, stream)


def gp_page_bounds_q8(kv: KV8Layer, ps: PageState, bounds: torch.Tensor, from_tokens: torch.Tensor | None = None,
                      max_update: int = 0, stream=None) -> None:
    """gp_page_bounds of an 8-bit cache (bounds bfloat16)."""
    _page_bounds("gp_page_bounds_q8", kv, torch.bfloat16, ps, bounds, from_tokens, max_update, stream)


def _lists(selected: torch.Tensor, R: int, Hkv: int) -> int:
    shape = selected.shape
    if selected.dtype != torch.int32 or len(shape) != 3 or shape[:2] != (R, Hkv):
        raise ValueError("selected: int32 [num_reqs, num_kv_heads, budget]")
    return shape[2]


def gp_select_pages(bounds: torch.Tensor, ps: PageState, q_post: torch.Tensor, keep_first: int, keep_last: int,
                    selected: torch.Tensor, ws: torch.Tensor, stream=None) -> None:
    """The logical pages each request and KV head is to read, into selected [R, Hkv, budget] int32."""
    c_ps = ps.c()
    pool, hkv, two, d = bounds.shape
    R, Hq, dq = q_post.shape
    budget = _lists(selected, R, hkv)
    if pool != c_ps.pool_pages or R != c_ps.num_reqs or dq != d or two != 2:
        raise ValueError("gp_select_pages: bounds [pool_pages, Hkv, 2, d] and q_post [R, Hq, d] of the page state")
    _on_device("gp_select_pages", None, ps, bounds, q_post, selected, ws)
    st = load().gp_select_pages(_ptr(bounds), _dtype_code(bounds), ctypes.byref(c_ps),
                                _of(q_post, bounds.dtype, "q_post"), Hq, hkv, d, budget, keep_first, keep_last,
                                _ptr(selected), _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "gp_select_pages")


def _decode_pages(name, kv, dtype, ps, selected, q_post, scale, out, ws, stream):
    c_kv, c_ps = kv.c(), ps.c()
    budget = _lists(selected, c_ps.num_reqs, c_kv.num_kv_heads)
    _queries(name, q_post, out, c_ps.num_reqs, c_kv.head_dim)
    _on_device(name, kv, ps, selected, q_post, out, ws)
    _check(getattr(load(), name)(ctypes.byref(c_kv), ctypes.byref(c_ps), _ptr(selected), budget,
                                 _of(q_post, dtype, "q_post"), q_post.shape[1], scale, _of(out, dtype, "out"), _ptr(ws),
                                 ws.numel(), _stream(stream)), name)


def gp_decode_attention_pages(kv: KVLayer, ps: PageState, selected: torch.Tensor, q_post: torch.Tensor, scale: float,
                              out: torch.Tensor, ws: torch.Tensor, stream=None) -> None:
    """Decode attention over the logical pages selected [R, Hkv, budget]."""
    _decode_pages("gp_decode_attention_pages", kv, kv.k.dtype, ps, selected, q_post, scale, out, ws, stream)


def gp_decode_attention_pages_q8(kv: KV8Layer, ps: PageState, selected: torch.Tensor, q_post: torch.Tensor,
                                 scale: float, out: torch.Tensor, ws: torch.Tensor, stream=None) -> None:
    """gp_decode_attention_pages over an 8-bit cache; q_post and out bfloat16."""
    _decode_pages("gp_decode_attention_pages_q8", kv, torch.bfloat16, ps, selected, q_post, scale, out, ws, stream)
