"""Thin ctypes binding of libhermes.so (argument marshalling only).

Every step of the streaming path runs in the library's HIP kernels; this
module only allocates device buffers with torch, passes raw pointers and the
current HIP stream, and turns negative return codes into exceptions.  If the
library has not been built it raises at import time: there is no fallback.
"""
from __future__ import annotations

import ctypes
import math
import os
from typing import Optional, Sequence

import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libhermes.so")
if not os.path.exists(_LIB_PATH):
    raise ImportError(f"{_LIB_PATH} is missing: build it with `python -m paper_2601_14724_amd.build`"
                      " (or __graft_entry__.build()) before using the HIP path")
lib = ctypes.CDLL(_LIB_PATH)

OK, EINVAL, ECAPACITY, ESTATE, EHIP, ENOTSUP = 0, -1, -2, -3, -4, -5
SHALLOW, MIDDLE, DEEP = 0, 1, 2
ALL_LAYERS = -1
MAX_LAYERS = 64
K_APPEND, K_ATTN, K_COLSUM, K_SELECT, K_GATHER, K_QUERY, K_SUMMARY, K_GUIDE, K_PACK = range(9)
KERNEL_NAMES = ("append", "attention", "colsum", "select", "gather", "query", "summary", "guide", "pack")
REINDEX_NONE, REINDEX_EAGER, REINDEX_LAZY = 0, 1, 2
SCORE_CHUNK, SCORE_GUIDANCE = 0, 1
PAGE_BF16, PAGE_FP4 = 0, 1
PAGE_BAD_ID, PAGE_BAD_LENGTH, PAGE_BAD_ROWS, PAGE_BAD_PARENT, PAGE_NO_ROOM = 1, 2, 4, 8, 16
BF16, FP32 = 0, 1
_MOST = 0x7FFFFFFF   # (ctypes would keep the low half of a greater number)

EXPORTED = ("hermes_workspace_bytes", "hermes_kv_init", "hermes_append_chunk",
            "hermes_append_chunk_at", "hermes_guidance_score", "hermes_compress",
            "hermes_append_chunk_mrope", "hermes_query_attend", "hermes_kv_rewind",
            "hermes_kv_view", "hermes_kv_view_rope", "hermes_kv_view_mrope",
            "hermes_budget_from_weights", "hermes_kv_destroy", "hermes_strerror",
            "hermes_select_topk", "hermes_profile_enable", "hermes_profile_read",
            "hermes_check_enable", "hermes_kv_init_static",
            "hermes_page_bytes", "hermes_page_workspace_bytes", "hermes_page_append",
            "hermes_page_attend", "hermes_page_read", "hermes_page_pack", "hermes_page_reorder",
            "hermes_beam_workspace_bytes", "hermes_beam_select", "hermes_weight_bytes",
            "hermes_weight_pack", "hermes_weight_workspace_bytes", "hermes_weight_product")
STATIC_WORKSPACE_BYTES = 128 << 20


class HermesConfig(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("max_chunk", ctypes.c_int32), ("max_cap", ctypes.c_int32),
                ("budget", ctypes.POINTER(ctypes.c_int32)),
                ("layer_class", ctypes.POINTER(ctypes.c_int8)),
                ("lambda_", ctypes.POINTER(ctypes.c_float)),
                ("omega0", ctypes.c_double), ("gamma", ctypes.c_double),
                ("forget_rate", ctypes.c_double), ("sm_scale", ctypes.c_double),
                ("alpha_mode", ctypes.c_int32), ("align_mode", ctypes.c_int32),
                ("force_scores", ctypes.c_int32),
                ("summary_mode", ctypes.c_int32), ("reindex_mode", ctypes.c_int32),
                ("rope_offset", ctypes.c_int32), ("rope_limit", ctypes.c_int32),
                ("rope_headroom", ctypes.c_int32), ("rope_theta", ctypes.c_double),
                ("scoring_mode", ctypes.c_int32), ("rope_axes", ctypes.c_int32),
                ("mrope_section", ctypes.c_int32 * 3)]


class LayerBuffers(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p * 2), ("v", ctypes.c_void_p * 2),
                ("pos", ctypes.c_void_p * 2), ("w", ctypes.c_void_p),
                ("s_dbg", ctypes.c_void_p), ("kept_dbg", ctypes.c_void_p),
                ("cap", ctypes.c_int32), ("init_len", ctypes.c_int32),
                ("rpos", ctypes.c_void_p * 2), ("rpos_h", ctypes.c_void_p * 2),
                ("rpos_w", ctypes.c_void_p * 2)]


class PagePoolStruct(ctypes.Structure):
    _fields_ = [("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("format", ctypes.c_int32), ("page_rows", ctypes.c_int32), ("n_pages", ctypes.c_int32),
                ("pages", ctypes.c_void_p), ("status", ctypes.c_void_p), ("sm_scale", ctypes.c_double),
                ("rope_theta", ctypes.c_double), ("rope_axes", ctypes.c_int32),
                ("mrope_section", ctypes.c_int32 * 3)]


class PageBatchStruct(ctypes.Structure):
    _fields_ = [("n_seqs", ctypes.c_int32), ("n_rows", ctypes.c_int32), ("max_rows", ctypes.c_int32),
                ("max_len", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("row_start", ctypes.c_void_p),
                ("kv_len", ctypes.c_void_p), ("tables", ctypes.c_void_p)]


class PageBeamsStruct(ctypes.Structure):
    _fields_ = [("n_groups", ctypes.c_int32), ("n_seqs", ctypes.c_int32), ("n_beams", ctypes.c_int32),
                ("max_pages", ctypes.c_int32), ("grow", ctypes.c_int32), ("parent", ctypes.c_void_p),
                ("room", ctypes.c_void_p), ("tables", ctypes.c_void_p), ("kv_len", ctypes.c_void_p),
                ("tables_out", ctypes.c_void_p), ("kv_len_out", ctypes.c_void_p)]


class BeamConfig(ctypes.Structure):
    _fields_ = [("n_seqs", ctypes.c_int32), ("n_beams", ctypes.c_int32), ("n_vocab", ctypes.c_int32),
                ("n_keep", ctypes.c_int32), ("logits_type", ctypes.c_int32), ("end_token", ctypes.c_int32),
                ("pad_token", ctypes.c_int32)]


class WeightStruct(ctypes.Structure):
    _fields_ = [("n_out", ctypes.c_int32), ("n_in", ctypes.c_int32), ("data", ctypes.c_void_p)]


_vp, _i32, _i64, _dbl = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_double
lib.hermes_workspace_bytes.restype = ctypes.c_size_t
lib.hermes_workspace_bytes.argtypes = [ctypes.POINTER(HermesConfig)]
lib.hermes_kv_init.restype = ctypes.c_int
lib.hermes_kv_init.argtypes = [ctypes.POINTER(HermesConfig), ctypes.POINTER(LayerBuffers), _vp,
                               ctypes.c_size_t, ctypes.POINTER(_vp)]
lib.hermes_kv_init_static.restype = ctypes.c_int
lib.hermes_kv_init_static.argtypes = [ctypes.POINTER(HermesConfig), ctypes.POINTER(LayerBuffers),
                                      ctypes.POINTER(_vp)]
lib.hermes_append_chunk.restype = ctypes.c_int
lib.hermes_append_chunk.argtypes = [_vp, _i32, _vp, _vp, _vp, _vp, _i32, _vp, _vp]
lib.hermes_append_chunk_at.restype = ctypes.c_int
lib.hermes_append_chunk_at.argtypes = [_vp, _i32, _vp, _vp, _vp, _vp, _vp, _i32, _vp, _vp]
lib.hermes_append_chunk_mrope.restype = ctypes.c_int
lib.hermes_append_chunk_mrope.argtypes = [_vp, _i32, _vp, _vp, _vp, _vp, _vp, _i32, _vp, _vp]
lib.hermes_kv_view_mrope.restype = ctypes.c_int
lib.hermes_kv_view_mrope.argtypes = [_vp, _i32, ctypes.POINTER(_vp), ctypes.POINTER(_vp),
                                     ctypes.POINTER(_vp)]
lib.hermes_guidance_score.restype = ctypes.c_int
lib.hermes_guidance_score.argtypes = [_vp, _i32, _vp, _vp, _vp, _i32, _vp]
lib.hermes_kv_view_rope.restype = ctypes.c_int
lib.hermes_kv_view_rope.argtypes = [_vp, _i32, ctypes.POINTER(_vp)]
lib.hermes_budget_from_weights.restype = ctypes.c_int
lib.hermes_budget_from_weights.argtypes = [ctypes.POINTER(_dbl), _i32, _i64, ctypes.POINTER(_i32)]
lib.hermes_compress.restype = ctypes.c_int
lib.hermes_compress.argtypes = [_vp, _vp]
lib.hermes_query_attend.restype = ctypes.c_int
lib.hermes_query_attend.argtypes = [_vp, _i32, _vp, _vp, _vp, _i32, _vp, _vp]
lib.hermes_kv_rewind.restype = ctypes.c_int
lib.hermes_kv_rewind.argtypes = [_vp]
lib.hermes_kv_view.restype = ctypes.c_int
lib.hermes_kv_view.argtypes = [_vp, _i32, ctypes.POINTER(_vp), ctypes.POINTER(_vp),
                               ctypes.POINTER(_vp), ctypes.POINTER(_i32)]
lib.hermes_kv_destroy.restype = None
lib.hermes_kv_destroy.argtypes = [_vp]
lib.hermes_strerror.restype = ctypes.c_char_p
lib.hermes_strerror.argtypes = [ctypes.c_int]
lib.hermes_select_topk.restype = ctypes.c_int
lib.hermes_select_topk.argtypes = [_vp, _i32, _i32, _vp, _vp]
lib.hermes_check_enable.restype = ctypes.c_int
lib.hermes_check_enable.argtypes = [_vp, ctypes.c_int]
lib.hermes_profile_enable.restype = ctypes.c_int
lib.hermes_profile_enable.argtypes = [_vp, ctypes.c_int]
lib.hermes_profile_read.restype = ctypes.c_int
lib.hermes_profile_read.argtypes = [_vp, ctypes.c_int, ctypes.POINTER(_dbl), ctypes.POINTER(_i64)]
_pool_p, _batch_p = ctypes.POINTER(PagePoolStruct), ctypes.POINTER(PageBatchStruct)
lib.hermes_page_bytes.restype = ctypes.c_size_t
lib.hermes_page_bytes.argtypes = [_pool_p]
lib.hermes_page_workspace_bytes.restype = ctypes.c_size_t
lib.hermes_page_workspace_bytes.argtypes = [_pool_p, _batch_p]
lib.hermes_page_append.restype = ctypes.c_int
lib.hermes_page_append.argtypes = [_pool_p, _batch_p, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _vp, _vp]
lib.hermes_page_attend.restype = ctypes.c_int
lib.hermes_page_attend.argtypes = [_pool_p, _batch_p, _vp, _i64, _vp, _vp, _vp, ctypes.c_size_t, _vp]
lib.hermes_page_read.restype = ctypes.c_int
lib.hermes_page_read.argtypes = [_pool_p, _batch_p, _vp, _vp, _vp]
lib.hermes_page_pack.restype = ctypes.c_int
lib.hermes_page_pack.argtypes = [_vp, _i32, _pool_p, _vp, _i32, _vp, _vp]
lib.hermes_page_reorder.restype = ctypes.c_int
lib.hermes_page_reorder.argtypes = [_pool_p, ctypes.POINTER(PageBeamsStruct), _vp]
_beam_p, _weight_p = ctypes.POINTER(BeamConfig), ctypes.POINTER(WeightStruct)
lib.hermes_beam_workspace_bytes.restype = ctypes.c_size_t
lib.hermes_beam_workspace_bytes.argtypes = [_beam_p]
lib.hermes_beam_select.restype = ctypes.c_int
lib.hermes_beam_select.argtypes = [_beam_p, _vp, _i64, _vp, _vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_size_t, _vp]
lib.hermes_weight_bytes.restype = ctypes.c_size_t
lib.hermes_weight_bytes.argtypes = [_weight_p]
lib.hermes_weight_pack.restype = ctypes.c_int
lib.hermes_weight_pack.argtypes = [_weight_p, _vp, _i64, _vp]
lib.hermes_weight_product.restype = ctypes.c_int
lib.hermes_weight_workspace_bytes.restype = ctypes.c_size_t
lib.hermes_weight_workspace_bytes.argtypes = [_weight_p, _i32]
lib.hermes_weight_product.argtypes = [_weight_p, _vp, _i64, _i32, _vp, _vp, _vp, _i32, _vp, ctypes.c_size_t, _vp]


class HermesError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: {lib.hermes_strerror(code).decode()} ({code})")
        self.code = code


def check(code: int, what: str) -> None:
    if code != OK:
        raise HermesError(code, what)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


# The current stream's handle without building a torch.cuda.Stream object for
# each call (2.8 us, a fifth of a one-token query's host time).
try:
    from torch._C import _cuda_getCurrentRawStream as _raw_stream, _cuda_getDevice as _device
except ImportError:   # a torch without a GPU build
    _raw_stream = None


def _stream() -> int:
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_device())


def _need(t: torch.Tensor, dtype: torch.dtype, shape: tuple, name: str) -> None:
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or tuple(t.shape) != shape:
        raise ValueError(f"{name}: expected {dtype} {shape}, got "
                         f"{getattr(t, 'dtype', None)} {tuple(getattr(t, 'shape', ()))}")
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name}: must be a contiguous device tensor")


def _on(index: int, fn, name: str, *args) -> None:
    """fn(*args, stream) with device `index` current, on its current stream."""
    if _raw_stream is not None and _device() == index:
        check(fn(*args, _raw_stream(index)), name)
    else:
        with torch.cuda.device(index):
            check(fn(*args, _stream()), name)


def budget_from_weights(weights: Sequence[float], total: int) -> list:
    """Per-layer budgets floor(w_i / sum w * total), residue to the last layer
    (the library's host helper)."""
    n = len(weights)
    w = (ctypes.c_double * n)(*[float(x) for x in weights])
    out = (ctypes.c_int32 * n)()
    check(lib.hermes_budget_from_weights(w, n, int(total), out), "hermes_budget_from_weights")
    return list(out)


def select_topk(keys: torch.Tensor, k: int) -> torch.Tensor:
    """Indices (ascending) of the k largest non-negative fp32 keys, ties to the
    higher index, computed by the library's TopK kernel."""
    _need(keys, torch.float32, (keys.numel(),), "keys")
    out = torch.empty(min(k, keys.numel()), dtype=torch.int32, device=keys.device)
    check(lib.hermes_select_topk(keys.data_ptr(), keys.numel(), k, out.data_ptr(), _stream()),
          "hermes_select_topk")
    return out


class HermesKV:
    """Per-layer KV caches managed by libhermes.

    Device memory (two ping-pong buffers per layer, positions, the attention
    mass, optional debug outputs and the workspace) is allocated here with
    torch; the library only receives pointers.  `init` optionally gives each
    layer's initial (k, v, pos) as device tensors of shapes [n][Hkv][d] bf16,
    [n][Hkv][d] bf16 and [n] int32, then optionally its RoPE positions [n]
    (rope_axes 1) or its (t, h, w) coordinates [3][n] int32 (rope_axes 3).
    """

    def __init__(self, n_layers: int, n_q_heads: int, n_kv_heads: int, head_dim: int,
                 budgets: Sequence[int], max_chunk: int, cap: Optional[int] = None,
                 init: Optional[Sequence[tuple]] = None,
                 layer_class: Optional[Sequence[int]] = None,
                 lambdas: Optional[Sequence[float]] = None, omega0: float = 0.75,
                 gamma: float = 0.6, forget_rate: float = 2.0 ** -10,
                 sm_scale: Optional[float] = None, alpha_mode: int = 0, align_mode: int = 0,
                 force_scores: bool = False, debug: bool = False, device: str = "cuda",
                 summary_mode: int = 0, reindex_mode: int = REINDEX_NONE, rope_offset: int = 0,
                 rope_limit: int = 0, rope_headroom: int = 0, rope_theta: float = 1.0e6,
                 scoring_mode: int = SCORE_CHUNK, rope_axes: int = 1,
                 mrope_section: Sequence[int] = (0, 0, 0), static_workspace: bool = False):
        self.L, self.Hq, self.Hkv, self.d = n_layers, n_q_heads, n_kv_heads, head_dim
        self.budgets = [int(b) for b in budgets]
        self.max_chunk = int(max_chunk)
        init_lens = [0] * n_layers if init is None else [int(t[0].shape[0]) for t in init]
        if cap is None:
            cap = max(max(init_lens), max(self.budgets) + int(bool(summary_mode))) + self.max_chunk
        self.rope_axes = 3 if rope_axes == 3 else 1
        self.keep_rpos = bool(summary_mode) or reindex_mode != REINDEX_NONE or self.rope_axes == 3
        self.cap = int(cap)
        self.device = torch.device(device)
        dev = self.device
        shp = (self.cap, n_kv_heads, head_dim)
        self.k = [[torch.zeros(shp, dtype=torch.bfloat16, device=dev) for _ in range(2)]
                  for _ in range(n_layers)]
        self.v = [[torch.zeros(shp, dtype=torch.bfloat16, device=dev) for _ in range(2)]
                  for _ in range(n_layers)]
        self.pos = [[torch.zeros(self.cap, dtype=torch.int32, device=dev) for _ in range(2)]
                    for _ in range(n_layers)]
        self.rpos = ([[torch.zeros(self.cap, dtype=torch.int32, device=dev) for _ in range(2)]
                      for _ in range(n_layers)] if self.keep_rpos else None)
        three = self.rope_axes == 3
        self.rpos_h = ([[torch.zeros(self.cap, dtype=torch.int32, device=dev) for _ in range(2)]
                        for _ in range(n_layers)] if three else None)
        self.rpos_w = ([[torch.zeros(self.cap, dtype=torch.int32, device=dev) for _ in range(2)]
                        for _ in range(n_layers)] if three else None)
        self.w = [torch.zeros(self.cap, dtype=torch.float32, device=dev) for _ in range(n_layers)]
        self.s_dbg = ([torch.zeros(self.cap, dtype=torch.float32, device=dev)
                       for _ in range(n_layers)] if debug else None)
        self.kept_dbg = ([torch.zeros(b, dtype=torch.int32, device=dev) for b in self.budgets]
                         if debug else None)
        if init is not None:
            for l, t in enumerate(init):
                k0, v0, p0 = t[:3]
                n = k0.shape[0]
                self.k[l][0][:n].copy_(k0)
                self.v[l][0][:n].copy_(v0)
                self.pos[l][0][:n].copy_(p0)
                if three and n > 0:   # (t, h, w) coordinates [3][n] (4th element)
                    if len(t) < 4:
                        raise ValueError("rope_axes 3: init needs (k, v, pos, thw)")
                    self.rpos[l][0][:n].copy_(t[3][0])
                    self.rpos_h[l][0][:n].copy_(t[3][1])
                    self.rpos_w[l][0][:n].copy_(t[3][2])
                elif self.keep_rpos and not three:   # RoPE positions (4th element), default the stream ones
                    self.rpos[l][0][:n].copy_(t[3] if len(t) > 3 else p0)
        self._budget_arr = (ctypes.c_int32 * n_layers)(*self.budgets)
        self._class_arr = ((ctypes.c_int8 * n_layers)(*layer_class)
                           if layer_class is not None else None)
        self._lambda_arr = ((ctypes.c_float * n_layers)(*lambdas) if lambdas is not None else None)
        cfg = HermesConfig()
        cfg.n_layers, cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim = (n_layers, n_q_heads,
                                                                     n_kv_heads, head_dim)
        cfg.max_chunk, cfg.max_cap = self.max_chunk, self.cap
        cfg.budget = self._budget_arr
        cfg.layer_class = (ctypes.cast(self._class_arr, ctypes.POINTER(ctypes.c_int8))
                           if self._class_arr is not None else None)
        cfg.lambda_ = (ctypes.cast(self._lambda_arr, ctypes.POINTER(ctypes.c_float))
                       if self._lambda_arr is not None else None)
        cfg.omega0, cfg.gamma, cfg.forget_rate = omega0, gamma, forget_rate
        cfg.sm_scale = sm_scale if sm_scale is not None else 0.0
        cfg.alpha_mode, cfg.align_mode, cfg.force_scores = alpha_mode, align_mode, int(force_scores)
        cfg.summary_mode, cfg.reindex_mode, cfg.scoring_mode = int(summary_mode), reindex_mode, scoring_mode
        cfg.rope_offset, cfg.rope_limit, cfg.rope_headroom = rope_offset, rope_limit, rope_headroom
        cfg.rope_theta = rope_theta
        cfg.rope_axes = int(rope_axes)
        for a in range(3):
            cfg.mrope_section[a] = int(mrope_section[a])
        self._cfg = cfg
        nbytes = lib.hermes_workspace_bytes(ctypes.byref(cfg))
        if nbytes == 0:
            raise HermesError(EINVAL, "hermes_workspace_bytes")
        # static_workspace: the library's own device scratch (hermes_kv_init_static)
        self.workspace = (None if static_workspace
                          else torch.empty(nbytes, dtype=torch.uint8, device=dev))
        bufs = (LayerBuffers * n_layers)()
        for l in range(n_layers):
            b = bufs[l]
            for p in range(2):
                b.k[p] = self.k[l][p].data_ptr()
                b.v[p] = self.v[l][p].data_ptr()
                b.pos[p] = self.pos[l][p].data_ptr()
            b.w = self.w[l].data_ptr()
            b.s_dbg = _ptr(self.s_dbg[l]) if debug else None
            b.kept_dbg = _ptr(self.kept_dbg[l]) if debug else None
            b.cap = self.cap
            b.init_len = init_lens[l]
            if self.keep_rpos:
                for p in range(2):
                    b.rpos[p] = self.rpos[l][p].data_ptr()
            if three:
                for p in range(2):
                    b.rpos_h[p] = self.rpos_h[l][p].data_ptr()
                    b.rpos_w[p] = self.rpos_w[l][p].data_ptr()
        self._bufs = bufs
        ctx = ctypes.c_void_p()
        if static_workspace:
            with torch.cuda.device(dev):
                check(lib.hermes_kv_init_static(ctypes.byref(cfg), bufs, ctypes.byref(ctx)),
                      "hermes_kv_init_static")
        else:
            check(lib.hermes_kv_init(ctypes.byref(cfg), bufs, self.workspace.data_ptr(), nbytes,
                                     ctypes.byref(ctx)), "hermes_kv_init")
        self.ctx = ctx

    # ------------------------------------------------------------------ calls
    def _check_inputs(self, q, k, v, n, layer):
        lead = () if layer != ALL_LAYERS else (self.L,)
        _need(q, torch.bfloat16, lead + (n, self.Hq, self.d), "q")
        _need(k, torch.bfloat16, lead + (n, self.Hkv, self.d), "k")
        _need(v, torch.bfloat16, lead + (n, self.Hkv, self.d), "v")

    def append(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, pos: torch.Tensor,
               layer: int = ALL_LAYERS, out: Optional[torch.Tensor] = None,
               rope_pos: Optional[torch.Tensor] = None,
               rope_thw: Optional[torch.Tensor] = None) -> torch.Tensor:
        n = q.shape[-3]
        self._check_inputs(q, k, v, n, layer)
        _need(pos, torch.int32, (n,), "pos")
        if out is None:
            out = torch.empty_like(q)
        if rope_thw is not None:
            _need(rope_thw, torch.int32, (3, n), "rope_thw")
            check(lib.hermes_append_chunk_mrope(self.ctx, layer, q.data_ptr(), k.data_ptr(),
                                                v.data_ptr(), pos.data_ptr(), rope_thw.data_ptr(),
                                                n, out.data_ptr(), _stream()),
                  "hermes_append_chunk_mrope")
        elif rope_pos is None:
            check(lib.hermes_append_chunk(self.ctx, layer, q.data_ptr(), k.data_ptr(),
                                          v.data_ptr(), pos.data_ptr(), n, out.data_ptr(),
                                          _stream()), "hermes_append_chunk")
        else:
            _need(rope_pos, torch.int32, (n,), "rope_pos")
            check(lib.hermes_append_chunk_at(self.ctx, layer, q.data_ptr(), k.data_ptr(),
                                             v.data_ptr(), pos.data_ptr(), rope_pos.data_ptr(), n,
                                             out.data_ptr(), _stream()), "hermes_append_chunk_at")
        return out

    def guidance(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                 layer: int = ALL_LAYERS) -> None:
        """Attention mass of the cached tokens from guidance-prompt rows."""
        n = q.shape[-3]
        self._check_inputs(q, k, v, n, layer)
        check(lib.hermes_guidance_score(self.ctx, layer, q.data_ptr(), k.data_ptr(), v.data_ptr(),
                                        n, _stream()), "hermes_guidance_score")

    def compress(self) -> None:
        check(lib.hermes_compress(self.ctx, _stream()), "hermes_compress")

    def query(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
              layer: int = ALL_LAYERS, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        n = q.shape[-3]
        self._check_inputs(q, k, v, n, layer)
        if out is None:
            out = torch.empty_like(q)
        check(lib.hermes_query_attend(self.ctx, layer, q.data_ptr(), k.data_ptr(), v.data_ptr(),
                                      n, out.data_ptr(), _stream()), "hermes_query_attend")
        return out

    def pack(self, pages: "KVPages", tables: torch.Tensor, kv_len: torch.Tensor, layer: int = ALL_LAYERS) -> None:
        """Packs the current cache of one layer, or of all, into the pages of `tables`
        (int32 [max_pages], or [L][max_pages]), and its length into kv_len (int32 [1] or [L])."""
        lead = () if layer != ALL_LAYERS else (self.L,)
        _need(tables, torch.int32, lead + (tables.shape[-1],), "tables")
        _need(kv_len, torch.int32, lead or (1,), "kv_len")
        for t in (tables, kv_len, self.k[0][0]):
            pages._on_device(t, "pack")
        pages._run(lib.hermes_page_pack, "hermes_page_pack", self.ctx, layer, pages._ref, tables.data_ptr(),
                   tables.shape[-1], kv_len.data_ptr())

    def rewind(self) -> None:
        check(lib.hermes_kv_rewind(self.ctx), "hermes_kv_rewind")

    def length(self, layer: int) -> int:
        ln = ctypes.c_int32()
        check(lib.hermes_kv_view(self.ctx, layer, None, None, None, ctypes.byref(ln)),
              "hermes_kv_view")
        return ln.value

    def view(self, layer: int):
        """(k, v, pos) tensors of the layer's current buffer, first `len` rows."""
        kp, vp, pp, ln = ctypes.c_void_p(), ctypes.c_void_p(), ctypes.c_void_p(), ctypes.c_int32()
        check(lib.hermes_kv_view(self.ctx, layer, ctypes.byref(kp), ctypes.byref(vp),
                                 ctypes.byref(pp), ctypes.byref(ln)), "hermes_kv_view")
        p = 0 if kp.value == self.k[layer][0].data_ptr() else 1
        n = ln.value
        return self.k[layer][p][:n], self.v[layer][p][:n], self.pos[layer][p][:n]

    def view_rope(self, layer: int) -> torch.Tensor:
        """RoPE positions of the layer's current buffer, first `len` rows."""
        rp = ctypes.c_void_p()
        check(lib.hermes_kv_view_rope(self.ctx, layer, ctypes.byref(rp)), "hermes_kv_view_rope")
        if not rp.value:
            raise ValueError("this cache keeps no RoPE positions")
        p = 0 if rp.value == self.rpos[layer][0].data_ptr() else 1
        return self.rpos[layer][p][:self.length(layer)]

    def view_mrope(self, layer: int) -> torch.Tensor:
        """(t, h, w) coordinates [3][len] of the layer's current buffer."""
        t, h, w = ctypes.c_void_p(), ctypes.c_void_p(), ctypes.c_void_p()
        check(lib.hermes_kv_view_mrope(self.ctx, layer, ctypes.byref(t), ctypes.byref(h),
                                       ctypes.byref(w)), "hermes_kv_view_mrope")
        if not t.value:
            raise ValueError("this cache keeps no M-RoPE coordinates")
        p = 0 if t.value == self.rpos[layer][0].data_ptr() else 1
        n = self.length(layer)
        return torch.stack([self.rpos[layer][p][:n], self.rpos_h[layer][p][:n],
                            self.rpos_w[layer][p][:n]])

    # -------------------------------------------------------------- profiling
    def check_preconditions(self, on: bool = True) -> None:
        """Device-side checks of positions and finiteness before each call."""
        check(lib.hermes_check_enable(self.ctx, int(on)), "hermes_check_enable")

    def profile(self, on: bool = True) -> None:
        check(lib.hermes_profile_enable(self.ctx, int(on)), "hermes_profile_enable")

    def profile_read(self, kernel_id: int):
        ms, cnt = ctypes.c_double(), ctypes.c_int64()
        check(lib.hermes_profile_read(self.ctx, kernel_id, ctypes.byref(ms), ctypes.byref(cnt)),
              "hermes_profile_read")
        return ms.value, cnt.value

    def close(self) -> None:
        if getattr(self, "ctx", None) is not None and self.ctx.value:
            lib.hermes_kv_destroy(self.ctx)
            self.ctx = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class PageBatch:
    """The sequences of a call on pages and their rows in its stacked inputs
    (hermes_page_batch): page ids `tables` int32 [n_seqs][max_pages], lengths `kv_len`
    int32 [n_seqs] with the call's own rows, and `row_start` int32 [n_seqs + 1] with
    `n_rows` stacked rows (None: one row a sequence).  The tensors are read by every
    call, and may change between calls.  `max_rows` and `max_len` (None: not known)
    only choose how the work is cut."""

    def __init__(self, tables: torch.Tensor, kv_len: torch.Tensor, row_start: Optional[torch.Tensor] = None,
                 n_rows: Optional[int] = None, max_rows: Optional[int] = None, max_len: Optional[int] = None):
        n = int(kv_len.shape[0])
        _need(kv_len, torch.int32, (n,), "kv_len")
        _need(tables, torch.int32, (n, tables.shape[-1]), "tables")
        if row_start is not None:
            _need(row_start, torch.int32, (n + 1,), "row_start")
            if n_rows is None:
                raise ValueError("n_rows: needed with row_start")
        elif n_rows not in (None, n):
            raise ValueError("n_rows: one row a sequence without row_start")
        for t in (tables, row_start):     # (a call compares the device of kv_len with its pool's)
            if t is not None and t.device != kv_len.device:
                raise ValueError(f"tables, kv_len and row_start: one device, got {t.device} and {kv_len.device}")
        self.tables, self.kv_len, self.row_start = tables, kv_len, row_start
        self.n_seqs, self.n_rows = n, n if n_rows is None else int(n_rows)
        b = PageBatchStruct()
        b.n_seqs, b.n_rows, b.max_pages = n, self.n_rows, tables.shape[-1]
        b.max_rows = 1 if row_start is None else int(max_rows or 0)
        b.max_len = int(max_len or 0)
        b.row_start, b.kv_len, b.tables = _ptr(row_start), kv_len.data_ptr(), tables.data_ptr()
        self._batch, self._ref = b, ctypes.byref(b)


class KVPages:
    """A pool of pages of K and V, in FP4 or bf16 (hermes_page_pool).

    `pages`: uint8 [n_pages][page bytes] to use as the pool (allocated here if None).
    The calls run on the current stream of the pool's device.  `faults()` reads and
    clears the PAGE_BAD_* bits that calls have noted."""

    def __init__(self, n_q_heads: int, n_kv_heads: int, head_dim: int, n_pages: int, page_rows: int = 64,
                 fmt: int = PAGE_FP4, sm_scale: Optional[float] = None, rope_theta: float = 1.0e6, rope_axes: int = 1,
                 mrope_section: Sequence[int] = (0, 0, 0), device: str = "cuda", pages: Optional[torch.Tensor] = None):
        p = PagePoolStruct()
        p.n_q_heads, p.n_kv_heads, p.head_dim, p.format = n_q_heads, n_kv_heads, head_dim, fmt
        p.page_rows, p.n_pages = page_rows, n_pages
        p.sm_scale = sm_scale if sm_scale is not None else 0.0
        p.rope_theta, p.rope_axes = rope_theta, rope_axes
        for i in range(3):
            p.mrope_section[i] = int(mrope_section[i])
        self.page_bytes = lib.hermes_page_bytes(ctypes.byref(p))
        if self.page_bytes == 0:              # (why: a call of no rows looks at the pool alone)
            p.pages = 16
            raise HermesError(lib.hermes_page_read(ctypes.byref(p), ctypes.byref(PageBatchStruct()), None, None, None),
                              "hermes_page_bytes")
        self.Hq, self.Hkv, self.d, self.axes = n_q_heads, n_kv_heads, head_dim, 3 if rope_axes == 3 else 1
        if pages is None:
            pages = torch.empty((n_pages, self.page_bytes), dtype=torch.uint8, device=device)
        _need(pages, torch.uint8, (n_pages, self.page_bytes), "pages")
        self.pages, self.device = pages, pages.device
        self._status = torch.zeros(1, dtype=torch.int32, device=self.device)
        p.pages, p.status = pages.data_ptr(), self._status.data_ptr()
        self._pool, self._ref, self._index = p, ctypes.byref(p), pages.get_device()

    # (a token's calls are a few microseconds on the device: their checks are kept short)
    def _run(self, fn, name: str, *args) -> None:
        """fn(*args, stream) with the pool's device current."""
        _on(self._index, fn, name, *args)

    def _on_device(self, t: torch.Tensor, name: str) -> None:
        if t.get_device() != self._index:
            raise ValueError(f"{name}: a tensor on {t.device}, the pages are on {self.device}")

    def _fits(self, t: torch.Tensor, dtype: torch.dtype, shape: tuple, name: str) -> None:
        if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
            raise ValueError(f"{name}: expected contiguous {dtype} {shape}, got {getattr(t, 'dtype', None)} "
                             f"{tuple(getattr(t, 'shape', ()))}")
        self._on_device(t, name)

    def _rows(self, t: torch.Tensor, n: int, heads: int, name: str) -> int:
        """Stride of rows [heads][d] of a bf16 tensor, which may lie apart."""
        if not isinstance(t, torch.Tensor) or t.dtype is not torch.bfloat16 or t.shape != (n, heads, self.d):
            raise ValueError(f"{name}: expected torch.bfloat16 {(n, heads, self.d)}, got "
                             f"{getattr(t, 'dtype', None)} {tuple(getattr(t, 'shape', ()))}")
        self._on_device(t, name)
        if n == 0:
            return heads * self.d
        rs, hs, es = t.stride()
        if es != 1 or (hs != self.d and heads > 1):
            raise ValueError(f"{name}: a row's heads must be contiguous")
        return rs if n > 1 else heads * self.d

    def append(self, batch: PageBatch, k: torch.Tensor, v: torch.Tensor, q: Optional[torch.Tensor] = None,
               rope: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
        """Rotates k (and q) to the positions `rope` (int32 [n_rows], or [3][n_rows]),
        stores k and v as the last rows of their sequences, and returns the rotated q."""
        n = batch.n_rows
        ks, vs = self._rows(k, n, self.Hkv, "k"), self._rows(v, n, self.Hkv, "v")
        qs, qp, op, rp = 0, None, None, None
        if q is not None:
            qs, qp = self._rows(q, n, self.Hq, "q"), q.data_ptr()
            if q_out is None:
                q_out = torch.empty(q.shape, dtype=torch.bfloat16, device=self.device)
            else:
                self._fits(q_out, torch.bfloat16, (n, self.Hq, self.d), "q_out")
        if q_out is not None:
            op = q_out.data_ptr()
        if rope is not None:
            self._fits(rope, torch.int32, (n,) if self.axes == 1 else (3, n), "rope")
            rp = rope.data_ptr()
        self._on_device(batch.kv_len, "batch")
        self._run(lib.hermes_page_append, "hermes_page_append", self._ref, batch._ref, qp, qs, k.data_ptr(), ks,
                  v.data_ptr(), vs, rp, op)
        return q_out

    def attend(self, batch: PageBatch, q: torch.Tensor, out: Optional[torch.Tensor] = None,
               lse: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Causal attention of every sequence's rows over its pages; lse: fp32
        [n_rows][n_q_heads], written if given."""
        n = batch.n_rows
        qs = self._rows(q, n, self.Hq, "q")
        if out is None:
            out = torch.empty(q.shape, dtype=torch.bfloat16, device=self.device)
        else:
            self._fits(out, torch.bfloat16, (n, self.Hq, self.d), "out")
        lp = wp = None
        if lse is not None:
            self._fits(lse, torch.float32, (n, self.Hq), "lse")
            lp = lse.data_ptr()
        self._on_device(batch.kv_len, "batch")
        nbytes = lib.hermes_page_workspace_bytes(self._ref, batch._ref)
        if nbytes:
            ws = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            wp = ws.data_ptr()
        self._run(lib.hermes_page_attend, "hermes_page_attend", self._ref, batch._ref, q.data_ptr(), qs, out.data_ptr(),
                  lp, wp, nbytes)
        return out

    def read(self, batch: PageBatch, k: Optional[torch.Tensor] = None, v: Optional[torch.Tensor] = None):
        """The stored (k, v) of the batch's rows, bf16 [n_rows][n_kv_heads][d]."""
        shape = (batch.n_rows, self.Hkv, self.d)
        if k is None:
            k = torch.empty(shape, dtype=torch.bfloat16, device=self.device)
        else:
            self._fits(k, torch.bfloat16, shape, "k")
        if v is None:
            v = torch.empty(shape, dtype=torch.bfloat16, device=self.device)
        else:
            self._fits(v, torch.bfloat16, shape, "v")
        self._on_device(batch.kv_len, "batch")
        self._run(lib.hermes_page_read, "hermes_page_read", self._ref, batch._ref, k.data_ptr(), v.data_ptr())
        return k, v

    def reorder(self, tables: torch.Tensor, kv_len: torch.Tensor, parent: torch.Tensor, room: torch.Tensor, grow: int = 1,
                tables_out: Optional[torch.Tensor] = None, kv_len_out: Optional[torch.Tensor] = None):
        """The (tables, kv_len) that beams go on with after a choice: beam j of sequence s continues
        beam parent[s][j] (int32 [n_seqs][n_beams]; -1: none), in every layer.  tables int32
        [n_seqs][n_beams][max_pages], or with layers before them; kv_len likewise without pages;
        room int32 [.., n_seqs][2], first page and number of pages of the beams' own pages, which
        the tables of no other group of beams name.
        Full pages are shared, a partly filled one that is not a beam's own is copied, and there
        is room for `grow` tokens more (hermes_page_reorder)."""
        if not isinstance(tables, torch.Tensor) or tables.dim() < 3:
            raise ValueError("tables: expected [n_seqs][n_beams][max_pages], or with layers before them")
        shape = tables.shape
        n_seqs, n_beams, max_pages = shape[-3:]
        self._fits(tables, torch.int32, shape, "tables")
        self._fits(kv_len, torch.int32, shape[:-1], "kv_len")
        self._fits(parent, torch.int32, (n_seqs, n_beams), "parent")
        self._fits(room, torch.int32, shape[:-2] + (2,), "room")
        n_groups = math.prod(shape[:-2])
        if n_groups > _MOST or n_beams > _MOST or max_pages > _MOST or not 0 <= grow <= _MOST:
            raise HermesError(EINVAL, "hermes_page_reorder")
        if tables_out is None:
            tables_out = torch.empty_like(tables)
        else:
            self._fits(tables_out, torch.int32, shape, "tables_out")
        if kv_len_out is None:
            kv_len_out = torch.empty_like(kv_len)
        else:
            self._fits(kv_len_out, torch.int32, shape[:-1], "kv_len_out")
        s = PageBeamsStruct(n_groups, n_seqs, n_beams, max_pages, grow, parent.data_ptr(), room.data_ptr(),
                            tables.data_ptr(), kv_len.data_ptr(), tables_out.data_ptr(), kv_len_out.data_ptr())
        self._run(lib.hermes_page_reorder, "hermes_page_reorder", self._ref, ctypes.byref(s))
        return tables_out, kv_len_out

    def faults(self) -> int:
        bits = int(self._status.item())
        self._status.zero_()
        return bits


def beam_select(logits: torch.Tensor, score: torch.Tensor, keep: int, done: Optional[torch.Tensor] = None,
                end_token: int = -1, pad_token: int = 0):
    """The `keep` best continuations of every sequence (hermes_beam_select): logits bf16 or fp32
    [n_seqs][n_beams][n_vocab], whose rows may lie apart; score fp32 [n_seqs][n_beams]; done
    int32 likewise, other than 0 where a beam has ended.  Returns score fp32, parent, token and
    done int32, all [n_seqs][keep], the best first; parent and token are -1 where there are fewer."""
    if not isinstance(logits, torch.Tensor) or logits.dim() != 3 or logits.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("logits: expected torch.bfloat16 or torch.float32 [n_seqs][n_beams][n_vocab]")
    n_seqs, n_beams, n_vocab = logits.shape
    index = logits.get_device()
    if index < 0:
        raise ValueError("logits: must be a device tensor")
    ss, stride, es = logits.stride()
    if logits.numel() == 0 or n_seqs * n_beams == 1:
        stride = max(n_vocab, 1)
    elif n_beams == 1:
        stride = ss
    elif n_seqs > 1 and ss != n_beams * stride:
        raise ValueError("logits: rows must lie evenly apart")
    if es != 1 and n_vocab > 1:
        raise ValueError("logits: a row must be contiguous")
    _beams_of(score, torch.float32, (n_seqs, n_beams), index, "score")
    if done is not None:
        _beams_of(done, torch.int32, (n_seqs, n_beams), index, "done")
    if (n_seqs > _MOST or n_beams > _MOST or n_vocab > _MOST or not 1 <= keep <= _MOST or not -1 <= end_token <= _MOST
            or not 0 <= pad_token <= _MOST):
        raise HermesError(EINVAL, "hermes_beam_select")
    cfg = BeamConfig(n_seqs, n_beams, n_vocab, keep, FP32 if logits.dtype is torch.float32 else BF16, end_token, pad_token)
    ref = ctypes.byref(cfg)
    nbytes = lib.hermes_beam_workspace_bytes(ref)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=logits.device)
    best, parent, token, ended = torch.empty((4, n_seqs, keep), dtype=torch.int32, device=logits.device).unbind(0)
    best = best.view(torch.float32)
    _on(index, lib.hermes_beam_select, "hermes_beam_select", ref, logits.data_ptr(), stride, score.data_ptr(), _ptr(done),
        best.data_ptr(), parent.data_ptr(), token.data_ptr(), ended.data_ptr(), ws.data_ptr(), nbytes)
    return best, parent, token, ended


def _beams_of(t: torch.Tensor, dtype: torch.dtype, shape: tuple, index: int, name: str) -> None:
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name}: expected contiguous {dtype} {shape}, got {getattr(t, 'dtype', None)} "
                         f"{tuple(getattr(t, 'shape', ()))}")
    if t.get_device() != index:
        raise ValueError(f"{name}: a tensor on {t.device}, the logits are on device {index}")


class PackedWeight:
    """A weight in 4 bits (hermes_weight), made of `dense`, bf16 [n_out][n_in], which is not kept.

    Calls run on the current stream of its device; the weight is laid out when it is made, on the
    stream that is current then."""

    def __init__(self, dense: torch.Tensor):
        if not isinstance(dense, torch.Tensor) or dense.dim() != 2 or dense.dtype is not torch.bfloat16:
            raise ValueError("dense: expected torch.bfloat16 [n_out][n_in]")
        if not dense.is_cuda or (dense.stride(1) != 1 and dense.shape[1] > 1):
            raise ValueError("dense: must be a device tensor with contiguous rows")
        self.n_out, self.n_in = dense.shape
        self.device, self._index = dense.device, dense.get_device()
        w = WeightStruct(self.n_out, self.n_in, None)
        nbytes = lib.hermes_weight_bytes(ctypes.byref(w)) if max(dense.shape) <= _MOST else 0
        if nbytes == 0:
            raise HermesError(EINVAL, "hermes_weight_bytes")
        self.data = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        w.data = self.data.data_ptr()
        self._weight, self._ref = w, ctypes.byref(w)
        _on(self._index, lib.hermes_weight_pack, "hermes_weight_pack", self._ref, dense.data_ptr(),
            dense.stride(0) if self.n_out > 1 else self.n_in)

    def product(self, x: torch.Tensor, bias: Optional[torch.Tensor] = None, add: Optional[torch.Tensor] = None,
                out: Optional[torch.Tensor] = None, dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
        """x [n_rows][n_in] (bf16, 16-byte aligned, rows a multiple of 8 elements apart) times the weight's
        transpose, plus bias [n_out] and add [n_rows][n_out] (bf16): [n_rows][n_out] of bf16 or fp32
        (`dtype`, or `out`'s).  out may be add."""
        if not isinstance(x, torch.Tensor) or x.dtype is not torch.bfloat16 or x.dim() != 2 or x.shape[1] != self.n_in:
            raise ValueError(f"x: expected torch.bfloat16 [n_rows][{self.n_in}], got {getattr(x, 'dtype', None)} "
                             f"{tuple(getattr(x, 'shape', ()))}")
        n = x.shape[0]
        if n > _MOST:
            raise HermesError(EINVAL, "hermes_weight_product")
        shape = (n, self.n_out)
        self._on_device(x, "x")
        bp = ap = None
        if bias is not None:
            self._fits(bias, torch.bfloat16, (self.n_out,), "bias")
            bp = bias.data_ptr()
        if add is not None:
            self._fits(add, torch.bfloat16, shape, "add")
            ap = add.data_ptr()
        if out is not None:
            dtype = out.dtype if isinstance(out, torch.Tensor) else dtype
        kind = FP32 if dtype is torch.float32 else BF16
        if kind == BF16 and dtype is not torch.bfloat16:
            raise ValueError(f"dtype: torch.bfloat16 or torch.float32, got {dtype}")
        if out is None:
            out = torch.empty(shape, dtype=dtype, device=self.device)
        else:
            self._fits(out, dtype, shape, "out")
        stride, es = x.stride()
        if n <= 1:
            stride = -(-self.n_in // 8) * 8
        if n and (es != 1 and self.n_in > 1 or stride % 8 != 0):
            raise ValueError("x: a row must be contiguous, and rows a multiple of 8 elements apart")
        wp, nbytes = None, lib.hermes_weight_workspace_bytes(self._ref, n)
        if nbytes:
            ws = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            wp = ws.data_ptr()
        _on(self._index, lib.hermes_weight_product, "hermes_weight_product", self._ref, x.data_ptr(), stride, n, bp, ap,
            out.data_ptr(), kind, wp, nbytes)
        return out

    def _on_device(self, t: torch.Tensor, name: str) -> None:
        if t.get_device() != self._index:
            raise ValueError(f"{name}: a tensor on {t.device}, the weight is on {self.device}")

    def _fits(self, t: torch.Tensor, dtype: torch.dtype, shape: tuple, name: str) -> None:
        if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
            raise ValueError(f"{name}: expected contiguous {dtype} {shape}, got {getattr(t, 'dtype', None)} "
                             f"{tuple(getattr(t, 'shape', ()))}")
        self._on_device(t, name)


def default_sm_scale(head_dim: int) -> float:
    return 1.0 / math.sqrt(head_dim)
