"""Thin ctypes binding of the latent-cache operators (include/taper_latent.h): argument marshalling only, over the library that
binding.py loads."""
from __future__ import annotations

import ctypes
from typing import Optional

import numpy as np

from . import binding
from .binding import TAPER_EINVAL, TaperError, _check, _dev, _i32

LATENT_EXPORTED = [
    "taper_latent_create", "taper_latent_destroy", "taper_latent_plan_build", "taper_latent_prompt_plan_build",
    "taper_latent_plan_free", "taper_latent_plan_export", "taper_latent_decode_step_attention", "taper_latent_prompt_attention",
    "taper_latent_append",
]


class taper_latent_config(ctypes.Structure):
    _fields_ = [("n_heads", ctypes.c_int), ("latent_dim", ctypes.c_int), ("rope_dim", ctypes.c_int), ("head_dim", ctypes.c_int),
                ("page_size", ctypes.c_int), ("scale", ctypes.c_float), ("device", ctypes.c_int)]


class taper_latent_item(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("seq0", "page0", "n_tokens", "row0", "n_rows", "part_row")]


_I32P = ctypes.POINTER(ctypes.c_int32)


class taper_latent_view(ctypes.Structure):
    _fields_ = [("n_seqs", ctypes.c_int32), ("n_groups", ctypes.c_int32), ("n_items", ctypes.c_int32),
                ("items", ctypes.POINTER(taper_latent_item)), ("piece_start", _I32P), ("piece_row", _I32P),
                ("n_partial_rows", ctypes.c_int64), ("tokens_unique", ctypes.c_int64), ("tokens_logical", ctypes.c_int64),
                ("device_bytes", ctypes.c_int64)]


_bound = None


def _library() -> ctypes.CDLL:
    global _bound
    lib = binding.load_library()
    if _bound is lib:
        return lib
    vp, ci, i64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64
    pvp = ctypes.POINTER(vp)
    lib.taper_latent_create.argtypes = [ctypes.POINTER(taper_latent_config), pvp]
    lib.taper_latent_destroy.argtypes = [vp]
    lib.taper_latent_destroy.restype = None
    lib.taper_latent_plan_build.argtypes = [vp, ci, vp, ci, vp, vp, vp, vp, i64, ci, vp, pvp]
    lib.taper_latent_prompt_plan_build.argtypes = [vp, ci, vp, ci, vp, vp, vp, vp, i64, vp, pvp]
    lib.taper_latent_plan_free.argtypes = [vp]
    lib.taper_latent_plan_free.restype = None
    lib.taper_latent_plan_export.argtypes = [vp, ctypes.POINTER(taper_latent_view)]
    lib.taper_latent_decode_step_attention.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp]
    lib.taper_latent_prompt_attention.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp]
    lib.taper_latent_append.argtypes = [vp, i64, vp, i64, vp, i64, vp, vp, i64, vp]
    _bound = lib
    return lib


def _stream_of(device: int, stream) -> int:
    """The stream's handle; without one, torch's current stream of the operator's device."""
    if stream is not None:
        return int(stream) if isinstance(stream, int) else int(stream.cuda_stream)
    if device < 0:
        return 0
    if binding._raw_stream is not None:
        return binding._raw_stream(device)
    import torch
    return int(torch.cuda.current_stream(device).cuda_stream)


class LatentPlan:
    """Integer metadata of a decode step or of a batch of prompts (taper_latent_plan); n_rows: rows of q and out."""

    def __init__(self, ctx: "LatentContext", handle: int, prompt: bool, n_rows: int, n_pool_pages: int):
        self.ctx, self._h, self.prompt, self.n_rows, self.n_pool_pages = ctx, handle, prompt, int(n_rows), int(n_pool_pages)

    def free(self):
        if self._h and self.ctx._h:  # (a plan hands its memory back to its context)
            _library().taper_latent_plan_free(self._h)
        self._h = 0

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass

    def export(self) -> dict:
        """taper_latent_plan_export, copied into numpy arrays."""
        v = taper_latent_view()
        _check(_library().taper_latent_plan_export(self._h, ctypes.byref(v)))
        arr = lambda p, n: np.ctypeslib.as_array(p, shape=(n,)).copy() if n else np.zeros(0, np.int32)
        items = np.ctypeslib.as_array(ctypes.cast(v.items, _I32P), shape=(v.n_items, 6)).copy()
        start = arr(v.piece_start, v.n_seqs + 1)
        return dict(n_seqs=v.n_seqs, n_groups=v.n_groups, items=items, item_fields=[f[0] for f in taper_latent_item._fields_],
                    piece_start=start, piece_row=arr(v.piece_row, int(start[-1])), n_partial_rows=int(v.n_partial_rows),
                    tokens_unique=int(v.tokens_unique), tokens_logical=int(v.tokens_logical), device_bytes=int(v.device_bytes))


class LatentContext:
    """taper_latent_ctx: shape and memory of plans.  device=-1 gives a host-only context."""

    def __init__(self, n_heads: int, latent_dim: int, head_dim: int, rope_dim: int = 64, page_size: int = 16,
                 scale: Optional[float] = None, device: int = 0):
        lib = _library()
        cfg = taper_latent_config(n_heads, latent_dim, rope_dim, head_dim, page_size,
                                  float(scale if scale is not None else (head_dim + rope_dim) ** -0.5), device)
        h = ctypes.c_void_p()
        _check(lib.taper_latent_create(ctypes.byref(cfg), ctypes.byref(h)))
        self._h, self.cfg = h.value, cfg
        self._q_row, self._out_row = int(n_heads) * (int(head_dim) + int(rope_dim)), int(n_heads) * int(head_dim)
        self._w, self._page = int(n_heads) * 2 * int(head_dim) * int(latent_dim), int(page_size) * (int(latent_dim) + int(rope_dim))

    def close(self):
        if self._h:
            _library().taper_latent_destroy(self._h)
            self._h = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def plan_build(self, block_table, branch_group, prefix_len, suffix_len, n_pool_pages: int, target_workgroups: int = 0,
                   seg_start=None, stream=None) -> LatentPlan:
        """Plan of a decode step.  seg_start: sequences see lists of private segments, of the lengths suffix_len (reduce phase)."""
        bt, grp, pl, sl = _i32(block_table), _i32(branch_group), _i32(prefix_len), _i32(suffix_len)
        ss = _i32(seg_start) if seg_start is not None else None
        if bt.ndim != 2 or not (len(grp) == len(pl) == bt.shape[0]) or (len(sl) != bt.shape[0] if ss is None else len(ss) != bt.shape[0] + 1 or ss[-1] != len(sl)):
            raise TaperError(TAPER_EINVAL, "block_table must be [S, max_blocks], the per-sequence arrays length S, seg_start length S + 1 ending at len(suffix_len)")
        h = ctypes.c_void_p()
        _check(_library().taper_latent_plan_build(self._h, bt.shape[0], bt.ctypes.data, bt.shape[1], grp.ctypes.data, pl.ctypes.data,
                                                  ss.ctypes.data if ss is not None else None, sl.ctypes.data, int(n_pool_pages),
                                                  int(target_workgroups), _stream_of(self.cfg.device, stream), ctypes.byref(h)))
        return LatentPlan(self, h.value, False, bt.shape[0], n_pool_pages)

    def prompt_plan_build(self, block_table, branch_group, prefix_len, suffix_len, new_len, n_pool_pages: int, stream=None) -> LatentPlan:
        """Plan for the last new_len[s] private tokens of each sequence as query rows."""
        bt, grp, pl, sl, nl = _i32(block_table), _i32(branch_group), _i32(prefix_len), _i32(suffix_len), _i32(new_len)
        if bt.ndim != 2 or not (len(grp) == len(pl) == len(sl) == len(nl) == bt.shape[0]):
            raise TaperError(TAPER_EINVAL, "block_table must be [S, max_blocks] and the per-sequence arrays length S")
        h = ctypes.c_void_p()
        _check(_library().taper_latent_prompt_plan_build(self._h, bt.shape[0], bt.ctypes.data, bt.shape[1], grp.ctypes.data, pl.ctypes.data,
                                                         sl.ctypes.data, nl.ctypes.data, int(n_pool_pages),
                                                         _stream_of(self.cfg.device, stream), ctypes.byref(h)))
        return LatentPlan(self, h.value, True, int(nl.sum(dtype=np.int64)), n_pool_pages)

    def _ptrs(self, plan: LatentPlan, q, w_up, pages, out, lse):
        d, n = self.cfg.device, plan.n_rows
        return (_dev(q, "q", n * self._q_row, "bfloat16", d), _dev(w_up, "w_up", self._w, "bfloat16", d),
                _dev(pages, "pages", plan.n_pool_pages * self._page, "bfloat16", d), _dev(out, "out", n * self._out_row, "bfloat16", d),
                _dev(lse, "lse", n * self.cfg.n_heads, "float32", d) if lse is not None else None)

    def decode_step_attention(self, plan: LatentPlan, q, w_up, pages, out, lse=None, stream=None):
        status = _bound.taper_latent_decode_step_attention(self._h, plan._h, *self._ptrs(plan, q, w_up, pages, out, lse), _stream_of(self.cfg.device, stream))
        if status:
            _check(status)

    def prompt_attention(self, plan: LatentPlan, q, w_up, pages, out, lse=None, stream=None):
        status = _bound.taper_latent_prompt_attention(self._h, plan._h, *self._ptrs(plan, q, w_up, pages, out, lse), _stream_of(self.cfg.device, stream))
        if status:
            _check(status)

    def append(self, latent, rope, slots, pages, n_pool_pages: int, stream=None):
        """Writes latent [n, latent_dim] and rope [n, rope_dim] (rows may be strided, so that both can be parts of one tensor) to the
        pool's slots [n]; slots outside the pool leave their token out."""
        d, n = self.cfg.device, int(slots.shape[0])
        rows = []
        for t, what, width in ((latent, "latent", self.cfg.latent_dim), (rope, "rope", self.cfg.rope_dim)):
            if t.dim() != 2 or t.shape[0] != n or t.shape[1] != width or (t.stride(1) != 1 and n > 0):
                raise TaperError(TAPER_EINVAL, f"{what} must be [{n}, {width}] with contiguous rows, got {tuple(t.shape)} with strides {t.stride()}")
            if str(t.dtype) != "torch.bfloat16" or t.device.type != "cuda" or (t.device.index or 0) != d:
                raise TaperError(TAPER_EINVAL, f"{what} must be bfloat16 on cuda:{d}, got {t.dtype} on {t.device}")
            rows += [t.data_ptr(), t.stride(0) if n > 1 else width]  # (torch gives the stride of a single row any value)
        status = _bound.taper_latent_append(self._h, n, *rows, _dev(slots, "slots", n, "int64", d),
                                            _dev(pages, "pages", int(n_pool_pages) * self._page, "bfloat16", d), int(n_pool_pages),
                                            _stream_of(d, stream))
        if status:
            _check(status)
