"""Thin ctypes binding of the page operators (include/taper_pages.h): argument marshalling only, over the library that binding.py
loads."""
from __future__ import annotations

import ctypes
from typing import Sequence

import numpy as np

from . import binding
from .binding import TAPER_EINVAL, TaperError, _check, _dev, _i32
from .latent import _stream_of

PAGES_EXPORTED = [
    "taper_page_pool_create", "taper_page_pool_destroy", "taper_page_pool_free_pages", "taper_page_pool_users",
    "taper_page_pool_alloc", "taper_page_pool_share", "taper_page_pool_release", "taper_page_pool_fork", "taper_page_pool_compact",
    "taper_pages_remap", "taper_mover_create", "taper_mover_destroy", "taper_pages_copy", "taper_pages_pack",
]
PAGE_KINDS = {"kv": 0, "latent": 1}


class taper_page_format(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int), ("n_heads", ctypes.c_int), ("dim", ctypes.c_int), ("page_size", ctypes.c_int), ("device", ctypes.c_int)]


_bound = None


def _library() -> ctypes.CDLL:
    global _bound
    lib = binding.load_library()
    if _bound is lib:
        return lib
    vp, ci, i32, i64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int32, ctypes.c_int64
    pvp, pi64, pi32 = ctypes.POINTER(vp), ctypes.POINTER(i64), ctypes.POINTER(i32)
    lib.taper_page_pool_create.argtypes = [i64, pvp]
    lib.taper_page_pool_destroy.argtypes = [vp]
    lib.taper_page_pool_destroy.restype = None
    lib.taper_page_pool_free_pages.argtypes = [vp]
    lib.taper_page_pool_free_pages.restype = i64
    lib.taper_page_pool_users.argtypes = [vp, i32]
    lib.taper_page_pool_users.restype = i32
    lib.taper_page_pool_alloc.argtypes = [vp, i64, vp]
    lib.taper_page_pool_share.argtypes = [vp, i64, vp]
    lib.taper_page_pool_release.argtypes = [vp, i64, vp, pi64]
    lib.taper_page_pool_fork.argtypes = [vp, vp, i64, ci, vp, pi32, pi32]
    lib.taper_page_pool_compact.argtypes = [vp, i64, vp, vp, pi64]
    lib.taper_pages_remap.argtypes = [i64, vp, i64, vp, vp]
    lib.taper_mover_create.argtypes = [ctypes.POINTER(taper_page_format), pvp]
    lib.taper_mover_destroy.argtypes = [vp]
    lib.taper_mover_destroy.restype = None
    lib.taper_pages_copy.argtypes = [vp, ci, vp, i64, vp, vp, i64, vp]
    lib.taper_pages_pack.argtypes = [vp, ci, vp, ci, vp, ci, vp, vp, vp, vp, vp, ci, i64, vp]
    _bound = lib
    return lib


class PagePool:
    """Who uses each page of a pool (taper_page_pool): host integers, no device memory."""

    def __init__(self, n_pages: int):
        h = ctypes.c_void_p()
        _check(_library().taper_page_pool_create(int(n_pages), ctypes.byref(h)))
        self._h, self.n_pages = h.value, int(n_pages)

    def close(self):
        if self._h:
            _library().taper_page_pool_destroy(self._h)
            self._h = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def free_pages(self) -> int:
        return _library().taper_page_pool_free_pages(self._h)

    def users(self, page: int) -> int:
        return _library().taper_page_pool_users(self._h, int(page))

    def alloc(self, n: int) -> np.ndarray:
        pages = np.zeros(max(0, int(n)), np.int32)
        _check(_library().taper_page_pool_alloc(self._h, int(n), pages.ctypes.data))
        return pages

    def share(self, pages):
        p = _i32(pages).ravel()
        _check(_library().taper_page_pool_share(self._h, len(p), p.ctypes.data))

    def release(self, pages) -> int:
        """One user less for each entry; returns how many pages became free."""
        p, freed = _i32(pages).ravel(), ctypes.c_int64()
        _check(_library().taper_page_pool_release(self._h, len(p), p.ctypes.data, ctypes.byref(freed)))
        return freed.value

    def fork(self, parent_row, n_tokens: int, page_size: int = 16):
        """(child row, (source, destination) of the page to copy or None) for a child of the run's first n_tokens tokens."""
        row = _i32(parent_row).ravel()
        n = (int(n_tokens) + page_size - 1) // page_size
        if n > len(row):
            raise TaperError(TAPER_EINVAL, f"{n_tokens} tokens need {n} pages, the row has {len(row)}")
        child, src, dst = np.zeros(max(0, n), np.int32), ctypes.c_int32(), ctypes.c_int32()
        _check(_library().taper_page_pool_fork(self._h, row.ctypes.data, int(n_tokens), int(page_size), child.ctypes.data,
                                               ctypes.byref(src), ctypes.byref(dst)))
        return child, ((src.value, dst.value) if src.value >= 0 else None)

    def compact(self, max_moves: int = -1):
        """(src, dst) of the moves that bring the live pages to the front; the pool counts them at their new places already."""
        most = self.n_pages if max_moves < 0 else min(int(max_moves), self.n_pages)
        src, dst, n = np.zeros(most, np.int32), np.zeros(most, np.int32), ctypes.c_int64()
        _check(_library().taper_page_pool_compact(self._h, most, src.ctypes.data, dst.ctypes.data, ctypes.byref(n)))
        return src[:n.value].copy(), dst[:n.value].copy()


def remap_pages(entries, src, dst) -> np.ndarray:
    """Block-table entries with the moved pages' new places (a new array)."""
    e, s, d = _i32(entries).copy(), _i32(src), _i32(dst)
    if s.shape != d.shape or s.ndim != 1:
        raise TaperError(TAPER_EINVAL, "src and dst must be lists of one length")
    _check(_library().taper_pages_remap(e.size, e.ctypes.data, len(s), s.ctypes.data, d.ctypes.data))
    return e


class PageMover:
    """taper_mover: moves pages and tokens of the pools of all layers.  device=-1 only checks arguments."""

    def __init__(self, kind, n_heads: int, dim: int, page_size: int = 16, device: int = 0):
        fmt = taper_page_format(PAGE_KINDS[kind] if isinstance(kind, str) else int(kind), int(n_heads), int(dim), int(page_size), int(device))
        h = ctypes.c_void_p()
        _check(_library().taper_mover_create(ctypes.byref(fmt), ctypes.byref(h)))
        self._h, self.format = h.value, fmt
        self._page = int(page_size) * int(n_heads) * int(dim) * (2 if fmt.kind == 0 else 1)

    @classmethod
    def kv(cls, n_kv_heads: int, head_dim: int, page_size: int = 16, device: int = 0) -> "PageMover":
        return cls("kv", n_kv_heads, head_dim, page_size, device)

    @classmethod
    def latent(cls, latent_dim: int, rope_dim: int = 64, page_size: int = 16, device: int = 0) -> "PageMover":
        return cls("latent", 1, latent_dim + rope_dim, page_size, device)

    def close(self):
        if self._h:
            _library().taper_mover_destroy(self._h)
            self._h = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _pools(self, pools: Sequence, n_pool_pages: int):
        ptrs = [_dev(p, "pool", int(n_pool_pages) * self._page, "bfloat16", self.format.device) for p in pools]
        return len(ptrs), (ctypes.c_void_p * max(1, len(ptrs)))(*ptrs)

    def copy(self, pools: Sequence, src, dst, n_pool_pages: int, stream=None):
        """Page dst[i] becomes a copy of page src[i] in every pool."""
        s, d = _i32(src), _i32(dst)
        if s.shape != d.shape or s.ndim != 1:
            raise TaperError(TAPER_EINVAL, "src and dst must be lists of one length")
        n, ptrs = self._pools(pools, n_pool_pages)
        _check(_library().taper_pages_copy(self._h, n, ptrs, len(s), s.ctypes.data, d.ctypes.data, int(n_pool_pages),
                                           _stream_of(self.format.device, stream)))

    def pack(self, pools: Sequence, block_table, prefix_len, seg_start, seg_len, dst_table, n_pool_pages: int, first_token=None, stream=None):
        """Each sequence's tokens (prefix, then segments) from first_token on, one after the other on the pages of dst_table."""
        bt, pl, ss, sl, dt = _i32(block_table), _i32(prefix_len), _i32(seg_start), _i32(seg_len), _i32(dst_table)
        ft = _i32(first_token) if first_token is not None else None
        S = len(pl)
        if bt.ndim != 2 or dt.ndim != 2 or not (bt.shape[0] == dt.shape[0] == len(ss) - 1 == S) or ss[-1] != len(sl) or (ft is not None and len(ft) != S):
            raise TaperError(TAPER_EINVAL, "block_table and dst_table must be [S, ...], prefix_len and first_token length S, seg_start length S + 1 ending at len(seg_len)")
        n, ptrs = self._pools(pools, n_pool_pages)
        _check(_library().taper_pages_pack(self._h, n, ptrs, S, bt.ctypes.data, bt.shape[1], pl.ctypes.data, ss.ctypes.data,
                                           sl.ctypes.data if len(sl) else None, ft.ctypes.data if ft is not None else None,
                                           dt.ctypes.data, dt.shape[1], int(n_pool_pages), _stream_of(self.format.device, stream)))
