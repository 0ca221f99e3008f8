"""Pages of a paged pool over the C-ABI library: handing out, giving back, forking sequences, compacting (include/tsv.h, "Pages
of a paged pool").  Argument marshalling and checks only.

A pool is a page table, a count of holders per page, the PLANES that hold the pages' contents (csa_kv, csa_ik, hca_kv, win_kv of
every layer; k and v of token caches) and the ROWS with what a sequence has besides (lengths, capacities, open-block states).
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Sequence

import torch

from . import binding as tsv
from .binding import TsvError, _lib, _p
from .tokens import ST_PAGE, ST_POOL, _bad, _device, _flat, _i32, _on, _workspace  # noqa: F401

MAX_LIST = 1024


class CPageArray(C.Structure):
    _fields_ = [("base", _p), ("bytes", C.c_int64)]


class CPagePool(C.Structure):
    _fields_ = [("page_table", _p), ("ref", _p), ("slots", C.c_int32), ("max_pages", C.c_int32), ("n_pages", C.c_int32), ("page_tokens", C.c_int32),
                ("planes", _p), ("rows", _p), ("n_planes", C.c_int32), ("n_rows", C.c_int32)]


_lib.tsv_pages_workspace_bytes.restype = C.c_size_t
_lib.tsv_pages_workspace_bytes.argtypes = [_p]
_lib.pages_assign.restype = C.c_int
_lib.pages_assign.argtypes = [_p, C.c_int32, _p, _p, _p, _p, C.c_size_t, _p, _p]
_lib.pages_free.restype = C.c_int
_lib.pages_free.argtypes = [_p, C.c_int32, _p, _p, _p, _p, _p]
_lib.pages_fork.restype = C.c_int
_lib.pages_fork.argtypes = [_p, C.c_int32, _p, _p, _p, _p, C.c_size_t, _p, _p]
_lib.pages_compact.restype = C.c_int
_lib.pages_compact.argtypes = [_p, _p, _p, C.c_size_t, _p]

_at = C.addressof


def counts_of(page_table: torch.Tensor, n_pages: int) -> torch.Tensor:
    """How many words of the table name each page (int32); words that name none of the pool's count for nothing."""
    held = page_table.flatten().long()
    return torch.zeros(n_pages, dtype=torch.int32, device=held.device).index_add_(0, held.clamp(0, n_pages - 1), ((held >= 0) & (held < n_pages)).int())


class PagePool:
    """Description of a pool over the caller's tensors, which it keeps: page_table [slots, max_pages] and ref [n_pages] (int32), planes
    (contiguous, the same share of each belongs to a page) and rows (contiguous, [slots, ...])."""

    def __init__(self, page_table: torch.Tensor, ref: torch.Tensor, page_tokens: int, planes: Sequence[torch.Tensor], rows: Sequence[torch.Tensor] = ()):
        if not isinstance(page_table, torch.Tensor) or page_table.dim() != 2 or not isinstance(ref, torch.Tensor):
            raise TsvError(tsv.ERR_SHAPE, "PagePool: expected page_table [slots, max_pages] and ref [n_pages]")
        slots, max_pages = page_table.shape
        n = ref.numel()
        self.page_table, self.ref, self.planes, self.rows = page_table, ref, list(planes), list(rows)
        for t, parts, what in [(t, n, "plane") for t in self.planes] + [(t, slots, "row array") for t in self.rows]:
            if not t.is_cuda or t.device != page_table.device or not t.is_contiguous() or t.numel() % parts:
                raise TsvError(tsv.ERR_SHAPE, f"PagePool: a {what} must be contiguous on {page_table.device} and divide into {parts}, got {tuple(t.shape)}")
        arrays = lambda ts, parts: (CPageArray * max(1, len(ts)))(*[CPageArray(t.data_ptr(), t.numel() // parts * t.element_size()) for t in ts])
        self._planes, self._rows = arrays(self.planes, n), arrays(self.rows, slots)
        dev = page_table.get_device()
        self.c = CPagePool(_flat("page_table", page_table, _i32, slots * max_pages, dev), _flat("ref", ref, _i32, n, dev), slots, max_pages, n,
                           page_tokens, _at(self._planes), _at(self._rows), len(self.planes), len(self.rows))
        self.device = dev

    @staticmethod
    def of_layers(caches: Sequence[tsv.LayerCache], ref: Optional[torch.Tensor] = None) -> "PagePool":
        """The pool behind the paged caches of layers that share one page table tensor and the size and number of its pages; ref: the counts, by
        default those that the table shows."""
        c0 = caches[0] if len(caches) else None
        if c0 is None or c0.page_table is None or any(c.page_table is None or c.page_table.data_ptr() != c0.page_table.data_ptr() for c in caches):
            raise TsvError(tsv.ERR_SHAPE, "PagePool.of_layers: the layers must share one page table")
        if any(c.page_tokens != c0.page_tokens or c.win_kv.shape[0] != c0.win_kv.shape[0] for c in caches):
            raise TsvError(tsv.ERR_SHAPE, f"PagePool.of_layers: page sizes {[c.page_tokens for c in caches]} and token rows {[c.win_kv.shape[0] for c in caches]} differ")
        n = c0.win_kv.shape[0] // c0.page_tokens
        if ref is None:
            ref = counts_of(c0.page_table, n)
        planes = [t for c in caches for t in (c.csa_kv, c.csa_ik, c.hca_kv, c.win_kv)]
        rows = [t for c in caches for t in (c.L, c.csa_cap, c.hca_cap, c.csa_mx, c.csa_s, c.csa_acc_kv, c.csa_acc_ik, c.hca_mx, c.hca_s, c.hca_acc_kv)]
        return PagePool(c0.page_table, ref, c0.page_tokens, planes, rows)


def alloc_workspace(pool: PagePool) -> torch.Tensor:
    n = int(_lib.tsv_pages_workspace_bytes(_at(pool.c)))
    if n == 0:
        raise TsvError(tsv.ERR_SHAPE, "tsv_pages_workspace_bytes")
    return torch.empty(n + 256, dtype=torch.uint8, device=pool.page_table.device)


def _here(pool: PagePool) -> int:
    dev = _device()
    if pool.device != dev:
        _bad("pool", "a pool", pool.page_table)
    return dev


def _count(where: str, t: torch.Tensor) -> int:
    try:
        return t.numel()
    except AttributeError:
        _bad(where, "an int32 tensor", t)


def pages_assign(pool: PagePool, slots: torch.Tensor, first: torch.Tensor, last: torch.Tensor, workspace: torch.Tensor, status: torch.Tensor,
                 stream=None) -> None:
    """Logical pages first[i] .. last[i] - 1 of slots[i] that have no page get the free ones with the lowest numbers."""
    n, dev = _count("slots", slots), _here(pool)
    wp, wn = _workspace(workspace, dev)
    r = _lib.pages_assign(_at(pool.c), n, _flat("slots", slots, _i32, n, dev), _flat("first", first, _i32, n, dev), _flat("last", last, _i32, n, dev), wp, wn,
                          _flat("status", status, _i32, n, dev), _on(stream, dev))
    if r:
        raise TsvError(r, "pages_assign")


def pages_free(pool: PagePool, slots: torch.Tensor, first: torch.Tensor, last: torch.Tensor, status: torch.Tensor, stream=None) -> None:
    """slots[i] gives up its logical pages first[i] .. last[i] - 1."""
    n, dev = _count("slots", slots), _here(pool)
    r = _lib.pages_free(_at(pool.c), n, _flat("slots", slots, _i32, n, dev), _flat("first", first, _i32, n, dev), _flat("last", last, _i32, n, dev),
                        _flat("status", status, _i32, n, dev), _on(stream, dev))
    if r:
        raise TsvError(r, "pages_free")


def pages_fork(pool: PagePool, src: torch.Tensor, dst: torch.Tensor, L: torch.Tensor, workspace: torch.Tensor, status: torch.Tensor, stream=None) -> None:
    """dst[i], a slot without pages, becomes a copy of src[i] with L[src[i]] tokens: full pages shared, the last one and the rows copied."""
    n, dev = _count("src", src), _here(pool)
    wp, wn = _workspace(workspace, dev)
    r = _lib.pages_fork(_at(pool.c), n, _flat("src", src, _i32, n, dev), _flat("dst", dst, _i32, n, dev), _flat("L", L, _i32, pool.c.slots, dev), wp, wn,
                        _flat("status", status, _i32, n, dev), _on(stream, dev))
    if r:
        raise TsvError(r, "pages_fork")


def pages_compact(pool: PagePool, n_used: torch.Tensor, workspace: torch.Tensor, stream=None) -> None:
    """The used pages move to the lowest numbers, contents, table and counts; n_used (int32, 1 value) becomes their number."""
    dev = _here(pool)
    wp, wn = _workspace(workspace, dev)
    r = _lib.pages_compact(_at(pool.c), _flat("n_used", n_used, _i32, 1, dev), wp, wn, _on(stream, dev))
    if r:
        raise TsvError(r, "pages_compact")
