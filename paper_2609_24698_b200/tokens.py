"""Token-level layers over the C-ABI library: norms and rotation of new queries and keys, attention over sinks and a sliding
window, and the token cache (include/tsv.h, "Token-level layers").  Argument marshalling and checks only.

    qk_norm_rope(...)        queries and keys of the new tokens, normed per head and rotated to their positions
    window_sink_attn(...)    their attention over the token cache and each other (chains or draft trees)
    token_commit(...)        accepted tokens' rows into the cache, lengths bumped

New tokens are packed: sequence b's are rows row0[b] .. row0[b] + n[b] - 1 of [rows, heads, d] tensors, whose rows may be
strided (column ranges of one projection).
"""
from __future__ import annotations

import ctypes as C
from dataclasses import dataclass, field
from struct import Struct
from typing import Optional

import torch

from . import binding as tsv
from .binding import TsvError, _aligned, _lib, _p

ST_PAGE, ST_POOL = 64, 128


class CTokShape(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("B", C.c_int32), ("H", C.c_int32), ("Hk", C.c_int32), ("d", C.c_int32), ("window", C.c_int32),
                ("n_sink", C.c_int32), ("max_n", C.c_int32), ("max_L", C.c_int64), ("sm_scale", C.c_float), ("reserved", C.c_int32)]


class CTokCache(C.Structure):
    _fields_ = [("L", _p), ("k", _p), ("v", _p), ("rows", C.c_int64), ("page_table", _p), ("page_tokens", C.c_int32), ("max_pages", C.c_int32)]


class CTokBatch(C.Structure):
    _fields_ = [("row0", _p), ("n", _p), ("parent", _p), ("rows", C.c_int64)]


class CTokRows(C.Structure):
    _fields_ = [("q", _p), ("k", _p), ("v", _p), ("q_ld", C.c_int64), ("k_ld", C.c_int64), ("v_ld", C.c_int64)]


_lib.qk_norm_rope.restype = C.c_int
_lib.qk_norm_rope.argtypes = [_p, _p, _p, _p, _p, _p, C.c_float, _p, C.c_int32, C.c_int32, C.c_int32, _p, C.c_int64, _p, C.c_int64, _p, _p]
_lib.tsv_tok_workspace_bytes.restype = C.c_size_t
_lib.tsv_tok_workspace_bytes.argtypes = [_p, C.c_int64]
_lib.window_sink_attn.restype = C.c_int
_lib.window_sink_attn.argtypes = [_p, _p, _p, _p, _p, _p, C.c_size_t, _p, _p]
_lib.token_commit.restype = C.c_int
_lib.token_commit.argtypes = [_p, _p, _p, _p, _p, C.c_int32, _p, _p, _p]

_at = C.addressof
# The structs of a call as bytes: ctypes takes some microseconds to make one, these are made anew for every call.
_pack_cache, _pack_batch, _pack_rows = Struct("3PqP2i").pack, Struct("3Pq").pack, Struct("3P3q").pack
assert Struct("3PqP2i").size == C.sizeof(CTokCache) and Struct("3Pq").size == C.sizeof(CTokBatch) and Struct("3P3q").size == C.sizeof(CTokRows)
_device, _raw_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
_i32, _i64, _f32 = torch.int32, torch.int64, torch.float32


def _on(stream, dev: int) -> int:
    return _raw_stream(dev) if stream is None else stream.cuda_stream


@dataclass
class TokenShape:
    """Shape of a token-level layer and of the calls on it (bounds size grids and workspace; fixed once made)."""
    dtype: str            # "fp32" | "bf16"
    B: int                # sequences
    H: int                # query heads
    Hk: int               # key/value heads
    d: int                # head dim
    window: int           # a query at p sees p - window + 1 .. p
    n_sink: int = 0       # and 0 .. n_sink - 1
    max_L: int = 1 << 20  # bound on L + new tokens of a sequence
    max_n: int = 1        # bound on new tokens of a sequence
    sm_scale: float = 0.0  # 0 -> 1/sqrt(d)
    c: CTokShape = field(init=False, repr=False, compare=False)

    def __post_init__(self):
        if self.dtype not in ("fp32", "bf16"):
            raise TsvError(tsv.ERR_SHAPE, "TokenShape")
        self.torch_dtype = torch.bfloat16 if self.dtype == "bf16" else torch.float32
        self.c = CTokShape(tsv.TSV_BF16 if self.dtype == "bf16" else tsv.TSV_FP32, self.B, self.H, self.Hk, self.d, self.window, self.n_sink,
                           self.max_n, self.max_L, float(self.sm_scale), 0)


def _bad(where: str, expected: str, t) -> None:
    got = f"{t.dtype} {tuple(t.shape)} with strides {t.stride()} on {t.device}" if isinstance(t, torch.Tensor) else repr(t)
    raise TsvError(tsv.ERR_SHAPE, f"{where}: expected {expected} on the current CUDA device, got {got}")


def _flat(where: str, t: torch.Tensor, dtype: torch.dtype, numel: int, dev: int) -> int:
    """Pointer of a contiguous tensor of at least `numel` elements on device dev."""
    try:                                      # (what is no tensor has no dtype: asking it first takes a microsecond a call)
        if t.dtype is dtype and t.numel() >= numel and t.is_contiguous() and t.get_device() == dev:
            return t.data_ptr()
    except AttributeError:
        pass
    _bad(where, f"a contiguous {dtype} tensor of {numel} elements", t)


def _maybe(where: str, t: Optional[torch.Tensor], dtype: torch.dtype, numel: int, dev: int) -> int:
    return 0 if t is None else _flat(where, t, dtype, numel, dev)


def _table(where: str, t: Optional[torch.Tensor], rows: int, dev: int):
    """Pointer and row length of an int32 table of at least `rows` rows; (0, 0) for None."""
    if t is None:
        return 0, 0
    try:
        _, ld = t.shape
    except (AttributeError, ValueError):
        _bad(where, f"an int32 tensor of {rows} rows", t)
    return _flat(where, t, _i32, rows * ld, dev), ld


def _workspace(workspace: torch.Tensor, dev: int):
    try:
        if workspace.get_device() == dev:
            return _aligned(workspace)
    except AttributeError:
        pass
    _bad("workspace", "a workspace", workspace)


def _vectors(where: str, t: torch.Tensor, dtype: torch.dtype, rows: int, heads: int, d: int, dev: int):
    """Pointer and row stride of a [>= rows, heads, d] tensor whose heads follow each other in a row."""
    try:
        s = t.shape
        if t.dtype is dtype and len(s) == 3 and s[0] >= rows and s[1] == heads and s[2] == d and t.get_device() == dev:
            ld, hs, es = t.stride()
            if es == 1 and (hs == d or heads == 1):
                return t.data_ptr(), (ld if s[0] > 1 else heads * d)
    except AttributeError:
        pass
    _bad(where, f"a {dtype} tensor [{rows}, {heads}, {d}] whose rows are contiguous", t)


def _rows(where: str, t: torch.Tensor) -> int:
    try:
        return t.shape[0]
    except (AttributeError, IndexError):
        _bad(where, "a tensor of rows", t)


@dataclass
class TokenBatch:
    """New tokens of B sequences: packed rows, chains or (parent given) draft trees."""
    row0: torch.Tensor                        # [B] int64
    n: torch.Tensor                           # [B] int32
    parent: Optional[torch.Tensor] = None     # [rows] int32, node of the same sequence, -1 for node 0

    def pack(self, B: int, rows: int, dev: int) -> bytes:
        return _pack_batch(_flat("row0", self.row0, _i64, B, dev), _flat("n", self.n, _i32, B, dev),
                           0 if self.parent is None else _flat("parent", self.parent, _i32, rows, dev), rows)


@dataclass
class TokenCache:
    """Committed keys (and values) of a layer, a row per token: a ring of n_sink + window rows per sequence, or pages."""
    L: torch.Tensor                           # [B] int32
    k: torch.Tensor                           # [..., Hk, d] rows
    v: Optional[torch.Tensor] = None          # None: the keys are the values
    page_table: Optional[torch.Tensor] = None  # [B, max_pages] int32
    page_tokens: int = 0
    ring: Optional[tuple] = None              # (n_sink, window) that the rows of a ring are laid out for, if known
    commits: bool = True                      # False: the sequences advance by another call, and token_commit refuses

    @staticmethod
    def of_layer(cache: tsv.LayerCache) -> "TokenCache":
        """The token-level KV of a verify layer, to be read: its window ring (n_sink = 0 and the layer's window then), or its pool's third
        physical layer.  L, compressed entries and open blocks of the layer advance together, by accept_and_refresh, so token_commit refuses."""
        ring = None if cache.page_table is not None else (0, cache.win_kv.shape[1])
        return TokenCache(cache.L, cache.win_kv, None, cache.page_table, cache.page_tokens, ring, False)

    def pack(self, shape: TokenShape, dev: int) -> bytes:
        dt, width, k, table = shape.torch_dtype, shape.Hk * shape.d, self.k, self.page_table
        if self.ring is not None and self.ring != (shape.n_sink, shape.window):
            raise TsvError(tsv.ERR_SHAPE, f"cache: rings of (n_sink, window) = {self.ring}, the shape has {(shape.n_sink, shape.window)}")
        kp, rows = _flat("cache.k", k, dt, width, dev), k.numel() // width
        tp, max_pages = _table("page_table", table, shape.B, dev)
        return _pack_cache(_flat("L", self.L, _i32, shape.B, dev), kp, _maybe("cache.v", self.v, dt, rows * width, dev), rows, tp, self.page_tokens, max_pages)


def alloc_token_cache(shape: TokenShape, values: bool = True, device="cuda") -> TokenCache:
    """Empty rings (L = 0) for the shape's sequences."""
    z = lambda: torch.zeros(shape.B, shape.n_sink + shape.window, shape.Hk, shape.d, dtype=shape.torch_dtype, device=device)
    return TokenCache(torch.zeros(shape.B, dtype=torch.int32, device=device), z(), z() if values else None, ring=(shape.n_sink, shape.window))


def alloc_token_pool(shape: TokenShape, n_pages: int, page_tokens: int, max_pages: int, values: bool = True, device="cuda") -> TokenCache:
    """An empty pool: no sequence holds a page yet (pages.pages_assign gives them out)."""
    z = lambda: torch.zeros(n_pages * page_tokens, shape.Hk, shape.d, dtype=shape.torch_dtype, device=device)
    return TokenCache(torch.zeros(shape.B, dtype=torch.int32, device=device), z(), z() if values else None,
                      torch.full((shape.B, max_pages), -1, dtype=torch.int32, device=device), page_tokens)


def alloc_workspace(shape: TokenShape, rows: int, device="cuda") -> torch.Tensor:
    """Workspace of window_sink_attn for calls of up to `rows` packed rows."""
    n = int(_lib.tsv_tok_workspace_bytes(_at(shape.c), rows))
    if n == 0:
        raise TsvError(tsv.ERR_SHAPE, "tsv_tok_workspace_bytes")
    return torch.empty(n + 256, dtype=torch.uint8, device=device)


def _raise(r: int, where: str) -> None:
    if r:
        raise TsvError(r, where)


def qk_norm_rope(shape: TokenShape, L: torch.Tensor, batch: TokenBatch, q: Optional[torch.Tensor], k: Optional[torch.Tensor],
                 q_out: Optional[torch.Tensor], k_out: Optional[torch.Tensor], wq: Optional[torch.Tensor], wk: Optional[torch.Tensor], eps: float,
                 inv_freq: Optional[torch.Tensor], first: int, pairs: bool, status: torch.Tensor, stream=None) -> None:
    """q [rows, H, d], k [rows, Hk, d] -> q_out, k_out (may be the inputs): per-head RMS norm with weights [d] fp32, then dims first ..
    first + 2 len(inv_freq) - 1 rotated to the tokens' positions; pairs: neighbouring dims turn together (else i and i + rot / 2)."""
    dt, dev = shape.torch_dtype, _device()
    some = q if q is not None else k
    if some is None:
        raise TsvError(tsv.ERR_NULL, "qk_norm_rope")
    rows, H, Hk, d = _rows("q" if q is not None else "k", some), shape.H, shape.Hk, shape.d
    qp = qo = kp = ko = ql = qol = kl = kol = 0
    if q is not None:
        (qp, ql), (qo, qol) = _vectors("q", q, dt, rows, H, d, dev), _vectors("q_out", q_out, dt, rows, H, d, dev)
    if k is not None:
        (kp, kl), (ko, kol) = _vectors("k", k, dt, rows, Hk, d, dev), _vectors("k_out", k_out, dt, rows, Hk, d, dev)
    rot = 0 if inv_freq is None else 2 * inv_freq.numel()
    r = _lib.qk_norm_rope(_at(shape.c), _flat("L", L, _i32, shape.B, dev), batch.pack(shape.B, rows, dev), _pack_rows(qp, kp, 0, ql, kl, 0),
                          _maybe("wq", wq, _f32, d, dev), _maybe("wk", wk, _f32, d, dev), eps, _maybe("inv_freq", inv_freq, _f32, rot // 2, dev), rot, first,
                          pairs, qo, qol, ko, kol, _flat("status", status, _i32, shape.B, dev), _on(stream, dev))
    if r:
        raise TsvError(r, "qk_norm_rope")


def _kv(shape: TokenShape, q: Optional[torch.Tensor], k: torch.Tensor, v: Optional[torch.Tensor], dev: int) -> bytes:
    dt, rows, Hk, d = shape.torch_dtype, _rows("k", k), shape.Hk, shape.d
    qp, qs = _vectors("q", q, dt, rows, shape.H, d, dev) if q is not None else (0, 0)
    kp, ks = _vectors("k", k, dt, rows, Hk, d, dev)
    vp, vs = _vectors("v", v, dt, rows, Hk, d, dev) if v is not None else (0, 0)
    return _pack_rows(qp, kp, vp, qs, ks, vs)


def window_sink_attn(shape: TokenShape, cache: TokenCache, batch: TokenBatch, q: torch.Tensor, k: torch.Tensor, v: Optional[torch.Tensor],
                     out: torch.Tensor, workspace: torch.Tensor, status: torch.Tensor, stream=None) -> None:
    """out [rows, H, d]: every new token's attention to the sinks and its window, committed (cache) and new (k, v) tokens."""
    dev = _device()
    (wp, wn), rows = _workspace(workspace, dev), _rows("k", k)
    r = _lib.window_sink_attn(_at(shape.c), cache.pack(shape, dev), batch.pack(shape.B, rows, dev), _kv(shape, q, k, v, dev),
                              _flat("out", out, shape.torch_dtype, rows * shape.H * shape.d, dev), wp, wn, _flat("status", status, _i32, shape.B, dev),
                              _on(stream, dev))
    if r:
        raise TsvError(r, "window_sink_attn")


def token_commit(shape: TokenShape, cache: TokenCache, batch: TokenBatch, k: torch.Tensor, v: Optional[torch.Tensor], status: torch.Tensor,
                 path: Optional[torch.Tensor] = None, count: Optional[torch.Tensor] = None, stream=None) -> None:
    """Rows of new tokens (all n[b] of a sequence, or the first count[b] nodes of path[b]) into the cache; L[b] grows by them."""
    if not cache.commits:
        raise TsvError(tsv.ERR_SHAPE, "token_commit: a verify layer's cache advances by accept_and_refresh, which keeps its compressed entries and open blocks with L")
    dev = _device()
    pp, ld = _table("path", path, shape.B, dev)
    r = _lib.token_commit(_at(shape.c), cache.pack(shape, dev), batch.pack(shape.B, _rows("k", k), dev), _kv(shape, None, k, v, dev), pp, ld, _maybe("count", count, _i32, shape.B, dev),
                          _flat("status", status, _i32, shape.B, dev), _on(stream, dev))
    if r:
        raise TsvError(r, "token_commit")
