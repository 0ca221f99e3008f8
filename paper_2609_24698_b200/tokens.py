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
from typing import Optional

import torch

from . import binding as tsv
from .binding import TsvError, _aligned, _lib, _p, _stream

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


def _check(where: str, t: Optional[torch.Tensor], dtype: torch.dtype, numel: int) -> int:
    """Pointer of a contiguous tensor of at least `numel` elements on the current device (None: 0)."""
    if t is None:
        return 0
    if t.dtype != dtype or t.numel() < numel or not t.is_contiguous():
        raise TsvError(tsv.ERR_SHAPE, f"{where}: expected a contiguous {dtype} tensor of {numel} elements, got {t.dtype} {tuple(t.shape)}")
    if not t.is_cuda or t.get_device() != torch.cuda.current_device():
        raise TsvError(tsv.ERR_SHAPE, f"{where}: the tensor is on {t.device}, not on the current CUDA device")
    return t.data_ptr()


def _vectors(where: str, t: torch.Tensor, dtype: torch.dtype, rows: int, heads: int, d: int):
    """Pointer and row stride of a [>= rows, heads, d] tensor whose heads follow each other in a row."""
    s = t.shape
    if t.dtype != dtype or len(s) != 3 or s[0] < rows or s[1] != heads or s[2] != d:
        raise TsvError(tsv.ERR_SHAPE, f"{where}: expected a {dtype} tensor [{rows}, {heads}, {d}], got {t.dtype} {tuple(s)}")
    st = t.stride()
    if (d > 1 and st[2] != 1) or (heads > 1 and st[1] != d):
        raise TsvError(tsv.ERR_SHAPE, f"{where}: the heads of a row must follow each other, strides are {st}")
    if not t.is_cuda or t.get_device() != torch.cuda.current_device():
        raise TsvError(tsv.ERR_SHAPE, f"{where}: the tensor is on {t.device}, not on the current CUDA device")
    return t.data_ptr(), (st[0] if s[0] > 1 else heads * d)


@dataclass
class TokenBatch:
    """New tokens of B sequences: packed rows, chains or (parent given) draft trees."""
    row0: torch.Tensor                        # [B] int64
    n: torch.Tensor                           # [B] int32
    parent: Optional[torch.Tensor] = None     # [rows] int32, node of the same sequence, -1 for node 0

    def struct(self, B: int, rows: int) -> CTokBatch:
        return CTokBatch(_check("row0", self.row0, torch.int64, B), _check("n", self.n, torch.int32, B),
                         _check("parent", self.parent, torch.int32, rows) or None, rows)


@dataclass
class TokenCache:
    """Committed keys (and values) of a layer, a row per token: a ring of n_sink + window rows per sequence, or pages."""
    L: torch.Tensor                           # [B] int32
    k: torch.Tensor                           # [..., Hk, d] rows
    v: Optional[torch.Tensor] = None          # None: the keys are the values
    page_table: Optional[torch.Tensor] = None  # [B, max_pages] int32
    page_tokens: int = 0

    @staticmethod
    def of_layer(cache: tsv.LayerCache) -> "TokenCache":
        """The token-level KV of a verify layer: its window ring, or its pool's third physical layer (n_sink = 0 for a ring)."""
        return TokenCache(cache.L, cache.win_kv, None, cache.page_table, cache.page_tokens)

    def struct(self, shape: TokenShape) -> CTokCache:
        dt, width = shape.torch_dtype, shape.Hk * shape.d
        rows = self.k.numel() // width
        k = _check("cache.k", self.k, dt, width)
        v = _check("cache.v", self.v, dt, rows * width)
        pt, mp = None, 0
        if self.page_table is not None:
            mp = self.page_table.shape[1]
            pt = _check("page_table", self.page_table, torch.int32, shape.B * mp)
        return CTokCache(_check("L", self.L, torch.int32, shape.B), k, v or None, rows, pt, self.page_tokens, mp)


def alloc_token_cache(shape: TokenShape, values: bool = True, device="cuda") -> TokenCache:
    """Empty rings (L = 0) for the shape's sequences."""
    z = lambda: torch.zeros(shape.B, shape.n_sink + shape.window, shape.Hk, shape.d, dtype=shape.torch_dtype, device=device)
    return TokenCache(torch.zeros(shape.B, dtype=torch.int32, device=device), z(), z() if values else None)


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
    dt, f32 = shape.torch_dtype, torch.float32
    some = q if q is not None else k
    if some is None:
        raise TsvError(tsv.ERR_NULL, "qk_norm_rope")
    rows = some.shape[0]
    b = batch.struct(shape.B, rows)
    qi = qo = ki = ko = (None, 0)
    if q is not None:
        qi, qo = _vectors("q", q, dt, rows, shape.H, shape.d), _vectors("q_out", q_out, dt, rows, shape.H, shape.d)
    if k is not None:
        ki, ko = _vectors("k", k, dt, rows, shape.Hk, shape.d), _vectors("k_out", k_out, dt, rows, shape.Hk, shape.d)
    io = CTokRows(qi[0], ki[0], None, qi[1], ki[1], 0)
    rot = 0 if inv_freq is None else 2 * inv_freq.numel()
    _raise(_lib.qk_norm_rope(_at(shape.c), _check("L", L, torch.int32, shape.B), _at(b), _at(io), _check("wq", wq, f32, shape.d),
                             _check("wk", wk, f32, shape.d), eps, _check("inv_freq", inv_freq, f32, rot // 2), rot, first, pairs, qo[0], qo[1],
                             ko[0], ko[1], _check("status", status, torch.int32, shape.B), _stream(stream)), "qk_norm_rope")


def _kv(shape: TokenShape, q: Optional[torch.Tensor], k: torch.Tensor, v: Optional[torch.Tensor]) -> CTokRows:
    dt, rows = shape.torch_dtype, k.shape[0]
    qp, qs = _vectors("q", q, dt, rows, shape.H, shape.d) if q is not None else (None, 0)
    kp, ks = _vectors("k", k, dt, rows, shape.Hk, shape.d)
    vp, vs = _vectors("v", v, dt, rows, shape.Hk, shape.d) if v is not None else (None, 0)
    return CTokRows(qp, kp, vp, qs, ks, vs)


def window_sink_attn(shape: TokenShape, cache: TokenCache, batch: TokenBatch, q: torch.Tensor, k: torch.Tensor, v: Optional[torch.Tensor],
                     out: torch.Tensor, workspace: torch.Tensor, status: torch.Tensor, stream=None) -> None:
    """out [rows, H, d]: every new token's attention to the sinks and its window, committed (cache) and new (k, v) tokens."""
    rows = k.shape[0]
    b, c, io = batch.struct(shape.B, rows), cache.struct(shape), _kv(shape, q, k, v)
    wp, wn = _aligned(workspace)
    _raise(_lib.window_sink_attn(_at(shape.c), _at(c), _at(b), _at(io), _check("out", out, shape.torch_dtype, rows * shape.H * shape.d), wp, wn,
                                 _check("status", status, torch.int32, shape.B), _stream(stream)), "window_sink_attn")


def token_commit(shape: TokenShape, cache: TokenCache, batch: TokenBatch, k: torch.Tensor, v: Optional[torch.Tensor], status: torch.Tensor,
                 path: Optional[torch.Tensor] = None, count: Optional[torch.Tensor] = None, stream=None) -> None:
    """Rows of new tokens (all n[b] of a sequence, or the first count[b] nodes of path[b]) into the cache; L[b] grows by them."""
    b, c, io = batch.struct(shape.B, k.shape[0]), cache.struct(shape), _kv(shape, None, k, v)
    ld = 0 if path is None else path.shape[1]
    _raise(_lib.token_commit(_at(shape.c), _at(c), _at(b), _at(io), _check("path", path, torch.int32, shape.B * ld) or None, ld,
                             _check("count", count, torch.int32, shape.B) or None, _check("status", status, torch.int32, shape.B), _stream(stream)),
           "token_commit")
