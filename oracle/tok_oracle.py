"""fp64 CPU restatement of the token-level and page operators (test infrastructure only): plain loops over sequences, tokens and
pages, from the definitions in include/tsv.h."""
from __future__ import annotations

from typing import List, Optional, Sequence, Set, Tuple

import numpy as np


def depths_and_kin(n: int, parent: Optional[Sequence[int]]) -> Tuple[List[int], List[Set[int]]]:
    """Depth of every new token, and the set of new tokens it may see (itself and, in a tree, its ancestors)."""
    if parent is None:
        return list(range(n)), [set(range(i + 1)) for i in range(n)]
    kin: List[Set[int]] = []
    for i in range(n):
        kin.append({i} | (kin[parent[i]] if parent[i] >= 0 else set()))
    return [len(k) - 1 for k in kin], kin


def ring_row(b: int, pos: int, n_sink: int, window: int) -> int:
    return b * (n_sink + window) + (pos if pos < n_sink else n_sink + (pos - n_sink) % window)


def attend(q: np.ndarray, k_new: np.ndarray, v_new: np.ndarray, k_old: np.ndarray, v_old: np.ndarray, window: int, n_sink: int, scale: float,
           parent: Optional[Sequence[int]] = None) -> Tuple[np.ndarray, np.ndarray, np.ndarray]:
    """One sequence: q [n, H, d], *_new [n, Hk, d], *_old [L, Hk, d] by position (fp64).  Returns the output, sum_j p_j |v_j| (what a
    relative error of the weights is multiplied by), and per (token, head) the largest sum |q| |k| * scale of a score."""
    n, H, d = q.shape
    L, G = k_old.shape[0], H // max(1, k_new.shape[1])
    depth, kin = depths_and_kin(n, parent)
    out, mag, reach = np.zeros((n, H, d)), np.zeros((n, H, d)), np.zeros((n, H))
    for i in range(n):
        p = L + depth[i]
        old = [j for j in range(L) if j > p - window or j < n_sink]
        new = [j for j in sorted(kin[i]) if L + depth[j] > p - window or L + depth[j] < n_sink]
        K = np.concatenate([k_old[old], k_new[new]])
        V = np.concatenate([v_old[old], v_new[new]])
        for h in range(H):
            with np.errstate(all="ignore"):
                s = K[:, h // G] @ q[i, h] * scale
                w = np.exp(s - s.max())
                w = w / w.sum()
                out[i, h] = (w[:, None] * V[:, h // G]).sum(0)
                mag[i, h] = (w[:, None] * np.abs(V[:, h // G])).sum(0)
                reach[i, h] = (np.abs(K[:, h // G]) @ np.abs(q[i, h])).max() * scale
    return out, mag, reach


def norm_rope(x: np.ndarray, w: Optional[np.ndarray], eps: float, pos: Sequence[int], inv_freq: np.ndarray, first: int, pairs: bool):
    """x [n, heads, d] fp64 -> the result, and the magnitudes |a| + |b| of the pair each value comes from."""
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    if w is not None:
        y = y * w
    z, mag = y.copy(), np.abs(y)
    half = len(inv_freq)
    for i, p in enumerate(pos):
        for j in range(half):
            a, b = (first + 2 * j, first + 2 * j + 1) if pairs else (first + j, first + half + j)
            c, s = np.cos(p * inv_freq[j]), np.sin(p * inv_freq[j])
            z[i, :, a] = y[i, :, a] * c - y[i, :, b] * s
            z[i, :, b] = y[i, :, a] * s + y[i, :, b] * c
            mag[i, :, a] = mag[i, :, b] = np.abs(y[i, :, a]) + np.abs(y[i, :, b])
    return z, mag


# ----------------------------------------------------------------------------- pages
class Pool:
    """Page table, counts and contents as plain arrays; the operations in the order of their definition."""

    def __init__(self, table: np.ndarray, ref: np.ndarray, page_tokens: int, planes: List[np.ndarray], rows: List[np.ndarray]):
        self.table, self.ref, self.page_tokens, self.planes, self.rows = table.copy(), ref.copy(), page_tokens, [p.copy() for p in planes], [r.copy() for r in rows]

    def _take(self, k: int) -> Optional[List[int]]:
        free = [p for p in range(len(self.ref)) if self.ref[p] == 0]
        return None if len(free) < k else free[:k]

    def assign(self, slots, first, last) -> List[int]:
        st, seen = [], set()
        for s, f, l in zip(slots, first, last):
            if not 0 <= s < len(self.table) or not 0 <= f <= l <= self.table.shape[1] or s in seen:
                st.append(64)
                continue
            seen.add(s)
            want = [lp for lp in range(f, l) if self.table[s, lp] < 0]
            got = self._take(len(want))
            st.append(0 if got is not None else 128)
            for lp, p in zip(want, got or []):
                self.table[s, lp], self.ref[p] = p, 1
        return st

    def free(self, slots, first, last) -> List[int]:
        st = []
        for s, f, l in zip(slots, first, last):
            if not 0 <= s < len(self.table) or not 0 <= f <= l <= self.table.shape[1]:
                st.append(64)
                continue
            st.append(0)
            for lp in range(f, l):
                p = self.table[s, lp]
                if p >= 0:
                    self.table[s, lp] = -1
                    self.ref[p] -= 1
        return st

    def fork(self, src, dst, L) -> List[int]:
        st, P = [], self.page_tokens
        before, L = self.table.copy(), list(L)
        for i, (a, z) in enumerate(zip(src, dst)):
            ok = 0 <= a < len(before) and 0 <= z < len(before) and z not in dst[:i] and z not in src and (before[z] < 0).all()
            if not ok or not 0 <= L[a] <= before.shape[1] * P:
                st.append(64)
                continue
            fresh = [lp for lp in range(before.shape[1]) if before[a, lp] >= 0 and lp >= L[a] // P]
            got = self._take(len(fresh))
            if got is None:
                st.append(128)
                continue
            st.append(0)
            for lp in range(before.shape[1]):
                if before[a, lp] >= 0 and lp < L[a] // P:
                    self.table[z, lp] = before[a, lp]
                    self.ref[before[a, lp]] += 1
            for lp, p in zip(fresh, got):
                self.table[z, lp], self.ref[p] = p, 1
                if lp == L[a] // P and L[a] % P:
                    for plane in self.planes:
                        plane[p] = plane[before[a, lp]]
            for r in self.rows:
                r[z] = r[a]
        return st

    def compact(self) -> int:
        used = int((self.ref != 0).sum())
        holes = [p for p in range(used) if self.ref[p] == 0]
        movers = [p for p in range(used, len(self.ref)) if self.ref[p] != 0]
        for p, h in zip(movers, holes):
            for plane in self.planes:
                plane[h] = plane[p]
            self.ref[h], self.ref[p] = self.ref[p], 0
            self.table[self.table == p] = h
        return used
