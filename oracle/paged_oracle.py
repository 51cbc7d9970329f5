"""Plain CPU definition of the paged cache and the attention over it (test
infrastructure): page tables, counts and copies as loops over rows and tokens,
attention in fp64.  It shares no code with the CUDA path."""
from __future__ import annotations

from dataclasses import dataclass
from typing import List, Optional, Sequence

import numpy as np


class PoolError(Exception):
    """A call that is refused as a whole: nothing has changed."""


@dataclass
class Pool:
    """k, v: [layers][pages][G][P][d] of any element type (copied, never computed with)."""

    k: np.ndarray
    v: np.ndarray
    table: np.ndarray   # [rows][max_pages]
    len: np.ndarray     # [rows]
    refs: np.ndarray    # [pages]

    @property
    def P(self) -> int:
        return self.k.shape[3]

    def pages_of(self, tokens: int) -> int:
        return -(-tokens // self.P)

    def _distinct(self, rows: Sequence[int]) -> None:
        if len(set(rows)) != len(rows) or any(r < 0 or r >= len(self.len) for r in rows):
            raise PoolError("rows")

    def _take(self, need: List[int]) -> List[List[int]]:
        """The lowest free pages for each need in turn."""
        free = [p for p in range(len(self.refs)) if self.refs[p] == 0]
        if sum(need) > len(free):
            raise PoolError("pages")
        out, at = [], 0
        for n in need:
            out.append(free[at:at + n])
            at += n
        return out

    def _copy(self, src: int, dst: int, slots: int) -> None:
        for x in (self.k, self.v):
            x[:, dst, :, :slots] = x[:, src, :, :slots]

    def extend(self, rows: Sequence[int], n_new: Sequence[int]) -> None:
        self._distinct(rows)
        need, shared = [], []
        for r, n in zip(rows, n_new):
            L = int(self.len[r])
            if n < 0 or L + n > self.table.shape[1] * self.P:
                raise PoolError("length")
            fill = L % self.P
            s = n > 0 and fill > 0 and self.refs[self.table[r, L // self.P]] > 1
            shared.append(s)
            need.append(self.pages_of(L + n) - self.pages_of(L) + int(s))
        taken = self._take(need)
        for r, n, s, new in zip(rows, n_new, shared, taken):
            L = int(self.len[r])
            at = self.pages_of(L)
            if s:
                at -= 1
                old = self.table[r, at]
                self._copy(old, new[0], L % self.P)
                self.refs[old] -= 1
            for j, p in enumerate(new):
                self.table[r, at + j] = p
                self.refs[p] = 1
            self.len[r] = L + n

    def fork(self, src: Sequence[int], dst: Sequence[int], deep: bool = False) -> None:
        self._distinct(dst)
        if any(self.len[d] != 0 for d in dst) or any(s < 0 or s >= len(self.len) for s in src):
            raise PoolError("rows")
        was = self.len.copy()
        need = [self.pages_of(int(was[s])) for s in src]
        taken = self._take(need) if deep else None
        for i, (s, d) in enumerate(zip(src, dst)):
            for j in range(need[i]):
                old = self.table[s, j]
                if deep:
                    p = taken[i][j]
                    self._copy(old, p, min(self.P, int(was[s]) - j * self.P))
                    self.table[d, j] = p
                    self.refs[p] = 1
                else:
                    self.table[d, j] = old
                    self.refs[old] += 1
            self.len[d] = was[s]

    def free(self, rows: Sequence[int]) -> None:
        self._distinct(rows)
        for r in rows:
            for j in range(self.pages_of(int(self.len[r]))):
                self.refs[self.table[r, j]] -= 1
            self.len[r] = 0

    def compact(self, rows: Sequence[int], L: Sequence[int], idx: Sequence[np.ndarray], w: int) -> None:
        """idx[i]: [layers][P or 1][B]."""
        self._distinct(rows)
        if any(self.len[r] != n for r, n in zip(rows, L)):
            raise PoolError("length")
        need = [self.pages_of(i.shape[2] + w) for i in idx]
        if any(n > self.table.shape[1] for n in need):
            raise PoolError("length")
        taken = self._take(need)
        for r, n, keep, new in zip(rows, L, idx, taken):
            old = self.table[r, :self.pages_of(n)].copy()
            for layer in range(self.k.shape[0]):
                for g in range(self.k.shape[2]):
                    at = np.concatenate([keep[layer, g if keep.shape[1] > 1 else 0], np.arange(n - w, n)])
                    for x in (self.k, self.v):
                        got = x[layer, old[at // self.P], g, at % self.P]
                        to = np.arange(len(at))
                        x[layer, np.asarray(new)[to // self.P], g, to % self.P] = got
            for p in old:
                self.refs[p] -= 1
            for j, p in enumerate(new):
                self.table[r, j] = p
                self.refs[p] = 1
            self.len[r] = keep.shape[2] + w

    def tokens(self, row: int, layer: int, x: np.ndarray) -> np.ndarray:
        """[G][len][d] of one row."""
        n = int(self.len[row])
        at = np.arange(n)
        return x[layer, self.table[row, at // self.P], :, at % self.P].swapaxes(0, 1)

    def store(self, row: int, layer: int, x: np.ndarray, new: np.ndarray) -> None:
        """new: [n][G][d] into the row's last n places."""
        n, L = len(new), int(self.len[row])
        for t in range(n):
            at = L - n + t
            x[layer, self.table[row, at // self.P], :, at % self.P] = new[t]


def seen_tree(L: int, n: int, mask: Sequence[int]) -> np.ndarray:
    """[n][L]: keys that each of the n drafted tokens of a row of L tokens sees."""
    out = np.zeros((n, L), bool)
    for t in range(n):
        for j in range(L):
            out[t, j] = j < L - n or bool(int(mask[t]) >> (j - (L - n)) & 1)
    return out


def seen_sink(L: int, n: int, n_sink: int, window: int) -> np.ndarray:
    out = np.zeros((n, L), bool)
    for t in range(n):
        i = L - n + t
        for j in range(i + 1):
            out[t, j] = j < n_sink or j > i - window
    return out


def attention(q: np.ndarray, k: np.ndarray, v: np.ndarray, seen: np.ndarray, spread: Optional[list] = None):
    """q [n][H][d], k and v [G][L][d], seen [n][L]: (o [n][H][d], lse [n][H]) in fp64.  `spread`
    takes sum_j p_j |v_j| of every output, the scale of a rounding of the weights."""
    n, H, d = q.shape
    G = k.shape[0]
    o, lse = np.zeros((n, H, d)), np.full((n, H), -np.inf)
    size = np.zeros((n, H, d))
    for t in range(n):
        at = np.flatnonzero(seen[t])
        if not len(at):
            continue
        for h in range(H):
            g = h * G // H
            z = k[g, at].astype(np.float64) @ q[t, h].astype(np.float64) / np.sqrt(d)
            top = z.max()
            e = np.exp(z - top)
            lse[t, h] = top + np.log(e.sum())
            p = e / e.sum()
            o[t, h] = p @ v[g, at].astype(np.float64)
            size[t, h] = p @ np.abs(v[g, at].astype(np.float64))
    if spread is not None:
        spread.append(size)
    return o, lse
