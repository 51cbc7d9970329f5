"""Shared by the tests of the paged cache: a pool on the device beside its plain
definition, and the bounds that the attention is held to."""
from __future__ import annotations

import numpy as np
import torch

from oracle import paged_oracle as O
from paper_2606_01790_gb300 import starkv as sk

D = 128


def state(layers=1, heads=28, kv_heads=4, window=8, **over) -> sk.State:
    return sk.init_state(sk.Config(n_layers=layers, n_heads=heads, n_kv_heads=kv_heads, window=window, **over))


class Pair:
    """One paged cache twice: tensors on the device, and the oracle's arrays."""

    def __init__(self, st, n_pages, P, n_rows, max_pages, seed=0, page_major=False, dev="cuda"):
        self.st, self.rng = st, np.random.default_rng(seed)
        nl, G = st.cfg.n_layers, st.cfg.n_kv_heads
        shape = (nl, n_pages, G, P, D)
        kv = []
        for _ in range(2):
            x = torch.from_numpy(self.rng.standard_normal(shape, dtype=np.float32)).to(torch.bfloat16).to(dev)
            if page_major:     # every layer of a page together
                x = x.transpose(0, 1).contiguous().transpose(0, 1)
            kv.append(x)
        self.pages = sk.Pages(k=kv[0], v=kv[1], table=torch.zeros((n_rows, max_pages), dtype=torch.int32, device=dev),
                              len=torch.empty(n_rows, dtype=torch.int32, device=dev),
                              refs=torch.empty(n_pages, dtype=torch.int32, device=dev))
        sk.pages_reset(st, self.pages)
        bits = [x.view(torch.int16).cpu().numpy().copy() for x in kv]
        self.ref = O.Pool(bits[0], bits[1], np.zeros((n_rows, max_pages), np.int32), np.zeros(n_rows, np.int32),
                          np.zeros(n_pages, np.int32))
        self.ws = sk.pages_workspace(st, self.pages, min(n_rows, 1024), 64)   # (a call takes 1024 rows at most)

    def ids(self, x):
        return torch.tensor(list(x), dtype=torch.int32, device=self.pages.k.device)

    def extend(self, rows, n_new):
        sk.pages_extend(self.st, self.pages, self.ids(rows), self.ids(n_new), self.ws)
        self.ref.extend(rows, n_new)

    def fork(self, src, dst, deep=False):
        sk.pages_fork(self.st, self.pages, self.ids(src), self.ids(dst), self.ws, deep=deep)
        self.ref.fork(src, dst, deep)

    def free(self, rows):
        sk.pages_free(self.st, self.pages, self.ids(rows))
        self.ref.free(rows)

    def check(self, errors=True):
        torch.cuda.synchronize()
        if errors:
            sk.check_device_error(self.st)
        r, p = self.ref, self.pages
        np.testing.assert_array_equal(p.len.cpu().numpy(), r.len)
        np.testing.assert_array_equal(p.refs.cpu().numpy(), r.refs)
        np.testing.assert_array_equal(p.table.cpu().numpy(), r.table)
        for x, y in ((p.k, r.k), (p.v, r.v)):
            np.testing.assert_array_equal(x.view(torch.int16).cpu().numpy(), y)

    def cache(self, row, layer):
        """K and V of a row in fp32, [G][L][d]."""
        out = []
        for x in (self.ref.k, self.ref.v):
            t = self.ref.tokens(row, layer, x).copy()
            out.append(torch.from_numpy(t).view(torch.bfloat16).float().numpy())
        return out


def check_attention(o, lse, q, k, v, seen, what=""):
    """One sequence against the oracle.  o is rounded to bf16 (2^-8 of its value).  Before
    that a weight p carries the error of its logit, dz <= 130 * 2^-24 * sum_i |q_i k_i| / sqrt(d) for a
    128-term fp32 sum, the normaliser the largest of them, two bf16 parts (16 bits) and fp32 sums of L
    terms, each relative to sum_j p_j |v_j|; lse that of its logits and fp32 rounding."""
    spread = []
    ro, rl = O.attention(q, k, v, seen, spread)
    n, H, _ = q.shape
    G, L, _ = k.shape
    for t in range(n):
        if not seen[t].any():
            assert np.all(o[t] == 0) and np.all(np.isneginf(lse[t])), (what, t)
            continue
        at = np.flatnonzero(seen[t])
        for h in range(H):
            g = h * G // H
            dz = 130 * 2.0**-24 * (np.abs(k[g, at]) @ np.abs(q[t, h])).max() / np.sqrt(D) + 2.0**-22
            tol = 2.0**-8 * np.abs(ro[t, h]) + (2.0**-15 + 4 * dz + (len(at) + 16) * 2.0**-24) * spread[0][t, h] + 1e-37
            err = np.abs(o[t, h] - ro[t, h])
            assert np.all(err <= tol), (what, t, h, float((err / tol).max()))
            tol = dz + (len(at) + 16) * 2.0**-24 + 2.0**-22 * abs(rl[t, h])
            assert abs(lse[t, h] - rl[t, h]) <= tol, (what, t, h, lse[t, h], rl[t, h], tol)
