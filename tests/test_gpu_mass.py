"""Attention mass and eviction by it on the GPU against the fp64 definition."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from paper_2606_01790_gb300 import starkv as sk

import paged_harness as PH

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

from test_gpu_paged_attention import built, filled, queries, random_tree, words  # noqa: E402,F401


def weighed(c, qs, seen_of, rows, counts, layer=0):
    """lse of the queries, from the definition, in place; [rows][G][tokens] of random mass on the device."""
    q = qs.q.float().cpu().numpy()
    lse = np.full(qs.lse.shape, 9.0, np.float32)
    for i, (r, n) in enumerate(zip(rows, counts)):
        k, v = c.cache(r, layer)
        if n:
            lse[i, :n] = O.attention(q[i, :n], k, v, seen_of(i, int(c.ref.len[r]), n))[1]
    qs.lse.copy_(torch.from_numpy(lse))


def make_mass(c, decay, seed=0, spare=0):
    nl, G = c.st.cfg.n_layers, c.st.cfg.n_kv_heads
    rows, cap = c.ref.table.shape[0], c.ref.table.shape[1] * c.ref.P + spare
    data = np.random.default_rng(seed).exponential(size=(nl, rows, G, cap)).astype(np.float32)
    return data, sk.Mass(torch.from_numpy(data).cuda(), decay)


def verify(c, qs, seen_of, rows, counts, before, mass, layer=0, errors=True):
    """Every row against the definition; other rows, layers and what lies behind a row's tokens untouched."""
    torch.cuda.synchronize()
    if errors:
        sk.check_device_error(c.st)
    got, want, tol = mass.data.cpu().numpy(), before.astype(np.float64), np.zeros(before.shape)
    q, lse = qs.q.float().cpu().numpy(), qs.lse.cpu().numpy()
    for i, (r, n) in enumerate(zip(rows, counts)):
        L = int(c.ref.len[r])
        if n:
            k, _ = c.cache(r, layer)
            off = []
            want[layer, r, :, :L] = O.mass(q[i, :n], k, lse[i, :n], seen_of(i, L, n), before[layer, r, :, :L], mass.decay, off)
            tol[layer, r, :, :L] = off[0]
    err = np.abs(got - want)
    assert np.all(err <= tol), (float((err - tol).max()), np.argwhere(~(err <= tol))[:5])


@pytest.mark.parametrize("P", [16, 64, 256])
@pytest.mark.parametrize("heads,kv_heads", [(28, 4), (8, 8), (12, 1), (40, 8)])
@pytest.mark.parametrize("T", [1, 5, 19, 64])
def test_mass_of_trees(P, heads, kv_heads, T):
    c = filled([T, T + 1, 63 + T, 64 + T, 200 + T, 517], P=P, heads=heads, kv_heads=kv_heads, seed=T)
    rng = np.random.default_rng(T)
    rows = [int(r) for r in rng.permutation(6)]
    counts = [T if i % 2 else int(rng.integers(0, T + 1)) for i in range(6)]
    masks = [random_tree(rng, n) for n in counts]
    qs = queries(c, 6, T, mask=words(masks, T), rows=c.ids(rows), n_tokens=c.ids(counts))
    seen = lambda i, L, n: O.seen_tree(L, n, masks[i])   # noqa: E731
    weighed(c, qs, seen, rows, counts)
    before, mass = make_mass(c, 0.75, spare=3)
    sk.tree_mass(c.st, c.pages, 0, qs, mass, c.ws)
    verify(c, qs, seen, rows, counts, before, mass)
    c.st.close()


@pytest.mark.parametrize("P", [16, 64, 128])
@pytest.mark.parametrize("n_sink,window", [(0, 1), (4, 64), (64, 100), (1, 1 << 20), (70, 37), (3, 0), (0, 0), (100000, 5), (0, 2**31 - 1)])
@pytest.mark.parametrize("T", [1, 3, 40])
def test_mass_under_windows_and_sinks(P, n_sink, window, T):
    c = filled([T, T + 7, 64 + T, 128, 391, 640], P=P, seed=window % 97)
    rng = np.random.default_rng(n_sink + T)
    rows = [int(r) for r in rng.permutation(6)]
    counts = [int(rng.integers(0, T + 1)) if i == 2 else T for i in range(6)]
    qs = queries(c, 6, T, rows=c.ids(rows), n_tokens=c.ids(counts))
    seen = lambda i, L, n: O.seen_sink(L, n, n_sink, window)   # noqa: E731
    weighed(c, qs, seen, rows, counts)
    before, mass = make_mass(c, 1.0 if T == 3 else 0.5)
    sk.sink_mass(c.st, c.pages, 0, qs, n_sink, window, mass, c.ws)
    verify(c, qs, seen, rows, counts, before, mass)
    c.st.close()


@pytest.mark.parametrize("heads,kv_heads,T", [(160, 1, 3), (256, 1, 1), (33, 3, 12), (32, 32, 5), (129, 1, 4)])
def test_mass_of_other_head_layouts(heads, kv_heads, T):
    c = filled([150, 77, 64], P=32, heads=heads, kv_heads=kv_heads, seed=heads)
    qs = queries(c, 3, T)
    seen = lambda i, L, n: O.seen_sink(L, n, 2, 100)   # noqa: E731
    weighed(c, qs, seen, [0, 1, 2], [T] * 3)
    before, mass = make_mass(c, 0.0)
    sk.sink_mass(c.st, c.pages, 0, qs, 2, 100, mass, c.ws)
    verify(c, qs, seen, [0, 1, 2], [T] * 3, before, mass)
    c.st.close()


@pytest.mark.parametrize("T,L,n_sink,window", [(700, 900, 5, 300), (333, 2100, 0, 1 << 20), (257, 257, 600, 40), (150, 4000, 130, 1000)])
def test_mass_of_chunks(T, L, n_sink, window):
    """Many query blocks: the cut pieces of a key tile are added up, the same way every time."""
    c = filled([L, T + 3, T], P=64, heads=8, kv_heads=2, seed=T)
    qs = queries(c, 3, T, scale=2.0, rows=c.ids([2, 0, 1]), n_tokens=c.ids([T, T, T // 3]))
    rows, counts = [2, 0, 1], [T, T, T // 3]
    ref = torch.zeros((3, T, 8))
    for i, (r, n) in enumerate(zip(rows, counts)):      # (normalisers by torch: the definition takes a while)
        k, _ = c.cache(r, 0)
        seen = torch.from_numpy(O.seen_sink(int(c.ref.len[r]), n, n_sink, window))
        for h in range(8):
            z = qs.q[i, :n, h].double().cpu() @ torch.from_numpy(k[h // 4]).double().T / np.sqrt(PH.D)
            ref[i, :n, h] = torch.where(seen, z, -torch.inf).logsumexp(-1).float()
    qs.lse.copy_(ref)
    before, mass = make_mass(c, 0.9)
    sk.sink_mass(c.st, c.pages, 0, qs, n_sink, window, mass, c.ws)
    verify(c, qs, lambda i, L, n: O.seen_sink(L, n, n_sink, window), rows, counts, before, mass)
    again = sk.Mass(torch.from_numpy(before).cuda(), 0.9)
    sk.sink_mass(c.st, c.pages, 0, qs, n_sink, window, again, c.ws)
    assert torch.equal(again.data, mass.data)
    c.st.close()


@pytest.mark.parametrize("page_major", [False, True])
def test_mass_reads_q_at_any_stride_and_a_mass_of_any_layout(page_major):
    n, T = 3, 5
    c = filled([90, 200, 33], P=32, layers=2, page_major=page_major)
    qs = queries(c, n, T)
    seen = lambda i, L, m: O.seen_sink(L, m, 1, 77)   # noqa: E731
    weighed(c, qs, seen, [0, 1, 2], [T] * 3, layer=1)
    qs.q = qs.q.permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3)      # heads outermost
    before, mass = make_mass(c, 0.3)
    other = sk.Mass(mass.data.permute(1, 2, 0, 3).contiguous().permute(2, 0, 1, 3), 0.3)
    sk.sink_mass(c.st, c.pages, 1, qs, 1, 77, other, c.ws)
    verify(c, qs, seen, [0, 1, 2], [T] * 3, before, other, layer=1)
    c.st.close()


def test_one_query_for_every_token_and_head():
    """Strides of 0: the same vector for all."""
    c = filled([70, 130], P=16, heads=8, kv_heads=2)
    qs = queries(c, 2, 20)
    qs.q = qs.q[:1, :1, :1].expand(2, 20, 8, PH.D)
    seen = lambda i, L, n: O.seen_sink(L, n, 0, 1 << 20)   # noqa: E731
    weighed(c, qs, seen, [0, 1], [20, 20])
    before, mass = make_mass(c, 1.0)
    sk.sink_mass(c.st, c.pages, 0, qs, 0, 1 << 20, mass, c.ws)
    verify(c, qs, seen, [0, 1], [20, 20], before, mass)
    c.st.close()


@pytest.mark.parametrize("T", [1, 6, 70])
def test_what_a_query_does_not_see_adds_nothing(T):
    """NaN and infinities in the slots behind the tokens, in keys out of every window, in queries that are none and in
    their lse; a seen NaN key has a NaN mass, and no other has."""
    lens, sinks, window = [200, 64 + T, 100], 3, 40
    c = filled(lens, P=64, heads=8, kv_heads=2)
    counts = [T, max(1, T // 2), T]
    bad = [float("nan"), float("inf"), float("-inf")]
    for r, L in enumerate(lens):
        for page, slots in ((c.ref.table[r, (L - 1) // 64], range((L - 1) % 64 + 1, 64)),):
            for s in slots:
                c.pages.k[0, int(page), :, s] = bad[s % 3]
        if L - counts[r] - window > 10:
            c.pages.k[0, int(c.ref.table[r, 0]), :, 7] = bad[r]      # behind the sinks, before every window
    c.pages.k[0, int(c.ref.table[2, (lens[2] - 1) // 64]), 1, (lens[2] - 1) % 64, 5] = float("nan")   # row 2's last token
    c.ref.k[:] = c.pages.k.view(torch.int16).cpu().numpy()
    qs = queries(c, 3, T, n_tokens=c.ids(counts))
    qs.lse.fill_(2.0)
    if counts[1] < T:
        qs.q[1, counts[1]:] = float("nan")
        qs.lse[1, counts[1]:] = float("nan")
    before, mass = make_mass(c, 0.5)
    sk.sink_mass(c.st, c.pages, 0, qs, sinks, window, mass, c.ws)
    torch.cuda.synchronize()
    sk.check_device_error(c.st)
    got = mass.data.cpu().numpy()
    nan = np.isnan(got)
    assert nan[0, 2, 1, lens[2] - 1] and nan.sum() == 1
    q, lse = qs.q.float().cpu().numpy(), qs.lse.cpu().numpy()
    for r, L in enumerate(lens):
        k, _ = c.cache(r, 0)
        k = np.where(np.isfinite(k), k, 0)
        off, n = [], counts[r]
        want = O.mass(q[r, :n], k, lse[r, :n], O.seen_sink(L, n, sinks, window), before[0, r, :, :L], 0.5, off)
        ok = ~nan[0, r, :, :L]
        assert np.all(np.abs(got[0, r, :, :L] - want)[ok] <= off[0][ok]), r
        np.testing.assert_array_equal(got[0, r, :, L:], before[0, r, :, L:])
    c.st.close()


def test_mass_where_normalisers_are_infinite():
    """lse +inf takes every weight; a query that sees nothing (lse -inf) adds nothing."""
    c = filled([50, 300], P=16, heads=8, kv_heads=2)
    qs = queries(c, 2, 3)
    qs.lse.fill_(float("inf"))
    before, mass = make_mass(c, 1.0)
    sk.sink_mass(c.st, c.pages, 0, qs, 0, 1 << 20, mass, c.ws)
    qs.lse.fill_(float("-inf"))
    sk.sink_mass(c.st, c.pages, 0, qs, 0, 0, mass, c.ws)
    torch.cuda.synchronize()
    sk.check_device_error(c.st)
    got = mass.data.cpu().numpy()
    for r, L in enumerate([50, 300]):
        np.testing.assert_array_equal(got[0, r, :, :L - 3], before[0, r, :, :L - 3])
        assert np.all(got[0, r, :, L - 3:L] == 0)
    c.st.close()


def test_sequences_that_do_not_fit_are_left_as_they_are():
    """A row out of range, counts out of range, a row shorter than its queries, a row named twice; the others go through."""
    lens = [40, 90, 3, 60, 70, 80]
    c = filled(lens, P=16, heads=8, kv_heads=2)
    rows, counts = [0, 99, 2, 3, 4, 4, 5], [5, 5, 5, 6, 2, 1, 4]
    seen = lambda i, L, n: O.seen_sink(L, n, 0, 50)   # noqa: E731
    good = [0, 6]
    qs = queries(c, 7, 5, rows=c.ids(rows), n_tokens=c.ids(counts))
    full = queries(c, 7, 5)
    part = sk.Queries(q=full.q, lse=full.lse)
    weighed(c, part, seen, [0, 0, 0, 0, 0, 0, 5], [5, 0, 0, 0, 0, 0, 4])
    qs.lse.copy_(part.lse)
    before, mass = make_mass(c, 0.5)
    sk.sink_mass(c.st, c.pages, 0, qs, 0, 50, mass, c.ws)
    torch.cuda.synchronize()
    assert sk.device_error_status(c.st) == sk.ERR_DEVICE
    some = sk.Queries(q=qs.q[good], lse=qs.lse[good])
    verify(c, some, seen, [0, 5], [5, 4], before, mass)
    c.st.close()


# ---------------------------------------------------------------- eviction

@pytest.mark.parametrize("per_head", [False, True])
@pytest.mark.parametrize("P,budget,window", [(16, 37, 8), (64, 0, 4), (32, 1, 1), (64, 300, 16), (128, 1500, 32)])
@pytest.mark.parametrize("kind", ["spread", "ties", "odd"])
def test_eviction(per_head, P, budget, window, kind):
    lens = [budget + window, budget + window + 1, budget + window + 700, 2500]
    st = PH.state(layers=2, heads=8, kv_heads=4, window=window, select_mode=int(per_head))
    need = [-(-x // P) for x in lens]
    c = PH.Pair(st, n_pages=sum(need) + 4 * (-(-(budget + window) // P)) + 2, P=P, n_rows=5, max_pages=max(need))
    c.extend([0, 1, 2, 4], lens)
    rng = np.random.default_rng(budget)
    data, mass = make_mass(c, 1.0, seed=P)
    if kind == "ties":
        data[:] = rng.integers(0, 4, data.shape)
    elif kind == "odd":
        data[:] = rng.standard_normal(data.shape)
        for x in (np.nan, np.inf, -np.inf, 0.0, -0.0, 3e38, 1e-45):
            data[rng.random(data.shape) < 0.01] = x
        if not per_head:       # (infinities of both signs in one sum: NaN, as in the definition)
            data[np.isneginf(data)] = -1.0
    mass.data.copy_(torch.from_numpy(data))
    rows, P_ = [2, 0, 4, 1], 4 if per_head else 1
    Ls = [lens[2], lens[0], lens[3], lens[1]]
    idx = [torch.full((2, P_, budget), -7, dtype=torch.int32, device="cuda") for _ in rows]
    metas = [rng.integers(0, 2**31, L).astype(np.int32) for L in Ls]
    outs = [torch.zeros((2, P_, budget + window), dtype=torch.int32, device="cuda") for _ in rows]
    seqs = [sk.Seq(L=L, budget=budget, idx=i, meta=torch.from_numpy(m).cuda(), meta_out=o)
            for L, i, m, o in zip(Ls, idx, metas, outs)]
    sk.pages_evict(st, c.pages, c.ids(rows), seqs, mass, c.ws)
    keep, want = [], data.copy()
    for r, L in zip(rows, Ls):
        past = data[:, r, :, :L - window].astype(np.float64)
        with np.errstate(invalid="ignore"):
            x = past if per_head else past.sum(1, keepdims=True)
        keep.append(np.stack([[O.heaviest(x[l, p], budget) for p in range(P_)] for l in range(2)]))
        at = np.concatenate([keep[-1], np.broadcast_to(np.arange(L - window, L), (2, P_, window))], -1)
        at = np.broadcast_to(at, (2, 4, budget + window))
        want[:, r, :, :budget + window] = np.take_along_axis(data[:, r], at, -1)
    c.ref.compact(rows, Ls, keep, window)
    c.check()
    np.testing.assert_array_equal(mass.data.cpu().numpy(), want)
    for i, k, m, o, L in zip(idx, keep, metas, outs, Ls):
        np.testing.assert_array_equal(i.cpu().numpy(), k)
        at = np.concatenate([k, np.broadcast_to(np.arange(L - window, L), (2, P_, window))], -1)
        np.testing.assert_array_equal(o.cpu().numpy(), m[at])
    st.close()


@pytest.mark.parametrize("per_head", [False, True])
def test_eviction_of_a_long_row(per_head):
    """Longer than what a block keeps of its keys."""
    L, budget, window, P = 150001, 60000, 8, 64
    st = PH.state(layers=1, heads=4, kv_heads=2, window=window, select_mode=int(per_head))
    c = PH.Pair(st, n_pages=4000, P=P, n_rows=1, max_pages=-(-L // P))
    c.extend([0], [L])
    data, mass = make_mass(c, 1.0)
    data[..., ::3] = np.round(data[..., ::3] * 4) / 4
    mass.data.copy_(torch.from_numpy(data))
    n = 2 if per_head else 1
    idx = torch.zeros((1, n, budget), dtype=torch.int32, device="cuda")
    sk.pages_evict(st, c.pages, None, [sk.Seq(L=L, budget=budget, idx=idx)], mass, c.ws)
    past = data[0, 0, :, :L - window].astype(np.float64)
    x = past if per_head else past.sum(0, keepdims=True)
    keep = np.stack([[O.heaviest(r, budget) for r in x]])
    np.testing.assert_array_equal(idx.cpu().numpy(), keep)
    c.ref.compact([0], [L], [keep], window)
    c.check()
    st.close()


def test_a_refused_eviction_changes_nothing():
    st = PH.state(layers=1, heads=8, kv_heads=2, window=4)
    c = PH.Pair(st, n_pages=7, P=16, n_rows=2, max_pages=6)
    c.extend([0, 1], [60, 40])
    data, mass = make_mass(c, 1.0)
    idx = [torch.full((1, 1, 20), -7, dtype=torch.int32, device="cuda") for _ in range(2)]
    for seqs, rows in (([sk.Seq(L=60, budget=20, idx=idx[0]), sk.Seq(L=40, budget=20, idx=idx[1])], [0, 1]),   # four pages, none free
                       ([sk.Seq(L=59, budget=20, idx=idx[0])], [0]), ([sk.Seq(L=60, budget=20, idx=idx[0])], [7])):
        sk.pages_evict(st, c.pages, c.ids(rows), seqs, mass, c.ws)
        torch.cuda.synchronize()
        assert sk.device_error_status(st) == sk.ERR_DEVICE
    c.check()
    np.testing.assert_array_equal(mass.data.cpu().numpy(), data)
    assert all(bool((i == -7).all()) for i in idx)
    # held back behind a refused call
    sk.pages_extend(st, c.pages, c.ids([0]), c.ids([100000]), c.ws)
    sk.pages_free(st, c.pages, c.ids([1]))
    sk.pages_evict(st, c.pages, c.ids([0]), [sk.Seq(L=60, budget=20, idx=idx[0])], mass, c.ws)
    torch.cuda.synchronize()
    assert sk.device_error_status(st) == sk.ERR_DEVICE
    np.testing.assert_array_equal(mass.data.cpu().numpy(), data)
    c.check()
    st.close()


def verify_on_device(c, qs, rows, counts, before, mass, seen_of):
    """``verify`` with the definition in 64 bits on the device, for calls whose oracle would take minutes: seen_of(i, L, n) is [n][L]
    there.  The same error is allowed."""
    torch.cuda.synchronize()
    sk.check_device_error(c.st)
    G, hg, P = c.st.cfg.n_kv_heads, c.st.cfg.n_heads // c.st.cfg.n_kv_heads, c.ref.P
    untouched = torch.from_numpy(before).cuda()
    for i, (r, n) in enumerate(zip(rows, counts)):
        L = int(c.ref.len[r])
        if n == 0:
            continue
        untouched[0, r, :, :L] = mass.data[0, r, :, :L]
        seen = seen_of(i, L, n)
        pages = c.pages.table[r, :-(-L // P)].long()
        for g in range(G):
            k = c.pages.k[0, pages, g].reshape(-1, PH.D)[:L].double()
            want = torch.from_numpy(before[0, r, g, :L]).cuda().double() * mass.decay
            want[L - n:] = 0
            off = 2.0**-23 * want.abs() + 1e-37
            for h in range(g * hg, (g + 1) * hg):
                q, lse = qs.q[i, :n, h].double(), qs.lse[i, :n, h].double()[:, None]
                z = q @ k.T / np.sqrt(PH.D)
                w = torch.where(seen, torch.exp(z - lse), 0.0)
                dz = 130 * 2.0**-24 * (q.abs() @ k.abs().T) / np.sqrt(PH.D) + 2.0**-22 * (z.abs() + lse.abs())
                want += w.sum(0)
                off += (w * (dz * (1 + dz) + 2.0**-21 + (n * hg + 8) * 2.0**-24)).sum(0)
            err = (mass.data[0, r, g, :L].double() - want).abs()
            assert bool((err <= off).all()), (i, g, float((err / off).max()), int((err / off).argmax()))
    assert torch.equal(untouched, mass.data)


def normalisers_on_device(c, qs, rows, counts, seen_of):
    G, hg, P = c.st.cfg.n_kv_heads, c.st.cfg.n_heads // c.st.cfg.n_kv_heads, c.ref.P
    for i, (r, n) in enumerate(zip(rows, counts)):
        L = int(c.ref.len[r])
        if n:
            seen = seen_of(i, L, n)
            pages = c.pages.table[r, :-(-L // P)].long()
            for g in range(G):
                k = c.pages.k[0, pages, g].reshape(-1, PH.D)[:L].double()
                z = torch.einsum("thd,jd->htj", qs.q[i, :n, g * hg:(g + 1) * hg].double(), k) / np.sqrt(PH.D)
                qs.lse[i, :n, g * hg:(g + 1) * hg] = torch.where(seen, z, -torch.inf).logsumexp(-1).T.float()


def sink_on_device(n_sink, window):
    def seen(i, L, n):
        j, pos = torch.arange(L, device="cuda"), torch.arange(L - n, L, device="cuda")[:, None]
        return (j <= pos) & ((j < n_sink) | (j > pos - window))
    return seen


@pytest.mark.parametrize("P,heads,kv_heads,T,n_sink,window", [
    (64, 28, 4, 1, 0, 1 << 20), (16, 28, 4, 1, 5, 700), (128, 28, 4, 18, 0, 1 << 20), (32, 28, 4, 30, 200, 900), (256, 8, 8, 3, 0, 100),
    (64, 28, 4, 90, 3, 1 << 20), (16, 32, 8, 300, 1000, 200), (64, 12, 1, 700, 0, 64)])
def test_mass_of_calls_with_many_tiles(P, heads, kv_heads, T, n_sink, window):
    """Groups of four tiles, whole and cut, that begin and end anywhere in a range: rows of one to 23 tiles, some of whose groups no
    token sees."""
    rng = np.random.default_rng(T)
    n = 120 // kv_heads
    lens = [int(x) for x in rng.integers(max(T, 100), 3000, n)]
    c = filled(lens, P=P, heads=heads, kv_heads=kv_heads, seed=T)
    rows = [int(r) for r in rng.permutation(n)]
    counts = [int(rng.integers(T // 2, T + 1)) if i else T for i in range(n)]
    qs = queries(c, n, T, rows=c.ids(rows), n_tokens=c.ids(counts), scale=1.5)
    seen = sink_on_device(n_sink, window)
    normalisers_on_device(c, qs, rows, counts, seen)
    before, mass = make_mass(c, 0.5)
    sk.sink_mass(c.st, c.pages, 0, qs, n_sink, window, mass, c.ws)
    verify_on_device(c, qs, rows, counts, before, mass, seen)
    again = sk.Mass(torch.from_numpy(before).cuda(), 0.5)
    sk.sink_mass(c.st, c.pages, 0, qs, n_sink, window, again, c.ws)
    assert torch.equal(again.data, mass.data)
    c.st.close()


@pytest.mark.parametrize("P,heads,kv_heads,T", [(64, 28, 4, 26), (16, 28, 4, 64), (128, 8, 2, 9)])
def test_mass_of_many_trees(P, heads, kv_heads, T):
    rng = np.random.default_rng(T)
    n = 30
    lens = [int(x) for x in rng.integers(T, 3000, n)]
    c = filled(lens, P=P, heads=heads, kv_heads=kv_heads, seed=T)
    rows = [int(r) for r in rng.permutation(n)]
    counts = [int(rng.integers(0, T + 1)) if i else T for i in range(n)]
    masks = [random_tree(rng, m) for m in counts]
    qs = queries(c, n, T, mask=words(masks, T), rows=c.ids(rows), n_tokens=c.ids(counts))

    def seen(i, L, m):
        out = torch.ones((m, L), dtype=torch.bool, device="cuda")
        out[:, L - m:] = torch.tensor([[x >> j & 1 for j in range(m)] for x in masks[i]], device="cuda").bool()
        return out
    normalisers_on_device(c, qs, rows, counts, seen)
    before, mass = make_mass(c, 0.9)
    sk.tree_mass(c.st, c.pages, 0, qs, mass, c.ws)
    verify_on_device(c, qs, rows, counts, before, mass, seen)
    c.st.close()


@pytest.mark.parametrize("per_head", [False, True])
def test_eviction_of_many_lengths_at_once(per_head):
    """Lengths about a block's threads and rounds, and about what it keeps of its keys, in one call."""
    past = [2, 511, 512, 513, 1024, 4095, 4096, 4097, 16384, 49151, 49152, 49153]
    P, window = 128, 4
    budgets = [1, 510, 256, 512, 1, 2047, 2048, 4096, 5000, 20000, 49151, 700]
    lens = [x + window for x in past]
    need = [-(-x // P) for x in lens]
    st = PH.state(layers=1, heads=4, kv_heads=2, window=window, select_mode=int(per_head))
    c = PH.Pair(st, n_pages=sum(need) + sum(-(-(b + window) // P) for b in budgets), P=P, n_rows=len(past), max_pages=max(need))
    c.extend(list(range(len(past))), lens)
    rng = np.random.default_rng(7)
    data, mass = make_mass(c, 1.0)
    data[:] = rng.random(data.shape)
    data[:, ::2] = np.round(data[:, ::2] * 256) / 256       # (many equal ones in every other row)
    mass.data.copy_(torch.from_numpy(data))
    n = 2 if per_head else 1
    idx = [torch.full((1, n, b), -7, dtype=torch.int32, device="cuda") for b in budgets]
    sk.pages_evict(st, c.pages, None, [sk.Seq(L=L, budget=b, idx=i) for L, b, i in zip(lens, budgets, idx)], mass, c.ws)
    keep, want = [], data.copy()
    for r, (x, b, L) in enumerate(zip(past, budgets, lens)):
        m = data[0, r, :, :x].astype(np.float64)
        keep.append(np.stack([[O.heaviest(y, b) for y in (m if per_head else m.sum(0, keepdims=True))]]))
        at = np.concatenate([keep[-1][0], np.broadcast_to(np.arange(x, L), (n, window))], -1)
        want[0, r, :, :b + window] = np.take_along_axis(data[0, r], np.broadcast_to(at, (2, b + window)), -1)
        np.testing.assert_array_equal(idx[r].cpu().numpy(), keep[-1], err_msg=str(x))
    np.testing.assert_array_equal(mass.data.cpu().numpy(), want)
    c.ref.compact(list(range(len(past))), lens, keep, window)
    c.check()
    st.close()
