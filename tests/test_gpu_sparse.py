"""Bounds of pages and attention over chosen pages on the GPU against the fp64 definition."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from paper_2606_01790_gb300 import starkv as sk

import paged_harness as PH

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

from test_gpu_paged_attention import built, filled, queries  # noqa: E402,F401


def reference_bounds(c, before, rows, counts, layers):
    want = before.copy()
    for r, n in zip(rows, counts):
        L = int(c.ref.len[r])
        for j in range((L - n) // c.ref.P, -(-L // c.ref.P) if n else 0):
            page = c.ref.table[r, j]
            for layer in layers:
                k = torch.from_numpy(c.ref.k[layer, page][:, :min(c.ref.P, L - j * c.ref.P)].copy()).view(torch.bfloat16).float().numpy()
                want[layer, page, :, 0], want[layer, page, :, 1] = k.min(1), k.max(1)
    return want


def fresh_bounds(c, seed=0):
    b = torch.from_numpy(np.random.default_rng(seed).standard_normal((c.st.cfg.n_layers, c.ref.k.shape[1], c.st.cfg.n_kv_heads, 2, PH.D),
                                                                    dtype=np.float32)).to(torch.bfloat16).cuda()
    return b, b.float().cpu().numpy()


@pytest.mark.parametrize("P", [16, 32, 64, 256])
@pytest.mark.parametrize("T", [1, 2, 17, 300])
@pytest.mark.parametrize("page_major", [False, True])
def test_bounds(P, T, page_major):
    lens = [1, T, T + 1, 64, 300 + T, 517]
    lens = [max(n, T) for n in lens]
    c = filled(lens, P=P, heads=8, kv_heads=2, layers=3, seed=T, page_major=page_major)
    for x in (c.pages.k[0, 1], c.pages.k[2, 2]):      # signed zeros, infinities and NaN among the keys
        x[0, :2, ::7] = float("inf")
        x[1, 2:4, 1::9] = float("-inf")
        x[0, 5, 3] = float("nan")
        x[1, 1:4, 4] = -0.0
    c.ref.k[:] = c.pages.k.view(torch.int16).cpu().numpy()
    bounds, before = fresh_bounds(c)
    rng = np.random.default_rng(T)
    rows = [int(r) for r in rng.permutation(6)] + [4]
    counts = [T if i % 2 else int(rng.integers(0, T + 1)) for i in range(7)]
    sk.pages_bounds(c.st, c.pages, 1, 2, bounds, T, rows=c.ids(rows), n_tokens=c.ids(counts))
    torch.cuda.synchronize()
    sk.check_device_error(c.st)
    np.testing.assert_array_equal(bounds.float().cpu().numpy(), reference_bounds(c, before, rows, counts, [1, 2]))
    sk.pages_bounds(c.st, c.pages, 0, 3, bounds, max(lens), n_tokens=c.pages.len)     # every page of every row
    torch.cuda.synchronize()
    sk.check_device_error(c.st)
    np.testing.assert_array_equal(bounds.float().cpu().numpy(), reference_bounds(c, before, range(6), lens, [0, 1, 2]))
    c.st.close()


def test_bounds_pass_over_what_does_not_fit():
    c = filled([40, 90, 3], P=16, heads=8, kv_heads=2)
    c.pages.table[1, 5] = 1000
    bounds, before = fresh_bounds(c)
    sk.pages_bounds(c.st, c.pages, 0, 1, bounds, 5, rows=c.ids([0, 77, -1, 2, 1, 0]), n_tokens=c.ids([5, 1, 1, 4, 5, 6]))
    torch.cuda.synchronize()
    assert sk.device_error_status(c.st) == sk.ERR_DEVICE
    np.testing.assert_array_equal(bounds.float().cpu().numpy(), reference_bounds(c, before, [0], [5], [0]))
    c.st.close()


def verify(c, qs, bounds, rows, counts, first, last, n_chosen, chosen, layer=0, errors=True):
    torch.cuda.synchronize()
    if errors:
        sk.check_device_error(c.st)
    o, lse, q = qs.o.float().cpu().numpy(), qs.lse.cpu().numpy(), qs.q.float().cpu().numpy()
    got, b = chosen.cpu().numpy(), bounds.float().cpu().numpy()
    G = c.st.cfg.n_kv_heads
    hg, P = c.st.cfg.n_heads // G, c.ref.P
    for i, (r, n) in enumerate(zip(rows, counts)):
        k, v = c.cache(r, layer)
        L = int(c.ref.len[r])
        for t in range(n):
            pos = L - n + t
            pages = c.ref.table[r, :pos // P + 1]
            for g in range(G):
                h = slice(g * hg, (g + 1) * hg)
                take = O.choose_pages(O.page_scores(q[i, t, h], b[layer, pages, g, 0], b[layer, pages, g, 1]), first, last, n_chosen)
                np.testing.assert_array_equal(got[i, t, g], take + [-1] * (n_chosen - len(take)), err_msg=str((i, t, g)))
                seen = np.zeros((1, L), bool)
                for j in take:
                    seen[0, j * P:min((j + 1) * P, pos + 1)] = True
                PH.check_attention(o[i, t:t + 1, h], lse[i, t:t + 1, h], q[i, t:t + 1, h], k[g:g + 1], v[g:g + 1], seen, what=(i, t, g))
        assert np.all(o[i, n:] == 9.0) and np.all(lse[i, n:] == 9.0) and np.all(got[i, n:] == -5), i


def bounded(c):
    bounds = sk.make_bounds(c.st, c.pages)
    bounds.fill_(float("nan"))      # of pages that no row holds
    sk.pages_bounds(c.st, c.pages, 0, c.st.cfg.n_layers, bounds, int(c.ref.len.max()), n_tokens=c.pages.len)
    return bounds


@pytest.mark.parametrize("P", [16, 64, 256])
@pytest.mark.parametrize("heads,kv_heads", [(28, 4), (8, 8), (12, 1), (40, 8)])
@pytest.mark.parametrize("T", [1, 5])
@pytest.mark.parametrize("first,last,n_chosen", [(0, 1, 1), (1, 2, 5), (2, 1, 12), (0, 3, 3), (1, 1, 1000)])
def test_sparse_attention(P, heads, kv_heads, T, first, last, n_chosen):
    lens = [T, T + 1, P, P + 1, 4 * P + 3, 1200, 6 * P]
    lens = [max(x, T) for x in lens]
    c = filled(lens, P=P, heads=heads, kv_heads=kv_heads, seed=T + n_chosen)
    bounds = bounded(c)
    rng = np.random.default_rng(n_chosen)
    rows = [int(r) for r in rng.permutation(7)]
    counts = [T if i != 2 else int(rng.integers(0, T + 1)) for i in range(7)]
    qs = queries(c, 7, T, rows=c.ids(rows), n_tokens=c.ids(counts))
    chosen = torch.full((7, T, kv_heads, n_chosen), -5, dtype=torch.int32, device="cuda")
    ws = sk.sparse_workspace(c.st, c.pages, 7, T, n_chosen)
    sk.sparse_attention(c.st, c.pages, 0, qs, bounds, first, last, n_chosen, ws, chosen_out=chosen)
    verify(c, qs, bounds, rows, counts, first, last, n_chosen, chosen)
    c.st.close()


@pytest.mark.parametrize("heads,kv_heads,T", [(160, 1, 3), (256, 1, 1), (33, 3, 12), (32, 32, 2)])
def test_sparse_attention_of_other_head_layouts(heads, kv_heads, T):
    c = filled([150, 77, 640], P=32, heads=heads, kv_heads=kv_heads, layers=2, seed=heads, page_major=True)
    bounds = bounded(c)
    qs = queries(c, 3, T)
    qs.q = qs.q.permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3)
    o = torch.full((T, 3, heads, PH.D), 9.0, dtype=torch.bfloat16, device="cuda")
    qs.o = o.transpose(0, 1)
    chosen = torch.full((3, T, kv_heads, 4), -5, dtype=torch.int32, device="cuda")
    ws = sk.sparse_workspace(c.st, c.pages, 3, T, 4)
    sk.sparse_attention(c.st, c.pages, 1, qs, bounds, 1, 1, 4, ws, chosen_out=chosen)
    verify(c, qs, bounds, [0, 1, 2], [T] * 3, 1, 1, 4, chosen, layer=1)
    c.st.close()


def test_a_chunk_of_more_queries_than_a_launch_takes():
    T = 1100
    c = filled([1300, 1200], P=16, heads=8, kv_heads=2)
    bounds = bounded(c)
    qs = queries(c, 2, T)
    chosen = torch.full((2, T, 2, 9), -5, dtype=torch.int32, device="cuda")
    ws = sk.sparse_workspace(c.st, c.pages, 2, T, 9)
    sk.sparse_attention(c.st, c.pages, 0, qs, bounds, 1, 2, 9, ws, chosen_out=chosen)
    torch.cuda.synchronize()
    sk.check_device_error(c.st)
    assert torch.isfinite(qs.o).all() and torch.isfinite(qs.lse).all()
    last = torch.tensor([1300, 1200]).view(2, 1, 1) - T + torch.arange(T).view(1, T, 1)
    assert torch.equal((chosen >= 0).sum(-1).cpu(), torch.minimum(last // 16 + 1, torch.tensor(9)).expand(2, T, 2))
    some = [0, 1, 150, 1023, 1024, 1099]
    o, lse, q = qs.o.float().cpu().numpy(), qs.lse.cpu().numpy(), qs.q.float().cpu().numpy()
    b, got = bounds.float().cpu().numpy(), chosen.cpu().numpy()
    for i, L in enumerate([1300, 1200]):
        k, v = c.cache(i, 0)
        for t in some:
            pos = L - T + t
            pages = c.ref.table[i, :pos // 16 + 1]
            for g in range(2):
                h = slice(4 * g, 4 * g + 4)
                take = O.choose_pages(O.page_scores(q[i, t, h], b[0, pages, g, 0], b[0, pages, g, 1]), 1, 2, 9)
                assert got[i, t, g].tolist() == take + [-1] * (9 - len(take))
                seen = np.zeros((1, L), bool)
                for j in take:
                    seen[0, j * 16:min((j + 1) * 16, pos + 1)] = True
                PH.check_attention(o[i, t:t + 1, h], lse[i, t:t + 1, h], q[i, t:t + 1, h], k[g:g + 1], v[g:g + 1], seen)
    c.st.close()


@pytest.mark.parametrize("kind", ["zero", "equal", "close", "huge", "tiny", "mixed"])
def test_which_of_close_scores_is_taken(kind):
    """Queries of zeros, pages alike, scores that differ in their last bits only, products past or under what 32 bits
    hold, scores that all but cancel: the choice is that of 64 bits, equal ones the lowest first."""
    n_pages, P = 300, 16
    c = filled([n_pages * P], P=P, heads=8, kv_heads=2)
    rng = np.random.default_rng(len(kind))
    bounds = sk.make_bounds(c.st, c.pages)
    base = rng.standard_normal((1, 1, 2, 2, PH.D))
    b = np.broadcast_to(base, tuple(bounds.shape)).copy()
    q = rng.standard_normal((1, 1, 8, PH.D))
    if kind == "zero":
        q[:] = 0
    if kind in ("close", "huge", "tiny"):
        big = rng.integers(0, 2, b.shape) * 2.0**rng.integers(0, 7, b.shape)      # changes of one bit in a few places
        b = b + (rng.random(b.shape) < 0.02) * big * 2.0**-9
    if kind == "huge":
        b, q = b * 2.0**100, q * 2.0**27
    if kind == "tiny":
        b, q = b * 2.0**-100, q * 2.0**-30
    if kind == "mixed":
        b = rng.standard_normal(b.shape) * 2.0**rng.integers(-30, 30, b.shape)
        b[..., PH.D // 2:] = -b[..., :PH.D // 2]      # products cancel
        q[..., PH.D // 2:] = q[..., :PH.D // 2]
        b[..., 0] += rng.standard_normal(b.shape[:-1]) * 2.0**-20
    bounds.copy_(torch.from_numpy(b))
    qs = queries(c, 1, 1)
    qs.q.copy_(torch.from_numpy(q))
    chosen = torch.full((1, 1, 2, 41), -5, dtype=torch.int32, device="cuda")
    ws = sk.sparse_workspace(c.st, c.pages, 1, 1, 41)
    sk.sparse_attention(c.st, c.pages, 0, qs, bounds, 1, 1, 41, ws, chosen_out=chosen)
    torch.cuda.synchronize()
    sk.check_device_error(c.st)
    bf, qf = bounds.double().cpu().numpy(), qs.q.double().cpu().numpy()
    for g in range(2):
        x = qf[0, 0, 4 * g:4 * g + 4]
        up, down = np.maximum(x, 0).sum(0), np.minimum(x, 0).sum(0)
        pages = c.ref.table[0, :n_pages]
        # every product has at most 8 + 10 bits: in units of the least place, whole numbers of any size
        exact = []
        for p in pages:
            from fractions import Fraction
            exact.append(sum(Fraction(u) * Fraction(h) + Fraction(d) * Fraction(l)
                             for u, d, l, h in zip(up, down, bf[0, p, g, 0], bf[0, p, g, 1])))
        order = sorted(range(1, n_pages - 1), key=lambda j: (-exact[j], j))
        want = sorted([0, n_pages - 1] + order[:39])
        got = chosen[0, 0, g].tolist()
        if kind in ("zero", "equal"):
            assert got == want
        else:      # 64 bits tell scores apart that differ by more than their sums' rounding
            size = [sum(abs(Fraction(u) * Fraction(h)) + abs(Fraction(d) * Fraction(l))
                        for u, d, l, h in zip(up, down, bf[0, p, g, 0], bf[0, p, g, 1])) for p in pages]
            edge = exact[order[38]]
            for j in set(got) ^ set(want):
                assert abs(exact[j] - edge) <= 2 * size[j] * Fraction(2)**-44, (g, j)
    c.st.close()


def test_pages_whose_bounds_are_not_numbers_come_first():
    P, n_pages = 16, 40
    c = filled([n_pages * P], P=P, heads=8, kv_heads=2)
    bounds = bounded(c)
    odd = {3: float("nan"), 17: float("inf"), 30: float("nan")}
    for j, x in odd.items():
        bounds[0, int(c.ref.table[0, j]), :, 1, 9] = x
    qs = queries(c, 1, 1)
    qs.q[..., 9] = 1.0
    chosen = torch.full((1, 1, 2, 6), -5, dtype=torch.int32, device="cuda")
    ws = sk.sparse_workspace(c.st, c.pages, 1, 1, 6)
    sk.sparse_attention(c.st, c.pages, 0, qs, bounds, 1, 2, 6, ws, chosen_out=chosen)
    assert chosen.cpu().tolist() == [[[[0, 3, 17, 30, 38, 39]] * 2]]
    c.st.close()


@pytest.mark.parametrize("T", [1, 4])
def test_pages_that_are_not_chosen_do_not_reach_an_output(T):
    """NaN and infinities in the K and V of pages that were not taken and behind the last token."""
    P = 64
    c = filled([1500, 700], P=P, heads=8, kv_heads=2)
    bounds = bounded(c)
    qs = queries(c, 2, T)
    chosen = torch.full((2, T, 2, 4), -5, dtype=torch.int32, device="cuda")
    ws = sk.sparse_workspace(c.st, c.pages, 2, T, 4)
    sk.sparse_attention(c.st, c.pages, 0, qs, bounds, 1, 1, 4, ws, chosen_out=chosen)
    clean = qs.o.clone(), qs.lse.clone(), chosen.clone()
    for i, L in enumerate([1500, 700]):
        for g in range(2):
            taken = set(chosen[i, :, g].flatten().tolist())
            for j in range(-(-L // P)):
                page = int(c.ref.table[i, j])
                if j not in taken:
                    c.pages.k[0, page, g] = float("nan")
                    c.pages.v[0, page, g] = float("inf")
                elif (j + 1) * P > L:
                    c.pages.k[0, page, g, L % P:] = float("inf")
                    c.pages.v[0, page, g, L % P:] = float("nan")
    for x in (qs.o, qs.lse, chosen):
        x.fill_(0)
    sk.sparse_attention(c.st, c.pages, 0, qs, bounds, 1, 1, 4, ws, chosen_out=chosen)
    torch.cuda.synchronize()
    sk.check_device_error(c.st)
    assert all(torch.equal(a, b) for a, b in zip((qs.o, qs.lse, chosen), clean))
    c.st.close()


def test_sequences_that_do_not_fit_have_zero_outputs():
    c = filled([40, 90, 3, 60], P=16, heads=8, kv_heads=2)
    bounds = bounded(c)
    rows, counts = [0, 99, 2, 1, 3], [5, 5, 5, 6, 2]
    qs = queries(c, 5, 5, rows=c.ids(rows), n_tokens=c.ids(counts))
    chosen = torch.full((5, 5, 2, 3), -5, dtype=torch.int32, device="cuda")
    ws = sk.sparse_workspace(c.st, c.pages, 5, 5, 3)
    sk.sparse_attention(c.st, c.pages, 0, qs, bounds, 1, 1, 3, ws, chosen_out=chosen)
    torch.cuda.synchronize()
    assert sk.device_error_status(c.st) == sk.ERR_DEVICE
    for i in (1, 2):
        assert torch.all(qs.o[i] == 0) and torch.all(torch.isneginf(qs.lse[i])) and torch.all(chosen[i] == -1)
    assert torch.all(qs.o[3] == 9) and torch.all(qs.lse[3] == 9) and torch.all(chosen[3] == -5)
    good = [0, 4]
    some = sk.Queries(q=qs.q[good], o=qs.o[good], lse=qs.lse[good])
    verify(c, some, bounds, [0, 3], [5, 2], 1, 1, 3, chosen[good])
    c.st.close()


@pytest.mark.parametrize("n_pages", [255, 257, 1026, 1027, 3000, 8194, 8195, 9500])
@pytest.mark.parametrize("kind", ["spread", "equal", "steps", "odd"])
def test_the_choice_among_many_pages(n_pages, kind):
    """On either side of what a thread, a pass over bins and shared memory hold; scores apart, all equal, in a few steps, with
    infinities and NaN among them."""
    P, first, last, n_chosen = 16, 1, 1, 70
    st = PH.state(layers=1, heads=4, kv_heads=2)
    pages = sk.Pages(k=torch.zeros((1, n_pages, 2, P, PH.D), dtype=torch.bfloat16, device="cuda"),
                     v=torch.zeros((1, n_pages, 2, P, PH.D), dtype=torch.bfloat16, device="cuda"),
                     table=torch.randperm(n_pages, generator=torch.Generator().manual_seed(1)).to(torch.int32).cuda()[None],
                     len=torch.tensor([n_pages * P - 3], dtype=torch.int32, device="cuda"),
                     refs=torch.ones(n_pages, dtype=torch.int32, device="cuda"))
    rng = np.random.default_rng(n_pages)
    b = rng.standard_normal((n_pages, 2, 2, PH.D)).astype(np.float32)
    if kind == "equal":
        b[:] = b[:1]
    if kind == "steps":
        b[:] = b[:1]
        b[:, :, 1, 3] = rng.integers(0, 3, (n_pages, 2))
    if kind == "odd":
        b[rng.integers(0, n_pages, 5), 0, 1, 7] = np.nan
        b[rng.integers(0, n_pages, 5), 1, 1, 7] = np.inf
        b[rng.integers(0, n_pages, 5), 1, 0, 8] = -np.inf
    bounds = torch.from_numpy(b)[None].to(torch.bfloat16).cuda()
    q = torch.from_numpy(rng.standard_normal((1, 1, 4, PH.D)).astype(np.float32)).to(torch.bfloat16).cuda()
    q[..., 7:9] = 0.5
    q[:, :, 0, 8] = -0.5
    qs = sk.Queries(q=q, o=torch.empty_like(q))
    chosen = torch.full((1, 1, 2, n_chosen), -5, dtype=torch.int32, device="cuda")
    ws = sk.sparse_workspace(st, pages, 1, 1, n_chosen)
    sk.sparse_attention(st, pages, 0, qs, bounds, first, last, n_chosen, ws, chosen_out=chosen)
    torch.cuda.synchronize()
    sk.check_device_error(st)
    bf, order, x = bounds[0].float().cpu().numpy(), pages.table[0].cpu().numpy(), q.float().cpu().numpy()[0, 0]
    for g in range(2):
        up, down = (f(x[2 * g:2 * g + 2], 0).astype(np.float64).sum(0) for f in (np.maximum, np.minimum))
        with np.errstate(invalid="ignore"):
            score = bf[order, g, 1].astype(np.float64) @ up + bf[order, g, 0].astype(np.float64) @ down
        assert chosen[0, 0, g].tolist() == O.choose_pages(score, first, last, n_chosen), g
    st.close()
