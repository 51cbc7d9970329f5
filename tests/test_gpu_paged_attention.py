"""Attention over the paged cache on the GPU against the fp64 definition: trees of
drafted tokens, sliding windows with sinks, and what must not reach an output."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from paper_2606_01790_gb300 import starkv as sk

import paged_harness as PH

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__
    __graft_entry__.build()


def filled(lens, P=64, heads=28, kv_heads=4, layers=1, seed=0, page_major=False, spare=3):
    """Rows of the given lengths in shuffled pages."""
    st = PH.state(layers=layers, heads=heads, kv_heads=kv_heads, window=1)
    need = [-(-n // P) for n in lens]
    c = PH.Pair(st, n_pages=sum(need) + spare, P=P, n_rows=len(lens), max_pages=max(max(need), 1) + 1, seed=seed,
                page_major=page_major)
    order = np.random.default_rng(seed + 1).permutation(sum(need) + spare)
    at = 0
    for r, (n, m) in enumerate(zip(lens, need)):
        c.ref.table[r, :m] = order[at:at + m]
        c.ref.refs[order[at:at + m]] = 1
        c.ref.len[r] = n
        at += m
    for x, y in ((c.pages.table, c.ref.table), (c.pages.len, c.ref.len), (c.pages.refs, c.ref.refs)):
        x.copy_(torch.from_numpy(y))
    return c


def queries(c, n, T, seed=0, scale=1.0, **over):
    H = c.st.cfg.n_heads
    q = torch.from_numpy(np.random.default_rng(seed).standard_normal((n, T, H, PH.D), dtype=np.float32) * scale)
    return sk.Queries(q=q.to(torch.bfloat16).cuda(), o=torch.full((n, T, H, PH.D), 9.0, dtype=torch.bfloat16, device="cuda"),
                      lse=torch.full((n, T, H), 9.0, device="cuda"), **over)


def random_tree(rng, T):
    mask = []
    for j in range(T):
        up = int(rng.integers(-1, j)) if j else -1
        mask.append((mask[up] if up >= 0 else 0) | 1 << j)
    return mask


def words(masks, T):
    out = np.zeros((len(masks), T), np.uint64)
    for i, m in enumerate(masks):
        out[i, :len(m)] = [x & (1 << 64) - 1 for x in m]
    return torch.from_numpy(out.view(np.int64)).cuda()


def verify(c, qs, seen_of, rows, counts, layer=0, errors=True):
    """Every sequence against the oracle; what lies behind its queries is untouched."""
    torch.cuda.synchronize()
    if errors:
        sk.check_device_error(c.st)
    o, lse, q = qs.o.float().cpu().numpy(), qs.lse.cpu().numpy(), qs.q.float().cpu().numpy()
    for i, (r, n) in enumerate(zip(rows, counts)):
        k, v = c.cache(r, layer)
        PH.check_attention(o[i, :n], lse[i, :n], q[i, :n], k, v, seen_of(i, int(c.ref.len[r]), n), what=f"seq {i}")
        assert np.all(o[i, n:] == 9.0) and np.all(lse[i, n:] == 9.0), i


@pytest.mark.parametrize("P", [16, 64, 256])
@pytest.mark.parametrize("heads,kv_heads", [(28, 4), (8, 8), (12, 1), (40, 8)])
@pytest.mark.parametrize("T", [1, 5, 19, 64])
def test_trees(P, heads, kv_heads, T):
    lens = [T, T + 1, 63 + T, 64 + T, 200 + T, 517]
    c = filled(lens, P=P, heads=heads, kv_heads=kv_heads, seed=T)
    rng = np.random.default_rng(T)
    rows = [int(r) for r in rng.permutation(6)]
    counts = [T if i % 2 else int(rng.integers(1, T + 1)) for i in range(6)]
    masks = [random_tree(rng, n) for n in counts]
    qs = queries(c, 6, T, mask=words(masks, T), rows=c.ids(rows), n_tokens=c.ids(counts))
    sk.tree_attention(c.st, c.pages, 0, qs, c.ws)
    verify(c, qs, lambda i, L, n: O.seen_tree(L, n, masks[i]), rows, counts)
    c.st.close()


@pytest.mark.parametrize("P", [16, 64, 128])
@pytest.mark.parametrize("n_sink,window", [(0, 1), (4, 64), (64, 100), (1, 1 << 20), (70, 37), (3, 0), (0, 0), (100000, 5), (0, 2**31 - 1)])
@pytest.mark.parametrize("T", [1, 3, 40])
def test_windows_and_sinks(P, n_sink, window, T):
    lens = [T, T + 7, 64 + T, 128, 391, 640]
    c = filled(lens, P=P, seed=window % 97)
    rng = np.random.default_rng(n_sink + T)
    rows = [int(r) for r in rng.permutation(6)]
    counts = [int(rng.integers(0, T + 1)) if i == 2 else T for i in range(6)]
    qs = queries(c, 6, T, rows=c.ids(rows), n_tokens=c.ids(counts))
    sk.sink_attention(c.st, c.pages, 0, qs, n_sink, window, c.ws)
    verify(c, qs, lambda i, L, n: O.seen_sink(L, n, n_sink, window), rows, counts)
    c.st.close()


@pytest.mark.parametrize("heads,kv_heads,T", [(160, 1, 3), (256, 1, 1), (33, 3, 12), (32, 32, 5)])
def test_other_head_layouts(heads, kv_heads, T):
    """More heads of a group than a query block has rows, odd numbers of them, one of each group."""
    c = filled([150, 77, 64], P=32, heads=heads, kv_heads=kv_heads, seed=heads)
    qs = queries(c, 3, T)
    sk.sink_attention(c.st, c.pages, 0, qs, 2, 100, c.ws)
    verify(c, qs, lambda i, L, n: O.seen_sink(L, n, 2, 100), [0, 1, 2], [T] * 3)
    c.st.close()


def test_more_query_blocks_than_a_launch_takes():
    """1024 rows of two blocks each go in two launches; sequences on both sides of the border."""
    n, T = 1024, 33
    c = filled([40 + i % 90 for i in range(n)], P=16, heads=8, kv_heads=2)
    rows = [int(r) for r in np.random.default_rng(0).permutation(n)]
    qs = queries(c, n, T, rows=c.ids(rows))
    sk.sink_attention(c.st, c.pages, 0, qs, 1, 60, c.ws)
    torch.cuda.synchronize()
    sk.check_device_error(c.st)
    pick = [0, 1, 510, 511, 512, 513, 1022, 1023]
    some = sk.Queries(q=qs.q[pick], o=qs.o[pick], lse=qs.lse[pick])
    verify(c, some, lambda i, L, m: O.seen_sink(L, m, 1, 60), [rows[i] for i in pick], [T] * len(pick))
    assert torch.isfinite(qs.o).all() and torch.isfinite(qs.lse).all()
    c.st.close()


def test_a_prompt_from_its_first_token():
    """T = L: every query sees what precedes it, the first only itself."""
    c = filled([300, 131], P=32)
    qs = queries(c, 2, 300, rows=None, n_tokens=c.ids([300, 131]))
    sk.sink_attention(c.st, c.pages, 0, qs, 2, 50, sk.pages_workspace(c.st, c.pages, 2, 300))
    verify(c, qs, lambda i, L, n: O.seen_sink(L, n, 2, 50), [0, 1], [300, 131])
    c.st.close()


def test_a_long_cache_many_pieces():
    c = filled([9001, 70, 4099], P=16)
    qs = queries(c, 3, 2)
    sk.sink_attention(c.st, c.pages, 0, qs, 4, 1 << 20, c.ws)
    verify(c, qs, lambda i, L, n: O.seen_sink(L, n, 4, 1 << 20), [0, 1, 2], [2, 2, 2])
    c.st.close()


def test_layers_strides_and_page_major_pools():
    """A query part of a fused projection, outputs head-major, layer 2 of a page-major pool."""
    c = filled([100, 333], P=16, layers=3, page_major=True)
    n, T, H = 2, 7, 28
    fused = torch.randn((T, n, H + 8, PH.D), device="cuda").to(torch.bfloat16)
    out = torch.full((H, n, T + 1, PH.D), 9.0, dtype=torch.bfloat16, device="cuda")
    qs = sk.Queries(q=fused[:, :, 4:H + 4].transpose(0, 1), o=out[:, :, :T].permute(1, 2, 0, 3),
                    lse=torch.empty((n, T, H), device="cuda"))
    sk.sink_attention(c.st, c.pages, 2, qs, 4, 90, c.ws)
    verify(c, qs, lambda i, L, m: O.seen_sink(L, m, 4, 90), [0, 1], [T, T], layer=2)
    assert torch.all(out[:, :, T] == 9.0)
    qs.lse = None      # optional
    before = qs.o.clone()
    out.zero_()
    sk.sink_attention(c.st, c.pages, 2, qs, 4, 90, c.ws)
    assert torch.equal(qs.o, before)
    c.st.close()


def test_masks_that_leave_queries_empty():
    T = 6
    c = filled([T, 80], P=16)
    masks = [[0, 1, 0, 0b1000, 0, 0b111111], [0] * T]
    qs = queries(c, 2, T, mask=words(masks, T))
    sk.tree_attention(c.st, c.pages, 0, qs, c.ws)
    verify(c, qs, lambda i, L, n: O.seen_tree(L, n, masks[i]), [0, 1], [T, T])
    assert torch.all(qs.o[0, 0] == 0) and torch.all(torch.isneginf(qs.lse[0, 0]))
    c.st.close()


@pytest.mark.parametrize("scale", [30.0, 300.0])
def test_logits_over_a_wide_range(scale):
    """Row references that move again and again, and weights that underflow."""
    c = filled([700, 450], P=64)
    qs = queries(c, 2, 3, scale=scale)
    sk.sink_attention(c.st, c.pages, 0, qs, 0, 600, c.ws)
    verify(c, qs, lambda i, L, n: O.seen_sink(L, n, 0, 600), [0, 1], [3, 3])
    c.st.close()


def test_values_of_every_magnitude():
    """Values far above and below fp16's range."""
    for scale in (1e30, 1e-30):
        c = filled([300], P=64)
        v = c.pages.v.float() * scale
        c.pages.v.copy_(v)
        c.ref.v[:] = c.pages.v.view(torch.int16).cpu().numpy()
        qs = queries(c, 1, 3)
        sk.sink_attention(c.st, c.pages, 0, qs, 0, 600, c.ws)
        verify(c, qs, lambda i, L, n: O.seen_sink(L, n, 0, 600), [0], [3])
        c.st.close()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_is_not_seen_does_not_reach_an_output(bad):
    """Slots behind the last token, free pages and tokens outside a window or a branch hold `bad`."""
    T, L = 8, 203
    c = filled([L, 90], P=64)
    mask = [[1 << j for j in range(T)], [1 << j | 1 for j in range(T)]]     # token 5 of row 0 is seen by itself only
    k0, v0 = c.cache(0, 0)
    k1, v1 = c.cache(1, 0)
    clean_k, clean_v = c.pages.k.clone(), c.pages.v.clone()
    for x in (c.pages.k, c.pages.v):
        held = torch.zeros(x.shape[1], dtype=torch.bool)
        for r, n in ((0, L), (1, 90)):
            for j in range(-(-n // 64)):
                p = int(c.ref.table[r, j])
                held[p] = True
                if j == n // 64:
                    x[0, p, :, n % 64:] = bad
        x[0, ~held.cuda()] = bad
        at = L - T + 5
        x[0, int(c.ref.table[0, at // 64]), :, at % 64] = bad
    qs = queries(c, 2, T, mask=words(mask, T))
    sk.tree_attention(c.st, c.pages, 0, qs, c.ws)
    torch.cuda.synchronize()
    sk.check_device_error(c.st)
    o, lse, q = qs.o.float().cpu().numpy(), qs.lse.cpu().numpy(), qs.q.float().cpu().numpy()
    for i, (k, v, n) in enumerate(((k0, v0, L), (k1, v1, 90))):
        seen = O.seen_tree(n, T, mask[i])
        for t in range(T):
            if i == 0 and t == 5:
                continue
            PH.check_attention(o[i, t:t + 1], lse[i, t:t + 1], q[i, t:t + 1], k, v, seen[t:t + 1], what=f"{i} {t}")
    assert not np.isfinite(o[0, 5]).any()
    # and under a window: everything before it but the sinks
    c.pages.k.copy_(clean_k)
    c.pages.v.copy_(clean_v)
    W, S = 70, 3
    for x in (c.pages.k, c.pages.v):
        for j in range(S, L - 4 - W + 1):
            x[0, int(c.ref.table[0, j // 64]), :, j % 64] = bad
    qs = queries(c, 2, 4)
    sk.sink_attention(c.st, c.pages, 0, qs, S, W, c.ws)
    verify(c, qs, lambda i, n, m: O.seen_sink(n, m, S, W), [0, 1], [4, 4])
    # a token that only the first of the queries still sees
    j = L - 4 - W + 1
    for x in (c.pages.v,):
        x[0, int(c.ref.table[0, j // 64]), :, j % 64] = bad
    sk.sink_attention(c.st, c.pages, 0, qs, S, W, c.ws)
    torch.cuda.synchronize()
    o, lse, q = qs.o.float().cpu().numpy(), qs.lse.cpu().numpy(), qs.q.float().cpu().numpy()
    assert not np.isfinite(o[0, 0]).any()
    seen = O.seen_sink(L, 4, S, W)
    for t in (1, 2, 3):
        PH.check_attention(o[0, t:t + 1], lse[0, t:t + 1], q[0, t:t + 1], k0, v0, seen[t:t + 1], what=f"window {t}")
    c.st.close()


def test_a_seen_value_that_is_not_finite_marks_its_column_only():
    T, L = 4, 150
    c = filled([L], P=64)
    at = L - T + 2
    c.pages.v[0, int(c.ref.table[0, at // 64]), 1, at % 64, 17] = float("inf")
    mask = [[0b0001, 0b0011, 0b0101, 0b1101]]
    qs = queries(c, 1, T, mask=words(mask, T))
    sk.tree_attention(c.st, c.pages, 0, qs, c.ws)
    o = qs.o.float().cpu()
    for t in range(T):
        for h in range(28):
            want_inf = t >= 2 and h // 7 == 1
            assert bool(torch.isinf(o[0, t, h, 17])) == want_inf, (t, h)
            assert torch.isfinite(torch.cat((o[0, t, h, :17], o[0, t, h, 18:]))).all(), (t, h)
    c.st.close()


def test_sequences_that_do_not_fit_are_reported_and_empty():
    c = filled([40, 90, 50], P=16)
    for rows, counts, reported in (([0, 7, 2], [3, 3, 3], 1), ([0, -1, 2], [3, 3, 3], 1), ([1, 0, 2], [3, 41, 3], 1)):
        T = max(counts)
        qs = queries(c, 3, T, rows=c.ids(rows), n_tokens=c.ids(counts))
        sk.sink_attention(c.st, c.pages, 0, qs, 2, 30, c.ws)
        torch.cuda.synchronize()
        assert sk.device_error_status(c.st) == sk.ERR_DEVICE
        n = counts[1]
        assert torch.all(qs.o[1, :n] == 0) and torch.all(torch.isneginf(qs.lse[1, :n]))
        for i in (0, 2):
            k, v = c.cache(rows[i], 0)
            PH.check_attention(qs.o[i, :3].float().cpu().numpy(), qs.lse[i, :3].cpu().numpy(), qs.q[i, :3].float().cpu().numpy(),
                               k, v, O.seen_sink(k.shape[1], 3, 2, 30), what=f"seq {i}")
    for counts in ([3, 4, 3], [3, -2, 3]):      # more queries than the call has room for, or fewer than none
        qs = queries(c, 3, 3, n_tokens=c.ids(counts))
        sk.sink_attention(c.st, c.pages, 0, qs, 2, 30, c.ws)
        torch.cuda.synchronize()
        assert sk.device_error_status(c.st) == sk.ERR_DEVICE
        assert torch.all(qs.o[1] == 9.0)
    # a page number that is not one
    c.pages.table[1, 2] = 1 << 28
    qs = queries(c, 3, 3)
    sk.sink_attention(c.st, c.pages, 0, qs, 0, 1000, c.ws)
    torch.cuda.synchronize()
    assert sk.device_error_status(c.st) == sk.ERR_DEVICE
    c.st.close()


def test_a_captured_call_replays_as_the_cache_grows():
    c = filled([60, 125], P=64, spare=8)
    qs = queries(c, 2, 1)
    rows, one = c.ids([0, 1]), c.ids([1, 1])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sk.pages_extend(c.st, c.pages, rows, one, c.ws)
        sk.sink_attention(c.st, c.pages, 0, qs, 4, 100, c.ws)
    for step in range(8):      # over the end of a page
        qs.q.copy_(torch.randn_like(qs.q))
        g.replay()
        c.ref.extend([0, 1], [1, 1])
        verify(c, qs, lambda i, L, n: O.seen_sink(L, n, 4, 100), [0, 1], [1, 1])
    c.check()
    c.st.close()


def test_the_same_bits_every_time():
    c = filled([3001, 500, 1700], P=32)
    qs = queries(c, 3, 9)
    sk.sink_attention(c.st, c.pages, 0, qs, 4, 1500, c.ws)
    first = qs.o.clone(), qs.lse.clone()
    for _ in range(5):
        c.ws.fill_(0xAB)
        sk.sink_attention(c.st, c.pages, 0, qs, 4, 1500, c.ws)
        assert torch.equal(qs.o, first[0]) and torch.equal(qs.lse, first[1])
    c.st.close()


def test_a_decoding_loop_over_a_compressed_cache():
    """The operators as they are used: prompts go into pages, are scored and selected from a contiguous copy of
    their keys, compressed where they are, branched, and each branch checks drafted tokens and keeps those it
    accepts.  The pool and every output are the oracle's."""
    w, nl = 8, 2
    st = sk.init_state(sk.Config(n_layers=nl, n_heads=28, n_kv_heads=4, window=w, grid_rows=8, grid_cols=8, max_seqs=2,
                                 n_warmup=0, n_ramp=0))
    c = PH.Pair(st, n_pages=60, P=16, n_rows=6, max_pages=20, seed=3)
    lens, B = [201, 137], 60
    c.extend([0, 1], lens)
    rng = np.random.default_rng(0)
    seqs = []
    for i, L in enumerate(lens):
        kv = torch.from_numpy(rng.standard_normal((2, 1, nl, L, 4, PH.D), dtype=np.float32)).to(torch.bfloat16).cuda()
        sk.pages_store(st, c.pages, 0, sk.Tokens(k=kv[0], v=kv[1], rows=c.ids([i])))
        for l in range(nl):
            for x, part in ((c.ref.k, kv[0]), (c.ref.v, kv[1])):
                c.ref.store(i, l, x, part[0, l].view(torch.int16).cpu().numpy())
        flat = torch.empty((1, nl, 4, L, PH.D), dtype=torch.bfloat16, device="cuda")
        sk.pages_load(st, c.pages, 0, sk.Tokens(k=flat.transpose(2, 3), rows=c.ids([i])))
        assert torch.equal(flat.transpose(2, 3), kv[0])
        q = torch.from_numpy(rng.standard_normal((nl, 28, w, PH.D), dtype=np.float32)).to(torch.bfloat16).cuda()
        meta = sk.meta_tensor(sk.pack_meta(np.arange(L) < 64, np.zeros(L), np.arange(L) // 8 % 8, np.arange(L) % 8)).cuda()
        seqs.append(sk.Seq(k=flat[0], q=q, meta=meta, L=L, budget=B, slot=i, S=torch.empty((nl, 4, L - w), device="cuda"),
                           idx=torch.empty((nl, 1, B), dtype=torch.int32, device="cuda"),
                           meta_out=torch.empty((nl, 1, B + w), dtype=torch.int32, device="cuda")))
    ws = sk.workspace(st, seqs)
    for l in range(nl):
        sk.score_layer(st, l, seqs, ws)
        sk.select(st, l, seqs, ws)
    sk.pages_compact(st, c.pages, c.ids([0, 1]), seqs, c.ws)
    c.ref.compact([0, 1], lens, [s.idx.cpu().numpy() for s in seqs], w)
    c.check()
    c.fork([0, 0, 1], [2, 4, 5])
    rows, T = [0, 2, 4, 5], 7
    for step in range(3):
        c.extend(rows, [T] * 4)
        masks = [random_tree(rng, T) for _ in rows]
        kv = torch.from_numpy(rng.standard_normal((2, 4, nl, T, 4, PH.D), dtype=np.float32)).to(torch.bfloat16).cuda()
        sk.pages_store(st, c.pages, 0, sk.Tokens(k=kv[0], v=kv[1], rows=c.ids(rows)))
        for i, r in enumerate(rows):
            for l in range(nl):
                for x, part in ((c.ref.k, kv[0]), (c.ref.v, kv[1])):
                    c.ref.store(r, l, x, part[i, l].view(torch.int16).cpu().numpy())
        for l in range(nl):
            qs = queries(c, 4, T, seed=10 * step + l, mask=words(masks, T), rows=c.ids(rows))
            sk.tree_attention(st, c.pages, l, qs, c.ws)
            verify(c, qs, lambda i, L, n: O.seen_tree(L, n, masks[i]), rows, [T] * 4, layer=l)
            qs = queries(c, 4, T, seed=10 * step + l, rows=c.ids(rows))
            sk.sink_attention(st, c.pages, l, qs, 4, 40, c.ws)
            verify(c, qs, lambda i, L, n: O.seen_sink(L, n, 4, 40), rows, [T] * 4, layer=l)
        c.check()
    c.free([0, 2, 4, 5, 1])
    c.check()
    assert int(c.pages.refs.sum()) == 0
    st.close()


def _reference(k, v, q, seen):
    """One sequence's attention in 64 bits on the GPU: k, v [G][L][d], q [n][H][d], seen [n][L]."""
    n, H, d = q.shape
    G = k.shape[0]
    z = torch.einsum("nghd,gld->nghl", q.double().view(n, G, H // G, d), k.double()) / d**0.5
    z = z.masked_fill(~seen[:, None, None], -torch.inf)
    p = z.softmax(-1)
    o, size = (torch.einsum("nghl,gld->nghd", p, x).reshape(n, H, d) for x in (v.double(), v.double().abs()))
    return o, size, torch.logsumexp(z, -1).reshape(n, H)


@pytest.mark.parametrize("heads,kv_heads,P,n,T,most", [(32, 8, 32, 64, 1, 14033), (28, 4, 64, 32, 26, 9000), (28, 4, 16, 6, 64, 20001)])
def test_ragged_batches_that_fill_the_gpu(heads, kv_heads, P, n, T, most):
    """Many ranges over long rows: loads, products and softmax of many units at once, rows whose last unit ends
    inside a page, pieces that ranges cut anywhere.  o is rounded to bf16 (2^-8 of its value), from sums that
    carry what check_attention counts (2^-15 for the weights, and logits of up to 14 here: 4 dz < 2^-13)."""
    g = torch.Generator(device="cuda").manual_seed(n)
    lens = [int(x) for x in np.random.default_rng(n).integers(most // 4, most, n)]
    lens[0] = most
    need = [-(-x // P) for x in lens]
    st = PH.state(heads=heads, kv_heads=kv_heads, window=1)
    pages = sk.make_pages(st, sum(need), P, n, max(need))
    for x in (pages.k, pages.v):
        x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
    order, at = torch.randperm(sum(need), generator=g, device="cuda").int(), 0
    for r, m in enumerate(need):
        pages.table[r, :m] = order[at:at + m]
        at += m
    pages.len.copy_(torch.tensor(lens, dtype=torch.int32))
    ws = sk.pages_workspace(st, pages, n, T)
    q = (2 * torch.randn((n, T, heads, PH.D), generator=g, device="cuda")).to(torch.bfloat16)
    o, lse = torch.empty_like(q), torch.empty((n, T, heads), device="cuda")
    mask = torch.tensor([[(1 << t + 1) - 1 if t < 63 else -1 for t in range(T)]] * n, device="cuda")
    for tree in (False, True):
        for _ in range(5):
            qs = sk.Queries(q=q, o=o, lse=lse, mask=mask)
            if tree:
                sk.tree_attention(st, pages, 0, qs, ws)
            else:
                sk.sink_attention(st, pages, 0, qs, 4, 4096, ws)
        sk.check_device_error(st)
        for r, L in enumerate(lens):
            ids = pages.table[r, :need[r]].long()
            k, v = (x[0, ids].transpose(0, 1).flatten(1, 2)[:, :L] for x in (pages.k, pages.v))
            j, i = torch.arange(L, device="cuda"), torch.arange(L - T, L, device="cuda")[:, None]
            seen = (j <= i) if tree else (j <= i) & ((j < 4) | (j > i - 4096))
            ro, size, rl = _reference(k, v, q[r], seen)
            err = (o[r].double() - ro).abs()
            tol = 2.0**-8 * ro.abs() + (2.0**-12 + L * 2.0**-24) * size
            assert bool((err <= tol).all()), (tree, r, float((err / tol).max()))
            assert float((lse[r].double() - rl).abs().max()) < 1e-4, (tree, r)
    st.close()


def test_values_that_are_not_finite_in_long_rows():
    """A NaN before the window's edge and one behind the drafted tokens of another branch, in rows of many units: the
    queries that do not see it are what they are without it, within the wait limit."""
    T = 20
    c = filled([20000, 9001], P=64, seed=4)
    clean = [c.cache(r, 0) for r in (0, 1)]
    S, W = 2, 19000
    j = 20000 - T - W + 1        # only the first query's window begins with it
    c.pages.v[0, int(c.ref.table[0, j // 64]), :, j % 64, 3] = float("nan")
    qs = queries(c, 2, T, seed=1)
    sk.sink_attention(c.st, c.pages, 0, qs, S, W, c.ws)
    torch.cuda.synchronize()
    sk.check_device_error(c.st)
    o, lse, q = qs.o.float().cpu().numpy(), qs.lse.cpu().numpy(), qs.q.float().cpu().numpy()
    assert np.isnan(o[0, 0, :, 3]).all() and np.isfinite(np.delete(o[0, 0], 3, axis=1)).all()
    for r, (k, v) in enumerate(clean):
        seen = O.seen_sink(k.shape[1], T, S, W)
        for t in (1, 7, T - 1):
            PH.check_attention(o[r, t:t + 1], lse[r, t:t + 1], q[r, t:t + 1], k, v, seen[t:t + 1], what=f"{r} {t}")
    c.st.close()


def test_a_row_twice_other_streams_and_two_graphs_on_one_workspace():
    c = filled([700, 333], P=64)
    T = 5
    masks = [random_tree(np.random.default_rng(i), T) for i in range(3)]
    rows = c.ids([0, 1, 0])
    a = queries(c, 3, T, seed=1, rows=rows, mask=words(masks, T))
    b = queries(c, 3, T, seed=2, rows=rows)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    sk.tree_attention(c.st, c.pages, 0, a, c.ws, stream=s)      # a stream given, and a current one
    with torch.cuda.stream(s):
        sk.sink_attention(c.st, c.pages, 0, b, 3, 200, c.ws)
    s.synchronize()
    tree, sink = (lambda i, L, n: O.seen_tree(L, n, masks[i])), (lambda i, L, n: O.seen_sink(L, n, 3, 200))
    verify(c, a, tree, [0, 1, 0], [T] * 3)
    verify(c, b, sink, [0, 1, 0], [T] * 3)
    graphs = []
    for call in (lambda: sk.tree_attention(c.st, c.pages, 0, a, c.ws), lambda: sk.sink_attention(c.st, c.pages, 0, b, 3, 200, c.ws)):
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        graphs.append(g)
    for step in range(6):      # in turn, on one stream
        qs, seen = ((a, tree), (b, sink))[step % 2]
        qs.q.copy_(torch.randn_like(qs.q))
        qs.o.fill_(9.0)
        graphs[step % 2].replay()
        verify(c, qs, seen, [0, 1, 0], [T] * 3)
    c.st.close()


def test_offsets_past_32_bits():
    """A row in the last pages of a pool of more than 2^32 elements gives the bits that it gives in a small one."""
    st = PH.state(heads=28, kv_heads=4, window=1)
    L, P = 500, 128
    per = 4 * P * PH.D
    big = sk.make_pages(st, (1 << 32) // per + 9, P, n_rows=1, max_pages=8)
    small = sk.make_pages(st, 5, P, n_rows=1, max_pages=8)
    big.refs[:-5] = 1
    ws, n = sk.pages_workspace(st, big, 1, 3), torch.tensor([L], dtype=torch.int32, device="cuda")
    k = torch.randn((2, 1, 1, L, 4, PH.D), device="cuda").to(torch.bfloat16)
    out = []
    for pages in (big, small):
        sk.pages_extend(st, pages, None, n, ws)
        sk.pages_store(st, pages, 0, sk.Tokens(k=k[0], v=k[1]))
        torch.manual_seed(0)
        q = torch.randn((1, 3, 28, PH.D), device="cuda").to(torch.bfloat16)
        o, lse = torch.empty_like(q), torch.empty((1, 3, 28), device="cuda")
        sk.sink_attention(st, pages, 0, sk.Queries(q=q, o=o, lse=lse), 2, 300, ws)
        out.append((o, lse))
    sk.check_device_error(st)
    assert int(big.table[0, 0]) == big.refs.numel() - 5 and int(small.table[0, 0]) == 0
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])
    st.close()


def test_rows_taken_key_by_key_run_into_no_wait_limit():
    """A value that is not finite before the first query's window in rows that are one piece each (as many rows as fill
    the GPU): the other queries' rows are taken again key by key, for longer than the wait limit, and the short rows
    that come after them in the same ranges are there too."""
    T, W, n = 18, 5900, 44
    lens = [6000 if i % 11 < 10 else 70 for i in range(n)]
    c = filled(lens, P=64, seed=2)
    clean = {r: c.cache(r, 0) for r in (0, 9, 10, 43)}
    for r in range(n):
        if lens[r] == 6000:
            j = 6000 - T - W + 1
            c.pages.v[0, int(c.ref.table[r, j // 64]), :, j % 64] = float("nan")
    sk.set_wait_limit(c.st, 2_000_000)
    qs = queries(c, n, T, seed=1)
    sk.sink_attention(c.st, c.pages, 0, qs, 2, W, c.ws)
    torch.cuda.synchronize()
    sk.check_device_error(c.st)
    o, lse, q = qs.o.float().cpu().numpy(), qs.lse.cpu().numpy(), qs.q.float().cpu().numpy()
    for r in range(n):
        assert np.isnan(o[r, 0]).all() == (lens[r] == 6000) and np.isfinite(o[r, 1:]).all(), r
    for r, (k, v) in clean.items():
        seen = O.seen_sink(k.shape[1], T, 2, W)
        for t in (1, T - 1):
            PH.check_attention(o[r, t:t + 1], lse[r, t:t + 1], q[r, t:t + 1], k, v, seen[t:t + 1], what=f"{r} {t}")
    c.st.close()


def same_where_not_finite(o, lse, q, k, v, clean, seen, what):
    """The NaNs and infinities of the definition, and elsewhere what the clean values give (an infinite V of a key does
    nothing to its other columns, nor to lse)."""
    with np.errstate(invalid="ignore", over="ignore"):
        want, _ = O.attention(q, k, v, seen)
    for kind in (np.isnan, np.isposinf, np.isneginf):
        np.testing.assert_array_equal(kind(o), kind(want), err_msg=f"{what} {kind.__name__}")
    rest, _ = O.attention(q, k, clean, seen)
    PH.check_attention(np.where(np.isfinite(want), o, rest), lse, q, k, clean, seen, what=what)


@pytest.mark.parametrize("scale", [1.0, 40.0])
@pytest.mark.parametrize("n,L,T,window", [(1, 1500, 1, 1 << 20), (1, 1500, 6, 900), (45, 700, 3, 1 << 20), (45, 700, 2, 300), (1, 9000, 19, 1 << 20)])
def test_seen_values_of_infinity(n, L, T, window, scale):
    """A V of infinity gives infinity in its column to every query that sees it, however its row is cut into pieces and
    whether every query sees all of a piece or not: at a row's largest weight (exactly 1, one part of it 0), at
    weights that are 0 in fp32 (logits of some hundreds), and NaN where both infinities meet."""
    c = filled([L] * n, P=64, seed=L)
    qs = queries(c, n, T, seed=3, scale=scale)
    pick = [0, n - 1] if n > 1 else [0]
    q = qs.q.float().cpu().numpy()
    clean = {r: c.cache(r, 0) for r in pick}
    for r in pick:
        k = clean[r][0]
        put = []
        for h, col, x in ((0, 17, np.inf), (8, 64, -np.inf), (27, 127, np.inf), (20, 3, np.nan)):
            z = k[h // 7] @ q[r, T - 1, h]
            z[:max(0, L - T - window + 1)] = -np.inf       # of the keys that every query sees
            put.append((int(z.argmax()), h // 7, col, x))
        put += [(L - T - 5, 0, 90, np.inf), (L - T - 70, 0, 90, -np.inf), (L - T - 100, 1, 40, -np.inf), (L - 1, 2, 0, np.inf)]
        for j, g, col, x in put:
            c.pages.v[0, int(c.ref.table[r, j // 64]), g, j % 64, col] = float(x)
    c.ref.v = c.pages.v.view(torch.int16).cpu().numpy()
    sk.sink_attention(c.st, c.pages, 0, qs, 0, window, c.ws)
    torch.cuda.synchronize()
    sk.check_device_error(c.st)
    o, lse = qs.o.float().cpu().numpy(), qs.lse.cpu().numpy()
    for r in pick:
        k, v = c.cache(r, 0)
        at = range(T) if T < 7 else (0, T - 1)
        for t in at:
            same_where_not_finite(o[r, t:t + 1], lse[r, t:t + 1], q[r, t:t + 1], k, v, clean[r][1], O.seen_sink(L, T, 0, window)[t:t + 1], f"{r} {t}")
    c.st.close()


@pytest.mark.parametrize("n,L,T,window", [(1, 1500, 1, 1 << 20), (1, 1500, 6, 900), (45, 700, 3, 1 << 20), (45, 700, 2, 300), (1, 9000, 19, 1 << 20)])
def test_logits_of_infinity(n, L, T, window):
    """K with an infinite element gives logits of +inf to some heads and -inf to the others: lse is +inf and o NaN
    where a logit is +inf, unless one is NaN (lse NaN); a logit of -inf is a weight of 0."""
    c = filled([L] * n, P=64, seed=L)
    qs = queries(c, n, T, seed=4)
    pick = [0, n - 1] if n > 1 else [0]
    for r, at in zip(pick, ((L - T - 5, L - T - 150, L - 1), (L - T - 290,))):
        for i, j in enumerate(at):
            c.pages.k[0, int(c.ref.table[r, j // 64]), i % 4, j % 64, 7 + i] = float("inf")
    j = L - T - 100
    c.pages.k[0, int(c.ref.table[pick[-1], j // 64]), :2, j % 64, 99] = float("nan")
    c.ref.k = c.pages.k.view(torch.int16).cpu().numpy()
    sk.sink_attention(c.st, c.pages, 0, qs, 0, window, c.ws)
    torch.cuda.synchronize()
    sk.check_device_error(c.st)
    o, lse, q = qs.o.float().cpu().numpy(), qs.lse.cpu().numpy(), qs.q.float().cpu().numpy()
    met = set()
    for r in pick:
        k, v = c.cache(r, 0)
        seen = O.seen_sink(L, T, 0, window)
        for t in range(T) if T < 7 else (0, T - 1):
            for h in range(28):
                z = k[h // 7, seen[t]] @ q[r, t, h]
                if np.isnan(z).any() or np.isposinf(z).any():
                    met.add("nan" if np.isnan(z).any() else "inf")
                    assert np.isnan(o[r, t, h]).all() and (np.isnan(lse[r, t, h]) if np.isnan(z).any() else np.isposinf(lse[r, t, h])), (r, t, h)
                    continue
                met.add("-inf" if np.isneginf(z).any() else "finite")
                see = seen[t:t + 1].copy()
                see[0, np.flatnonzero(seen[t])[np.isneginf(z)]] = False
                kk = np.where(np.isfinite(k), k, 0)
                g = slice(h // 7, h // 7 + 1)
                PH.check_attention(o[r, t:t + 1, h:h + 1], lse[r, t:t + 1, h:h + 1], q[r, t:t + 1, h:h + 1], kk[g], v[g], see, what=f"{r} {t} {h}")
    assert {"inf", "nan", "-inf", "finite"} <= met
    c.st.close()


@pytest.mark.parametrize("n,L,T", [(1, 1500, 1), (1, 1500, 9), (45, 300, 3)])
def test_logits_that_are_all_minus_infinity(n, L, T):
    """o is 0 / 0 and lse -inf where a query sees keys and every logit is -inf; o is 0 where it sees none."""
    c = filled([L] * n, P=64, seed=L)
    qs = queries(c, n, T, seed=5)
    c.pages.k[0, :, 2, :, 31] = float("-inf")
    q = qs.q.float().cpu().numpy()
    for n_sink, window in ((0, 1 << 20), (3, 150), (0, 0)):
        sk.sink_attention(c.st, c.pages, 0, qs, n_sink, window, c.ws)
        torch.cuda.synchronize()
        sk.check_device_error(c.st)
        o, lse = qs.o.float().cpu().numpy(), qs.lse.cpu().numpy()
        for r in range(n):
            for t in range(T):
                for h in range(14, 21):
                    if window and q[r, t, h, 31] > 0:
                        assert np.isnan(o[r, t, h]).all() and np.isneginf(lse[r, t, h]), (r, t, h)
                    elif window:
                        assert np.isnan(o[r, t, h]).all() and np.isposinf(lse[r, t, h]), (r, t, h)
                if not window:
                    assert np.all(o[r, t] == 0) and np.all(np.isneginf(lse[r, t]))
                else:
                    assert np.isfinite(o[r, t, :14]).all() and np.isfinite(o[r, t, 21:]).all()
    c.st.close()


@pytest.mark.parametrize("heads,T", [(160, 64), (128, 63), (256, 64)])
def test_trees_of_many_query_blocks(heads, T):
    """80 blocks of a sequence (no gang's worth of CTAs is left over by a second one), 63 (two gangs) and 128."""
    c = filled([T + 90, T, 300], P=32, heads=heads, kv_heads=1, seed=heads)
    rng = np.random.default_rng(T)
    masks = [random_tree(rng, T) for _ in range(3)]
    qs = queries(c, 3, T, mask=words(masks, T))
    sk.tree_attention(c.st, c.pages, 0, qs, c.ws)
    torch.cuda.synchronize()
    sk.check_device_error(c.st)
    o, lse, q = qs.o.float().cpu().numpy(), qs.lse.cpu().numpy(), qs.q.float().cpu().numpy()
    for i, L in enumerate((T + 90, T, 300)):
        k, v = c.cache(i, 0)
        seen = O.seen_tree(L, T, masks[i])
        for t in sorted({0, 1, T // 2, T - 1}):
            PH.check_attention(o[i, t:t + 1], lse[i, t:t + 1], q[i, t:t + 1], k, v, seen[t:t + 1], what=f"{i} {t}")
    assert np.isfinite(o).all() and np.isfinite(lse).all()
    c.st.close()


def test_queries_of_infinity():
    """Logits of both infinities from a query with an infinite element: lse +inf and o NaN; the other heads' are their own."""
    c = filled([700, 75], P=64)
    qs = queries(c, 2, 2, seed=6)
    qs.q[:, 0, 3, 5], qs.q[:, 1, 20, 90] = float("inf"), float("-inf")
    sk.sink_attention(c.st, c.pages, 0, qs, 0, 500, c.ws)
    torch.cuda.synchronize()
    sk.check_device_error(c.st)
    o, lse, q = qs.o.float().cpu().numpy(), qs.lse.cpu().numpy(), qs.q.float().cpu().numpy()
    for r in range(2):
        k, v = c.cache(r, 0)
        seen = O.seen_sink(k.shape[1], 2, 0, 500)
        for t in range(2):
            for h in range(28):
                if (t, h) in ((0, 3), (1, 20)):
                    assert np.isnan(o[r, t, h]).all() and np.isposinf(lse[r, t, h]), (r, t, h)
                else:
                    PH.check_attention(o[r, t:t + 1, h:h + 1], lse[r, t:t + 1, h:h + 1], q[r, t:t + 1, h:h + 1], k[h // 7:h // 7 + 1],
                                       v[h // 7:h // 7 + 1], seen[t:t + 1], what=f"{r} {t} {h}")
    c.st.close()
