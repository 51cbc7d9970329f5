"""The paged cache on the GPU against its plain definition: tables, lengths, page
counts and every bit of the pool after each call; what is refused changes nothing."""
import numpy as np
import pytest
import torch

from paper_2606_01790_gb300 import starkv as sk

import paged_harness as PH

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__
    __graft_entry__.build()


def _error(st):
    torch.cuda.synchronize()
    return sk.device_error_status(st)


@pytest.mark.parametrize("P,page_major,layers,G", [(16, False, 1, 4), (64, True, 3, 4), (32, False, 2, 8), (128, False, 1, 1),
                                                   (256, True, 2, 2)])
def test_random_calls_match_the_definition(P, page_major, layers, G):
    st = PH.state(layers=layers, heads=8, kv_heads=G)
    c = PH.Pair(st, n_pages=70, P=P, n_rows=12, max_pages=9, seed=P, page_major=page_major)
    rng = np.random.default_rng(P + 1)
    for step in range(25):
        used = [r for r in range(12) if c.ref.len[r]]
        empty = [r for r in range(12) if not c.ref.len[r]]
        op = rng.integers(0, 4)
        if op == 0 or not used:
            rows = [int(r) for r in rng.permutation(12)[:rng.integers(1, 5)]]
            c.extend(rows, [int(min(rng.integers(0, 2 * P), 9 * P - c.ref.len[r])) for r in rows])
        elif op == 1 and empty:
            dst = [int(r) for r in rng.permutation(empty)[:rng.integers(1, 4)]]
            c.fork([int(rng.choice(used)) for _ in dst], dst)
        elif op == 2 and empty:
            c.fork([int(rng.choice(used))], [empty[0]], deep=True)
        elif op == 3 and len(used) > 3:
            c.free([int(r) for r in rng.permutation(used)[:2]])
        c.check()
    st.close()


@pytest.mark.parametrize("n", [1, 300, 1024])
def test_many_rows_in_one_call(n):
    st = PH.state(heads=4, kv_heads=1)
    c = PH.Pair(st, n_pages=3 * n + 5, P=16, n_rows=2 * n, max_pages=3)
    rows = [int(r) for r in np.random.default_rng(1).permutation(2 * n)[:n]]
    c.extend(rows, [7 + i % 33 for i in range(n)])
    c.check()
    others = [r for r in range(2 * n) if r not in set(rows)]
    c.fork(rows, others)
    c.extend(others, [i % 5 for i in range(n)])      # many copies of shared last pages; rows that need nothing
    c.check()
    c.free(rows[::2])
    c.check()
    st.close()


def test_a_large_pool_hands_out_its_lowest_free_pages():
    st = PH.state(heads=1, kv_heads=1)
    n_pages = 300_000
    pages = sk.make_pages(st, n_pages, 16, n_rows=3, max_pages=150_000)
    ws = sk.pages_workspace(st, pages, 3)
    ids = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    g = torch.Generator().manual_seed(3)
    taken = torch.rand(n_pages, generator=g) < 0.5
    pages.refs.copy_(taken.int())
    free = torch.nonzero(~taken)[:, 0].int()
    sk.pages_extend(st, pages, ids(0, 2), ids(16 * 100_000 - 3, 16 * 20_000), ws)
    torch.cuda.synchronize()
    sk.check_device_error(st)
    assert torch.equal(pages.table[0, :100_000].cpu(), free[:100_000])
    assert torch.equal(pages.table[2, :20_000].cpu(), free[100_000:120_000])
    assert pages.len.tolist() == [16 * 100_000 - 3, 0, 16 * 20_000]
    assert int(pages.refs.sum()) == int(taken.sum()) + 120_000 and int(pages.refs.max()) == 1
    sk.pages_free(st, pages, ids(2, 0))
    torch.cuda.synchronize()
    assert torch.equal(pages.refs.cpu(), taken.int())
    st.close()


def _compact(c, rows, budgets, w, seed=0, meta=True):
    rng = np.random.default_rng(seed)
    nl, G = c.st.cfg.n_layers, c.st.cfg.n_kv_heads
    sets = sk.sel_rows(c.st.cfg)
    seqs, idx, metas = [], [], []
    for i, (r, B) in enumerate(zip(rows, budgets)):
        L = int(c.ref.len[r])
        keep = np.stack([[np.sort(rng.permutation(L - w)[:B]) for _ in range(sets)] for _ in range(nl)]).astype(np.int32)
        idx.append(keep.reshape(nl, sets, B))
        m = rng.integers(-2**31, 2**31, (nl, sets, L)).astype(np.int32)
        metas.append(m)
        seqs.append(sk.Seq(L=L, budget=B, slot=i, idx=torch.from_numpy(idx[-1]).cuda() if B else None,
                           meta=torch.from_numpy(m).cuda() if meta else None, meta_layer_stride=sets * L,
                           meta_group_stride=L if sets > 1 else 0,
                           meta_out=torch.full((nl, sets, B + w), 7, dtype=torch.int32, device="cuda")))
    lens = [s.L for s in seqs]
    sk.pages_compact(c.st, c.pages, c.ids(rows), seqs, c.ws)
    c.ref.compact(rows, lens, idx, w)
    c.check()
    for s, keep, m in zip(seqs, idx, metas):
        at = np.concatenate([keep, np.broadcast_to(np.arange(s.L - w, s.L), (nl, sets, w))], -1)
        want = np.take_along_axis(m, at, -1) if meta else np.full(at.shape, 7)
        np.testing.assert_array_equal(s.meta_out.cpu().numpy(), want)


@pytest.mark.parametrize("per_head", [False, True])
@pytest.mark.parametrize("P", [16, 64, 128])
def test_compaction_of_rows_that_share_pages(P, per_head):
    w = 8
    st = PH.state(layers=2, window=w, max_seqs=4, select_mode=int(per_head))
    c = PH.Pair(st, n_pages=1600 // P + 40, P=P, n_rows=6, max_pages=700 // P + 2, seed=9, page_major=True)
    c.extend([0, 3, 5], [333, w, 577])
    c.fork([0, 5], [1, 2])
    c.check()
    _compact(c, [1, 5, 3], [100, 0, 0], w)       # a branch, only the window, a row that is its window
    _compact(c, [0], [333 - w], w, seed=2)       # everything kept
    _compact(c, [2], [64], w, seed=3, meta=False)
    st.close()


def test_compaction_of_more_than_one_batch():
    w, n = 8, 37
    st = PH.state(heads=4, kv_heads=2, window=w, max_seqs=n)
    c = PH.Pair(st, n_pages=400, P=16, n_rows=n, max_pages=8)
    c.extend(range(n), [20 + 2 * i for i in range(n)])
    rows = [int(r) for r in np.random.default_rng(5).permutation(n)]
    _compact(c, rows, [(int(c.ref.len[r]) - w) // 2 for r in rows], w)
    st.close()


def test_compaction_reports_an_index_outside_the_past_tokens():
    st = PH.state(heads=4, kv_heads=1, window=8)
    c = PH.Pair(st, n_pages=20, P=16, n_rows=1, max_pages=8)
    c.extend([0], [40])
    idx = torch.tensor([[0, 5, 32]], dtype=torch.int32, device="cuda")     # 32 is a window token
    sk.pages_compact(st, c.pages, None, [sk.Seq(L=40, budget=3, idx=idx)], c.ws)
    assert _error(st) == sk.ERR_DEVICE
    assert c.pages.len.tolist() == [11]
    st.close()


@pytest.mark.parametrize("P,T,page_major", [(16, 1, False), (64, 1, True), (16, 45, True), (128, 200, False)])
def test_store_and_load(P, T, page_major):
    st = PH.state(layers=3)
    c = PH.Pair(st, n_pages=900 // P + 12, P=P, n_rows=4, max_pages=300 // P + 2, page_major=page_major)
    c.extend([2, 0, 3], [T + 13, 250, T])
    rows, counts = [0, 3, 2], [T, max(0, T - 1), T]
    rng = np.random.default_rng(4)
    G, n = 4, 3
    # (k, v) of one fused projection: strided, token-major, a query part between
    fused = torch.from_numpy(rng.standard_normal((n, 2, T, 3, G, PH.D), dtype=np.float32)).to(torch.bfloat16).cuda()
    tok = sk.Tokens(k=fused[:, :, :, 0], v=fused[:, :, :, 2], rows=c.ids(rows), n_tokens=c.ids(counts))
    sk.pages_store(st, c.pages, 1, tok)
    bits = fused.view(torch.int16).cpu().numpy()
    for i, (r, m) in enumerate(zip(rows, counts)):
        L = int(c.ref.len[r])
        for l in range(2):
            for x, part in ((c.ref.k, 0), (c.ref.v, 2)):
                for t in range(m):     # the first m of the T are the row's last m tokens
                    at = L - m + t
                    x[1 + l, c.ref.table[r, at // P], :, at % P] = bits[i, l, t, part]
    c.check()
    # head-major, and keys only
    back = torch.full((n, 1, G, T + 2, PH.D), 3.0, dtype=torch.bfloat16, device="cuda")
    got = back[:, :, :, :T].transpose(2, 3)
    sk.pages_load(st, c.pages, 2, sk.Tokens(k=got, rows=c.ids(rows), n_tokens=c.ids(counts)))
    c.check()
    for i, m in enumerate(counts):
        assert torch.equal(got[i, 0, :m].cpu(), fused[i, 1, :m, 0].cpu())
        assert torch.all(back[i, :, :, m:] == 3.0)
    st.close()


def test_a_shared_page_is_not_written_to():
    st = PH.state(heads=4, kv_heads=2)
    c = PH.Pair(st, n_pages=12, P=16, n_rows=3, max_pages=4)
    c.extend([0], [20])
    c.fork([0], [1])
    k = torch.zeros((1, 1, 6, 2, PH.D), dtype=torch.bfloat16, device="cuda")
    sk.pages_store(st, c.pages, 0, sk.Tokens(k=k, v=k, rows=c.ids([1])))
    assert _error(st) == sk.ERR_DEVICE
    c.check()
    c.extend([1], [6])       # now the last page is its own, and holds the 6 tokens
    sk.pages_store(st, c.pages, 0, sk.Tokens(k=k, v=k, rows=c.ids([1])))
    for x in (c.ref.k, c.ref.v):
        c.ref.store(1, 0, x, np.zeros((6, 2, PH.D), np.int16))
    c.check()
    st.close()


REFUSED = {
    "no room in the pool": lambda c: sk.pages_extend(c.st, c.pages, c.ids([2, 3]), c.ids([64, 33]), c.ws),
    "no room in the table": lambda c: sk.pages_extend(c.st, c.pages, c.ids([2, 0]), c.ids([1, 60]), c.ws),
    "a row twice": lambda c: sk.pages_extend(c.st, c.pages, c.ids([2, 2]), c.ids([1, 1]), c.ws),
    "a row out of range": lambda c: sk.pages_extend(c.st, c.pages, c.ids([2, 4]), c.ids([1, 1]), c.ws),
    "a negative row": lambda c: sk.pages_free(c.st, c.pages, c.ids([-1, 0])),
    "fewer than no tokens": lambda c: sk.pages_extend(c.st, c.pages, c.ids([0]), c.ids([-1]), c.ws),
    "a branch into a full row": lambda c: sk.pages_fork(c.st, c.pages, c.ids([0, 0]), c.ids([2, 1]), c.ws),
    "two branches into one row": lambda c: sk.pages_fork(c.st, c.pages, c.ids([0, 1]), c.ids([2, 2]), c.ws),
    "a branch from nowhere": lambda c: sk.pages_fork(c.st, c.pages, c.ids([9]), c.ids([2]), c.ws),
    "no room for a deep copy": lambda c: sk.pages_fork(c.st, c.pages, c.ids([0, 0]), c.ids([2, 3]), c.ws, deep=True),
    "a row freed twice": lambda c: sk.pages_free(c.st, c.pages, c.ids([0, 1, 0])),
    "another length": lambda c: sk.pages_compact(c.st, c.pages, c.ids([0]), [sk.Seq(L=39, budget=0)], c.ws),
    "no room to compact": lambda c: sk.pages_compact(
        c.st, c.pages, c.ids([0, 1]), [sk.Seq(L=40, budget=32, slot=0, idx=torch.arange(32, dtype=torch.int32, device="cuda")),
                                       sk.Seq(L=50, budget=42, slot=1, idx=torch.arange(42, dtype=torch.int32, device="cuda"))],
        c.ws),
}


@pytest.mark.parametrize("what", sorted(REFUSED))
def test_refused_calls_change_nothing(what):
    st = PH.state(heads=4, kv_heads=1, window=8, max_seqs=2)
    c = PH.Pair(st, n_pages=13, P=16, n_rows=4, max_pages=6)
    c.extend([0, 1], [40, 50])       # 7 of 13 pages
    if what in ("no room to compact", "no room for a deep copy"):
        c.extend([3], [16])
        c.free([3]) if what == "no room for a deep copy" else None
        c.ref.refs[12] = 1           # and one page that somebody else holds
        c.pages.refs[12] = 1
    c.check()
    REFUSED[what](c)
    assert _error(st) == sk.ERR_DEVICE
    c.check()
    st.close()


def test_a_wrong_page_number_is_reported_and_not_followed():
    st = PH.state(heads=4, kv_heads=1, window=8)
    c = PH.Pair(st, n_pages=13, P=16, n_rows=2, max_pages=6)
    c.extend([0], [40])
    for bad in (-1, 13, 1 << 30):
        c.pages.table[0, 2] = bad
        k = torch.zeros((1, 1, 40, 1, PH.D), dtype=torch.bfloat16, device="cuda")
        sk.pages_load(st, c.pages, 0, sk.Tokens(k=k, rows=c.ids([0])))
        assert _error(st) == sk.ERR_DEVICE
        sk.pages_store(st, c.pages, 0, sk.Tokens(k=k[:, :, :3], rows=c.ids([0])))
        assert _error(st) == sk.ERR_DEVICE
        sk.pages_extend(st, c.pages, c.ids([0]), c.ids([3]), c.ws)      # would look at that page's count
        assert _error(st) == sk.ERR_DEVICE
        c.pages.table[0, 2] = c.ref.table[0, 2].item()
        c.check()
    for bad in (-5, 97, 1 << 30):     # lengths that the table cannot hold
        c.pages.len[0] = bad
        sk.pages_free(st, c.pages, c.ids([0]))
        assert _error(st) == sk.ERR_DEVICE
        c.pages.len[0] = 40
        c.check()
    st.close()


def test_captured_calls_replay_with_what_the_arrays_hold():
    """extend and store, captured once, append a token per replay, page after page."""
    st = PH.state(layers=2, heads=4, kv_heads=2)
    c = PH.Pair(st, n_pages=40, P=16, n_rows=3, max_pages=8)
    c.extend([0, 1], [14, 30])
    c.fork([1], [2])
    rows, one = c.ids([0, 1, 2]), c.ids([1, 1, 1])
    k = torch.zeros((3, 2, 1, 2, PH.D), dtype=torch.bfloat16, device="cuda")
    tok = sk.Tokens(k=k, v=k, rows=rows)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sk.pages_extend(st, c.pages, rows, one, c.ws)
        sk.pages_store(st, c.pages, 0, tok)
    for step in range(20):
        k.fill_(float(step + 1))
        g.replay()
        word = torch.tensor(float(step + 1), dtype=torch.bfloat16).view(torch.int16).item()
        c.ref.extend([0, 1, 2], [1, 1, 1])
        for r in range(3):
            for l in range(2):
                for x in (c.ref.k, c.ref.v):
                    c.ref.store(r, l, x, np.full((1, 2, PH.D), word, np.int16))
        c.check()
    st.close()


def test_a_captured_compaction_replays():
    """free, fork and compact, captured once: each replay drops the branch, branches again and compresses the branch."""
    w, B = 8, 20
    st = PH.state(layers=2, heads=4, kv_heads=2, window=w)
    c = PH.Pair(st, n_pages=30, P=16, n_rows=2, max_pages=8)
    c.extend([0], [77])
    idx = torch.arange(0, 2 * B, 2, dtype=torch.int32, device="cuda").expand(2, 1, B).contiguous()
    seq, src, dst = sk.Seq(L=77, budget=B, idx=idx), c.ids([0]), c.ids([1])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sk.pages_free(st, c.pages, dst)
        sk.pages_fork(st, c.pages, src, dst, c.ws)
        sk.pages_compact(st, c.pages, dst, [seq], c.ws)
    for step in range(4):
        idx += 1          # (other tokens each time: the index is read on the device)
        g.replay()
        c.ref.free([1])
        c.ref.fork([0], [1])
        c.ref.compact([1], [77], [idx.cpu().numpy()], w)
        c.check()
    st.close()


def test_offsets_past_32_bits():
    """A pool of more than 2^32 elements: its last pages are stored to, copied and read back."""
    st = PH.state(heads=4, kv_heads=4)
    per = 4 * 256 * PH.D
    n_pages = (1 << 32) // per + 40
    pages = sk.make_pages(st, n_pages, 256, n_rows=3, max_pages=4)
    pages.refs[: n_pages - 6] = 1
    ws = sk.pages_workspace(st, pages, 2)
    ids = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    sk.pages_extend(st, pages, ids(0), ids(300), ws)
    k = torch.randn((1, 1, 300, 4, PH.D), device="cuda").to(torch.bfloat16)
    sk.pages_store(st, pages, 0, sk.Tokens(k=k, v=k.neg()))
    sk.pages_fork(st, pages, ids(0), ids(1), ws, deep=True)
    sk.pages_fork(st, pages, ids(0), ids(2), ws)
    sk.pages_extend(st, pages, ids(2), ids(1), ws)
    got, gotv = torch.zeros((2, 1, 300, 4, PH.D), dtype=torch.bfloat16, device="cuda"), None
    gotv = torch.zeros_like(got)
    sk.pages_load(st, pages, 0, sk.Tokens(k=got, v=gotv, rows=ids(0, 1)))
    torch.cuda.synchronize()
    sk.check_device_error(st)
    assert pages.table[0, 0].item() == n_pages - 6
    assert torch.equal(got, k.expand(2, -1, -1, -1, -1)) and torch.equal(gotv, -got)
    got = got[:1, :, :44].clone()
    tail = torch.zeros((1, 1, 45, 4, PH.D), dtype=torch.bfloat16, device="cuda")
    sk.pages_load(st, pages, 0, sk.Tokens(k=tail, rows=ids(2)))
    assert torch.equal(tail[:, :, :44], k[:, :, 256:])
    st.close()


def test_a_stream_of_its_own():
    st = PH.state(heads=4, kv_heads=2)
    c = PH.Pair(st, n_pages=30, P=16, n_rows=2, max_pages=8)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    rows, n = c.ids([1]), c.ids([37])
    sk.pages_extend(st, c.pages, rows, n, c.ws, stream=s)
    c.ref.extend([1], [37])
    k = torch.ones((1, 1, 37, 2, PH.D), dtype=torch.bfloat16, device="cuda")
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        sk.pages_store(st, c.pages, 0, sk.Tokens(k=k, v=k, rows=rows))
    s.synchronize()
    one = torch.ones((), dtype=torch.bfloat16).view(torch.int16).item()
    for x in (c.ref.k, c.ref.v):
        c.ref.store(1, 0, x, np.full((37, 2, PH.D), one, np.int16))
    c.check()
    st.close()


BAD_POOLS = [dict(k=None), dict(k=8), dict(table=2), dict(refs=None), dict(page_size=48), dict(page_size=8), dict(page_size=512),
             dict(n_pages=0), dict(n_pages=(1 << 20) + 1), dict(n_rows=0), dict(n_rows=65537), dict(max_pages=0),
             dict(max_pages=1 << 21), dict(page_stride=4 * 16 * 128 - 8), dict(page_stride=4 * 16 * 128 + 4),
             dict(layer_stride=-8), dict(layer_stride=8), dict(page_stride=1 << 38)]


@pytest.mark.parametrize("over", BAD_POOLS, ids=str)
def test_a_pool_that_is_none_is_refused_on_the_host(over):
    import ctypes as C
    st = PH.state(layers=2, heads=8, kv_heads=4)
    c = PH.Pair(st, n_pages=4, P=16, n_rows=2, max_pages=2)
    pg = c.pages.to_c()
    for name, x in over.items():
        old = getattr(pg, name)
        setattr(pg, name, old + x if name in ("k", "table") and x else x)
    L = sk.lib()
    n = C.c_size_t(0)
    want = (sk.ERR_INVALID_ARG, sk.ERR_UNSUPPORTED)
    assert L.starkv_pages_workspace_bytes(st.handle, C.byref(pg), 1, 1, C.byref(n)) in want
    assert L.starkv_pages_reset(st.handle, C.byref(pg), None) in want
    assert L.starkv_pages_free(st.handle, C.byref(pg), None, 1, None) in want
    c.check()
    st.close()


def test_calls_that_do_not_fit_are_refused_on_the_host():
    import ctypes as C
    st = PH.state(layers=2, heads=8, kv_heads=4, window=8, max_seqs=2)
    c = PH.Pair(st, n_pages=9, P=16, n_rows=2, max_pages=4)
    c.extend([0, 1], [33, 20])
    L, pg, ws = sk.lib(), c.pages.to_c(), (c.ws.data_ptr(), c.ws.numel())
    one, ids = c.ids([1, 1]), c.ids([0, 1])
    inv, uns = (sk.ERR_INVALID_ARG,), (sk.ERR_UNSUPPORTED,)
    P = C.byref(pg)
    assert L.starkv_pages_extend(st.handle, P, None, None, 2, *ws, None) in inv
    assert L.starkv_pages_extend(st.handle, P, None, one.data_ptr() + 1, 2, *ws, None) in inv
    assert L.starkv_pages_extend(st.handle, P, None, one.data_ptr(), -1, *ws, None) in inv
    assert L.starkv_pages_extend(st.handle, P, None, one.data_ptr(), 1025, *ws, None) in uns
    assert L.starkv_pages_extend(st.handle, P, None, one.data_ptr(), 2, ws[0], 255, None) in inv
    assert L.starkv_pages_extend(st.handle, P, None, one.data_ptr(), 2, ws[0] + 16, ws[1], None) in inv
    assert L.starkv_pages_fork(st.handle, P, None, ids.data_ptr(), 1, 0, *ws, None) in inv
    assert L.starkv_pages_fork(st.handle, P, ids.data_ptr(), ids.data_ptr(), 1, 2, *ws, None) in inv
    for seq in (sk.Seq(L=7), sk.Seq(L=33, budget=26), sk.Seq(L=33, budget=3),
                sk.Seq(L=33, meta=c.ids(range(33)))):
        with pytest.raises(sk.StarkvError) as e:
            sk.pages_compact(st, c.pages, None, [seq], c.ws)
        assert e.value.status == sk.ERR_INVALID_ARG
    k = torch.zeros((2, 2, 4, 4, PH.D), dtype=torch.bfloat16, device="cuda")
    for layer0, bad in ((1, k), (-1, k), (3, k[:, :1])):
        with pytest.raises(sk.StarkvError):
            sk.pages_store(st, c.pages, layer0, sk.Tokens(k=bad))
    wide = torch.zeros((2, 2, 4, 4, PH.D + 4), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(sk.StarkvError):       # rows that do not start on 16 bytes
        sk.pages_store(st, c.pages, 0, sk.Tokens(k=wide[..., :PH.D]))
    q = torch.zeros((2, 3, 8, PH.D), dtype=torch.bfloat16, device="cuda")
    o = torch.zeros_like(q)
    mask = torch.ones((2, 3), dtype=torch.int64, device="cuda")
    with pytest.raises(sk.StarkvError):       # two sequences into one place
        sk.pages_load(st, c.pages, 0, sk.Tokens(k=k[:1].expand(2, 2, 4, 4, PH.D)))
    calls = [lambda: sk.sink_attention(st, c.pages, 0, sk.Queries(q=q, o=q), 1, 4, c.ws),
             lambda: sk.tree_attention(st, c.pages, 2, sk.Queries(q=q, o=o, mask=mask), c.ws),
             lambda: sk.tree_attention(st, c.pages, 0, sk.Queries(q=q, o=o), c.ws),
             lambda: sk.sink_attention(st, c.pages, 0, sk.Queries(q=q, o=o), -1, 4, c.ws),
             lambda: sk.sink_attention(st, c.pages, 0, sk.Queries(q=q, o=o), 1, -4, c.ws),
             lambda: sk.sink_attention(st, c.pages, 0, sk.Queries(q=q, o=o[:, :1].expand(2, 3, 8, PH.D)), 1, 4, c.ws),
             lambda: sk.tree_attention(st, c.pages, 0, sk.Queries(q=q[:, :1].expand(2, 65, 8, PH.D), o=torch.zeros(
                 (2, 65, 8, PH.D), dtype=torch.bfloat16, device="cuda"), mask=torch.ones((2, 65), dtype=torch.int64, device="cuda")),
                 c.ws)]
    for call in calls:
        with pytest.raises(sk.StarkvError):
            call()
    for call in (lambda: sk.pages_free(st, c.pages, ids.long()), lambda: sk.pages_free(st, c.pages, ids.cpu()),
                 lambda: sk.pages_extend(st, c.pages, ids[:1], one, c.ws)):
        with pytest.raises(ValueError):
            call()
    # nothing to do is no error
    sk.pages_extend(st, c.pages, ids[:0], one[:0], c.ws)
    sk.pages_free(st, c.pages, ids[:0])
    sk.sink_attention(st, c.pages, 0, sk.Queries(q=q[:0], o=o[:0]), 1, 4, c.ws)
    sk.sink_attention(st, c.pages, 0, sk.Queries(q=q[:, :0], o=o[:, :0]), 1, 4, c.ws)
    sk.pages_store(st, c.pages, 0, sk.Tokens(k=k[:, :, :0]))
    c.check()
    st.close()


ON_HELD_PAGES = {
    "fork": lambda c, r, dst: sk.pages_fork(c.st, c.pages, c.ids([r]), c.ids([dst]), c.ws),
    "fork deep": lambda c, r, dst: sk.pages_fork(c.st, c.pages, c.ids([r]), c.ids([dst]), c.ws, deep=True),
    "free": lambda c, r, dst: sk.pages_free(c.st, c.pages, c.ids([r])),
    "compact": lambda c, r, dst: sk.pages_compact(c.st, c.pages, c.ids([r]), [sk.Seq(L=int(c.ref.len[r]), budget=0)], c.ws),
}


@pytest.mark.parametrize("at", [0, 3, 1100, 1299])
@pytest.mark.parametrize("what", sorted(ON_HELD_PAGES))
def test_a_call_on_a_row_with_a_wrong_page_changes_nothing(what, at):
    """A number that is no page, or a page that no row holds, anywhere among the pages of the call's row (the first
    1,024 are one block's): nothing is counted, moved or branched, and the branch's row keeps what it held."""
    st = PH.state(heads=1, kv_heads=1, window=8)
    c = PH.Pair(st, n_pages=4000, P=16, n_rows=4, max_pages=1400)
    c.extend([2, 0, 1], [16 * 1300, 16 * 1300 - 5, 70])
    c.free([2])                    # its entries stay behind: pages that are free now
    good = int(c.ref.table[0, at])
    for bad in (-1, 4000, 1 << 30, 3999):
        c.pages.table[0, at] = bad
        ON_HELD_PAGES[what](c, 0, 2)
        assert _error(st) == sk.ERR_DEVICE
        c.ref.table[0, at] = bad
        c.check()
        c.pages.table[0, at] = c.ref.table[0, at] = good
        c.check()
    ON_HELD_PAGES[what](c, 0, 2)   # and with the right one it is carried out
    assert _error(st) == sk.OK
    st.close()


def test_extending_a_row_whose_last_page_nobody_holds_changes_nothing():
    st = PH.state(heads=4, kv_heads=1, window=8)
    c = PH.Pair(st, n_pages=13, P=16, n_rows=2, max_pages=6)
    c.extend([0], [40])
    c.pages.refs[2] = c.ref.refs[2] = 0
    sk.pages_extend(st, c.pages, c.ids([0]), c.ids([3]), c.ws)
    assert _error(st) == sk.ERR_DEVICE
    c.check()
    st.close()


def test_calls_behind_a_refused_one_are_held_back_until_it_is_reported():
    """A store queued behind an extend that found no page would write over the row's last tokens; whatever else would
    change the pool counts on the refused call just as much."""
    st = PH.state(layers=2, heads=4, kv_heads=2, window=8, max_seqs=2)
    c = PH.Pair(st, n_pages=8, P=16, n_rows=4, max_pages=6)
    other = PH.Pair(st, n_pages=8, P=16, n_rows=2, max_pages=4)
    c.extend([0, 1], [40, 50])       # 7 of 8 pages, none shared
    k = torch.zeros((1, 2, 30, 2, PH.D), dtype=torch.bfloat16, device="cuda")
    tok = sk.Tokens(k=k, v=k, rows=c.ids([0]))
    keep = torch.arange(20, dtype=torch.int32, device="cuda").expand(2, 1, 20).contiguous()
    sk.pages_extend(st, c.pages, c.ids([0]), c.ids([30]), c.ws)       # needs two pages
    sk.pages_store(st, c.pages, 0, tok)
    for call in (lambda: sk.pages_extend(st, c.pages, c.ids([2]), c.ids([3]), c.ws),      # each would do by itself
                 lambda: sk.pages_fork(st, c.pages, c.ids([0]), c.ids([2]), c.ws),
                 lambda: sk.pages_fork(st, c.pages, c.ids([0]), c.ids([2]), c.ws, deep=True),
                 lambda: sk.pages_compact(st, c.pages, c.ids([0]), [sk.Seq(L=40, budget=20, idx=keep)], c.ws),
                 lambda: sk.pages_free(st, c.pages, c.ids([1])),
                 lambda: sk.pages_extend(st, other.pages, other.ids([1]), other.ids([3]), other.ws)):
        call()
        sk.pages_store(st, c.pages, 1, sk.Tokens(k=k[:, :1], v=k[:, :1], rows=c.ids([1])))
    got = torch.empty((1, 2, 40, 2, PH.D), dtype=torch.bfloat16, device="cuda")
    sk.pages_load(st, c.pages, 0, sk.Tokens(k=got, rows=c.ids([0])))          # reading goes on
    assert _error(st) == sk.ERR_DEVICE
    c.check()
    other.check()
    for layer in range(2):
        want = c.ref.tokens(0, layer, c.ref.k).swapaxes(0, 1)
        np.testing.assert_array_equal(got[0, layer].view(torch.int16).cpu().numpy(), want)
    c.free([1])                      # reported: the pool is as the refused call found it, and the call may be made again
    c.extend([0], [30])
    sk.pages_store(st, c.pages, 0, tok)
    for layer in range(2):
        for x in (c.ref.k, c.ref.v):
            c.ref.store(0, layer, x, np.zeros((30, 2, PH.D), np.int16))
    c.check()
    st.close()


def test_captured_steps_stop_where_the_pool_is_full():
    """extend and store of a token, replayed past the last free page: the row keeps every token that it took."""
    st = PH.state(layers=1, heads=4, kv_heads=1, window=8)
    c = PH.Pair(st, n_pages=3, P=16, n_rows=2, max_pages=6)
    c.extend([0], [20])
    rows, one = c.ids([0]), c.ids([1])
    k = torch.zeros((1, 1, 1, 1, PH.D), dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sk.pages_extend(st, c.pages, rows, one, c.ws)
        sk.pages_store(st, c.pages, 0, sk.Tokens(k=k, v=k, rows=rows))
    for step in range(40):
        k.fill_(float(step + 1))
        g.replay()
        if int(c.ref.len[0]) < 48:
            c.ref.extend([0], [1])
            word = torch.tensor(float(step + 1), dtype=torch.bfloat16).view(torch.int16).item()
            for x in (c.ref.k, c.ref.v):
                c.ref.store(0, 0, x, np.full((1, 1, PH.D), word, np.int16))
        c.check(errors=False)
    assert _error(st) == sk.ERR_DEVICE
    c.check()
    st.close()


def test_errors_of_a_store_hold_nothing_back():
    st = PH.state(heads=4, kv_heads=2)
    c = PH.Pair(st, n_pages=12, P=16, n_rows=3, max_pages=4)
    c.extend([0], [20])
    c.fork([0], [1])
    k = torch.zeros((1, 1, 6, 2, PH.D), dtype=torch.bfloat16, device="cuda")
    sk.pages_store(st, c.pages, 0, sk.Tokens(k=k, v=k, rows=c.ids([1])))      # into a shared page: passed over
    c.extend([1], [6])
    sk.pages_store(st, c.pages, 0, sk.Tokens(k=k, v=k, rows=c.ids([1])))
    for x in (c.ref.k, c.ref.v):
        c.ref.store(1, 0, x, np.zeros((6, 2, PH.D), np.int16))
    assert _error(st) == sk.ERR_DEVICE
    c.check()
    st.close()


@pytest.mark.parametrize("n,twins", [(3, [(0, 2)]), (40, [(3, 39), (4, 5)]), (1024, [(0, 1023), (100, 101), (300, 900)])])
def test_a_store_that_names_a_row_twice_leaves_that_row_alone(n, twins):
    """Two sequences' tokens for the same places, far apart in the call or next to each other: neither is written and
    it is reported; the others are.  A sequence that brings no tokens is no rival (a padded batch), and to load a row
    twice is nothing wrong."""
    st = PH.state(layers=2, heads=4, kv_heads=2)
    c = PH.Pair(st, n_pages=2 * n + 3, P=16, n_rows=n, max_pages=3)
    c.extend(range(n), [3 + i % 20 for i in range(n)])
    T = 3
    rows = [int(r) for r in np.random.default_rng(n).permutation(n)]
    k = torch.from_numpy(np.random.default_rng(1).standard_normal((2, n, 2, T, 2, PH.D), dtype=np.float32)).to(torch.bfloat16).cuda()
    for padded in (False, True):
        named, counts = list(rows), [T] * n
        for a, b in twins:
            named[b] = named[a]
            counts[b] = 0 if padded else T
        sk.pages_store(st, c.pages, 0, sk.Tokens(k=k[0], v=k[1], rows=c.ids(named), n_tokens=c.ids(counts)))
        assert _error(st) == (sk.OK if padded else sk.ERR_DEVICE)
        lone = [i for i in range(n) if counts[i] and (padded or named.count(named[i]) == 1)]
        for i in lone:
            for layer in range(2):
                for x, part in ((c.ref.k, k[0]), (c.ref.v, k[1])):
                    c.ref.store(named[i], layer, x, part[i, layer].view(torch.int16).cpu().numpy())
        c.check()
        k = k.flip(0)
    back = torch.empty((2, 2, T, 2, PH.D), dtype=torch.bfloat16, device="cuda")
    sk.pages_load(st, c.pages, 0, sk.Tokens(k=back, rows=c.ids([rows[1], rows[1]])))
    assert _error(st) == sk.OK and torch.equal(back[0], back[1])
    st.close()


def test_compaction_looks_at_no_slot():
    """More rows than the state has slots, all with the default one: compaction touches no slot's state."""
    w = 8
    st = PH.state(heads=4, kv_heads=2, window=w, max_seqs=1)
    c = PH.Pair(st, n_pages=40, P=16, n_rows=3, max_pages=8)
    c.extend([0, 1, 2], [60, 33, 90])
    idx = [np.arange(b, dtype=np.int32).reshape(1, 1, b) for b in (20, 5, 40)]
    sk.pages_compact(st, c.pages, None, [sk.Seq(L=int(c.ref.len[i]), budget=x.size, idx=torch.from_numpy(x).cuda())
                                         for i, x in enumerate(idx)], c.ws)
    c.ref.compact([0, 1, 2], [60, 33, 90], idx, w)
    c.check()
    st.close()


def test_outputs_whose_rows_meet_are_refused_on_the_host():
    """Strides that each step over a row and still let two rows share elements; axes in any order, or interleaved without meeting, are taken."""
    st = PH.state(layers=2, heads=8, kv_heads=4)
    c = PH.Pair(st, n_pages=9, P=16, n_rows=2, max_pages=4)
    c.extend([0, 1], [20, 20])
    bf = dict(dtype=torch.bfloat16, device="cuda")
    flat, D = torch.zeros(1 << 16, **bf), PH.D
    q = torch.zeros((2, 3, 8, D), **bf)
    for strides in ((3 * D, D, D), (8 * D, 8 * D, D), (24 * D, 7 * D, D), (23 * D, 8 * D, D), (D, 2 * D, 3 * D), (1 << 47, 1 << 62, D)):
        with pytest.raises((sk.StarkvError, RuntimeError)):
            sk.sink_attention(st, c.pages, 0, sk.Queries(q=q, o=flat.as_strided((2, 3, 8, D), (*strides, 1))), 1, 40, c.ws)
    for strides in ((24 * D, 8 * D, D), (D, 2 * D, 6 * D), (3 * D, D, 6 * D), (50 * D, 9 * D, D), (3 * D, 2 * D, 8 * D)):
        sk.sink_attention(st, c.pages, 0, sk.Queries(q=q, o=flat.as_strided((2, 3, 8, D), (*strides, 1))), 1, 40, c.ws)
    for strides in ((D, D, D, D), (24 * D, 12 * D, 4 * D, 2 * D), (24 * D, 11 * D, 4 * D, D), (12 * D, 12 * D, 4 * D, D)):
        with pytest.raises(sk.StarkvError):
            sk.pages_load(st, c.pages, 0, sk.Tokens(k=flat.as_strided((2, 2, 3, 4, D), (*strides, 1))))
    k = torch.zeros((2, 2, 3, 4, D), **bf)
    with pytest.raises(sk.StarkvError):
        sk.pages_load(st, c.pages, 0, sk.Tokens(k=k, v=k))
    for strides in ((24 * D, 12 * D, 4 * D, D), (D, 24 * D, 8 * D, 2 * D), (24 * D, 12 * D, D, 3 * D)):
        sk.pages_load(st, c.pages, 0, sk.Tokens(k=flat.as_strided((2, 2, 3, 4, D), (*strides, 1))))
    c.check()
    st.close()
