"""Attention mass, eviction, page bounds and chosen pages as they are used: one after another over growing rows, captured
and replayed, on other streams, far into large tensors; and what is refused on the host."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from paper_2606_01790_gb300 import starkv as sk

import paged_harness as PH

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

from test_gpu_mass import make_mass, weighed, verify as verify_mass  # noqa: E402
from test_gpu_paged_attention import built, filled, queries  # noqa: E402,F401
from test_gpu_sparse import bounded, verify as verify_sparse  # noqa: E402


@pytest.mark.parametrize("per_head", [False, True])
def test_decoding_with_eviction_and_chosen_pages(per_head):
    """Rows grow by tokens, are attended over, weighed and evicted from when they are long, branch, and are read through chosen
    pages: every call against the definition."""
    layers, G, H, P, w, budget = 2, 2, 8, 16, 4, 40
    st = PH.state(layers=layers, heads=H, kv_heads=G, window=w, select_mode=int(per_head))
    c = PH.Pair(st, n_pages=90, P=P, n_rows=4, max_pages=12)
    mass, bounds = sk.make_mass(st, c.pages, decay=0.9), sk.make_bounds(st, c.pages)
    ref_mass = np.zeros(tuple(mass.data.shape))
    rng = np.random.default_rng(int(per_head))
    ws = sk.sparse_workspace(st, c.pages, 4, 16, 5)
    evictions = 0

    def tokens(rows, T):
        """T new tokens of each row: stored, bounded, attended over with a window, weighed."""
        n = len(rows)
        ids = c.ids(rows)
        c.extend(rows, [T] * n)
        kv = torch.from_numpy(rng.standard_normal((2, n, layers, T, G, PH.D), dtype=np.float32)).to(torch.bfloat16).cuda()
        sk.pages_store(st, c.pages, 0, sk.Tokens(k=kv[0], v=kv[1], rows=ids))
        for i, r in enumerate(rows):
            for layer in range(layers):
                for x, part in ((c.ref.k, kv[0]), (c.ref.v, kv[1])):
                    c.ref.store(r, layer, x, part[i, layer].view(torch.int16).cpu().numpy())
        sk.pages_bounds(st, c.pages, 0, layers, bounds, T, rows=ids)
        for layer in range(layers):
            qs = queries(c, n, T, seed=int(rng.integers(1 << 30)), rows=ids)
            sk.sink_attention(st, c.pages, layer, qs, 2, 50, c.ws)
            sk.sink_mass(st, c.pages, layer, qs, 2, 50, mass, c.ws)
            torch.cuda.synchronize()
            lse, q = qs.lse.cpu().numpy(), qs.q.float().cpu().numpy()
            for i, r in enumerate(rows):
                L = int(c.ref.len[r])
                k, v = c.cache(r, layer)
                seen, off = O.seen_sink(L, T, 2, 50), []
                want = O.mass(q[i], k, lse[i], seen, ref_mass[layer, r, :, :L], 0.9, off)
                got = mass.data[layer, r, :, :L].cpu().numpy()
                assert np.all(np.abs(got - want) <= off[0]), (layer, r)
                ref_mass[layer, r, :, :L] = got       # (from here on what the device has: choices hang on the last bit)
                PH.check_attention(qs.o[i].float().cpu().numpy(), lse[i], q[i], k, v, seen)

    def evict(rows):
        Ls = [int(c.ref.len[r]) for r in rows]
        idx = [torch.zeros((layers, G if per_head else 1, budget), dtype=torch.int32, device="cuda") for _ in rows]
        sk.pages_evict(st, c.pages, c.ids(rows), [sk.Seq(L=L, budget=budget, idx=i) for L, i in zip(Ls, idx)], mass, c.ws)
        keep = []
        for r, L in zip(rows, Ls):
            past = ref_mass[:, r, :, :L - w]
            x = past if per_head else past.sum(1, keepdims=True)
            keep.append(np.stack([[O.heaviest(p, budget) for p in y] for y in x]))
            at = np.concatenate([keep[-1], np.broadcast_to(np.arange(L - w, L), (*keep[-1].shape[:2], w))], -1)
            ref_mass[:, r, :, :budget + w] = np.take_along_axis(ref_mass[:, r], np.broadcast_to(at, (layers, G, budget + w)), -1)
        for i, k in zip(idx, keep):
            np.testing.assert_array_equal(i.cpu().numpy(), k)
        c.ref.compact(rows, Ls, keep, w)
        sk.pages_bounds(st, c.pages, 0, layers, bounds, budget + w, rows=c.ids(rows))

    tokens([0, 1], 13)
    for step in range(18):
        tokens([0, 1] if step < 9 else [0, 1, 2], int(rng.integers(1, 16)))
        if step == 8:      # a branch takes its source's mass along
            c.fork([1], [2])
            mass.data[:, 2] = mass.data[:, 1]
            ref_mass[:, 2] = ref_mass[:, 1]
        long = [r for r in range(3) if c.ref.len[r] >= budget + w + 20]
        if long:
            evict(long)
            evictions += 1
        rows = [r for r in range(3) if c.ref.len[r] > 0]
        qs = queries(c, len(rows), 1, seed=step, rows=c.ids(rows))
        chosen = torch.full((len(rows), 1, G, 4), -5, dtype=torch.int32, device="cuda")
        sk.sparse_attention(st, c.pages, 1, qs, bounds, 1, 1, 4, ws, chosen_out=chosen)
        verify_sparse(c, qs, bounds, rows, [1] * len(rows), 1, 1, 4, chosen, layer=1)
        c.check()
        for r in rows:
            L = int(c.ref.len[r])
            np.testing.assert_array_equal(mass.data[:, r, :, :L].cpu().numpy(), ref_mass[:, r, :, :L].astype(np.float32))
    assert evictions >= 3
    # the bounds of every page that a row holds are those of its keys
    b = bounds.float().cpu().numpy()
    for r in range(3):
        for j in range(-(-int(c.ref.len[r]) // P)):
            fill = min(P, int(c.ref.len[r]) - j * P)
            k = torch.from_numpy(c.ref.k[:, c.ref.table[r, j]][:, :, :fill].copy()).view(torch.bfloat16).float().numpy()
            np.testing.assert_array_equal(b[:, c.ref.table[r, j]], np.stack([k.min(2), k.max(2)], 2))
    st.close()


def test_captured_calls_replay_with_what_the_arrays_hold_then():
    """Two graphs over one workspace, replayed in turn, with lengths, counts, queries and masses that change between."""
    c = filled([300, 150, 77], P=16, heads=8, kv_heads=2)
    bounds = bounded(c)
    T = 40
    counts, rows = c.ids([40, 3, 17]), c.ids([2, 0, 1])
    qs = queries(c, 3, T, rows=rows, n_tokens=counts)
    sp = queries(c, 3, 2, seed=5, rows=rows)
    chosen = torch.full((3, 2, 2, 6), -5, dtype=torch.int32, device="cuda")
    ws = torch.empty(max(sk.sparse_workspace(c.st, c.pages, 3, 2, 6).numel(), c.ws.numel()), dtype=torch.uint8, device="cuda")
    before, mass = make_mass(c, 0.5)
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):      # (a first call outside a capture)
        sk.sink_attention(c.st, c.pages, 0, qs, 1, 90, ws)
        sk.sink_mass(c.st, c.pages, 0, qs, 1, 90, mass, ws)
        sk.sparse_attention(c.st, c.pages, 0, sp, bounds, 1, 1, 6, ws, chosen_out=chosen)
    torch.cuda.synchronize()
    with torch.cuda.graph(graphs[0]):
        sk.sink_attention(c.st, c.pages, 0, qs, 1, 90, ws)
        sk.sink_mass(c.st, c.pages, 0, qs, 1, 90, mass, ws)
    with torch.cuda.graph(graphs[1]):
        sk.pages_bounds(c.st, c.pages, 0, 1, bounds, 2, rows=rows)
        sk.sparse_attention(c.st, c.pages, 0, sp, bounds, 1, 1, 6, ws, chosen_out=chosen)
    for lens, n in (([300, 150, 77], [40, 3, 17]), ([211, 149, 60], [1, 40, 0]), ([300, 33, 70], [9, 40, 33])):
        c.pages.len.copy_(torch.tensor(lens, dtype=torch.int32))
        c.ref.len[:] = lens
        counts.copy_(torch.tensor(n, dtype=torch.int32))
        sk.pages_bounds(c.st, c.pages, 0, 1, bounds, 300, n_tokens=c.pages.len)
        mass.data.copy_(torch.from_numpy(before))
        for x in (qs.o, qs.lse, sp.o, sp.lse):
            x.fill_(9.0)
        chosen.fill_(-5)
        graphs[0].replay()
        graphs[1].replay()
        graphs[1].replay()
        verify_mass(c, qs, lambda i, L, m: O.seen_sink(L, m, 1, 90), [2, 0, 1], n, before, mass)
        verify_sparse(c, sp, bounds, [2, 0, 1], [2] * 3, 1, 1, 6, chosen)
    c.st.close()


def test_a_captured_eviction():
    st = PH.state(layers=1, heads=8, kv_heads=2, window=4)
    c = PH.Pair(st, n_pages=40, P=16, n_rows=2, max_pages=8)
    c.extend([0], [100])
    data, mass = make_mass(c, 1.0)
    idx = torch.zeros((1, 1, 30), dtype=torch.int32, device="cuda")
    seqs, dst, src = [sk.Seq(L=100, budget=30, idx=idx)], c.ids([1]), c.ids([0])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sk.pages_fork(st, c.pages, src, dst, c.ws)
        mass.data[:, 1].copy_(mass.data[:, 0])
        sk.pages_evict(st, c.pages, dst, seqs, mass, c.ws)
    for i in range(3):
        data = np.random.default_rng(i).exponential(size=data.shape).astype(np.float32)
        mass.data.copy_(torch.from_numpy(data))
        c.free([1])
        g.replay()
        c.ref.fork([0], [1])
        keep = O.heaviest(data[0, 0, :, :96].astype(np.float64).sum(0), 30)
        c.ref.compact([1], [100], [keep[None, None]], 4)
        c.check()
        np.testing.assert_array_equal(idx[0, 0].cpu().numpy(), keep)
        at = np.concatenate([keep, np.arange(96, 100)])
        np.testing.assert_array_equal(mass.data[0, 1, :, :34].cpu().numpy(), data[0, 0][:, at])
    st.close()


def test_calls_on_another_stream():
    """In the order of the stream that a call names, with work of the current one on either side."""
    c = filled([900, 640], P=32, heads=8, kv_heads=2)
    bounds = bounded(c)
    side = torch.cuda.Stream()
    rows, counts = [0, 1], [5, 5]
    qs, sp = queries(c, 2, 5), queries(c, 2, 1, seed=2)
    seen = lambda i, L, n: O.seen_sink(L, n, 0, 300)   # noqa: E731
    weighed(c, qs, seen, rows, counts)
    before, mass = make_mass(c, 0.5)
    chosen = torch.full((2, 1, 2, 6), -5, dtype=torch.int32, device="cuda")
    ws = sk.sparse_workspace(c.st, c.pages, 2, 5, 6)
    torch.cuda._sleep(2_000_000)
    side.wait_stream(torch.cuda.current_stream())
    sk.sink_mass(c.st, c.pages, 0, qs, 0, 300, mass, ws, stream=side)
    sk.pages_bounds(c.st, c.pages, 0, 1, bounds, 3, stream=side)
    sk.sparse_attention(c.st, c.pages, 0, sp, bounds, 1, 1, 6, ws, chosen_out=chosen, stream=side.cuda_stream)
    torch.cuda.current_stream().wait_stream(side)
    verify_mass(c, qs, seen, rows, counts, before, mass)
    verify_sparse(c, sp, bounds, rows, [1, 1], 1, 1, 6, chosen)
    c.st.close()


def test_masses_behind_a_refused_call_are_held_back():
    """A mass call counts on the tokens of the extend in front of it."""
    c = filled([40, 60], P=16, heads=8, kv_heads=2)
    qs = queries(c, 2, 3)
    weighed(c, qs, lambda i, L, n: O.seen_sink(L, n, 0, 99), [0, 1], [3, 3])
    before, mass = make_mass(c, 0.5)
    sk.pages_extend(c.st, c.pages, c.ids([0]), c.ids([100000]), c.ws)
    sk.sink_mass(c.st, c.pages, 0, qs, 0, 99, mass, c.ws)
    torch.cuda.synchronize()
    assert sk.device_error_status(c.st) == sk.ERR_DEVICE
    np.testing.assert_array_equal(mass.data.cpu().numpy(), before)
    sk.sink_mass(c.st, c.pages, 0, qs, 0, 99, mass, c.ws)
    verify_mass(c, qs, lambda i, L, n: O.seen_sink(L, n, 0, 99), [0, 1], [3, 3], before, mass)
    c.st.close()


def test_offsets_past_32_bits():
    """Masses, bounds and keys that lie more than 2^32 bytes, and 2^31 elements, into their tensors."""
    P, G, H = 16, 1, 4
    st = PH.state(layers=1, heads=H, kv_heads=G, window=2)
    n_pages, n_rows, max_pages = 40, 3, 12
    stride = 150_000_000                      # elements between pages, masses of rows, bounds of pages
    i32 = dict(dtype=torch.int32, device="cuda")
    kv = [torch.empty(39 * stride + P * PH.D, dtype=torch.bfloat16, device="cuda").as_strided(
        (1, n_pages, G, P, PH.D), (40 * stride, stride, P * PH.D, PH.D, 1)) for _ in range(2)]
    rng = np.random.default_rng(0)
    small = [torch.from_numpy(rng.standard_normal((1, n_pages, G, P, PH.D), dtype=np.float32)).to(torch.bfloat16) for _ in range(2)]
    for x, y in zip(kv, small):
        x.copy_(y)
    pages = sk.Pages(k=kv[0], v=kv[1], table=torch.zeros((n_rows, max_pages), **i32), len=torch.zeros(n_rows, **i32),
                     refs=torch.zeros(n_pages, **i32))
    lens = [180, 33, 150]
    order = rng.permutation(n_pages)
    ref = O.Pool(small[0].view(torch.int16).numpy().copy(), small[1].view(torch.int16).numpy().copy(),
                 np.zeros((n_rows, max_pages), np.int32), np.array(lens, np.int32), np.zeros(n_pages, np.int32))
    at = 0
    for r, n in enumerate(lens):
        m = -(-n // P)
        ref.table[r, :m] = order[at:at + m]
        ref.refs[order[at:at + m]] = 1
        at += m
    for x, y in ((pages.table, ref.table), (pages.len, ref.len), (pages.refs, ref.refs)):
        x.copy_(torch.from_numpy(y))

    class C:      # what the checks look at
        pass
    c = C()
    c.st, c.pages, c.ref = st, pages, ref
    c.cache = lambda r, layer: PH.Pair.cache(c, r, layer)
    cap = max_pages * P
    data = torch.empty(2 * 20 * stride + cap, device="cuda").as_strided((1, n_rows, G, cap), (60 * stride, 20 * stride, cap, 1))
    before = rng.exponential(size=(1, n_rows, G, cap)).astype(np.float32)
    data.copy_(torch.from_numpy(before))
    mass = sk.Mass(data, 0.5)
    ws = sk.sparse_workspace(st, pages, 3, 4, 5)
    qs = queries(c, 3, 4)
    seen = lambda i, L, n: O.seen_sink(L, n, 0, 100)   # noqa: E731
    weighed(c, qs, seen, [0, 1, 2], [4] * 3)
    sk.sink_mass(st, pages, 0, qs, 0, 100, mass, ws)
    verify_mass(c, qs, seen, [0, 1, 2], [4] * 3, before, mass)
    bounds = torch.empty(39 * stride + 2 * PH.D, dtype=torch.bfloat16, device="cuda").as_strided(
        (1, n_pages, G, 2, PH.D), (40 * stride, stride, 2 * PH.D, PH.D, 1))
    sk.pages_bounds(st, pages, 0, 1, bounds, 180, n_tokens=pages.len)
    chosen = torch.full((3, 4, G, 5), -5, **i32)
    sk.sparse_attention(st, pages, 0, qs, bounds, 1, 1, 5, ws, chosen_out=chosen)
    verify_sparse(c, qs, bounds, [0, 1, 2], [4] * 3, 1, 1, 5, chosen)
    now = mass.data.cpu().numpy()
    idx = torch.zeros((1, 1, 20), **i32)
    sk.pages_evict(st, pages, torch.tensor([2], **i32), [sk.Seq(L=150, budget=20, idx=idx)], mass, ws)
    keep = O.heaviest(now[0, 2, 0, :148], 20)
    ref.compact([2], [150], [keep[None, None]], 2)
    torch.cuda.synchronize()
    sk.check_device_error(st)
    np.testing.assert_array_equal(idx[0, 0].cpu().numpy(), keep)
    np.testing.assert_array_equal(pages.table.cpu().numpy(), ref.table)
    for x, y in zip(kv, (ref.k, ref.v)):
        np.testing.assert_array_equal(x.contiguous().view(torch.int16).cpu().numpy(), y)
    np.testing.assert_array_equal(mass.data[0, 2, 0, :22].cpu().numpy(), now[0, 2, 0, np.concatenate([keep, [148, 149]])])
    st.close()


def test_calls_without_work():
    c = filled([40, 20], P=16, heads=8, kv_heads=2)
    before, mass = make_mass(c, 0.5)
    bounds = bounded(c)
    was = bounds.clone()
    z = lambda n, T: sk.Queries(q=torch.zeros((n, T, 8, PH.D), dtype=torch.bfloat16, device="cuda"),   # noqa: E731
                                o=torch.full((n, T, 8, PH.D), 9.0, dtype=torch.bfloat16, device="cuda"),
                                lse=torch.zeros((n, T, 8), device="cuda"), mask=torch.zeros((n, T), dtype=torch.int64, device="cuda"))
    ws = sk.sparse_workspace(c.st, c.pages, 2, 1, 3)
    for n, T in ((0, 1), (2, 0)):
        sk.sink_mass(c.st, c.pages, 0, z(n, T), 0, 1, mass, ws)
        sk.tree_mass(c.st, c.pages, 0, z(n, T), mass, ws)
        sk.sparse_attention(c.st, c.pages, 0, z(n, T), bounds, 0, 1, 3, ws)
    none = z(2, 1)
    none.n_tokens = c.ids([0, 0])
    sk.sink_mass(c.st, c.pages, 0, none, 0, 1, mass, ws)
    sk.tree_mass(c.st, c.pages, 0, none, mass, ws)
    sk.sparse_attention(c.st, c.pages, 0, none, bounds, 0, 1, 3, ws)
    assert torch.all(none.o == 9)
    sk.pages_bounds(c.st, c.pages, 0, 0, bounds, 4)
    sk.pages_bounds(c.st, c.pages, 0, 1, bounds, 0)
    sk.pages_bounds(c.st, c.pages, 0, 1, bounds, 4, n_tokens=c.ids([0, 0]))
    sk.pages_evict(c.st, c.pages, c.ids([]), [], mass, c.ws)
    torch.cuda.synchronize()
    sk.check_device_error(c.st)
    np.testing.assert_array_equal(mass.data.cpu().numpy(), before)
    assert torch.equal(bounds.nan_to_num(7.0), was.nan_to_num(7.0))
    c.st.close()


def test_calls_that_do_not_fit_are_refused_on_the_host():
    c = filled([40, 60], P=16, heads=8, kv_heads=2, layers=2)
    st, pages = c.st, c.pages
    cap = pages.table.shape[1] * 16
    bounds, mass = sk.make_bounds(st, pages), sk.make_mass(st, pages)
    qs = queries(c, 2, 3)
    deep = queries(c, 2, 65)
    deep.mask = torch.zeros((2, 65), dtype=torch.int64, device="cuda")
    ws = sk.sparse_workspace(st, pages, 2, 3, 4)
    flat = torch.zeros(1 << 16, device="cuda")
    narrow = flat.as_strided((2, 2, 2, cap), (4 * cap, 2 * cap, cap - 1, 1))       # rows of two heads meet
    fb = torch.zeros(1 << 16, dtype=torch.bfloat16, device="cuda")
    met = fb.as_strided((2, pages.k.shape[1], 2, 2, 128), (256, 512, 256, 128, 1))     # layers inside pages, and through them
    bad = [
        lambda: sk.sink_mass(st, pages, 2, qs, 0, 1, mass, ws), lambda: sk.sink_mass(st, pages, -1, qs, 0, 1, mass, ws),
        lambda: sk.sink_mass(st, pages, 0, qs, -1, 1, mass, ws), lambda: sk.sink_mass(st, pages, 0, qs, 0, -1, mass, ws),
        lambda: sk.sink_mass(st, pages, 0, qs, 0, 1, sk.Mass(mass.data, float("nan")), ws),
        lambda: sk.sink_mass(st, pages, 0, qs, 0, 1, sk.Mass(mass.data, float("inf")), ws),
        lambda: sk.sink_mass(st, pages, 0, qs, 0, 1, sk.Mass(mass.data, -0.5), ws),
        lambda: sk.sink_mass(st, pages, 0, qs, 0, 1, sk.Mass(narrow), ws),
        lambda: sk.sink_mass(st, pages, 0, qs, 0, 1, mass, ws[:1000]), lambda: sk.tree_mass(st, pages, 0, qs, mass, ws),
        lambda: sk.tree_mass(st, pages, 0, deep, mass, ws),
        lambda: sk.pages_evict(st, pages, None, [sk.Seq(L=40, budget=41, idx=torch.zeros((2, 1, 41), dtype=torch.int32, device="cuda"))],
                               mass, c.ws),
        lambda: sk.pages_evict(st, pages, None, [sk.Seq(L=40, budget=3)], mass, c.ws),
        lambda: sk.pages_evict(st, pages, None, [sk.Seq(L=40)], sk.Mass(narrow), c.ws),
        lambda: sk.pages_bounds(st, pages, 0, 3, bounds, 4), lambda: sk.pages_bounds(st, pages, -1, 1, bounds, 4),
        lambda: sk.pages_bounds(st, pages, 0, 1, bounds, -1), lambda: sk.pages_bounds(st, pages, 0, 1, bounds, (1 << 24) + 1),
        lambda: sk.pages_bounds(st, pages, 0, 1, met, 4),
        lambda: sk.sparse_attention(st, pages, 0, qs, bounds, 0, 0, 4, ws), lambda: sk.sparse_attention(st, pages, 0, qs, bounds, -1, 1, 4, ws),
        lambda: sk.sparse_attention(st, pages, 0, qs, bounds, 3, 2, 4, ws), lambda: sk.sparse_attention(st, pages, 0, qs, bounds, 0, 1, 0, ws),
        lambda: sk.sparse_attention(st, pages, 2, qs, bounds, 0, 1, 4, ws), lambda: sk.sparse_attention(st, pages, 0, qs, met, 0, 1, 4, ws),
        lambda: sk.sparse_attention(st, pages, 0, qs, bounds, 0, 1, 4, ws[:-256]),
        lambda: sk.sparse_workspace(st, pages, 1025, 1, 4), lambda: sk.sparse_workspace(st, pages, 1, -1, 4),
        lambda: sk.sparse_workspace(st, pages, 1, 1, 0),
    ]
    before = mass.data.clone()
    for i, call in enumerate(bad):
        with pytest.raises(sk.StarkvError) as e:
            call()
        assert e.value.status in (sk.ERR_INVALID_ARG, sk.ERR_UNSUPPORTED), i
    same = sk.Queries(q=qs.q, o=qs.q)
    with pytest.raises(sk.StarkvError):
        sk.sparse_attention(st, pages, 0, same, bounds, 0, 1, 4, ws)
    torch.cuda.synchronize()
    sk.check_device_error(st)
    assert torch.equal(mass.data, before)
    c.check()
    st.close()


def test_a_workspace_for_more_serves_fewer():
    """Of rows, queries or pages; also where the scores of all queries would not fit one launch's share of it."""
    st = PH.state(layers=1, heads=8, kv_heads=8)
    c = PH.Pair(st, n_pages=300, P=16, n_rows=4, max_pages=100_000)
    c.extend([0, 1], [2000, 600])
    bounds = bounded(c)
    ws = sk.sparse_workspace(st, c.pages, 4, 40, 5000)
    for n, T, n_chosen in ((4, 40, 5000), (2, 40, 7), (1, 3, 5000), (2, 40, 3)):
        assert sk.sparse_workspace(st, c.pages, n, T, n_chosen).numel() <= ws.numel()
        qs = queries(c, min(n, 2), T, rows=c.ids([0, 1][:n]))
        sk.sparse_attention(st, c.pages, 0, qs, bounds, 1, 1, n_chosen, ws)
        torch.cuda.synchronize()
        sk.check_device_error(st)
        assert torch.isfinite(qs.o).all()
    st.close()
