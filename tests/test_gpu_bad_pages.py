"""Page numbers that are none in a table's rows: what the calls that weigh tokens and choose pages do with them."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from paper_2606_01790_gb300 import starkv as sk

import paged_harness as PH

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

from test_gpu_mass import make_mass  # noqa: E402
from test_gpu_paged_attention import built, filled, queries, random_tree, words  # noqa: E402,F401
from test_gpu_sparse import bounded  # noqa: E402


@pytest.mark.parametrize("P", [16, 64, 256])
@pytest.mark.parametrize("kind,T", [("sink", 1), ("sink", 6), ("sink", 200), ("tree", 3), ("tree", 40)])
def test_tokens_of_a_page_that_is_none_keep_their_mass(P, kind, T):
    """In the middle of a row, at its start and under its newest tokens; seen by the queries or not (a window of 90: the
    first tokens only fade).  Other tokens get what the definition says."""
    lens = [1500, 700, 900, 800]
    c = filled(lens, P=P, heads=8, kv_heads=2, seed=T)
    bad = {0: [(1, -1)], 1: [((700 - 1) // P, len(c.ref.refs))], 2: [(0, 1 << 30), (900 // P - 1, -(1 << 31))]}
    for r, entries in bad.items():
        for at, x in entries:
            c.pages.table[r, at] = x      # (the definition's table keeps the page)
    masks = [random_tree(np.random.default_rng(i), T) for i in range(4)] if kind == "tree" else None
    qs = queries(c, 4, T, mask=words(masks, T) if masks else None)
    qs.lse.fill_(-3.0)                    # (a logit of 0, as of a key of zeros, would weigh 20)
    before, mass = make_mass(c, 0.5)
    if kind == "tree":
        sk.tree_mass(c.st, c.pages, 0, qs, mass, c.ws)
    else:
        sk.sink_mass(c.st, c.pages, 0, qs, 2, 90, mass, c.ws)
    torch.cuda.synchronize()
    assert sk.device_error_status(c.st) == sk.ERR_DEVICE
    got, q, lse = mass.data.cpu().numpy(), qs.q.float().cpu().numpy(), qs.lse.cpu().numpy()
    for r, L in enumerate(lens):
        k, _ = c.cache(r, 0)
        off = []
        seen = O.seen_tree(L, T, masks[r]) if masks else O.seen_sink(L, T, 2, 90)
        want = O.mass(q[r], k, lse[r], seen, before[0, r, :, :L], 0.5, off)
        none = np.zeros(L, bool)
        for at, _ in bad.get(r, []):
            none[at * P:(at + 1) * P] = True
        np.testing.assert_array_equal(got[0, r, :, :L][:, none], before[0, r, :, :L][:, none], err_msg=str(r))
        assert np.all((np.abs(got[0, r, :, :L] - want) <= off[0])[:, ~none]), r
        np.testing.assert_array_equal(got[0, r, :, L:], before[0, r, :, L:])
    c.st.close()


@pytest.mark.parametrize("n_pages", [30, 300, 9000])
def test_a_page_that_is_none_is_reported_by_a_choice_that_passes_it_over(n_pages):
    """It scores 0: the queries take others, and the outputs are theirs."""
    P, bad = 16, [3, n_pages // 2, n_pages - 4]
    c = filled([n_pages * P], P=P, heads=4, kv_heads=2)
    bounds = bounded(c)
    qs = queries(c, 1, 1)
    chosen = [torch.full((1, 1, 2, 9), -5, dtype=torch.int32, device="cuda") for _ in range(2)]
    ws = sk.sparse_workspace(c.st, c.pages, 1, 1, 9)
    sk.sparse_attention(c.st, c.pages, 0, qs, bounds, 1, 2, 9, ws, chosen_out=chosen[0])
    sk.check_device_error(c.st)
    assert not set(bad) & set(chosen[0].flatten().tolist())      # (bounds of normal keys score above 0)
    clean = qs.o.clone(), qs.lse.clone()
    for at, x in zip(bad, (-1, len(c.ref.refs), 1 << 30)):
        for number in (x, int(c.ref.table[0, at])):
            c.pages.table[0, at] = number
            for y in (qs.o, qs.lse):
                y.fill_(9.0)
            sk.sparse_attention(c.st, c.pages, 0, qs, bounds, 1, 2, 9, ws, chosen_out=chosen[1])
            torch.cuda.synchronize()
            assert sk.device_error_status(c.st) == (sk.ERR_DEVICE if number == x else sk.OK), (at, x)
            assert torch.equal(chosen[0], chosen[1]) and torch.equal(clean[0], qs.o) and torch.equal(clean[1], qs.lse)
    c.st.close()


def test_a_page_that_is_none_and_is_taken_counts_as_zeros():
    """As in the attention over whole rows."""
    P = 16
    c = filled([20 * P - 5], P=P, heads=4, kv_heads=2)
    bounds = bounded(c)
    page = int(c.ref.table[0, 0])
    c.ref.k[:, page], c.ref.v[:, page] = 0, 0
    c.pages.table[0, 0] = -7
    qs = queries(c, 1, 1)
    chosen = torch.full((1, 1, 2, 6), -5, dtype=torch.int32, device="cuda")
    ws = sk.sparse_workspace(c.st, c.pages, 1, 1, 6)
    sk.sparse_attention(c.st, c.pages, 0, qs, bounds, 1, 1, 6, ws, chosen_out=chosen)
    torch.cuda.synchronize()
    assert sk.device_error_status(c.st) == sk.ERR_DEVICE
    k, v = c.cache(0, 0)
    o, lse, q = qs.o.float().cpu().numpy(), qs.lse.cpu().numpy(), qs.q.float().cpu().numpy()
    for g in range(2):
        take = chosen[0, 0, g].tolist()
        assert take[0] == 0 and take[-1] == 19
        seen = np.zeros((1, 20 * P - 5), bool)
        for j in take:
            seen[0, j * P:(j + 1) * P] = True
        h = slice(2 * g, 2 * g + 2)
        PH.check_attention(o[0, :, h], lse[0, :, h], q[0, :, h], k[g:g + 1], v[g:g + 1], seen)
    c.st.close()
