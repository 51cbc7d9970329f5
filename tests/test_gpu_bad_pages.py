"""Page numbers that are none in a table's rows: what the calls that weigh tokens do with them."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from paper_2606_01790_gb300 import starkv as sk

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

from test_gpu_mass import make_mass  # noqa: E402
from test_gpu_paged_attention import built, filled, queries, random_tree, words  # noqa: E402,F401


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
