"""Evictions of rows that are longer than what a block keeps of its keys: what moves with the tokens."""
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
from test_gpu_paged_attention import built  # noqa: E402,F401


@pytest.mark.parametrize("per_head", [False, True])
@pytest.mark.parametrize("kind", ["spread", "ties"])
@pytest.mark.parametrize("L,budget", [(60003, 100), (60003, 59000), (150001, 60000)])
def test_masses_of_a_long_row_move_with_its_tokens(per_head, kind, L, budget):
    window, P, layers = 8, 256, 2
    st = PH.state(layers=layers, heads=4, kv_heads=2, window=window, select_mode=int(per_head))
    m, kept = -(-L // P), -(-(budget + window) // P)
    c = PH.Pair(st, n_pages=m + 2 + kept, P=P, n_rows=2, max_pages=m)
    c.extend([1, 0], [L, 300])
    data, mass = make_mass(c, 1.0, seed=budget)
    if kind == "ties":
        data[:] = np.round(data * 8) / 8
    mass.data.copy_(torch.from_numpy(data))
    n = 2 if per_head else 1
    idx = torch.full((layers, n, budget), -7, dtype=torch.int32, device="cuda")
    sk.pages_evict(st, c.pages, c.ids([1]), [sk.Seq(L=L, budget=budget, idx=idx)], mass, c.ws)
    past = data[:, 1, :, :L - window].astype(np.float64)
    x = past if per_head else past.sum(1, keepdims=True)
    keep = np.stack([[O.heaviest(r, budget) for r in y] for y in x])
    np.testing.assert_array_equal(idx.cpu().numpy(), keep)
    at = np.concatenate([keep, np.broadcast_to(np.arange(L - window, L), (layers, n, window))], -1)
    want = data.copy()
    want[:, 1, :, :budget + window] = np.take_along_axis(data[:, 1], np.broadcast_to(at, (layers, 2, budget + window)), -1)
    np.testing.assert_array_equal(mass.data.cpu().numpy(), want)
    c.ref.compact([1], [L], [keep], window)
    c.check()
    st.close()
