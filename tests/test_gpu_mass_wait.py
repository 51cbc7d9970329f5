"""A mass call whose waits run out: a long chunk of a prompt, whose keys stay while hundreds of query blocks pass, under a
limit that this takes longer than.  Every wait ends, the status says so, and no token's mass is anything but what it was
or what the call makes of it."""
import time

import numpy as np
import pytest
import torch

from paper_2606_01790_gb300 import starkv as sk

import paged_harness as PH

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

from test_gpu_paged_attention import built  # noqa: E402,F401


def test_masses_of_a_call_whose_waits_run_out():
    n, T, H, G, P = 8, 10000, 64, 8, 256
    st = PH.state(layers=1, heads=H, kv_heads=G)
    m = -(-T // P)
    rng = np.random.default_rng(0)
    k = torch.from_numpy(rng.standard_normal((1, m, G, P, PH.D), dtype=np.float32)).to(torch.bfloat16).cuda()
    i32 = dict(dtype=torch.int32, device="cuda")
    pages = sk.Pages(k=k, v=torch.zeros_like(k), table=torch.arange(m, **i32).expand(n, m).contiguous(),
                     len=torch.full((n,), T, **i32), refs=torch.full((m,), n, **i32))
    q = torch.from_numpy(rng.standard_normal((1, 1, H, PH.D), dtype=np.float32)).to(torch.bfloat16).cuda().expand(n, T, H, PH.D)
    qs = sk.Queries(q=q, lse=torch.full((n, T, H), 3.0, device="cuda"))
    before = torch.from_numpy(rng.exponential(size=(1, n, G, m * P)).astype(np.float32)).cuda()
    mass = sk.Mass(before.clone(), 0.5)
    ws = sk.pages_workspace(st, pages, n, T)
    sk.sink_mass(st, pages, 0, qs, 0, 1 << 20, mass, ws)
    sk.check_device_error(st)
    after = mass.data.clone()
    assert bool(torch.isfinite(after).all())

    mass.data.copy_(before)
    ws.fill_(0xFF)                       # (parts that the call does not write are NaN)
    sk.set_wait_limit(st, 1)
    t0 = time.perf_counter()
    sk.sink_mass(st, pages, 0, qs, 0, 1 << 20, mass, ws)
    torch.cuda.synchronize()
    took = time.perf_counter() - t0
    assert sk.device_error_status(st) == sk.ERR_TIMEOUT
    assert took < 6                      # (the copies in flight at the end of a CTA are waited for, 2 s at most)
    was, new = mass.data == before, mass.data == after
    assert bool((was | new).all()), int((~(was | new)).sum())
    assert not bool(new.all())

    sk.set_wait_limit(st, 1_000_000_000)
    mass.data.copy_(before)
    sk.sink_mass(st, pages, 0, qs, 0, 1 << 20, mass, ws)
    sk.check_device_error(st)
    assert torch.equal(mass.data, after)
    st.close()
