"""Attention mass, eviction, page bounds and chosen pages without a GPU: struct layouts, checks of arguments, and pins of
the definitions that the GPU tests compare with."""
import ctypes
import importlib.util
import shutil
import subprocess
from pathlib import Path

import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from paper_2606_01790_gb300 import build as B
from paper_2606_01790_gb300 import starkv as sk

ROOT = Path(__file__).resolve().parents[1]


@pytest.fixture(scope="module")
def library():
    B.build()
    return sk.lib()


class _State:     # what the binding reads of a state
    cfg = sk.Config(n_layers=2, n_heads=8, n_kv_heads=4)
    handle = None


def _pages():
    k = torch.zeros((2, 5, 4, 16, 128), dtype=torch.bfloat16)
    i32 = dict(dtype=torch.int32)
    return sk.Pages(k=k, v=torch.zeros_like(k), table=torch.zeros((3, 4), **i32), len=torch.zeros(3, **i32), refs=torch.zeros(5, **i32))


def test_struct_layouts_match_the_header(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    structs = [("starkv_mass", sk.CMass), ("starkv_bounds", sk.CBounds)]
    lines = []
    for name, c in structs:
        lines.append(f'  printf("%zu\\n", sizeof({name}));')
        lines += [f'  printf("%zu\\n", offsetof({name}, {f[0]}));' for f in c._fields_]
    src = tmp_path / "probe.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "starkv.h"\nint main(void) {\n' + "\n".join(lines) + "\n  return 0;\n}\n")
    exe = tmp_path / "probe"
    subprocess.run([cc, "-std=c99", "-Wall", "-Werror", f"-I{ROOT / 'include'}", str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    want = []
    for _, c in structs:
        want.append(ctypes.sizeof(c))
        want += [getattr(c, f[0]).offset for f in c._fields_]
    assert got == want


def test_calls_without_a_state_are_refused(library):
    pg, qs, m, b, n = sk.CPages(), sk.CQueries(), sk.CMass(), sk.CBounds(), ctypes.c_size_t(0)
    r = ctypes.byref
    calls = [
        library.starkv_tree_mass(None, r(pg), 0, r(qs), r(m), None, 0, None),
        library.starkv_sink_mass(None, r(pg), 0, r(qs), 0, 1, r(m), None, 0, None),
        library.starkv_pages_evict(None, r(pg), None, None, 1, r(m), None, 0, None),
        library.starkv_pages_bounds(None, r(pg), 0, 1, r(b), None, None, 1, 1, None),
        library.starkv_sparse_workspace_bytes(None, r(pg), 1, 1, 1, r(n)),
        library.starkv_sparse_attention(None, r(pg), 0, r(qs), r(b), 0, 1, 1, None, None, 0, None),
    ]
    assert all(c == sk.ERR_INVALID_ARG for c in calls)


@pytest.mark.parametrize("data", [
    torch.zeros((2, 3, 4, 64), dtype=torch.float64), torch.zeros((2, 3, 4)), torch.zeros((2, 3, 4, 128))[..., ::2],
    torch.zeros((1, 3, 4, 64)), torch.zeros((2, 2, 4, 64)), torch.zeros((2, 3, 8, 64)), torch.zeros((2, 3, 4, 63))],
    ids=lambda t: f"{tuple(t.shape)}-{t.dtype}")
def test_the_binding_checks_a_mass(data):
    st, pages = _State(), _pages()
    sk._c_mass(st, pages, sk.Mass(torch.zeros((2, 3, 4, 70)), 0.5))
    with pytest.raises(ValueError):
        sk._c_mass(st, pages, sk.Mass(data))


@pytest.mark.parametrize("bounds", [
    torch.zeros((2, 5, 4, 2, 128)), torch.zeros((2, 5, 4, 128), dtype=torch.bfloat16),
    torch.zeros((2, 4, 4, 2, 128), dtype=torch.bfloat16), torch.zeros((2, 5, 2, 4, 128), dtype=torch.bfloat16).transpose(2, 3)],
    ids=lambda t: f"{tuple(t.shape)}-{t.dtype}")
def test_the_binding_checks_bounds(bounds):
    st, pages = _State(), _pages()
    sk._c_bounds(st, pages, torch.zeros((5, 2, 4, 2, 128), dtype=torch.bfloat16).transpose(0, 1))
    with pytest.raises(ValueError):
        sk._c_bounds(st, pages, bounds)


def test_the_binding_checks_the_tensors_of_a_call():
    st, pages = _State(), _pages()
    q, mass = torch.zeros((2, 3, 8, 128), dtype=torch.bfloat16), sk.Mass(torch.zeros((2, 3, 4, 64)))
    bounds, ws = torch.zeros((2, 5, 4, 2, 128), dtype=torch.bfloat16), torch.zeros(256, dtype=torch.uint8)
    lse = torch.zeros((2, 3, 8))
    for call in (lambda: sk.sink_mass(st, pages, 0, sk.Queries(q=q), 0, 1, mass, ws),                    # no normalisers
                 lambda: sk.tree_mass(st, pages, 0, sk.Queries(q=q, lse=lse[:1]), mass, ws),
                 lambda: sk.sink_mass(st, pages, 0, sk.Queries(q=q, lse=lse.double()), 0, 1, mass, ws),
                 lambda: sk.sparse_attention(st, pages, 0, sk.Queries(q=q), bounds, 0, 1, 2, ws),       # no o
                 lambda: sk.sparse_attention(st, pages, 0, sk.Queries(q=q, o=q.clone()), bounds, 0, 1, 2, ws,
                                             chosen_out=torch.zeros((2, 3, 4, 3), dtype=torch.int32)),
                 lambda: sk.sparse_attention(st, pages, 0, sk.Queries(q=q, o=q.clone()), bounds, 0, 1, 2, ws,
                                             chosen_out=torch.zeros((2, 3, 4, 2), dtype=torch.int64)),
                 lambda: sk.pages_bounds(st, pages, 0, 1, bounds, 4, rows=torch.zeros(2, dtype=torch.int64)),
                 lambda: sk.pages_bounds(st, pages, 0, 1, bounds, 4, rows=torch.zeros(2, dtype=torch.int32),
                                         n_tokens=torch.zeros(3, dtype=torch.int32)),
                 lambda: sk.pages_bounds(st, pages, 0, 1, bounds, 4)):                                   # host memory
        with pytest.raises(ValueError):
            call()
    st.cfg = sk.Config(n_layers=2, n_heads=8, n_kv_heads=4, window=8)
    with pytest.raises(ValueError, match="seq 0: idx"):
        sk.pages_evict(st, pages, None, [sk.Seq(L=40, budget=3, idx=torch.zeros((2, 1, 3), dtype=torch.int64))], mass, ws)


def test_a_mass_call_packs_queries_without_an_output(monkeypatch):
    st, pages = _State(), _pages()
    monkeypatch.setattr(sk, "_on", lambda *a: None)
    q, lse = torch.zeros((5, 2, 8, 128), dtype=torch.bfloat16).transpose(0, 1), torch.zeros((2, 5, 8))
    got = sk.CQueries.from_buffer_copy(sk._c_queries(st, pages, sk.Queries(q=q, lse=lse), True))
    assert (got.q, got.lse, got.n, got.T, got.q_seq_stride, got.q_token_stride) == (q.data_ptr(), lse.data_ptr(), 2, 5, *q.stride()[:2])


def test_the_definition_of_mass_against_softmax():
    """The weights of a query add up to 1 per head, over what it sees."""
    rng = np.random.default_rng(0)
    q, k = rng.standard_normal((5, 6, 16)), rng.standard_normal((2, 40, 16))
    seen = O.seen_sink(40, 5, 3, 9)
    _, lse = O.attention(q, k, k, seen)
    had = rng.random((2, 40))
    m = O.mass(q, k, lse, seen, had, 0.5)
    z = torch.einsum("thd,hjd->thj", torch.from_numpy(q), torch.from_numpy(k).repeat_interleave(3, 0)) / 4
    p = z.masked_fill(~torch.from_numpy(seen)[:, None], -torch.inf).softmax(-1).view(5, 2, 3, 40).sum((0, 2)).numpy()
    had[:, 35:] = 0
    np.testing.assert_allclose(m, 0.5 * had + p, rtol=1e-12, atol=1e-14)
    assert abs((m - 0.5 * had).sum() - 30) < 1e-10


def test_the_definitions_of_the_choices():
    assert O.heaviest(np.array([1, 3, 2, 3, np.nan, 3, 0]), 3).tolist() == [1, 3, 4]
    assert O.heaviest(np.array([np.inf, np.nan, 1]), 1).tolist() == [0]
    rng = np.random.default_rng(1)
    q, k = rng.standard_normal((4, 8)), rng.standard_normal((6, 16, 8))
    s = O.page_scores(q, k.min(1), k.max(1))
    assert np.all(s >= (k @ q.sum(0)).max(1))      # no key's logits add up to more
    assert O.choose_pages([5, 1, 7, 7, 2, 0], 1, 1, 4) == [0, 2, 3, 5]
    assert O.choose_pages([5, 1, 7, 7, 2, 0], 0, 1, 2) == [2, 5]
    assert O.choose_pages([5, 1, np.nan], 1, 1, 3) == [0, 1, 2]


def test_the_two_cpu_definitions_agree():
    """The plain forms that the performance cases are timed with, on the CPU, against the loops of the oracle."""
    spec = importlib.util.spec_from_file_location("more_operators_cpu", ROOT / "perf" / "more_operators.py")
    M = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(M)
    M.DEV = "cpu"

    def cache(s, r, layer=1):
        L, P = int(s["len"][r]), s["page"]
        at = np.arange(L)
        return [x[layer].float().numpy()[s["table"].numpy()[r, at // P], :, at % P].swapaxes(0, 1) for x in (s["k"], s["v"])]

    for c in (M._case("x", "mass", heads=8, n=2, ctx=60, page=16, T=5, ragged=True, tree=True, decay=0.5),
              M._case("x", "mass", heads=8, n=2, ctx=60, page=16, T=5, ragged=True, tree=False, sinks=2, window=20, decay=0.5)):
        s = M.prepare(c, 2)
        before = s["mass"].clone().numpy()
        got = M.run(s)["mass"].numpy()
        for i, (r, n) in enumerate(zip(s["rows"].tolist(), s["n_tokens"].tolist())):
            L = int(s["len"][r])
            seen = O.seen_tree(L, n, s["mask"][i].tolist()) if c["tree"] else O.seen_sink(L, n, 2, 20)
            want = O.mass(s["q"][i, :n].float().numpy(), cache(s, r)[0], s["lse"][i, :n].numpy(), seen, before[1, r, :, :L], 0.5)
            np.testing.assert_allclose(got[1, r, :, :L], want, rtol=1e-5, atol=1e-7)
            np.testing.assert_array_equal(got[1, r, :, L:], before[1, r, :, L:])
    c = M._case("x", "evict", heads=8, n=2, ctx=70, page=16, ragged=True, budget=20, window=4, per_head=False)
    s = M.prepare(c, 3)
    p = O.Pool(s["k"].view(torch.int16).numpy().copy(), s["v"].view(torch.int16).numpy().copy(), s["table"].numpy().copy(),
               s["len"].numpy().copy(), s["refs"].numpy().copy())
    mass, lens = s["mass"].numpy().copy(), s["len"][:2].tolist()
    M.run(s)
    p.fork([0, 1], [2, 3])
    keep = [np.stack([[O.heaviest(mass[l, r, :, :L - 4].astype(np.float64).sum(0), 20)] for l in range(2)]) for r, L in enumerate(lens)]
    p.compact([2, 3], lens, keep, 4)
    for a, b in ((s["table"], p.table), (s["len"], p.len), (s["refs"], p.refs), (s["k"].view(torch.int16), p.k), (s["idx"], np.stack(keep))):
        np.testing.assert_array_equal(a.numpy(), b)
    c = M._case("x", "sparse", heads=8, n=2, ctx=200, page=16, T=3, ragged=True, first=1, last=1, chosen=5)
    s = M.prepare(c, 4)
    got = M.run(s)
    b = s["bounds"].float().numpy()
    for i, (r, n) in enumerate(zip(s["rows"].tolist(), s["n_tokens"].tolist())):
        L = int(s["len"][r])
        k, v = cache(s, r)
        for t in range(n):
            pages = s["table"].numpy()[r, :(L - n + t) // 16 + 1]
            for g in range(4):
                q = s["q"][i, t, 2 * g:2 * g + 2].float().numpy()
                take = O.choose_pages(O.page_scores(q, b[1, pages, g, 0], b[1, pages, g, 1]), 1, 1, 5)
                assert got["chosen"][i, t, g].tolist() == take + [-1] * (5 - len(take))
                seen = np.zeros((1, L), bool)
                for j in take:
                    seen[0, j * 16:min(j * 16 + 16, L - n + t + 1)] = True
                o, lse = O.attention(q[None], k[g:g + 1], v[g:g + 1], seen)
                np.testing.assert_allclose(got["lse"][i, t, 2 * g:2 * g + 2].numpy(), lse[0], rtol=2e-6)
                np.testing.assert_allclose(got["o"][i, t, 2 * g:2 * g + 2].float().numpy(), o[0], rtol=2**-7, atol=1e-5)


def test_a_masss_tensor_is_checked_once_and_stays_its_own():
    m = sk.Mass(torch.zeros((2, 3, 4, 64)), 0.5)
    with pytest.raises(AttributeError):
        m.data = torch.zeros((2, 3, 4, 64))
    with pytest.raises(AttributeError):
        m.decay = 1.0
    got = sk.CMass.from_buffer_copy(sk._c_mass(_State(), _pages(), m))
    assert (got.mass, got.layer_stride, got.row_stride, got.group_stride, got.decay) == (m.data.data_ptr(), 768, 256, 64, 0.5)


@pytest.mark.parametrize("decay", [0, 0.98, float("inf"), 1e300])
def test_a_packed_mass_is_the_struct(decay):
    data = torch.zeros((2, 3, 4, 70))[:, 1:]
    c = sk.CMass.from_buffer_copy(sk.Mass(data, decay)._packed)
    assert (c.mass, c.layer_stride, c.row_stride, c.group_stride) == (data.data_ptr(), 3 * 4 * 70, 4 * 70, 70)
    assert c.decay == ctypes.c_float(decay).value      # (past 32 bits: infinity, which the calls refuse)
    one = sk.CMass.from_buffer_copy(sk.Mass(torch.zeros((1, 1, 1, 70)).expand(1, 1, 1, 70), decay)._packed)
    assert (one.layer_stride, one.row_stride, one.group_stride) == (70, 70, 70)
