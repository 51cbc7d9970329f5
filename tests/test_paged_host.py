"""The paged cache without a GPU: struct layouts, checks of arguments on the host,
and pins of the definition that the GPU tests compare with."""
import ctypes
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


def test_struct_layouts_match_the_header(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    structs = [("starkv_pages", sk.CPages), ("starkv_tokens", sk.CTokens), ("starkv_queries", sk.CQueries)]
    lines = []
    for name, c in structs:
        lines.append(f'  printf("%zu\\n", sizeof({name}));')
        lines += [f'  printf("%zu\\n", offsetof({name}, {f[0]}));' for f in c._fields_]
    lines.append('  printf("%d\\n", (int)STARKV_NUM_KERNELS);')
    src = tmp_path / "probe.c"
    src.write_text('#include <stdio.h>\n#include "starkv.h"\nint main(void) {\n' + "\n".join(lines) + "\n  return 0;\n}\n")
    exe = tmp_path / "probe"
    subprocess.run([cc, "-std=c99", "-Wall", "-Werror", f"-I{ROOT / 'include'}", str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    want = []
    for _, c in structs:
        want.append(ctypes.sizeof(c))
        want += [getattr(c, f[0]).offset for f in c._fields_]
    assert got == want + [len(sk.KERNELS)]


def test_calls_without_a_state_or_pages_are_refused(library):
    pg, tok, qs, n = sk.CPages(), sk.CTokens(), sk.CQueries(), ctypes.c_size_t(0)
    calls = [
        library.starkv_pages_workspace_bytes(None, ctypes.byref(pg), 1, 1, ctypes.byref(n)),
        library.starkv_pages_reset(None, ctypes.byref(pg), None),
        library.starkv_pages_extend(None, ctypes.byref(pg), None, None, 1, None, 0, None),
        library.starkv_pages_fork(None, ctypes.byref(pg), None, None, 1, 0, None, 0, None),
        library.starkv_pages_free(None, ctypes.byref(pg), None, 1, None),
        library.starkv_pages_compact(None, ctypes.byref(pg), None, None, 1, None, 0, None),
        library.starkv_pages_store(None, ctypes.byref(pg), 0, 1, ctypes.byref(tok), None),
        library.starkv_pages_load(None, ctypes.byref(pg), 0, 1, ctypes.byref(tok), None),
        library.starkv_tree_attention(None, ctypes.byref(pg), 0, ctypes.byref(qs), None, 0, None),
        library.starkv_sink_attention(None, ctypes.byref(pg), 0, ctypes.byref(qs), 0, 1, None, 0, None),
    ]
    assert all(c == sk.ERR_INVALID_ARG for c in calls)


class _State:     # what the binding reads of a state
    cfg = sk.Config(n_layers=2, n_heads=8, n_kv_heads=4)
    handle = None


def _pages(**over):
    a = dict(k=torch.zeros((2, 5, 4, 16, 128), dtype=torch.bfloat16), table=torch.zeros((3, 4), dtype=torch.int32),
             len=torch.zeros(3, dtype=torch.int32), refs=torch.zeros(5, dtype=torch.int32))
    a["v"] = torch.zeros_like(a["k"])
    a.update(over)
    return sk.Pages(**a)


@pytest.mark.parametrize("over", [
    dict(k=torch.zeros((2, 5, 4, 16, 128))), dict(v=torch.zeros((2, 5, 4, 32, 128), dtype=torch.bfloat16)),
    dict(v=torch.zeros((5, 2, 4, 16, 128), dtype=torch.bfloat16).transpose(0, 1)),
    dict(table=torch.zeros((3, 4), dtype=torch.int64)), dict(table=torch.zeros(12, dtype=torch.int32)),
    dict(table=torch.zeros((4, 3), dtype=torch.int32).t()), dict(len=torch.zeros(4, dtype=torch.int32)),
    dict(refs=torch.zeros(6, dtype=torch.int32)), dict(refs=torch.zeros(5))])
def test_the_binding_checks_a_pool(over):
    _pages().to_c()
    with pytest.raises(ValueError):
        _pages(**over).to_c()


def test_the_binding_checks_the_tensors_of_a_call():
    st, pages = _State(), _pages()
    for call in (lambda: sk.pages_reset(st, pages),                                       # host memory
                 lambda: sk.pages_free(st, pages, torch.zeros(1, dtype=torch.int32)),
                 lambda: sk.pages_reset(st, _pages(k=torch.zeros((1, 5, 4, 16, 128), dtype=torch.bfloat16),
                                                   v=torch.zeros((1, 5, 4, 16, 128), dtype=torch.bfloat16)))):
        with pytest.raises(ValueError):
            call()
    bf = dict(dtype=torch.bfloat16)
    for bad in (sk.Tokens(k=torch.zeros((1, 2, 3, 4, 64), **bf)), sk.Tokens(k=torch.zeros((1, 2, 3, 8, 128), **bf)),
                sk.Tokens(k=torch.zeros((1, 2, 3, 128, 4), **bf).transpose(3, 4)),
                sk.Tokens(k=torch.zeros((1, 2, 3, 4, 128))),
                sk.Tokens(k=torch.zeros((1, 2, 3, 4, 128), **bf), v=torch.zeros((1, 2, 4, 3, 128), **bf).transpose(2, 3))):
        with pytest.raises(ValueError):
            sk._c_tokens(st, pages, bad)
    q = torch.zeros((2, 3, 8, 128), **bf)
    for bad in (sk.Queries(q=q, o=q[:1]), sk.Queries(q=q.float(), o=q), sk.Queries(q=q[:, :, :4], o=q[:, :, :4]),
                sk.Queries(q=q, o=torch.zeros((2, 3, 8, 256), **bf)[..., ::2])):
        with pytest.raises(ValueError):
            sk._c_queries(st, pages, bad)


def test_packed_calls_equal_the_ctypes_structs(monkeypatch):
    st, pages = _State(), _pages()
    monkeypatch.setattr(sk, "_on", lambda *a: None)
    bf, i32 = dict(dtype=torch.bfloat16), dict(dtype=torch.int32)
    k, rows, n = torch.zeros((3, 2, 5, 4, 128), **bf), torch.zeros(3, **i32), torch.ones(3, **i32)
    want = sk.CTokens(k.data_ptr(), 0, rows.data_ptr(), n.data_ptr(), 3, 5, *k.stride()[:4])
    assert sk._c_tokens(st, pages, sk.Tokens(k=k, rows=rows, n_tokens=n)) == bytes(want)
    q, o = torch.zeros((5, 3, 8, 128), **bf).transpose(0, 1), torch.zeros((3, 5, 8, 128), **bf)
    lse, mask = torch.zeros((3, 5, 8)), torch.zeros((3, 5), dtype=torch.int64)
    want = sk.CQueries(q.data_ptr(), o.data_ptr(), lse.data_ptr(), mask.data_ptr(), rows.data_ptr(), 0, 3, 5, *q.stride()[:3],
                       *o.stride()[:3])
    assert sk._c_queries(st, pages, sk.Queries(q=q, o=o, lse=lse, mask=mask, rows=rows)) == bytes(want)
    # an axis of one entry is never stepped along, whatever its stride
    x = torch.empty_strided((1, 1, 8, 128), (7, 5, 256, 1), **bf)
    got = sk.CQueries.from_buffer_copy(sk._c_queries(st, pages, sk.Queries(q=x, o=x)))
    assert (got.q_seq_stride, got.q_token_stride, got.q_head_stride) == (128, 128, 256)
    with pytest.raises(AttributeError):      # a pool's tensors are checked once, and stay its own
        pages.k = k


def test_the_definition_of_attention_against_torch():
    rng = np.random.default_rng(0)
    q, k, v = rng.standard_normal((5, 6, 16)), rng.standard_normal((2, 40, 16)), rng.standard_normal((2, 40, 16))
    seen = O.seen_sink(40, 5, 3, 9)
    o, lse = O.attention(q, k, v, seen)
    tq, tk, tv = (torch.from_numpy(x) for x in (q, k, v))
    z = torch.einsum("thd,hjd->htj", tq, tk.repeat_interleave(3, 0)) / 4
    z = z.masked_fill(~torch.from_numpy(seen), -torch.inf)
    np.testing.assert_allclose(lse, torch.logsumexp(z, -1).T.numpy(), rtol=1e-13)
    np.testing.assert_allclose(o, torch.einsum("htj,hjd->thd", z.softmax(-1), tv.repeat_interleave(3, 0)).numpy(), rtol=1e-11, atol=1e-13)


def test_what_queries_see():
    assert O.seen_sink(6, 2, 1, 2).astype(int).tolist() == [[1, 0, 0, 1, 1, 0], [1, 0, 0, 0, 1, 1]]
    assert O.seen_sink(3, 3, 0, 9).astype(int).tolist() == [[1, 0, 0], [1, 1, 0], [1, 1, 1]]
    assert O.seen_tree(4, 2, [0b01, 0b10]).astype(int).tolist() == [[1, 1, 1, 0], [1, 1, 0, 1]]
    assert O.seen_tree(2, 2, [0, 0b111]).astype(int).tolist() == [[0, 0], [1, 1]]


def test_the_definition_of_the_pool():
    kv = [np.arange(2 * 6 * 1 * 4 * 3, dtype=np.int64).reshape(2, 6, 1, 4, 3) + 1000 * i for i in range(2)]
    p = O.Pool(kv[0], kv[1], np.zeros((4, 4), int), np.zeros(4, int), np.zeros(6, int))
    p.extend([1], [6])
    assert p.table[1, :2].tolist() == [0, 1] and p.refs.tolist() == [1, 1, 0, 0, 0, 0]
    p.fork([1], [0])
    assert p.refs.tolist() == [2, 2, 0, 0, 0, 0] and p.len.tolist() == [6, 6, 0, 0]
    before = p.k.copy()
    p.extend([0, 1], [1, 0])       # row 0 copies the shared page's two filled slots; row 1 needs nothing
    assert p.table[0, :2].tolist() == [0, 2] and p.refs.tolist() == [2, 1, 1, 0, 0, 0]
    assert np.array_equal(p.k[:, 2, :, :2], before[:, 1, :, :2]) and np.array_equal(p.k[:, 2, :, 2:], before[:, 2, :, 2:])
    rows = p.tokens(0, 1, p.k).copy()
    p.compact([0], [7], [np.array([[[1, 4]], [[0, 2]]])], 2)
    assert p.table[0, :1].tolist() == [3] and p.refs.tolist() == [1, 1, 0, 1, 0, 0]
    assert np.array_equal(p.tokens(0, 1, p.k), rows[:, [0, 2, 5, 6]])
    with pytest.raises(O.PoolError):
        p.extend([2, 3], [8, 8])       # three free pages
    assert p.len.tolist() == [4, 6, 0, 0]
    p.free([0, 1])
    assert p.refs.sum() == 0 and p.len.sum() == 0


def test_the_two_cpu_definitions_agree():
    """The plain forms that the performance cases are timed with, on the CPU, against the loops of the oracle."""
    import importlib.util
    spec = importlib.util.spec_from_file_location("operators_cpu", ROOT / "perf" / "operators.py")
    M = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(M)
    M.DEV = "cpu"
    c = M._case("x", "fork", layers=2, n=5, sources=2, ctx=70, ragged=True, page=16, T=20)
    s = M.prepare(c, 1)
    p = O.Pool(s["k"].view(torch.int16).numpy().copy(), s["v"].view(torch.int16).numpy().copy(), s["table"].numpy().copy(),
               s["len"].numpy().copy(), s["refs"].numpy().copy())
    M.run(s)
    p.fork(s["src"].tolist(), s["dst"].tolist())
    p.extend(s["dst"].tolist(), s["n_new"].tolist())
    for a, b in ((s["table"], p.table), (s["len"], p.len), (s["refs"], p.refs), (s["k"].view(torch.int16), p.k)):
        np.testing.assert_array_equal(a.numpy(), b)
    c = M._case("x", "tree", heads=8, n=2, ctx=40, page=16, T=9, ragged=True)
    s = M.prepare(c, 2)
    got = M.run(s)
    for i, (r, n) in enumerate(zip(s["rows"].tolist(), s["n_tokens"].tolist())):
        L = int(s["len"][r])
        at = np.arange(L)
        k, v = (x[1].float().numpy()[s["table"].numpy()[r, at // 16], :, at % 16].swapaxes(0, 1) for x in (s["k"], s["v"]))
        o, lse = O.attention(s["q"][i, :n].float().numpy(), k, v, O.seen_tree(L, n, s["mask"][i].tolist()))
        np.testing.assert_allclose(got["lse"][i, :n].numpy(), lse, rtol=2e-6)
        np.testing.assert_allclose(got["o"][i, :n].float().numpy(), o, rtol=2**-7, atol=1e-5)


@pytest.mark.parametrize("over,what", [
    (dict(idx=torch.zeros((2, 1, 3), dtype=torch.int64)), "idx"), (dict(idx=torch.zeros((1, 1, 3), dtype=torch.int32)), "idx"),
    (dict(idx=torch.zeros((2, 1, 4), dtype=torch.int32)), "idx"), (dict(idx=torch.zeros((2, 1, 3))), "idx"),
    (dict(meta_out=torch.zeros((2, 1, 10), dtype=torch.int32)), "meta_out"), (dict(meta_out=torch.zeros(21, dtype=torch.int32)), "meta_out"),
    (dict(meta_out=torch.zeros((2, 1, 11), dtype=torch.int64)), "meta_out"), (dict(meta=torch.zeros(39, dtype=torch.int32)), "meta"),
    (dict(meta=torch.zeros(79, dtype=torch.int32), meta_layer_stride=40), "meta"), (dict(meta=torch.zeros(40, dtype=torch.int64)), "meta")],
    ids=lambda x: x if isinstance(x, str) else str(tuple(next(iter(x.values())).shape)))
def test_the_binding_checks_what_a_compaction_keeps(over, what):
    """idx as 64-bit words would be read as pairs of 32-bit ones, and a short meta_out be written past its end."""
    st, pages = _State(), _pages()
    st.cfg = sk.Config(n_layers=2, n_heads=8, n_kv_heads=4, window=8)
    seq = dict(L=40, budget=3, idx=torch.zeros((2, 1, 3), dtype=torch.int32), meta=torch.zeros(40, dtype=torch.int32),
               meta_out=torch.zeros((2, 1, 11), dtype=torch.int32))
    ws = torch.zeros(256, dtype=torch.uint8)
    with pytest.raises(ValueError, match="pages on cpu"):     # all is well with it but the device
        sk.pages_compact(st, pages, None, [sk.Seq(**seq)], ws)
    with pytest.raises(ValueError, match=f"seq 1: {what}"):
        sk.pages_compact(st, pages, None, [sk.Seq(**seq), sk.Seq(**{**seq, **over})], ws)


def test_the_binding_refuses_a_workspace_that_is_not_what_it_says():
    """An expanded tensor has more elements than bytes behind it."""
    st, pages = _State(), _pages()
    ws, ids = torch.zeros(1, dtype=torch.uint8).expand(1 << 30), torch.zeros(2, dtype=torch.int32)
    q = torch.zeros((1, 1, 8, 128), dtype=torch.bfloat16)
    qs = sk.Queries(q=q, o=torch.zeros_like(q), mask=torch.zeros((1, 1), dtype=torch.int64))
    for call in (lambda: sk.pages_extend(st, pages, None, ids, ws), lambda: sk.pages_fork(st, pages, ids, ids, ws),
                 lambda: sk.pages_compact(st, pages, None, [sk.Seq(L=40)], ws), lambda: sk.tree_attention(st, pages, 0, qs, ws),
                 lambda: sk.sink_attention(st, pages, 0, qs, 1, 1, ws)):
        with pytest.raises(ValueError, match="contiguous"):
            call()
