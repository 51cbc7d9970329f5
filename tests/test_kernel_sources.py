"""Rules of the CUDA sources that no run can show to be broken without hanging a GPU:
read from the text.  CPU only."""
import re
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parents[1] / "paper_2606_01790_gb300" / "csrc"


def functions(name):
    """{function: body without comments} of the functions of a source file whose
    brace opens on the line of their closing parenthesis."""
    text = re.sub(r"//[^\n]*", "", (CSRC / name).read_text())
    out = {}
    for m in re.finditer(r"^[^\n;{}=]*?\b(\w+)\((?:[^(){};]|\([^()]*\))*\)\s*\{", text, flags=re.M):
        if m.group(1) in ("if", "for", "while", "switch"):
            continue
        depth, i = 1, m.end()
        while depth:
            depth += {"{": 1, "}": -1}.get(text[i], 0)
            i += 1
        out[m.group(1)] = text[m.end():i - 1]
    return out


@pytest.mark.parametrize("helper", ["cluster_sync", "cluster_arrive", "cluster_wait", "named_bar_sync", "tmem_dealloc"])
def test_barriers_that_want_a_converged_warp_converge_it(helper):
    """An aligned barrier has no time limit: reached by a diverged warp it may
    never complete.  Callers have per-lane branches right before these."""
    body = functions("ptx.cuh")[helper]
    assert "__syncwarp();" in body and body.index("__syncwarp();") < body.index("asm")


def test_no_other_source_issues_such_a_barrier_itself():
    for path in sorted(CSRC.glob("*.cu*")):
        if path.name != "ptx.cuh":
            assert not re.search(r'"[^"]*(barrier\.cluster|bar\.sync|tcgen05\.dealloc)', path.read_text()), path.name


@pytest.mark.parametrize("role", ["mma_s_loop", "mma_pv_loop", "softmax_unit", "softmax_loop", "convert_loop"])
def test_warp_wide_attention_roles_leave_together(role):
    """Lanes that read another role's failure flag one by one may disagree, and those
    that stay then wait for the others in the next warp vote for ever.  These
    roles learn of a failure only through warp_wait's vote, at every wait; the
    final wait for their own products is the one that goes on regardless."""
    body = functions("attn.cu")[role]
    assert "abort" not in body
    assert "warp_wait(" in body
    assert re.findall(r"\bmbar_wait\(([^,]*),", body) == (["&ctl->drain"] if role.startswith("mma") else [])


def test_every_attention_wait_sees_another_roles_failure():
    body = functions("attn.cu")["warp_wait"]
    assert body.index("ctl->abort") < body.index("__all_sync(") < body.index("mbar_wait(")


@pytest.mark.parametrize("source,role", [("score.cu", "producer_loop"), ("attn.cu", "k_loader"), ("attn.cu", "v_loader")])
def test_loaders_see_every_copy_land(source, role):
    """A loader that is past its last load when another role gives up still keeps
    the block until its copies are in: they would land in another block's shared
    memory.  The waits for them stand at the function's top level."""
    body = functions(source)[role]
    depth, found = 0, []
    for line in body.split("\n"):
        if "drain_limit(" in line:
            found.append((depth, line))
        depth += line.count("{") - line.count("}")
    assert found and all(d == 0 for d, _ in found)
    assert not re.search(r"if \(ctl->abort\)\s*\{?\s*for", body)


@pytest.mark.parametrize("role", ["load_loop", "mma_s_loop", "mma_pv_loop", "softmax_unit", "softmax_loop"])
def test_warp_wide_paged_attention_roles_leave_together(role):
    """As in the window attention: these roles learn of a failure through a vote only, and wait on regardless
    for nothing but their own products and copies."""
    body = functions("paged_attn.cu")[role]
    assert "abort" not in body
    assert "warp_wait(" in body
    alone = [w for w in re.findall(r"\bmbar_wait\(([^,]*),", body)]
    assert alone == {"load_loop": ["&full[i]"], "mma_s_loop": ["&ctl->drain"], "mma_pv_loop": ["&ctl->drain"]}.get(role, [])


def test_paged_attention_asks_two_barriers_at_once_only_where_either_order_is_right():
    """A parity cannot tell a phase from the one two before it, and two questions may be answered in either
    order: only barriers whose previous phase the asking warp has waited for itself may share a vote.  The loader's
    and the softmax's (rings that the products go round) do; a piece's end asks one after the other."""
    f = functions("paged_attn.cu")
    assert {name for name, body in f.items() if "warp_wait2(" in body} == {"mma_s_loop", "mma_pv_loop"}
    assert "warp_wait2" not in f["softmax_loop"] and f["softmax_loop"].count("ml_full, pc & 1, p.wait_ns) && warp_wait(") == 1
    loop = f["softmax_loop"]
    assert loop.index("p_empty[before % kPlaces]") < loop.index("v_full[stage]") < loop.index("v4[x] =")


def test_the_paged_loader_sees_every_copy_land():
    body = functions("paged_attn.cu")["load_loop"]
    depth, found = 0, []
    for line in body.split("\n"):
        if "drain_limit(" in line:
            found.append(depth)
        depth += line.count("{") - line.count("}")
    assert found == [0]


def test_page_bookkeeping_writes_to_peers_only_once_all_of_them_run():
    """A peer's shared memory may be written once that CTA is known to have started, which only a cluster barrier
    shows: every thread arrives before the call's first reads and waits before the first such write."""
    body = functions("pages.cu")["k_book"]
    first = body.index("dsmem_")
    arrive, wait = body.index("cluster_arrive();"), body.index("cluster_wait();")
    assert arrive < body.index("griddep_wait();") < wait < first < body.index("cluster_sync();")
    assert body.count("cluster_arrive();") == body.count("cluster_wait();") == 1
    assert "return" not in body[arrive:wait]
