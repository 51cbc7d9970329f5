"""Rules of the sources of the attention mass and the choice of pages that no run can show to be broken without
hanging a GPU: read from the text.  CPU only."""
import re

import pytest

from test_kernel_sources import functions


@pytest.mark.parametrize("role", ["key_loop", "query_loop", "mma_loop", "weigh_loop"])
def test_roles_of_the_mass_kernel_leave_together(role):
    """They learn of a failure through a vote at a wait only, and wait on regardless for nothing but their own
    products and copies."""
    body = functions("mass.cu")[role]
    assert "abort" not in body and "warp_wait(" in body
    alone = re.findall(r"\bmbar_wait\(([^,]*),", body)
    assert alone == {"key_loop": ["&ctl->k_full[i]"], "mma_loop": ["&ctl->drain"]}.get(role, [])
    assert "mbar_try_wait" not in body


def test_every_wait_of_the_mass_kernel_sees_another_roles_failure():
    body = functions("mass.cu")["warp_wait"]
    assert body.index("ctl->abort") < body.index("mbar_wait(") < body.rindex("__all_sync(")


def test_the_key_loader_sees_every_copy_land():
    body = functions("mass.cu")["key_loop"]
    depth, found = 0, []
    for line in body.split("\n"):
        if "drain_limit(" in line:
            found.append(depth)
        depth += line.count("{") - line.count("}")
    assert found == [0]


def test_queries_are_handed_over_when_they_have_landed_and_the_tensor_core_may_see_them():
    body = functions("mass.cu")["query_loop"]
    order = [body.index(x) for x in ("cp_async16(", "cp_async_wait();", "fence_proxy_async_smem();", "__syncwarp();", "mbar_arrive(&ctl->q_full")]
    assert order == sorted(order)


def test_scores_go_to_another_cta_only_once_it_is_known_to_run():
    """Every thread of the cluster arrives, waits once on either way, and meets the others again before the first
    CTA reads and the others leave."""
    body = functions("sparse.cu")["k_page_choose"]
    arrive, wait, meet = body.index("cluster_arrive();"), body.index("cluster_wait();"), body.index("cluster_sync();")
    first = body.index("dsmem_")
    assert arrive < wait < first < meet
    assert body.count("cluster_arrive();") == 1 and body.count("cluster_sync();") == 1 and body.count("cluster_wait();") == 2
    assert "return" not in re.sub(r"auto \w+ = \[&\].*?\};", "", body[arrive:meet], flags=re.S)
    assert body.rindex("dsmem_") < meet
