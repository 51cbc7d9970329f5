"""What the sum of a mass call's parts takes of CTAs that have not written theirs: read from the text, since which of
them a refusal on another stream reaches is a matter of time.  CPU only."""
from test_kernel_sources import functions


def test_a_cta_that_is_held_back_has_no_parts_to_add_up():
    """A refusal may reach some CTAs of a running call: their ranges are empty, and the groups that they would have had
    a part of keep their mass."""
    f = functions("mass.cu")
    held = f["plan"].index("held = __shfl_sync(kFull, latched, 0) & kErrHeld;")
    assert held < f["plan"].index("if (held) fb = fe;") < f["plan"].index("ctl->held = held;") < f["plan"].rindex("__syncthreads();")
    body = f["k_mass"]
    assert body.index("plan(p, ctl") < body.index("s.failed = ctl->held;") < body.index("p.split[blockIdx.x] = s;")


def test_a_cta_that_gave_up_says_so_when_its_roles_are_done():
    body, after = functions("mass.cu")["k_mass"], "if (threadIdx.x == 0 && p.cut && ctl->abort) p.split[blockIdx.x].failed = 1;"
    assert body.index("p.split[blockIdx.x] = s;") < body.rindex("__syncthreads();") < body.index(after)
    total = functions("mass.cu")["k_mass_sum"]
    assert total.index("failed |= p.split[c].failed;") < total.index("if (!failed) *mass")


def test_the_key_loaders_wait_for_all_of_their_copies_together():
    """A slot whose other half never comes has no end to wait for: the limit is one for all slots, as the header says."""
    body = functions("mass.cu")["key_loop"]
    assert "if (in_time && (used >> i & 1)) in_time = mbar_wait(&ctl->k_full[i]," in body
