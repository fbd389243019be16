"""The time-out path of the attention over the cache, read from the source: every wait is internal to a CTA, so no input makes one
run out, and what the kernels do after one can only be stated about the code (nothing is launched here)."""
import os
import re

import pytest

from conftest import ROOT

CSRC = os.path.join(ROOT, "paper_2505_15141_b200", "csrc")
KERNELS = ["bs_cache_attention.cu", "bs_cache_attention_rows.cu"]


def _accumulator(name):
    """The accumulator warps' part of a kernel, without comments."""
    src = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
    a = src.index("} else if (warp < 8) {")
    return src[a:src.index("} else {\n", src.index("ca_advance(p, cur, nt);", a))]


@pytest.mark.parametrize("name", KERNELS)
def test_accumulator_warps_leave_together_before_they_branch_on_the_marks(name):
    """A warp whose wait gave up does not know whether there are marks; barriers of the four warps that depend on them, or that
    come after the item's tiles at all, are met by all or by none only if the warps voted on leaving first."""
    src = _accumulator(name)
    wait = src.index("ca_wait(smem_u32(&b_l[buf])")
    vote = re.compile(r"if \(ca_bar_any\([^;{]*!ok\)\) \{ ok = false; break; \}")
    at = vote.search(src, wait)
    assert at, "no vote behind the wait for the sums"
    assert not re.search(r"s_nan_any|s_ml\[|if \(nans\)|ca_bar_any", src[wait:at.start()])
    # behind the vote `ok` is the same for all and does not change within the item: no vote, no branch on it
    rest = src[at.end():]
    assert "ok" not in re.findall(r"\bok\b", rest[:rest.index("mbar_arrive(smem_u32(&b_lfree")])
    assert not vote.search(rest)


@pytest.mark.parametrize("name", KERNELS)
def test_nothing_is_in_flight_when_a_cta_that_gave_up_ends(name):
    """A producer that had issued its last copy, or an issuer its last product, before another role gave up has left its own loop:
    the drain has to come behind the barrier at which all roles meet, and before tensor memory goes back."""
    src = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
    end = src[:src.index("tc_free(")].rindex("__syncthreads();")
    assert re.search(r"if \(s_abort\) ca_drain<RING>\(warp, b_full, s_tiles, &b_drain\);", src[end:src.index("tc_free(")])
    head = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "bs_cache_attention.cuh")).read())
    body = head[head.index("void ca_drain("):]
    body = body[:body.index("\n}\n")]
    assert body.index("warp < 2") < body.index("b_full[warp]") < body.index("cp.async.wait_all") < body.index("warp == 2") < body.index("ca_commit")
    produce = head[head.index("void ca_produce("):head.index("void ca_drain(")]
    assert "s_tiles[kv] = tile;" in produce and "mbar_wait" not in produce


def test_a_time_out_is_kept_where_the_host_can_read_it(lib):
    head = open(os.path.join(CSRC, "bs_cache_attention.cuh")).read()
    give_up = head[head.index("void ca_give_up("):]
    assert "*p.abort = 1u;" in give_up[:give_up.index("\n}\n")]
    f = lib._lib.bs_cache_get_device_status
    assert f(None, 1 << 20, None) == lib.BS_ERR_INVALID_ARG
    assert f(4096 + 16, 1 << 20, None) == lib.BS_ERR_WORKSPACE
    assert f(4096, 64, None) == lib.BS_ERR_WORKSPACE
