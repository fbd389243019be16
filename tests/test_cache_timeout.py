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
