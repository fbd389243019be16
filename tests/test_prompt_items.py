"""How the CTAs of bs_prompt_attention take their items: the kernel's own header, run on the host with CTA numbers in orders that a GPU
does not give on demand (no GPU needed)."""
import os
import re
import subprocess

import numpy as np
import pytest

from conftest import ROOT

KEYS = 128


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("items") / "items")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wno-unknown-pragmas", "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROOT, "paper_2505_15141_b200", "csrc"), "-o", out, os.path.join(ROOT, "tests", "prompt_items_host.cpp")], check=True)
    return out


def _run(program, cu, T, Hkv, TQ, numbers, running):
    text = " ".join(map(str, [T, Hkv, TQ, len(cu) - 1, *cu, running, len(numbers), *numbers]))
    out = subprocess.run([program], input=text, capture_output=True, text=True, check=True, timeout=120).stdout.split("\n")
    items = [tuple(map(int, ln.split()[1:])) for ln in out if ln.startswith("item")]
    status = [int(ln.split()[2]) for ln in out if ln.startswith("status")]
    return items, status


def _grid(T, B, Hkv, TQ):
    return (T // (2 * TQ) + B) * Hkv


def _want(cu, good, Hkv, TQ):
    """Every item once: (row0, n, i0, h, nt0, nt1)."""
    out = []
    for lo, hi, ok in zip(cu[:-1], cu[1:], good):
        n = hi - lo if ok else 0
        for i0 in range(0, n, 2 * TQ):
            tiles = [-(-min(n, i0 + k * TQ) // KEYS) if i0 + (k - 1) * TQ < n else 0 for k in (1, 2)]
            out += [(lo, n, i0, h, *tiles) for h in range(Hkv)]
    return sorted(out)


def _ragged(B, most, seed):
    rng = np.random.default_rng(seed)
    n = rng.integers(0, most, B)
    n[rng.random(B) < 0.2] = 0
    return np.concatenate([[0], np.cumsum(n)]).tolist()


ORDERS = {
    "ascending": lambda g, rng: list(range(g)),
    "descending": lambda g, rng: list(range(g))[::-1],
    "any": lambda g, rng: rng.permutation(g).tolist(),
    "the last first": lambda g, rng: [g - 1] + list(range(g - 1)),
}


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("B,most,Hkv,TQ", [(1, 3000, 1, 128), (5, 700, 2, 32), (40, 700, 3, 25), (100, 400, 1, 18), (70, 2, 4, 64), (33, 1500, 2, 128)])
def test_every_item_is_taken_once_whatever_the_order_of_the_numbers(program, B, most, Hkv, TQ, order):
    cu = _ragged(B, most, B + TQ)
    T = cu[-1] + 3
    for running in (1, 7):
        grid = _grid(T, B, Hkv, TQ)
        numbers = ORDERS[order](grid, np.random.default_rng(B))
        items, status = _run(program, cu, T, Hkv, TQ, numbers, min(running, grid))
        assert sorted(i[1:] for i in items) == _want(cu, [True] * B, Hkv, TQ)
        assert not any(status)


def test_the_longest_items_of_32_sequences_come_first(program):
    cu, T = _ragged(70, 900, 5), 70 * 900
    items, _ = _run(program, cu, T, 2, 64, list(range(_grid(T, 70, 2, 64))), 1)
    group = [max(b for b in range(70) if cu[b] == i[1] and cu[b + 1] > cu[b]) // 32 for i in items]
    assert group == sorted(group)
    for g in range(3):
        starts = [i[3] for i, k in zip(items, group) if k == g]
        assert starts == sorted(starts, reverse=True)


def test_bad_lengths_in_the_second_group(program):
    """Sequences whose lengths make no sense have no items, those around them have all of theirs."""
    cu = _ragged(60, 500, 9)
    T = cu[-1]
    cu[41] = cu[40] - 1                                       # 40 descends, 41 begins before its predecessor's end
    good = [True] * 60
    good[40] = False
    cu[41] = max(cu[41], 0)
    cu[60] = T + 1                                            # behind the last token
    good[59] = False
    cu[20], good[19], good[20] = -1, False, False
    for order in ORDERS:
        numbers = ORDERS[order](_grid(T, 60, 2, 32), np.random.default_rng(3))
        items, status = _run(program, cu, T, 2, 32, numbers, 5)
        bad = [b for b in range(60) if status[b]]
        assert set(bad) >= {19, 20, 40, 59} and set(bad) <= {19, 20, 40, 41, 59} and set(status) <= {0, 64}
        assert sorted(i[1:] for i in items) == _want(cu, [b not in bad for b in range(60)], 2, 32)


@pytest.mark.parametrize("cu", [[0, 100, 60, 90], [0, 100, 60, 90, 210], [50, 120, 10, 60, 130], [0, 200, 0, 200], [0, 80, 80, 20, 90, 90, 150],
                                [0, 500, 100, 150], [100, 40, 60, 50, 70, 80]])
@pytest.mark.parametrize("before", [0, 30, 31, 40])
def test_a_row_belongs_to_one_sequence_at_most(program, cu, before):
    """Lengths that go back: a sequence that begins before the end of an earlier one would write its rows again, in whatever order the
    CTAs run.  It is reported, the earlier one is whole; also when the earlier one is among the 32 before."""
    cu = [0] * before + cu
    B, T = len(cu) - 1, 210
    ends, good = 0, []
    for lo, hi in zip(cu[:-1], cu[1:]):
        sane = 0 <= lo <= hi <= T
        good.append(sane and lo >= ends)
        if sane:
            ends = max(ends, hi)
    for order in ("ascending", "any"):
        items, status = _run(program, cu, T, 2, 16, ORDERS[order](_grid(T, B, 2, 16), np.random.default_rng(1)), 4)
        assert status == [0 if g else 64 for g in good]
        assert sorted(i[1:] for i in items) == _want(cu, good, 2, 16)
    rows = [r for lo, hi, g in zip(cu[:-1], cu[1:], good) if g for r in range(lo, hi)]
    assert len(rows) == len(set(rows))


def test_a_wait_may_last_as_long_as_the_longest_item(program):
    """Three waits do (for an item's place, for V that is seen in part, of the warps whose row tile an item lacks).  A tile of keys takes
    3150 cycles, measured; a healthy call has four times that, and a second, at every length that is not refused."""
    for T in [1, 130, 16384, 635000 * KEYS, 80000000, 2 ** 30 - 1, 2 ** 30]:
        limit = int(subprocess.run([program, str(T)], capture_output=True, text=True, check=True).stdout)
        assert 2000000000 + 4 * 3150 * -(-T // KEYS) <= limit <= 2 ** 38
        assert limit < 2.2e9 or T > 10 ** 6                   # what does not end ends in about a second in calls of usual lengths


def test_every_wait_of_the_kernel_has_this_limit():
    src = open(os.path.join(ROOT, "paper_2505_15141_b200", "csrc", "bs_prompt_attention.cu")).read()
    assert src.count("try_wait.parity") == 1 and "kWaitCycles" not in src
    assert src.count("clock64() - t0 <= limit);") == 1 and src.count("p.limit = pa_wait_limit(T);") == 1
    waits = re.findall(r"pa_wait(?:<true>)?\((?!const)(.*)", src)
    assert len(waits) == 6 and all("p.limit, &s_abort)" in w for w in waits)
