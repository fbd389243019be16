"""Rounds of the key / value cache over many plans: the oracle against a plain count of every sequence's tokens, and the host-side
refusals of bs_cache_plan_next (no kernel is launched here)."""
import numpy as np
import pytest

from oracle import cache as oc

P = 4096                                                  # a non-NULL, aligned pointer that is never followed


@pytest.mark.parametrize("seed", range(20))
def test_refused_sequences_keep_nothing(seed):
    """A pool too small for the batch: every round the verification returns an out_len for every sequence, refused ones too."""
    rng = np.random.default_rng(seed)
    B, bt, W, nb = 6, 16, 8, 7
    seq, held, table = np.zeros(B, int), np.zeros(B, int), np.full((B, W), -1)
    free, kept, cu, refused = list(range(nb)), None, None, 0
    length = [0] * B                                      # tokens that were written and kept
    for _ in range(12):
        was = None if cu is None else np.diff(cu)
        ended = rng.random(B) < 0.1
        for b in np.nonzero(ended)[0]:                    # the sequence ends and another takes its place
            seq[b], length[b] = 0, 0
            if kept is not None:
                kept[b] = 0
        if kept is not None:
            length = [n + int(k) * int(g > 0) for n, k, g in zip(length, kept, was)]
        new = rng.integers(0, 9, B)
        r = oc.plan(seq, kept, new, 1, None, bt, table, held, free, int(new.sum()) + B, cu)
        assert not (r["status"] & oc.BAD_LENGTH).any()
        assert r["seq_len"].tolist() == length
        seq, held, table, free, cu = r["seq_len"], r["held"], r["table"], r["free"], r["cu_new"]
        refused += int((r["status"] != 0).sum())
        kept = np.array([int(rng.integers(1, n + 2)) for n in new])
    assert refused > 3


def test_more_kept_than_granted_is_a_bad_length():
    table, held = np.array([[0, 1], [2, 3]]), np.array([2, 2])
    r = oc.plan(np.array([3, 3]), np.array([5, 4]), np.array([1, 1]), 0, None, 16, table, held, [], 8, np.array([0, 4, 8]))
    assert r["status"].tolist() == [oc.BAD_LENGTH, 0] and r["seq_len"].tolist() == [3, 7]


@pytest.mark.parametrize("seed", range(10))
def test_shared_blocks_are_nobodys_to_return(seed):
    """Sequences behind a common prefix come and go: its blocks never reach the stack, every other block has one place."""
    rng = np.random.default_rng(seed)
    B, bt, W, nb, sh = 5, 16, 32, 30, 2
    prefix = [7, 3]
    table = np.full((B, W), -1)
    table[:, :sh] = prefix
    seq, held, free, cu, kept = np.full(B, sh * bt), np.full(B, sh), [b for b in range(nb) if b not in prefix], None, None
    for _ in range(15):
        shared = np.full(B, sh)
        r = oc.plan(seq, kept, rng.integers(0, 30, B), 0, None, bt, table, held, free, 500, cu, shared)
        seq, held, table, free, cu = r["seq_len"], r["held"], r["table"], r["free"], r["cu_new"]
        assert not (r["status"] & oc.BAD_LENGTH).any() and (table[:, :sh] == prefix).all()
        used = [int(x) for b in range(B) for x in table[b, sh:held[b]]] + [int(x) for x in free]
        assert sorted(used + prefix) == list(range(nb))
        kept = np.minimum(np.diff(cu), rng.integers(0, 30, B))
        for b in np.nonzero(rng.random(B) < 0.3)[0]:      # it ends; the next one begins behind the same prefix
            seq[b], kept[b] = sh * bt, 0
    # all end, the last reader lets go: every block is back
    r = oc.plan(np.zeros(B, int), None, np.zeros(B, int), 0, None, bt, table, held, free, 1, None, np.array([0] + [sh] * (B - 1)))
    assert sorted(int(x) for x in r["free"]) == list(range(nb)) and r["held"].tolist() == [0] + [sh] * (B - 1)


def test_new_tokens_inside_shared_blocks_are_a_bad_length():
    table = np.array([[0, 1], [0, 1], [0, 2], [0, -1]])
    r = oc.plan(np.array([16, 15, 31, 0]), None, np.array([1, 1, 0, 1]), 0, None, 16, table, np.array([1, 1, 2, 0]), [5, 6], 8, None,
                np.array([1, 1, 2, 1]))
    assert r["status"].tolist() == [0, oc.BAD_LENGTH, 0, oc.BAD_LENGTH]


def test_plan_next_refuses(lib):
    f = lib._lib.bs_cache_plan_next

    def call(seq=P, last=P, shared=P, new=P, extra=1, B=4, bt=16, table=P, W=8, held=P, free=P, nb=64, nfree=P, kv=P, cu=P, slots=P, T=16):
        return f(seq, None, last, shared, new, extra, None, B, bt, table, W, held, free, nb, nfree, kv, cu, slots, None, T, None, None)

    for kw in ({"seq": None}, {"new": None}, {"table": None}, {"held": None}, {"free": None}, {"nfree": None}, {"kv": None},
               {"cu": None}, {"slots": None}, {"B": 0}, {"W": 0}, {"nb": 0}, {"T": 0}, {"extra": -1}):
        assert call(**kw) == lib.BS_ERR_INVALID_ARG, kw
    for kw in ({"bt": 8}, {"bt": 256}, {"B": lib.BS_MAX_BATCH + 1}, {"W": lib.BS_MAX_SEQ_BLOCKS + 1}, {"nb": 1 << 27, "bt": 16}):
        assert call(**kw) == lib.BS_ERR_UNSUPPORTED, kw
