"""Rounds of the key / value cache in which sequences are refused or share a prefix, on the GPU (needs a B200): a sequence that got
no slots keeps nothing, whatever the verification of the batch says about it; shared blocks are neither returned nor written."""
import numpy as np
import pytest
import torch

from oracle import cache as oc

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device=DEV)


class Pool:
    """Plans of a batch on the device beside the oracle's, call by call; cu_new is one array, read and written by every call."""

    def __init__(self, B, bt, W, n_blocks, T):
        self.bt, self.T, self.nb = bt, T, n_blocks
        self.seq, self.held, self.table, self.free = np.zeros(B, int), np.zeros(B, int), np.full((B, W), -1), list(range(n_blocks))
        self.cu = np.zeros(B + 1, int)
        self.d = dict(seq=_i32(self.seq), held=_i32(self.held), table=_i32(self.table), free=_i32(self.free), n_free=_i32([n_blocks]),
                      kv=_i32([0] * B), cu=_i32(self.cu), slots=_i32([0] * T), pos=_i32([0] * T), status=_i32([0] * B))

    def plan(self, lib, kept, new, extra=0, shared=None):
        d = self.d
        d["seq"].copy_(_i32(self.seq))
        lib.bs_cache_plan(d["seq"], kept, _i32(new), extra, None, self.bt, d["table"], d["held"], d["free"], d["n_free"], d["kv"], d["cu"],
                          d["slots"], d["pos"], d["status"], last_cu=d["cu"],
                          n_shared=None if shared is None else _i32(shared))
        torch.cuda.synchronize()
        r = oc.plan(self.seq, None if kept is None else kept.cpu().numpy(), np.asarray(new), extra, None, self.bt, self.table, self.held,
                    self.free, self.T, self.cu, shared)
        for n, k in (("seq", "seq_len"), ("held", "held"), ("table", "table"), ("kv", "kv_len"), ("cu", "cu_new"), ("slots", "slot_map"),
                     ("pos", "positions"), ("status", "status")):
            assert np.array_equal(d[n].cpu().numpy(), r[k]), n
        nf = int(d["n_free"].item())
        assert d["free"][:nf].cpu().tolist() == [int(x) for x in r["free"]]
        self.seq, self.held, self.table, self.free, self.cu = r["seq_len"], r["held"], r["table"], r["free"], r["cu_new"]
        return r


@pytest.mark.parametrize("B,T", [(5, 200), (1100, 9000)])  # the second: slots in a launch of their own, sequences in two passes
def test_a_pool_that_runs_out_in_the_middle(lib, B, T):
    """Prompts, then rounds with the verification's raw out_len as `kept`: lengths stay those of the tokens that were written."""
    rng = np.random.default_rng(B)
    p = Pool(B, 16, 8, B + 1, T)
    new = rng.integers(1, 20 if B < 10 else 8, B)
    p.plan(lib, None, new)
    kept, refused, length = new, 0, np.zeros(B, int)
    for _ in range(8):
        length += np.where(np.diff(p.cu) > 0, kept, 0)
        gamma = rng.integers(0, 7, B)
        r = p.plan(lib, _i32(kept), gamma, 1)
        assert np.array_equal(p.seq, length)
        refused += int((r["status"] != 0).sum())
        kept = rng.integers(0, 7, B) % (gamma + 1) + 1    # of every sequence, refused or not
        gone = rng.random(B) < 0.2
        p.seq[gone], length[gone], kept[gone] = 0, 0, 0
    assert refused > 3


def test_more_kept_than_granted_is_flagged(lib):
    p = Pool(3, 16, 4, 12, 64)
    p.plan(lib, None, [20, 5, 7])
    r = p.plan(lib, _i32([20, 6, 3]), [1, 1, 1])
    assert r["status"].tolist() == [0, lib.BS_DEV_BAD_LENGTH, 0] and r["seq_len"].tolist() == [20, 0, 3]


def test_the_path_of_a_refused_tree_moves_nothing(lib):
    """Sequence 0's tree gets no block; the verification accepts nodes 2, 4 of both trees all the same."""
    p = Pool(2, 16, 4, 3, 64)
    p.plan(lib, None, [14, 20])
    kept = _i32([14, 20])
    r = p.plan(lib, kept, [5, 5])
    assert r["status"].tolist() == [lib.BS_DEV_NO_BLOCKS, 0] and r["cu_new"].tolist() == [0, 0, 5]
    kc = torch.randint(0, 127, (3, 2, 16, 64), device=DEV, dtype=torch.uint8)
    vc, ks, vs = kc.flip(0).contiguous(), torch.ones(3, 2, device=DEV), torch.ones(3, 2, device=DEV)
    # room for the path inside the first block, so that only the plan's word keeps it where it is
    p.d["seq"][0] = 9
    was = [x.clone() for x in (kc, vc)]
    lib.bs_cache_keep_path(_i32([[2, 4, -1, -1]] * 2), _i32([2, 2]), p.d["seq"], p.d["table"], kc, ks, vc, vs, p.d["status"])
    torch.cuda.synchronize()
    own = p.d["table"][0, 0].item()
    for x, w in zip((kc, vc), was):
        assert torch.equal(x[own], w[own]) and not torch.equal(x, w)
    assert p.d["status"].tolist() == [lib.BS_DEV_NO_BLOCKS, 0]


@pytest.mark.parametrize("B,T", [(6, 300), (1100, 20000)])
def test_sequences_behind_a_common_prefix_come_and_go(lib, B, T):
    rng = np.random.default_rng(B + 1)
    bt, W, sh, nb, H, d = 16, 10, 3, 5 * B + 3, 2, 64
    prefix = [2, 0, 4]
    p = Pool(B, bt, W, nb, T)
    p.table[:, :sh] = prefix
    p.seq[:], p.held[:], p.free = sh * bt, sh, [b for b in range(nb) if b not in prefix]
    for n, x in (("table", p.table), ("held", p.held), ("n_free", [len(p.free)])):
        p.d[n].copy_(_i32(x))
    p.d["free"][:len(p.free)] = _i32(p.free)
    codes = [torch.randint(0, 127, (nb, H, bt, d), device=DEV, dtype=torch.uint8) for _ in range(2)]
    scales = [torch.full((nb, H), 2.0 ** -9, device=DEV) for _ in range(2)]
    was = [x[prefix].clone() for x in codes + scales]
    kept, shared = None, np.full(B, sh)
    for _ in range(6):
        r = p.plan(lib, kept, rng.integers(0, 14, B), 1, shared)
        assert not (r["status"] & lib.BS_DEV_BAD_LENGTH).any()
        x = torch.randn(T, H, d, device=DEV)              # far above what the present scales hold: a block written to changes
        lib.bs_cache_append(x, x, p.d["slots"], codes[0], scales[0], codes[1], scales[1])
        torch.cuda.synchronize()
        assert all(torch.equal(a[prefix], w) for a, w in zip(codes + scales, was))
        kept = rng.integers(0, 15, B) % np.maximum(np.diff(p.cu), 1)
        gone = rng.random(B) < 0.25
        p.seq[gone], kept[gone] = sh * bt, 0
        kept = _i32(kept)
    p.seq[:] = 0                                          # all end; the last reader lets the prefix go
    p.plan(lib, None, np.zeros(B, int), 0, np.array([0] + [sh] * (B - 1)))
    assert sorted(p.free) == list(range(nb))


def test_new_tokens_inside_shared_blocks_are_flagged(lib):
    p = Pool(4, 16, 4, 8, 64)
    p.table[:3, 0], p.held[:] = 0, [1, 1, 2, 0]
    p.table[2, 1] = 1
    p.seq[:], p.free = [16, 15, 31, 0], [5, 6]
    for n, x in (("table", p.table), ("held", p.held), ("n_free", [2])):
        p.d[n].copy_(_i32(x))
    p.d["free"][:2] = _i32([5, 6])
    r = p.plan(lib, None, [1, 1, 0, 1], 0, [1, 1, 2, 1])
    assert r["status"].tolist() == [0, lib.BS_DEV_BAD_LENGTH, 0, lib.BS_DEV_BAD_LENGTH]


@pytest.mark.parametrize("T", [64, 9000])
def test_captured_plans_follow_refusals_on_the_device(lib, T):
    """One captured plan, replayed: kept, the new tokens and the shared blocks change between replays, cu_new is read and written."""
    rng = np.random.default_rng(3)
    B, sh = 6, 1
    p = Pool(B, 16, 8, 10, T)
    p.table[:, 0], p.seq[:], p.held[:], p.free = 9, 16, 1, [b for b in range(10) if b != 9]
    kept, new, shared = _i32([0] * B), _i32([0] * B), _i32([sh] * B)
    d = p.d

    def load():
        for n, x in (("seq", p.seq), ("table", p.table), ("held", p.held), ("n_free", [len(p.free)]), ("cu", p.cu)):
            d[n].copy_(_i32(x))
        d["free"][:len(p.free)] = _i32(p.free)

    def step():
        lib.bs_cache_plan(d["seq"], kept, new, 1, None, 16, d["table"], d["held"], d["free"], d["n_free"], d["kv"], d["cu"], d["slots"],
                          d["pos"], d["status"], last_cu=d["cu"], n_shared=shared)

    load()
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    load()
    refused = 0
    for _ in range(12):
        n, k = rng.integers(3, 12, B), rng.integers(0, 5, B)
        new.copy_(_i32(n))
        kept.copy_(_i32(k))
        g.replay()
        torch.cuda.synchronize()
        r = oc.plan(p.seq, k, n, 1, None, 16, p.table, p.held, p.free, T, p.cu, [sh] * B)
        for name, key in (("seq", "seq_len"), ("held", "held"), ("table", "table"), ("kv", "kv_len"), ("cu", "cu_new"), ("slots", "slot_map"),
                          ("pos", "positions"), ("status", "status")):
            assert np.array_equal(d[name].cpu().numpy(), r[key]), name
        p.seq, p.held, p.table, p.free, p.cu = r["seq_len"], r["held"], r["table"], r["free"], r["cu_new"]
        refused += int((r["status"] & lib.BS_DEV_NO_BLOCKS != 0).sum())
    assert refused > 0
