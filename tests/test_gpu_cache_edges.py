"""The attention over the key / value cache at the edges of what its header allows (needs a B200)."""
import numpy as np
import pytest
import torch

from test_gpu_cache import Case

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_a_time_out_is_reported_without_a_status_array(lib):
    """No input makes a wait run out, so its word is put into the workspace by hand: a wait that gave up in any kernel leaves the
    same one, also for a call without a status array."""
    c = Case(1, [300, 20], [3, 2], 8, 2, 128, 16)
    ws = lib.new_cache_workspace(8, 2, 128, DEV)
    want = c.run(lib, ws=ws)
    lib.bs_cache_get_device_status(ws)
    n = torch.cuda.get_device_properties(0).multi_processor_count
    ws.view(torch.int32)[n] = 1                           # behind the arrival counters, one per multiprocessor
    with pytest.raises(lib.BanditSpecError) as e:
        lib.bs_cache_get_device_status(ws)
    assert e.value.code == lib.BS_ERR_TIMEOUT
    lib.bs_workspace_init(ws)
    lib.bs_cache_get_device_status(ws, torch.cuda.current_stream())
    assert torch.equal(c.run(lib, ws=ws), want)
    lib.bs_cache_get_device_status(ws)


LANES = [4, 8, 16, 40]                                    # with four query heads a key head: tiles of 16, 32, 64, 128 rows


def _scales(c, i, f):
    """Sets the scales of K (i = 0) or V (1): f(position of the block's first token, block) where a block is in use."""
    for b, kv in enumerate(c.kv):
        for j in range(-(-kv // c.bt)):
            c.scales[i][c.table[b, j]] = f(j * c.bt, c.table[b, j])


@pytest.mark.parametrize("max_new", LANES)
@pytest.mark.parametrize("rising", [False, True])
def test_scales_of_v_far_apart_in_different_tiles(lib, rising, max_new):
    """2^96 between the tiles of a sequence: a tile whose values vanish beside another's still has its share of the softmax sum."""
    c = Case(21, [400, 130, 3000], [4, 3, 2], 8, 2, 128, 16, q_mul=0.5)
    _scales(c, 1, lambda pos, blk: 2.0 ** (-64 if (pos // 128 % 2 == 0) == rising else 32))
    c.check(c.run(lib, max_new=max_new))


@pytest.mark.parametrize("max_new", LANES)
def test_scales_of_v_far_apart_in_one_tile(lib, max_new):
    c = Case(22, [400, 130], [4, 3], 8, 2, 128, 16, q_mul=0.5)
    _scales(c, 1, lambda pos, blk: 2.0 ** (-64 if pos // 16 % 2 else 32))
    c.check(c.run(lib, max_new=max_new))


@pytest.mark.parametrize("max_new", LANES)
@pytest.mark.parametrize("e", [-64, 100])
def test_scales_of_v_at_the_ends_of_their_range(lib, e, max_new):
    c = Case(23, [400, 130, 3000], [4, 3, 2], 8, 2, 128, 16, q_mul=2.0)
    _scales(c, 1, lambda pos, blk: 2.0 ** e)
    c.check(c.run(lib, max_new=max_new))


@pytest.mark.parametrize("max_new", LANES)
@pytest.mark.parametrize("e", [-100, 100])
def test_scales_of_k_and_queries_far_from_one(lib, e, max_new):
    c = Case(24, [400, 130], [4, 3], 8, 2, 128, 16, q_mul=2.0 ** (-6 - e))
    _scales(c, 0, lambda pos, blk: 2.0 ** e)
    c.check(c.run(lib, max_new=max_new))


@pytest.mark.parametrize("max_new", LANES)
@pytest.mark.parametrize("d", [64, 128])
def test_scales_that_are_no_powers_of_two(lib, d, max_new):
    c = Case(25, [400, 130, 77], [4, 3, 5], 8, 2, d, 16, q_mul=2.0, spread=2.0)
    rng = np.random.default_rng(25)
    for s in c.scales:
        s *= rng.uniform(1.0, 2.0, s.shape).astype(np.float32)
    c.check(c.run(lib, max_new=max_new))


@pytest.mark.parametrize("max_new", LANES)
def test_trees_of_a_root_alone(lib, max_new):
    c = Case(26, [100, 33, 4], [1, 2, 1], 8, 2, 128, 16)
    c.parent = np.zeros((3, 0), int)
    st = torch.zeros(3, dtype=torch.int32, device=DEV)
    out = c.run(lib, max_new=max_new, status=st)
    assert st.tolist() == [0, lib.BS_DEV_BAD_LENGTH, 0] and (out[1:3] == 7.0).all()
    c.check(out, seqs=[0, 2])


@pytest.mark.parametrize("max_new", [1, 4, 8, 16, 40])
@pytest.mark.parametrize("d", [64, 128])
def test_trees_larger_than_max_new(lib, d, max_new):
    """max_new chooses the tile: a tree's rows may fall into several of them."""
    rng = np.random.default_rng(d)
    new = [32, 7, 20, 1]
    c = Case(27, [200, 90, 5, 128], new, 16, 4, d, 16, q_mul=2.0)
    c.parent = np.array([[int(rng.integers(0, k)) for k in range(1, n)] + [0] * (32 - n) for n in new])
    st = torch.zeros(4, dtype=torch.int32, device=DEV)
    c.check(c.run(lib, max_new=max_new, status=st))
    assert not st.any()


@pytest.mark.parametrize("max_new", LANES)
def test_bad_data_without_a_status_array(lib, max_new):
    c = Case(28, [60, 200, 30, 40, 50], [3, 2, 4, 2, 4], 8, 2, 128, 16)
    c.parent = np.array([[0, 1, 2]] * 4 + [[0, 9, -1]])
    good = c.run(lib, max_new=max_new)                    # its last tree has bad parents
    st = torch.zeros(5, dtype=torch.int32, device=DEV)
    assert torch.equal(c.run(lib, max_new=max_new, status=st), good) and st.tolist() == [0, 0, 0, 0, lib.BS_DEV_BAD_TREE]
    c.kv[1] = c.table.shape[1] * 16 + 1
    c.table[2, 1] = -7
    out = c.run(lib, max_new=max_new)
    assert torch.equal(out[:3], good[:3]) and (out[3:5] == 7.0).all() and torch.equal(out[9:], good[9:])


@pytest.mark.parametrize("B", [600, 1500, 4096])
@pytest.mark.parametrize("max_new", LANES)
def test_more_sequences_than_threads(lib, B, max_new):
    """A thread looks after several sequences when the work is cut into shares; 4096 is the largest batch."""
    rng = np.random.default_rng(B)
    new = [int(n) for n in rng.integers(0, 4, B)]
    c = Case(B, rng.integers(0, 70, B).tolist(), new, 4, 1, 64, 64, q_mul=2.0)
    st, ws, dev = torch.zeros(B, dtype=torch.int32, device=DEV), lib.new_cache_workspace(4, 1, 64, DEV), c.device()
    out = c.run(lib, max_new=max_new, status=st, ws=ws, dev=dev)
    assert not st.any()
    c.check(out, seqs=[0, 1, B - 2, B - 1] + sorted(int(b) for b in rng.integers(0, B, 60)))
    assert torch.equal(c.run(lib, max_new=max_new, ws=ws, dev=dev), out)


@pytest.mark.parametrize("max_new", LANES)
@pytest.mark.parametrize("tree", [False, True])
def test_a_round_without_new_tokens_writes_nothing(lib, tree, max_new):
    c = Case(29, [100, 0, 33], [0, 0, 0], 8, 2, 128, 16)
    c.parent = np.zeros((3, 4), int) if tree else None
    st = torch.zeros(3, dtype=torch.int32, device=DEV)
    assert (c.run(lib, max_new=max_new, status=st) == 7.0).all() and not st.any()
