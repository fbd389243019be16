"""The oracle of the key / value cache against independent statements, and the host-side refusals of bs_cache_*
(no kernel is launched here)."""
import numpy as np
import pytest
import torch

from oracle import cache as oc


def test_e4m3_table_and_rounding_against_torch():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(oc.VALUES, want, equal_nan=True)
    g = torch.Generator().manual_seed(0)
    x = torch.randn(200000, generator=g) * torch.exp(4 * torch.randn(200000, generator=g))
    mid = torch.tensor((oc.VALUES[:126] + oc.VALUES[1:127]) / 2, dtype=torch.float32)      # ties
    x = torch.cat([x, mid, -mid, torch.tensor([0.0, -0.0, 448.0, 464.0, 465.0, 1e30, -1e30])])
    want = x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(oc.encode(x.double().numpy()), want)
    assert np.isnan(oc.VALUES[oc.encode(np.array([np.nan]))[0]])
    assert oc.VALUES[oc.encode(np.array([np.inf, -np.inf]))].tolist() == [448.0, -448.0]


def test_block_scale_is_the_smallest_power_of_two():
    rng = np.random.default_rng(1)
    for x in list(np.exp(rng.normal(size=200) * 12)) + [448.0, 448.0 * 2 ** 9, 448.0000001, 1e-30, 0.0]:
        s = oc.block_scale(np.array([x, -x / 3]))
        assert s >= 2.0 ** -64 and np.log2(s) == round(np.log2(s)) and x <= 448 * s
        assert s == 2.0 ** -64 or x > 448 * s / 2
    assert oc.block_scale(np.array([np.inf, np.nan, 3.0])) == oc.block_scale(np.array([3.0]))


def test_a_plan_given_back_restores_the_stack_and_blocks_are_never_shared():
    rng = np.random.default_rng(2)
    for _ in range(50):
        B, bt, W = int(rng.integers(1, 9)), 16, 12
        seq = rng.integers(0, 60, B)
        held = -(-seq // bt)
        order = rng.permutation(int(held.sum()) + 40)
        table = np.full((B, W), -1)
        at = 0
        for b in range(B):
            table[b, :held[b]] = order[at:at + held[b]]
            at += held[b]
        free = [int(x) for x in order[at:]]
        r = oc.plan(seq, None, rng.integers(0, 40, B), 1, None, bt, table, held, free, 10_000)
        used = [int(x) for x in r["table"].ravel() if x >= 0] + list(r["free"])
        assert sorted(used) == sorted(order.tolist())
        ok = r["status"] == 0
        assert np.array_equal(r["held"][ok], -(-r["kv_len"][ok] // bt))
        back = oc.plan(r["seq_len"], None, np.zeros(B, int), 0, None, bt, r["table"], r["held"], r["free"], 1)
        assert back["free"] == free and np.array_equal(back["table"], table)


def test_growing_scale_leaves_normal_codes_exact():
    rng = np.random.default_rng(3)
    codes, scale = np.zeros((1, 1, 16, 64), np.uint8), np.ones((1, 1))
    x = rng.normal(size=(16, 1, 64))
    for i in range(16):                                   # token by token, sizes growing by 2^i
        oc.append(x[i:i + 1] * 2.0 ** (i % 4), np.array([i]), codes, scale, 16)
    for i in range(16):
        y = x[i, 0] * 2.0 ** (i % 4)
        got = oc.VALUES[codes[0, 0, i]] * scale[0, 0]
        assert (np.abs(got - y) <= np.maximum(np.abs(y) * 2.0 ** -4, scale[0, 0] * 2.0 ** -9)).all()


def test_tree_mask_and_attention_against_softmax():
    assert oc.sees(4, 2, [0, 1, 0]).astype(int).tolist() == [[1, 1, 1, 0, 0, 0], [1, 1, 1, 1, 0, 0], [1, 1, 1, 1, 1, 0], [1, 1, 1, 0, 0, 1]]
    assert np.array_equal(oc.sees(5, 3), oc.sees(5, 3, [0, 1, 2, 3]))
    assert not oc.sees(3, -2)[:2].any() and oc.sees(3, -2)[2].all()
    rng = np.random.default_rng(4)
    kc, vc = rng.integers(0, 126, (3, 2, 16, 64)).astype(np.uint8), rng.integers(0, 126, (3, 2, 16, 64)).astype(np.uint8)
    ks, vs = 2.0 ** rng.integers(-3, 3, (3, 2)), 2.0 ** rng.integers(-3, 3, (3, 2))
    q = rng.normal(size=(3, 4, 64)) * 0.01
    got = oc.attention(q, np.array([2, 0, 1]), 41, kc, ks, vc, vs, 0.125)
    k = torch.tensor((oc.VALUES[kc] * ks[:, :, None, None])[[2, 0, 1]]).transpose(0, 1).reshape(2, 48, 64)[:, :41]
    v = torch.tensor((oc.VALUES[vc] * vs[:, :, None, None])[[2, 0, 1]]).transpose(0, 1).reshape(2, 48, 64)[:, :41]
    want = torch.nn.functional.scaled_dot_product_attention(
        torch.tensor(q).transpose(0, 1), k.repeat_interleave(2, 0), v.repeat_interleave(2, 0),
        attn_mask=torch.tensor(oc.sees(3, 38)), scale=0.125).transpose(0, 1)
    assert np.abs(got - want.numpy()).max() < 1e-9


# ---- refusals: on the host, before anything is launched ---------------------------------------

P = 4096                                                  # a non-NULL, aligned pointer that is never followed


def test_plan_refuses(lib):
    f = lib._lib.bs_cache_plan

    def call(seq=P, kept=None, new=P, extra=1, B=4, bt=16, table=P, W=8, held=P, free=P, nb=64, nfree=P, kv=P, cu=P, slots=P, T=16):
        return f(seq, kept, new, extra, None, B, bt, table, W, held, free, nb, nfree, kv, cu, slots, None, T, None, None)

    for kw in ({"seq": None}, {"new": None}, {"table": None}, {"held": None}, {"free": None}, {"nfree": None}, {"kv": None},
               {"cu": None}, {"slots": None}, {"B": 0}, {"W": 0}, {"nb": 0}, {"T": 0}, {"extra": -1}):
        assert call(**kw) == lib.BS_ERR_INVALID_ARG, kw
    for kw in ({"bt": 8}, {"bt": 24}, {"bt": 256}, {"bt": 0}, {"B": lib.BS_MAX_BATCH + 1}, {"W": lib.BS_MAX_SEQ_BLOCKS + 1},
               {"nb": 1 << 27, "bt": 16}):
        assert call(**kw) == lib.BS_ERR_UNSUPPORTED, kw


def test_append_refuses(lib):
    f = lib._lib.bs_cache_append

    def call(k=P, v=P, dt=lib.BS_BF16, kt=1024, kh=128, vt=1024, vh=128, slots=P, T=4, H=8, d=128, kc=P, ks=P, vc=P, vs=P, nb=8, bt=16):
        return f(k, v, dt, kt, kh, vt, vh, slots, T, H, d, kc, ks, vc, vs, nb, bt, None)

    for kw in ({"k": None}, {"v": None}, {"slots": None}, {"kc": None}, {"ks": None}, {"vc": None}, {"vs": None}, {"T": 0}, {"H": 0},
               {"d": 0}, {"nb": 0}, {"bt": 0}, {"dt": 5}, {"k": P + 2}, {"vc": P + 8}):
        assert call(**kw) == lib.BS_ERR_INVALID_ARG, kw
    for kw in ({"d": 96}, {"d": 256}, {"bt": 8}, {"bt": 48}, {"kt": 1028}, {"vh": 100}, {"dt": lib.BS_F32, "kh": 130}):
        assert call(**kw) == lib.BS_ERR_UNSUPPORTED, kw


def test_attention_refuses(lib):
    f = lib._lib.bs_cache_attention

    def call(q=P, qt=4096, qh=128, cu=P, kv=P, table=P, W=8, par=None, N=0, kc=P, ks=P, vc=P, vs=P, nb=8, bt=16, B=2, T=4, Hq=32, H=8,
             d=128, mn=2, sc=0.1, out=P, ot=4096, oh=128, ws=P, n=1 << 30):
        return f(q, qt, qh, cu, kv, table, W, par, N, kc, ks, vc, vs, nb, bt, B, T, Hq, H, d, mn, sc, out, ot, oh, None, ws, n, None)

    for kw in ({"q": None}, {"cu": None}, {"kv": None}, {"table": None}, {"kc": None}, {"ks": None}, {"vc": None}, {"vs": None},
               {"out": None}, {"ws": None}, {"B": 0}, {"T": 0}, {"W": 0}, {"mn": 0}, {"Hq": 0}, {"H": 0}, {"Hq": 30}, {"q": P + 2},
               {"out": P + 8}, {"kc": P + 4}, {"sc": float("nan")}, {"sc": float("inf")}, {"N": -1}):
        assert call(**kw) == lib.BS_ERR_INVALID_ARG, kw
    for kw in ({"d": 96}, {"bt": 8}, {"Hq": 130, "H": 2}, {"B": lib.BS_MAX_BATCH + 1}, {"par": P, "N": 32}, {"qt": 4100}, {"oh": 4},
               {"W": lib.BS_MAX_SEQ_BLOCKS + 1}):
        assert call(**kw) == lib.BS_ERR_UNSUPPORTED, kw
    for kw in ({"n": 100}, {"ws": P + 16}):
        assert call(**kw) == lib.BS_ERR_WORKSPACE, kw
    assert lib._lib.bs_cache_workspace_bytes(32, 8, 128) > 0
    for bad in ((30, 8, 128), (0, 8, 128), (8, 0, 64), (130, 2, 64), (8, 8, 96)):
        assert lib._lib.bs_cache_workspace_bytes(*bad) == 0


def test_keep_path_refuses(lib):
    f = lib._lib.bs_cache_keep_path

    def call(on=P, acc=P, seq=P, B=2, N=7, table=P, W=8, H=8, d=128, kc=P, ks=P, vc=P, vs=P, nb=8, bt=16):
        return f(on, acc, seq, B, N, table, W, H, d, kc, ks, vc, vs, nb, bt, None, None)

    for kw in ({"on": None}, {"acc": None}, {"seq": None}, {"table": None}, {"kc": None}, {"ks": None}, {"vc": None}, {"vs": None},
               {"B": 0}, {"N": 0}, {"W": 0}, {"H": 0}, {"d": 0}, {"kc": P + 8}):
        assert call(**kw) == lib.BS_ERR_INVALID_ARG, kw
    for kw in ({"N": 32}, {"d": 80}, {"bt": 4}, {"B": lib.BS_MAX_BATCH + 1}):
        assert call(**kw) == lib.BS_ERR_UNSUPPORTED, kw


def test_binding_checks_shapes_and_types(lib):
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(AssertionError):
        lib._i32(torch.zeros(4, dtype=torch.int64), 4)
    with pytest.raises(AssertionError):
        lib._i32(i32(4), 5)
    kc, ks = lib.new_cache(4, 2, 16, 64, device="cpu")
    with pytest.raises(AssertionError):
        lib._cache_args(kc, ks[:, :1], kc, ks)
    with pytest.raises(AssertionError):
        lib._cache_args(kc, ks, kc[:2], ks)
    with pytest.raises(AssertionError):
        lib._cache_args(kc.float(), ks, kc, ks)
