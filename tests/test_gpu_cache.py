"""The key / value cache of a round on the GPU against the oracle (needs a B200), through the C ABI: bs_cache_plan,
bs_cache_append, bs_cache_attention, bs_cache_keep_path, and rounds of all of them together.

Whole numbers, codes and scales are compared bit for bit.  Tolerance of the attention, from its arithmetic: out =
sum_j w_j v_j / sum_j p_j, and per row and element

  2^-8 |out|                        rounding to bf16
  (2^-8 + 2^-11) sum_j p_j |v_j|    a probability is two e4m3 terms (each half a step of 2^-4) after fp16 (2^-11)
  2^-18 a_T sum_{j in T} |code_j|   floor of the second term: half of the smallest subnormal 2^-9, probabilities of a
                                    tile T scaled so that its largest p_j s_j, a_T, becomes 2^8
  2 B sum_j p_j |v_j|               B: error of an exponent, scale (2^-17 max|q| sum_d |k_d| + 2^-18 sum_d |q_d k_d|) (queries
                                    below the range of the split; accumulation, measured 2^-20 of the largest product)
                                    plus 2^-21 (|t| + 64) for t itself in fp32, its shift by log2 of the scale and ex2
"""
import numpy as np
import pytest
import torch

from oracle import cache as oc

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device=DEV)


class Case:
    """A cache with blocks in a shuffled order, everything that may not be read filled with NaN codes, NaN scales and
    block numbers far outside."""

    def __init__(self, seed, ctx, new, Hq, Hkv, d, bt, q_mul=1.0, pad=3, spread=1.0):
        rng = np.random.default_rng(seed)
        self.ctx, self.new, self.bt, self.d, self.Hq, self.Hkv = list(ctx), list(new), bt, d, Hq, Hkv
        self.kv = [max(0, c + n) for c, n in zip(ctx, new)]
        held = [-(-k // bt) for k in self.kv]
        nb = sum(held) + 4
        order = rng.permutation(nb)
        W = max(held) + 2
        self.table = np.full((len(new), W), 1 << 30, np.int64)
        at = 0
        for b, h in enumerate(held):
            self.table[b, :h] = order[at:at + h]
            at += h
        self.codes, self.scales = [], []
        for _ in range(2):
            c = np.full((nb, Hkv, bt, d), 0x7F, np.uint8)
            s = np.full((nb, Hkv), np.nan, np.float32)
            for b, k in enumerate(self.kv):
                for j in range(held[b]):
                    n = min(bt, k - j * bt)
                    c[self.table[b, j], :, :n] = oc.encode(rng.normal(size=(Hkv, n, d)) * 60.0)
                    s[self.table[b, j]] = 2.0 ** (-6 + np.round(spread * rng.normal(size=Hkv)))
            self.codes.append(c)
            self.scales.append(s)
        self.cu = np.concatenate([[0], np.cumsum(self.new)])
        self.T = int(self.cu[-1]) + pad
        self.q = torch.tensor(rng.normal(size=(self.T, Hq, d)) * q_mul, dtype=torch.bfloat16)
        self.scale = d ** -0.5
        self.parent = None

    def device(self):
        f8 = [torch.tensor(c, device=DEV).view(torch.float8_e4m3fn) for c in self.codes]
        sc = [torch.tensor(s, device=DEV) for s in self.scales]
        return f8[0], sc[0], f8[1], sc[1]

    def run(self, lib, max_new=None, status=None, ws=None, q=None, out=None, dev=None):
        kc, ks, vc, vs = dev or self.device()
        q = self.q.to(DEV) if q is None else q
        out = torch.full((self.T, self.Hq, self.d), 7.0, dtype=torch.bfloat16, device=DEV) if out is None else out
        ws = lib.new_cache_workspace(self.Hq, self.Hkv, self.d, DEV) if ws is None else ws
        par = None if self.parent is None else _i32(self.parent)
        lib.bs_cache_attention(q, _i32(self.cu), _i32(self.kv), _i32(self.table), par, kc, ks, vc, vs,
                               max(1, max(self.new)) if max_new is None else max_new, self.scale, out, status, ws)
        torch.cuda.synchronize()
        return out

    def want(self, b):
        return oc.attention(self.q[self.cu[b]:self.cu[b + 1]].double().numpy(), self.table[b], self.kv[b], self.codes[0],
                            self.scales[0].astype(np.float64), self.codes[1], self.scales[1].astype(np.float64), self.scale,
                            None if self.parent is None else self.parent[b])

    def tolerance(self, b):
        q = self.q[self.cu[b]:self.cu[b + 1]].double().numpy()
        n, kv, bt, d = self.new[b], self.kv[b], self.bt, self.d
        G, see = self.Hq // self.Hkv, oc.sees(n, kv - n, None if self.parent is None else self.parent[b])
        nb = -(-kv // bt)
        blocks = self.table[b, :nb]
        tol = np.zeros((n, self.Hq, d))
        for h in range(self.Hkv):
            k = (oc.VALUES[self.codes[0][blocks, h]] * self.scales[0][blocks, h][:, None, None].astype(np.float64)).reshape(-1, d)[:kv]
            code = np.abs(oc.VALUES[self.codes[1][blocks, h]].reshape(-1, d)[:kv])
            s = np.repeat(self.scales[1][blocks, h].astype(np.float64), bt)[:kv]
            for g in range(G):
                for i in range(n):
                    idx = np.nonzero(see[i])[0]
                    if not idx.size:
                        continue
                    qi = q[i, h * G + g]
                    t = k[idx] @ qi * self.scale
                    p = np.exp(t - t.max())
                    p /= p.sum()
                    mass = p @ (s[idx, None] * code[idx])
                    B = abs(self.scale) * (2.0 ** -17 * np.abs(qi).max() * np.abs(k[idx]).sum(1) + 2.0 ** -18 * (np.abs(k[idx]) @ np.abs(qi))).max()
                    B += 2.0 ** -21 * (np.abs(t).max() + 64)
                    floor = np.zeros(d)
                    for T in np.unique(idx // 128):
                        m = idx // 128 == T
                        floor += 2.0 ** -18 * (p[m] * s[idx[m]]).max() * code[idx[m]].sum(0)
                    tol[i, h * G + g] = (2.0 ** -8 + 2.0 ** -11 + 2 * B) * mass + floor
        return tol

    def check(self, out, seqs=None):
        o = out.double().cpu().numpy()
        worst = 0.0
        for b in range(len(self.new)) if seqs is None else seqs:
            if not self.new[b]:
                continue
            want = self.want(b)
            got = o[self.cu[b]:self.cu[b + 1]]
            tol = self.tolerance(b) + 2.0 ** -8 * np.abs(want) + 1e-30
            assert np.isfinite(got).all(), (b, np.argwhere(~np.isfinite(got))[:4])
            worst = max(worst, float((np.abs(got - want) / tol).max()))
        assert worst <= 1.0, worst
        assert (o[self.cu[-1]:] == 7.0).all()             # rows behind the last sequence
        return worst


# ---- attention -----------------------------------------------------------------------------------

@pytest.mark.parametrize("bt", [16, 64])
def test_one_token(lib, bt):
    c = Case(1, [4], [1], 8, 2, 128, bt)
    c.check(c.run(lib))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("ctx", [0, 1, 15, 16, 126, 127, 128, 129, 255, 300, 1023])
def test_one_token_at_block_and_tile_edges(lib, d, ctx):
    c = Case(ctx, [ctx], [1], 8, 2, d, 16)
    c.check(c.run(lib))


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (5, 5), (8, 2), (28, 4), (16, 2), (40, 1), (64, 1)])
@pytest.mark.parametrize("d", [64, 128])
def test_head_groups(lib, Hq, Hkv, d):
    c = Case(Hq + d, [100, 0, 333, 17], [1, 3, 2, 9], Hq, Hkv, d, 32, q_mul=2.0)
    c.check(c.run(lib))


@pytest.mark.parametrize("bt", [16, 32, 64, 128])
@pytest.mark.parametrize("d", [64, 128])
def test_ragged_round(lib, d, bt):
    ctx = [0, 1, 500, 127, 128, 77, 260, 3, 1000, 64]
    new = [5, 0, 9, 3, 0, 7, 1, 2, 4, 0]
    c = Case(bt, ctx, new, 16, 4, d, bt, q_mul=3.0)
    st = torch.zeros(len(new), dtype=torch.int32, device=DEV)
    c.check(c.run(lib, status=st))
    assert not st.any()


@pytest.mark.parametrize("max_new", [1, 3, 6, 8, 100])
def test_every_tile_width_gives_the_result(lib, max_new):
    c = Case(7, [200, 90, 5], [9, 4, 20], 16, 4, 128, 16, q_mul=2.0)
    c.check(c.run(lib, max_new=max_new))


@pytest.mark.parametrize("G", [1, 4, 7])
def test_piece_of_a_prompt(lib, G):
    c = Case(G, [0, 150], [300, 77], 2 * G, 2, 128, 16, q_mul=2.0)
    c.check(c.run(lib))


@pytest.mark.parametrize("max_new", [4, 5, 16, 32])
def test_split_over_many_ctas(lib, max_new):
    c = Case(3, [20000], [5], 4, 1, 128, 64, q_mul=3.0)
    c.check(c.run(lib, max_new=max_new))
    c = Case(4, [9000, 1, 5000], [2, 3, 1], 7, 1, 64, 16, q_mul=3.0)
    c.check(c.run(lib, max_new=max_new))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,new,max_new", [(2, [1, 3, 8], 8), (4, [8, 1, 5], 8), (8, [8, 3, 1], 8), (4, [16, 40, 3], 40)])
def test_many_short_items(lib, d, G, new, max_new):
    """Many more sequences than CTAs, a tile or two each: every CTA walks through a row of items, of the four tile widths."""
    rng = np.random.default_rng(G)
    B = 500
    new = [new[b % 3] if b % 11 else 0 for b in range(B)]
    ctx = rng.integers(0, 150, B).tolist()
    c = Case(G, ctx, new, 2 * G, 2, d, 16, q_mul=2.0)
    st = torch.zeros(B, dtype=torch.int32, device=DEV)
    ws, dev = lib.new_cache_workspace(2 * G, 2, d, DEV), c.device()
    out = c.run(lib, max_new=max_new, status=st, ws=ws, dev=dev)
    assert not st.any()
    c.check(out, seqs=[0, 1, 2, 3, 250, 251, 252, 497, 498, 499])
    for _ in range(20):
        assert torch.equal(c.run(lib, max_new=max_new, ws=ws, dev=dev), out)


def _random_parents(rng, n, N):
    return [int(rng.integers(0, k)) for k in range(1, n)] + [int(rng.integers(-5, 50)) for _ in range(N - max(n - 1, 0))]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 4, 8])
def test_trees(lib, d, G):
    rng = np.random.default_rng(G + d)
    new = [1, 32, 15, 2, 0, 13, 7]
    c = Case(G, [0, 100, 120, 250, 9, 3, 640], new, 2 * G, 2, d, 16, q_mul=2.0)
    c.parent = np.array([_random_parents(rng, n, 31) for n in new])
    st = torch.zeros(len(new), dtype=torch.int32, device=DEV)
    c.check(c.run(lib, status=st))
    assert not st.any()


def test_a_chain_shaped_tree_is_the_chain(lib):
    c = Case(5, [100, 33], [6, 9], 8, 2, 128, 16)
    a = c.run(lib)
    c.parent = np.array([list(range(8))] * 2)
    assert torch.equal(c.run(lib), a)


def test_bad_trees_are_flagged_and_hang_under_the_root(lib):
    c = Case(6, [40, 40, 40], [5, 5, 5], 8, 2, 64, 16)
    c.parent = np.array([[0, 1, 2, 3], [0, 2, 9, -1], [0, 0, 0, 0]])
    st = torch.zeros(3, dtype=torch.int32, device=DEV)
    out = c.run(lib, status=st)
    assert st.tolist() == [0, lib.BS_DEV_BAD_TREE, 0]
    c.check(out)                                          # the oracle reads a bad parent as the root, too
    c.parent = np.array([[0], [0], [0]])                  # room for one drafted node, five rows
    st.zero_()
    assert (c.run(lib, status=st)[:15] == 7.0).all()
    assert st.tolist() == [lib.BS_DEV_BAD_LENGTH] * 3


@pytest.mark.parametrize("max_new", [4, 8, 16, 40])
def test_rows_that_see_nothing_are_zero(lib, max_new):
    c = Case(8, [-3, 20, -9], [5, 2, 4], 8, 2, 128, 16)   # fewer cached tokens than new ones; none at all
    out = c.run(lib, max_new=max_new)
    c.check(out)
    assert (out[:3] == 0).all() and (out[7:11] == 0).all()


@pytest.mark.parametrize("max_new", [4, 8, 16, 40])     # tiles of 16, 32, 64 and 128 rows
@pytest.mark.parametrize("d", [64, 128])
def test_nan_and_infinity_stay_with_those_who_see_them(lib, d, max_new):
    c = Case(9, [100, 50], [6, 3], 8, 2, d, 16)
    blk, off = c.table[0, 103 // 16], 103 % 16
    c.codes[1][blk, 1, off, 5] = 0x7F                     # V of new token 3 of sequence 0, head 1
    c.codes[1][blk, 1, off, 57] = 0xFF
    c.codes[0][c.table[0, 105 // 16], 0, 105 % 16, 3] = 0x7F   # K of its token 5, head 0
    c.q[c.cu[1] + 1, 2, 9] = float("inf")                 # a query of sequence 1
    c.q[c.cu[1] + 2, 7, 1] = float("nan")
    out = c.run(lib, max_new=max_new).float().cpu().numpy()
    bad = np.zeros(out.shape, bool)
    bad[3:6, 4:8, 5] = bad[3:6, 4:8, 57] = True
    bad[5, 0:4] = True
    bad[c.cu[1] + 1, 2] = bad[c.cu[1] + 2, 7] = True
    assert np.array_equal(np.isnan(out), bad)
    for b, seq in ((0, slice(0, 6)), (1, slice(6, 9))):
        with np.errstate(invalid="ignore"):
            want, tol = c.want(b), c.tolerance(b)
        ok = ~bad[seq] & np.isfinite(want) & np.isfinite(tol)
        assert ok.sum() > 0.5 * ok.size
        assert (np.abs(out[seq] - want)[ok] <= (tol + 2.0 ** -8 * np.abs(want))[ok]).all()


@pytest.mark.parametrize("max_new", [4, 16, 40])        # tokens as lanes, rows as lanes (64, 128)
@pytest.mark.parametrize("kind", ["v_scales", "k_scales", "sharp", "flat", "tiny_q", "negative_scale"])
def test_values_far_apart(lib, kind, max_new):
    c = Case(10, [400, 130], [4, 3], 8, 2, 128, 16, q_mul={"sharp": 40.0, "flat": 1e-3, "tiny_q": 1e-30}.get(kind, 2.0))
    rng = np.random.default_rng(0)
    if kind == "v_scales":                                # blocks 2^44 apart inside one tile, and a block of zeros
        c.scales[1] = np.where(np.isnan(c.scales[1]), c.scales[1], 2.0 ** rng.integers(-24, 20, c.scales[1].shape)).astype(np.float32)
        c.codes[1][c.table[0, 2]] = 0
        c.scales[1][c.table[0, 2]] = 2.0 ** -64
    if kind == "k_scales":
        c.scales[0] = np.where(np.isnan(c.scales[0]), c.scales[0], 2.0 ** rng.integers(-20, -3, c.scales[0].shape)).astype(np.float32)
    if kind == "negative_scale":
        c.scale = -c.scale
    c.check(c.run(lib, max_new=max_new))


def test_strides_and_a_padded_batch(lib):
    c = Case(11, [60, 200], [3, 2], 8, 2, 128, 16, pad=11)
    big = torch.full((c.T, 24, 128), float("nan"), dtype=torch.bfloat16, device=DEV)
    big[:, 8:16] = c.q.to(DEV)
    o = torch.full((c.T, 2, 8, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    out = c.run(lib, q=big[:, 8:16], out=o[:, 1])
    c.check(out)
    assert (o[:, 0] == 7.0).all()


@pytest.mark.parametrize("max_new", [4, 16])
def test_sequences_share_the_blocks_of_a_common_prefix(lib, max_new):
    c = Case(41, [100, 300, 90], [3, 4, 2], 16, 4, 128, 16, q_mul=2.0)
    c.table[1, :5] = c.table[2, :5] = c.table[0, :5]
    c.check(c.run(lib, max_new=max_new))


def test_bad_lengths_and_blocks_are_flagged(lib):
    c = Case(12, [60, 200, 30, 40], [3, 2, 4, 2], 8, 2, 128, 16)
    good = c.run(lib)
    c.kv[1] = c.table.shape[1] * 16 + 1
    st = torch.zeros(4, dtype=torch.int32, device=DEV)
    out = c.run(lib, status=st)
    assert st.tolist() == [0, lib.BS_DEV_BAD_LENGTH, 0, 0] and (out[3:5] == 7.0).all()
    assert torch.equal(out[:3], good[:3]) and torch.equal(out[5:], good[5:])
    c.kv[1] = 202
    c.table[2, 1] = -7
    st.zero_()
    out = c.run(lib, status=st)
    assert st.tolist() == [0, 0, lib.BS_DEV_BAD_BLOCK, 0]
    assert torch.equal(out[:5], good[:5]) and torch.equal(out[9:], good[9:])
    c.table[2, 1] = 0
    c.cu[2] = 2                                           # not ascending
    st.zero_()
    c.run(lib, status=st)
    assert st[1].item() == lib.BS_DEV_BAD_LENGTH


@pytest.mark.parametrize("max_new", [4, 8, 16, 32])
def test_repeats_bit_for_bit_and_leaves_the_workspace_clear(lib, max_new):
    c = Case(13, [3000, 700, 1], [5, 9, 2], 8, 2, 128, 16, q_mul=2.0)
    ws, dev = lib.new_cache_workspace(8, 2, 128, DEV), c.device()
    first = c.run(lib, ws=ws, dev=dev, max_new=max_new)
    c.check(first)
    for _ in range(200):
        assert torch.equal(c.run(lib, ws=ws, dev=dev, max_new=max_new), first)
    assert not ws[:592].any()                             # arrival counters


def test_two_streams_with_a_workspace_each(lib):
    cs = [Case(14 + i, [2000 + 500 * i, 300], [4, 6], 8, 2, 128, 16, q_mul=2.0) for i in range(2)]
    want = [c.run(lib) for c in cs]
    streams, ws, dev = [torch.cuda.Stream() for _ in cs], [lib.new_cache_workspace(8, 2, 128, DEV) for _ in cs], [c.device() for c in cs]
    args = [(c.q.to(DEV), _i32(c.cu), _i32(c.kv), _i32(c.table)) for c in cs]
    outs = [torch.full_like(w, 7.0) for w in want]
    torch.cuda.synchronize()
    for _ in range(50):
        for i in range(2):
            q, cu, kv, tb = args[i]
            lib.bs_cache_attention(q, cu, kv, tb, None, *dev[i], 6, cs[i].scale, outs[i], None, ws[i], stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(outs[i], want[i])


def test_captured_graph_follows_lengths_on_the_device(lib):
    a, b = Case(16, [900, 64], [3, 5], 8, 2, 64, 32), Case(17, [17, 1300], [4, 2], 8, 2, 64, 32)
    want = [a.run(lib), b.run(lib)]
    nb, W, T = max(x.codes[0].shape[0] for x in (a, b)), max(x.table.shape[1] for x in (a, b)), max(a.T, b.T)
    kc, ks = lib.new_cache(nb, 2, 32, 64)
    vc, vs = lib.new_cache(nb, 2, 32, 64)
    q, out = torch.zeros(T, 8, 64, dtype=torch.bfloat16, device=DEV), torch.zeros(T, 8, 64, dtype=torch.bfloat16, device=DEV)
    cu, kv, table = _i32([0, 0, 0]), _i32([0, 0]), torch.zeros(2, W, dtype=torch.int32, device=DEV)
    ws = lib.new_cache_workspace(8, 2, 64, DEV)

    def step():
        lib.bs_cache_attention(q, cu, kv, table, None, kc, ks, vc, vs, 5, a.scale, out, None, ws)

    step()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]   # two graphs that share a workspace, replayed in turn
    for g in graphs:
        with torch.cuda.graph(g):
            step()
    for rep in range(6):
        x = (a, b)[rep % 2]
        dev = x.device()
        for dst, src in ((kc.view(torch.uint8), dev[0].view(torch.uint8)), (ks, dev[1]), (vc.view(torch.uint8), dev[2].view(torch.uint8)), (vs, dev[3])):
            dst[:src.shape[0]] = src
        q[:x.T] = x.q.to(DEV)
        cu.copy_(_i32(x.cu))
        kv.copy_(_i32(x.kv))
        table[:, :x.table.shape[1]] = _i32(x.table)
        out.fill_(7.0)
        graphs[rep // 3].replay()
        torch.cuda.synchronize()
        assert torch.equal(out[:x.T], want[rep % 2])


def test_long_cache_block_offsets_beyond_32_bits(lib):
    nb, H, bt, d = 140000, 2, 128, 128                    # 4.6e9 bytes of codes for K
    kc = torch.zeros(nb, H, bt, d, dtype=torch.uint8, device=DEV)
    vc = torch.zeros(nb, H, bt, d, dtype=torch.uint8, device=DEV)
    ks, vs = torch.ones(nb, H, device=DEV), torch.ones(nb, H, device=DEV)
    c = Case(18, [300], [2], 8, H, d, bt)
    far = [nb - 1, nb - 7, 139000]
    for j in range(3):
        for dst, src in ((kc, c.codes[0]), (vc, c.codes[1])):
            dst[far[j]] = torch.tensor(src[c.table[0, j]], device=DEV)
        for dst, src in ((ks, c.scales[0]), (vs, c.scales[1])):
            dst[far[j]] = torch.tensor(src[c.table[0, j]], device=DEV)
    want = c.run(lib)
    c.table[0, :3] = far
    got = c.run(lib, dev=(kc, ks, vc, vs))
    assert torch.equal(got, want)
    x = torch.randn(2, H, d, device=DEV, dtype=torch.bfloat16)
    slots = _i32([far[0] * bt + 5, far[0] * bt + 6])
    lib.bs_cache_append(x, x, slots, kc, ks, vc, vs)
    y = kc[far[0], :, 5:7].view(torch.float8_e4m3fn).float() * ks[far[0]][:, None, None]
    assert (y - x.float().transpose(0, 1)).abs().max() <= x.float().abs().max() * 2.0 ** -4


# ---- append --------------------------------------------------------------------------------------

def _append_case(lib, seed, runs, H, d, bt, dtype, mul=None, fused=False):
    """runs: (block, offset, count) in order; a negative block: `count` skipped tokens."""
    rng = np.random.default_rng(seed)
    nb = max(r[0] for r in runs) + 3
    slots = np.concatenate([np.full(n, blk) if blk < 0 else blk * bt + off + np.arange(n) for blk, off, n in runs])
    T = len(slots)
    x = torch.randn(2, T, H, d, generator=torch.Generator().manual_seed(seed), dtype=torch.float32)
    x *= torch.tensor(np.exp(2 * rng.normal(size=(2, T, 1, 1))), dtype=torch.float32) if mul is None else mul
    x = x.to(dtype)
    codes = [oc.encode(rng.normal(size=(nb, H, bt, d)) * 100) for _ in range(2)]
    scales = [(2.0 ** rng.integers(-9, -3, (nb, H))).astype(np.float32) for _ in range(2)]
    dev = [torch.tensor(c, device=DEV) for c in codes], [torch.tensor(s, device=DEV) for s in scales]
    if fused:                                             # heads of q, k and v side by side
        big = torch.zeros(T, 4 * H, d, dtype=dtype, device=DEV)
        big[:, 2 * H:3 * H], big[:, 3 * H:] = x[0].to(DEV), x[1].to(DEV)
        k, v = big[:, 2 * H:3 * H], big[:, 3 * H:]
    else:
        k, v = x[0].to(DEV), x[1].to(DEV)
    return x, slots, codes, scales, dev, k, v


def _append_check(lib, x, slots, codes, scales, dev, k, v, bt):
    (kc, vc), (ks, vs) = dev
    lib.bs_cache_append(k, v, _i32(slots), kc, ks, vc, vs)
    torch.cuda.synchronize()
    for i, (c, s) in enumerate(((kc, ks), (vc, vs))):
        want_c, want_s = codes[i].copy(), scales[i].copy()
        oc.append(x[i].double().numpy(), slots, want_c, want_s, bt)
        assert np.array_equal(s.cpu().numpy(), want_s), i
        got = c.cpu().numpy()
        nan = (got & 0x7F) == 0x7F
        assert np.array_equal(nan, (want_c & 0x7F) == 0x7F) and np.array_equal(got[~nan], want_c[~nan]), i


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bt", [16, 32, 64, 128])
def test_append_runs(lib, dtype, d, bt):
    runs = [(3, 0, 1), (1, 5, 3), (-1, 0, 2), (0, 0, bt), (5, bt - 1, 1), (6, 0, 7), (8, 0, bt), (9, 0, bt // 2 + 1), (4, 3, bt - 3), (-1, 0, 5)]
    a = _append_case(lib, bt + d, runs, 3, d, bt, dtype, fused=True)
    _append_check(lib, *a, bt)


def test_append_one_token(lib):
    _append_check(lib, *_append_case(lib, 1, [(0, 0, 1)], 1, 128, 16, torch.bfloat16), 16)
    _append_check(lib, *_append_case(lib, 2, [(2, 15, 1)], 8, 64, 16, torch.bfloat16), 16)


@pytest.mark.parametrize("H", [2, 4, 8])
@pytest.mark.parametrize("bt", [16, 128])
def test_append_many_tokens(lib, bt, H):
    """A group of warps looks after 4 tokens, 8, or a block's worth of them; runs that cross its borders."""
    runs, blk = [], 0
    rng = np.random.default_rng(bt)
    while sum(r[2] for r in runs) < 4500:
        n, off = int(rng.integers(1, 300)), int(rng.integers(0, bt))
        while n:
            m = min(n, bt - off)
            runs.append((blk, off, m))
            blk, off, n = blk + 1, 0, n - m
    _append_check(lib, *_append_case(lib, bt, runs, H, 64, bt, torch.bfloat16), bt)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_append_special_values(lib, dtype):
    runs = [(0, 0, 4), (1, 2, 4), (2, 0, 3), (3, 1, 2)]
    a = _append_case(lib, 5, runs, 2, 64, 16, dtype)
    x, k, v = a[0], a[5], a[6]
    for i, val in enumerate((float("inf"), float("-inf"), float("nan"), 3.0e38, 0.0, -0.0, 1e-38, 1e-30)):
        x[0, i % 13, 0, i] = val
        x[1, (i * 5) % 13, 1, 63 - i] = val
    x[:, 8:11] = 0.0                                      # a block of zeros
    k.copy_(x[0])
    v.copy_(x[1])
    _append_check(lib, *a, 16)


def test_append_slots_outside_the_cache_are_skipped(lib):
    a = list(_append_case(lib, 6, [(0, 0, 3), (1, 0, 2)], 2, 64, 16, torch.bfloat16))
    a[1] = a[1].copy()
    a[1][3:] = [2 ** 31 - 1, a[2][0].shape[0] * 16]
    _append_check(lib, *a, 16)


def test_append_misaligned_views_are_refused(lib):
    kc, ks = lib.new_cache(2, 1, 16, 64)
    x = torch.zeros(3, 1, 68, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(lib.BanditSpecError):
        lib.bs_cache_append(x[:, :, :64], x[:, :, :64], _i32([0, 1, 2]), kc, ks, kc.clone(), ks.clone())
    with pytest.raises(AssertionError):
        y = torch.zeros(3, 64, 1, dtype=torch.bfloat16, device=DEV).transpose(1, 2)[:, :, ::1]
        lib.bs_cache_append(torch.zeros(3, 1, 128, device=DEV)[:, :, ::2], y, _i32([0, 1, 2]), kc, ks, kc, ks)


# ---- plan ------------------------------------------------------------------------------------------

class Plan:
    def __init__(self, rng, B, bt, W, n_blocks, max_len):
        self.bt = bt
        self.seq = rng.integers(0, max_len + 1, B)
        self.held = np.minimum(W, -(-self.seq // bt) + rng.integers(0, 3, B))
        self.held = np.maximum(self.held, -(-self.seq // bt))
        order = rng.permutation(n_blocks)
        self.table = np.full((B, W), -1)
        at = 0
        for b in range(B):
            self.table[b, :self.held[b]] = order[at:at + self.held[b]]
            at += self.held[b]
        self.free = [int(x) for x in order[at:]]
        self.n_blocks = n_blocks

    def check(self, lib, kept, new, extra, active, T):
        B = len(self.seq)
        dev = dict(seq=_i32(self.seq), table=_i32(self.table), held=_i32(self.held), n_free=_i32([len(self.free)]),
                   free=_i32(self.free + [-1] * (self.n_blocks - len(self.free))))
        o = {n: torch.full((k,), -77, dtype=torch.int32, device=DEV)
             for n, k in (("kv_len", B), ("cu_new", B + 1), ("slot_map", T), ("positions", T), ("status", B))}
        act = None if active is None else torch.tensor(active, dtype=torch.uint8, device=DEV)
        lib.bs_cache_plan(dev["seq"], None if kept is None else _i32(kept), _i32(new), extra, act, self.bt, dev["table"], dev["held"],
                          dev["free"], dev["n_free"], o["kv_len"], o["cu_new"], o["slot_map"], o["positions"], o["status"])
        torch.cuda.synchronize()
        r = oc.plan(self.seq, kept, new, extra, active, self.bt, self.table, self.held, self.free, T)
        for n in o:
            assert np.array_equal(o[n].cpu().numpy(), r[n]), n
        assert np.array_equal(dev["seq"].cpu().numpy(), r["seq_len"])
        assert np.array_equal(dev["held"].cpu().numpy(), r["held"])
        assert np.array_equal(dev["table"].cpu().numpy(), r["table"])
        nf = int(dev["n_free"].item())
        assert nf == len(r["free"]) and dev["free"][:nf].cpu().tolist() == [int(x) for x in r["free"]]
        self.seq, self.table, self.held, self.free = r["seq_len"], r["table"], r["held"], r["free"]
        return r


@pytest.mark.parametrize("B,bt", [(1, 16), (3, 128), (64, 16), (700, 32), (1025, 16), (4096, 64)])
def test_plan_rounds(lib, B, bt):
    rng = np.random.default_rng(B)
    p = Plan(rng, B, bt, 40, B * 42 + 5, 20 * bt)
    kept = None
    for _ in range(6):
        new = rng.integers(0, 9, B)
        act = (rng.random(B) < 0.9).astype(np.uint8) if B > 3 else None
        r = p.check(lib, kept, new, 1, act, int(new.sum()) + B + 3)
        assert not (r["status"] & lib.BS_DEV_NO_BLOCKS).any()
        got = r["cu_new"][1:] - r["cu_new"][:-1]
        kept = np.where(got > 0, rng.integers(0, 10, B) % np.maximum(got, 1) + 1, 0)


def test_plan_large_slot_maps(lib):
    rng = np.random.default_rng(5)
    p = Plan(rng, 90, 16, 200, 90 * 100, 0)
    new = rng.integers(0, 1500, 90)
    p.check(lib, None, new, 0, None, int(new.sum()) + 777)
    p.check(lib, new, np.zeros(90, int), 0, None, 20000)  # they are kept; surplus is given back
    p.seq[::2] = 0                                        # half of the sequences end
    p.check(lib, None, np.where(np.arange(90) % 2, 1, 0), 0, None, 9000)


@pytest.mark.parametrize("T", [64, 9000])
def test_plan_runs_out_of_blocks_and_of_room(lib, T):
    rng = np.random.default_rng(T)
    for _ in range(8):
        p = Plan(rng, 40, 16, 30, 40 * 12, 100)
        p.free = p.free[:int(rng.integers(0, 30))]
        r = p.check(lib, None, rng.integers(0, 60, 40), 1, None, T)
        assert (r["status"] & (lib.BS_DEV_NO_BLOCKS | lib.BS_DEV_NO_ROOM)).any()


def test_plan_flags_bad_lengths(lib):
    rng = np.random.default_rng(7)
    p = Plan(rng, 8, 16, 10, 200, 100)
    p.seq[1], p.seq[3] = -1, p.held[3] * 16 + 1
    p.held[5] = 11
    new = np.array([1, 1, 1, 1, -4, 1, 170, 2])
    r = p.check(lib, None, new, 0, None, 300)
    assert r["status"].tolist() == [0, 64, 0, 64, 64, 64, 64, 0]


def test_plan_given_back_restores_the_stack(lib):
    rng = np.random.default_rng(8)
    p = Plan(rng, 50, 16, 30, 50 * 30, 200)
    p.check(lib, None, np.zeros(50, int), 0, None, 8)     # nobody holds more than it needs
    free, table = list(p.free), p.table.copy()
    p.check(lib, None, rng.integers(0, 100, 50), 1, None, 6000)
    p.check(lib, None, np.zeros(50, int), 0, None, 8)
    assert p.free == free and np.array_equal(p.table, table)


# ---- keep path ---------------------------------------------------------------------------------------

@pytest.mark.parametrize("d,bt", [(64, 16), (128, 16), (128, 32), (64, 128), (128, 64)])
def test_keep_path(lib, d, bt):
    rng = np.random.default_rng(d + bt)
    B, N, H = 24, 31, 3
    base = rng.integers(0, 3 * bt, B)
    paths = []
    for b in range(B):
        tau = int(rng.integers(0, N + 1)) if b else N
        paths.append(sorted(rng.choice(np.arange(1, N + 1), tau, replace=False).tolist()))
    W = (3 * bt + 33) // bt + 2
    table = rng.permutation(B * W).reshape(B, W)
    codes = [oc.encode(rng.normal(size=(B * W, H, bt, d)) * 100) for _ in range(2)]
    scales = [(2.0 ** rng.integers(-14, 3, (B * W, H))).astype(np.float32) for _ in range(2)]
    dev_c, dev_s = [torch.tensor(c, device=DEV) for c in codes], [torch.tensor(s, device=DEV) for s in scales]
    nodes = np.full((B, N), -1)
    for b, p in enumerate(paths):
        nodes[b, :len(p)] = p
    st = torch.zeros(B, dtype=torch.int32, device=DEV)
    lib.bs_cache_keep_path(_i32(nodes), _i32([len(p) for p in paths]), _i32(base), _i32(table), dev_c[0], dev_s[0], dev_c[1], dev_s[1], st)
    torch.cuda.synchronize()
    assert not st.any()
    for i in range(2):
        for b in range(B):
            oc.keep_path(paths[b], int(base[b]), table[b], codes[i], scales[i], bt)
        assert np.array_equal(dev_s[i].cpu().numpy(), scales[i])
        assert np.array_equal(dev_c[i].cpu().numpy(), codes[i])


def test_keep_path_leaves_bad_sequences_alone(lib):
    B, N, W = 7, 6, 3
    table = np.arange(B * W).reshape(B, W)
    table[4, 1] = B * W
    nodes = np.array([[2, 5, -1, -1, -1, -1]] * B)
    nodes[1, :2] = [5, 2]                                 # not ascending
    nodes[2, :2] = [2, 7]                                 # no such node
    acc, base = np.array([2, 2, 2, -1, 2, 2, 2]), np.array([10, 10, 10, 10, 10, -1, 43])
    kc, ks = lib.new_cache(B * W, 1, 16, 64)
    kc = torch.randint(0, 127, kc.shape, device=DEV, dtype=torch.uint8)
    vc, was = kc.clone(), kc.clone()
    st = torch.zeros(B, dtype=torch.int32, device=DEV)
    lib.bs_cache_keep_path(_i32(nodes), _i32(acc), _i32(base), _i32(table), kc, ks, vc, ks.clone(), st)
    # sequence 4 moves positions 12 and 15 to 11 and 12: all in its first block, the bad second one is not touched
    assert st.tolist() == [0, lib.BS_DEV_BAD_TREE, lib.BS_DEV_BAD_TREE, lib.BS_DEV_BAD_LENGTH, 0, lib.BS_DEV_BAD_LENGTH,
                           lib.BS_DEV_BAD_LENGTH]
    same = (kc == was).flatten(1).all(1).view(B, W)
    assert same[[1, 2, 3, 5, 6]].all() and not same[0, 0] and not same[4, 0] and same[4, 1:].all()


def test_keep_path_flags_bad_blocks(lib):
    table = np.arange(6).reshape(2, 3)
    table[0, 1], table[1, 1] = 6, -1
    kc, ks = torch.randint(0, 127, (6, 2, 16, 128), device=DEV, dtype=torch.uint8), torch.ones(6, 2, device=DEV)
    was, st = kc.clone(), _i32([lib.BS_DEV_BAD_TREE, 0])  # bits are added to what is there
    # sources at 15 and 18, destinations at 14 and 15: the second source lies in a bad block
    nodes = _i32([[2, 5, -1, -1, -1]] * 2)
    lib.bs_cache_keep_path(nodes, _i32([2, 2]), _i32([13, 13]), _i32(table), kc, ks, kc.clone(), ks.clone(), st)
    assert st.tolist() == [lib.BS_DEV_BAD_TREE | lib.BS_DEV_BAD_BLOCK, lib.BS_DEV_BAD_BLOCK]
    assert torch.equal(kc, was)


# ---- rounds ----------------------------------------------------------------------------------------------

@pytest.mark.parametrize("tree", [False, True])
def test_rounds_end_to_end(lib, tree):
    """Prompt, then rounds as a decoder runs them: arms -> plan -> append -> attention -> verification -> path -> plan.
    A shadow of every kept token's keys and values in order is what the cache has to stand for."""
    B, V, Hq, Hkv, d, bt, rounds = 5, 512, 8, 2, 64, 16, 6
    g = torch.Generator(device=DEV).manual_seed(11)
    rng = np.random.default_rng(11)
    shapes = [[0, 1, 2], [0, 0, 1, 1, 2, 2], [0, 0, 0]]
    Nmax = 6
    arms = [len(s) for s in shapes] if tree else [1, 4, 6]
    state = lib.new_bandit(lib.BS_UCB, B, arms, device=DEV)
    nb, W = 200, 30
    order = rng.permutation(nb)
    seq_len, held, table = _i32([0] * B), _i32([0] * B), _i32(np.full((B, W), -1))
    free, n_free = _i32(order), _i32([nb])
    caches = lib.new_cache(nb, Hkv, bt, d) + lib.new_cache(nb, Hkv, bt, d)
    T = 200
    e = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)  # noqa: E731
    kv_len, cu, slots, pos, status = e(B), e(B + 1), e(T), e(T), e(B)
    ws, vws = lib.new_cache_workspace(Hq, Hkv, d, DEV), lib.new_workspace(B, Nmax, V, DEV)
    shadow = [[] for _ in range(B)]                       # kept (k, v) of every sequence
    prompt = [20, 1, 33, 16, 7]
    kept = None

    def step(n_new, extra, parent):
        lib.bs_cache_plan(seq_len, kept, n_new, extra, None, bt, table, held, free, n_free, kv_len, cu, slots, pos, status)
        k, v = (torch.randn(T, Hkv, d, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
        q = (2 * torch.randn(T, Hq, d, generator=g, device=DEV)).to(torch.bfloat16)
        out = torch.full((T, Hq, d), 7.0, dtype=torch.bfloat16, device=DEV)
        lib.bs_cache_append(k, v, slots, *caches)
        lib.bs_cache_attention(q, cu, kv_len, table, parent, *caches, 7, d ** -0.5, out, status, ws)
        torch.cuda.synchronize()
        assert not status.any()
        c, L, c0 = cu.cpu().numpy(), kv_len.cpu().numpy(), seq_len.cpu().numpy()
        want_pos = np.concatenate([c0[b] + np.arange(c[b + 1] - c[b]) for b in range(B)])
        assert np.array_equal(pos.cpu().numpy()[:c[-1]], want_pos)
        x = Case.__new__(Case)                            # the cache as it is, checked like any other
        x.ctx, x.new, x.bt, x.d, x.Hq, x.Hkv = list(c0), list(c[1:] - c[:-1]), bt, d, Hq, Hkv
        x.kv, x.cu, x.T, x.q, x.scale = [int(l) for l in L], c, T, q.cpu(), d ** -0.5
        x.table = table.cpu().numpy()
        x.codes = [caches[0].view(torch.uint8).cpu().numpy(), caches[2].view(torch.uint8).cpu().numpy()]
        x.scales = [caches[1].cpu().numpy(), caches[3].cpu().numpy()]
        x.parent = None if parent is None else parent.cpu().numpy()
        x.check(out)
        return k.float().cpu().numpy(), v.float().cpu().numpy(), c

    def check_shadow():
        tb, L = table.cpu().numpy(), seq_len.cpu().numpy()
        for b in range(B):
            assert len(shadow[b]) == L[b]
            for t, rows in enumerate(shadow[b]):
                blk, off = tb[b, t // bt], t % bt
                for i in range(2):
                    s = caches[2 * i + 1][blk].cpu().numpy()[:, None]
                    y = caches[2 * i][blk, :, off].float().cpu().numpy() * s
                    assert (np.abs(y - rows[i]) <= np.maximum(np.abs(rows[i]) * 2.0 ** -4, s * 2.0 ** -10)).all()

    k, v, c = step(_i32(prompt), 0, None)
    for b in range(B):
        shadow[b] += [(k[i], v[i]) for i in range(c[b], c[b + 1])]
    kept = _i32(prompt)
    arm, gamma, u = e(B), e(B), torch.rand(B, device=DEV, generator=g)
    acc, on, ot, ol = e(B), e(B, Nmax), e(B, Nmax + 1), e(B)
    sp, sn = _i32([s + [0] * (Nmax - len(s)) for s in shapes]), _i32([len(s) for s in shapes])
    parent, nn = e(B, Nmax), e(B)
    moved = 0
    for _ in range(rounds):
        lib.bs_bandit_select(state, lib.BS_UCB, B, 3, None, None, arm, gamma)
        target = torch.randn(B, Nmax + 1, V, generator=g, device=DEV)
        if tree:
            lib.bs_tree_expand_shapes(sp, sn, arm, parent, nn)
            best = target.argmax(2)
            up = best.gather(1, parent.long())
            rnd = torch.randint(0, V, (B, Nmax), generator=g, device=DEV)
            tokens = torch.where(torch.rand(B, Nmax, device=DEV, generator=g) < 0.6, up, rnd).to(torch.int32)
            k, v, c = step(nn, 1, parent)
            lib.bs_tree_verify_greedy(target, parent, tokens, nn, acc, on, ot, ol, vws)
            lib.bs_cache_keep_path(on, acc, seq_len, table, *caches, status)
        else:
            tokens = torch.where(torch.rand(B, Nmax, device=DEV, generator=g) < 0.7, target.argmax(2)[:, :Nmax], 3).to(torch.int32)
            k, v, c = step(gamma, 1, None)
            lib.bs_softmax_verify(target, None, tokens, gamma, None, 0.0, acc, None, None, vws)
            lib.bs_residual_sample(target, None, tokens, gamma, acc, None, 0.0, ot, ol, vws)
        lib.bs_bandit_update(state, lib.BS_UCB, B, 3, arm, ol)
        torch.cuda.synchronize()
        assert not status.any()
        tau, path = acc.cpu().numpy(), on.cpu().numpy()
        for b in range(B):
            rows = [0] + (path[b, :tau[b]].tolist() if tree else list(range(1, tau[b] + 1)))
            moved += rows != list(range(len(rows)))
            shadow[b] += [(k[c[b] + r], v[c[b] + r]) for r in rows]
        kept = ol.clone()
    lib.bs_cache_plan(seq_len, kept, e(B), 0, None, bt, table, held, free, n_free, kv_len, cu, slots, pos, status)
    check_shadow()
    assert moved > 0 or not tree
    seq_len.zero_()                                       # all sequences end: every block comes back
    lib.bs_cache_plan(seq_len, None, e(B), 0, None, bt, table, held, free, n_free, kv_len, cu, slots, pos, status)
    assert n_free.item() == nb and sorted(free.tolist()) == list(range(nb)) and not held.any()
