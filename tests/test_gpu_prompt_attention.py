"""bs_prompt_attention on the GPU against attention in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import prompt as op

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _cu(n):
    return torch.tensor(np.concatenate([[0], np.cumsum(n)]).tolist(), dtype=torch.int32, device=DEV)


def _inputs(n, Hq, Hkv, d, seed, spread=2.0, extra=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    qkv = torch.randn(sum(n) + extra, Hq + 2 * Hkv, d, generator=g, device=DEV)
    qkv[:, :Hq] *= spread
    qkv = qkv.to(torch.bfloat16)
    return qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]


def _exact(q, k, v, n, scale):
    """out, sum p |v| and the largest sum |q_c k_c| of every row, in fp64, head by head."""
    G = q.shape[1] // k.shape[1]
    out, size = torch.zeros(q.shape, dtype=torch.float64, device=DEV), torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    reach = torch.zeros(q.shape[:2], dtype=torch.float64, device=DEV)
    lo = 0
    for m in n:
        for h in range(q.shape[1]):
            a, b, c = q[lo:lo + m, h].double(), k[lo:lo + m, h // G].double(), v[lo:lo + m, h // G].double()
            see = torch.ones(m, m, dtype=torch.bool, device=DEV).tril()
            p = torch.softmax((a @ b.T * scale).masked_fill(~see, float("-inf")), 1) if m else a.new_zeros(0, 0)
            out[lo:lo + m, h], size[lo:lo + m, h] = p @ c, p @ c.abs()
            reach[lo:lo + m, h] = (a.abs() @ b.abs().T * scale).masked_fill(~see, 0.0).amax(1) if m else 0.0
        lo += m
    return out, size, reach


def _check(got, q, k, v, n, scale):
    """A probability is rounded to bf16 (2^-8), the result again; a score is off by at most 2^-21 of its sum of magnitudes (products
    in the tensor cores: 2^-22, scaling: 2^-23), which changes a probability, and the sum of them, by as much; the exponential and
    the sums of up to 2^14 terms add 2^-13 at most."""
    out, size, reach = _exact(q, k, v, n, scale)
    T = sum(n)
    tol = 2.0 ** -8 * out.abs() + (2.0 ** -8 + 2.0 ** -13 + 2 * 2.0 ** -21 * reach[..., None]) * size
    err = (got.double() - out).abs()[:T]
    bad = ~(err <= 1.01 * tol[:T])
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist(), float((err / tol[:T]).nan_to_num(1e9).max()))


CASES = [([1], 1, 1, 128), ([1], 8, 1, 64), ([5], 4, 4, 64), ([128], 1, 1, 128), ([129], 1, 1, 128), ([127, 1, 0, 130], 2, 1, 64), ([256], 2, 2, 128),
         ([257], 1, 1, 64), ([300, 7, 64, 513], 8, 2, 128), ([1000], 7, 1, 128), ([65, 200], 28, 4, 64), ([640], 64, 1, 64), ([33, 385], 48, 1, 128),
         ([2049], 4, 1, 128), ([1] * 70, 4, 2, 64), ([0, 0, 3], 3, 3, 128), ([1500, 2], 16, 16, 64), ([700, 699], 5, 1, 128)]


@pytest.mark.parametrize("n,Hq,Hkv,d", CASES)
def test_attention(lib, n, Hq, Hkv, d):
    q, k, v = _inputs(n, Hq, Hkv, d, seed=sum(n) + Hq)
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    status = torch.zeros(len(n), dtype=torch.int32, device=DEV)
    lib.bs_prompt_attention(q, k, v, _cu(n), d ** -0.5, out, status)
    assert not status.any()
    _check(out, q, k, v, n, d ** -0.5)


def test_against_the_plain_oracle(lib):
    n, Hq, Hkv, d = [3, 40, 1, 130], 4, 2, 64
    q, k, v = _inputs(n, Hq, Hkv, d, seed=3)
    out = torch.zeros(q.shape, dtype=torch.bfloat16, device=DEV)
    lib.bs_prompt_attention(q, k, v, _cu(n), 0.2, out)
    want, size = op.attention(*(x.double().cpu().numpy() for x in (q, k, v)), _cu(n).tolist(), 0.2)
    assert (np.abs(out.double().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -12) * size).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("spread,shift", [(40.0, 0.0), (0.01, 0.0), (3.0, 30.0)])
def test_scores_that_grow(lib, d, spread, shift):
    """Maxima that move far and often, that hardly differ, that drift along the keys."""
    n = [900, 130]
    q, k, v = _inputs(n, 4, 2, d, seed=11, spread=spread)
    if shift:
        k = k.clone()
        k[:, :, 0] += shift * torch.arange(sum(n), device=DEV, dtype=torch.float32)[:, None].to(torch.bfloat16) / 100
        q = q.clone()
        q[:, :, 0] = 2.0
    out = torch.zeros(q.shape, dtype=torch.bfloat16, device=DEV)
    lib.bs_prompt_attention(q, k, v, _cu(n), d ** -0.5, out)
    _check(out, q, k, v, n, d ** -0.5)


@pytest.mark.parametrize("layout", ["heads first", "padded rows", "contiguous"])
def test_layouts(lib, layout):
    n, Hq, Hkv, d = [200, 77], 4, 2, 64
    q, k, v = _inputs(n, Hq, Hkv, d, seed=4)
    def lay(x):
        if layout == "heads first":
            return x.transpose(0, 1).contiguous().transpose(0, 1)
        if layout == "padded rows":
            y = torch.zeros(x.shape[0], x.shape[1] + 3, d + 8, dtype=x.dtype, device=DEV)
            y[:, 1:1 + x.shape[1], :d] = x
            return y[:, 1:1 + x.shape[1], :d]
        return x.contiguous()
    base = torch.zeros(q.shape, dtype=torch.bfloat16, device=DEV)
    lib.bs_prompt_attention(q, k, v, _cu(n), 0.125, base)
    out = lay(torch.zeros(q.shape, dtype=torch.bfloat16, device=DEV))
    lib.bs_prompt_attention(lay(q), lay(k), lay(v), _cu(n), 0.125, out)
    assert torch.equal(out, base)


def test_rows_behind_the_sequences_and_strange_neighbours(lib):
    """Rows behind the last sequence stay; what they hold, and what other sequences hold, does not matter."""
    n, Hq, Hkv, d = [130, 40, 300], 4, 2, 128
    q, k, v = (x.clone() for x in _inputs(n, Hq, Hkv, d, seed=6, extra=100))
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    lib.bs_prompt_attention(q, k, v, _cu(n), d ** -0.5, out)
    assert (out[sum(n):] == 7.0).all()
    want = out.clone()
    for x in (q, k, v):
        x[sum(n):] = float("nan")
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    lib.bs_prompt_attention(q, k, v, _cu(n), d ** -0.5, out)
    assert torch.equal(out, want)
    for x in (q, k, v):
        x[130:170] = float("inf")                             # the second sequence
    lib.bs_prompt_attention(q, k, v, _cu(n), d ** -0.5, out)
    assert torch.equal(out[:130], want[:130]) and torch.equal(out[170:470], want[170:470])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("at", [0, 5, 127, 128, 300, 399])
def test_later_tokens_leave_no_trace(lib, d, at):
    """NaN and infinities in a token's key and value reach the rows that see it, and no other."""
    n, Hq, Hkv = [400], 4, 1
    q, k, v = (x.clone() for x in _inputs(n, Hq, Hkv, d, seed=8))
    want = torch.zeros(q.shape, dtype=torch.bfloat16, device=DEV)
    lib.bs_prompt_attention(q, k, v, _cu(n), d ** -0.5, want)
    out = torch.zeros_like(want)
    v[at, 0, 3], v[min(at + 1, 399), 0, 60] = float("nan"), float("-inf")
    lib.bs_prompt_attention(q, k, v, _cu(n), d ** -0.5, out)
    clean = torch.ones(d, dtype=torch.bool, device=DEV)
    clean[[3, 60]] = False
    assert torch.equal(out[..., clean], want[..., clean])
    assert torch.equal(out[:at], want[:at]) and not torch.isfinite(out[at:, :, 3]).any()
    second = min(at + 1, 399)
    assert torch.equal(out[:second, :, 60], want[:second, :, 60]) and not torch.isfinite(out[second:, :, 60]).any()
    k[at] = float("nan")
    lib.bs_prompt_attention(q, k, v, _cu(n), d ** -0.5, out)
    assert torch.equal(out[:at], want[:at]) and torch.isnan(out[at:]).all()


def test_scores_of_minus_infinity(lib):
    """Keys that score -inf have no weight, in the first tile as in a later one; a row that sees nothing else is NaN."""
    n, d = [300], 64
    q, k, v = (x.clone() for x in _inputs(n, 1, 1, d, seed=9))
    q[:, :, 0] = 1.0
    k[:150, :, 0] = float("-inf")
    k[200:210, :, 0] = float("-inf")
    out = torch.zeros(q.shape, dtype=torch.bfloat16, device=DEV)
    lib.bs_prompt_attention(q, k, v, _cu(n), 0.125, out)
    assert torch.isnan(out[:150]).all()
    keep = [j for j in range(300) if j >= 150 and not 200 <= j < 210]
    t = (q[:, 0].double() @ k[keep, 0].double().T * 0.125)
    see = torch.tensor(keep, device=DEV)[None] <= torch.arange(300, device=DEV)[:, None]
    p = torch.softmax(t.masked_fill(~see, float("-inf")), 1)[150:]
    want, size = p @ v[keep, 0].double(), p @ v[keep, 0].double().abs()
    assert ((out[150:, 0].double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -12) * size).all()


def test_bad_lengths(lib):
    n, d = [100, 50, 60], 64
    q, k, v = _inputs(n, 2, 1, d, seed=10)
    want = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    lib.bs_prompt_attention(q, k, v, _cu(n), 0.125, want)
    T = sum(n)

    def call(cu):
        out, status = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV), torch.zeros(len(cu) - 1, dtype=torch.int32, device=DEV)
        lib.bs_prompt_attention(q, k, v, torch.tensor(cu, dtype=torch.int32, device=DEV), 0.125, out, status)
        return out, [s == lib.BS_DEV_BAD_LENGTH for s in status.tolist()], status.tolist()

    out, bad, raw = call([0, 100, 150, T + 1])
    assert bad == [False, False, True] and torch.equal(out[:150], want[:150]) and (out[150:] == 7.0).all()
    out, bad, raw = call([0, 100, 60, T])
    assert bad == [False, True, True] and torch.equal(out[:100], want[:100])     # 100 + 150 tokens of 210
    out, bad, raw = call([-5, 100, 150, T])
    assert bad == [True, False, False] and (out[:100] == 7.0).all() and torch.equal(out[100:], want[100:])
    assert not any(s for s, b in zip(raw, bad) if not b)


def test_streams_graphs_and_repeats(lib):
    n, d = [513, 300, 1, 77], 128
    q, k, v = (x.contiguous() for x in _inputs(n, 8, 2, d, seed=12))
    cu = _cu(n)
    want = torch.zeros(q.shape, dtype=torch.bfloat16, device=DEV)
    lib.bs_prompt_attention(q, k, v, cu, d ** -0.5, want)
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in range(3)], [torch.zeros_like(want) for _ in range(3)]
    for s, o in zip(streams, outs):                           # several at once: no workspace is shared
        s.wait_stream(torch.cuda.current_stream())
        for _ in range(5):
            lib.bs_prompt_attention(q, k, v, cu, d ** -0.5, o, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    graph, out = torch.cuda.CUDAGraph(), torch.zeros_like(want)
    with torch.cuda.graph(graph):
        lib.bs_prompt_attention(q, k, v, cu, d ** -0.5, out)
    short = _cu([100, 2, 3, 500])                             # other lengths in the captured call's array
    cu.copy_(short)
    lib.bs_prompt_attention(q, k, v, cu, d ** -0.5, want.zero_())
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want) and (out[605:] == 0).all()


def test_long_prompt(lib):
    n, d = [9001], 128
    q, k, v = _inputs(n, 2, 1, d, seed=13)
    out = torch.zeros(q.shape, dtype=torch.bfloat16, device=DEV)
    lib.bs_prompt_attention(q, k, v, _cu(n), d ** -0.5, out)
    _check(out, q, k, v, n, d ** -0.5)


def test_reports_stay_within_the_batch(lib):
    """Sequences that overlap hold more tokens than there are: those are reported, and nothing behind the batch."""
    q, k, v = _inputs([210], 2, 1, 64, seed=14)
    around = torch.zeros(64, dtype=torch.int32, device=DEV)
    out = torch.zeros(q.shape, dtype=torch.bfloat16, device=DEV)
    lib.bs_prompt_attention(q, k, v, torch.tensor([0, 100, 60, 210], dtype=torch.int32, device=DEV), 0.125, out, around[8:11])
    assert around[8:11].tolist() == [0, lib.BS_DEV_BAD_LENGTH, lib.BS_DEV_BAD_LENGTH]
    assert not around[:8].any() and not around[11:].any()


def test_rows_that_two_sequences_claim(lib):
    """A sequence that begins before the end of an earlier one writes nothing, although there are tokens enough for both."""
    q, k, v = _inputs([210], 2, 1, 64, seed=15)
    want = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    lib.bs_prompt_attention(q, k, v, torch.tensor([0, 100], dtype=torch.int32, device=DEV), 0.125, want)
    out, status = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV)
    lib.bs_prompt_attention(q, k, v, torch.tensor([0, 100, 60, 90], dtype=torch.int32, device=DEV), 0.125, out, status)
    assert status.tolist() == [0, lib.BS_DEV_BAD_LENGTH, lib.BS_DEV_BAD_LENGTH] and torch.equal(out, want)


def _ragged(B, most, seed):
    rng = np.random.default_rng(seed)
    n = rng.integers(0, most, B)
    n[rng.random(B) < 0.15] = 0
    n[-1] = most                                              # the last of them has the most items
    return n.tolist()


# items of a call against the SMs: 4 x 148 are 592
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,Hq,Hkv", [(_ragged(60, 700, 1), 21, 3), (_ragged(100, 300, 2), 15, 3), (_ragged(45, 600, 3), 16, 16), ([3000], 40, 40),
                                      ([1200, 1], 128, 2), ([129] * 70, 8, 8), ([257, 1, 128] * 30, 12, 12)])
def test_ctas_that_take_many_items(lib, n, Hq, Hkv, d):
    """Three items and more a CTA: slots, barriers and rings are used again, over groups of 32 sequences and all lengths."""
    TQ = 128 // (Hq // Hkv)
    assert sum(-(-m // (2 * TQ)) for m in n) * Hkv > 3 * 148
    q, k, v = _inputs(n, Hq, Hkv, d, seed=sum(n) + Hq)
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    status = torch.zeros(len(n), dtype=torch.int32, device=DEV)
    lib.bs_prompt_attention(q, k, v, _cu(n), d ** -0.5, out, status)
    assert not status.any()
    _check(out, q, k, v, n, d ** -0.5)
    again = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    lib.bs_prompt_attention(q, k, v, _cu(n), d ** -0.5, again)
    assert torch.equal(out, again)


@pytest.mark.parametrize("d", [64, 128])
def test_bad_lengths_among_many_sequences(lib, d):
    """One in the second group of 32: its rows stay, all others are as without it."""
    n, Hq, Hkv = _ragged(60, 700, 4), 21, 3
    q, k, v = _inputs(n, Hq, Hkv, d, seed=16)
    cu, T = _cu(n), sum(n)
    want = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    lib.bs_prompt_attention(q, k, v, cu, d ** -0.5, want)
    cu[41] = T + 5                                            # 40 ends behind the tokens, 41 descends
    out, status = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV), torch.zeros(60, dtype=torch.int32, device=DEV)
    lib.bs_prompt_attention(q, k, v, cu, d ** -0.5, out, status)
    assert [b for b in range(60) if status[b]] == [40, 41]
    lo, hi = sum(n[:40]), sum(n[:42])
    assert hi > lo and (out[lo:hi] == 7.0).all()
    assert torch.equal(out[:lo], want[:lo]) and torch.equal(out[hi:], want[hi:])


def test_no_time_out_without_a_status_array(lib):
    q, k, v = _inputs([210], 2, 1, 64, seed=17)
    out = torch.zeros(q.shape, dtype=torch.bfloat16, device=DEV)
    lib.bs_prompt_attention(q, k, v, _cu([210]), 0.125, out)
    lib.bs_prompt_get_device_status()
    side = torch.cuda.Stream()
    lib.bs_prompt_attention(q, k, v, _cu([210]), 0.125, out, stream=side)
    lib.bs_prompt_get_device_status(q.device, side)
