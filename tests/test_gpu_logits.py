"""bs_logits_adjust and bs_history_update on the GPU against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import logits as ol

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _ints(v):
    return torch.tensor(np.asarray(v).tolist(), dtype=torch.int32, device=DEV)


def _round(B, R, V, dtype, seed, tree, lists=True, n_masks=3):
    """Everything at once, from a seed, as host arrays and as the arguments of a call."""
    rng = np.random.default_rng(seed)
    N = max(R - 1, 1)
    h = dict(gamma=rng.integers(0, R, B), drafted=rng.integers(0, min(V, 12), (B, N)),
             parent=np.array([[rng.integers(0, j + 1) for j in range(N)] for _ in range(B)]) if tree else None,
             history=(rng.random((B, V)) < 0.3) * rng.integers(0, 9, (B, V)),
             r=1 + rng.random(B), p=rng.normal(size=B), f=rng.normal(size=B))
    count = rng.integers(0, 80, B) if lists else np.zeros(B, int)
    h["begin"] = np.concatenate([[0], np.cumsum(count)])
    h["bt"] = rng.integers(0, V, count.sum())
    h["bt"][rng.random(count.sum()) < 0.4] = V - 1            # many times the same
    h["bv"] = rng.normal(size=count.sum()) * 3
    share = np.array([0.0, 0.5, 0.97])[np.arange(n_masks) % 3]
    h["allowed"] = rng.random((n_masks, V)) < share[:, None]
    h["row"] = rng.integers(-1, n_masks, (B, R))
    words = -(-V // 32)
    bits = np.zeros((n_masks, words * 32), np.uint64)
    bits[:, :V] = h["allowed"]
    packed = (bits.reshape(n_masks, words, 32) << np.arange(32, dtype=np.uint64)).sum(2).astype(np.uint32).view(np.int32)
    fl = lambda v: torch.tensor(v, dtype=torch.float32, device=DEV)  # noqa: E731
    x = torch.tensor(rng.normal(size=(B, R, V)) * 4, device=DEV).to(dtype)
    a = dict(draft_tokens=_ints(h["drafted"]), node_parent=None if h["parent"] is None else _ints(h["parent"]),
             history=torch.tensor(h["history"], dtype=torch.int16, device=DEV), repetition=fl(h["r"]), presence=fl(h["p"]), frequency=fl(h["f"]),
             bias_begin=_ints(h["begin"]), bias_tokens=_ints(h["bt"]), bias_values=fl(h["bv"]),
             masks=torch.tensor(packed, device=DEV), mask_row=_ints(h["row"]))
    for n in ("r", "p", "f"):
        h[n] = h[n].astype(np.float32).astype(np.float64)
    h["bv"] = h["bv"].astype(np.float32).astype(np.float64)
    return x, _ints(h["gamma"]), a, h


def _want(x, h, b, row, a, masks=True):
    on = [int(h["drafted"][b, n - 1]) for n in ol.path(None if h["parent"] is None else h["parent"][b], row)] if a.get("draft_tokens") is not None else []
    lo, hi = h["begin"][b], h["begin"][b + 1]
    bias = list(zip(h["bt"][lo:hi], h["bv"][lo:hi])) if a.get("bias_begin") is not None else []
    m = h["row"][b, row] if a.get("mask_row") is not None else -1
    pen = any(a.get(n) is not None for n in ("repetition", "presence", "frequency"))
    want = ol.adjust_row(x, h["history"][b] if pen and a.get("history") is not None else None, on if pen else (), h["r"][b] if a.get("repetition") is not None else 1.0,
                         h["p"][b] if a.get("presence") is not None else 0.0, h["f"][b] if a.get("frequency") is not None else 0.0, bias,
                         h["allowed"][m] if m >= 0 else None)
    # what the fp32 steps work on: a step is off by at most 2^-24 of the largest number it handles
    size = np.abs(x) * h["r"][b] + (np.abs(h["f"][b]) * (h["history"][b] // 2 + len(on)) + np.abs(h["p"][b]))
    steps = np.full(len(x), 4.0 + len(on))
    for t, v in bias:
        size[t] += abs(v)
        steps[t] += 1
    return want, size * steps * 2.0 ** -24


def _compare(out, x0, gamma, extra, rows, h, a, dtype, untouched):
    out, x0 = out.double().cpu().numpy(), x0.double().cpu().numpy()
    half = 2.0 ** -8 if dtype is torch.bfloat16 else 0.0      # fp32: its rounding is among the steps
    for b in range(out.shape[0]):
        for r in range(out.shape[1]):
            if not rows[0] <= r < min(rows[1], int(gamma[b]) + extra):
                assert np.array_equal(out[b, r], untouched[b, r]), (b, r)
                continue
            want, tol = _want(x0[b, r], h, b, r, a)
            masked = np.isinf(want)
            assert (out[b, r][masked] == -np.inf).all()
            err = np.abs(out[b, r][~masked] - want[~masked])
            bound = 1.01 * half * np.abs(want[~masked]) + tol[~masked] * 1.01
            assert (err <= bound).all(), (b, r, (err / bound).max())


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,R,V", [(1, 1, 1), (3, 5, 1000), (2, 9, 4096), (5, 16, 2051), (2, 32, 264), (4, 3, 7), (3, 4, 2049), (2, 2, 36)])
def test_adjust(lib, B, R, V, dtype, tree, in_place):
    x, gamma, a, h = _round(B, R, V, dtype, seed=V + R, tree=tree)
    out = x.clone() if in_place else torch.full_like(x, 3.0)
    before = out.clone().double().cpu().numpy()
    status = torch.zeros(B, dtype=torch.int32, device=DEV)
    lib.bs_logits_adjust(out if in_place else x, out, gamma, 1, status=status, **a)
    _compare(out, x, gamma, 1, (0, R), h, a, dtype, before)
    assert not status.any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("which", [("history", "repetition"), ("history", "presence"), ("history", "frequency"), ("draft_tokens", "frequency", "repetition"),
                                   ("bias_begin", "bias_tokens", "bias_values"), ("masks", "mask_row"), ("history",), ("draft_tokens",), ()])
def test_each_rule_alone(lib, which, dtype):
    B, R, V = 3, 6, 1544
    x, gamma, a, h = _round(B, R, V, dtype, seed=5, tree=False)
    a = {n: a[n] for n in which}
    for in_place in (False, True):
        out = x.clone() if in_place else torch.full_like(x, 3.0)
        before = out.double().cpu().numpy()
        lib.bs_logits_adjust(out if in_place else x, out, gamma, 1, **a)
        _compare(out, x, gamma, 1, (0, R), h, a, dtype, before)


def test_rows_of_drafting(lib):
    """Draft rows one position at a time (extra 0), and all rows without a gamma."""
    B, R, V = 4, 5, 520
    x, gamma, a, h = _round(B, R, V, torch.float32, seed=9, tree=False)
    for row in range(R):
        out = torch.full_like(x, 3.0)
        lib.bs_logits_adjust(x, out, gamma, 0, rows=(row, row + 1), **a)
        _compare(out, x, gamma, 0, (row, row + 1), h, a, torch.float32, np.full(x.shape, 3.0))
    out = torch.full_like(x, 3.0)
    lib.bs_logits_adjust(x, out, None, 0, **a)
    _compare(out, x, [R] * B, 0, (0, R), h, a, torch.float32, None)


def test_special_values(lib):
    V = 512
    x = torch.randn(1, 2, V, device=DEV)
    x[0, 0, :4] = torch.tensor([float("nan"), float("inf"), float("-inf"), float("nan")], device=DEV)
    x[0, 1] = x[0, 0]
    hist = torch.full((1, V), 5, dtype=torch.int16, device=DEV)
    masks = torch.full((2, V // 32), -1, dtype=torch.int32, device=DEV)
    masks[0, 0] = ~9                                          # tokens 0 and 3 forbidden
    masks[1] = 0                                              # nothing allowed
    out = torch.empty_like(x)
    one = torch.ones(1, device=DEV)
    lib.bs_logits_adjust(x, out, None, 0, history=hist, repetition=2 * one, presence=one, frequency=one, masks=masks, mask_row=_ints([[0, 1]]))
    got = out.cpu().numpy()
    assert got[0, 0, 0] == got[0, 0, 2] == got[0, 0, 3] == -np.inf and got[0, 0, 1] == np.inf
    assert np.isfinite(got[0, 0, 4:]).all() and (got[0, 1] == -np.inf).all()


def test_bad_data_is_reported_and_left_out(lib):
    B, R, V = 6, 4, 300
    x, gamma, a, h = _round(B, R, V, torch.float32, seed=3, tree=True)
    g = [3] * B
    g[0] = 9                                                  # outside
    a["draft_tokens"][1, 0] = V
    h["drafted"][1, 0] = V
    a["node_parent"][2, 1] = 2                                # itself
    h["parent"][2, 1] = 2
    a["mask_row"][3, 0] = 3
    h["row"][3, 0] = -1
    a["mask_row"][3, 2] = -2
    h["row"][3, 2] = -1
    h["begin"][5], h["begin"][6] = 0, len(h["bt"])            # of sequence 5: everything, with a token outside
    a["bias_tokens"][0] = -1
    h["bt"][0] = -1
    begin = h["begin"].copy()
    begin[4] = begin[5] + 1                                   # sequence 4 descends; sequence 3 gets what comes
    a["bias_begin"] = _ints(begin)
    h["begin"] = begin
    status = torch.zeros(B, dtype=torch.int32, device=DEV)
    out = torch.full_like(x, 3.0)
    lib.bs_logits_adjust(x, out, _ints(g), 1, status=status, **a)
    s = status.tolist()
    assert s[0] & lib.BS_DEV_BAD_GAMMA and s[1] & lib.BS_DEV_BAD_TOKEN and s[2] & lib.BS_DEV_BAD_TREE
    assert s[3] & lib.BS_DEV_BAD_MASK and s[4] & lib.BS_DEV_BAD_LENGTH and s[5] & lib.BS_DEV_BAD_TOKEN
    g[0] = 0
    keep = [0, 1, 2, 3, 5]
    got, x0 = out.double().cpu().numpy(), x.double().cpu().numpy()
    for b in keep:
        for r in range(R):
            if r > g[b]:
                assert (got[b, r] == 3.0).all()
                continue
            hb = dict(h, bt=np.where((h["bt"] < 0) | (h["bt"] >= V), 0, h["bt"]), bv=np.where((h["bt"] < 0) | (h["bt"] >= V), 0.0, h["bv"]))
            want, tol = _want(x0[b, r], hb, b, r, a)
            inf = np.isinf(want)
            assert (got[b, r][inf] == -np.inf).all() and (np.abs(got[b, r][~inf] - want[~inf]) <= 1.01 * tol[~inf]).all(), (b, r)


# ---- history --------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("V", [1, 31, 8191, 8192, 8193, 20001, 128256])
@pytest.mark.parametrize("B", [1, 3])
def test_history(lib, B, V):
    rng = np.random.default_rng(V)
    hist = lib.new_history(B, V)
    hist += 7                                                 # left over
    lens = rng.integers(0, 3000, B)
    prompts = [rng.integers(0, V, n).tolist() for n in lens]
    W = 9
    emitted = rng.integers(0, min(V, 5), (B, W))
    m = rng.integers(0, W + 1, B)
    fresh = np.ones(B, int)
    if B > 1:
        fresh[1] = 0                                          # goes on
    want = ol.enter(np.full((B, V), 7), fresh, prompts, [emitted[b, :m[b]] for b in range(B)])
    cu = np.concatenate([[0], np.cumsum(lens)])
    flat = _ints(sum(prompts, []) + [0])
    status = torch.zeros(B, dtype=torch.int32, device=DEV)
    lib.bs_history_update(hist, torch.tensor(fresh.tolist(), dtype=torch.uint8, device=DEV), _ints(cu), flat, _ints(emitted), _ints(m), status)
    assert np.array_equal(hist.cpu().numpy(), want) and not status.any()
    for _ in range(3):                                        # rounds
        lib.bs_history_update(hist, out_tokens=_ints(emitted), out_len=_ints(m))
        want = ol.enter(want, emitted=[emitted[b, :m[b]] for b in range(B)])
    assert np.array_equal(hist.cpu().numpy(), want)
    lib.bs_history_update(hist, cu_prompt=_ints(cu), prompt_tokens=flat)     # pieces of prompts, nothing fresh
    want = ol.enter(want, prompts=prompts)
    assert np.array_equal(hist.cpu().numpy(), want)


def test_history_counts_stop_at_the_largest(lib):
    hist = lib.new_history(2, 10)
    hist[0, 3], hist[0, 4], hist[1, 3] = 2 * ol.MOST - 2 + 1, 2 * ol.MOST, 1
    tokens = _ints([[3, 3, 3, 4], [3, 3, 3, 3]])
    lib.bs_history_update(hist, out_tokens=tokens, out_len=_ints([4, 4]))
    assert hist[0, 3] == 2 * ol.MOST + 1 and hist[0, 4] == 2 * ol.MOST and hist[1, 3] == 9


def test_history_bad_data(lib):
    B, V, W = 5, 100, 4
    hist = lib.new_history(B, V)
    status = torch.zeros(B, dtype=torch.int32, device=DEV)
    tokens = _ints([[1, -1, 2, 3], [4, 5, 100, 6], [7, 7, 7, 7], [8, 8, 8, 8], [9, 9, 9, 9]])
    lib.bs_history_update(hist, out_tokens=tokens, out_len=_ints([4, 4, 5, -1, 2]), status=status)
    want = ol.enter(np.zeros((B, V)), emitted=[[1, 2, 3], [4, 5, 6], [], [], [9, 9]])
    assert np.array_equal(hist.cpu().numpy(), want)
    bad = lib.BS_DEV_BAD_TOKEN, lib.BS_DEV_BAD_LENGTH
    assert status.tolist() == [bad[0], bad[0], bad[1], bad[1], 0]
    status.zero_()
    lib.bs_history_update(hist, torch.ones(B, dtype=torch.uint8, device=DEV), _ints([0, 2, 1, 3, 9, 3]), _ints([1, 200, 3, 4]), status=status)
    want = ol.enter(np.zeros((B, V)), prompts=[[1, 200], [], [200, 3], [], []])
    assert np.array_equal(hist.cpu().numpy(), want)
    assert status.tolist() == [bad[0], bad[1], bad[0], bad[1], bad[1]]


def test_adjust_reads_what_rounds_entered(lib):
    """A prompt, a round's tokens and the next round's rows, captured and replayed."""
    B, R, V = 2, 4, 1000
    x = torch.randn(B, R, V, device=DEV)
    hist = lib.new_history(B, V)
    gamma, drafted = _ints([3, 1]), _ints([[5, 6, 5], [900, 1, 1]])
    one = torch.ones(B, device=DEV)
    prompt, cu, emitted, m = _ints([5, 7, 7, 900]), _ints([0, 3, 4]), _ints([[5, 8, 8, 0], [1, 1, 1, 1]]), _ints([3, 4])
    fresh = torch.ones(B, dtype=torch.uint8, device=DEV)
    out = torch.zeros_like(x)

    def step():
        lib.bs_history_update(hist, fresh, cu, prompt)
        lib.bs_history_update(hist, out_tokens=emitted, out_len=m)
        lib.bs_logits_adjust(x, out, gamma, 1, draft_tokens=drafted, history=hist, repetition=1.5 * one, presence=one, frequency=0.25 * one)

    step()
    first = out.clone()
    want = ol.enter(np.zeros((B, V)), prompts=[[5, 7, 7], [900]], emitted=[[5, 8, 8], [1, 1, 1, 1]])
    assert np.array_equal(hist.cpu().numpy(), want)
    for b in range(B):
        for r in range(int(gamma[b]) + 1):
            w = ol.adjust_row(x[b, r].cpu().numpy(), want[b], drafted[b, :r].tolist(), 1.5, 1.0, 0.25)
            assert np.abs(out[b, r].cpu().numpy() - w).max() < 1e-5
    params = [1.5 * one, one, 0.25 * one]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lib.bs_history_update(hist, fresh, cu, prompt)
        lib.bs_history_update(hist, out_tokens=emitted, out_len=m)
        lib.bs_logits_adjust(x, out, gamma, 1, draft_tokens=drafted, history=hist, repetition=params[0], presence=params[1], frequency=params[2])
    out.zero_()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, first) and np.array_equal(hist.cpu().numpy(), want)


@pytest.mark.parametrize("extra", [0, 1])
@pytest.mark.parametrize("begin", [0, 1])
@pytest.mark.parametrize("changed", [1, 200])
def test_any_gamma_outside_the_range_is_zero(lib, changed, begin, extra):
    """Up to the ends of int32, where a sum with `extra` would wrap; one changed element in a block of the vocabulary, and many."""
    R, V, far = 4, 256, 2 ** 31
    gammas = [far - 1, far - 2, -far, -1, R - extra + 1, R - extra, 0]
    B = len(gammas)
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn(B + 2, R, V, generator=g, device=DEV)    # rows in front and behind: nothing is written there
    out = torch.full_like(x, 3.0)
    hist = torch.zeros(B, V, dtype=torch.int16, device=DEV)
    hist[:, :changed] = 5
    half = torch.full((B,), 0.5, device=DEV)
    status = torch.zeros(B, dtype=torch.int32, device=DEV)
    lib.bs_logits_adjust(x[1:-1], out[1:-1], _ints(gammas), extra, rows=(begin, R), history=hist, presence=half, status=status)
    bad = [not 0 <= v <= R - extra for v in gammas]
    assert status.tolist() == [lib.BS_DEV_BAD_GAMMA if v else 0 for v in bad]
    want = torch.full_like(x, 3.0)
    for b, v in enumerate(gammas):
        end = (0 if bad[b] else v) + extra
        want[b + 1, begin:end] = x[b + 1, begin:end] - 0.5 * (hist[b] > 0)
    assert torch.equal(out, want)


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [512, 515])
def test_a_row_has_its_bits_whatever_else_is_drafted(lib, V, dtype, tree):
    """How many elements of a block of the vocabulary change, on all rows together, decides how they are worked on; a row's result
    must not show it: tokens of other branches and behind the row, left over beyond gamma, in a call of its own or of all rows."""
    rng = np.random.default_rng(V + tree)
    R, N, fills = 8, 7, list(range(20, 44))                   # 32 is where the work changes
    B = len(fills)
    hist = np.zeros((B, V), np.int16)
    for b, n in enumerate(fills):
        hist[b, rng.permutation(250)[:n]] = rng.integers(1, 12, n)
    x = rng.normal(size=(B, R, V)) * 4
    x[:, :, 7] = -0.0
    x[:, :, rng.permutation(V)[:20]] = -0.0
    x = torch.tensor(x, device=DEV).to(dtype)
    parent = np.array([[rng.integers(0, j + 1) for j in range(N)] for _ in range(B)]) if tree else None
    drafted = rng.integers(0, 250, (B, N))
    drafted[:, 1], drafted[:, 4] = drafted[:, 0], drafted[:, 0]    # the same one more than once
    fl = lambda lo, hi: torch.tensor(rng.uniform(lo, hi, B), dtype=torch.float32, device=DEV)  # noqa: E731
    rules = dict(history=torch.tensor(hist, device=DEV), repetition=fl(1.1, 1.7), presence=fl(-0.5, 1.0), frequency=fl(-0.3, 0.9),
                 bias_begin=_ints(np.arange(B + 1) * 3), bias_tokens=_ints(rng.integers(0, 250, 3 * B)),
                 bias_values=torch.tensor(rng.normal(size=3 * B), dtype=torch.float32, device=DEV),
                 node_parent=None if parent is None else _ints(parent))
    bits = torch.int16 if dtype is torch.bfloat16 else torch.int32
    base = torch.zeros_like(x)
    lib.bs_logits_adjust(x, base, _ints([R - 1] * B), 1, draft_tokens=_ints(drafted), **rules)
    for row in range(R):
        other = rng.integers(0, 250, (B, N))
        for b in range(B):
            for n in ol.path(None if parent is None else parent[b], row):
                other[b, n - 1] = drafted[b, n - 1]
        for in_place in (False, True):
            for only in (False, True):
                out = x.clone() if in_place else torch.zeros_like(x)
                lib.bs_logits_adjust(out if in_place else x, out, _ints([row] * B), 1, rows=(row if only else 0, R), draft_tokens=_ints(other), **rules)
                differ = out[:, row].view(bits) != base[:, row].view(bits)
                assert not differ.any(), (row, in_place, only, int(differ.sum()))


def test_lists_at_the_far_end_of_their_arrays(lib):
    """Entries 2^31 - 12 to 2^31 - 2 of the biases, the last that 32 bits can number; the tokens of a prompt there."""
    n, far, V = 2 ** 31 - 1, 10, 300
    whole = torch.empty(n + 64, dtype=torch.int32, device=DEV)    # both arrays in one: their last entries lie apart
    tokens, values = whole[:n], whole[64:].view(torch.float32)
    at = [3, 299, 7, 3, 0, 255, 256, 3, 11, 12]
    tokens[-far:] = _ints(at)
    values[-far:] = torch.arange(1, far + 1, device=DEV)
    x = torch.zeros(2, 2, V, device=DEV)
    out = torch.full_like(x, 9.0)
    status = torch.zeros(2, dtype=torch.int32, device=DEV)
    lib.bs_logits_adjust(x, out, None, 0, bias_begin=_ints([n - far, n - 4, n]), bias_tokens=tokens, bias_values=values, status=status)
    want = torch.zeros(2, 2, V)
    for i, t in enumerate(at):
        want[0 if i < far - 4 else 1, :, t] += i + 1.0
    assert torch.equal(out.cpu(), want) and not status.any()
    hist = lib.new_history(2, V)
    lib.bs_history_update(hist, cu_prompt=_ints([n - far, n - 4, n]), prompt_tokens=tokens, status=status)
    assert np.array_equal(hist.cpu().numpy(), ol.enter(np.zeros((2, V)), prompts=[at[:-4], at[-4:]])) and not status.any()


def test_a_prompt_as_long_as_its_array_can_be(lib):
    """2^31 - 1 tokens of one sequence, all entered, the last ones among them; in a history that begins anew."""
    n, V = 2 ** 31 - 1, 64
    tokens = torch.zeros(n, dtype=torch.int32, device=DEV)
    tokens[-3:] = _ints([5, 63, 64])
    hist, status = lib.new_history(1, V), torch.zeros(1, dtype=torch.int32, device=DEV)
    lib.bs_history_update(hist, torch.ones(1, dtype=torch.uint8, device=DEV), _ints([0, n]), tokens, status=status)
    want = np.zeros((1, V))
    want[0, [0, 5, 63]] = 1
    assert np.array_equal(hist.cpu().numpy(), want) and status.tolist() == [lib.BS_DEV_BAD_TOKEN]
