"""bs_rotary on the GPU against the fp64 oracle: layouts, parts of the head, strides, scalings, far positions, trees."""
import numpy as np
import pytest
import torch

from oracle import prompt as op

pytestmark = pytest.mark.gpu
DEV = "cuda"
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _check(got, x, positions, f, amplitude, interleaved, dtype):
    """A result is rounded once (half a step); before that: the sine and cosine are off by at most 5 half steps of fp32 (angle, two
    units of the function, amplitude) and products and sum by 3, each of at most |a| + |b| times the amplitude."""
    x = x.double().cpu().numpy()
    want = op.rotate(x, positions, f, amplitude, interleaved)
    half = len(f)
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    size = np.abs(x)
    size[..., a], size[..., b] = (np.abs(x[..., a]) + np.abs(x[..., b]),) * 2
    tol = (1.01 * HALF[dtype] if dtype is torch.bfloat16 else 0.0) * np.abs(want) + 8 * 2.0 ** -24 * amplitude * size + 1e-38
    err = np.abs(got.double().cpu().numpy() - want)
    assert (err <= tol).all(), (err / tol).max()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,Hq,Hkv,d,rot", [(1, 1, 1, 64, 64), (5, 32, 8, 128, 128), (37, 7, 1, 128, 32), (9, 4, 2, 64, 24), (3, 3, 0, 64, 2),
                                            (2500, 4, 1, 64, 64), (11, 2, 2, 80, 20), (6, 1, 1, 34, 6), (4, 2, 1, 256, 256)])
def test_rotation(lib, T, Hq, Hkv, d, rot, dtype, interleaved):
    g = torch.Generator(device=DEV).manual_seed(T + rot)
    q = torch.randn(T, Hq, d, generator=g, device=DEV).to(dtype)
    k = torch.randn(T, Hkv, d, generator=g, device=DEV).to(dtype) if Hkv else None
    pos = torch.randint(0, 200000, (T,), generator=g, device=DEV, dtype=torch.int32)
    table = lib.new_rotary_table(rot, 500000.0)
    qo, ko = torch.zeros_like(q), None if k is None else torch.zeros_like(k)
    lib.bs_rotary(q, k, pos, table, interleaved, qo, ko)
    f, amplitude = op.frequencies(rot, 500000.0)
    _check(qo, q, pos.tolist(), f, amplitude, interleaved, dtype)
    if k is not None:
        _check(ko, k, pos.tolist(), f, amplitude, interleaved, dtype)
    lib.bs_rotary(q, k, pos, table, interleaved, q, k)        # in place: the same bits
    assert torch.equal(q, qo) and (k is None or torch.equal(k, ko))


@pytest.mark.parametrize("scaling,kw", [("linear", {"factor": 4.0}), ("bands", {"factor": 8.0, "low": 1.0, "high": 4.0, "original": 8192}),
                                        ("yarn", {"factor": 32.0, "low": 1.0, "high": 32.0, "original": 4096})])
def test_scalings_at_far_positions(lib, scaling, kw):
    pos = [0, 1, 131071, 1000003, 2 ** 31 - 1]
    q = torch.randn(len(pos), 2, 64, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV)
    out = torch.empty_like(q)
    lib.bs_rotary(q, None, _ints(pos), lib.new_rotary_table(64, 10000.0, scaling, **kw), False, out, None)
    f, amplitude = op.frequencies(64, 10000.0, scaling, **kw)
    assert (amplitude != 1.0) == (scaling == "yarn")
    # the oracle's own angle: a frequency and the product are off by half a step of fp64 each, 2^31 radians x 2^-52
    x = q.double().cpu().numpy()
    want = op.rotate(x, pos, f, amplitude, False)
    size = np.abs(x[..., :32]) + np.abs(x[..., 32:])
    tol = (8 * 2.0 ** -24 + 2.0 ** -20 * (np.array(pos) > 2 ** 30)[:, None, None]) * amplitude * np.concatenate([size, size], 2)
    assert (np.abs(out.double().cpu().numpy() - want) <= tol).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pad", [8, 4, 2, 1])
def test_views_and_untouched_rows(lib, dtype, pad):
    """Views of a fused projection whose rows start on every alignment; rows without a position stay as they are."""
    T, H, d, rot = 13, 3, 64, 32
    g = torch.Generator(device=DEV).manual_seed(pad)
    fused = torch.randn(T, H * d * 3 + pad, generator=g, device=DEV).to(dtype)
    q = fused[:, pad:pad + 2 * H * d].view(T, 2 * H, d) if pad % 2 == 0 else torch.as_strided(fused, (T, 2 * H, d), (fused.stride(0), d, 1), pad)
    k = torch.as_strided(fused, (T, H, d), (fused.stride(0), d, 1), pad + 2 * H * d)
    pos = torch.arange(T, device=DEV, dtype=torch.int32) * 7
    pos[4] = pos[12] = -1
    qo, ko = torch.full((T, 2 * H, d), 5.0, device=DEV, dtype=dtype), torch.full((H, T, d), 5.0, device=DEV, dtype=dtype).transpose(0, 1)
    lib.bs_rotary(q, k, pos, lib.new_rotary_table(rot), True, qo, ko)
    f, amplitude = op.frequencies(rot, 10000.0)
    live = [t for t in range(T) if pos[t] >= 0]
    for x, y in ((q, qo), (k, ko)):
        _check(y[live], x[live], pos[live].tolist(), f, amplitude, True, dtype)
        assert (y[[4, 12]] == 5.0).all()
    before = fused.clone()
    lib.bs_rotary(q, k, pos, lib.new_rotary_table(rot), True, q, k)
    assert torch.equal(q[live], qo[live]) and torch.equal(k[live], ko[live])
    assert torch.equal(fused[[4, 12]], before[[4, 12]]) and torch.equal(fused[:, :pad], before[:, :pad])
    if 3 * H * d + pad > pad + 3 * H * d:
        assert torch.equal(fused[:, pad + 3 * H * d:], before[:, pad + 3 * H * d:])


@pytest.mark.parametrize("B", [1, 33, 70, 1100])
def test_trees(lib, B):
    """A node is rotated to its depth; rows behind the tree's table, or behind the last sequence, stay."""
    rng = np.random.default_rng(B)
    N = 31 if B < 1000 else 3
    n = rng.integers(0, N + 2, B)
    if B > 2:
        n[1] = 0
        n[2] = N + 3                                          # more rows than nodes
    parent = np.array([[rng.integers(0, j + 1) for j in range(N)] for _ in range(B)])
    parent[0, 0] = -4                                         # nonsense counts as the root
    if N > 4:
        parent[0, 4] = 9
    cu = np.concatenate([[0], np.cumsum(n)])
    T = int(cu[-1]) + 2
    ctx = rng.integers(0, 5000, B)
    pos = np.full(T, 77)
    for b in range(B):
        pos[cu[b]:cu[b + 1]] = ctx[b] + np.arange(n[b])
    q = torch.randn(T, 2, 64, generator=torch.Generator(device=DEV).manual_seed(2), device=DEV)
    out = torch.full_like(q, 9.0)
    lib.bs_rotary(q, None, _ints(pos.tolist()), lib.new_rotary_table(64), False, out, None, cu_new=_ints(cu.tolist()), node_parent=_ints(parent.tolist()))
    f, amplitude = op.frequencies(64, 10000.0)
    want = [int(ctx[b]) + op.depth(parent[b], r) if r <= N else -1 for b in range(B) for r in range(n[b])] + [-1, -1]
    live = [t for t, w in enumerate(want) if w >= 0]
    _check(out[live], q[live], [want[t] for t in live], f, amplitude, False, torch.float32)
    gone = [t for t, w in enumerate(want) if w < 0]
    assert (out[gone] == 9.0).all()
    # trees of a root alone
    lib.bs_rotary(q, None, _ints(pos.tolist()), lib.new_rotary_table(64), False, out, None, cu_new=_ints(cu.tolist()),
                  node_parent=torch.zeros(B, 0, dtype=torch.int32, device=DEV))
    roots = [int(cu[b]) for b in range(B) if n[b]]
    _check(out[roots], q[roots], pos[roots].tolist(), f, amplitude, False, torch.float32)


def test_special_values_and_streams(lib):
    q = torch.randn(4, 1, 64, device=DEV, dtype=torch.bfloat16)
    q[1, 0, 3], q[2, 0, 5] = float("nan"), float("inf")
    pos, table = _ints([3, 4, 5, 6]), lib.new_rotary_table(64)
    out = torch.zeros_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    lib.bs_rotary(q, None, pos, table, False, out, None, stream=side)
    side.synchronize()
    bad = ~torch.isfinite(out)
    assert bad.sum() == 4 and bad[1, 0, [3, 35]].all() and bad[2, 0, [5, 37]].all()
    graph = torch.cuda.CUDAGraph()
    other = torch.zeros_like(out)
    with torch.cuda.graph(graph):
        lib.bs_rotary(q, None, pos, table, False, other, None)
    pos += 1
    graph.replay()
    torch.cuda.synchronize()
    lib.bs_rotary(q, None, pos, table, False, out, None)
    torch.cuda.synchronize()
    assert torch.equal(out.view(torch.int16), other.view(torch.int16))


@pytest.mark.parametrize("scaling,kw", [("none", {}), ("linear", {"factor": 3.0}), ("bands", {"factor": 8.0, "low": 1.0, "high": 4.0, "original": 8192})])
def test_angles_at_the_farthest_positions(lib, scaling, kw):
    """Pairs (1, 0) become cosine and sine.  The angle is off by 2^-31 turns and rounded by 2^-26: 1.62 x 2^-24 radians; the functions are
    off by two units of 2^-24 at most, the result by half of one."""
    from test_rotary_frequencies import exact_turns
    from decimal import Decimal
    pos = [2 ** 24 + 1, 2 ** 27 - 3, 2 ** 30 + 7, 2 ** 31 - 2, 2 ** 31 - 1]
    q = torch.zeros(len(pos), 1, 128, device=DEV)
    q[..., :64] = 1.0
    out = torch.empty_like(q)
    lib.bs_rotary(q, None, _ints(pos), lib.new_rotary_table(128, 10000.0, scaling, **kw), False, out, None)
    turns = np.array([[float((f * p) % Decimal(1)) for f in exact_turns(128, 10000.0, scaling, **kw)] for p in pos])
    want = np.concatenate([np.cos(2 * np.pi * turns), np.sin(2 * np.pi * turns)], 1)
    err = np.abs(out[:, 0].double().cpu().numpy() - want)
    assert err.max() <= 4.2 * 2.0 ** -24, err.max() * 2 ** 24
