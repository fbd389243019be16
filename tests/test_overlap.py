"""Outputs that overlap inputs are refused before anything is launched; views of one buffer that only lie between one another are not
(no GPU needed)."""
import os
import subprocess

import numpy as np
import pytest

from conftest import ROOT


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("overlap") / "overlap")
    subprocess.run(["g++", "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2505_15141_b200", "csrc"), "-o", out,
                    os.path.join(ROOT, "tests", "overlap_host.cpp")], check=True)
    return out


def _bytes(at, st, sh, T, H, d, e):
    return {at + t * st * e + h * sh * e + k for t in range(T) for h in range(H) for k in range(d * e)}


def _ask(program, cases):
    out = subprocess.run([program], input="\n".join(" ".join(map(str, a + b)) for a, b in cases), capture_output=True, text=True, check=True)
    return [int(x) for x in out.stdout.split()]


def test_against_every_byte(program):
    """Small arrays of any layout with one token stride; with strides that differ nothing apart is taken for overlapping."""
    rng = np.random.default_rng(0)
    cases = []
    for _ in range(6000):
        T, d, e = int(rng.integers(1, 6)), int(rng.integers(1, 5)), int(rng.choice([1, 2, 4]))
        Ha, Hb = (int(rng.integers(0, 5)) for _ in range(2))
        kind = rng.integers(0, 5)
        sh = d * int(rng.integers(1, 4))
        st = int(rng.integers(1, 60)) if kind == 0 else sh * 5 + int(rng.integers(0, 8)) if kind < 3 else d
        shb = sh if kind else int(rng.integers(0, 30))
        if kind == 3:                                         # heads first
            sh = shb = d * T + int(rng.integers(0, 4))
        if kind == 4:                                         # without gaps
            sh = shb = d
            st, stb = d * Ha, d * Hb
        if rng.random() < 0.1 and kind != 4:
            st = -st
        if rng.random() < 0.1:
            sh, shb = -sh, -shb
        if kind != 4:
            stb = st if rng.random() < 0.85 else int(rng.integers(0, 60))
        elif rng.random() < 0.5:
            stb, shb = int(rng.integers(0, 60)), int(rng.integers(0, 20))
        cases.append(((1000, st, sh, T, Ha, d, e), (1000 + int(rng.integers(-150, 150)) * (e if rng.random() < 0.9 else 1), stb, shb, T, Hb, d, e)))
    got = _ask(program, cases)
    assert len(got) == len(cases) and 500 < sum(got) < 5500
    for (a, b), g in zip(cases, got):
        want = bool(_bytes(*a) & _bytes(*b))
        dense = lambda x: len(_bytes(*x)) == max(_bytes(*x), default=0) - min(_bytes(*x), default=0) + 1 and x[1] >= 0 and x[2] >= x[5]  # noqa: E731
        if a[1] == b[1] or a[3] == 1 or (dense(a) and a[1] in (a[5], a[4] * a[5])) or (dense(b) and b[1] in (b[5], b[4] * b[5])):
            assert g == want, (a, b)
        else:
            assert not g or want, (a, b)


def test_views_of_a_fused_projection(program):
    """Large ones: 2^20 tokens of 32 + 8 + 8 heads of 128, and results in the same buffer."""
    at, T, st = 1 << 40, 1 << 20, (32 + 8 + 8 + 32) * 128
    part = lambda first, heads: (at + first * 256, st, 128, T, heads, 128, 2)  # noqa: E731
    q, k, v, out = part(0, 32), part(32, 8), part(40, 8), part(48, 32)
    inner = lambda i: (at + i * 256, st, 4 * 128, T, 8, 128, 2)  # noqa: E731  -- head by head
    far = (at + (1 << 62), st, 128, T, 32, 128, 2)
    got = _ask(program, [(q, k), (k, v), (v, out), (out, q), (q, q), (q, part(31, 8)), (part(79, 8), q), (inner(0), inner(3)), (inner(1), inner(1)), (q, far)])
    assert got == [0, 0, 0, 0, 1, 1, 1, 0, 1, 0]


# ---- the library refuses them: sizes and pointers as a call would bring them, none of which is read ------------------------------

AT = 1 << 30


def _attention(lib, **kw):
    a = dict(q=AT, q_t=256, q_h=64, k=2 * AT, k_t=128, k_h=64, v=3 * AT, v_t=128, v_h=64, cu=AT, B=2, T=100, Hq=4, Hkv=2, d=64, scale=0.1, out=4 * AT, o_t=256,
             o_h=64, status=None, stream=None)
    a.update(kw)
    return lib._lib.bs_prompt_attention(*a.values())


@pytest.mark.parametrize("kw", [{"out": AT}, {"out": AT + 99 * 512}, {"out": AT - 99 * 512}, {"out": 2 * AT}, {"out": 3 * AT + 16}, {"out": 3 * AT - 99 * 512 - 400},
                                {"q_t": 768, "q": AT, "o_t": 768, "out": AT + 256}, {"out": AT, "o_t": 512}, {"T": 1, "out": AT + 128, "o_t": 8}])
def test_attention_into_its_inputs(lib, kw):
    assert _attention(lib, **kw) == lib.BS_ERR_INVALID_ARG


def _rotary(lib, **kw):
    a = dict(q=AT, q_t=256, q_h=64, k=2 * AT, k_t=128, k_h=64, dtype=1, pos=AT, freq=AT, amplitude=1.0, rot=64, inter=0, cu=None, parent=None, B=0, N=0,
             T=100, Hq=4, Hkv=2, d=64, qo=3 * AT, qo_t=256, qo_h=64, ko=4 * AT, ko_t=128, ko_h=64, stream=None)
    a.update(kw)
    return lib._lib.bs_rotary(*a.values())


@pytest.mark.parametrize("kw", [{"qo": AT + 2}, {"qo": AT, "qo_t": 264}, {"qo": AT, "qo_h": 72}, {"qo": 2 * AT}, {"ko": AT + 512 * 50}, {"ko": 2 * AT + 128},
                                {"qo": 4 * AT}, {"ko": 3 * AT + 512 * 99}, {"qo": AT, "Hkv": 0, "k": None, "ko": None, "qo_t": 512}])
def test_rotation_into_other_inputs(lib, kw):
    assert _rotary(lib, **kw) == lib.BS_ERR_INVALID_ARG


@pytest.mark.parametrize("out", [AT + 4, AT + 4 * (2 * 5 * 100 - 1), AT - 4, AT - 4 * (2 * 5 * 100 - 1)])
def test_adjusted_logits_that_overlap_the_others(lib, out):
    assert lib._lib.bs_logits_adjust(AT, out, 0, None, 1, 0, 5, None, None, 0, None, None, None, None, None, None, None, 0, None, 0, None, 2, 5, 100,
                                     None, None) == lib.BS_ERR_INVALID_ARG
