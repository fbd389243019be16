"""What the calls around the cache refuse before anything is launched: in the library, by sizes and pointers, and in the Python
binding, by types and places (no GPU needed); the frequencies of the rotation, which are computed on the host."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import logits as ol
from oracle import prompt as op
from test_cache_binding import Placed

AT = 1 << 20                                                  # an address that nothing reads: every call below is refused


def _attention(lib, **kw):
    a = dict(q=AT, q_t=256, q_h=64, k=AT, k_t=256, k_h=64, v=AT, v_t=256, v_h=64, cu=AT, B=2, T=0, Hq=4, Hkv=2, d=64, scale=0.1, out=AT, o_t=256,
             o_h=64, status=None, stream=None)
    assert set(kw) <= set(a)
    a.update(kw)
    return lib._lib.bs_prompt_attention(*a.values())


@pytest.mark.parametrize("code,kw", [
    (0, {}), (0, {"q": None, "k": None, "v": None, "out": None}),                       # no tokens: nothing to do
    (1, {"B": 0}), (1, {"T": -1}), (1, {"cu": None}), (1, {"Hq": 0}), (1, {"Hkv": 0}), (1, {"Hq": 5}), (1, {"d": 0}), (1, {"T": 3, "q": None}),
    (1, {"T": 3, "out": None}), (1, {"scale": 0.0}), (1, {"scale": -1.0}), (1, {"scale": float("nan")}), (1, {"scale": float("inf")}),
    (1, {"q": AT + 8}), (1, {"k": AT + 2}), (1, {"v": AT + 4}), (1, {"out": AT + 8}), (3, {"d": 96}), (3, {"d": 256}), (3, {"Hq": 130}),
    (3, {"B": 4097}), (3, {"q_t": 260}), (3, {"k_h": 4}), (3, {"v_t": 1}), (3, {"o_h": 12}), (3, {"k_t": -256}), (3, {"T": 2 ** 31 - 1, "Hq": 128, "Hkv": 128, "B": 4096})])
def test_attention_refusals(lib, code, kw):
    assert _attention(lib, **kw) == code


def _rotary(lib, **kw):
    a = dict(q=AT, q_t=256, q_h=64, k=AT, k_t=128, k_h=64, dtype=1, pos=AT, freq=AT, amplitude=1.0, rot=64, inter=0, cu=None, parent=None, B=0, N=0,
             T=0, Hq=4, Hkv=2, d=64, qo=AT, qo_t=256, qo_h=64, ko=AT, ko_t=128, ko_h=64, stream=None)
    assert set(kw) <= set(a)
    a.update(kw)
    return lib._lib.bs_rotary(*a.values())


@pytest.mark.parametrize("code,kw", [
    (0, {}), (0, {"Hq": 0, "q": None, "qo": None}), (1, {"T": -1}), (1, {"Hq": -1}), (1, {"Hq": 0, "Hkv": 0}), (1, {"freq": None}), (1, {"T": 1, "pos": None}),
    (1, {"dtype": 2}), (1, {"T": 1, "q": None}), (1, {"T": 1, "qo": None}), (1, {"T": 1, "k": None}), (1, {"T": 1, "ko": None}), (1, {"amplitude": float("nan")}),
    (1, {"parent": AT}), (1, {"parent": AT, "cu": AT}), (1, {"parent": AT, "cu": AT, "B": 1, "N": -1}), (3, {"parent": AT, "cu": AT, "B": 1, "N": 32}),
    (3, {"parent": AT, "cu": AT, "B": 4097, "N": 3}), (3, {"rot": 0}), (3, {"rot": 66}), (3, {"rot": 7}), (3, {"rot": 258, "d": 512}), (3, {"d": 65}), (3, {"Hq": 5000})])
def test_rotary_refusals(lib, code, kw):
    assert _rotary(lib, **kw) == code


def _adjust(lib, **kw):
    a = dict(x=AT, y=AT, dtype=0, gamma=AT, extra=1, r0=0, r1=5, tok=None, parent=None, N=0, hist=None, rep=None, pres=None, freq=None, bb=None, bt=None,
             bv=None, n_bias=0, masks=None, n_masks=0, row=None, B=2, R=5, V=100, status=None, stream=None)
    assert set(kw) <= set(a)
    a.update(kw)
    return lib._lib.bs_logits_adjust(*a.values())


@pytest.mark.parametrize("code,kw", [
    (1, {"x": None}), (1, {"y": None}), (1, {"B": 0}), (1, {"R": 0}), (1, {"V": 0}), (1, {"N": -1}), (1, {"n_bias": -1}), (1, {"n_masks": -1}), (1, {"dtype": 5}),
    (1, {"extra": 2}), (1, {"extra": -1}), (1, {"r0": -1}), (1, {"r0": 4, "r1": 3}), (1, {"r1": 6}), (3, {"B": 4097}), (3, {"R": 33, "r1": 33}), (3, {"V": (1 << 20) + 1}),
    (3, {"N": 32}), (1, {"tok": AT, "N": 3}), (1, {"parent": AT, "N": 4}), (1, {"rep": AT}), (1, {"freq": AT}), (1, {"pres": AT}), (1, {"bb": AT, "n_bias": 1}),
    (1, {"bb": AT, "bt": AT, "n_bias": 1}), (1, {"row": AT, "n_masks": 1})])
def test_adjust_refusals(lib, code, kw):
    assert _adjust(lib, **kw) == code


@pytest.mark.parametrize("code,kw", [
    (0, {}), (1, {"hist": None}), (1, {"hist": AT + 1}), (1, {"B": 0}), (1, {"V": 0}), (1, {"Tp": -1}), (1, {"W": -1}), (1, {"cu": AT, "Tp": 1}), (1, {"len": AT, "W": 1}),
    (3, {"B": 4097}), (3, {"V": (1 << 20) + 1}), (3, {"W": 33})])
def test_history_refusals(lib, code, kw):
    a = dict(hist=AT, B=2, V=10, fresh=None, cu=None, prompt=None, Tp=0, tok=None, len=None, W=0, status=None, stream=None)
    a.update(kw)
    assert lib._lib.bs_history_update(*a.values()) == code


# ---- frequencies ----------------------------------------------------------------------------------------------

@pytest.mark.parametrize("rot", [2, 24, 64, 128, 256])
@pytest.mark.parametrize("scaling,kw", [("none", {}), ("linear", {"factor": 4.0}), ("bands", {"factor": 8.0, "low": 1.0, "high": 4.0, "original": 8192}),
                                        ("yarn", {"factor": 32.0, "low": 1.0, "high": 32.0, "original": 4096}), ("yarn", {"factor": 1.0, "low": 2.0, "high": 3.0, "original": 1})])
def test_frequencies(lib, rot, scaling, kw):
    """Held in whole multiples of 2^-64 turns: half a step, 2 pi 2^-65 radians, beside the few last bits of two fp64 computations."""
    table = lib.new_rotary_table(rot, 500000.0, scaling, **kw, device="cpu")
    f, amplitude = op.frequencies(rot, 500000.0, scaling, **kw)
    got = table.freq.numpy().view(np.uint64).astype(np.float64) * 2.0 ** -64 * 2 * np.pi
    assert table.rot == rot and (np.abs(got - f) <= 2.0 ** -48 * f + 2 * np.pi * 2.0 ** -65).all() and abs(table.amplitude - amplitude) <= 2.0 ** -24 * amplitude


@pytest.mark.parametrize("code,kw", [
    (1, {"base": 1.0}), (1, {"base": float("nan")}), (1, {"base": float("inf")}), (3, {"rot": 0}), (3, {"rot": 3}), (3, {"rot": 258}),
    (1, {"scaling": "linear", "factor": 0.5}), (1, {"scaling": "yarn", "factor": float("nan")}), (1, {"scaling": "bands", "low": 0.0}),
    (1, {"scaling": "bands", "low": 4.0, "high": 4.0}), (1, {"scaling": "yarn", "original": 0.0})])
def test_frequencies_refusals(lib, code, kw):
    with pytest.raises(lib.BanditSpecError) as e:
        lib.new_rotary_table(kw.pop("rot", 64), **kw, device="cpu")
    assert e.value.code == code


def test_frequencies_need_somewhere_to_go(lib):
    f = lib._lib.bs_rotary_frequencies
    one, amplitude = np.zeros(1, np.uint64), C.c_float()
    assert f(0, 2, 10.0, 1.0, 1.0, 2.0, 1.0, None, C.byref(amplitude)) == lib.BS_ERR_INVALID_ARG
    assert f(0, 2, 10.0, 1.0, 1.0, 2.0, 1.0, one.ctypes.data_as(C.c_void_p), None) == lib.BS_ERR_INVALID_ARG
    assert f(7, 2, 10.0, 1.0, 1.0, 2.0, 1.0, one.ctypes.data_as(C.c_void_p), C.byref(amplitude)) == lib.BS_ERR_INVALID_ARG


# ---- the binding's own checks ---------------------------------------------------------------------------------

def _calls(lib):
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    f = lambda *s: torch.zeros(*s)  # noqa: E731
    q, k = torch.zeros(6, 4, 64, dtype=torch.bfloat16), torch.zeros(6, 2, 64, dtype=torch.bfloat16)
    B, R, V, N = 3, 4, 40, 3
    table = lib.new_rotary_table(64, device="cpu")
    return {
        "bs_prompt_attention": ([q, k, k.clone(), i(B + 1), 0.1, q.clone(), i(B)], {}, 6),
        "bs_rotary": ([q, k, i(6), table, True, q.clone(), k.clone()], {"cu_new": i(B + 1), "node_parent": i(B, N)}, 7),
        "bs_history_update": ([torch.zeros(B, V, dtype=torch.int16)], {"fresh": torch.ones(B, dtype=torch.uint8), "cu_prompt": i(B + 1), "prompt_tokens": i(7),
                                                                     "out_tokens": i(B, R), "out_len": i(B), "status": i(B)}, 7),
        "bs_logits_adjust": ([f(B, R, V), f(B, R, V), i(B), 1], {"draft_tokens": i(B, N), "node_parent": i(B, N), "history": torch.zeros(B, V, dtype=torch.int16),
                                                               "repetition": f(B), "presence": f(B), "frequency": f(B), "bias_begin": i(B + 1), "bias_tokens": i(5),
                                                               "bias_values": f(5), "masks": i(2, 2), "mask_row": i(B, R), "status": i(B)}, 15),
    }


NAMES = ["bs_prompt_attention", "bs_rotary", "bs_history_update", "bs_logits_adjust"]


def _place(lib, x, index=0):
    if isinstance(x, torch.Tensor):
        return Placed(x, index)
    if isinstance(x, lib.RotaryTable):
        return lib.RotaryTable(Placed(x.freq, 0), x.amplitude, x.rot)
    return x


@pytest.mark.parametrize("name", NAMES)
def test_every_tensor_has_to_be_on_the_calls_gpu(lib, monkeypatch, name):
    made = []
    monkeypatch.setattr(lib, "_call", lambda fn, where, *a: made.append(where))
    args, kw, count = _calls(lib)[name]
    fn = getattr(lib, name)
    fn(*[_place(lib, x) for x in args], **{k: _place(lib, x) for k, x in kw.items()})
    assert made == [name]
    tensors = [n for n, x in enumerate(args) if isinstance(x, torch.Tensor)] + list(kw)
    assert len(tensors) == count
    for which in tensors:
        for index in (-1, 1):
            a, k = [_place(lib, x) for x in args], {n: _place(lib, x) for n, x in kw.items()}
            (k if isinstance(which, str) else a)[which].index = index
            with pytest.raises(AssertionError, match="GPU"):
                fn(*a, **k)
    if name == "bs_rotary":
        a, k = [_place(lib, x) for x in args], {n: _place(lib, x) for n, x in kw.items()}
        a[3].freq.index = 1
        with pytest.raises(AssertionError, match="GPU"):
            fn(*a, **k)
    assert len(made) == 1


@pytest.mark.parametrize("name", NAMES)
def test_types_and_sizes(lib, monkeypatch, name):
    """Each tensor in turn has another type, or one element too many."""
    monkeypatch.setattr(lib, "_call", lambda *a: None)
    args, kw, _ = _calls(lib)[name]
    for which in [n for n, x in enumerate(args) if isinstance(x, torch.Tensor)] + list(kw):
        for change in ("type", "size"):
            a, k = [_place(lib, x) for x in args], {n: _place(lib, x) for n, x in kw.items()}
            x = (k if isinstance(which, str) else a)[which]
            if change == "type":
                x.t = x.t.to(torch.float64 if x.t.is_floating_point() else torch.int64)
            elif which in ("prompt_tokens", "bias_tokens", "bias_values", "masks"):
                continue                                      # any number goes; pairs are looked at below
            else:
                x.t = torch.cat([x.t, x.t[:1]])
            if (name, which, change) in (("bs_history_update", 0, "size"), ("bs_prompt_attention", 3, "size")):
                with pytest.raises(AssertionError):           # the other tensors no longer fit it
                    getattr(lib, name)(*a, **k)
                continue
            with pytest.raises((AssertionError, TypeError)):
                getattr(lib, name)(*a, **k)
    if name == "bs_logits_adjust":
        k = {n: _place(lib, x) for n, x in kw.items()}
        k["bias_values"].t = torch.zeros(6)
        with pytest.raises(AssertionError):
            lib.bs_logits_adjust(*[_place(lib, x) for x in args], **k)
        for gone in ("bias_begin", "bias_tokens", "bias_values", "masks", "mask_row"):
            k = {n: _place(lib, x) for n, x in kw.items() if n != gone}
            with pytest.raises(AssertionError):
                lib.bs_logits_adjust(*[_place(lib, x) for x in args], **k)


def test_last_dimension_has_to_be_contiguous(lib, monkeypatch):
    monkeypatch.setattr(lib, "_call", lambda *a: None)
    args, _, _ = _calls(lib)["bs_prompt_attention"]
    for which in (0, 1, 2, 5):
        a = [_place(lib, x) for x in args]
        a[which].t = a[which].t.transpose(1, 2).contiguous().transpose(1, 2)
        with pytest.raises(AssertionError, match="last dimension"):
            lib.bs_prompt_attention(*a)
    args, kw, _ = _calls(lib)["bs_rotary"]
    for which in (0, 1, 5, 6):
        a = [_place(lib, x) for x in args]
        a[which].t = a[which].t.transpose(1, 2).contiguous().transpose(1, 2)
        with pytest.raises(AssertionError, match="last dimension"):
            lib.bs_rotary(*a)


def test_trees_without_drafts_are_not_chains(lib, monkeypatch):
    seen = []
    monkeypatch.setattr(lib, "_call", lambda fn, where, index, stream, *a: seen.append(a))
    args, kw, _ = _calls(lib)["bs_rotary"]
    lib.bs_rotary(*[_place(lib, x) for x in args], cu_new=Placed(kw["cu_new"]), node_parent=Placed(torch.zeros(3, 0, dtype=torch.int32)))
    lib.bs_rotary(*[_place(lib, x) for x in args])
    assert seen[0][13] and seen[0][14:16] == (3, 0) and seen[1][13] is None


# ---- the oracles themselves ----------------------------------------------------------------------------------

def test_oracle_of_the_rotation():
    """Scores of rotated queries and keys depend on the difference of the positions alone; lengths are kept."""
    rng = np.random.default_rng(0)
    f, _ = op.frequencies(16, 10000.0)
    x, y = rng.normal(size=(1, 1, 20)), rng.normal(size=(1, 1, 20))
    for inter in (False, True):
        s = [float((op.rotate(x, [a + 7], f, 1.0, inter) * op.rotate(y, [a], f, 1.0, inter)).sum()) for a in (0, 3, 1000)]
        assert np.ptp(s) < 1e-9
        assert np.isclose(np.linalg.norm(op.rotate(x, [5], f, 1.0, inter)), np.linalg.norm(x))
        assert np.array_equal(op.rotate(x, [-1], f, 1.0, inter), x)
    assert op.depth([0, 0, 1, 3, 9], 4) == 3 and op.depth([0, 0, 1, 3, 9], 5) == 1 and op.depth([-1], 1) == 1


def test_oracle_of_the_attention():
    rng = np.random.default_rng(1)
    q, k, v = rng.normal(size=(5, 4, 8)), rng.normal(size=(5, 2, 8)), rng.normal(size=(5, 2, 8))
    out, size = op.attention(q, k, v, [0, 2, 2, 5], 0.3)
    assert np.allclose(out[0], v[0].repeat(2, 0)) and np.allclose(out[2], v[2].repeat(2, 0))
    p = np.exp(0.3 * k[2:4, 1] @ q[3, 2])
    assert np.allclose(out[3, 2], (p / p.sum()) @ v[2:4, 1]) and (size >= np.abs(out) - 1e-12).all()


def test_oracle_of_the_logits():
    hist = ol.enter(np.zeros((1, 6)), prompts=[[1, 1, 2]], emitted=[[2, 3, 3]])
    assert hist.tolist() == [[0, 1, 3, 4, 0, 0]]
    x = ol.adjust_row([1.0, 1.0, -1.0, 2.0, 0.5, 0.0], hist[0], drafted=[4, 3], r=2.0, p=0.25, f=0.5, bias=[(0, 1.0), (0, 0.5)], allowed=[1, 1, 1, 1, 1, 0])
    assert x.tolist() == [2.5, 0.5, -2.75, -0.75, -0.5, -np.inf]
    assert ol.path(None, 3) == [3, 2, 1] and ol.path([0, 0, 1, 2], 4) == [4, 2] and ol.path([7], 1) == [1]
    assert ol.enter([[2 * ol.MOST + 1]], emitted=[[0]]).tolist() == [[2 * ol.MOST + 1]]


@pytest.mark.parametrize("scale,code", [(3.4e38, 1), (2.4e38, 1), (2.3e38, 0), (1e-45, 0)])
def test_attention_refuses_a_scale_that_is_infinite_in_base_two(lib, scale, code):
    """The kernel works with softmax_scale x log2(e), 1.4427 of it; the largest float is 3.4028e38."""
    assert _attention(lib, scale=scale) == code


@pytest.mark.parametrize("kw", [{"x": AT + 2, "y": AT + (1 << 24)}, {"y": AT + (1 << 24) + 1}, {"dtype": 1, "x": AT + 1, "y": AT + 1}, {"tok": AT, "N": 4, "hist": AT + 1, "rep": AT}])
def test_adjust_refuses_pointers_between_elements(lib, kw):
    assert _adjust(lib, **kw) == lib.BS_ERR_INVALID_ARG


@pytest.mark.parametrize("dtype,off", [(1, 1), (0, 1), (0, 2)])
@pytest.mark.parametrize("which", ["q", "qo", "k", "ko"])
def test_rotary_refuses_pointers_between_elements(lib, which, dtype, off):
    at = {"q": AT, "qo": 2 * AT, "k": 3 * AT, "ko": 4 * AT}
    assert _rotary(lib, dtype=dtype, T=5, **dict(at, **{which: at[which] + off})) == lib.BS_ERR_INVALID_ARG
