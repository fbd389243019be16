"""What the Python binding of the cache calls refuses by itself, before the library is called (no GPU needed)."""
import subprocess
import sys

import pytest
import torch

from conftest import ROOT


@pytest.mark.parametrize("which", [0, 2])
@pytest.mark.parametrize("dtype", [torch.float8_e5m2, torch.int8, torch.bool])
def test_codes_of_another_type_are_refused(lib, dtype, which):
    """One byte is not enough: e5m2 read as e4m3 gives other numbers without a word."""
    kc, ks = lib.new_cache(4, 2, 16, 64, device="cpu")
    args = [kc, ks, kc.clone(), ks.clone()]
    args[which] = torch.zeros(kc.shape, dtype=torch.uint8).view(dtype)
    with pytest.raises(AssertionError, match="float8_e4m3fn"):
        lib._cache_args(*args)


def test_the_binding_imports_without_torchs_private_calls(lib):
    """A torch without CUDA has neither torch._C._cuda_getCurrentRawStream nor torch._C._cuda_getDevice."""
    code = """
import torch
for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"):
    if hasattr(torch._C, name):
        delattr(torch._C, name)
from paper_2505_15141_b200 import binding
assert callable(binding._raw_stream) and callable(binding._current_gpu)
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr


class Placed:
    """A tensor in host memory that says it is on GPU `index`."""

    def __init__(self, t, index=0):
        self.t, self.index = t, index

    def get_device(self):
        return self.index

    @property
    def device(self):
        return torch.device("cuda", self.index) if self.index >= 0 else torch.device("cpu")

    def __getattr__(self, name):
        return getattr(self.t, name)


def _calls(lib):
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    B, W, N, T, H = 3, 4, 5, 8, 2
    kc, ks = lib.new_cache(6, H, 16, 64, device="cpu")
    x = torch.zeros(T, H, 64, dtype=torch.bfloat16)
    q, ws = torch.zeros(T, 4, 64, dtype=torch.bfloat16), torch.zeros(1 << 10, dtype=torch.uint8)
    cache = [kc, ks, kc.clone(), ks.clone()]
    plan = [i(B), i(B), i(B), 1, torch.ones(B, dtype=torch.uint8), 16, i(B, W), i(B), i(6), i(1), i(B), i(B + 1), i(T), i(T), i(B)]
    return {
        "bs_cache_plan": (plan, {}),
        "bs_cache_plan (next)": (plan, {"last_cu": i(B + 1), "n_shared": i(B)}),
        "bs_cache_append": ([x, x.clone(), i(T)] + cache, {}),
        "bs_cache_attention": ([q, i(B + 1), i(B), i(B, W), i(B, N)] + cache + [4, 0.1, q.clone(), i(B), ws], {}),
        "bs_cache_get_device_status": ([ws], {}),
        "bs_cache_keep_path": ([i(B, N), i(B), i(B), i(B, W)] + cache + [i(B)], {}),
    }


@pytest.mark.parametrize("name", ["bs_cache_plan", "bs_cache_plan (next)", "bs_cache_append", "bs_cache_attention",
                                  "bs_cache_get_device_status", "bs_cache_keep_path"])
def test_every_tensor_has_to_be_on_the_calls_gpu(lib, monkeypatch, name):
    """A pointer into host memory, or into another GPU's, would fault in the kernel: each argument in turn is elsewhere."""
    made = []
    monkeypatch.setattr(lib, "_call", lambda fn, where, *a: made.append(where))
    fn = getattr(lib, name.split()[0])
    args, kw = _calls(lib)[name]

    def place(x, index=0):
        return Placed(x, index) if isinstance(x, torch.Tensor) else x

    fn(*[place(x) for x in args], **{k: place(x) for k, x in kw.items()})
    assert made == [name.split()[0]]
    tensors = [n for n, x in enumerate(args) if isinstance(x, torch.Tensor)] + [k for k, x in kw.items()]
    assert len(tensors) == {"bs_cache_plan": 13, "bs_cache_plan (next)": 15, "bs_cache_append": 7, "bs_cache_attention": 12,
                            "bs_cache_get_device_status": 1, "bs_cache_keep_path": 9}[name]
    elsewhere = (-1,) if len(tensors) == 1 else (-1, 1)
    for which in tensors:
        for index in elsewhere:
            a, k = [place(x) for x in args], {n: place(x) for n, x in kw.items()}
            (k if isinstance(which, str) else a)[which].index = index
            with pytest.raises(AssertionError, match="GPU"):
                fn(*a, **k)
    with pytest.raises(AssertionError, match="GPU"):         # all of them in host memory
        fn(*[place(x, -1) for x in args], **{k: place(x, -1) for k, x in kw.items()})
    assert len(made) == 1


def test_trees_without_drafts_are_not_chains(lib, monkeypatch):
    """An empty tensor has no address, and NULL means chains."""
    seen = []
    monkeypatch.setattr(lib, "_call", lambda fn, where, index, stream, *a: seen.append(a))
    args, _ = _calls(lib)["bs_cache_attention"]
    args[4] = torch.zeros(3, 0, dtype=torch.int32)
    lib.bs_cache_attention(*[Placed(x) if isinstance(x, torch.Tensor) else x for x in args])
    args[4] = None
    lib.bs_cache_attention(*[Placed(x) if isinstance(x, torch.Tensor) else x for x in args])
    assert seen[0][7] and seen[0][8] == 0 and seen[1][7] is None and seen[1][8] == 0
