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


def test_the_binding_imports_without_torchs_private_stream_call(lib):
    """A torch without CUDA has no torch._C._cuda_getCurrentRawStream."""
    code = """
import torch
if hasattr(torch._C, "_cuda_getCurrentRawStream"):
    del torch._C._cuda_getCurrentRawStream
from paper_2505_15141_b200 import binding
assert callable(binding._raw_stream)
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
