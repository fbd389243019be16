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
