"""The time-out path of bs_prompt_attention, read from the source: every wait is internal to a CTA, so no input makes one run out, and
what the kernel does after one can only be stated about the code (nothing is launched here)."""
import os
import re

from conftest import ROOT

SRC = re.sub(r"//[^\n]*", "", open(os.path.join(ROOT, "paper_2505_15141_b200", "csrc", "bs_prompt_attention.cu")).read())


def _end():
    """From the barrier at which all roles meet."""
    at = SRC.index("if (s_abort) {")
    return SRC[SRC.rindex("__syncthreads();", 0, at):SRC.index("tc_free(tmem", at)]


def test_every_role_tells_that_it_gave_up():
    body = SRC[SRC.index("if (warp == 10) {"):SRC.index("if (s_abort) {")]
    assert body.count("s_abort = 1;") == 5            # scheduler, copies, products, softmax, V


def test_nothing_is_in_flight_when_a_cta_that_gave_up_ends():
    """Copies of the ring, those by way of the V warp, queries; products and the launch control's answer before the roles meet."""
    end = _end()
    assert end.index("s_copies") < end.index("pa_wait<true>(&b_full") < end.index("pa_wait<true>(&b_part") < end.index("pa_wait<true>(&b_qfull")
    before = SRC[:SRC.index("if (s_abort) {")]
    assert before.count("pa_wait<true>(&b_drain, 0, p.limit, &s_abort)") == 1
    assert before.count("if (asked != answered) pa_wait<true>(&b_next, answered & 1, p.limit, &s_abort);") == 1


def test_a_time_out_is_kept_where_the_host_can_read_it():
    """With or without a status array, behind the drain."""
    end = _end()
    at = end.index("g_pa_gave_up = 1u;")
    assert end.index("pa_wait<true>(&b_qfull") < at < end.index("if (p.status) atomicOr(p.status, BS_DEV_TIMEOUT);")
    assert "p.status" not in end[:at]
    read = SRC[SRC.index("bs_prompt_get_device_status("):]
    read = read[:read.index("\n}\n")]
    assert read.index("cudaGetSymbolAddress(&at, g_pa_gave_up)") < read.index("cudaMemcpyAsync(&gave_up, at") < read.index("cudaStreamSynchronize")
    assert read.index("cudaMemsetAsync(at, 0") < read.index("return gave_up ? BS_ERR_TIMEOUT : BS_OK;")


def test_the_answer_is_taken_on_the_gpu_asked_for(lib, monkeypatch):
    seen = []
    monkeypatch.setattr(lib, "_call", lambda fn, where, index, stream: seen.append((where, index, stream)))
    lib.bs_prompt_get_device_status("cuda:3", 17)
    lib.bs_prompt_get_device_status(stream=None, device="cuda:0")
    assert seen == [("bs_prompt_get_device_status", 3, 17), ("bs_prompt_get_device_status", 0, None)]
