"""What the selective head's calls in C refuse at their limits: nothing here reaches a GPU."""
import ctypes

import pytest
import torch

from paper_1806_04965_b200 import SrError, operators, selective
from tests.test_selective_cpu import INVALID, conv_desc, conv_run, conv_step, scan_desc, scan_run, scan_step

P3 = ctypes.c_void_p(1 << 23)


@pytest.mark.parametrize("batch", [(1 << 31) - (1 << 16) + 1, (1 << 31) - 31, (1 << 31) - 1])
def test_sequences_that_32_bits_cannot_count_past_are_refused(batch):
    """A search over the sequences adds 31 to their number, a launch over them 65534."""
    small = dict(batch=batch, channels=1)
    strides = dict(x=(batch, 1), out=(batch, 1))
    assert conv_run(conv_desc(width=2, frames=4, **small, **strides), offsets=P3) == INVALID
    assert conv_run(conv_desc(width=2, frames=4, **small, **strides)) == INVALID
    assert conv_step(conv_desc(width=2, **small, **strides)) == INVALID
    d = scan_desc(states=1, groups=1, frames=40, **small)
    size, plan = ctypes.c_size_t(), selective._ScanPlan()
    assert scan_run(d, offsets=P3) == INVALID and scan_run(d) == INVALID and scan_step(d) == INVALID
    for packed in (0, 1):
        assert selective._library().sr_selective_scan_workspace_bytes(ctypes.byref(d), packed, ctypes.byref(size)) == INVALID
        assert selective._library().sr_selective_scan_plan(ctypes.byref(d), packed, 148, ctypes.byref(plan)) == INVALID
    assert selective._library().sr_selective_scan_plan(ctypes.byref(scan_desc(batch=(1 << 31) - (1 << 16), channels=1, states=1, groups=1, frames=1)), 0, 148, ctypes.byref(plan)) == 0


@pytest.mark.parametrize("run,step,desc,channels", [(conv_run, conv_step, conv_desc, 64), (scan_run, scan_step, scan_desc, 64)], ids=["conv", "scan"])
def test_outputs_on_top_of_each_other_are_refused(run, step, desc, channels):
    for frame, sequence in ((0, channels), (channels - 1, 1000), (2 * channels, 0), (2 * channels, channels - 1), (0, 0)):
        assert run(desc(out=(frame, sequence))) == INVALID, (frame, sequence)
    for frame in (0, 1, channels - 1):
        assert run(desc(out=(frame, channels)), offsets=P3) == INVALID, frame
    for sequence in (0, channels - 1):
        assert step(desc(out=(0, sequence))) == INVALID, sequence


def test_sizes_beyond_32_bits_are_not_cut_off():
    """2^32 + 5 sequences are not 5."""
    many = (1 << 32) + 5
    x, w, a, b = torch.zeros(1, 1, 1).expand(1, many, 1), torch.zeros(1, 1), torch.zeros(1, 1), torch.zeros(1, 1, 1, 1).expand(1, many, 1, 1)
    calls = [lambda: selective._conv_desc("causal_conv_run", x, w, None, False, 2, False, many, x), lambda: selective._conv_desc("causal_conv_step", x[0], w, None, False, 1, True, many, x[0]),
             lambda: selective._scan_desc("selective_scan_run", x, x, a, b, b, None, None, None, True, 2, False, many, x),
             lambda: selective.scan_plan(torch.float32, many, 1, 1, 1, sms=148), lambda: selective.scan_plan(torch.float32, 1, 1, many, 1, sms=148),
             lambda: operators.attention_plan(torch.float32, many, 1, 1, 1, 8, 8, sms=148), lambda: operators.attention_plan(torch.float32, 1, 1, 1, 1, 8, many, sms=148)]
    for k, call in enumerate(calls):
        with pytest.raises(SrError):
            call()
            pytest.fail("call %d was taken" % k)
