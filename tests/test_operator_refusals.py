"""What the temporal head's operators refuse before anything reaches a GPU."""
import pytest
import torch

import paper_1806_04965_b200 as sr
from paper_1806_04965_b200 import SrError


@pytest.mark.parametrize("name, value", [("rows", 5000), ("rows", 1 << 40), ("rows", 1 << 70), ("cols", 96), ("cols", 0), ("rows", -1), ("format", "mx8"), ("format", "mx6"),
                                         ("data", torch.zeros(4, 16, dtype=torch.uint8)), ("data", torch.zeros(4, 64, dtype=torch.uint8)[:, ::2]),
                                         ("data", torch.zeros(4, 32, dtype=torch.int8)), ("scales", torch.zeros(4, dtype=torch.uint8))])
def test_a_microscaled_matrix_that_no_longer_fits_its_buffers_is_refused(name, value):
    # its attributes can be assigned after it was made; a kernel would read behind the buffers' ends
    good, bad = sr.Microscaled.empty(4, 64, "mx4", "cpu"), sr.Microscaled.empty(4, 64, "mx4", "cpu")
    setattr(bad, name, value)
    for call in (lambda: bad.values(), lambda: sr.product(good, bad), lambda: sr.product(bad, good), lambda: sr.product(bad, bad)):
        with pytest.raises(SrError, match="sizes|out of range|format"):
            call()


def test_an_argument_without_a_truth_value_raises_its_own_error():
    import numpy as np
    m = sr.Microscaled.empty(4, 64, "mx4", "cpu")
    with pytest.raises((SrError, ValueError)):                  # not a SystemError of a call that returned with an exception set
        sr.product(m, m, relu=np.array([1, 2]))


def test_status_of_something_that_is_no_cuda_device_is_refused():
    for call in (sr.operator_status, sr.operator_reset):
        with pytest.raises(SrError, match="CUDA device"):
            call("cpu")
