"""What the operators' Python entry points make of their arguments before they ask for a GPU."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2111_00705_amd as P
from paper_2111_00705_amd import operators


@pytest.mark.parametrize("bounds", [[2.7], [-1, 0.5], [float("nan")], [float("inf")], [2 ** 31], [-2 ** 31 - 1], [2 ** 70],
                                    np.array([2 ** 32 + 1]), np.array([0, 2 ** 33], dtype=np.uint64), np.array(["1"])],
                         ids=repr)
def test_bounds_that_are_no_32_bit_numbers_are_refused(bounds):
    s = torch.zeros(1, 1, 3, 4)
    with pytest.raises(ValueError, match="bounds must be whole numbers"):
        P.rel_bias_softmax(s, torch.zeros(len(bounds) + 1, 1), bounds)
    with pytest.raises(ValueError, match="bounds must be whole numbers"):
        P.rel_bias_softmax_backward(s, s, bounds, torch.zeros(1, len(bounds) + 1, 1))


@pytest.mark.parametrize("bounds", [[], [-3, 0, 5], (1, 2), np.array([-2 ** 31, 2 ** 31 - 1]), np.array([1.0, 4.0]), np.arange(6, dtype=np.uint8)[::2],
                                    torch.tensor([-1, 7]), np.array([3, 4], dtype=np.int32), np.arange(6, dtype=np.int32)[::2]], ids=repr)
def test_bounds_come_as_they_are(bounds):
    b = operators._bounds(bounds)
    assert b.dtype == np.int32 and b.flags.c_contiguous and b.tolist() == [int(x) for x in bounds]


def test_bounds_have_one_dimension():
    assert operators._bounds(3).tolist() == [3]                  # one bound
    for bounds in ([[1, 2]], np.zeros((2, 2), dtype=np.int32)):
        with pytest.raises(ValueError, match="one-dimensional"):
            operators._bounds(bounds)


def test_a_temperature_whose_reciprocal_leaves_fp32_in_units_of_log_2_is_refused():
    rows = C.c_int64(0)                                          # nothing to do: what is not refused returns at once
    for call in (lambda t: P.lib().comp_ams_distill(None, None, None, None, None, rows, 100, 100, 5, t, 0, None),
                 lambda t: P.lib().comp_ams_distill_backward(None, None, None, None, None, None, rows, 100, 100, 100, 5, t, 0, None),
                 lambda t: P.lib().comp_ams_distill_grad(None, None, None, None, None, None, rows, 100, 100, 100, 5, t, 0, None)):
        assert call(3.5e-39) == P.EINVAL and call(1e-45) == P.EINVAL
        assert call(1e-38) == P.OK and call(1.0) == P.OK
