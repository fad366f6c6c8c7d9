"""What the binding of the site norm, the residual tail and the checkpoints refuses before it reaches the library, and so
without a GPU."""
import os

import numpy as np
import pytest

from paper_2111_07383_amd import _abi
from paper_2111_07383_amd import binding as B

pytestmark = pytest.mark.skipif(not os.path.exists(_abi.LIB_PATH), reason="libssconv.so not built")


@pytest.mark.parametrize("bad", [2.5, -0.5, "2", float("inf"), float("nan"), 2 ** 32 + 2, -2 ** 31])
def test_orders_and_multiplicities_are_whole_numbers(bad):
    """A fraction is not cut off, and a number past 32 bits not taken for its lowest bits."""
    for f in (((0, bad),), ((bad, 1),), ((0, 3), (1, bad)), [[0, bad]]):
        for call in (B.gate_fields, B.packed_blocks):
            with pytest.raises((ValueError, OverflowError)):
                call(f)


def test_whole_numbers_of_any_type():
    want = ((0, 3), (1, 2), (0, 2))
    for f in (((0, 3), (1, 2)), [[0, 3], [1, 2]], ((0.0, 3.0), (1, np.int64(2))), np.array([[0, 3], [1, 2]])):
        assert B.gate_fields(f) == want and all(type(v) is int for e in B.gate_fields(f) for v in e)


def test_stream_of_another_device():
    """The tensors are those of the current device, and a launch on another device's stream would reach them from there."""
    class Stream:
        device_index, cuda_stream = 1, 4096

    assert B._raw_stream(Stream, 1) == 4096
    with pytest.raises(ValueError):
        B._raw_stream(Stream, 0)
