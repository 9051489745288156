"""What the rotary call refuses and takes, on the CPU: with bad arguments nothing is enqueued."""
import ctypes

import pytest
import torch

INVALID, MISALIGNED = -1, -3


@pytest.fixture(scope="module")
def b():
    from paper_2503_15758_amd import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("freq, taken", [(2.0 ** 64, False), (-2.0 ** 64, False), (1e300, False), (float("nan"), False), (-float("inf"), False),
                                         (2.0 ** 64 - 2 ** 11, True), (-2.0 ** 63, True), (5e-324, True), (0.0, True)])
def test_frequencies_too_large(b, freq, taken):
    """From 2^64 on the part of a turn is beyond the bits that it is formed with."""
    freqs = torch.tensor([1.0, freq], dtype=torch.float64)
    d = b.RotaryDesc(rows=10, hdim=128, pairs=2, axes=1, sets=1, in_dtype=1, out_dtype=1, freqs=freqs.data_ptr(), axis=None, positions=0x10000)
    # (a tensor that is not aligned is refused behind the frequencies)
    t = b.RotaryTensor(x=0x10008, y=0x20000, heads=1)
    assert b.lib().a2d_rotary(ctypes.byref(d), 1, ctypes.byref(t), None) == (MISALIGNED if taken else INVALID)
