"""Temperatures that the distilling calls refuse, before a device is touched."""
import ctypes

import pytest

from paper_2605_24058_amd import binding

VALUE, NO_DEVICE = 3, 6
BUF = [(i + 1) << 40 for i in range(8)]     # addresses that are never followed


@pytest.mark.parametrize("u,accepted", [(1e-39, False), (2.0 ** -149, False), (2.0 ** -126, True), (3e38, True)])
def test_temperatures_are_normal_numbers(u, accepted):
    import torch
    if accepted and torch.cuda.is_available():
        pytest.skip("the addresses above are not memory")
    lib = binding.load_library()
    w = ctypes.byref(binding.Teacher(BUF[1], BUF[2], None, 3, u, 1.0, 0.0))
    want = NO_DEVICE if accepted else VALUE
    assert lib.lordba_distill(BUF[0], 0, w, None, BUF[3], BUF[4], None, 4, 100, None) == want
    assert lib.lordba_distill_backward(BUF[5], BUF[0], 0, BUF[4], w, BUF[6], 4, 100, None) == want
