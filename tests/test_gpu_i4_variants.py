"""The projections, the gated block and their gradients on 4-bit weights, on the shapes that reach the kernels' remaining variants: against 64 bits, on guarded memory."""
import pytest

import i4_variants
import test_gpu_i4_parity as parity

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    return torch


@pytest.mark.parametrize("shift", [0, 1], ids=["aligned", "by-one"])
@pytest.mark.parametrize("T,d_in,d_out,group,zeros", i4_variants.SHAPES)
def test_linear_and_gradient(torch, T, d_in, d_out, group, zeros, shift):
    parity.test_linear_and_gradient(torch, T, d_in, d_out, group, zeros, shift)


@pytest.mark.parametrize("shift", [0, 1], ids=["aligned", "by-one"])
@pytest.mark.parametrize("T,d_in,d_ff,group,zeros", i4_variants.SHAPES)
def test_gated_and_gradient(torch, T, d_in, d_ff, group, zeros, shift):
    parity.test_gated_and_gradient(torch, T, d_in, d_ff, group, zeros, shift)
