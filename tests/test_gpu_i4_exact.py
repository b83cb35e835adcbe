"""Long contractions of the products with 4-bit weights, exact to the last column: both sides of the length up to which tiles take them, the refills of the activations that the
kernels for few tokens hold, offsets of rows near the end of 32 bits."""
import pytest

import i4_exact
from paper_2605_24058_amd import binding

pytestmark = pytest.mark.gpu
M = 1 << 22
SIZES = [(3, M + 1, 24, 128), (8, M, 24, 32), (40, M, 24, 128), (40, M - 1, 24, 64), (40, M + 8, 24, 128), (1030, M, 264, 128), (1030, M - 3, 264, 32), (2100, M // 4, 264, 64),
         (2100, M // 4 - 3, 264, 128)]


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    return torch


@pytest.fixture(autouse=True)
def give_back(torch):
    yield
    torch.cuda.empty_cache()     # (tensors of some tens of GB)


def made(torch, T, k, rows, cols, group):
    gen = torch.Generator(device="cuda").manual_seed(T + k)
    return i4_exact.acts(torch, gen, T, k), i4_exact.weights(torch, gen, rows, cols, group)


@pytest.mark.parametrize("T,k,n,group", SIZES)
def test_linear(torch, T, k, n, group):
    x, W = made(torch, T, k, n, k, group)
    assert i4_exact.same(binding.lordba_linear_i4(x, binding.lordba_layout_i4(*W, group)), i4_exact.product(torch, x, *W, group))


@pytest.mark.parametrize("T,k,n,group", SIZES)
def test_linear_gradient(torch, T, k, n, group):
    g, W = made(torch, T, k, k, n, group)
    assert i4_exact.same(binding.lordba_linear_i4_backward(g, binding.lordba_layout_i4(*W, group, transposed=True)), i4_exact.product(torch, g, *W, group, back=True))


@pytest.mark.parametrize("T,k,n,group", SIZES)
def test_gate_and_up(torch, T, k, n, group):
    x, W = made(torch, T, k, 2 * n, k, group)
    _, kept = binding.lordba_gated_i4(x, binding.lordba_layout_i4(*W, group, halves=2), save=True)
    want = i4_exact.product(torch, x, *W, group)
    assert i4_exact.same(kept[0], want[:, :n]) and i4_exact.same(kept[1], want[:, n:])


@pytest.mark.parametrize("T,k,n,group", SIZES)
def test_gated_gradient(torch, T, k, n, group):
    # up = 2 at a gate of 0, where sigma is 1/2: dgate = dh; a gate of 16, where sigma rounds to 1: dup = 16 dh
    dh, W = made(torch, T, k, 2 * k, n, group)
    laid = binding.lordba_layout_i4(*W, group, halves=2, transposed=True)
    kept = torch.zeros(2, T, k, dtype=torch.float16, device="cuda")
    kept[0, :, 1::2], kept[1, :, ::2] = 16, 2
    dx, dgu = binding.lordba_gated_i4_backward(dh, kept, laid)
    assert torch.equal(dgu[0, :, ::2], dh[:, ::2]) and torch.equal(dgu[1, :, 1::2], 16 * dh[:, 1::2]) and not bool(dgu[0, :, 1::2].any()) and not bool(dgu[1, :, ::2].any())
    want = i4_exact.product(torch, dgu[0], *(t[:k] for t in W), group, back=True) + i4_exact.product(torch, dgu[1], *(t[k:] for t in W), group, back=True)
    assert i4_exact.same(dx, want)
