"""Rows with one entry far above the others in two digits: every result inside half a step per entry, and the error of the whole what the header says,
8.9e-6 of the norm for each unit of largest / rms beside the 2.1e-4 of the rounding to fp16."""
import numpy as np
import pytest

import i8_checks as c

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    c.binding.load_library()
    return torch


def rows(rng, T, n, outlier):
    v = rng.standard_normal((T, n))
    if outlier:
        v[np.arange(T), rng.integers(0, n, size=T)] = outlier
    return v.astype(np.float16)


def check(torch, got, want, err, numbers):
    c.near(got, want, err)
    # Roundings to steps are uniform and independent: step / sqrt(12) of each entry, a weight's rms times that per result, and the result's rms is the rows'
    # times the weight's: largest / (D sqrt(12) rms).  fp16 rounds by 2^-11 / sqrt(3) of a value times 0.72 at most (uniform mantissas), 2.1e-4.
    # T x n such errors average to within 10 %.
    ratio = numbers.abs().amax(dim=1) / numbers.square().mean(dim=1).sqrt()
    size = want.square().sum(dim=1)
    stated = float((((8.9e-6 * ratio) ** 2 + 2.1e-4 ** 2) * size).sum().div(size.sum()).sqrt())
    seen = float((got.double() - want).norm() / want.norm())
    assert 0.9 * stated <= seen <= 1.1 * stated, (seen, stated)


@pytest.mark.parametrize("outlier", [0, 30, 100, 300])
def test_projections(torch, outlier):
    rng = np.random.default_rng(outlier)
    T, n, k = 96, 700, 4096
    W, _ = c.weights(rng, n, k)
    ws = np.full(n, 1e-3, np.float32)
    x, w = rows(rng, T, k, outlier), torch.from_numpy(W).cuda()
    xd, wsd = torch.from_numpy(x).cuda(), torch.from_numpy(ws).cuda()
    y = c.binding.lordba_linear_i8(xd, c.binding.lordba_layout_i8(w), wsd, digits=2)
    check(torch, y, *c.row_error(torch, xd.double(), 2.0 ** -22 * xd.double().abs(), np.full(k, 1e-3, np.float32), w, 2), xd.double())
    # the gradient contracts the other side: rows of g times one scale each
    one = torch.full((k,), 1e-3, device="cuda")
    dx = c.binding.lordba_linear_i8_backward(xd, c.binding.lordba_layout_i8(w), one)
    check(torch, dx, *c.row_error(torch, xd.double(), 2.0 ** -22 * xd.double().abs(), np.full(k, 1e-3, np.float32), w, 2), xd.double())


@pytest.mark.parametrize("outlier", [0, 30, 100, 300])
def test_the_gated_gradient(torch, outlier):
    rng = np.random.default_rng(7 + outlier)
    T, n, F = 96, 700, 2048
    W, _ = c.weights(rng, n, 2 * F)
    ws = np.full(2 * F, 1e-3, np.float32)
    dh, gate_up = rows(rng, T, F, outlier), rng.standard_normal((2, T, F)).astype(np.float16)
    w = torch.from_numpy(W).cuda()
    dx, dgu = c.binding.lordba_gated_i8_backward(torch.from_numpy(dh).cuda(), torch.from_numpy(gate_up).cuda(), c.binding.lordba_layout_i8(w), torch.from_numpy(ws).cuda())
    dg, du, eg, eu = c.gated_gradient(torch, dh, gate_up)
    both = torch.cat([dg, du], dim=1)
    check(torch, dx, *c.row_error(torch, both, torch.cat([eg, eu], dim=1), ws, w, 2), both)
