"""Gates and ups past the range of fp16: h is a finite number for many of them, so their gradients have to be numbers too."""
import numpy as np
import pytest

import i8_checks as c

pytestmark = pytest.mark.gpu
LARGEST = 65504.0


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    c.binding.load_library()
    return torch


# one launch with the rows, the small tiles and the large ones; even and odd widths, whole tiles and ragged ones
@pytest.mark.parametrize("T,F,digits", [(2, 40, 1), (2, 41, 2), (70, 64, 1), (65, 131, 2), (768, 8320, 1), (768, 8320, 2), (385, 5505, 1)])
def test_a_gate_past_the_range_has_finite_gradients(torch, T, F, digits):
    # x = (600, 0): one weight of 127 gives +-76200, which is exact in every digit; up and gate get the rest from the addends
    rng = np.random.default_rng(F)
    W = np.zeros((2 * F, 2), np.int8)
    kind = np.arange(F) % 5
    W[:F, 0] = np.choose(kind, [-127, 127, 0, 0, -127])
    W[F:, 0] = np.choose(kind, [0, 0, 127, -127, 127])
    x, ws = np.zeros((T, 2), np.float16), np.ones(2 * F, np.float32)
    x[:, 0] = 600
    add = rng.uniform(0.001, 0.01, size=(2, T, F)).astype(np.float16)     # (76200 x 0.01 stays inside the range of h)
    add[0][:, kind >= 2] -= np.float16(12)                                # (silu(-12) = -7.4e-5: so does its product with 76200)
    w = torch.from_numpy(W).cuda()
    q, s = c.rows_of(x, None, digits)
    gate, up, h, eg, eu, eh = c.gated(torch, q, s, w, ws, add)
    assert float(gate.abs().max()) > 70000 < float(up.abs().max()) and float(h.abs().max()) < 1000
    for shift in (0, 1):
        mem = c.Memory(torch)
        got, kept = mem.output((T, F), torch.float16, shift), mem.output((2, T, F), torch.float16, shift)
        space = c.workspace(mem, T, 2, digits)
        c.call(torch, "lordba_gated_i8", mem.input(x), mem.input(c.binding.lordba_layout_i8(w)), mem.input(ws), mem.input(add), got, kept, space, space.numel(),
               T, 2, F, digits)
        mem.unchanged()
        c.near(got, h, eh)
        c.near(kept[0], gate.clamp(-LARGEST, LARGEST), eg)
        c.near(kept[1], up.clamp(-LARGEST, LARGEST), eu)
    dh = rng.uniform(0.1, 0.5, size=(T, F)).astype(np.float16)
    dx, dgu = c.binding.lordba_gated_i8_backward(torch.from_numpy(dh).cuda(), kept, c.binding.lordba_layout_i8(w, True), torch.from_numpy(ws).cuda())
    dg, du, eg, eu = c.gated_gradient(torch, dh, kept.cpu().numpy())
    c.near(dgu[0], dg, eg)
    c.near(dgu[1], du, eu)
    assert bool(torch.isfinite(dgu).all()) and not bool(torch.isnan(dx).any())
    # what the largest number stands for differs from the gate itself by the flat parts of silu only
    d = torch.from_numpy(dh).cuda().double()
    sigma, rest = torch.sigmoid(gate), torch.sigmoid(-gate)
    inside = up.abs() <= LARGEST
    c.near(dgu[0][inside], (d * up * sigma * (1 + gate * rest))[inside], (d * up).abs()[inside] * 2.0 ** -10)   # (up is kept in fp16)


def test_what_is_no_number_is_kept_as_none(torch):
    T, F = 40, 70
    add = np.zeros((2, T, F), np.float16)
    add[0, 3, 5], add[1, 20, 69], add[0, 7, 7], add[1, 39, 0] = np.nan, np.nan, np.inf, -np.inf
    W = torch.zeros(2 * F, 9, dtype=torch.int8, device="cuda")
    h, kept = c.binding.lordba_gated_i8(torch.ones(T, 9, dtype=torch.float16, device="cuda"), c.binding.lordba_layout_i8(W), torch.ones(2 * F, device="cuda"),
                                        addends=torch.from_numpy(add).cuda(), save=True)
    want = np.where(np.isinf(add), np.sign(add) * LARGEST, add.astype(np.float64))
    got = kept.cpu().numpy().astype(np.float64)
    assert np.array_equal(got, want, equal_nan=True)
    assert np.isnan(h.cpu().numpy()[[3, 20, 7], [5, 69, 7]]).all()     # (infinity times an up of 0)
