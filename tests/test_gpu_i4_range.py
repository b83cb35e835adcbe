"""The gated block on 4-bit weights where gate, up and the gradients with respect to them pass the range of fp16: what comes of them is a number for many, and has to be that number."""
import numpy as np
import pytest

import i4_checks
import i8_checks
from paper_2605_24058_amd import binding

pytestmark = pytest.mark.gpu
LARGEST = 65504.0

# T, d_in, d_ff, group, zero points, the kernel of the product (two planes of d_ff columns, d_in outputs)
CASES = [(3, 40, 64, 32, True, "few"), (5, 33, 70, 128, False, "few"), (2, 9, 5, 32, True, "few"), (8, 4200, 136, 64, True, "few"), (8, 8200, 43, 64, False, "few"),
         (12, 24, 2056, 64, True, "tile32"), (17, 3001, 777, 128, False, "tile32"), (17, 4104, 136, 32, False, "tile64"), (777, 40, 43, 64, True, "tile64"),
         (17, 4099, 40, 128, True, "tile128"), (100, 8200, 41, 32, True, "tile128"), (2100, 1991, 40, 128, False, "tile256"), (2100, 2000, 45, 32, True, "tile256")]


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    return torch


def inputs(torch, T, d_in, F, group, zeros):
    """Every third token has a few gradients past the range: a gate that the forward pass kept as the largest number, an up of that size beside a gate of some units."""
    rng = np.random.default_rng(T + F)
    codes, scale, zero = i4_checks.weights(torch, rng, 2 * F, d_in, group, zeros)
    scale = scale * min(1.0, d_in ** 0.5 / 64)      # (dx stays inside the range)
    codes[:, ::5] = 8 if zero is None else zero[:, torch.arange(0, d_in, 5) // group]     # weights of 0 in every row
    dh, gate_up = i8_checks.acts(rng, T, F), i8_checks.acts(rng, 2 * T, F).reshape(2, T, F)
    for t in range(1, T, 3):
        for j, (gate, up, d) in zip(rng.choice(F, size=3, replace=False), ((LARGEST, 0.01, 2.0), (3.0, -LARGEST, 1.5), (LARGEST, 0.02, -3.0))):
            gate_up[0, t, j], gate_up[1, t, j], dh[t, j] = gate, up, d
    return codes, scale, zero, dh, gate_up


def expected(torch, codes, scale, zero, group, dg, du, eg, eu, rounded):
    """dx and the bound of its error: of the 64-bit dgate and dup, or of the numbers that they are kept as"""
    W = i4_checks.real(torch, codes, scale, zero, group, rounded).cuda()
    both, err = torch.cat([dg, du], dim=1), torch.cat([eg, eu], dim=1)
    want, sums = i4_checks.product(torch, both, W.t().contiguous())
    return want, sums + torch.mm(err, W.abs())


@pytest.mark.parametrize("shift", [0, 1], ids=["aligned", "by-one"])
@pytest.mark.parametrize("T,d_in,F,group,zeros,kernel", CASES)
def test_gradients_past_the_range(torch, T, d_in, F, group, zeros, kernel, shift):
    assert shift or i4_checks.kernel(T, F, d_in, 2, backward=True) == kernel
    codes, scale, zero, dh, gate_up = inputs(torch, T, d_in, F, group, zeros)
    mem = i8_checks.Memory(torch)
    laid = binding.lordba_layout_i4(codes.cuda(), scale.cuda(), None if zero is None else zero.cuda(), group, halves=2, transposed=True)
    dx, dgu = mem.output((T, d_in), torch.float16, shift), mem.output((2, T, F), torch.float16, shift)
    i8_checks.call(torch, "lordba_gated_i4_backward", mem.input(dh, shift), mem.input(gate_up, shift), laid.codes, laid.scale, laid.zero, dx, dgu, T, d_in, F, group)
    mem.unchanged()
    dg, du, eg, eu = i8_checks.gated_gradient(torch, dh, gate_up)
    i8_checks.near(dgu[0], dg, eg)
    i8_checks.near(dgu[1], du, eu)
    past = torch.isinf(dgu).any(dim=2).any(dim=0)
    assert past.cpu().tolist() == [t % 3 == 1 for t in range(T)]
    none = torch.zeros_like(eg[~past])
    i8_checks.near(dx[~past], *expected(torch, codes, scale, zero, group, dgu[0][~past].double(), dgu[1][~past].double(), none, none, True))
    want, err = expected(torch, codes, scale, zero, group, dg[past], du[past], eg[past], eu[past], False)
    assert float(want.abs().max()) < LARGEST
    i8_checks.near(dx[past], want, err)


@pytest.mark.parametrize("T,d_in,F,group,zeros,kernel", CASES[::3])
def test_what_is_no_number_stays_in_its_token(torch, T, d_in, F, group, zeros, kernel):
    codes, scale, zero, dh, gate_up = inputs(torch, T, d_in, F, group, zeros)
    scale = scale.abs() + 0.001
    laid = binding.lordba_layout_i4(codes.cuda(), scale.cuda(), None if zero is None else zero.cuda(), group, halves=2, transposed=True)
    call = lambda d, gu: binding.lordba_gated_i4_backward(torch.from_numpy(d).cuda(), torch.from_numpy(gu).cuda(), laid)
    dx, dgu = call(dh, gate_up)
    dh2, gate_up2 = dh.copy(), gate_up.copy()
    dh2[0, F - 1], gate_up2[1, T - 1, 0], dh2[T - 1, 0] = np.inf, np.nan, 1.0
    dx2, dgu2 = call(dh2, gate_up2)
    others = torch.ones(T, dtype=torch.bool, device="cuda")
    others[0] = others[T - 1] = False
    assert torch.equal(dx2[others], dx[others]) and torch.equal(dgu2[:, others], dgu[:, others])
    assert not bool(torch.isfinite(dx2[0]).any()) and bool(torch.isnan(dx2[T - 1]).all())


@pytest.mark.parametrize("shift", [0, 1], ids=["aligned", "by-one"])
@pytest.mark.parametrize("T,d_in,F,group,kernel", [(2, 2, 40, 32, "few"), (5, 40, 41, 64, "few"), (40, 528, 1501, 128, "tile32"), (17, 264, 1991, 32, "tile64"), (17, 40, 1991, 64, "tile128"),
                                                   (200, 40, 8200, 128, "tile256"), (200, 40, 8199, 32, "tile256")])
def test_a_gate_past_the_range_has_finite_gradients(torch, T, d_in, F, group, kernel, shift):
    # x = (600, 0, ...): one weight of 15 x 8 gives +-72000; gate and up get the rest from the addends, and silu(-12) = -7.4e-5, so their product with 72000 is small
    assert shift or i4_checks.kernel(T, d_in, F, gated=True) == kernel
    rng, kind = np.random.default_rng(F), np.arange(F) % 5
    sign = np.concatenate([np.choose(kind, [-1, 1, 0, 0, -1]), np.choose(kind, [0, 0, 1, -1, 0])])
    zero = np.where(sign < 0, 15, np.where(sign > 0, 0, 6)).astype(np.uint8)[:, None].repeat(-(-d_in // group), axis=1)
    codes = np.repeat(zero[:, :1], d_in, axis=1)
    codes[:, 0] = np.where(sign < 0, 0, np.where(sign > 0, 15, 6))
    x = np.zeros((T, d_in), np.float16)
    x[:, 0] = 600
    add = rng.uniform(0.001, 0.01, size=(2, T, F)).astype(np.float16)
    add[0][:, kind >= 2] -= np.float16(12)
    cu = lambda a: torch.from_numpy(a).cuda()
    plain = cu(codes), torch.full(zero.shape, 8.0, dtype=torch.float16, device="cuda"), cu(zero)
    mem = i8_checks.Memory(torch)
    h, kept = mem.output((T, F), torch.float16, shift), mem.output((2, T, F), torch.float16, shift)
    laid = binding.lordba_layout_i4(*plain, group, halves=2)
    i8_checks.call(torch, "lordba_gated_i4", mem.input(x, shift), laid.codes, laid.scale, laid.zero, mem.input(add, shift), h, kept, T, d_in, F, group)
    mem.unchanged()
    base = cu(600.0 * 120.0 * sign)
    gate, up = base[:F] + cu(add[0]).double(), base[F:] + cu(add[1]).double()
    silu = gate * torch.sigmoid(gate)
    assert float(gate.abs().max()) > 70000 < float(up.abs().max()) and float((silu * up).abs().max()) < 1000
    # (the product is exact; the addition is rounded)
    eg, eu = gate.abs() * 2.0 ** -24, up.abs() * 2.0 ** -24
    i8_checks.near(h, silu * up, 1.1 * up.abs() * eg + silu.abs() * eu + (silu * up).abs() * 2.0 ** -18 * (1 + gate.abs() / 16))
    i8_checks.near(kept[0], gate.clamp(-LARGEST, LARGEST), eg)
    i8_checks.near(kept[1], up.clamp(-LARGEST, LARGEST), eu)
    dh = rng.uniform(0.1, 0.5, size=(T, F)).astype(np.float16)
    dx, dgu = binding.lordba_gated_i4_backward(cu(dh), kept, binding.lordba_layout_i4(*plain, group, halves=2, transposed=True))
    dg, du, eg, eu = i8_checks.gated_gradient(torch, dh, kept.cpu().numpy())
    i8_checks.near(dgu[0], dg, eg)
    i8_checks.near(dgu[1], du, eu)
    assert bool(torch.isfinite(dgu).all()) and not bool(torch.isnan(dx).any())


def test_what_is_no_number_is_kept_as_none(torch):
    for T, F in ((4, 70), (40, 70), (200, 1000)):
        add = np.zeros((2, T, F), np.float16)
        add[0, 3, 5], add[1, T // 2, 69], add[0, 1, 7], add[1, T - 1, 0] = np.nan, np.nan, np.inf, -np.inf
        W = binding.lordba_layout_i4(torch.full((2 * F, 9), 8, dtype=torch.uint8, device="cuda"), torch.ones(2 * F, 1, dtype=torch.float16, device="cuda"), group=32, halves=2)
        h, kept = binding.lordba_gated_i4(torch.ones(T, 9, dtype=torch.float16, device="cuda"), W, addends=torch.from_numpy(add).cuda(), save=True)
        want = np.where(np.isinf(add), np.sign(add) * LARGEST, add.astype(np.float64))
        assert np.array_equal(kept.cpu().numpy().astype(np.float64), want, equal_nan=True)
        assert np.isnan(h.cpu().numpy()[[3, T // 2, 1], [5, 69, 7]]).all()     # (infinity times an up of 0)


@pytest.mark.parametrize("T,d_in,F,group,zeros,kernel", CASES[1::4])
def test_gradients_past_the_range_in_graphs_and_on_two_streams(torch, T, d_in, F, group, zeros, kernel):
    codes, scale, zero, dh, gate_up = inputs(torch, T, d_in, F, group, zeros)
    laid = binding.lordba_layout_i4(codes.cuda(), scale.cuda(), None if zero is None else zero.cuda(), group, halves=2, transposed=True)
    d, gu = torch.from_numpy(dh).cuda(), torch.from_numpy(gate_up).cuda()
    call = lambda **kw: binding.lordba_gated_i4_backward(d, gu, laid, **kw)
    want = [t.clone() for t in call()]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    both = [call(stream=s) for s in streams]      # at once
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for got in both for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for k in range(4):                            # tokens in range, and past it again
        d.copy_(torch.from_numpy(dh).cuda() * (0.125 if k % 2 == 0 else 1.0))
        graph.replay()
        torch.cuda.synchronize()
        again = call()
        assert all(torch.equal(a, b) for a, b in zip(out, again)), k
        assert bool(torch.isinf(out[1]).any()) is (k % 2 == 1) and bool(torch.isfinite(out[0]).all())
