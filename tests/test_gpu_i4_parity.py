"""The 4-bit projections, their gradients and the gated block against their definitions in 64 bits, on guarded memory."""
import numpy as np
import pytest

import i4_checks
import i8_checks
from paper_2605_24058_amd import binding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    return torch


def laid_out(torch, mem, codes, scale, zero, group, halves=1, transposed=False):
    """The three laid-out tensors on guarded memory, made there from the guarded plain ones."""
    lib = binding.load_library()
    rows, cols = codes.shape
    n = lib.lordba_i4_scale_count(rows, cols, group, halves, int(transposed))
    plain = [mem.input(codes), mem.input(scale, 1), None if zero is None else mem.input(zero, 1)]
    out = [mem.output((lib.lordba_i4_code_bytes(rows, cols, halves, int(transposed)),), torch.uint8), mem.output((n,), torch.float16),
           None if zero is None else mem.output((n,), torch.float16)]
    i8_checks.call(torch, "lordba_layout_i4", *plain, *out, rows, cols, group, halves, int(transposed))
    return out


def acts(torch, rng, rows, cols):
    return torch.from_numpy(i8_checks.acts(rng, rows, cols)).cuda()


@pytest.mark.parametrize("shift", [0, 1], ids=["aligned", "by-one"])
@pytest.mark.parametrize("T,d_in,d_out,group,zeros", i4_checks.SHAPES)
def test_linear_and_gradient(torch, T, d_in, d_out, group, zeros, shift):
    rng = np.random.default_rng(T + d_in)
    mem = i8_checks.Memory(torch)
    codes, scale, zero = i4_checks.weights(torch, rng, d_out, d_in, group, zeros)
    x, g = mem.input(acts(torch, rng, T, d_in), shift), mem.input(acts(torch, rng, T, d_out), shift)
    for backward in (False, True):
        W = i4_checks.real(torch, codes, scale, zero, group, rounded=backward or i4_checks.kernel(T, d_in, d_out, aligned=shift == 0, fine_zeros=zeros and group == 32) != "few").cuda()
        y = mem.output((T, d_in if backward else d_out), torch.float16, shift)
        i8_checks.call(torch, "lordba_linear_i4" + "_backward" * backward, g if backward else x, *laid_out(torch, mem, codes, scale, zero, group, 1, backward), y,
                       T, d_in, d_out, group)
        want, err = i4_checks.product(torch, (g if backward else x).double(), W.t().contiguous() if backward else W)
        i8_checks.near(y, want, err)
    mem.unchanged()


@pytest.mark.parametrize("shift", [0, 1], ids=["aligned", "by-one"])
@pytest.mark.parametrize("T,d_in,d_ff,group,zeros", i4_checks.SHAPES)
def test_gated_and_gradient(torch, T, d_in, d_ff, group, zeros, shift):
    rng = np.random.default_rng(T + d_in + 1)
    mem = i8_checks.Memory(torch)
    codes, scale, zero = i4_checks.weights(torch, rng, 2 * d_ff, d_in, group, zeros)
    x, add, dh = mem.input(acts(torch, rng, T, d_in), shift), mem.input(torch.randn(2, T, d_ff).half().cuda(), shift), mem.input(acts(torch, rng, T, d_ff), shift)
    W = i4_checks.real(torch, codes, scale, zero, group, rounded=i4_checks.kernel(T, d_in, d_ff, gated=True, aligned=shift == 0, fine_zeros=zeros and group == 32) != "few").cuda()
    L = laid_out(torch, mem, codes, scale, zero, group, 2)
    both, err = i4_checks.product(torch, x.double(), W)
    for addends, keep in ((add, True), (None, False)):
        h, kept = mem.output((T, d_ff), torch.float16, shift), mem.output((2, T, d_ff), torch.float16, shift) if keep else None
        i8_checks.call(torch, "lordba_gated_i4", x, *L, addends, h, kept, T, d_in, d_ff, group)
        gate, up = (both[:, p * d_ff:(p + 1) * d_ff] + (addends[p].double() if keep else 0) for p in (0, 1))
        eg, eu = err[:, :d_ff] + gate.abs() * 2.0 ** -23, err[:, d_ff:] + up.abs() * 2.0 ** -23
        silu = gate * torch.sigmoid(gate)
        # |silu'| <= 1.1; silu itself: the exponential's and the quotient's roundings, 2^-18 with the argument's 2^-24 |gate| in it
        i8_checks.near(h, silu * up, 1.1 * up.abs() * eg + silu.abs() * eu + (silu * up).abs() * 2.0 ** -18 * (1 + gate.abs() / 16))
        if keep:
            i8_checks.near(kept[0], gate, eg)
            i8_checks.near(kept[1], up, eu)
    gate_up = torch.from_numpy(i8_checks.acts(rng, 2 * T, d_ff)).view(2, T, d_ff)
    dx, dgu = mem.output((T, d_in), torch.float16, shift), mem.output((2, T, d_ff), torch.float16, shift)
    i8_checks.call(torch, "lordba_gated_i4_backward", dh, mem.input(gate_up, shift), *laid_out(torch, mem, codes, scale, zero, group, 2, True), dx, dgu, T, d_in, d_ff,
                   group)
    dg, du, eg, eu = i8_checks.gated_gradient(torch, dh.cpu().numpy(), gate_up.numpy())
    i8_checks.near(dgu[0], dg, eg)
    i8_checks.near(dgu[1], du, eu)
    # dx is the product of the numbers that dgate_up holds
    Wt = i4_checks.real(torch, codes, scale, zero, group, rounded=True).cuda().t().contiguous()
    i8_checks.near(dx, *i4_checks.product(torch, torch.cat([dgu[0], dgu[1]], dim=1).double(), Wt))
    mem.unchanged()


@pytest.mark.parametrize("T", [3, 100])
def test_subnormal_weights(torch, T):
    # scales of some 1e-7: the products scale * (code - zero) are subnormal fp16 numbers, whole multiples of the smallest
    rng = np.random.default_rng(5)
    codes, scale, zero = i4_checks.weights(torch, rng, 96, 200, 64, True, tiny=True)
    x, g = acts(torch, rng, T, 200) * 64, acts(torch, rng, T, 96) * 64
    dev = [codes.cuda(), scale.cuda(), zero.cuda()]
    W = i4_checks.real(torch, codes, scale, zero, 64, rounded=False).cuda()
    assert float(W.abs().max()) < 2.0 ** -14 and torch.equal(W, W.half().double())
    i8_checks.near(binding.lordba_linear_i4(x, binding.lordba_layout_i4(*dev, 64)), *i4_checks.product(torch, x.double(), W))
    dx = binding.lordba_linear_i4_backward(g, binding.lordba_layout_i4(*dev, 64, transposed=True))
    i8_checks.near(dx, *i4_checks.product(torch, g.double(), W.t().contiguous()))


@pytest.mark.parametrize("T", [2, 20, 90])
@pytest.mark.parametrize("d_in", [256, 200, 201])
def test_rows_that_hold_no_numbers_spoil_no_others(torch, T, d_in):
    rng = np.random.default_rng(T)
    codes, scale, zero = i4_checks.weights(torch, rng, 70, d_in, 64, True)
    scale = scale.abs() + 0.001
    codes[codes == zero[:, torch.arange(d_in) // 64]] += 1      # (no weight is 0; a code of 16 counts as 0)
    codes %= 16
    zero[zero == codes[:, ::64]] = 0
    codes[:, -1] = 9
    zero[:, -1] = 3
    x, g = acts(torch, rng, T, d_in), acts(torch, rng, T, 70)
    L, Lt = (binding.lordba_layout_i4(codes.cuda(), scale.cuda(), zero.cuda(), 64, transposed=t) for t in (False, True))
    y, dx = binding.lordba_linear_i4(x, L), binding.lordba_linear_i4_backward(g, Lt)
    x2, g2 = x.clone(), g.clone()
    x2[1, -1], g2[1, 3] = float("inf"), float("nan")
    y2, dx2 = binding.lordba_linear_i4(x2, L), binding.lordba_linear_i4_backward(g2, Lt)
    others = torch.arange(T, device="cuda") != 1
    assert torch.equal(y2[others], y[others]) and torch.equal(dx2[others], dx[others])
    assert bool((y2[1] == float("inf")).all())       # weight 6 times a positive scale there; padding adds nothing
    assert bool(torch.isnan(dx2[1]).all())


@pytest.mark.parametrize("T", [2, 100])
@pytest.mark.parametrize("d_in", [200, 201])
def test_padding_behind_large_scales(torch, T, d_in):
    # weights of 0 under scales whose other multiples pass the range of fp16: nothing behind a row's end comes into its sums
    codes = torch.full((40, d_in), 3, dtype=torch.uint8, device="cuda")
    scale = torch.full((40, -(-d_in // 128)), 60000.0, dtype=torch.float16, device="cuda")
    zero = torch.full(scale.shape, 3, dtype=torch.uint8, device="cuda")
    x = torch.randn(T, d_in, device="cuda").half()
    y = binding.lordba_linear_i4(x, binding.lordba_layout_i4(codes, scale, zero))
    assert bool((y == 0).all())


def test_a_tuple_will_do(torch):
    codes, scale, zero = binding.lordba_quantize_i4(torch.randn(64, 96, device="cuda").half(), 32, True)
    W, x = binding.lordba_layout_i4(codes, scale, zero, 32), torch.randn(5, 96, device="cuda").half()
    y = binding.lordba_linear_i4(x, W)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for W2, stream in ((tuple(W), None), (tuple(W), side)):
        y2 = binding.lordba_linear_i4(x, W2, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(y2, y)


def test_more_workgroups_than_one_launch_takes(torch):
    # and results behind the first 2^32 bytes
    T, d_in, d_out = 300001, 5, 8192
    rng = np.random.default_rng(4)
    codes, scale, zero = i4_checks.weights(torch, rng, d_out, d_in, 32, True)
    W = i4_checks.real(torch, codes, scale, zero, 32, rounded=False).cuda()
    x = torch.randn(T, d_in, device="cuda", generator=torch.Generator("cuda").manual_seed(4)).half()
    y = binding.lordba_linear_i4(x, binding.lordba_layout_i4(codes.cuda(), scale.cuda(), zero.cuda(), 32))
    for t in range(0, T, 10000):
        i8_checks.near(y[t:t + 10000], *i4_checks.product(torch, x[t:t + 10000].double(), W))


@pytest.mark.parametrize("T,k,n", [(40, 1 << 22, 24), (40, (1 << 22) + 8, 24), (3, (1 << 22) + 1, 24)])
@pytest.mark.parametrize("backward", [False, True])
def test_long_contractions(torch, T, k, n, backward):
    rng = np.random.default_rng(k + T)
    codes, scale, zero = i4_checks.weights(torch, rng, *((k, n) if backward else (n, k)), 128, True)
    W = i4_checks.real(torch, codes, scale, zero, 128, rounded=backward or i4_checks.kernel(T, k, n) != "few").cuda()
    x = torch.randn(T, k, device="cuda", generator=torch.Generator("cuda").manual_seed(T)).half()
    laid = binding.lordba_layout_i4(codes.cuda(), scale.cuda(), zero.cuda(), transposed=backward)
    y = binding.lordba_linear_i4_backward(x, laid) if backward else binding.lordba_linear_i4(x, laid)
    i8_checks.near(y, *i4_checks.product(torch, x.double(), W.t().contiguous() if backward else W))


def test_the_low_four_bits_count(torch):
    codes, scale, zero = binding.lordba_quantize_i4(torch.randn(64, 200, device="cuda").half(), 64, True)
    for transposed in (False, True):
        a = binding.lordba_layout_i4(codes, scale, zero, 64, transposed=transposed)
        b = binding.lordba_layout_i4(codes ^ 0xf0, scale, zero ^ 0xf0, 64, transposed=transposed)
        assert torch.equal(a.codes, b.codes) and torch.equal(a.scale, b.scale) and torch.equal(a.zero, b.zero)


def test_no_tokens(torch):
    codes, scale, _ = binding.lordba_quantize_i4(torch.randn(64, 96, device="cuda").half(), 32)
    x, g = torch.empty(0, 96, dtype=torch.float16, device="cuda"), torch.empty(0, 64, dtype=torch.float16, device="cuda")
    assert binding.lordba_linear_i4(x, binding.lordba_layout_i4(codes, scale, group=32)).shape == (0, 64)
    assert binding.lordba_linear_i4_backward(g, binding.lordba_layout_i4(codes, scale, group=32, transposed=True)).shape == (0, 96)
    h, kept = binding.lordba_gated_i4(x, binding.lordba_layout_i4(codes, scale, group=32, halves=2), save=True)
    dx, dgu = binding.lordba_gated_i4_backward(h, kept, binding.lordba_layout_i4(codes, scale, group=32, halves=2, transposed=True))
    assert h.shape == (0, 32) and kept.shape == dgu.shape == (2, 0, 32) and dx.shape == (0, 96)


@pytest.mark.parametrize("zero_points", [False, True])
@pytest.mark.parametrize("group,rows,cols", [(32, 5, 33), (64, 70, 200), (128, 33, 1000), (128, 4, 9), (128, 1, 1)])
def test_quantiser(torch, group, rows, cols, zero_points):
    rng = np.random.default_rng(cols)
    w = rng.standard_normal((rows, cols)).astype(np.float16)
    w[0, :] = 0
    if rows > 2:
        w[1] = np.abs(w[1]) + 1     # one sign only
        w[2] *= np.float16(1e-6)    # subnormal scales
    codes, scale, zero = binding.lordba_quantize_i4(torch.from_numpy(w).cuda(), group, zero_points)
    # the definition in fp32, group by group (rows of whole groups, padded with what changes nothing)
    groups = -(-cols // group)
    v = np.zeros((rows, groups * group), np.float32)
    v[:, :cols] = w
    v = v.reshape(rows, groups, group)
    low, high = v.min(axis=2), v.max(axis=2)      # (a padded 0 is in the range by definition)
    low, high = np.minimum(low, 0), np.maximum(high, 0)
    s = ((high - low) / np.float32(15) if zero_points else np.maximum(high, -low) / np.float32(7)).astype(np.float16)
    f = s.astype(np.float32)
    flat = f == 0
    f1 = np.where(flat, np.float32(1), f)
    z = np.where(flat, 0, np.minimum(np.rint(-low / f1), 15)) if zero_points else np.full(s.shape, 8)
    q = np.where(flat[..., None], z[..., None], np.clip(np.rint((v / f1[..., None]).astype(np.float32) + z[..., None].astype(np.float32)), 0, 15))
    assert np.array_equal(scale.cpu().numpy(), s)     # (as numbers: the sign of a 0 is nothing)
    assert np.array_equal(codes.cpu().numpy(), q.reshape(rows, -1)[:, :cols].astype(np.uint8))
    assert (zero is None) is not zero_points and (zero is None or np.array_equal(zero.cpu().numpy(), z.astype(np.uint8)))
    # a weight is off by half a step, and by what the ends of the range lose to the scale's rounding (2^-11 of 8 or 15 steps, or a subnormal's half step)
    if zero_points:
        back = f[..., None] * (q - z[..., None])
        # (zero and code are rounded apart: half a step each)
        assert (np.abs(back - v) <= 1.02 * f[..., None] + np.float32(2.0 ** -25) * 15).all()


def test_a_group_without_numbers(torch):
    w = torch.randn(3, 96, device="cuda").half()
    w[1, 40] = float("nan")
    w[2, 0] = float("inf")
    for zero_points in (False, True):
        _, scale, _ = binding.lordba_quantize_i4(w, 32, zero_points)
        assert torch.isnan(scale).cpu().tolist() == [[False] * 3, [False, True, False], [True, False, False]]


@pytest.mark.parametrize("T", [1, 48, 300])
def test_streams_and_graphs(torch, T):
    gen = torch.Generator(device="cuda").manual_seed(3)
    half = lambda *s: torch.randn(s, generator=gen, device="cuda").half()
    F, d = 160, 200
    codes, scale, zero = binding.lordba_quantize_i4(half(2 * F, d) / 14, 32, True)
    L, Lt = (binding.lordba_layout_i4(codes, scale, zero, 32, halves=2, transposed=t) for t in (False, True))
    M, Mt = (binding.lordba_layout_i4(codes, scale, zero, 32, transposed=t) for t in (False, True))
    x, dh, g = half(T, d), half(T, F), half(T, 2 * F)

    def calls():
        h, kept = binding.lordba_gated_i4(x, L, save=True)
        return [h, kept, *binding.lordba_gated_i4_backward(dh, kept, Lt), binding.lordba_linear_i4(x, M), binding.lordba_linear_i4_backward(g, Mt)]

    want = [t.clone() for t in calls()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    h, kept = binding.lordba_gated_i4(x, L, save=True, stream=side)
    got = [h, kept, *binding.lordba_gated_i4_backward(dh, kept, Lt, stream=side), binding.lordba_linear_i4(x, M, stream=side.cuda_stream),
           binding.lordba_linear_i4_backward(g, Mt, stream=side)]
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = calls()
    for k in range(4):      # other inputs in the same memory, eager work in between
        for t in (x, dh, g):
            t.copy_(half(*t.shape))
        graph.replay()
        torch.cuda.synchronize()
        again = calls()
        assert all(torch.equal(a, b) for a, b in zip(out, again)), k


@pytest.mark.parametrize("T", [7, 100])
def test_the_gradient_is_the_adjoint(torch, T):
    # <g, x W^T> = <g W, x>, up to the roundings of y and dx to fp16 and of the weights
    rng = np.random.default_rng(8)
    codes, scale, zero = (t.cuda() for t in i4_checks.weights(torch, rng, 300, 260, 32, True))
    x, g = acts(torch, rng, T, 260), acts(torch, rng, T, 300)
    y = binding.lordba_linear_i4(x, binding.lordba_layout_i4(codes, scale, zero, 32)).double()
    dx = binding.lordba_linear_i4_backward(g, binding.lordba_layout_i4(codes, scale, zero, 32, transposed=True)).double()
    W = i4_checks.real(torch, codes.cpu(), scale.cpu(), zero.cpu(), 32, False).cuda()
    size = float((g.double().abs() @ (x.double().abs() @ W.abs().t().contiguous()).t().contiguous()).diagonal().sum())
    assert abs(float((g.double() * y).sum() - (dx * x.double()).sum())) <= 4 * 2.0 ** -11 * size


def test_plain_and_other_ways_agree(torch, monkeypatch):
    gen = torch.Generator(device="cuda").manual_seed(4)
    half = lambda *s: torch.randn(s, generator=gen, device="cuda").half()
    T, d, F = 9, 70, 34
    codes, scale, zero = binding.lordba_quantize_i4(half(2 * F, d), 32, True)
    L, Lt = (binding.lordba_layout_i4(codes, scale, zero, 32, halves=2, transposed=t) for t in (False, True))
    M, Mt = (binding.lordba_layout_i4(codes, scale, None, 32, transposed=t) for t in (False, True))
    x, dh, g, kept, add = half(T, d), half(T, F), half(T, 2 * F), half(2, T, F), half(2, T, F)
    calls = [lambda: binding.lordba_linear_i4(x, M), lambda: binding.lordba_linear_i4(x, M, y_out=torch.empty_like(g)), lambda: binding.lordba_linear_i4_backward(g, Mt),
             lambda: binding.lordba_gated_i4(x, L), lambda: binding.lordba_gated_i4(x, L, addends=add, save=True),
             lambda: binding.lordba_gated_i4_backward(dh, kept, Lt)]
    taken, both = [], []
    real = binding._plain_call
    for plain in (True, False):
        monkeypatch.setattr(binding, "_plain_call", lambda *a: (lambda r: (taken.append(r is not None), r)[1])(real(*a)) if plain else None)
        both.append([c() for c in calls])
    assert taken == [True] * len(calls)
    flat = lambda v: [t for r in v for t in (r if isinstance(r, tuple) else (r,))]
    assert all(torch.equal(a, b) for a, b in zip(flat(both[0]), flat(both[1])))
    # refused the same way both ways: other types, shapes, layouts
    bad = [lambda: binding.lordba_linear_i4(x.float(), M), lambda: binding.lordba_linear_i4(x[:, :-1].contiguous(), M), lambda: binding.lordba_linear_i4(x, Mt),
           lambda: binding.lordba_linear_i4(x, L), lambda: binding.lordba_linear_i4(x.t(), M), lambda: binding.lordba_linear_i4(x, M, y_out=x),
           lambda: binding.lordba_linear_i4(x, M._replace(cols=71)), lambda: binding.lordba_linear_i4(x, M._replace(codes=M.codes[:-16])),
           lambda: binding.lordba_linear_i4(x, M._replace(group=64)), lambda: binding.lordba_linear_i4(x, tuple(M)[:-1]), lambda: binding.lordba_linear_i4_backward(g, M),
           lambda: binding.lordba_gated_i4(x, M), lambda: binding.lordba_gated_i4(x, L, addends=add[0]), lambda: binding.lordba_gated_i4(x, L, addends=add.float()),
           lambda: binding.lordba_gated_i4_backward(dh, kept[0], Lt), lambda: binding.lordba_gated_i4_backward(dh[:, 1:].contiguous(), kept, Lt)]
    for k, call in enumerate(bad):
        for plain in (True, False):
            monkeypatch.setattr(binding, "_plain_call", real if plain else lambda *a: None)
            with pytest.raises((TypeError, ValueError)):
                call()
