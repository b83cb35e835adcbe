"""The calls around the branch through the C interface on tensors with guarded surroundings: results that are numbers and near 64 bits, nothing
read from outside (NaN lies there), nothing written outside (checked), inputs as they were."""
import numpy as np
import pytest

import i8_checks as c
from i8_checks import call, near
from test_gpu_i8_parity import GATED, REGIMES, SHAPES


def test_what_near_refuses():
    one, none = np.ones((2, 3)), np.zeros((2, 3))
    good = one.astype(np.float16)
    near(good, one, none)
    past = np.full((2, 3), -1e5)
    near(np.full((2, 3), -np.inf, np.float16), past, none)
    near(np.full((2, 3), -65504, np.float16), np.full((2, 3), -65510.0), none)
    bad = good.copy()
    for v in (np.nan, np.inf, -np.inf, 1.002, 0):
        bad[1, 2] = v
        with pytest.raises(AssertionError):
            near(bad, one, none)
    for want, err in ((np.full((2, 3), np.nan), none), (np.full((2, 3), np.inf), none), (one, np.full((2, 3), np.nan))):
        with pytest.raises(AssertionError):
            near(good, want, err)
    with pytest.raises(AssertionError):
        near(np.full((2, 3), np.inf, np.float16), past, none)
    with pytest.raises(AssertionError):
        near(np.full((2, 3), -65504, np.float16), past, none)


def test_what_memory_refuses():
    import torch

    def fresh():
        mem = c.Memory(torch, "cpu")
        x = mem.input(np.arange(5, dtype=np.float16), 3)
        s, w = mem.input(np.ones((2, 3), np.float32), 1), mem.input(np.ones(7, np.int8), 16)
        y = mem.output((3, 5), torch.float16, 1)
        for t, item, lead in ((x, 2, 3), (s, 4, 1), (w, 1, 16), (y, 2, 1)):
            assert (t.data_ptr() - lead * item) % 64 == 0 and t.is_contiguous()
        for (big, _, _), t in ((mem.kept[0], x), (mem.kept[1], s)):     # what follows and precedes an input are NaN of its type
            at, n = t.data_ptr() - big.data_ptr(), t.numel() * t.element_size()
            assert big[at + n:at + n + 64].view(t.dtype).isnan().all() and big[at - 64:at].view(t.dtype).isnan().all()
        y.fill_(7)
        mem.unchanged()
        return mem, x, y

    for entry, where in ((0, -1), (0, 0), (3, -1), (3, 3 * 5 * 2)):     # in front of the input, in it, in front of the output, behind it
        mem, x, y = fresh()
        big = mem.kept[entry][0]
        big[(x if entry == 0 else y).data_ptr() - big.data_ptr() + where] ^= 1
        with pytest.raises(AssertionError):
            mem.unchanged()


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    c.binding.load_library()
    return torch


def ids(s):
    return "T%d_%dx%d" % s


SHIFTS = (0, 1)     # elements behind 64 aligned bytes; matrices of int8 16 of them


@pytest.mark.gpu
@pytest.mark.parametrize("digits", [1, 2])
@pytest.mark.parametrize("shape", SHAPES + REGIMES, ids=ids)
def test_linear(torch, shape, digits):
    check_linear(torch, *shape, digits)


def check_linear(torch, T, d_in, d_out, digits, shifts=SHIFTS):
    rng = np.random.default_rng(T + 7 * d_in + 13 * d_out)
    W, ws = c.weights(rng, d_out, d_in)
    x = c.acts(rng, T, d_in)
    w = torch.from_numpy(W).cuda()
    want, err = c.product(torch, *c.rows_of(x, None, digits), w, ws)
    for shift in shifts:
        mem = c.Memory(torch)
        y = mem.output((T, d_out), torch.float16, shift)
        space = c.workspace(mem, T, d_in, digits)
        call(torch, "lordba_linear_i8", mem.input(x, shift), mem.input(c.binding.lordba_layout_i8(w), 16 * shift), mem.input(ws, shift), y, space, space.numel(),
             T, d_in, d_out, digits)
        mem.unchanged()
        near(y, want, err)


@pytest.mark.gpu
@pytest.mark.parametrize("digits", [1, 2])
@pytest.mark.parametrize("shape", SHAPES + [s for s in REGIMES if s[1] <= 14000], ids=ids)
def test_linear_backward(torch, shape, digits):
    check_linear_backward(torch, *shape, digits)


def check_linear_backward(torch, T, d_in, d_out, digits, shifts=SHIFTS):
    rng = np.random.default_rng(T + 5 * d_in + 11 * d_out)
    W, ws = c.weights(rng, d_out, d_in)
    g = c.acts(rng, T, d_out)
    w = torch.from_numpy(W).cuda()
    want, err = c.product(torch, *c.rows_of(g, ws, digits), w.t().contiguous(), np.ones(d_in, np.float32))
    for shift in shifts:
        mem = c.Memory(torch)
        dx = mem.output((T, d_in), torch.float16, shift)
        space = c.workspace(mem, T, d_out, digits)
        call(torch, "lordba_linear_i8_backward", mem.input(g, shift), mem.input(c.binding.lordba_layout_i8(w, True), 16 * shift), mem.input(ws, shift), dx, space,
             space.numel(), T, d_in, d_out, digits)
        mem.unchanged()
        near(dx, want, err)


@pytest.mark.gpu
@pytest.mark.parametrize("digits", [1, 2])
@pytest.mark.parametrize("shape", GATED, ids=ids)
def test_gated(torch, shape, digits):
    check_gated(torch, *shape, digits)


def check_gated(torch, T, d_in, F, digits, shifts=SHIFTS, ways=((True, True), (False, True), (True, False), (False, False))):
    """ways: (with addends, kept) of the calls; a shift of its own for the outputs where it is a pair"""
    rng = np.random.default_rng(T + 17 * d_in + 3 * F)
    W, ws = c.weights(rng, 2 * F, d_in)
    ws = (ws * 2).astype(np.float32)
    x, addends = c.acts(rng, T, d_in), c.acts(rng, 2 * T, F).reshape(2, T, F)
    w = torch.from_numpy(W).cuda()
    q, s = c.rows_of(x, None, digits)
    for add in {a: None for a, _ in ways}:
        gate, up, h, eg, eu, eh = c.gated(torch, q, s, w, ws, addends if add else None)
        for keep in [k for a, k in ways if a == add]:
            for shift in shifts:
                mem = c.Memory(torch)
                shift, out = shift if isinstance(shift, tuple) else (shift, shift)
                got = mem.output((T, F), torch.float16, out)
                kept = mem.output((2, T, F), torch.float16, out) if keep else None
                space = c.workspace(mem, T, d_in, digits)
                call(torch, "lordba_gated_i8", mem.input(x, shift), mem.input(c.binding.lordba_layout_i8(w), 16 * shift), mem.input(ws, shift),
                     mem.input(addends, shift) if add else None, got, kept, space, space.numel(), T, d_in, F, digits)
                mem.unchanged()
                near(got, h, eh)
                if keep:
                    near(kept[0], gate, eg)
                    near(kept[1], up, eu)


GATED_BACKWARD = GATED + [(2, 40, 2049), (2, 33, 4097), (2, 20, 8200), (2, 17, 16390), (4, 83, 12871), (70, 30, 3000), (1100, 2100, 130), (512, 40, 7), (600, 33, 515)]


@pytest.mark.gpu
@pytest.mark.parametrize("digits", [1, 2])
@pytest.mark.parametrize("shape", GATED_BACKWARD, ids=ids)
def test_gated_backward(torch, shape, digits):
    check_gated_backward(torch, *shape, digits)


def check_gated_backward(torch, T, d_in, F, digits, shifts=SHIFTS):
    rng = np.random.default_rng(T + 19 * d_in + 7 * F)
    W, ws = c.weights(rng, 2 * F, d_in)
    dh, gate_up = c.acts(rng, T, F), (c.acts(rng, 2 * T, F) * np.float16(2)).reshape(2, T, F)
    gate_up[0, 0, 0], gate_up[0, -1, -1] = -60000, 200     # (the exponential of the first overflows)
    w = torch.from_numpy(W).cuda()
    dg, du, eg, eu = c.gated_gradient(torch, dh, gate_up)
    both, err = torch.cat([dg, du], dim=1), torch.cat([eg, eu], dim=1)
    want, ex = c.row_error(torch, both, err, ws, w.t().contiguous(), digits)
    for shift in shifts:
        mem = c.Memory(torch)
        dx, dgu = mem.output((T, d_in), torch.float16, shift), mem.output((2, T, F), torch.float16, shift)
        space = c.workspace(mem, T, 2 * F, digits)
        call(torch, "lordba_gated_i8_backward", mem.input(dh, shift), mem.input(gate_up, shift), mem.input(c.binding.lordba_layout_i8(w, True), 16 * shift),
             mem.input(ws, shift), dx, dgu, space, space.numel(), T, d_in, F, digits)
        mem.unchanged()
        near(dgu[0], dg, eg)
        near(dgu[1], du, eu)
        near(dx, want, ex)


@pytest.mark.gpu
@pytest.mark.parametrize("digits", [1, 2])
@pytest.mark.parametrize("scaled", [False, True])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (4, 64), (5, 511), (9, 512), (2, 513), (7, 1023), (1030, 1025), (1100, 2047), (3, 2049), (2, 4097), (2, 8193), (2, 16385), (2, 33000)])
def test_rows(torch, rows, cols, scaled, digits):
    rng = np.random.default_rng(rows * 1000003 + cols)
    x = c.acts(rng, rows, cols)
    cs = rng.uniform(0.01, 3.0, size=cols).astype(np.float32) if scaled else None
    want, scales = c.rows_of(x, cs, digits)
    for shift in (0, 3):
        mem = c.Memory(torch)
        q, s = mem.output((digits, rows, c.binding.lordba_i8_row_bytes(cols)), torch.int8, 16 * shift), mem.output((rows,), torch.float32, shift)
        call(torch, "lordba_quantize_rows", mem.input(x, shift), None if cs is None else mem.input(cs, shift), q, s, rows, cols, digits)
        mem.unchanged()
        assert np.array_equal(s.cpu().numpy(), scales)
        for k in range(digits):     # the definition's own operations: the same integers, zeros behind the columns
            assert np.array_equal(q[k, :, :cols].cpu().numpy(), want[k]) and not q[k, :, cols:].any()


@pytest.mark.gpu
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("rows,cols", [(1, 1), (5, 3), (64, 64), (65, 129), (130, 1000), (300, 77), (1, 1025), (2051, 3)])
def test_layouts(torch, rows, cols, transposed):
    rng = np.random.default_rng(rows + cols)
    W = rng.integers(-128, 128, size=(rows, cols), dtype=np.int8)
    want = W.T if transposed else W
    for shift in (0, 5):
        mem = c.Memory(torch)
        out = mem.output((want.shape[0], c.binding.lordba_i8_row_bytes(want.shape[1])), torch.int8, 16 * shift)
        call(torch, "lordba_layout_i8", mem.input(W, shift), out, rows, cols, int(transposed))
        mem.unchanged()
        got = out.cpu().numpy()
        assert np.array_equal(got[:, :want.shape[1]], want) and not got[:, want.shape[1]:].any()


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 7, 8, 9, 255, 2047, 2048, 2049, 100003])
@pytest.mark.parametrize("base", [False, True])
def test_dropout(torch, n, base):
    from test_gpu_dropout import kept

    rng = np.random.default_rng(n)
    x, b = rng.standard_normal(n).astype(np.float16), rng.standard_normal(n).astype(np.float16)
    keep, factor = kept(n, 0.3, 5, 1 << 40)
    part = np.where(keep, x.astype(np.float64) * factor, 0)
    want = part + b.astype(np.float64) * base
    for shift in (0, 1, 2, 5):
        mem = c.Memory(torch)
        y = mem.output((n,), torch.float16, shift)
        call(torch, "lordba_dropout", mem.input(x, 2 * shift), mem.input(b, 3 * shift) if base else None, y, n, 0.3, 5, 1 << 40, None)
        mem.unchanged()
        near(y.cpu().numpy(), want, (np.abs(part) + np.abs(want)) * 2.0 ** -22)   # (the factor, the product and the sum in fp32)
