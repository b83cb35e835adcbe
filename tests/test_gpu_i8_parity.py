"""GPU parity of the 8-bit projections, the gated block and its backward pass against 64-bit arithmetic.

Bounds.  Integer sums are exact, so given the rows' integers q and scales s, y = s w sum(q W) is off by the conversions to fp32 (2^-24 of
what is converted), three fp32 operations and one rounding to fp16: 2^-11 of the value (2^-25 among the subnormals), and F32 = 2^-21 of
256 |sum hi| + |sum lo| for the rest, with a factor of two to spare.  A row in D = 127 or 32512 steps is off by half a step per entry and by
the two fp32 roundings of v * (D / amax), D * 2^-23 steps."""
import numpy as np
import pytest

from paper_2605_24058_amd import binding

pytestmark = pytest.mark.gpu

F32, F16, SUB = 2.0 ** -21, 2.0 ** -11, 2.0 ** -25
DEPTH = {1: 127, 2: 32512}

# (T, d_in, d_out): one row, block edges of 16 / 64 / 128 / 256 tokens and columns on both sides, one column, widths that no vector divides
SHAPES = [(1, 1, 1), (1, 4096, 64), (2, 7, 5), (5, 130, 127), (8, 512, 512), (15, 64, 66), (16, 63, 65), (17, 129, 130), (31, 1000, 33), (33, 257, 1),
          (64, 384, 200), (65, 128, 257), (100, 999, 301), (127, 1025, 128), (129, 640, 129), (255, 96, 511), (257, 2047, 96), (300, 64, 1030),
          (513, 320, 260), (1, 11008, 129), (3, 13824, 40), (700, 200, 700)]


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    binding.load_library()
    return torch


def weights(rng, n, k, full=False):
    """int8 [n, k] and fp32 scales [n]; full: every value from -128 on"""
    W = rng.integers(-128 if full else -127, 128, size=(n, k), dtype=np.int64).astype(np.int8)
    return W, (rng.uniform(0.2, 2.0, size=n) / (70 * np.sqrt(k))).astype(np.float32)


def acts(rng, rows, cols, zero_rows=True):
    x = rng.standard_normal((rows, cols)).astype(np.float32)
    x[:, ::37] *= 8
    if zero_rows and rows > 4:
        x[rows // 2] = 0
    return x.astype(np.float16)


def place(torch, a, shift):
    """`a` on the GPU, its first element `shift` elements behind a 16-byte boundary, NaN around it."""
    t = torch.from_numpy(np.ascontiguousarray(a))
    big = torch.full((t.numel() + 64,), float("nan"), dtype=t.dtype, device="cuda:0")
    v = big[16 + shift:16 + shift + t.numel()].view(t.shape)
    v.copy_(t)
    return v


def host(t):
    return t.cpu().numpy()


def integers(torch, x, col_scale, digits):
    """The rows as the library holds them: (integer parts [digits] as int64 [rows, cols], scale as float64)."""
    q, s = binding.lordba_quantize_rows(x, col_scale, digits)
    cols = x.shape[1]
    q = host(q).astype(np.int64).reshape(digits, x.shape[0], -1)
    assert not q[:, :, cols:].any()   # what lies behind the columns is zero
    return q[:, :, :cols], host(s).astype(np.float64)


def sums(q, W):
    """sum q W^T of each digit, exact (float64 holds them: below 2^53)"""
    return [p.astype(np.float64) @ W.astype(np.float64).T for p in q]


def product(q, s, W, w_scale):
    """y and the bound of its error before the rounding to fp16"""
    parts = sums(q, W)
    value = parts[0] if len(parts) == 1 else 256 * parts[0] + parts[1]
    size = np.abs(parts[0]) if len(parts) == 1 else 256 * np.abs(parts[0]) + np.abs(parts[1])
    f = s[:, None] * w_scale[None, :].astype(np.float64)
    return value * f, size * f * F32


def near(got, want, err):
    """got: fp16 of a value within err of want"""
    off = np.abs(got.astype(np.float64) - want)
    limit = np.abs(want) * F16 + err * 1.01 + SUB
    bad = off > limit
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:3].tolist(), float((off / limit).max()))


@pytest.mark.parametrize("digits", [1, 2])
@pytest.mark.parametrize("scaled", [False, True])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (4, 64), (5, 511), (9, 512), (2, 513), (7, 1023), (6, 1024), (3, 2049), (2, 4096), (3, 4097), (2, 8193),
                                       (2, 16385), (2, 33000), (1, 131071)])
def test_rows(torch, rows, cols, scaled, digits):
    rng = np.random.default_rng(rows * 1000003 + cols)
    x = acts(rng, rows, cols)
    cs = rng.uniform(0.01, 3.0, size=cols).astype(np.float32) if scaled else None
    for shift in (0, 3):
        xd = place(torch, x, shift)
        q, s = integers(torch, xd, None if cs is None else place(torch, cs, shift), digits)
        v = x.astype(np.float64) * (1.0 if cs is None else cs.astype(np.float64))
        amax, D = np.abs(v).max(axis=1), DEPTH[digits]
        assert np.all(np.abs(s - amax / D) <= amax / D * 2.0 ** -22)
        if digits == 2:
            assert np.abs(q[0]).max() <= 127
        whole = q[0] if digits == 1 else 256 * q[0] + q[1]
        assert np.abs(whole).max() <= D
        step = np.where(amax > 0, amax / D, 1.0)[:, None]
        assert np.all(np.abs(whole - v / step) <= 0.5 + D * 2.0 ** -21)   # (with a column scale: one rounding more)


def test_rows_without_numbers_and_the_smallest(torch):
    x = np.ones((6, 300), dtype=np.float16)
    x[1, 7] = np.inf
    x[2, 299] = np.nan
    x[3] = 0
    x[4] = np.float16(6e-8)      # the smallest subnormal
    x[5, 1:] = 65504
    for digits in (1, 2):
        q, s = integers(torch, place(torch, x, 1), None, digits)
        assert np.isnan(s[[1, 2]]).all() and np.isfinite(s[[0, 3, 4, 5]]).all()
        assert not q[:, 1:4].any() and s[3] == 0
        whole = q[0] if digits == 1 else 256 * q[0] + q[1]
        assert (whole[4] == DEPTH[digits]).all() and (whole[5, 1:] == DEPTH[digits]).all()
    cs = torch.full((300,), 1e-38, device="cuda:0")
    q, s = binding.lordba_quantize_rows(place(torch, np.ones((2, 300), np.float16), 0), cs)
    assert not q.any() and not s.any()   # below 2^-100 a row counts as zeros


@pytest.mark.parametrize("rows,cols", [(1, 1), (5, 3), (64, 64), (65, 129), (130, 1000), (300, 77)])
def test_layouts(torch, rows, cols):
    rng = np.random.default_rng(rows + cols)
    W = rng.integers(-128, 128, size=(rows, cols), dtype=np.int64).astype(np.int8)
    w = torch.from_numpy(W).cuda()
    for transposed, want in ((False, W), (True, W.T)):
        out = host(binding.lordba_layout_i8(w, transposed))
        assert out.shape == (want.shape[0], binding.lordba_i8_row_bytes(want.shape[1]))
        assert np.array_equal(out[:, :want.shape[1]], want) and not out[:, want.shape[1]:].any()


@pytest.mark.parametrize("digits", [1, 2])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "T%d_%dx%d" % s)
def test_linear(torch, shape, digits):
    T, d_in, d_out = shape
    rng = np.random.default_rng(T + 7 * d_in + 13 * d_out)
    W, ws = weights(rng, d_out, d_in, full=True)
    Wl = binding.lordba_layout_i8(torch.from_numpy(W).cuda())
    x = acts(rng, T, d_in)
    for shift in (0, 1):
        xd, sd = place(torch, x, shift), place(torch, ws, shift)
        y = host(binding.lordba_linear_i8(xd, Wl, sd, digits=digits, y_out=place(torch, np.zeros((T, d_out), np.float16), shift)))
        near(y, *product(*integers(torch, xd, None, digits), W, ws))
    # against x itself: half a step of the row per entry
    if digits == 2:
        want = x.astype(np.float64) @ (W * ws[:, None].astype(np.float64)).T
        half = 0.51 * np.abs(x).max(axis=1).astype(np.float64) / DEPTH[2]
        near(y, want, half[:, None] * (np.abs(W).sum(axis=1) * ws.astype(np.float64))[None, :] + F32 * np.abs(want) * 4)


@pytest.mark.parametrize("digits", [1, 2])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "T%d_%dx%d" % s)
def test_linear_backward(torch, shape, digits):
    T, d_in, d_out = shape
    rng = np.random.default_rng(T + 5 * d_in + 11 * d_out)
    W, ws = weights(rng, d_out, d_in)
    Wt = binding.lordba_layout_i8(torch.from_numpy(W).cuda(), transposed=True)
    g = place(torch, acts(rng, T, d_out), 1)
    sd = torch.from_numpy(ws).cuda()
    dx = host(binding.lordba_linear_i8_backward(g, Wt, sd, digits=digits))
    near(dx, *product(*integers(torch, g, sd, digits), W.T, np.ones(d_in, np.float32)))
    if digits == 2:   # the formula
        gw = host(g).astype(np.float64) * ws
        half = 0.51 * np.abs(gw).max(axis=1) / DEPTH[2]
        near(dx, gw @ W.astype(np.float64), half[:, None] * np.abs(W.astype(np.float64)).sum(axis=0)[None, :] + 4 * F32 * np.abs(gw) @ np.abs(W))
        assert np.array_equal(dx, host(binding.lordba_linear_i8_backward(g, Wt, sd)))   # (the default)


# Every tile and way of working: 256 x 256 (whole, ragged, odd widths), 256 x 128, 128 x 128, 64 x 64 and below, steps shared by several workgroups (few rows
# or columns, long contractions), and a few tokens whose rows the product's workgroups make (multiples of 8 columns, 16-byte aligned)
REGIMES = [(2100, 300, 4200), (2048, 520, 4095), (1030, 260, 4100), (512, 700, 4096), (600, 250, 1111), (40, 5000, 70), (3, 9000, 40), (16, 131071, 3), (20, 3000, 33),
           (130, 2100, 20), (1, 4096, 515), (2, 6000, 100), (7, 1024, 64), (1, 13824, 33), (3, 4104, 37), (16, 64, 8), (16, 880, 31), (158, 34321, 771),
           (237, 37461, 34), (113, 27294, 500), (165, 14105, 68), (64, 13824, 2100), (128, 2600, 4096), (60, 2000, 3500),
           (1, 4095, 300), (2, 2047, 65), (1, 9, 40), (2, 1, 33)]


@pytest.mark.parametrize("digits", [1, 2])
@pytest.mark.parametrize("shape", REGIMES, ids=lambda s: "T%d_%dx%d" % s)
def test_linear_regimes(torch, shape, digits):
    T, d_in, d_out = shape
    rng = np.random.default_rng(T + 23 * d_in + 29 * d_out)
    W, ws = weights(rng, d_out, d_in)
    Wl = binding.lordba_layout_i8(torch.from_numpy(W).cuda())
    x, sd = torch.from_numpy(acts(rng, T, d_in)).cuda(), torch.from_numpy(ws).cuda()
    y = binding.lordba_linear_i8(x, Wl, sd, digits=digits)
    near(host(y), *product(*integers(torch, x, None, digits), W, ws))
    for _ in range(2):   # the same again, in a workspace that holds anything
        junk = torch.full((binding.lordba_i8_workspace_bytes(T, d_in, digits),), 0xA5, dtype=torch.uint8, device="cuda")
        assert torch.equal(binding.lordba_linear_i8(x, Wl, sd, digits=digits, workspace=junk), y)


@pytest.mark.parametrize("shape", [(2053, 320, 4096), (2048, 256, 4090), (1024, 300, 3001), (512, 260, 2048), (4, 6000, 30), (20, 3000, 17), (1, 4096, 100), (3, 2048, 50),
                                   (1, 6144, 9), (267, 20889, 85), (17, 14034, 400), (114, 9500, 282), (700, 500, 640),
                                   (1, 2047, 70), (2, 1001, 33)], ids=lambda s: "T%d_%dx%d" % s)
def test_gated_regimes(torch, shape):
    T, d_in, F = shape
    rng = np.random.default_rng(T + 31 * d_in + 37 * F)
    W, ws = weights(rng, 2 * F, d_in)
    Wl, sd = binding.lordba_layout_i8(torch.from_numpy(W).cuda()), torch.from_numpy(ws).cuda()
    x, add = torch.from_numpy(acts(rng, T, d_in)).cuda(), acts(rng, 2 * T, F, zero_rows=False).reshape(2, T, F)
    ad = torch.from_numpy(add).cuda()
    h, kept = binding.lordba_gated_i8(x, Wl, sd, addends=ad, save=True)
    gate, up, want, eg, eu = gated(*integers(torch, x, None, 1), W, ws, add, F)
    near(host(kept)[0], gate, eg)
    near(host(kept)[1], up, eu)
    silu = np.abs(gate) / (1 + np.exp(-gate))
    near(host(h), want, 1.1 * np.abs(up) * eg + silu * eu + np.abs(want) * 2.0 ** -18 * (1 + np.abs(gate) / 16))
    # addends that start in the middle of a word take another way to the same sums
    other = place(torch, add, 1)
    h2, kept2 = binding.lordba_gated_i8(x, Wl, sd, addends=other, save=True)
    assert torch.equal(h2, h) and torch.equal(kept2, kept)
    none = binding.lordba_gated_i8(x, Wl, sd)
    zero = binding.lordba_gated_i8(x, Wl, sd, addends=torch.zeros_like(ad))
    assert torch.equal(none, zero)


@pytest.mark.parametrize("shape", [(4, 83, 12871), (3, 65, 6926), (70, 30, 3000), (1100, 2100, 130)], ids=lambda s: "T%d_%dx%d" % s)
def test_gated_backward_regimes(torch, shape):
    test_gated_backward(torch, shape, 2)


def test_the_linear_gradient_is_the_difference(torch):
    # y is linear in x: <dx, v> = <g, W v> for any v, here v of the size of x
    rng = np.random.default_rng(3)
    T, d_in, d_out = 45, 301, 205
    W, ws = weights(rng, d_out, d_in)
    w = torch.from_numpy(W).cuda()
    sd = torch.from_numpy(ws).cuda()
    v, g = acts(rng, T, d_in), acts(rng, T, d_out)
    cu = lambda a: torch.from_numpy(a).cuda()
    dx = host(binding.lordba_linear_i8_backward(cu(g), binding.lordba_layout_i8(w, True), sd)).astype(np.float64)
    y = host(binding.lordba_linear_i8(cu(v), binding.lordba_layout_i8(w), sd, digits=2)).astype(np.float64)
    # every factor is off by less than 2^-10 of its size (fp16, the digits), with independent signs at most in the sum of sizes
    for t in range(T):
        assert abs(dx[t] @ v[t] - g[t] @ y[t]) <= 2.0 ** -10 * (np.abs(dx[t]) @ np.abs(v[t]) + np.abs(g[t]) @ np.abs(y[t]))


def gated(q, s, W, ws, add, F):
    """gate, up, h in 64 bits and the bounds of the errors of gate and up"""
    y, err = product(q, s, W, ws)
    y, err = y.reshape(len(y), 2, F), err.reshape(len(y), 2, F)
    if add is not None:
        y = y + add.transpose(1, 0, 2).astype(np.float64)
        err = err + F32 * np.abs(y)
    gate, up = y[:, 0], y[:, 1]
    with np.errstate(over="ignore"):
        h = gate / (1 + np.exp(-gate)) * up
    return gate, up, h, err[:, 0], err[:, 1]


GATED = [(1, 1, 1), (1, 512, 300), (3, 130, 7), (8, 257, 64), (16, 64, 15), (17, 128, 129), (33, 1000, 33), (64, 100, 127), (65, 640, 128), (130, 333, 257),
         (257, 128, 260), (1, 4096, 40), (520, 192, 130)]


@pytest.mark.parametrize("digits", [1, 2])
@pytest.mark.parametrize("addends", [False, True])
@pytest.mark.parametrize("shape", GATED, ids=lambda s: "T%d_%dx%d" % s)
def test_gated(torch, shape, addends, digits):
    T, d_in, F = shape
    rng = np.random.default_rng(T + 17 * d_in + 3 * F)
    W, ws = weights(rng, 2 * F, d_in)
    ws = (ws * 2).astype(np.float32)
    Wl, sd = binding.lordba_layout_i8(torch.from_numpy(W).cuda()), torch.from_numpy(ws).cuda()
    x = place(torch, acts(rng, T, d_in), 1)
    add = acts(rng, 2 * T, F, zero_rows=False).reshape(2, T, F) if addends else None
    ad = None if add is None else place(torch, add, 1)
    h, kept = binding.lordba_gated_i8(x, Wl, sd, addends=ad, digits=digits, save=True)
    gate, up, want, eg, eu = gated(*integers(torch, x, None, digits), W, ws, add, F)
    near(host(kept)[0], gate, eg)
    near(host(kept)[1], up, eu)
    # |d silu| <= 1.1; silu itself is off by the exponential's and the quotient's roundings, 2^-18 with the argument's 2^-24 |gate| in it
    silu = np.abs(gate) / (1 + np.exp(-gate))
    near(host(h), want, 1.1 * np.abs(up) * eg + silu * eu + np.abs(want) * 2.0 ** -18 * (1 + np.abs(gate) / 16))
    assert np.array_equal(host(h), host(binding.lordba_gated_i8(x, Wl, sd, addends=ad, digits=digits)))


def gated_loss_parts(dh, gate, up):
    sigma = 1 / (1 + np.exp(-gate))
    return dh * up * sigma * (1 + gate * (1 - sigma)), dh * gate * sigma


def test_the_gated_gradient_formula_is_the_difference():
    rng = np.random.default_rng(8)
    gate, up, dh = rng.standard_normal((3, 200)) * 3
    dg, du = gated_loss_parts(dh, gate, up)
    f = lambda g, u: dh * g / (1 + np.exp(-g)) * u
    e = 1e-5
    # central differences: e^2 |f'''| / 6, |f'''| < |dh up|, and 2^-53 |f| / e
    assert np.all(np.abs((f(gate + e, up) - f(gate - e, up)) / (2 * e) - dg) <= np.abs(dh * up) * e * e + 1e-10 * (1 + np.abs(f(gate, up))))
    assert np.all(np.abs((f(gate, up + e) - f(gate, up - e)) / (2 * e) - du) <= 1e-10 * (1 + np.abs(f(gate, up))))


@pytest.mark.parametrize("digits", [1, 2])
@pytest.mark.parametrize("shape", GATED + [(2, 40, 2049), (2, 33, 4097), (2, 20, 8200), (2, 17, 16390)], ids=lambda s: "T%d_%dx%d" % s)
def test_gated_backward(torch, shape, digits):
    T, d_in, F = shape
    rng = np.random.default_rng(T + 19 * d_in + 7 * F)
    W, ws = weights(rng, 2 * F, d_in)
    Wt, sd = binding.lordba_layout_i8(torch.from_numpy(W).cuda(), True), torch.from_numpy(ws).cuda()
    dh, gu = acts(rng, T, F), (acts(rng, 2 * T, F) * np.float16(2)).reshape(2, T, F)
    gu[0, 0, 0] = -60000   # (the exponential of that overflows)
    dx, dgu = binding.lordba_gated_i8_backward(place(torch, dh, 1), place(torch, gu, 1), Wt, sd, digits=digits)
    d, gate, up = dh.astype(np.float64), gu[0].astype(np.float64), gu[1].astype(np.float64)
    with np.errstate(over="ignore"):
        sigma = 1 / (1 + np.exp(-gate))
        dg, du = gated_loss_parts(d, gate, up)
    # roundings: 2^-18 of each factor's parts (sigma, 1 - sigma absolutely: 2^-22)
    eg = np.abs(d * up) * (sigma * (1 + np.abs(gate) * (1 - sigma)) * 2.0 ** -18 + sigma * np.abs(gate) * 2.0 ** -21)
    eu = np.abs(du) * 2.0 ** -18 * (1 + np.abs(gate) / 16)
    near(host(dgu)[0], dg, eg)
    near(host(dgu)[1], du, eu)
    rows = np.concatenate([dg, du], axis=1) * ws
    err = np.concatenate([eg, eu], axis=1) * ws
    half = 0.51 * np.abs(rows).max(axis=1) / DEPTH[digits]
    w = np.abs(W.astype(np.float64))
    near(host(dx), rows @ W.astype(np.float64), half[:, None] * w.sum(axis=0)[None, :] + (err + 4 * F32 * np.abs(rows)) @ w)


def test_rows_without_numbers_stay_by_themselves(torch):
    rng = np.random.default_rng(5)
    T, d_in, F = 37, 200, 70
    W, ws = weights(rng, 2 * F, d_in)
    w, sd = torch.from_numpy(W).cuda(), torch.from_numpy(ws).cuda()
    x = acts(rng, T, d_in)
    clean = [host(binding.lordba_linear_i8(torch.from_numpy(x).cuda(), binding.lordba_layout_i8(w), sd, digits=k)) for k in (1, 2)]
    x[3, 5], x[20, 199] = np.inf, np.nan
    rest = np.delete(np.arange(T), [3, 20])
    for k in (1, 2):
        y = host(binding.lordba_linear_i8(torch.from_numpy(x).cuda(), binding.lordba_layout_i8(w), sd, digits=k))
        assert np.isnan(y[[3, 20]]).all() and np.array_equal(y[rest], clean[k - 1][rest])
    h = host(binding.lordba_gated_i8(torch.from_numpy(x).cuda(), binding.lordba_layout_i8(w), sd))
    assert np.isnan(h[[3, 20]]).all() and np.isfinite(h[rest]).all()
    g = acts(rng, T, F)
    g[11, 0] = -np.inf
    gu = acts(rng, 2 * T, F).reshape(2, T, F)
    dx, _ = binding.lordba_gated_i8_backward(torch.from_numpy(g).cuda(), torch.from_numpy(gu).cuda(), binding.lordba_layout_i8(w, True), sd)
    dx = host(dx)
    assert np.isnan(dx[11]).all() and np.isfinite(np.delete(dx, 11, axis=0)).all()


def test_no_rows(torch):
    Wl = binding.lordba_layout_i8(torch.zeros(10, 20, dtype=torch.int8, device="cuda"))
    Wt = binding.lordba_layout_i8(torch.zeros(10, 20, dtype=torch.int8, device="cuda"), True)
    s = torch.ones(10, device="cuda")
    e = lambda *sh: torch.empty(sh, dtype=torch.float16, device="cuda")
    assert binding.lordba_linear_i8(e(0, 20), Wl, s).shape == (0, 10)
    assert binding.lordba_linear_i8_backward(e(0, 10), Wt, s).shape == (0, 20)
    assert binding.lordba_gated_i8(e(0, 20), Wl, s).shape == (0, 5)
    dx, dgu = binding.lordba_gated_i8_backward(e(0, 5), e(2, 0, 5), Wt, s)
    assert dx.shape == (0, 20) and dgu.shape == (2, 0, 5)
    q, sc = binding.lordba_quantize_rows(e(0, 20))
    assert q.shape == (0, binding.lordba_i8_row_bytes(20)) and sc.shape == (0,)


def test_results_pass_the_range_of_fp16_as_infinities(torch):
    W = np.full((3, 64), 127, dtype=np.int8)
    x = torch.full((2, 64), 60000.0, dtype=torch.float16, device="cuda")
    y = host(binding.lordba_linear_i8(x, binding.lordba_layout_i8(torch.from_numpy(W).cuda()), torch.tensor([1.0, -1.0, 1e-7], device="cuda")))
    assert np.isposinf(y[:, 0]).all() and np.isneginf(y[:, 1]).all() and np.isfinite(y[:, 2]).all()


def test_the_longest_sums_stay_inside_32_bits(torch):
    k = binding.I8_MAX_COLUMNS
    W = torch.full((2, k), -128, dtype=torch.int8, device="cuda")
    x = torch.full((3, k), -1.0, dtype=torch.float16, device="cuda")
    y = host(binding.lordba_linear_i8(x, binding.lordba_layout_i8(W), torch.full((2,), 1e-4, device="cuda"))).astype(np.float64)
    want = 128 * k * 1e-4
    assert np.all(np.abs(y - want) <= want * (F16 + F32))
    g = torch.full((3, k), -1.0, dtype=torch.float16, device="cuda")
    Wt = torch.full((2, binding.lordba_i8_row_bytes(k)), -128, dtype=torch.int8, device="cuda")
    Wt[:, k:] = 0
    dx = host(binding.lordba_linear_i8_backward(g, Wt, torch.full((k,), 1e-4, device="cuda"))).astype(np.float64)
    assert np.all(np.abs(dx - want) <= want * (F16 + F32))


def test_matrices_past_4_gib(torch):
    # weights, rows, and results whose bytes pass 32 bits: sampled entries
    n, k = (1 << 25) // 8 + 40, 1025
    gen = torch.Generator(device="cuda").manual_seed(1)
    W = torch.randint(-127, 128, (n, 1280), generator=gen, device="cuda", dtype=torch.int8)
    assert W.shape[1] == binding.lordba_i8_row_bytes(k) and W.numel() > 1 << 32
    W[:, k:] = 0
    ws = torch.full((n,), 1e-3, device="cuda")
    x = torch.randn(2, k, generator=gen, device="cuda").half()
    y = binding.lordba_linear_i8(x, W, ws)
    pick = torch.tensor([0, 1, 12345, n // 2, n - 41, n - 2, n - 1], device="cuda")
    near(host(y[:, pick]), *product(*integers(torch, x, None, 1), host(W[pick])[:, :k], host(ws[pick])))
    # as rows of activations: T * row bytes past 32 bits, a few columns out
    T = n
    xs = W[:, :k].half()
    w = torch.randint(-127, 128, (5, k), generator=gen, device="cuda", dtype=torch.int8)
    y = binding.lordba_linear_i8(xs, binding.lordba_layout_i8(w), torch.full((5,), 1e-3, device="cuda"))
    some = xs[pick].contiguous()
    near(host(y[pick]), *product(*integers(torch, some, None, 1), host(w), np.full(5, 1e-3, np.float32)))


def test_more_rows_than_a_launch(torch):
    # the row kernels take 2^21 rows a launch
    T, d_in, F = (1 << 21) + 77, 3, 4
    rng = np.random.default_rng(9)
    W, ws = weights(rng, 2 * F, d_in)
    Wt, sd = binding.lordba_layout_i8(torch.from_numpy(W).cuda(), True), torch.from_numpy(ws).cuda()
    gen = torch.Generator(device="cuda").manual_seed(2)
    dh, gu = torch.randn(T, F, generator=gen, device="cuda").half(), torch.randn(2, T, F, generator=gen, device="cuda").half()
    dx, dgu = binding.lordba_gated_i8_backward(dh, gu, Wt, sd)
    pick = torch.tensor([0, 1, (1 << 21) - 1, 1 << 21, (1 << 21) + 1, T - 1], device="cuda")
    one, many = binding.lordba_gated_i8_backward(dh[pick], gu[:, pick].contiguous(), Wt, sd)
    assert torch.equal(dx[pick], one) and torch.equal(dgu[:, pick], many)
    d, gate, up = host(dh[pick]).astype(np.float64), *host(gu[:, pick]).astype(np.float64)
    near(host(many)[0], gated_loss_parts(d, gate, up)[0], np.abs(d * up) * 2.0 ** -17 * (1 + np.abs(gate)))


@pytest.mark.parametrize("T,d_in,F", [(50, 300, 90), (2100, 260, 2100), (60, 9000, 40), (2, 512, 64)])
def test_streams_and_graphs(torch, T, d_in, F):
    rng = np.random.default_rng(6)
    W, ws = weights(rng, 2 * F, d_in)
    w, sd = torch.from_numpy(W).cuda(), torch.from_numpy(ws).cuda()
    Wl, Wt = binding.lordba_layout_i8(w), binding.lordba_layout_i8(w, True)
    x, dh = torch.from_numpy(acts(rng, T, d_in)).cuda(), torch.from_numpy(acts(rng, T, F)).cuda()
    g = torch.from_numpy(acts(rng, T, 2 * F)).cuda()

    def step(stream=None):
        h, kept = binding.lordba_gated_i8(x, Wl, sd, save=True, stream=stream)
        dx, dgu = binding.lordba_gated_i8_backward(dh, kept, Wt, sd, stream=stream)
        return (binding.lordba_linear_i8(x, Wl, sd, stream=stream), binding.lordba_linear_i8_backward(g, Wt, sd, stream=stream), h, kept, dx, dgu)

    want = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream, 0):
        side.wait_stream(torch.cuda.current_stream())
        got = step(stream)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(4):
        x.copy_(torch.from_numpy(acts(np.random.default_rng(100 + k), T, d_in)))
        eager = step()
        for o in out:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, eager)), k


def test_refusals(torch):
    e = lambda *sh, dt=torch.float16: torch.zeros(sh, dtype=dt, device="cuda")
    Wl, Wt, s = binding.lordba_layout_i8(e(10, 20, dt=torch.int8)), binding.lordba_layout_i8(e(10, 20, dt=torch.int8), True), e(10, dt=torch.float32)
    lin, back, gat, gback, rows = (binding.lordba_linear_i8, binding.lordba_linear_i8_backward, binding.lordba_gated_i8, binding.lordba_gated_i8_backward,
                                   binding.lordba_quantize_rows)
    for call in (lambda: lin(e(3, 20).float(), Wl, s), lambda: lin(e(3, 20).cpu(), Wl, s), lambda: lin(e(3, 40)[:, ::2], Wl, s), lambda: lin(e(3, 20), Wl.float(), s),
                 lambda: lin(e(3, 20), Wl, s.half()), lambda: back(e(3, 10).float(), Wt, s), lambda: gat(e(3, 20), Wl, s, addends=e(2, 3, 5).float()),
                 lambda: gback(e(3, 5), e(2, 3, 5).float(), Wt, s), lambda: rows(e(3, 20).float()), lambda: rows(e(3, 20), e(20)),
                 lambda: binding.lordba_layout_i8(e(3, 20)), lambda: lin(e(3, 20), Wl, s, y_out=e(3, 10).float())):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: lin(e(3, 400), Wl, s), lambda: lin(e(3, 20), Wl, e(11, dt=torch.float32)), lambda: lin(e(20), Wl, s), lambda: lin(e(3, 20), Wl, s, digits=3),
                 lambda: back(e(3, 11), Wt, s), lambda: gat(e(3, 20), Wl, s, addends=e(2, 3, 6)), lambda: gback(e(3, 5), e(2, 4, 5), Wt, s),
                 lambda: gat(e(3, 20), Wl, e(9, dt=torch.float32)), lambda: rows(e(3, 20), e(21, dt=torch.float32)), lambda: rows(e(3, 20), digits=0),
                 lambda: lin(e(3, 20), Wl, s, y_out=e(3, 11)), lambda: binding.lordba_layout_i8(e(3, dt=torch.int8))):
        with pytest.raises(ValueError):
            call()
    small = torch.empty(64, dtype=torch.uint8, device="cuda")
    with pytest.raises(binding.LordbaError, match="workspace"):
        lin(e(3, 20), Wl, s, workspace=small)
    both = e(3, 20)
    with pytest.raises(binding.LordbaError, match="overlaps"):
        lin(both, Wl, s, y_out=both.view(-1)[:30].view(3, 10))
