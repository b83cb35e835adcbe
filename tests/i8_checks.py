"""What the tests of the 8-bit projections, the gated block and dropout compare with and call through: a comparison that no NaN passes, tensors
with guarded surroundings, the calls through the C interface on them, and the definitions in 64 bits.

Bounds.  Integer sums are exact, so given a row's integers q and scale s, y = s w sum(q W) is off by the conversions to fp32 (2^-24 of what is
converted), three fp32 operations and one rounding to fp16: 2^-11 of the value (2^-25 among the subnormals), and F32 = 2^-21 of
256 |sum hi| + |sum lo| for the rest, with a factor of two to spare."""
import numpy as np

from paper_2605_24058_amd import binding

F32, F16, SUB = 2.0 ** -21, 2.0 ** -11, 2.0 ** -25
DEPTH = {1: 127, 2: 32512}
LARGEST, OVERFLOWS = 65504.0, 65520.0     # of fp16: the largest number, and where rounding gives an infinity


def near(got, want, err):
    """got: fp16 of a value within err of want.  want and err are numbers; got is one too, but an infinity of want's sign where want is past the
    range of fp16 by more than err (either within err of its end).  numpy arrays or torch tensors alike."""
    if not isinstance(got, np.ndarray):
        import torch

        got, want, err = got.double(), want.double(), torch.as_tensor(err, dtype=torch.float64, device=got.device)
        finite, large = torch.isfinite, (got.abs() == float("inf")) & (got * want > 0)
    else:
        got, want, err = got.astype(np.float64), np.asarray(want, np.float64), np.asarray(err, np.float64)
        with np.errstate(invalid="ignore"):
            finite, large = np.isfinite, (np.abs(got) == np.inf) & (got * want > 0)
    assert bool(finite(want).all()) and bool(finite(err).all()), "the expected values are no numbers"
    limit = abs(want) * F16 + err * 1.01 + SUB
    with np.errstate(invalid="ignore"):
        good = (abs(got - want) <= limit) & (abs(want) - err * 1.01 < OVERFLOWS) | large & (abs(want) + err * 1.01 >= OVERFLOWS)
    assert bool(good.all()), (int((~good).sum()), [int(v) for v in (~good).reshape(-1).nonzero()[0].reshape(-1)[:3]])


GUARD = 512     # bytes on both sides


class Memory:
    """Tensors on the GPU whose surroundings are known: NaN around floating-point inputs (bytes of 0x7F around others), 0xA5 around and in outputs.
    unchanged() says that what lies around them all, and in the inputs, is as it was."""

    def __init__(self, torch, device="cuda"):
        self.torch, self.device, self.kept = torch, device, []

    def _place(self, nbytes, shift, fill):
        big = self.torch.empty(nbytes + 2 * GUARD + 64, dtype=self.torch.uint8, device=self.device)
        if fill is None:
            big[:big.numel() // 2 * 2].view(self.torch.float16).fill_(float("nan"))
            big[big.numel() // 2 * 2:] = 0xFF
        else:
            big.fill_(fill)
        start = GUARD + (-(big.data_ptr() + GUARD)) % 64 + shift
        return big, start

    def input(self, a, shift=0):
        """`a` (a numpy array or a tensor), its first byte `shift` elements behind a 64-byte boundary."""
        torch = self.torch
        t = torch.from_numpy(np.ascontiguousarray(a)) if isinstance(a, np.ndarray) else a
        big, start = self._place(t.numel() * t.element_size(), shift * t.element_size(), None if t.is_floating_point() else 0x7F)
        if t.dtype == torch.float32:     # (two NaN of 16 bits are no NaN of 32)
            big[start % 4:][:(big.numel() - start % 4) // 4 * 4].view(torch.float32).fill_(float("nan"))
        v = big[start:start + t.numel() * t.element_size()].view(t.dtype).view(t.shape)
        v.copy_(t)
        self.kept.append((big, big.clone(), None))
        return v

    def output(self, shape, dtype, shift=0):
        item = self.torch.empty(0, dtype=dtype).element_size()
        n = int(np.prod(shape)) * item
        big, start = self._place(n, shift * item, 0xA5)
        self.kept.append((big, big.clone(), (start, start + n)))
        return big[start:start + n].view(dtype).view(shape)

    def unchanged(self):
        if self.device == "cuda":
            self.torch.cuda.synchronize()
        for big, before, written in self.kept:
            if written is None:
                assert self.torch.equal(big, before), "an input or what is around it was written to"
            else:
                assert self.torch.equal(big[:written[0]], before[:written[0]]), "written in front of an output"
                assert self.torch.equal(big[written[1]:], before[written[1]:]), "written behind an output"


def call(torch, name, *args):
    """A call of the C interface on the current stream; tensors go as pointers, None as NULL."""
    st = getattr(binding.load_library(), name)(*[a.data_ptr() if hasattr(a, "data_ptr") else a for a in args], torch.cuda.current_stream().cuda_stream)
    if st != 0:
        raise binding.LordbaError(st, name)


def workspace(mem, T, cols, digits):
    return mem.output((binding.lordba_i8_workspace_bytes(T, cols, digits),), mem.torch.uint8)


# ---- inputs ----
def weights(rng, n, k):
    """int8 [n, k], every value from -128 on, and fp32 scales [n]"""
    return rng.integers(-128, 128, size=(n, k), dtype=np.int8), (rng.uniform(0.2, 2.0, size=n) / (70 * np.sqrt(k))).astype(np.float32)


def acts(rng, rows, cols):
    """N(0, 1), some channels eight times as large, a row of zeros"""
    x = rng.standard_normal((rows, cols), dtype=np.float32)
    x[:, ::37] *= 8
    if rows > 4:
        x[rows // 2] = 0
    return x.astype(np.float16)


# ---- definitions ----
def rows_of(x, col_scale, digits):
    """The rows' integers by the header's definition in fp32: (parts [digits] of int8 [rows, cols], scales fp32 [rows])."""
    v = x.astype(np.float32) if col_scale is None else x.astype(np.float32) * col_scale
    amax = np.abs(v).max(axis=1)
    zero = amax == 0
    D = np.float32(DEPTH[digits])
    inverse = np.where(zero, np.float32(0), D / np.where(zero, np.float32(1), amax))
    q = np.rint(v * inverse[:, None]).astype(np.int32)
    if digits == 1:
        return [q.astype(np.int8)], amax / D
    hi = (q + 128) >> 8
    return [hi.astype(np.int8), (q - 256 * hi).astype(np.int8)], amax / D


def sums(torch, q, W):
    """The digits' sums with W [n, k] (a tensor of int8), exact in 64 bits: (value, 256 |hi| + |lo|)."""
    Wd = W.double().t().contiguous()
    parts = [torch.mm(torch.from_numpy(p).cuda().double(), Wd) for p in q]
    if len(parts) == 1:
        return parts[0], parts[0].abs()
    return 256 * parts[0] + parts[1], 256 * parts[0].abs() + parts[1].abs()


def product(torch, q, s, W, w_scale):
    """y and the bound of its error before the rounding to fp16"""
    value, size = sums(torch, q, W)
    f = torch.from_numpy(s).cuda().double()[:, None] * torch.from_numpy(w_scale).cuda().double()[None, :]
    return value * f, size * f * F32


def gated(torch, q, s, W, w_scale, addends):
    """gate, up, h and the bounds of the errors of the three.  addends: numpy [2, T, F] or None"""
    y, err = product(torch, q, s, W, w_scale)
    F = y.shape[1] // 2
    (gate, up), (eg, eu) = y.split(F, dim=1), err.split(F, dim=1)
    if addends is not None:
        a = torch.from_numpy(addends).cuda().double()
        gate, up = gate + a[0], up + a[1]
        eg, eu = eg + F32 * gate.abs(), eu + F32 * up.abs()
    silu = gate * torch.sigmoid(gate)
    # |d silu| <= 1.1; silu itself is off by the exponential's and the quotient's roundings, 2^-18 with the argument's 2^-24 |gate| in it
    eh = 1.1 * up.abs() * eg + silu.abs() * eu + (silu * up).abs() * 2.0 ** -18 * (1 + gate.abs() / 16)
    return gate, up, silu * up, eg, eu, eh


def gated_gradient(torch, dh, gate_up):
    """dgate, dup and the bounds of their errors before the rounding to fp16; numpy fp16 in, 64-bit tensors out"""
    d, gate, up = (torch.from_numpy(a).cuda().double() for a in (dh, gate_up[0], gate_up[1]))
    sigma, rest = torch.sigmoid(gate), torch.sigmoid(-gate)
    dg, du = d * up * sigma * (1 + gate * rest), d * gate * sigma
    # 2^-18 of each factor's parts; sigma and 1 - sigma absolutely: 2^-22
    eg = (d * up).abs() * (sigma * (1 + gate.abs() * rest) * 2.0 ** -18 + sigma * gate.abs() * 2.0 ** -21)
    return dg, du, eg, du.abs() * 2.0 ** -18 * (1 + gate.abs() / 16)


def row_error(torch, values, err, w_scale, Wt, digits):
    """dx = (values w_scale) Wt^T and its error: half a step of the row's largest number per entry (two hundredths of one for the fp32 roundings of
    the step), the numbers' own errors, and fp32 roundings of the products.  Wt: int8 [n, k]."""
    s = torch.from_numpy(w_scale).cuda().double()
    rows, W = values * s, Wt.double()
    half = 0.51 * (rows.abs() + err * s).amax(dim=1, keepdim=True) / DEPTH[digits]
    A = W.abs()
    return torch.mm(rows, W.t().contiguous()), half * A.sum(dim=1)[None, :] + torch.mm(err * s + 4 * F32 * rows.abs(), A.t().contiguous())
