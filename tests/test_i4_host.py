"""Host-side checks of the 4-bit projections and of the teacher's loss that need no GPU: sizes, and every refusal before a device is touched."""
import ctypes

import pytest
import torch

from paper_2605_24058_amd import binding

OK, NULL, DIM, VALUE, ALIAS, ALIGN, NO_DEVICE = 0, 1, 2, 3, 4, 5, 6


@pytest.fixture(scope="module")
def lib():
    return binding.load_library()


def test_sizes(lib):
    # rows to pairs of 16-row blocks, columns to blocks of 128: 1 KiB each; a half each for itself
    for args, blocks in (((1, 1, 1, 0), 2), ((32, 128, 1, 0), 2), ((33, 129, 1, 0), 8), ((33, 129, 1, 1), 10), ((66, 129, 2, 0), 16), ((66, 129, 2, 1), 20)):
        assert lib.lordba_i4_code_bytes(*args) == 1024 * blocks, args
    for args, scales in (((33, 129, 64, 1, 0), 4 * 4 * 16), ((33, 129, 32, 1, 1), 5 * 128), ((66, 129, 128, 2, 0), 8 * 2 * 16), ((66, 129, 128, 2, 1), 2 * 256)):
        assert lib.lordba_i4_scale_count(*args) == scales, args
    for bad in ((0, 5, 1, 0), (5, 0, 1, 0), (5, 5, 2, 0), (5, 5, 3, 0), (5, 5, 0, 0), ((1 << 24) + 1, 5, 1, 0), (5, (1 << 24) + 1, 1, 0)):
        assert lib.lordba_i4_code_bytes(*bad) == 0 and lib.lordba_i4_scale_count(*bad[:2], 128, *bad[2:]) == 0
    assert [lib.lordba_i4_scale_count(5, 5, g, 1, 0) for g in (0, 16, 48, 256, -128)] == [0] * 5
    assert lib.lordba_i4_code_bytes(1 << 24, 1 << 24, 1, 0) == 1 << 47     # (no 32-bit arithmetic)


# addresses that are never followed: every call below is refused, or finds no device
BUF = [(i + 1) << 40 for i in range(10)]


def linear(lib, f, x=BUF[0], c=BUF[1], s=BUF[2], z=BUF[3], y=BUF[4], T=4, d_in=100, d_out=60, group=32):
    return getattr(lib, f)(x, c, s, z, y, T, d_in, d_out, group, None)


@pytest.mark.parametrize("f", ["lordba_linear_i4", "lordba_linear_i4_backward"])
def test_linear_refusals(lib, f):
    for name in ("x", "c", "s", "y"):
        assert linear(lib, f, **{name: None}) == NULL
    for kw in ({"T": -1}, {"d_in": 0}, {"d_out": 0}, {"d_in": (1 << 24) + 1}, {"d_out": (1 << 24) + 1}, {"T": 1 << 31}):
        assert linear(lib, f, **kw) == DIM
    for group in (0, 16, 33, 256, -32):
        assert linear(lib, f, group=group) == VALUE
    for kw in ({"x": BUF[0] + 1}, {"c": BUF[1] + 8}, {"s": BUF[2] + 2}, {"z": BUF[3] + 8}, {"y": BUF[4] + 1}):
        assert linear(lib, f, **kw) == ALIGN
    for kw in ({"y": BUF[0]}, {"y": BUF[1] + 16}, {"y": BUF[2]}, {"y": BUF[3] + 32}):
        assert linear(lib, f, **kw) == ALIAS
    assert linear(lib, f, T=0, x=None, y=None) == OK


def gated(lib, f, a=BUF[0], b=BUF[1], c=BUF[2], s=BUF[3], z=BUF[4], d=BUF[5], e=BUF[6], T=4, d_in=100, d_ff=60, group=64):
    if f == "lordba_gated_i4":     # x, codes, scale, zero, addends, h, gate_up
        return lib.lordba_gated_i4(a, c, s, z, b, d, e, T, d_in, d_ff, group, None)
    return lib.lordba_gated_i4_backward(a, b, c, s, z, d, e, T, d_in, d_ff, group, None)   # dh, gate_up, codes, scale, zero, dx, dgate_up


@pytest.mark.parametrize("f", ["lordba_gated_i4", "lordba_gated_i4_backward"])
def test_gated_refusals(lib, f):
    optional = ("b", "e", "z") if f == "lordba_gated_i4" else ("z",)
    for name in ("a", "b", "c", "s", "d", "e"):
        if name not in optional:
            assert gated(lib, f, **{name: None}) == NULL
    for kw in ({"T": -1}, {"d_in": 0}, {"d_ff": 0}, {"d_ff": (1 << 23) + 1}):
        assert gated(lib, f, **kw) == DIM
    assert gated(lib, f, group=96) == VALUE
    for kw in ({"a": BUF[0] + 1}, {"b": BUF[1] + 1}, {"c": BUF[2] + 4}, {"s": BUF[3] + 8}, {"z": BUF[4] + 2}, {"d": BUF[5] + 1}, {"e": BUF[6] + 1}):
        assert gated(lib, f, **kw) == ALIGN
    for kw in ({"d": BUF[0]}, {"d": BUF[2] + 2}, {"e": BUF[0] + 2}, {"e": BUF[1]}, {"d": BUF[6] + 40}, {"e": BUF[3]}, {"d": BUF[4] + 16}):
        assert gated(lib, f, **kw) == ALIAS
    assert gated(lib, f, T=0, a=None, d=None) == OK


def test_quantiser_and_layout_refusals(lib):
    quant = lambda w=BUF[0], c=BUF[1], s=BUF[2], z=BUF[3], n=4, k=100, g=32: lib.lordba_quantize_i4(w, c, s, z, n, k, g, None)
    for name in ("w", "c", "s"):
        assert quant(**{name: None}) == NULL
    assert quant(n=-1) == quant(k=0) == quant(n=(1 << 24) + 1) == quant(k=(1 << 24) + 1) == DIM and quant(g=48) == VALUE
    assert quant(w=BUF[0] + 1) == quant(s=BUF[2] + 1) == ALIGN
    for kw in ({"c": BUF[0]}, {"s": BUF[0] + 2}, {"z": BUF[0]}, {"s": BUF[1]}, {"z": BUF[2]}):
        assert quant(**kw) == ALIAS
    assert quant(n=0) == OK
    lay = lambda c=BUF[0], s=BUF[1], z=BUF[2], o=BUF[3], os=BUF[4], oz=BUF[5], n=4, k=100, g=64, h=1, t=0: lib.lordba_layout_i4(c, s, z, o, os, oz, n, k, g, h, t, None)
    for name in ("c", "s", "o", "os", "oz"):
        assert lay(**{name: None}) == NULL
    assert lay(n=0) == lay(k=0) == lay(n=(1 << 24) + 1) == DIM
    assert lay(g=1) == lay(h=0) == lay(h=3) == lay(n=5, h=2) == VALUE
    assert lay(s=BUF[1] + 1) == lay(o=BUF[3] + 8) == lay(os=BUF[4] + 2) == lay(oz=BUF[5] + 8) == ALIGN
    for kw in ({"o": BUF[0]}, {"os": BUF[1]}, {"oz": BUF[2]}, {"os": BUF[3] + 1024}, {"oz": BUF[4]}, {"o": BUF[2]}):
        assert lay(**kw) == ALIAS


def distill(lib, z=BUF[0], kind=0, index=BUF[1], top=BUF[2], labels=BUF[3], k=5, u=1.0, soft=1.0, hard=0.5, dl=BUF[4], loss=BUF[5], kept=BUF[6], dz=BUF[7], T=4, V=100,
            backward=False, teacher=True):
    w = ctypes.byref(binding.Teacher(index, top, labels, k, u, soft, hard)) if teacher else None
    if backward:
        return lib.lordba_distill_backward(dl, z, kind, kept, w, dz, T, V, None)
    return lib.lordba_distill(z, kind, w, dl, loss, kept, dz, T, V, None)


@pytest.mark.parametrize("backward", [False, True])
def test_distill_refusals(lib, backward):
    f = lambda **kw: distill(lib, backward=backward, **kw)
    inf, nan = float("inf"), float("nan")
    for kw in ({"z": None}, {"teacher": False}, {"index": None}, {"top": None}, {"dl": None}, {"dz": None}, {"kept" if backward else "loss": None}):
        assert f(**kw) == NULL, kw
    for kw in ({"T": -1}, {"T": 1 << 31}, {"V": 0}, {"V": (1 << 24) + 1}, {"k": -1}, {"k": 1025}):
        assert f(**kw) == DIM, kw
    for kw in ({"kind": 2}, {"kind": -1}, {"u": 0.0}, {"u": -1.0}, {"u": nan}, {"u": inf}, {"soft": nan}, {"soft": inf}, {"hard": -inf}):
        assert f(**kw) == VALUE, kw
    for kw in ({"z": BUF[0] + 1}, {"z": BUF[0] + 2, "kind": 1}, {"index": BUF[1] + 2}, {"top": BUF[2] + 1}, {"labels": BUF[3] + 1}, {"dl": BUF[4] + 2}, {"kept": BUF[6] + 2},
               {"dz": BUF[7] + 1}):
        assert f(**kw) == ALIGN, kw
    for kw in ({"dz": BUF[0] + 2}, {"dz": BUF[0] - 2}, {"dz": BUF[1]}, {"dz": BUF[2]}, {"dz": BUF[3]}, {"dz": BUF[4]}, {"dz": BUF[6]}):
        assert f(**kw) == ALIAS, kw
    if not backward:
        for kw in ({"loss": BUF[0]}, {"loss": BUF[0], "dz": BUF[0]}, {"kept": BUF[0], "dz": BUF[0]}, {"loss": BUF[6] + 4}, {"loss": BUF[4]}, {"kept": BUF[3]}):
            assert f(**kw) == ALIAS, kw
    assert f(T=0, z=None, dl=None, dz=None, loss=None, kept=None) == OK


def test_accepted_arguments_reach_the_device_check(lib):
    if torch.cuda.is_available():
        pytest.skip("the addresses above are not memory")
    for f in ("lordba_linear_i4", "lordba_linear_i4_backward"):
        assert linear(lib, f) == linear(lib, f, z=None) == linear(lib, f, x=BUF[0] + 2, y=BUF[4] + 2, group=128) == NO_DEVICE
    for f in ("lordba_gated_i4", "lordba_gated_i4_backward"):
        assert gated(lib, f) == gated(lib, f, z=None) == NO_DEVICE
    assert gated(lib, "lordba_gated_i4", b=None, e=None) == NO_DEVICE
    assert distill(lib) == distill(lib, dz=BUF[0]) == distill(lib, dl=None, dz=None) == distill(lib, kept=None) == NO_DEVICE
    assert distill(lib, k=0, index=None, top=None, kind=1) == distill(lib, labels=None) == NO_DEVICE
    assert distill(lib, backward=True) == distill(lib, backward=True, dz=BUF[0]) == NO_DEVICE


def test_what_the_binding_refuses():
    half, byte = torch.zeros(4, 100, dtype=torch.float16), torch.zeros(4, 100, dtype=torch.uint8)
    W = binding.WeightsI4(byte, half, None, 4, 100, 32, 1, False)
    with pytest.raises(TypeError, match="x must be"):
        binding.lordba_linear_i4(half, W)
    with pytest.raises(TypeError, match="codes must be"):
        binding.lordba_layout_i4(byte, half)
    with pytest.raises(TypeError, match="w must be"):
        binding.lordba_quantize_i4(half)
    with pytest.raises(TypeError, match="dh must be"):
        binding.lordba_gated_i4_backward(half, half, W)
    with pytest.raises(TypeError, match="logits must be"):
        binding.lordba_distill(half)
    with pytest.raises(TypeError, match="logits must be a contiguous float16 or float32"):
        binding.lordba_distill(half.bfloat16())
    m = binding._load_torch_module()
    for name, n in (("linear_i4", 4), ("linear_i4_backward", 4), ("gated_i4", 5), ("gated_i4_backward", 4), ("distill", 10), ("distill_backward", 11)):
        f = getattr(m, name)      # what is not plain is left to the binding
        assert f(*[half] * n) is None and f(*[None] * n) is None and f(*["x"] * n) is None and f(*[W] * n) is None and f(half) is None, name


def test_tensors_of_two_devices_are_refused():
    class On:
        def __init__(self, device):
            self.device = torch.device("cuda", device)

    with pytest.raises(ValueError, match="one device"):
        with binding._on_device(None, On(0), None, On(0), On(1)):
            pass
