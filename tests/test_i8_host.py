"""Host-side checks of the 8-bit projections and of dropout that need no GPU: sizes, and every refusal before a device is touched."""
import ctypes

import pytest

from paper_2605_24058_amd import binding

OK, NULL, DIM, VALUE, ALIAS, ALIGN, NO_DEVICE, WORKSPACE = 0, 1, 2, 3, 4, 5, 6, 9


@pytest.fixture(scope="module")
def lib():
    return binding.load_library()


def test_sizes(lib):
    assert [binding.lordba_i8_row_bytes(c) for c in (1, 128, 129, 4096, 131071)] == [256, 256, 256, 4096, 131072]
    assert [binding.lordba_i8_row_bytes(c) for c in (0, -1, 131072)] == [0, 0, 0]
    assert binding.lordba_i8_workspace_bytes(3, 200, 1) >= 3 * 256 + 12
    assert binding.lordba_i8_workspace_bytes(3, 200, 2) >= 6 * 256 + 12
    for args in ((-1, 200, 1), (3, 0, 1), (3, 131072, 1), (3, 200, 0), (3, 200, 3), (1 << 31, 200, 1)):
        assert binding.lordba_i8_workspace_bytes(*args) == 0


# addresses that are never followed: every call below is refused, or finds no device
BUF = [(i + 1) << 32 for i in range(8)]
BIG = 1 << 30


def linear(lib, f, x=BUF[0], W=BUF[1], s=BUF[2], y=BUF[3], ws=BUF[4], n=BIG, T=4, d_in=100, d_out=60, digits=1):
    return getattr(lib, f)(x, W, s, y, ws, n, T, d_in, d_out, digits, None)


@pytest.mark.parametrize("f", ["lordba_linear_i8", "lordba_linear_i8_backward"])
def test_linear_refusals(lib, f):
    for name in ("x", "W", "s", "y", "ws"):
        assert linear(lib, f, **{name: None}) == NULL
    for kw in ({"T": -1}, {"d_in": 0}, {"d_out": 0}, {"d_in" if f == "lordba_linear_i8" else "d_out": 131072}, {"d_out": (1 << 24) + 1}, {"T": 1 << 31}):
        assert linear(lib, f, **kw) == DIM
    for digits in (0, 3, -1):
        assert linear(lib, f, digits=digits) == VALUE
    assert linear(lib, f, n=100) == WORKSPACE
    for kw in ({"x": BUF[0] + 1}, {"W": BUF[1] + 8}, {"s": BUF[2] + 2}, {"y": BUF[3] + 1}, {"ws": BUF[4] + 8}):
        assert linear(lib, f, **kw) == ALIGN
    for kw in ({"y": BUF[0]}, {"y": BUF[1] + 16}, {"y": BUF[2]}, {"y": BUF[4] + 64}, {"ws": BUF[0]}, {"ws": BUF[1]}):
        assert linear(lib, f, **kw) == ALIAS
    assert linear(lib, f, T=0, x=None, y=None, ws=None, n=0) == OK


def gated(lib, f, a=BUF[0], b=BUF[1], s=BUF[2], c=BUF[3], d=BUF[4], e=BUF[5], ws=BUF[6], n=BIG, T=4, d_in=100, d_ff=60, digits=1):
    if f == "lordba_gated_i8":     # x, W, w_scale, addends, h, gate_up
        return lib.lordba_gated_i8(a, b, s, c, d, e, ws, n, T, d_in, d_ff, digits, None)
    return lib.lordba_gated_i8_backward(a, c, b, s, d, e, ws, n, T, d_in, d_ff, digits, None)   # dh, gate_up, Wt, w_scale, dx, dgate_up


@pytest.mark.parametrize("f", ["lordba_gated_i8", "lordba_gated_i8_backward"])
def test_gated_refusals(lib, f):
    optional = ("c", "e") if f == "lordba_gated_i8" else ()
    for name in ("a", "b", "s", "c", "d", "e", "ws"):
        if name not in optional:
            assert gated(lib, f, **{name: None}) == NULL
    for kw in ({"T": -1}, {"d_in": 0}, {"d_ff": 0}, {"d_in": 131072} if f == "lordba_gated_i8" else {"d_ff": 65536}):
        assert gated(lib, f, **kw) == DIM
    assert gated(lib, f, digits=3) == VALUE
    assert gated(lib, f, n=100) == WORKSPACE
    for kw in ({"a": BUF[0] + 1}, {"b": BUF[1] + 4}, {"s": BUF[2] + 1}, {"c": BUF[3] + 1}, {"d": BUF[4] + 1}, {"e": BUF[5] + 1}, {"ws": BUF[6] + 1}):
        assert gated(lib, f, **kw) == ALIGN
    for kw in ({"d": BUF[0]}, {"d": BUF[1] + 2}, {"e": BUF[0] + 2}, {"e": BUF[3]}, {"d": BUF[5] + 40}, {"ws": BUF[3]}, {"e": BUF[6]}):
        assert gated(lib, f, **kw) == ALIAS
    assert gated(lib, f, T=0, a=None, d=None, ws=None, n=0) == OK


def test_rows_and_layout_refusals(lib):
    rows = lambda x=BUF[0], cs=BUF[1], q=BUF[2], s=BUF[3], n=4, k=100, digits=1: lib.lordba_quantize_rows(x, cs, q, s, n, k, digits, None)
    for name in ("x", "q", "s"):
        assert rows(**{name: None}) == NULL
    assert rows(n=-1) == rows(k=0) == rows(k=131072) == DIM and rows(digits=0) == VALUE
    for kw in ({"x": BUF[0] + 1}, {"cs": BUF[1] + 1}, {"q": BUF[2] + 4}, {"s": BUF[3] + 2}):
        assert rows(**kw) == ALIGN
    for kw in ({"q": BUF[0]}, {"s": BUF[0]}, {"q": BUF[1]}, {"s": BUF[2] + 16}, {"s": BUF[1]}):
        assert rows(**kw) == ALIAS
    assert rows(n=0) == OK
    lay = lambda w=BUF[0], o=BUF[1], n=4, k=100, t=0: lib.lordba_layout_i8(w, o, n, k, t, None)
    assert lay(w=None) == lay(o=None) == NULL
    assert lay(n=0) == lay(k=0) == lay(k=131072) == lay(n=131072, t=1) == lay(n=(1 << 24) + 1) == DIM
    assert lay(o=BUF[1] + 8) == ALIGN and lay(o=BUF[0] + 16) == ALIAS


def test_dropout_refusals(lib):
    nan = float("nan")
    f = lambda x=BUF[0], b=BUF[1], y=BUF[2], n=100, p=0.5, o=BUF[3]: lib.lordba_dropout(x, b, y, n, p, 1, 2, o, None)
    assert f(x=None) == f(y=None) == NULL
    assert f(n=-1) == f(n=(1 << 38) + 1) == DIM
    assert f(p=-0.1) == f(p=1.1) == f(p=nan) == VALUE
    assert f(x=BUF[0] + 1) == f(b=BUF[1] + 1) == f(y=BUF[2] + 1) == f(o=BUF[3] + 4) == ALIGN
    assert f(y=BUF[0] + 2) == f(y=BUF[1] + 2) == f(y=BUF[3] - 100) == ALIAS
    assert f(n=0, x=None, y=None) == OK


def test_accepted_arguments_reach_the_device_check(lib):
    import torch
    if torch.cuda.is_available():
        pytest.skip("the addresses above are not memory")
    assert linear(lib, "lordba_linear_i8") == linear(lib, "lordba_linear_i8_backward") == NO_DEVICE
    assert gated(lib, "lordba_gated_i8") == gated(lib, "lordba_gated_i8", c=None, e=None) == gated(lib, "lordba_gated_i8_backward") == NO_DEVICE
    assert lib.lordba_dropout(BUF[0], None, BUF[0], 100, 0.5, 1, 2, None, None) == NO_DEVICE     # in place
    assert lib.lordba_dropout(BUF[0], BUF[1], BUF[1], 100, 0.5, 1, 2, None, None) == NO_DEVICE
    assert ctypes.c_int(lib.lordba_layout_i8(BUF[0], BUF[1], 4, 100, 1, None)).value == NO_DEVICE
