"""The C++ module behind the calls around the branch: the plain case gives what the binding's own way gives, bit for bit, and everything else is left to
the binding."""
import pytest
import torch

from paper_2605_24058_amd import binding

CALLS = (("linear_i8", 7), ("linear_i8_backward", 7), ("gated_i8", 8), ("gated_i8_backward", 7), ("dropout", 8))


def test_what_is_not_plain_is_left_to_the_binding():
    m = binding._load_torch_module()
    t = torch.zeros(2, 2, dtype=torch.float16)
    for name, n in CALLS:
        f = getattr(m, name)
        assert f(*[t] * n) is None and f(*[None] * n) is None and f(*["x"] * n) is None and f(t) is None, name


def both(monkeypatch, call):
    got = []
    for plain in (True, False):
        with monkeypatch.context() as mp:
            if not plain:
                mp.setattr(binding, "_plain_call", lambda *a: None)
            try:
                got.append(call())
                torch.cuda.synchronize()
            except Exception as e:  # noqa: BLE001 - the type is what is compared
                got.append(type(e))
    return got


def same(a, b):
    if isinstance(a, tuple):
        return isinstance(b, tuple) and len(a) == len(b) and all(same(u, v) for u, v in zip(a, b))
    if isinstance(a, torch.Tensor):
        return isinstance(b, torch.Tensor) and a.dtype == b.dtype and a.shape == b.shape and torch.equal(a.view(torch.int16), b.view(torch.int16))
    return a is b


def case():
    g = torch.Generator().manual_seed(4)
    T, d_in, F = 9, 70, 33
    half = lambda *s: torch.randn(s, generator=g).half().cuda()
    W = torch.randint(-127, 128, (2 * F, d_in), generator=g, dtype=torch.int8).cuda()
    s = torch.rand(2 * F, generator=g).cuda() / 500
    return dict(x=half(T, d_in), g=half(T, 2 * F), dh=half(T, F), kept=half(2, T, F), W=binding.lordba_layout_i8(W), Wt=binding.lordba_layout_i8(W, True), s=s,
                add=half(2, T, F), y=half(T, 2 * F), base=half(T, d_in))


@pytest.mark.gpu
def test_plain_calls(monkeypatch):
    c = case()
    calls = [lambda: binding.lordba_linear_i8(c["x"], c["W"], c["s"]), lambda: binding.lordba_linear_i8(c["x"], c["W"], c["s"], digits=2),
             lambda: binding.lordba_linear_i8(c["x"], c["W"], c["s"], y_out=torch.empty_like(c["y"])),
             lambda: binding.lordba_linear_i8_backward(c["g"], c["Wt"], c["s"]), lambda: binding.lordba_linear_i8_backward(c["g"], c["Wt"], c["s"], digits=1),
             lambda: binding.lordba_gated_i8(c["x"], c["W"], c["s"]), lambda: binding.lordba_gated_i8(c["x"], c["W"], c["s"], addends=c["add"], save=True),
             lambda: binding.lordba_gated_i8(c["x"], c["W"], c["s"], addends=c["add"], digits=2),
             lambda: binding.lordba_gated_i8_backward(c["dh"], c["kept"], c["Wt"], c["s"]), lambda: binding.lordba_dropout(c["x"], 0.3, 5),
             lambda: binding.lordba_dropout(c["x"], 0.3, (1 << 64) - 1, (1 << 64) - 1, y_base=c["base"]), lambda: binding.lordba_dropout(c["x"], 0, 5),
             lambda: binding.lordba_dropout(c["x"], 0.3, 5, offset_dev=torch.tensor([3], device="cuda"))]
    module = binding._load_torch_module()
    taken = []
    for name, _ in CALLS:     # each call above but the one with an integer p is taken by the module
        f = getattr(module, name)
        assert callable(f)
    real = binding._plain_call
    monkeypatch.setattr(binding, "_plain_call", lambda *a: (lambda r: (taken.append(r is not None), r)[1])(real(*a)))
    for k, call in enumerate(calls):
        a, b = both(monkeypatch, call)
        assert not isinstance(a, type) and same(a, b), k
    assert taken.count(False) == 1 and len(taken) == len(calls)
    y = torch.empty_like(c["y"])
    assert binding.lordba_linear_i8(c["x"], c["W"], c["s"], y_out=y) is y
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = binding.lordba_linear_i8(c["x"], c["W"], c["s"], stream=side)
    side.synchronize()
    assert same(other, calls[0]())


@pytest.mark.gpu
def test_spoiled_arguments(monkeypatch):
    # another type, not contiguous, on the CPU, shorter, one more dimension, not a tensor: the same exception type or the same result both ways
    c = case()
    spoil = (lambda t: t.double(), lambda t: torch.stack((t, t), -1)[..., 0], lambda t: t.cpu(), lambda t: t[..., :-1].contiguous(), lambda t: t[None])
    for f, names in ((binding.lordba_linear_i8, ("x", "W", "s")), (binding.lordba_linear_i8_backward, ("g", "Wt", "s")), (binding.lordba_gated_i8, ("x", "W", "s", "add")),
                     (binding.lordba_gated_i8_backward, ("dh", "kept", "Wt", "s"))):
        for k in range(len(names)):
            for bad in spoil:
                args = [bad(c[n]) if i == k else c[n] for i, n in enumerate(names)]
                a, b = both(monkeypatch, lambda: f(*args))
                assert same(a, b), (f.__name__, names[k])
