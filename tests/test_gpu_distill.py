"""What tokens lose against a teacher's top logits, and its gradient, against the definition in 64 bits and against differences.

Bounds.  A probability exp((z - m) / u) / sum: the argument, up to A = (max z - min z over what counts) / u + |lse|, is off by 4 * 2^-24 A (differences, factor,
logarithm), the exponential by 2^-22, the sum by one step of 2^-24 for each of the terms a thread adds, V / 256 and some, and 64 for the joining.  rel(V, A) is their sum, doubled."""
import numpy as np
import pytest

import i8_checks
from paper_2605_24058_amd import binding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    return torch


def rel(V, A):
    return 2 * (4 * 2.0 ** -24 * A + 2.0 ** -22 + (V / 256 + 64) * 2.0 ** -24)


def reference(torch, z, index, top, labels, u, soft, hard, weight):
    """loss, gradient and the bounds of both (before a rounding of the gradient to its type), in 64 bits on the CPU.  Entries and labels that are not there: below 0."""
    z = z.double().cpu()
    T, V = z.shape
    loss, grad, el, eg = (torch.zeros(T, dtype=torch.float64), torch.zeros(T, V, dtype=torch.float64), torch.zeros(T, dtype=torch.float64),
                          torch.zeros(T, V, dtype=torch.float64))
    for t in range(T):
        w = float(weight[t])
        some = [] if index is None else [(int(v), float(l)) for v, l in zip(index[t], top[t]) if 0 <= int(v) < V and float(l) != -np.inf]
        finite = z[t][z[t] > -np.inf]
        span = float(finite.max() - finite.min()) if len(finite) else 0.0
        if some and soft:
            l = torch.tensor([s[1] for s in some], dtype=torch.float64) / u
            log_p, log_q = torch.log_softmax(l, 0), torch.log_softmax(z[t] / u, 0)
            A = span / u + np.log(V) + float(l.max() - l.min())
            for (v, _), lp in zip(some, log_p):
                p = lp.exp()
                if p > 0:
                    loss[t] += soft * u * u * p * (lp - log_q[v])
                    el[t] += abs(soft) * u * u * p * (rel(V, A) + (lp.abs() + log_q[v].abs()) * (rel(V, A) + 2.0 ** -21))
                grad[t, v] -= w * soft * u * p
                eg[t, v] += abs(w * soft * u) * p * (rel(1024, A) + 2.0 ** -21)
            q = log_q.exp()
            grad[t] += w * soft * u * q
            eg[t] += abs(w * soft * u) * q * (rel(V, A) + 2.0 ** -21)
        if labels is not None and 0 <= int(labels[t]) < V and hard:
            c, log_r = int(labels[t]), torch.log_softmax(z[t], 0)
            A = span + np.log(V)
            loss[t] -= hard * log_r[c]
            el[t] += abs(hard) * (rel(V, A) + log_r[c].abs() * 2.0 ** -21 + A * 2.0 ** -22)
            grad[t] += w * hard * log_r.exp()
            grad[t, c] -= w * hard
            eg[t] += abs(w * hard) * log_r.exp() * (rel(V, A) + 2.0 ** -21)
            eg[t, c] += abs(w * hard) * 2.0 ** -23
    # (exponentials below the range of fp32 are 0)
    return loss, grad, el + 2.0 ** -100, eg + 2.0 ** -100


def check(torch, loss, grad, want):
    wl, wg, el, eg = want
    assert bool((abs(loss.double().cpu() - wl) <= 1.01 * el + abs(wl) * 2.0 ** -23).all()), (loss.cpu() - wl, el)
    if grad is not None:
        if grad.dtype == torch.float16:
            i8_checks.near(grad.cpu(), wg, eg)
        else:
            assert bool((abs(grad.double().cpu() - wg) <= 1.01 * eg + abs(wg) * 2.0 ** -23).all())


def case(torch, T, V, k, kind, seed=0, spread=2.0):
    rng = np.random.default_rng(seed + V)
    z = torch.from_numpy((rng.standard_normal((T, V)) * spread).astype(np.float32)).to(kind)
    index = torch.from_numpy(rng.integers(0, V, size=(T, k)).astype(np.int32))       # (some stand twice where k is not small beside V)
    index[torch.from_numpy(rng.random((T, k)) < 0.15)] = -1
    top = torch.from_numpy((rng.standard_normal((T, k)) * 3).astype(np.float32)).to(kind)
    labels = torch.from_numpy(rng.integers(0, V, size=T).astype(np.int32))
    if k:
        labels[0] = int(index[0, 0]) if int(index[0, 0]) >= 0 else 0     # a label that the teacher names too
    if T > 2:
        index[1], labels[1] = -1, -100        # neither
        index[2] = -1                         # no teacher
    if T > 4:
        labels[3] = V                         # no label: outside
        index[4, :] = V + 5 if k else -1
    weight = torch.from_numpy((rng.uniform(0.2, 3, size=T) * (64 if kind is torch.float16 else 1)).astype(np.float32))
    return z, index, top, labels, weight


SIZES = [(1, 1, 1), (2, 2, 3), (5, 7, 4), (6, 8, 0), (3, 9, 1), (6, 15, 17), (4, 511, 5), (5, 1000, 64), (3, 4103, 16), (3, 8191, 1024), (2, 32000, 16), (2, 50001, 50),
         (1, 131072, 7), (1, 200003, 3)]


@pytest.mark.parametrize("wide", [False, True], ids=["fp16", "fp32"])
@pytest.mark.parametrize("u,soft,hard", [(1.0, 1.0, 0.0), (1.0, 0.7, 0.3), (2.0, 1.0, 0.5), (0.5, 0.0, 1.0), (4.0, 1.0, 0.0)])
@pytest.mark.parametrize("T,V,k", SIZES)
def test_loss_and_gradient(torch, T, V, k, u, soft, hard, wide):
    kind = torch.float32 if wide else torch.float16
    z, index, top, labels, weight = case(torch, T, V, k, kind)
    want = reference(torch, z, index, top, labels, u, soft, hard, weight)
    mem = i8_checks.Memory(torch)
    shift = V % 3
    dz, di, dt, dl, dw = mem.input(z, shift), mem.input(index) if k else None, mem.input(top, shift) if k else None, mem.input(labels), mem.input(weight)
    w = binding.Teacher(di.data_ptr() if k else None, dt.data_ptr() if k else None, dl.data_ptr(), k, u, soft, hard)
    import ctypes
    lib, st = binding.load_library(), torch.cuda.current_stream().cuda_stream
    loss, grad = mem.output((T,), torch.float32), mem.output((T, V), kind, (shift + 1) % 4)
    assert lib.lordba_distill(dz.data_ptr(), int(wide), ctypes.byref(w), dw.data_ptr(), loss.data_ptr(), None, grad.data_ptr(), T, V, st) == 0
    check(torch, loss, grad, want)
    loss2, kept, grad2 = mem.output((T,), torch.float32), mem.output((T, 3), torch.float32), mem.output((T, V), kind, shift)
    assert lib.lordba_distill(dz.data_ptr(), int(wide), ctypes.byref(w), None, loss2.data_ptr(), kept.data_ptr(), None, T, V, st) == 0
    assert lib.lordba_distill_backward(dw.data_ptr(), dz.data_ptr(), int(wide), kept.data_ptr(), ctypes.byref(w), grad2.data_ptr(), T, V, st) == 0
    check(torch, loss2, grad2, want)
    mem.unchanged()
    inplace = z.cuda()
    args = (index.cuda(), top.cuda()) if k else (None, None)
    loss3, grad3 = binding.lordba_distill(inplace, *args, labels.cuda(), u, soft, hard, weight.cuda(), d_logits_out=inplace)
    assert grad3.data_ptr() == inplace.data_ptr()
    check(torch, loss3, grad3, want)


@pytest.mark.parametrize("wide", [False, True], ids=["fp16", "fp32"])
def test_infinities_and_empty_rows(torch, wide):
    kind, inf, nan = (torch.float32 if wide else torch.float16), float("inf"), float("nan")
    V, k = 300, 4
    z, index, top, labels, weight = case(torch, 8, V, k, kind, seed=3)
    index[:] = torch.arange(8 * k).view(8, k).int()
    labels[:] = 200
    z[0, 100:150] = -inf                      # masked vocabulary
    z[1, :] = nan; index[1], labels[1] = -1, -100       # a token without teacher and label: what its logits hold does not matter
    z[2, 7] = nan
    z[3, :] = -inf
    z[4, 9] = inf
    top[5, 0] = -inf                          # an entry of probability 0: not there
    top[6, 1] = nan
    z[7, :] = 60000.0 if not wide else 3e38   # the ends of the range
    z[7, 5] = -60000.0 if not wide else -3e38
    loss, grad = binding.lordba_distill(z.cuda(), index.cuda(), top.cuda(), labels.cuda(), 2.0, 1.0, 0.5, weight.cuda())
    kept_loss, kept = binding.lordba_distill(z.cuda(), index.cuda(), top.cuda(), labels.cuda(), 2.0, 1.0, 0.5)
    grad2 = binding.lordba_distill_backward(weight.cuda(), z.cuda(), kept, index.cuda(), top.cuda(), labels.cuda(), 2.0, 1.0, 0.5)
    good = [0, 5]
    want = reference(torch, z[good], index[good], top[good], labels[good], 2.0, 1.0, 0.5, weight[good])
    check(torch, loss[good], grad[good], want)
    check(torch, kept_loss[good], grad2[good], want)
    for g in (grad, grad2):
        assert bool((g[0, 100:150] == 0).all())
        assert bool((g[1] == 0).all())
        assert bool(torch.isnan(g[[2, 3, 4]]).all())
        assert torch.isnan(g[6]).cpu().nonzero()[:, 0].tolist() == index[6].tolist()
        assert bool(torch.isfinite(g[7]).all())
    assert float(loss[1]) == 0 and bool(torch.isnan(loss[[2, 3, 4, 6]]).all()) and torch.equal(loss.isnan(), kept_loss.isnan())
    # an entry that the student holds impossible: infinitely much is lost, its gradient is what the teacher wants
    z[0, 0] = -inf
    loss, grad = binding.lordba_distill(z[:1].contiguous().cuda(), index[:1].cuda(), top[:1].cuda(), None, 1.0, d_loss=weight[:1].cuda())
    assert float(loss) == inf and bool(torch.isfinite(grad).all()) and float(grad[0, 0]) < 0


def test_more_tokens_than_one_launch_takes(torch):
    T, V = (1 << 24) + 1000, 3
    z = torch.randn(T, V, device="cuda", generator=torch.Generator("cuda").manual_seed(3))
    index = (torch.arange(T, device="cuda", dtype=torch.int32) % V)[:, None].contiguous()
    loss, grad = binding.lordba_distill(z, index, torch.zeros(T, 1, device="cuda"), d_loss=torch.ones(T, device="cuda"))
    log_q = torch.log_softmax(z.double(), 1)
    want = -log_q.gather(1, index.long())[:, 0]      # (one entry: p = 1)
    A = (z.amax(1) - z.amin(1)).double() + np.log(V)
    assert bool((abs(loss - want) <= 1.01 * (rel(V, A) + want * (rel(V, A) + 2.0 ** -21)) + want * 2.0 ** -23).all())
    want = log_q.exp()
    err = want * (rel(V, A) + 2.0 ** -21)[:, None]
    want.scatter_add_(1, index.long(), -torch.ones(T, 1, dtype=torch.float64, device="cuda"))
    err.scatter_add_(1, index.long(), (rel(1024, A) + 2.0 ** -21)[:, None])
    assert bool((abs(grad - want) <= 1.01 * err + abs(want) * 2.0 ** -23).all())


def test_differences(torch):
    # central differences of the loss: off by h^2 / 6 times the third derivative (for each term at most 1 / u^3 of its factor u^2, 1) and by the loss's error / h
    V, k, u, soft, hard, h = 40, 6, 2.0, 1.0, 0.5, 2.0 ** -5
    z, index, top, labels, _ = case(torch, 1, V, k, torch.float32, seed=9)
    rest = index.cuda(), top.cuda(), labels.cuda(), u, soft, hard
    loss, grad = binding.lordba_distill(z.cuda(), *rest, torch.ones(1, device="cuda"))
    up, _ = binding.lordba_distill((z + h * torch.eye(V)).cuda(), *(t.expand(V, *t.shape[1:]).contiguous() for t in rest[:3]), u, soft, hard)
    down, _ = binding.lordba_distill((z - h * torch.eye(V)).cuda(), *(t.expand(V, *t.shape[1:]).contiguous() for t in rest[:3]), u, soft, hard)
    el = float(reference(torch, z, index, top, labels, u, soft, hard, torch.ones(1))[2])
    assert float(((up - down) / (2 * h) - grad[0]).abs().max()) <= h * h / 6 * (soft / u + hard) + 2.0 * el / h


@pytest.mark.parametrize("V", [1001, 32000])
def test_streams_graphs_and_repetition(torch, V):
    z, index, top, labels, weight = (t.cuda() for t in case(torch, 37, V, 12, torch.float16))
    call = lambda **kw: binding.lordba_distill(z, index, top, labels, 2.0, 1.0, 0.5, weight, **kw)
    want = [t.clone() for t in call()]
    assert all(torch.equal(a, b) for a, b in zip(call(), want))       # bit for bit
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = call(stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))

    def both():
        loss, kept = binding.lordba_distill(z, index, top, labels, 2.0, 1.0, 0.5)
        return [loss, binding.lordba_distill_backward(weight, z, kept, index, top, labels, 2.0, 1.0, 0.5), *call()]

    both()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    for k in range(4):
        z.copy_(torch.randn_like(z))
        graph.replay()
        torch.cuda.synchronize()
        again = both()
        assert all(torch.equal(a, b) for a, b in zip(out, again)), k


def test_plain_and_other_ways_agree(torch, monkeypatch):
    z, index, top, labels, weight = (t.cuda() for t in case(torch, 6, 100, 4, torch.float32))
    loss, kept = binding.lordba_distill(z, index, top, labels, 2.0, 1.0, 0.5)
    calls = [lambda: binding.lordba_distill(z, index, top, labels, 2.0, 1, 0.5, weight), lambda: binding.lordba_distill(z, index, top),
             lambda: binding.lordba_distill(z, labels=labels, hard=1.0), lambda: binding.lordba_distill(z.half(), index, top.half(), d_loss=weight),
             lambda: (binding.lordba_distill_backward(weight, z, kept, index, top, labels, 2.0, 1.0, 0.5),)]
    bad = [lambda: binding.lordba_distill(z, index), lambda: binding.lordba_distill(z, index.long(), top), lambda: binding.lordba_distill(z, index, top.half()),
           lambda: binding.lordba_distill(z, index[:3].contiguous(), top), lambda: binding.lordba_distill(z, index, top, labels[:2]),
           lambda: binding.lordba_distill(z, index, top, d_logits_out=z), lambda: binding.lordba_distill(z, index, top, d_loss=weight[:2]),
           lambda: binding.lordba_distill(z.t(), index, top), lambda: binding.lordba_distill(z[0], index, top), lambda: binding.lordba_distill(z.double(), index, top),
           lambda: binding.lordba_distill_backward(weight, z, kept[:, 0].contiguous(), index, top), lambda: binding.lordba_distill(z.cpu(), index, top)]
    real, taken, both = binding._plain_call, [], []
    for plain in (True, False):
        monkeypatch.setattr(binding, "_plain_call", lambda *a: (lambda r: (taken.append(r is not None), r)[1])(real(*a)) if plain else None)
        both.append([c() for c in calls])
        for call in bad:
            with pytest.raises((TypeError, ValueError)):
                call()
    assert taken[:len(calls)] == [True] * len(calls)
    assert all(torch.equal(a, b) for u, v in zip(*both) for a, b in zip(u, v))
    for kw in ({"temperature": 0.0}, {"temperature": float("nan")}, {"soft": float("inf")}):
        with pytest.raises(binding.LordbaError):
            binding.lordba_distill(z, index, top, **kw)
