"""That the loss against a teacher and its gradient take every entry of a row once, wherever the row starts and however long it is: rows of equal logits, whose sums are their
entries' number, and rows in which one entry outweighs all others."""
import ctypes

import numpy as np
import pytest

import i8_checks
from paper_2605_24058_amd import binding

pytestmark = pytest.mark.gpu
# shorter than a 16-byte piece, around one, around what 64, 256, 512 and 1024 threads hold in fp16 and in fp32, rows that they read in turns
LENGTHS = [1, 3, 9, 17, 513, 1023, 1027, 1028, 2047, 2055, 2056, 4099, 4100, 8191, 8199, 8200, 16387, 16388, 32771, 32775, 32776, 50001, 65543, 65544, 131072, 200003]


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    return torch


def threads(V, pieces_of, step):
    """As in csrc/lordba_distill.hip: the workgroup of a row, and the pieces that a turn of it takes"""
    pieces = V // pieces_of
    for most, n, short in ((256, 64, True), (1024, 256, True), (4096, 512 if step else 256, step), (8192, 1024 if step else 512, step)):
        if pieces <= most:
            return n, n if short else 4 * n
    return 1024, 4096


def run(torch, mem, z, index, top, labels, u, soft, hard, weight, shift, step):
    """(loss, kept or None, gradient) in one pass or two, on guarded memory"""
    wide, (T, V) = z.dtype == torch.float32, z.shape
    dz, di, dt, dl, dw = mem.input(z, shift), mem.input(index), mem.input(top), mem.input(labels), mem.input(weight)
    teacher = ctypes.byref(binding.Teacher(di.data_ptr(), dt.data_ptr(), dl.data_ptr(), index.shape[1], u, soft, hard))
    loss, grad = mem.output((T,), torch.float32), mem.output((T, V), z.dtype, shift)
    lib, st = binding.load_library(), torch.cuda.current_stream().cuda_stream
    if step:
        assert lib.lordba_distill(dz.data_ptr(), int(wide), teacher, dw.data_ptr(), loss.data_ptr(), None, grad.data_ptr(), T, V, st) == 0
        kept = None
    else:
        kept = mem.output((T, 3), torch.float32)
        assert lib.lordba_distill(dz.data_ptr(), int(wide), teacher, None, loss.data_ptr(), kept.data_ptr(), None, T, V, st) == 0
        assert lib.lordba_distill_backward(dw.data_ptr(), dz.data_ptr(), int(wide), kept.data_ptr(), teacher, grad.data_ptr(), T, V, st) == 0
    mem.unchanged()
    return loss.double().cpu(), None if kept is None else kept.double().cpu(), grad.double().cpu()


@pytest.mark.parametrize("kind,shift", [("float16", s) for s in range(8)] + [("float32", s) for s in range(4)])
@pytest.mark.parametrize("V", LENGTHS)
def test_equal_logits_are_counted(torch, V, kind, shift):
    # exp(z - m) is 1: sums of ones are exact below 2^24, and so the kept sums are the numbers of entries, those of -infinity left out
    rng, T, kind = np.random.default_rng(V + shift), 9, getattr(torch, kind)
    z = np.full((T, V), 1.5, np.float32)
    for t in range(0, T, 2):
        z[t, rng.random(V) < (0.3, 0.9)[t % 4 // 2]] = -np.inf
    label = rng.integers(0, V, size=T).astype(np.int32)
    z[np.arange(T), label] = 1.5
    n = torch.from_numpy((z > -np.inf).sum(axis=1)).double()
    args = torch.from_numpy(z).to(kind), torch.from_numpy(label[:, None].copy()), torch.zeros(T, 1, dtype=kind), torch.from_numpy(label)
    weight = torch.full((T,), 1.0)
    mem = i8_checks.Memory(torch)
    for u, soft, hard in ((1.0, 1.0, 0.0), (2.0, 0.5, 0.25), (4.0, 0.0, 1.0)):
        for step in (False, True):
            loss, kept, grad = run(torch, mem, *args, u, soft, hard, weight, shift, step)
            if kept is not None:
                assert bool((kept[:, 0] == 1.5).all()) and torch.equal(kept[:, 1], n) and torch.equal(kept[:, 2], n), (u, step)
            # loss: soft u^2 log n + hard log n; the logarithm to 2^-23, four roundings
            want = (soft * u * u + hard) * torch.log(n)
            assert bool((abs(loss - want) <= want * 6 * 2.0 ** -24).all()), (u, step, loss, want)
            # gradient: (soft u + hard) / n, less soft u + hard at the label.  (a quotient, a product with it, the factor, for both terms, and their sum; the exponential of 0 is 1)
            factor = soft * u + hard
            want = torch.where(torch.from_numpy(z) > -np.inf, factor / n[:, None], 0.0).double()
            want[torch.arange(T), torch.from_numpy(label).long()] -= factor
            err = want.abs() * 8 * 2.0 ** -24
            err[torch.arange(T), torch.from_numpy(label).long()] += factor * 4 * 2.0 ** -24
            if kind is torch.float16:
                i8_checks.near(grad, want, err)
            else:
                assert bool((abs(grad - want) <= err + 2.0 ** -149).all()), (u, step)


def edges(V, head, pieces_of, n, turn):
    """Entries where a way through the row begins or ends: the row, its aligned pieces, turns of the workgroup"""
    last = head + (V - head) // pieces_of * pieces_of
    at = {0, head - 1, head, head + pieces_of - 1, last - 1, last, V - 1, last - pieces_of}
    for turns in {1, 2, 3, 4, (V - head) // pieces_of // turn}:
        for d in (-1, 0):
            at |= {head + turns * turn * pieces_of + d, head + turns * n * pieces_of + d}
    return sorted(e for e in at if 0 <= e < V)


@pytest.mark.parametrize("step", [False, True], ids=["two passes", "one pass"])
@pytest.mark.parametrize("kind,shift", [("float16", s) for s in (0, 1, 4, 7)] + [("float32", s) for s in (0, 1, 3)])
@pytest.mark.parametrize("V", LENGTHS[2:])
def test_one_entry_outweighs_all(torch, V, kind, shift, step):
    rng, kind = np.random.default_rng(V + shift), getattr(torch, kind)
    item = torch.empty(0, dtype=kind).element_size()
    N = 16 // item
    n, turn = threads(V, N, step)
    T = len(edges(V, 0, N, n, turn)) + 2
    z = rng.standard_normal((T, V)).astype(np.float32)
    for t in range(T):
        at = edges(V, min(V, -(shift + t * V) % N), N, n, turn)
        z[t, at[t % len(at)]] = 40       # e^40 against 2e5 e^0.5: all but 1e-12; at twice the temperature all but 1e-3
    index = torch.from_numpy(rng.integers(0, V, size=(T, 1)).astype(np.int32))
    labels = torch.from_numpy(rng.integers(0, V, size=T).astype(np.int32))
    z = torch.from_numpy(z).to(kind)
    weight, u, soft, hard = torch.full((T,), 1.0), 2.0, 0.5, 0.25
    loss, _, grad = run(torch, i8_checks.Memory(torch), z, index, torch.zeros(T, 1, dtype=kind), labels, u, soft, hard, weight, shift, step)
    log_q, log_r = torch.log_softmax(z.double() / u, dim=1), torch.log_softmax(z.double(), dim=1)
    i, c = index.long(), labels.long()[:, None]
    want = -soft * u * u * log_q.gather(1, i)[:, 0] - hard * log_r.gather(1, c)[:, 0]
    # a lost or doubled entry is worth 0.7 at least; arguments up to 50 are off by 4 roundings, so are the logarithms, the sums by one for each of a thread's terms
    rel = 2 * (8 * 50 + V / n + 64) * 2.0 ** -24
    assert bool((abs(loss - want) <= 3 * rel + want.abs() * 2.0 ** -22).all()), (loss, want)
    q, r = log_q.exp(), log_r.exp()
    want = soft * u * q + hard * r
    err = want * rel + 2.0 ** -100
    want.scatter_add_(1, i, torch.full((T, 1), -soft * u, dtype=torch.float64))
    want.scatter_add_(1, c, torch.full((T, 1), -hard, dtype=torch.float64))
    err.scatter_add_(1, i, torch.full((T, 1), 2.0 ** -21, dtype=torch.float64))
    err.scatter_add_(1, c, torch.full((T, 1), 2.0 ** -21, dtype=torch.float64))
    if kind is torch.float16:
        i8_checks.near(grad, want, err)
    else:
        assert bool((abs(grad - want) <= err + want.abs() * 2.0 ** -23).all())
