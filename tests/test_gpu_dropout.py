"""Dropout against Philox4x32-10 written out in numpy: which elements are kept, exactly; what they become, to the roundings."""
import numpy as np
import pytest

from paper_2605_24058_amd import binding


def philox(counter, key):
    """counter: [n, 4], key: two words; the published generator's ten rounds"""
    m = np.uint64(0xFFFFFFFF)
    c = [counter[:, i].astype(np.uint64) for i in range(4)]
    k = [np.uint64(key[0]), np.uint64(key[1])]
    for _ in range(10):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> np.uint64(32)) ^ c[1] ^ k[0], q & m, (p >> np.uint64(32)) ^ c[3] ^ k[1], p & m]
        k = [(k[0] + np.uint64(0x9E3779B9)) & m, (k[1] + np.uint64(0xBB67AE85)) & m]
    return np.stack(c, axis=1).astype(np.uint32)


def test_the_generator_gives_the_published_vectors():
    # known answers that are published with the generator
    f = 0xFFFFFFFF
    for counter, key, want in (([0] * 4, (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
                               ([f] * 4, (f, f), (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
                               ([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))):
        assert tuple(philox(np.array([counter], dtype=np.uint64), key)[0]) == want


def draws(start, n, seed, offset):
    """the draws of elements start .. start + n - 1 (start a multiple of 8)"""
    g = np.arange(start // 8, (start + n + 7) // 8, dtype=np.uint64)
    w = np.uint64(0xFFFFFFFF)
    c = np.stack([g & w, g >> np.uint64(32), np.full_like(g, offset & 0xFFFFFFFF), np.full_like(g, offset >> 32)], axis=1)
    return philox(c, (seed & 0xFFFFFFFF, seed >> 32)).reshape(-1).view(np.uint16)[:n]


def kept(n, p, seed, offset):
    least = int(np.rint(p * 65536))
    return draws(0, n, seed, offset) >= least, (65536 / (65536 - least) if least < 65536 else 0.0)


@pytest.fixture(scope="module")
def torch():
    import torch
    binding.load_library()
    return torch


def shifted(torch, a, shift):
    big = torch.full((a.size + 32,), float("nan"), dtype=torch.float16, device="cuda")
    v = big[8 + shift:8 + shift + a.size].view(a.shape)
    v.copy_(torch.from_numpy(a))
    return v


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 7, 8, 9, 255, 2047, 2048, 2049, 100003])
@pytest.mark.parametrize("p", [0.0, 1e-5, 0.05, 0.1, 0.5, 0.999, 1.0])
def test_mask_and_values(torch, n, p):
    rng = np.random.default_rng(n)
    seed, offset = 0x123456789ABCDEF1, 0xFEDCBA9876543210
    keep, factor = kept(n, p, seed, offset)
    for shift in (0, 1):
        ones = shifted(torch, np.ones(n, np.float16), shift)
        y = binding.lordba_dropout(ones, p, seed, offset, y_out=shifted(torch, np.ones(n, np.float16), 2 * shift)).cpu().numpy()
        assert np.array_equal(y != 0, keep & (p < 1))
        x, b = rng.standard_normal(n).astype(np.float16), rng.standard_normal(n).astype(np.float16)
        for base in (None, b):
            got = binding.lordba_dropout(shifted(torch, x, shift), p, seed, offset, y_base=None if base is None else shifted(torch, base, 3 * shift)).cpu().numpy()
            part = np.where(keep, x.astype(np.float64) * factor, 0)
            want = part + (0 if base is None else base.astype(np.float64))
            # fp32: the factor, the product and the sum are rounded (3 * 2^-24 of the parts), then fp16
            with np.errstate(over="ignore"):
                limit = np.abs(want) * 2.0 ** -11 + (np.abs(part) + np.abs(want)) * 2.0 ** -22 + 2.0 ** -25
            big = np.abs(want) > 65504
            assert np.all(np.abs(got.astype(np.float64) - want)[~big] <= limit[~big]) and np.all(np.isinf(got[big]))


@pytest.mark.gpu
def test_what_is_dropped_may_be_anything(torch):
    n, p = 5000, 0.3
    keep, _ = kept(n, p, 5, 6)
    x = np.where(np.arange(n) % 2, np.nan, np.inf).astype(np.float16)
    y = binding.lordba_dropout(torch.from_numpy(x).cuda(), p, 5, 6).cpu().numpy()
    assert np.all(y[~keep] == 0) and not np.isfinite(y[keep]).any()


@pytest.mark.gpu
def test_seeds_and_offsets(torch):
    x = torch.ones(64, 100, dtype=torch.float16, device="cuda")
    a = binding.lordba_dropout(x, 0.5, 1, 2)
    assert torch.equal(a, binding.lordba_dropout(x, 0.5, 1, 2))
    for seed, offset in ((2, 2), (1, 3), (1 + (1 << 32), 2), (1, 2 + (1 << 32))):
        assert not torch.equal(a, binding.lordba_dropout(x, 0.5, seed, offset))
    # the mask of an element does not depend on the shape around it
    assert torch.equal(a.view(-1)[:1000], binding.lordba_dropout(x.view(-1)[:1000], 0.5, 1, 2))
    # (1, 2 + (1 << 32)) as the host's part and the device's
    dev = torch.tensor([(1 << 32) - 5], device="cuda")
    assert torch.equal(binding.lordba_dropout(x, 0.5, 1, 7, offset_dev=dev), binding.lordba_dropout(x, 0.5, 1, 2 + (1 << 32)))


@pytest.mark.gpu
def test_the_backward_pass_is_the_forward_pass_on_the_gradient(torch):
    # y is linear in x with the same mask: sum(g y(x)) = sum(y(g) x), here in numbers that no rounding touches
    rng = np.random.default_rng(2)
    x, g = (torch.from_numpy(rng.integers(-8, 9, size=(37, 111)).astype(np.float16)).cuda() for _ in range(2))
    y, dx = binding.lordba_dropout(x, 0.5, 9, 4), binding.lordba_dropout(g, 0.5, 9, 4)
    assert (y.double() * g.double()).sum().item() == (dx.double() * x.double()).sum().item()
    base = torch.from_numpy(rng.integers(-8, 9, size=(37, 111)).astype(np.float16)).cuda()
    assert torch.equal(binding.lordba_dropout(g, 0.5, 9, 4, y_base=base), dx + base)
    # in place on either operand
    want = dx + base
    g2, b2 = g.clone(), base.clone()
    assert binding.lordba_dropout(g2, 0.5, 9, 4, y_base=base, y_out=g2) is g2 and torch.equal(g2, want)
    assert binding.lordba_dropout(g, 0.5, 9, 4, y_base=b2, y_out=b2) is b2 and torch.equal(b2, want)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [(1 << 32) + 4104, (1 << 34) + 4104], ids=["2^32", "2^34"])   # (the second takes two launches)
def test_more_than_32_bits_of_elements(torch, n):
    p, seed = 0.25, 77
    x = torch.ones(n, dtype=torch.float16, device="cuda")
    y = binding.lordba_dropout(x, p, seed, 3, y_out=x)
    for start in (0, (1 << 31) - 64, (1 << 32) - 64, (1 << 32) + 4000, (n - 4104) - 64, n - 104):
        m = min(128, n - start)
        got = y[start:start + m].cpu().numpy()
        assert np.array_equal(got != 0, draws(start, m, seed, 3) >= 16384)
    share = sum(float((part != 0).sum()) for part in y.split(1 << 31)) / n
    assert abs(share - 0.75) <= 6 * np.sqrt(0.75 * 0.25 / n)
    assert binding.lordba_dropout(x[:0], p, seed).numel() == 0


@pytest.mark.gpu
def test_streams_and_graphs(torch):
    x = torch.randn(3000, device="cuda").half()
    want = binding.lordba_dropout(x, 0.1, 4, 1)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        got = binding.lordba_dropout(x, 0.1, 4, 1, stream=stream)
        side.synchronize()
        assert torch.equal(got, want)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = binding.lordba_dropout(x, 0.1, 4, 1, offset_dev=step)
    for k in (1, 0, 7, 2):
        step.fill_(k)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, binding.lordba_dropout(x, 0.1, 4, 1 + k))


@pytest.mark.gpu
def test_refusals(torch):
    x = torch.zeros(4, 6, dtype=torch.float16, device="cuda")
    for call in (lambda: binding.lordba_dropout(x.float(), 0.1, 1), lambda: binding.lordba_dropout(x.cpu(), 0.1, 1), lambda: binding.lordba_dropout(x.t(), 0.1, 1),
                 lambda: binding.lordba_dropout(x, 0.1, 1, y_base=x.float()), lambda: binding.lordba_dropout(x, 0.1, 1, offset_dev=x)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: binding.lordba_dropout(x, 0.1, -1), lambda: binding.lordba_dropout(x, 0.1, 1, 1 << 64), lambda: binding.lordba_dropout(x, 0.1, 1, y_base=x[:2]),
                 lambda: binding.lordba_dropout(x, 0.1, 1, offset_dev=torch.zeros(2, dtype=torch.int64, device="cuda"))):
        with pytest.raises(ValueError):
            call()
    for p in (-0.1, 1.5, float("nan")):
        with pytest.raises(binding.LordbaError):
            binding.lordba_dropout(x, p, 1)
