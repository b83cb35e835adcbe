"""The exact products of i4_exact tell a result from what is nearly one: on the CPU, with the sums themselves."""
import torch

import i4_exact


def made(k):
    gen = torch.Generator().manual_seed(k)
    x, (codes, scale, zero) = i4_exact.acts(torch, gen, 3, k), i4_exact.weights(torch, gen, 24, k, 128)
    return x.double(), i4_exact.real(torch, codes, scale, zero, 128)


def test_a_lost_a_doubled_and_a_moved_column_show():
    k = (1 << 20) + 8
    x, W = made(k)
    y = x @ W.t()
    got = y.half()
    assert i4_exact.same(got, y)
    assert float((x.abs() @ W.abs().t()).max()) < 2.0 ** 23 and float(y.abs().median()) < 1024     # (halves: exact in fp32 whatever the order)
    assert not i4_exact.same(torch.zeros_like(got), y) and not i4_exact.same(-got, y)
    at = i4_exact.columns(k)
    for c in at[:20] + at[len(at) // 2:len(at) // 2 + 20] + at[-40:]:
        part = torch.outer(x[:, c], W[:, c])
        assert not i4_exact.same((y - part).half(), y) and not i4_exact.same((y + part).half(), y), c
        moved = torch.outer(x[:, c], W[:, c - 1 if c else 1])
        assert not i4_exact.same((y - part + moved).half(), y), c


def test_every_refill_is_covered():
    # a workgroup for few tokens holds up to 85 blocks of three tokens in LDS: every such span has one of the columns
    k = (1 << 22) + 1
    blocks = sorted({c // 128 for c in i4_exact.columns(k)})
    assert max(b - a for a, b in zip(blocks, blocks[1:])) <= 61


def test_the_product_in_parts_is_the_product():
    k = (1 << 17) * 2 + 77
    gen = torch.Generator().manual_seed(1)
    x, (codes, scale, zero) = i4_exact.acts(torch, gen, 2, k), i4_exact.weights(torch, gen, 5, k, 64)
    assert torch.equal(i4_exact.product(torch, x, codes, scale, zero, 64), x.double() @ i4_exact.real(torch, codes, scale, zero, 64).t())
    codes, scale, zero = i4_exact.weights(torch, gen, k, 5, 64)
    assert torch.equal(i4_exact.product(torch, x, codes, scale, zero, 64, back=True), x.double() @ i4_exact.real(torch, codes, scale, zero, 64))
