"""Products with 4-bit weights that are exact at any length: activations of -1, 0 and 1, scales that are powers of two, so that every sum is a whole number of halves below 2^23
and rounded once, to fp16.  A column that is lost, read twice or multiplied with another's weight changes a result by a half at least; sums stay mostly below 1024, where fp16 holds that."""


def columns(k, planes=1):
    """Where something begins or ends: the row, blocks of 128 columns (every power of two of them, and a prime apart, so that every place of a loop over some hundred blocks comes by),
    pieces of eight at both ends."""
    at = set(range(min(k, 16))) | {k - 1 - i for i in range(min(k, 16))}
    blocks = -(-k // 128)
    for b in {1 << i for i in range(blocks.bit_length())} | set(range(0, blocks, 61)) | {blocks - 1, blocks - 2}:
        at |= {128 * b - 1, 128 * b, 128 * b + 1}
    at |= {k // 128 * 128 + i for i in (-1, 0, 1, 7, 8, 31, 32)}
    return sorted(c for c in at if 0 <= c < k)


def acts(torch, gen, T, k):
    """fp16 [T, k] on the generator's device: some 1500 entries a row, those of columns() among them"""
    dev = gen.device
    sign = lambda *s: torch.randint(0, 2, s, generator=gen, device=dev).half() * 2 - 1
    x = torch.zeros(T, k, dtype=torch.float16, device=dev)
    for t in range(T):
        some = torch.randint(0, k, (min(k, 700),), generator=gen, device=dev)
        x[t, some] = sign(len(some))
    at = torch.tensor(columns(k), device=dev)
    x[:, at] = sign(T, len(at))
    return x


def weights(torch, gen, rows, cols, group):
    """codes, scale (1/2, 1, a few 0 and -1), zero on the generator's device"""
    dev = gen.device
    groups = -(-cols // group)
    draw = lambda high, *s: torch.randint(0, high, s, generator=gen, device=dev, dtype=torch.uint8)
    kind = draw(16, rows, groups)
    scale = torch.where(kind < 8, 0.5, 1.0).half()
    scale[kind == 15], scale[kind == 14] = -1.0, 0.0
    return draw(16, rows, cols), scale, draw(16, rows, groups)


def real(torch, codes, scale, zero, group, first=0):
    """W in 64 bits, of codes from column `first` of a matrix on"""
    column = torch.arange(first, first + codes.shape[1], device=codes.device) // group
    return scale.double()[:, column] * (codes.double() - zero.double()[:, column])


def product(torch, x, codes, scale, zero, group, back=False):
    """x W^T, or x W, in 64 bits, some columns of the contraction at a time"""
    step, y = 1 << 17, 0.0
    for c in range(0, x.shape[1], step):
        if back:
            W = real(torch, codes[c:c + step], scale[c:c + step], zero[c:c + step], group)
        else:
            W = real(torch, codes[:, c:c + step], scale, zero, group, c).t().contiguous()
        y = y + torch.mm(x[:, c:c + step].double(), W)
    return y


def same(got, want):
    """got, fp16, is the rounded sum: want in 64 bits, exact"""
    return got.shape == want.shape and bool((got == want.half()).all())
