"""What the tests of the 4-bit projections compare with: inputs, and the definitions in 64 bits with the bounds of what the kernels may be off by.

Bounds.  Sums are fp32: a product of two fp16 numbers is exact there, a sum over K columns adds them in steps of 32 or fewer and joins the waves' parts.  With an
error of 2^-23 (a truncation at worst) of the sum of magnitudes for each of K / 32 steps, 32 additions inside one, 16 parts and a few more,
    sums(K) = (K / 32 + 64) * 2^-23 * sum |x| |W|.
With a few tokens a group's scale is multiplied on in fp32: in the same bound.  The result is rounded to fp16 once (near() of i8_checks counts that)."""
import numpy as np

FEW = 64    # tokens up to which the forward products take the weights as they are


def weights(torch, rng, rows, cols, group, zeros, tiny=False):
    """codes uint8 [rows, cols] of every value, scale fp16 [rows, groups] (a few 0 and negative ones), zero uint8 or None, as CPU tensors"""
    groups = -(-cols // group)
    scale = rng.uniform(0.2, 2.0, size=(rows, groups)) / (8 * np.sqrt(cols)) * (1e-5 if tiny else 1)
    scale[rng.random(scale.shape) < 0.02] *= -1
    scale[rng.random(scale.shape) < 0.02] = 0
    codes = torch.from_numpy(rng.integers(0, 16, size=(rows, cols), dtype=np.uint8))
    zero = torch.from_numpy(rng.integers(0, 16, size=scale.shape, dtype=np.uint8)) if zeros else None
    return codes, torch.from_numpy(scale.astype(np.float16)), zero


def real(torch, codes, scale, zero, group, rounded):
    """W in 64 bits; rounded: each weight to fp16, as the products of many tokens and of gradients take it"""
    column = torch.arange(codes.shape[1]) // group
    z = 8.0 if zero is None else zero.double()[:, column]
    W = scale.double()[:, column] * (codes.double() - z)
    return W.half().double() if rounded else W


def product(torch, x, W):
    """x W^T and the bound of the sums' error; 64-bit tensors on the GPU"""
    Wt = W.t().contiguous()
    return torch.mm(x, Wt), torch.mm(x.abs(), Wt.abs()) * ((W.shape[1] / 32 + 64) * 2.0 ** -23)
