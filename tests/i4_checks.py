"""What the tests of the 4-bit projections compare with: inputs, and the definitions in 64 bits with the bounds of what the kernels may be off by.

Bounds.  Sums are fp32: a product of two fp16 numbers is exact there, a sum over K columns adds them in steps of 32 or fewer and joins the waves' parts.  With an
error of 2^-23 (a truncation at worst) of the sum of magnitudes for each of K / 32 steps, 32 additions inside one, 16 parts and a few more,
    sums(K) = (K / 32 + 64) * 2^-23 * sum |x| |W|.
With the kernel for few tokens a group's scale is multiplied on in fp32: in the same bound.  The result is rounded to fp16 once (near() of i8_checks counts that)."""
import ctypes
import functools
import os
import subprocess
import tempfile

import numpy as np

from paper_2605_24058_amd import binding

KERNELS = ("few", "tile32", "tile64", "tile128", "tile256", "square64")    # (the last: forward, one matrix, aligned rows)
# T, d_in, d_out (d_ff), group, zero points: one token and one column; ends of groups, of blocks of 128 columns, of 32 rows; both sides of the kernels' limits; odd
# widths; rows that start anywhere; tiles of every size whole and with all sizes ragged; contractions of fewer blocks than a workgroup has parts and of many
SHAPES = [(1, 1, 1, 32, True), (1, 128, 32, 128, False), (2, 31, 33, 32, True), (3, 127, 31, 64, False), (8, 129, 65, 128, True), (16, 256, 64, 64, True),
          (17, 257, 95, 32, False), (33, 640, 96, 128, False), (40, 1000, 130, 64, True), (64, 384, 100, 32, True), (64, 2176, 48, 128, True),
          (65, 384, 96, 128, False), (65, 129, 127, 32, True), (127, 1000, 257, 64, True), (128, 256, 128, 128, False), (200, 100, 300, 32, False),
          (333, 392, 1031, 64, False), (513, 130, 515, 128, True), (1030, 264, 4104, 32, True), (2200, 384, 2049, 64, False), (2048, 128, 6144, 128, True),
          (100, 5, 700, 32, True), (70, 7, 3, 64, False), (5, 4, 9, 32, False), (1, 5000, 40, 128, True), (7, 4200, 70, 32, False), (16, 4104, 4200, 64, False),
          (32, 3328, 520, 128, True), (48, 2050, 1001, 64, False), (96, 2048, 1024, 32, True), (256, 1288, 4136, 128, False), (300, 1032, 1032, 32, True),
          (260, 5000, 264, 64, True), (640, 2056, 1536, 64, True), (1500, 520, 2056, 128, False), (1024, 1024, 4096, 32, False), (1100, 4104, 776, 128, True),
          (4100, 264, 520, 64, True), (2500, 1025, 700, 32, True), (40, 4104, 2072, 64, True), (64, 8192, 2048, 32, False), (60, 8200, 2051, 128, True),
          (61, 8264, 1991, 64, False), (3, 300, 8300, 128, True), (8, 1030, 8321, 32, False), (1, 8400, 264, 64, True), (7, 8320, 130, 128, False), (500, 1032, 2048, 32, False),
          (63, 2056, 10001, 64, True), (130, 2112, 4096, 128, False)]


@functools.lru_cache(None)
def _choice():
    """The choice of the kernel (csrc/lordba_i4_choice.h), compiled for the host."""
    with tempfile.TemporaryDirectory() as d:
        with open(os.path.join(d, "choice.cpp"), "w") as f:
            f.write('#include "lordba_i4_choice.h"\nextern "C" int kernel(long long T, long long k, long long b, long long n, int g, int a, int w, int f) '
                    "{ return i4_kernel(T, k, b, n, g != 0, a != 0, w != 0, f != 0); }\n")
        subprocess.run([os.environ.get("CXX", "g++"), "-O1", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-fPIC", "-shared", "-I", binding._CSRC, f.name, "-o",
                        os.path.join(d, "choice.so")], check=True, capture_output=True, timeout=120)
        f = ctypes.CDLL(os.path.join(d, "choice.so")).kernel
    f.restype, f.argtypes = ctypes.c_int, [ctypes.c_longlong] * 4 + [ctypes.c_int] * 4
    return f


def kernel(T, columns, n, planes=1, gated=False, aligned=True, backward=False, fine_zeros=False):
    """Which kernel contracts `planes` planes of `columns` columns with n outputs (gated: of each half)."""
    return KERNELS[_choice()(T, columns, planes * -(-columns // 128), n, gated, aligned and columns % 8 == 0, backward, fine_zeros)]


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
