"""A workspace of the 8-bit calls that is sized for the longest batch of a program serves every shorter one: accepted (no GPU), with the same results (GPU)."""
import numpy as np
import pytest

import i8_checks as c
import i8_shapes as shapes
from paper_2605_24058_amd import binding
from test_i8_host import BUF, NO_DEVICE, WORKSPACE, gated, linear


@pytest.mark.parametrize("longest,digits", [(513, 1), (600, 1), (300, 2), (257, 2), (4096, 1)])
def test_a_workspace_for_the_longest_batch_is_accepted_for_shorter_ones(longest, digits):
    import torch

    if torch.cuda.is_available():
        pytest.skip("the addresses are not memory")
    lib = binding.load_library()
    far = dict(x=1 << 40, W=2 << 40, s=3 << 40, y=4 << 40, ws=5 << 40)
    for cols in (100, 2048, 4096, 30000):
        n = binding.lordba_i8_workspace_bytes(longest, cols, digits)
        for T in sorted({1, 5, 64, 255, 256, 257, 300, 511, 512, 513, 600, longest} & set(range(longest + 1))):
            for d in range(1, digits + 1):
                for k in (cols, 1 + cols // 2):
                    kw = dict(far, n=n, T=T, digits=d)
                    assert linear(lib, "lordba_linear_i8", d_in=k, d_out=60, **kw) == NO_DEVICE, (T, k, d)
                    assert linear(lib, "lordba_linear_i8_backward", d_in=60, d_out=k, **kw) == NO_DEVICE, (T, k, d)
                    kw = dict(a=1 << 40, b=2 << 40, s=3 << 40, c=4 << 40, d=5 << 40, e=6 << 40, ws=7 << 40, n=n, T=T, digits=d)
                    assert gated(lib, "lordba_gated_i8", d_in=k, d_ff=60, **kw) == NO_DEVICE, (T, k, d)
                    assert gated(lib, "lordba_gated_i8_backward", d_in=60, d_ff=k // 2 or 1, **kw) == NO_DEVICE, (T, k, d)
        # what the rows' integers and scales need, it has to have
        assert linear(lib, "lordba_linear_i8", **dict(far, n=longest * binding.lordba_i8_row_bytes(cols) * digits, T=longest, d_in=cols, digits=digits)) == WORKSPACE
    assert linear(lib, "lordba_linear_i8", y=BUF[4] + 64, n=binding.lordba_i8_workspace_bytes(600, 2048), T=64, d_in=2048) == 4   # (y in the rows)


@pytest.mark.gpu
@pytest.mark.parametrize("shape,digits", [(s, d) for (g, d, t), some in shapes.SHARED.items() if not g for s in some[-1:]], ids=str)
def test_the_same_results_without_room_for_shared_sums(shape, digits):
    import torch

    T, cols, n = shape
    rng = np.random.default_rng(T + cols + n)
    W, ws = c.weights(rng, 2 * n, cols)
    w, x = torch.from_numpy(W).cuda(), c.acts(rng, T, cols)
    add = c.acts(rng, 2 * T, n).reshape(2, T, n)
    full = binding.lordba_i8_workspace_bytes(T, cols, digits)
    results = []
    for size in (full, full - 1, binding.lordba_i8_workspace_bytes(512 // digits + 1, cols, digits)):
        if size <= T * binding.lordba_i8_row_bytes(cols) * digits:
            continue     # (so much longer a row than a batch that it has no room for this one)
        mem = c.Memory(torch)
        y, h, kept = mem.output((T, 2 * n), torch.float16), mem.output((T, n), torch.float16), mem.output((2, T, n), torch.float16)
        space = mem.output((size,), torch.uint8)
        args = mem.input(x), mem.input(binding.lordba_layout_i8(w)), mem.input(ws)
        c.call(torch, "lordba_linear_i8", *args, y, space, size, T, cols, 2 * n, digits)
        c.call(torch, "lordba_gated_i8", *args, mem.input(add), h, kept, space, size, T, cols, n, digits)
        mem.unchanged()
        results.append((y, h, kept))
    assert len(results) >= 2
    c.near(results[0][0], *c.product(torch, *c.rows_of(x, None, digits), w, ws))
    for other in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], other))
