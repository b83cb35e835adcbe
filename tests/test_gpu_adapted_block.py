"""The adapted feed-forward block: its forward and backward pass against the same block in 64 bits, built from the block's own frozen weights, signs and
masks; and that fitting the adapters lowers the loss."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    return torch


def reference(torch, block, x, step, dy):
    """y, dx and the branches' scale gradients by 64-bit autograd.  The carriers are constants here, so are the masks."""
    from paper_2605_24058_amd import binding as lb

    def mask(shape, offset):
        return lb.lordba_dropout(torch.ones(shape, dtype=torch.float16, device="cuda"), block.p, block.seed, offset).double()

    leaf = lambda t: t.double().requires_grad_()
    scales = {n: [leaf(s) for s in a.half] for n, a in block.adapters.items()}

    def branch(name, v):
        a = block.adapters[name]
        A, B = (torch.where(l >= 0, 1.0, -1.0).double() for l in a.latents)
        s_in, s_rank, s_out = scales[name]
        return ((v * s_in) @ A.t().contiguous() * s_rank) @ B.t().contiguous() * s_out

    def rows(q, scale, cols):
        return q[:, :cols].double() * scale.double()[:, None]

    def held_in_8_bits(v):     # the rows' rounding is what the forward pass does; its gradient is taken as that of the identity
        s = v.detach().abs().amax(dim=1, keepdim=True) / 127
        return v + (torch.round(v / s) * s - v).detach()

    Wgu, Wd = rows(block.gate_up, block.gate_up_scale, block.d_model), rows(block.down, block.down_scale, block.d_ff)
    xv = leaf(x)
    xd = xv * mask(x.shape, 2 * step)
    g, u = (held_in_8_bits(xv) @ Wgu.t().contiguous()).chunk(2, dim=1)
    gate, up = g + branch("gate", xd), u + branch("up", xd)
    h = gate * torch.sigmoid(gate) * up
    h = h + (h.detach().half().double() - h.detach())      # (h is an fp16 tensor)
    y = held_in_8_bits(h) @ Wd.t().contiguous() + branch("down", h * mask(h.shape, 2 * step + 1))
    y.backward(dy.double())
    return y.detach(), xv.grad, {n: [s.grad for s in v] for n, v in scales.items()}


@pytest.mark.parametrize("tokens,d_model,d_ff,r", [(96, 256, 512, 16), (33, 129, 301, 5)])
def test_a_step_against_64_bits(torch, tokens, d_model, d_ff, r):
    from paper_2605_24058_amd import adapted_block

    block = adapted_block.AdaptedBlock(d_model, d_ff, r, p=0.1, seed=11)
    gen = torch.Generator(device="cuda").manual_seed(2)
    x, dy = (torch.randn(tokens, d_model, generator=gen, device="cuda").half() for _ in range(2))
    y, saved = block.forward(x, 3)
    dx, grads = block.backward(dy, saved)
    want_y, want_dx, want = reference(torch, block, x, 3, dy)
    rel = lambda a, b: float((a.double() - b).norm() / b.norm())
    # fp16 tensors between the calls (2^-11 each, a handful of them) and the few entries of the second product's rows that fall to the other side of a
    # rounding to 8 bits because h is off by an fp16 rounding: some 2^-11 * 127 / 3 of them, by one step of 1 / 127 of the largest
    assert rel(y, want_y) <= 4e-3
    assert rel(dx, want_dx) <= 4e-3
    for name in want:
        for k, w in zip(("d_s_in", "d_s_rank", "d_s_out"), want[name]):
            assert rel(grads[name][k], w) <= 4e-3, (name, k)


def test_serving_is_training_without_dropout(torch):
    from paper_2605_24058_amd import adapted_block

    block = adapted_block.AdaptedBlock(256, 320, 8, p=0.0)
    x = torch.randn(40, 256, device="cuda").half()
    y, _ = block.forward(x, 0)
    one = torch.cat([block.serve(x[k:k + 1].contiguous()) for k in range(3)])
    full = block.serve(x)
    rel = lambda a, b: float((a.double() - b.double()).norm() / b.double().norm())
    assert rel(full, y) <= 2e-3 and rel(one, y[:3]) <= 2e-3   # (other kernels of the branch for other lengths: sums in another order)


def test_fitting_lowers_the_loss(torch):
    from paper_2605_24058_amd import adapted_block

    block = adapted_block.AdaptedBlock(256, 512, 16)
    x = torch.randn(128, 256, device="cuda").half()
    losses = adapted_block.fit(block, x, adapted_block.stronger(block, x), 12)
    assert all(np.isfinite(losses)) and losses[-1] < losses[0]
