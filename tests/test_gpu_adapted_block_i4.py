"""The adapted feed-forward block on 4-bit weights, and its adapters learning from a teacher's top logits through a head on 4-bit weights: against the same block, head and
loss in 64 bits, in a captured graph, and from the command line."""
import subprocess
import sys

import pytest

from paper_2605_24058_amd import binding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    return torch


def weights(torch, W):
    """A laid-out matrix W in 64 bits, by the products themselves: unit rows through the input gradient (each weight rounded to fp16 there: exact to 2^-11)."""
    eye = torch.eye(W.rows, dtype=torch.float16, device="cuda")
    if W.halves == 1:
        return binding.lordba_linear_i4_backward(eye, W).double()
    # (the gated block's: dx of dgate = dh with up = 1 at gate = 0, where sigma = 1/2)
    F = W.rows // 2
    kept = torch.zeros(2, F, F, dtype=torch.float16, device="cuda")
    kept[1] = 2
    gate, _ = binding.lordba_gated_i4_backward(eye[:F, :F].contiguous(), kept, W)
    kept[0], kept[1] = 40, 0       # dgate = 0, dup = dh * 40
    up, _ = binding.lordba_gated_i4_backward(eye[:F, :F].contiguous(), kept, W)
    return torch.cat([gate.double(), up.double() / 40])


def reference(torch, block, x, step, head=None):
    """(y or logits as a function of leaves, the leaves): x and the adapters' scales"""
    def mask(shape, offset):
        return binding.lordba_dropout(torch.ones(shape, dtype=torch.float16, device="cuda"), block.p, block.seed, offset).double()

    leaf = lambda t: t.double().requires_grad_()
    scales = {n: [leaf(s) for s in a.half] for n, a in block.adapters.items()}

    def branch(name, v):
        a = block.adapters[name]
        A, B = (torch.where(l >= 0, 1.0, -1.0).double() for l in a.latents)
        s_in, s_rank, s_out = scales[name]
        return ((v * s_in) @ A.t().contiguous() * s_rank) @ B.t().contiguous() * s_out

    xv = leaf(x)
    xd = xv * mask(x.shape, 2 * step)
    g, u = (xv @ weights(torch, block.gate_up_t).t().contiguous()).chunk(2, dim=1)
    gate, up = g + branch("gate", xd), u + branch("up", xd)
    h = gate * torch.sigmoid(gate) * up
    y = h @ weights(torch, block.down_t).t().contiguous() + branch("down", h * mask(h.shape, 2 * step + 1))
    return (y if head is None else y @ weights(torch, head.Wt).t().contiguous()), xv, scales


def rel(a, b):
    return float((a.double() - b).norm() / b.norm())


@pytest.mark.parametrize("tokens,d_model,d_ff,r", [(96, 256, 512, 16), (33, 129, 301, 5), (5, 200, 320, 8)])
def test_a_step_against_64_bits(torch, tokens, d_model, d_ff, r):
    from paper_2605_24058_amd import adapted_block

    block = adapted_block.AdaptedBlock(d_model, d_ff, r, p=0.1, seed=11, bits=4)
    gen = torch.Generator(device="cuda").manual_seed(2)
    x, dy = (torch.randn(tokens, d_model, generator=gen, device="cuda").half() for _ in range(2))
    y, saved = block.forward(x, 3)
    dx, grads = block.backward(dy, saved)
    want, xv, scales = reference(torch, block, x, 3)
    want.backward(dy.double())
    # fp16 tensors between the calls and fp16 weights on both sides: a dozen roundings of 2^-11 at most, each on part of the sum
    assert rel(y, want.detach()) <= 4e-3 and rel(dx, xv.grad) <= 4e-3
    for name, leaves in scales.items():
        for k, s in zip(("d_s_in", "d_s_rank", "d_s_out"), leaves):
            assert rel(grads[name][k], s.grad) <= 4e-3, (name, k)


@pytest.mark.parametrize("tokens,V", [(64, 1000), (11, 333)])
def test_learning_from_a_teacher_against_64_bits(torch, tokens, V):
    from paper_2605_24058_amd import adapted_block

    block, head = adapted_block.AdaptedBlock(128, 256, 8, p=0.1, seed=5, bits=4), adapted_block.Head(V, 128)
    x = torch.randn(tokens, 128, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").half()
    teacher = adapted_block.best(head.logits(adapted_block.stronger(block, x).half()), 7)
    loss, grads = adapted_block.distil_step(block, head, x, teacher, 1)
    logits, _, scales = reference(torch, block, x, 1, head)
    u = 2.0
    log_q = torch.log_softmax(logits / u, dim=1).gather(1, teacher[0].long())
    log_p = torch.log_softmax(teacher[1].double() / u, dim=1)
    want = u * u * (log_p.exp() * (log_p - log_q)).sum(dim=1)
    (1024 * want.mean()).backward()
    # the logits are off by a few roundings of 2^-11 of their size (some 3 standard deviations here), the losses by as much
    assert float((loss.double() - want.detach()).abs().max()) <= 0.05 and rel(loss, want.detach()) <= 2e-2
    for name, leaves in scales.items():
        for k, s in zip(("d_s_in", "d_s_rank", "d_s_out"), leaves):
            assert rel(grads[name][k], s.grad) <= 1e-2, (name, k)


def test_serving_is_training_without_dropout(torch):
    from paper_2605_24058_amd import adapted_block

    block = adapted_block.AdaptedBlock(256, 320, 8, p=0.0, bits=4)
    x = torch.randn(40, 256, device="cuda").half()
    y, _ = block.forward(x, 0)
    one = torch.cat([block.serve(x[k:k + 1].contiguous()) for k in range(3)])
    # (other kernels for other lengths: weights rounded to fp16 or not, sums in another order)
    assert rel(block.serve(x), y.double()) <= 3e-3 and rel(one, y[:3].double()) <= 3e-3


def test_a_captured_step(torch):
    from paper_2605_24058_amd import adapted_block

    block, head = adapted_block.AdaptedBlock(128, 192, 8, bits=4), adapted_block.Head(515, 128)
    x = torch.randn(50, 128, device="cuda").half()
    teacher = adapted_block.best(head.logits(x), 5)

    def step():
        loss, grads = adapted_block.distil_step(block, head, x, teacher, 2)
        return [loss] + [grads[n][k] for n in grads for k in ("d_latentA", "d_latentB", "d_s_in", "d_s_rank", "d_s_out")]

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(3):
        x.copy_(torch.randn_like(x))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, step())), k


@pytest.mark.parametrize("more", [["--bits", "4"], ["--bits", "8", "--vocab", "600"], ["--bits", "4", "--vocab", "601", "--top", "4"]])
def test_the_command_runs(more):
    out = subprocess.run([sys.executable, "-m", "paper_2605_24058_amd.adapted_block", "--tokens", "40", "--d-model", "128", "--d-ff", "200", "--rank", "4", "--steps", "2"] +
                         more, capture_output=True, text=True, timeout=110)
    assert out.returncode == 0, out.stderr[-2000:]
    assert "step   1  loss" in out.stdout and "finite: True" in out.stdout
