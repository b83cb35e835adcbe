"""A feed-forward block (gate, up, down) whose frozen weights are held in 8 or in 4 bits and whose three projections carry LoRDBA adapters:
the library's calls in the order in which a training loop and a serving loop make them.

    python -m paper_2605_24058_amd.adapted_block [--tokens 512] [--d-model 1024] [--d-ff 2752] [--rank 16] [--steps 20] [--bits 4] [--vocab 8192 [--top 16]]

fits the adapters to what the same block answers with stronger branches, prints the loss, then answers as a decode step would.  With --vocab the
answers go through a frozen head on 4-bit weights, and what the adapters learn from are the stronger block's top logits.
"""
from __future__ import annotations

import argparse

import torch

from . import binding as lb


class Adapter:
    """Latent carriers and scales in fp32 (what training keeps), packed carriers and fp16 scales (what the kernels take)."""

    def __init__(self, d_in: int, d_out: int, r: int, generator):
        new = lambda *s: torch.randn(s, generator=generator, device="cuda")
        self.latents = [new(r, d_in) / d_in ** 0.5, new(d_out, r) / r ** 0.5]
        self.scales = [torch.full((d_in,), 1 / d_in ** 0.5, device="cuda"), torch.full((r,), 0.05, device="cuda"), torch.ones(d_out, device="cuda")]
        self.pack()

    def pack(self) -> None:
        self.packed = lb.lordba_pack_latents(*self.latents)          # (A, B, A^T, B^T)
        self.half = [s.half() for s in self.scales]

    def branch(self, x, base):
        """base + branch(x), and the rank-r intermediate for the backward pass"""
        return lb.lordba_forward_save_t(x, *self.packed[:2], *self.half, base)

    def branch_backward(self, x, g, t, dx_base, kappa):
        """The gradients; "dx" is dx_base plus the branch's input gradient."""
        return lb.lordba_backward(x, g, self.packed[0], *self.packed[2:], *self.half, *self.latents, kappa, dx_base=dx_base, t_saved=t)

    def step(self, grads, rate: float) -> None:
        for p, k in zip(self.latents + self.scales, ("d_latentA", "d_latentB", "d_s_in", "d_s_rank", "d_s_out")):
            p -= rate * grads[k] / grads[k].norm().clamp_min(1e-12) * p.norm()     # (normalised: the gradients' sizes differ widely)
        self.pack()


def frozen_in_4_bits(w, group: int = 128, halves: int = 1):
    """fp16 weights as the 4-bit projections take them, and as their input gradients do."""
    plain = lb.lordba_quantize_i4(w, group, zero_points=True)
    return tuple(lb.lordba_layout_i4(*plain, group, halves=halves, transposed=t) for t in (False, True))


class AdaptedBlock:
    """y = down(silu(gate(x)) * up(x)), each projection its frozen 8-bit part plus its adapter's branch."""

    def __init__(self, d_model: int, d_ff: int, r: int, p: float = 0.05, seed: int = 0, bits: int = 8):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.d_model, self.d_ff, self.p, self.seed, self.bits = d_model, d_ff, p, seed, bits
        # the frozen weights, laid out once; the transposed layouts are what the input gradients contract with
        half = lambda n, k: (torch.randn(n, k, generator=gen, device="cuda") / k ** 0.5).half()
        gate_up, down = torch.cat([half(d_ff, d_model), half(d_ff, d_model)]), half(d_model, d_ff)
        if bits == 4:
            self.gate_up, self.gate_up_t = frozen_in_4_bits(gate_up, halves=2)
            self.down, self.down_t = frozen_in_4_bits(down)
        elif bits == 8:
            self.gate_up, self.gate_up_scale = lb.lordba_quantize_rows(gate_up)
            self.down, self.down_scale = lb.lordba_quantize_rows(down)
            self.gate_up_t = lb.lordba_layout_i8(self.gate_up[:, :d_model].contiguous(), transposed=True)
            self.down_t = lb.lordba_layout_i8(self.down[:, :d_ff].contiguous(), transposed=True)
        else:
            raise ValueError("bits must be 8 or 4")
        self.adapters = {name: Adapter(*shape, r, gen) for name, shape in
                         (("gate", (d_model, d_ff)), ("up", (d_model, d_ff)), ("down", (d_ff, d_model)))}

    # the four products with the frozen weights
    def _gated(self, x, addends, save=False):
        if self.bits == 4:
            return lb.lordba_gated_i4(x, self.gate_up, addends=addends, save=save)
        return lb.lordba_gated_i8(x, self.gate_up, self.gate_up_scale, addends=addends, save=save)

    def _gated_backward(self, dh, kept):
        if self.bits == 4:
            return lb.lordba_gated_i4_backward(dh, kept, self.gate_up_t)
        return lb.lordba_gated_i8_backward(dh, kept, self.gate_up_t, self.gate_up_scale)

    def _down(self, h):
        return lb.lordba_linear_i4(h, self.down) if self.bits == 4 else lb.lordba_linear_i8(h, self.down, self.down_scale)

    def _down_backward(self, dy):
        return lb.lordba_linear_i4_backward(dy, self.down_t) if self.bits == 4 else lb.lordba_linear_i8_backward(dy, self.down_t, self.down_scale)

    def serve(self, x):
        """The block in inference: no dropout, nothing kept."""
        zero = x.new_zeros(2, x.shape[0], self.d_ff)
        add = torch.empty_like(zero)
        for k, name in enumerate(("gate", "up")):
            a = self.adapters[name]
            lb.lordba_forward(x, *a.packed[:2], *a.half, zero[k], y_out=add[k])
        h = self._gated(x, add)
        a = self.adapters["down"]
        return lb.lordba_forward(h, *a.packed[:2], *a.half, self._down(h))

    def forward(self, x, step: int):
        """The block in training: the branches see their inputs through dropout.  Returns y and what the backward pass needs (no masks: they follow
        from the seed and the offsets 2 * step and 2 * step + 1)."""
        xd = lb.lordba_dropout(x, self.p, self.seed, 2 * step)
        zero = x.new_zeros(x.shape[0], self.d_ff)
        (gate, t_gate), (up, t_up) = (self.adapters[n].branch(xd, zero) for n in ("gate", "up"))
        h, kept = self._gated(x, torch.stack([gate, up]), save=True)
        hd = lb.lordba_dropout(h, self.p, self.seed, 2 * step + 1)
        y, t_down = self.adapters["down"].branch(hd, self._down(h))
        return y, (xd, hd, kept, t_gate, t_up, t_down, step)

    def backward(self, dy, saved, kappa: float = 100.0):
        """dx and each adapter's gradients."""
        xd, hd, kept, t_gate, t_up, t_down, step = saved
        grads = {"down": self.adapters["down"].branch_backward(hd, dy, t_down, torch.zeros_like(hd), kappa)}
        # the branch's input gradient passes its mask again, and the base path's is added on the way
        dh = lb.lordba_dropout(grads["down"]["dx"], self.p, self.seed, 2 * step + 1, y_base=self._down_backward(dy))
        dx, dgate_up = self._gated_backward(dh, kept)
        grads["gate"] = self.adapters["gate"].branch_backward(xd, dgate_up[0], t_gate, torch.zeros_like(xd), kappa)
        grads["up"] = self.adapters["up"].branch_backward(xd, dgate_up[1], t_up, grads["gate"]["dx"], kappa)     # (both branches have the same input)
        return lb.lordba_dropout(grads["up"]["dx"], self.p, self.seed, 2 * step, y_base=dx), grads


def fit(block: AdaptedBlock, x, target, steps: int, rate: float = 0.02):
    """Gradient descent of the adapters on mean |y - target|^2; the loss of every step."""
    losses = []
    for step in range(steps):
        y, saved = block.forward(x, step)
        miss = y.float() - target
        losses.append(miss.square().mean().item())
        _, grads = block.backward(miss.half(), saved, kappa=2.0)
        for name, adapter in block.adapters.items():
            adapter.step(grads[name], rate)
    return losses


class Head:
    """A frozen projection onto a vocabulary, on 4-bit weights."""

    def __init__(self, vocab: int, d_model: int, seed: int = 1):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.W, self.Wt = frozen_in_4_bits((torch.randn(vocab, d_model, generator=gen, device="cuda") / d_model ** 0.5).half())

    def logits(self, y):
        return lb.lordba_linear_i4(y, self.W)

    def backward(self, d_logits):
        return lb.lordba_linear_i4_backward(d_logits, self.Wt)


def best(logits, k: int):
    """A teacher's k best entries, as lordba_distill takes them."""
    top = torch.topk(logits.float(), k, dim=1)
    return top.indices.int(), top.values.to(logits.dtype)


def distil_step(block: AdaptedBlock, head: Head, x, teacher, step: int, temperature: float = 2.0, kappa: float = 2.0):
    """One pass through block, head and loss and back: the tokens' losses and the adapters' gradients of their mean, times 1024 (entries of the gradient with
    respect to the logits are probabilities over the tokens' number: fp16 holds them so)."""
    y, saved = block.forward(x, step)
    logits = head.logits(y)
    weight = torch.full((x.shape[0],), 1024.0 / x.shape[0], device=x.device)
    loss, d_logits = lb.lordba_distill(logits, *teacher, temperature=temperature, d_loss=weight, d_logits_out=logits)
    return loss, block.backward(head.backward(d_logits), saved, kappa)[1]


def distil(block: AdaptedBlock, head: Head, x, teacher, steps: int, rate: float = 0.02):
    """Gradient descent of the adapters on what the tokens lose against the teacher's top logits (top_index, top_logits); the mean loss of every step."""
    losses = []
    for step in range(steps):
        loss, grads = distil_step(block, head, x, teacher, step)
        losses.append(loss.mean().item())
        for name, adapter in block.adapters.items():
            adapter.step(grads[name], rate)
    return losses


def stronger(block: AdaptedBlock, x, factor: float = 2.0):
    """What the block answers with every branch `factor` times as large."""
    for a in block.adapters.values():
        a.half[1] *= factor
    y = block.serve(x).float()
    for a in block.adapters.values():
        a.pack()
    return y


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("tokens", 512), ("d-model", 1024), ("d-ff", 2752), ("rank", 16), ("steps", 20), ("bits", 8), ("vocab", 0), ("top", 16)):
        p.add_argument("--" + name, type=int, default=value)
    a = p.parse_args()
    block = AdaptedBlock(a.d_model, a.d_ff, a.rank, bits=a.bits)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(a.tokens, a.d_model, generator=gen, device="cuda").half()
    target = stronger(block, x)
    if a.vocab:
        head = Head(a.vocab, a.d_model)
        losses = distil(block, head, x, best(head.logits(target.half()), a.top), a.steps)
    else:
        losses = fit(block, x, target, a.steps)
    for k in range(0, a.steps, max(1, a.steps // 10)):
        print("step %3d  loss %.6f" % (k, losses[k]))
    print("step %3d  loss %.6f" % (a.steps - 1, losses[-1]))
    y = block.serve(x[:1].contiguous())
    if a.vocab:
        print("one token: best entry %d" % int(head.logits(y).argmax()))
    print("one token: |y| = %.4f, finite: %s" % (y.float().norm().item(), bool(torch.isfinite(y).all())))


if __name__ == "__main__":
    main()
