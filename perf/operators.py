"""Passes through the operators that stand around an adapter branch: the frozen base projection in 8 bits, the gated feed-forward
block on such weights, and dropout of a branch's input.  Kinds of pass ("op"):

  linear       y = x W^T on 8-bit weights: the rows of x are held in 8 bits with a scale each, y in fp16
  linear_grad  the gradient with respect to x of such a projection, dx = g W
  gated        h = silu(x Wg^T + a_g) * (x Wu^T + a_u); with "train" gate and up are returned too, with "addends" the two branch
               outputs a_g and a_u of adapters come in
  gated_grad   from dh and the kept gate and up: the gradients with respect to gate, up and x
  dropout      y = x with elements dropped at probability p, the others scaled; with "base" a tensor is added (the backward pass:
               the base path's gradient plus that of the branch)

Definition of the 8-bit rows: amax = max |x| over the row, q = rint(x * 127 / amax), scale = amax / 127; a row of zeros stays zeros.
Weights are int8 with an fp32 scale per output channel.  The gradients are those of y = x W^T at the weights' exact values.
Definition of the dropout mask: Philox4x32-10 with the counter (element index / 8, offset) in 64 bits each and the seed as the key;
element e of its eight takes 16 bits, (word e / 2 >> 16 (e mod 2)) mod 65536, and is kept if these are at least rint(65536 p); what is kept
is scaled by 65536 / (65536 - rint(65536 p)).
"""
import functools
import math

import numpy as np
import torch

own = False  # True: `run` calls this repository's kernels; False: elementary operations in 32 bits


# ------------------------------------------------------------------------------------------------ cases ----
def _case(op, T, d_in, d_out, train=False, addends=False, base=False, p=0.0, pad=0):
    return dict(op=op, T=T, d_in=d_in, d_out=d_out, train=train, addends=addends, base=base, p=p, pad=pad)


def listed():
    return [
        # One token through one square projection: a decode step's call, where latency counts.
        dict(_case("linear", 1, 4096, 4096), name="linear_decode"),
        # A decode step of 64 sequences through the wide projection.
        dict(_case("linear", 64, 4096, 11008), name="linear_decode_64"),
        # A chunk of a prompt through a head with an odd number of outputs behind an odd number of features, some rows padding.
        dict(_case("linear", 301, 1001, 3001, pad=40), name="linear_odd"),
        # Prefill of 4096 tokens back to the narrow side of a layer.
        dict(_case("linear", 4096, 11008, 4096), name="linear_prefill"),
        # A training step's input gradient of a square projection.
        dict(_case("linear_grad", 2048, 4096, 4096), name="linear_grad_square"),
        # The input gradient of the widest projection on a long batch.
        dict(_case("linear_grad", 8192, 5120, 13824), name="linear_grad_large"),
        # A decode step of eight sequences through the gated block, adapters on both projections.
        dict(_case("gated", 8, 4096, 11008, addends=True), name="gated_decode"),
        # The forward pass of a training step of the block: gate and up are kept for the backward pass.
        dict(_case("gated", 2048, 4096, 11008, train=True, addends=True), name="gated_train"),
        # Its backward pass.
        dict(_case("gated_grad", 2048, 4096, 11008), name="gated_grad"),
        # A short ragged batch of a small block with odd widths, some rows padding.
        dict(_case("gated_grad", 77, 999, 2731, pad=9), name="gated_grad_odd"),
        # Dropout of a branch's input in training.
        dict(_case("dropout", 2048, 4096, 4096, p=0.05), name="dropout"),
        # Its backward pass on a long batch of the widest input, the base path's gradient added.
        dict(_case("dropout", 8192, 13824, 13824, p=0.1, base=True), name="dropout_grad_large"),
    ]


_MOST = 2.0 * 8192 * 5120 * 13824


def draw(rng):
    def size(low, high):
        return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))))

    op = rng.choice(["linear", "linear_grad", "gated", "gated_grad", "dropout"])
    T = size(1, 8192)
    d_in, d_out = size(64, 13824), size(64, 13824)
    while 2.0 * T * d_in * d_out * (2 if op.startswith("gated") else 1) > 0.9 * _MOST:
        T = max(1, T // 2)
    pad = T // 8 if rng.random() < 0.25 else 0
    if op == "dropout":
        return _case(op, T, d_in, d_in, base=rng.random() < 0.5, p=rng.choice([0.05, 0.1, 0.25, 0.5]), pad=pad)
    if op == "gated":
        return _case(op, T, d_in, d_out, train=rng.random() < 0.5, addends=rng.random() < 0.7, pad=pad)
    return _case(op, T, d_in, d_out, pad=pad)


# ----------------------------------------------------------------------------------------------- inputs ----
def _inputs(case, seed):
    """The tensors of a pass from the seed alone.  Activations are N(0, 1) with a few channels eight times as large, as the inputs of
    projections have them; `pad` rows at the end are zeros (padding of a batch).  Weights are N(0, 1 / d) in 8 bits."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    T, d_in, d_out, op = case["T"], case["d_in"], case["d_out"], case["op"]

    def normal(*shape, std=1.0):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * std

    def acts(cols, large=False):
        a = normal(T, cols)
        if large:
            a = a * torch.where(torch.rand(cols, generator=gen, device="cuda") < 0.005, 8.0, 1.0)
        if case["pad"]:
            a[T - case["pad"]:] = 0
        return a.half()

    if op == "dropout":
        s = dict(x=acts(d_in), p=case["p"], seed=int(seed) * 2654435761 % (1 << 62), offset=int(seed) % 1000003 + (1 << 33))
        s["base"] = acts(d_in) if case["base"] else None
        return s
    channels = 2 * d_out if op.startswith("gated") else d_out
    W = normal(channels, d_in, std=1 / math.sqrt(d_in))
    w_scale = (W.abs().amax(dim=1) / 127).contiguous()
    s = dict(W=(W / w_scale[:, None]).round().to(torch.int8), w_scale=w_scale)
    if op in ("linear", "gated"):
        s["x"] = acts(d_in, large=True)
        s["addends"] = torch.stack([acts(d_out), acts(d_out)]) if case["addends"] else None
    if op == "linear_grad":
        s["g"] = acts(d_out)
    if op == "gated_grad":
        s["dh"], s["gate_up"] = acts(d_out), torch.stack([acts(d_out), acts(d_out)])
    return s


def prepare(case, seed):
    s = dict(_inputs(case, seed), op=case["op"], train=case["train"])
    if own and "W" in s:  # the weights as a program keeps them: rows laid out once, transposed for the gradients
        from paper_2605_24058_amd import binding

        s["W"] = binding.lordba_layout_i8(s["W"], transposed=case["op"].endswith("_grad"))
    return s


# -------------------------------------------------------------------------------------------- plain form ----
def _rows_in_8_bits(x):
    x = x.float()
    amax = x.abs().amax(dim=1, keepdim=True)
    zero = amax == 0
    inverse = torch.where(zero, 0.0, 127.0 / amax.masked_fill(zero, 1.0))
    return (x * inverse).round(), amax / 127.0


def _product(q, scale, W, w_scale):
    return q @ W.float().t() * scale * w_scale


def _philox_round(state, _):
    (a, b, c, d), (k0, k1) = state
    low = 0xFFFFFFFF
    first, second = a * 0xD2511F53, c * 0xCD9E8D57  # (of the wrapped products bits 0 .. 63 are right)
    words = ((second >> 32) & low) ^ b ^ k0, second & low, ((first >> 32) & low) ^ d ^ k1, first & low
    return words, ((k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low)


def _kept(n, p, seed, offset, device):
    """Which of n elements are kept, and the factor of those."""
    group = torch.arange((n + 7) // 8, device=device, dtype=torch.int64)
    low = 0xFFFFFFFF
    start = (group & low, group >> 32, torch.full_like(group, offset & low), torch.full_like(group, offset >> 32)), (seed & low, seed >> 32)
    words, _ = functools.reduce(_philox_round, range(10), start)
    bits = torch.stack([v for w in words for v in (w & 0xFFFF, w >> 16)], dim=1).reshape(-1)[:n]
    least = int(round(p * 65536))
    return bits >= least, 65536.0 / (65536 - least) if least < 65536 else 0.0


def _plain(s):
    op = s["op"]
    if op == "linear":
        return _product(*_rows_in_8_bits(s["x"]), s["W"], s["w_scale"]).half()
    if op == "linear_grad":
        return ((s["g"].float() * s["w_scale"]) @ s["W"].float()).half()
    if op == "gated":
        q, scale = _rows_in_8_bits(s["x"])
        gate, up = _product(q, scale, s["W"], s["w_scale"]).chunk(2, dim=1)
        if s["addends"] is not None:
            gate, up = gate + s["addends"][0].float(), up + s["addends"][1].float()
        h = (gate / (1 + torch.exp(-gate)) * up).half()
        return (h, torch.stack([gate, up]).half()) if s["train"] else h
    if op == "gated_grad":
        gate, up, dh = s["gate_up"][0].float(), s["gate_up"][1].float(), s["dh"].float()
        sigma = 1 / (1 + torch.exp(-gate))
        dgate, dup = dh * up * sigma * (1 + gate * (1 - sigma)), dh * gate * sigma
        dx = (torch.cat([dgate, dup], dim=1) * s["w_scale"]) @ s["W"].float()
        return dx.half(), torch.stack([dgate, dup]).half()
    keep, factor = _kept(s["x"].numel(), s["p"], s["seed"], s["offset"], s["x"].device)
    y = torch.where(keep.view(s["x"].shape), s["x"].float() * factor, 0.0)
    return (y if s["base"] is None else y + s["base"].float()).half()


# ------------------------------------------------------------------------------------------------- passes ----
def run(s):
    if not own:
        return _plain(s)
    from paper_2605_24058_amd import binding

    op = s["op"]
    if op == "linear":
        return binding.lordba_linear_i8(s["x"], s["W"], s["w_scale"])
    if op == "linear_grad":
        return binding.lordba_linear_i8_backward(s["g"], s["W"], s["w_scale"])
    if op == "gated":
        return binding.lordba_gated_i8(s["x"], s["W"], s["w_scale"], addends=s["addends"], save=s["train"])
    if op == "gated_grad":
        return binding.lordba_gated_i8_backward(s["dh"], s["gate_up"], s["W"], s["w_scale"])
    return binding.lordba_dropout(s["x"], s["p"], s["seed"], s["offset"], y_base=s["base"])


def work(case):
    T, d_in, d_out, op = case["T"], case["d_in"], case["d_out"], case["op"]
    if op == "dropout":
        return {"bytes": T * d_in * (6.0 if case["base"] else 4.0), "flops": 2.0 * T * d_in}
    if op.startswith("linear"):
        return {"bytes": 2.0 * T * (d_in + d_out) + d_in * d_out + 4.0 * d_out, "flops": 2.0 * T * d_in * d_out}
    weights = 2.0 * d_out * d_in + 8.0 * d_out
    if op == "gated":
        return {"bytes": weights + 2.0 * T * (d_in + d_out * (1 + 2 * case["train"] + 2 * case["addends"])), "flops": 4.0 * T * d_in * d_out}
    return {"bytes": weights + 2.0 * T * (d_in + 5 * d_out), "flops": 4.0 * T * d_in * d_out}


# ------------------------------------------------------------------------------------------------ 64 bits ----
def _philox_words(groups, seed, offset):
    mask, shift = np.uint64(0xFFFFFFFF), np.uint64(32)
    n = np.arange(groups, dtype=np.uint64)
    c = [n & mask, n >> shift, np.full_like(n, offset & 0xFFFFFFFF), np.full_like(n, offset >> 32)]
    k = [np.uint64(seed & 0xFFFFFFFF), np.uint64(seed >> 32)]
    for i in range(10):
        if i:
            k = [(k[0] + np.uint64(0x9E3779B9)) & mask, (k[1] + np.uint64(0xBB67AE85)) & mask]
        m0, m1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(m1 >> shift) ^ c[1] ^ k[0], m1 & mask, (m0 >> shift) ^ c[3] ^ k[1], m0 & mask]
    return np.stack(c, axis=1).astype(np.uint32)


def exact(case, seed):
    s, op = _inputs(case, seed), case["op"]
    T, d_in, d_out = case["T"], case["d_in"], case["d_out"]
    if op == "dropout":
        n = T * d_in
        draws = _philox_words(-(-n // 8), s["seed"], s["offset"]).view(np.uint16).reshape(-1)[:n]
        least = int(round(s["p"] * 65536))
        y = torch.from_numpy(draws >= least).to("cuda").view(T, d_in) * s["x"].double() * (65536.0 / (65536 - least))
        return y + s["base"].double() if s["base"] is not None else y
    W = s["W"].double() * s["w_scale"].double()[:, None]
    if op == "linear_grad":
        return torch.mm(s["g"].double(), W)
    if op == "gated_grad":
        gate, up = s["gate_up"].double()
        dh = s["dh"].double()
        silu = gate * torch.sigmoid(gate)
        slope = torch.sigmoid(gate) + silu * torch.sigmoid(-gate)
        grads = torch.stack([dh * up * slope, dh * silu])
        return torch.addmm(torch.mm(grads[0], W[:d_out]), grads[1], W[d_out:]), grads
    x = s["x"].double()
    step = x.abs().max(dim=1).values.clamp_min(1e-300) / 127
    x8 = torch.round(x / step[:, None]) * step[:, None]
    if op == "linear":
        return torch.mm(x8, W.t().contiguous())
    gate, up = torch.mm(x8, W[:d_out].t().contiguous()), torch.mm(x8, W[d_out:].t().contiguous())
    if s["addends"] is not None:
        gate, up = gate + s["addends"][0].double(), up + s["addends"][1].double()
    h = gate * torch.sigmoid(gate) * up
    return (h, torch.stack([gate, up])) if case["train"] else h
