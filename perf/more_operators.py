"""Passes through the operators of a 4-bit base model: the frozen projections on 4-bit weights with group scales, their input gradients,
the gated feed-forward block on such weights, and the loss by which adapters learn from a teacher.  Kinds of pass ("op"):

  linear       y = x W^T, x and y in fp16
  linear_grad  the gradient with respect to x of such a projection, dx = g W
  gated        h = silu(x Wg^T + a_g) * (x Wu^T + a_u); with "train" gate and up are returned too, with "addends" the two branch
               outputs a_g and a_u of adapters come in
  gated_grad   from dh and the kept gate and up: the gradients with respect to gate, up and x
  distill      from a student's logits and a teacher's top logits, for every token: the loss, and its gradient with respect to the logits;
               "step": both in one pass with the tokens' weights known before, otherwise the loss first and the gradient behind it

Definition of the weights: W[j, i] = scale[j, i / group] * (code[j, i] - zero[j, i / group]), codes and zeros whole numbers from 0 to 15 (zeros that
are not given are 8), scales in fp16.
Definition of the loss of a token with logits z, temperature u, teacher's logits l_i at the vocabulary entries v_i (those with a v_i below 0 are
absent) and a label c (below 0: none):
    p = softmax over the entries i that are there of l_i / u;   q = softmax(z / u);   r = softmax(z)
    loss = soft * u^2 * sum_i p_i (log p_i - log q[v_i]) - hard * log r[c]
each of the two terms being 0 where there is no entry, no label.  Gradient: weight of the token times
    soft * u * (q - sum_i p_i onehot(v_i)) + hard * (r - onehot(c)).
"""
import math

import torch

own = False  # True: `run` calls this repository's kernels; False: elementary operations in 32 bits


# ------------------------------------------------------------------------------------------------ cases ----
def _case(op, T, d_in, d_out, group=128, zeros=False, train=False, addends=False, pad=0):
    return dict(op=op, T=T, d_in=d_in, d_out=d_out, group=group, zeros=zeros, train=train, addends=addends, pad=pad)


def _loss(T, V, k, u=1.0, hard=0.0, step=True, wide=False, pad=0):
    return dict(op="distill", T=T, V=V, k=k, u=u, hard=hard, step=step, wide=wide, pad=pad)


def listed():
    return [
        # One token through one square projection: a decode step's call, where latency counts.
        dict(_case("linear", 1, 4096, 4096), name="linear_decode"),
        # A prompt of 56 tokens through the wide projection of a model whose weights came with zero points.
        dict(_case("linear", 56, 4096, 11008, group=64, zeros=True), name="linear_prompt_56"),
        # A chunk of a prompt through a head with an odd number of outputs behind an odd number of features, some rows padding.
        dict(_case("linear", 301, 1001, 3001, group=32, zeros=True, pad=40), name="linear_odd"),
        # Prefill of 4096 tokens back to the narrow side of a layer.
        dict(_case("linear", 4096, 11008, 4096), name="linear_prefill"),
        # A training step's input gradient of a square projection.
        dict(_case("linear_grad", 2048, 4096, 4096), name="linear_grad_square"),
        # The input gradient of a head with an odd number of outputs on a short batch.
        dict(_case("linear_grad", 77, 999, 2731, group=32, zeros=True, pad=9), name="linear_grad_odd"),
        # A decode step of eight sequences through the gated block, adapters on both projections.
        dict(_case("gated", 8, 4096, 11008, addends=True), name="gated_decode"),
        # The forward pass of a training step of the block: gate and up are kept for the backward pass.
        dict(_case("gated", 2048, 4096, 11008, train=True, addends=True), name="gated_train"),
        # Its backward pass.
        dict(_case("gated_grad", 2048, 4096, 11008), name="gated_grad"),
        # The backward pass of a short ragged batch of a small block, smaller groups.
        dict(_case("gated_grad", 150, 512, 1376, group=64, zeros=True, pad=11), name="gated_grad_small"),
        # A training step's loss on 2048 tokens with a teacher's 16 best of 32000 entries, kept in fp16: loss and gradient at once.
        dict(_loss(2048, 32000, 16, pad=100), name="distill_step"),
        # Loss, then gradient of a short batch with labels beside the teacher, over a vocabulary of odd size, logits in fp32.
        dict(_loss(333, 50001, 50, u=2.0, hard=0.5, step=False, wide=True, pad=33), name="distill_pair_odd"),
    ]


_MOST = 4.0 * 2048 * 4096 * 11008


def draw(rng):
    def size(low, high):
        return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))))

    op = rng.choice(["linear", "linear", "linear_grad", "gated", "gated_grad", "distill"])
    T = size(1, 8192)
    pad = T // 8 if rng.random() < 0.25 else 0
    if op == "distill":
        V = size(500, 131072)
        while T * V > 2048 * 32000:
            T = max(1, T // 2)
        return _loss(T, V, size(1, 128), u=rng.choice([1.0, 1.0, 2.0, 4.0]), hard=rng.choice([0.0, 0.25, 1.0]), step=rng.random() < 0.6,
                     wide=rng.random() < 0.4, pad=T // 8 if pad else 0)
    d_in, d_out = size(64, 13824), size(64, 13824)
    while 2.0 * T * d_in * d_out * (2 if op.startswith("gated") else 1) > 0.9 * _MOST:
        T = max(1, T // 2)
    return _case(op, T, d_in, d_out, group=rng.choice([32, 64, 128]), zeros=rng.random() < 0.5, train=op == "gated" and rng.random() < 0.5,
                 addends=op == "gated" and rng.random() < 0.7, pad=min(pad, T // 8))


# ----------------------------------------------------------------------------------------------- inputs ----
def _weights(normal, rows, cols, group, zeros):
    """N(0, 1 / cols) rounded to 4 bits group by group: codes uint8 [rows, cols], scale fp16 [rows, groups], zero uint8 [rows, groups] or None."""
    groups = -(-cols // group)
    w = torch.nn.functional.pad(normal(rows, cols, std=1 / math.sqrt(cols)), (0, groups * group - cols)).view(rows, groups, group)
    if zeros:  # the range of a group, 0 in it
        low, high = w.amin(dim=2).clamp_max(0), w.amax(dim=2).clamp_min(0)
        scale = ((high - low) / 15).half()
        zero = (-low / scale.float()).round().clamp(0, 15)
    else:
        scale = (w.abs().amax(dim=2) / 7).half()
        zero = torch.full_like(scale, 8, dtype=torch.float32)
    codes = (w / scale.float()[:, :, None] + zero[:, :, None]).round().clamp(0, 15).to(torch.uint8)
    codes = codes.view(rows, groups * group)[:, :cols].contiguous()
    return dict(codes=codes, scale=scale, zero=zero.to(torch.uint8) if zeros else None)


def _inputs(case, seed):
    """The tensors of a pass from the seed alone.  Activations are N(0, 1) with a few channels eight times as large, as the inputs of
    projections have them; `pad` rows at the end are zeros (padding of a batch), for the loss rows without teacher and label."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    T, pad, op = case["T"], case["pad"], case["op"]

    def normal(*shape, std=1.0):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * std

    if op == "distill":
        V, k = case["V"], case["k"]
        kind = torch.float32 if case["wide"] else torch.float16
        logits = normal(T, V, std=2.0).to(kind)
        best = torch.topk(logits.float() + normal(T, V), k, dim=1)
        index = best.indices.int()
        index[:, k - k // 4:][torch.rand((T, k // 4), generator=gen, device="cuda") < 0.2] = -1  # (a teacher that gave fewer)
        labels = torch.randint(0, V, (T,), generator=gen, device="cuda", dtype=torch.int32)
        labels[::7] = -100
        weight = torch.full((T,), 65536.0 / T, device="cuda") if not case["wide"] else torch.full((T,), 1.0 / T, device="cuda")
        if pad:
            index[T - pad:], labels[T - pad:] = -1, -100
        return dict(logits=logits, index=index.contiguous(), top=best.values.to(kind).contiguous(), labels=labels if case["hard"] else None,
                    weight=weight, u=case["u"], hard=case["hard"])

    def acts(cols, large=False):
        a = normal(T, cols)
        if large:
            a = a * torch.where(torch.rand(cols, generator=gen, device="cuda") < 0.005, 8.0, 1.0)
        if pad:
            a[T - pad:] = 0
        return a.half()

    d_in, d_out = case["d_in"], case["d_out"]
    s = _weights(normal, 2 * d_out if op.startswith("gated") else d_out, d_in, case["group"], case["zeros"])
    if op in ("linear", "gated"):
        s["x"] = acts(d_in, large=True)
        s["addends"] = torch.stack([acts(d_out), acts(d_out)]) if case["addends"] else None
    if op == "linear_grad":
        s["g"] = acts(d_out)
    if op == "gated_grad":
        s["dh"], s["gate_up"] = acts(d_out), torch.stack([acts(d_out), acts(d_out)])
    return s


def prepare(case, seed):
    s = dict(_inputs(case, seed), **{key: case[key] for key in ("op", "train", "group", "step") if key in case})
    if own and "codes" in s:  # the weights as a program keeps them: laid out once, transposed for the gradients
        from paper_2605_24058_amd import binding

        s["W"] = binding.lordba_layout_i4(s.pop("codes"), s.pop("scale"), s.pop("zero"), case["group"],
                                          halves=2 if case["op"].startswith("gated") else 1, transposed=case["op"].endswith("_grad"))
    return s


# -------------------------------------------------------------------------------------------- plain form ----
def _real(s):
    cols = s["codes"].shape[1]
    spread = lambda v: v.float().repeat_interleave(s["group"], dim=1)[:, :cols]
    return (s["codes"].float() - (8.0 if s["zero"] is None else spread(s["zero"]))) * spread(s["scale"])


def _plain_loss(s):
    z, u, soft = s["logits"].float(), s["u"], 1.0
    there = s["index"] >= 0
    some = there.any(dim=1)
    at = s["index"].clamp_min(0).long()
    top = torch.where(there, s["top"].float() / u, float("-inf"))
    top = torch.where(some[:, None], top, 0.0)
    e = torch.exp(top - top.amax(dim=1, keepdim=True))
    total = e.sum(dim=1, keepdim=True)
    p = torch.where(there, e / total, 0.0)
    log_p = torch.where(there, top - top.amax(dim=1, keepdim=True) - torch.log(total), 0.0)
    largest = z.amax(dim=1, keepdim=True)
    exps = torch.exp((z - largest) / u)
    sums = exps.sum(dim=1, keepdim=True)
    log_q = (torch.gather(z, 1, at) - largest) / u - torch.log(sums)
    loss = soft * u * u * torch.where(there, p * (log_p - log_q), 0.0).sum(dim=1)
    grad = torch.where(some[:, None], exps / sums, 0.0).scatter_add(1, at, -p) * (soft * u)
    if s["labels"] is not None:
        labelled = s["labels"] >= 0
        c = s["labels"].clamp_min(0).long()[:, None]
        exps = torch.exp(z - largest)
        sums = exps.sum(dim=1, keepdim=True)
        loss = loss - s["hard"] * torch.where(labelled, (torch.gather(z, 1, c) - largest - torch.log(sums))[:, 0], 0.0)
        hard = (exps / sums).scatter_add(1, c, torch.full_like(sums, -1.0))
        grad = grad + s["hard"] * torch.where(labelled[:, None], hard, 0.0)
    return loss, (grad * s["weight"][:, None]).to(s["logits"].dtype)


def _plain(s):
    op = s["op"]
    if op == "distill":
        return _plain_loss(s)
    W = _real(s)
    if op == "linear":
        return (s["x"].float() @ W.t()).half()
    if op == "linear_grad":
        return (s["g"].float() @ W).half()
    if op == "gated":
        gate, up = (s["x"].float() @ W.t()).chunk(2, dim=1)
        if s["addends"] is not None:
            gate, up = gate + s["addends"][0].float(), up + s["addends"][1].float()
        h = (gate / (1 + torch.exp(-gate)) * up).half()
        return (h, torch.stack([gate, up]).half()) if s["train"] else h
    gate, up, dh = s["gate_up"][0].float(), s["gate_up"][1].float(), s["dh"].float()
    sigma = 1 / (1 + torch.exp(-gate))
    dgate, dup = dh * up * sigma * (1 + gate * (1 - sigma)), dh * gate * sigma
    return (torch.cat([dgate, dup], dim=1) @ W).half(), torch.stack([dgate, dup]).half()


# ------------------------------------------------------------------------------------------------- passes ----
def run(s):
    if not own:
        return _plain(s)
    from paper_2605_24058_amd import binding

    op = s["op"]
    if op == "linear":
        return binding.lordba_linear_i4(s["x"], s["W"])
    if op == "linear_grad":
        return binding.lordba_linear_i4_backward(s["g"], s["W"])
    if op == "gated":
        return binding.lordba_gated_i4(s["x"], s["W"], addends=s["addends"], save=s["train"])
    if op == "gated_grad":
        return binding.lordba_gated_i4_backward(s["dh"], s["gate_up"], s["W"])
    teacher = s["index"], s["top"], s["labels"]
    if s["step"]:
        return binding.lordba_distill(s["logits"], *teacher, temperature=s["u"], hard=s["hard"], d_loss=s["weight"])
    loss, kept = binding.lordba_distill(s["logits"], *teacher, temperature=s["u"], hard=s["hard"])
    return loss, binding.lordba_distill_backward(s["weight"], s["logits"], kept, *teacher, temperature=s["u"], hard=s["hard"])


def work(case):
    T, op = case["T"], case["op"]
    if op == "distill":
        size = 4.0 if case["wide"] else 2.0
        return {"bytes": T * case["V"] * size * (2 if case["step"] else 3) + T * (case["k"] * (4 + size) + 12), "flops": 8.0 * T * case["V"]}
    d_in, d_out = case["d_in"], case["d_out"]
    groups = -(-d_in // case["group"])
    weights = d_out * (d_in / 2.0 + groups * (2.5 if case["zeros"] else 2.0))
    if op.startswith("linear"):
        return {"bytes": 2.0 * T * (d_in + d_out) + weights, "flops": 2.0 * T * d_in * d_out}
    planes = d_in + d_out * (1 + 2 * case["train"] + 2 * case["addends"]) if op == "gated" else d_in + 5 * d_out
    return {"bytes": 2 * weights + 2.0 * T * planes, "flops": 4.0 * T * d_in * d_out}


# ------------------------------------------------------------------------------------------------ 64 bits ----
def _exact_loss(case, s):
    z, u = s["logits"].double(), case["u"]
    T, V = z.shape
    # the teacher as a row of the whole vocabulary
    l = torch.where(s["index"] >= 0, s["top"].double(), float("-inf")) / u
    teacher = torch.softmax(l, dim=1).nan_to_num(0.0)
    logs = torch.log_softmax(z / u, dim=1)
    loss = torch.zeros(T, dtype=torch.float64, device=z.device)
    grad = torch.zeros_like(z)
    rows = torch.arange(T, device=z.device)
    for i in range(case["k"]):
        on = s["index"][:, i] >= 0
        v, p = s["index"][on, i].long(), teacher[on, i]
        loss[on] += u * u * (torch.xlogy(p, p) - p * logs[rows[on], v])
        grad[rows[on], v] -= u * p
    some = (s["index"] >= 0).any(dim=1)
    grad[some] += u * logs[some].exp()
    if case["hard"]:
        on = s["labels"] >= 0
        logs = torch.log_softmax(z[on], dim=1)
        c = s["labels"][on].long()
        loss[on] -= case["hard"] * logs.gather(1, c[:, None])[:, 0]
        grad[on] += case["hard"] * logs.exp()
        grad[rows[on], c] -= case["hard"]
    return loss, grad * s["weight"].double()[:, None]


def exact(case, seed):
    s, op = _inputs(case, seed), case["op"]
    if op == "distill":
        return _exact_loss(case, s)
    d_in, d_out = case["d_in"], case["d_out"]
    column = torch.arange(d_in, device="cuda") // case["group"]
    zero = 8.0 if s["zero"] is None else s["zero"].double()[:, column]
    W = s["scale"].double()[:, column] * (s["codes"].double() - zero)
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
    if op == "linear":
        return torch.mm(x, W.t().contiguous())
    gate, up = torch.mm(x, W[:d_out].t().contiguous()), torch.mm(x, W[d_out:].t().contiguous())
    if s["addends"] is not None:
        gate, up = gate + s["addends"][0].double(), up + s["addends"][1].double()
    h = gate * torch.sigmoid(gate) * up
    return (h, torch.stack([gate, up])) if case["train"] else h
