"""Cases of the language model's loss and of activations kept in 8 bits.

What a training program does between the embedding and the gradients' clip:
the head's cross entropy over the whole vocabulary with the gradients of the
hidden states and of the table; scoring tokens with it, without gradients;
linear layers and gated activations that keep their inputs in 8 bits for the
backward pass; and the 8-bit form by itself.  Sizes are this repository's
model layouts (GPT 1.3B, Llama 7B and 13B, and the small layout of its tests)
with whole batches of tokens, and odd ones between.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
BLOCK = 32  # columns that share a scale


def listed():
    return [
        # the tests' two-layer layout: a training step whose launches and latency count
        {"name": "head_small", "op": "head", "tokens": 96, "length": 48, "vocab": 320, "dim": 64, "type": "bf16",
         "grad": "bf16"},
        # fp16 training with a loss scale, odd sizes, padded sequences
        {"name": "head_fp16_odd", "op": "head", "tokens": 2331, "length": 777, "vocab": 32003, "dim": 1157,
         "type": "fp16", "grad": "fp16", "masked": 0.2, "scale": 65536.0},
        # one training batch of the GPT 1.3B layout, some of the sequences padded
        {"name": "head_gpt_8x2048", "op": "head", "tokens": 16384, "length": 2048, "vocab": 50304, "dim": 2048,
         "type": "bf16", "grad": "bf16", "masked": 0.05},
        # one token's loss, Llama 7B
        {"name": "score_one_token", "op": "score", "tokens": 1, "length": 1, "vocab": 32000, "dim": 4096,
         "type": "bf16"},
        # every token's loss over a long sequence, Llama 13B
        {"name": "score_13b_4096", "op": "score", "tokens": 4096, "length": 4096, "vocab": 32000, "dim": 5120,
         "type": "bf16"},
        # the tests' layout, up projection
        {"name": "linear8_small", "op": "linear8", "tokens": 96, "rows": 176, "cols": 64, "type": "bf16",
         "grad": "bf16"},
        # odd sizes, fp16, the weight's gradient kept in fp32
        {"name": "linear8_fp16_odd", "op": "linear8", "tokens": 2999, "rows": 3085, "cols": 1157, "type": "fp16",
         "grad": "fp32"},
        # a training batch through the GPT 1.3B layout's up projection
        {"name": "linear8_gpt_8x2048", "op": "linear8", "tokens": 16384, "rows": 8192, "cols": 2048, "type": "bf16",
         "grad": "bf16"},
        # the GPT layout's activation without a gate, odd sizes, fp32
        {"name": "gate8_gelu_odd", "op": "gate8", "tokens": 1501, "cols": 3085, "type": "fp32", "kind": "gelu"},
        # Llama 7B's gated activation over a training batch, both halves from one product
        {"name": "gate8_7b_8x2048", "op": "gate8", "tokens": 16384, "cols": 11008, "type": "bf16", "kind": "silu",
         "gated": True, "halves": True},
        # one layer's normed input of the tests' layout, kept and restored
        {"name": "act8_small", "op": "act8", "tokens": 96, "cols": 64, "type": "bf16"},
        # the hidden states of a large batch of Llama 13B
        {"name": "act8_13b_65536", "op": "act8", "tokens": 65536, "cols": 5120, "type": "bf16"},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return w["bytes"] / 4e12 + w["flops"] / 1e14


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(["head", "head", "score", "linear8", "linear8", "gate8", "act8"])
        c = {"op": op}
        if op in ("head", "score"):
            length = rng.choice([1, 1, 7, 128, 1000, 2048])
            c.update(length=length, tokens=length * _log_uniform(rng, 1, max(1, 16384 // length)),
                     vocab=_log_uniform(rng, 300, 131072), dim=_log_uniform(rng, 48, 8192),
                     type=rng.choice(["bf16", "bf16", "fp16"]))
            if rng.random() < 0.8:
                c["dim"] = (c["dim"] + 7) // 8 * 8
            if rng.random() < 0.4:
                c["masked"] = rng.choice([0.02, 0.3])
            if rng.random() < 0.3:
                c["factor"] = 0.5
        elif op == "linear8":
            c.update(tokens=_log_uniform(rng, 1, 32768), rows=_log_uniform(rng, 48, 14000),
                     cols=_log_uniform(rng, 48, 14000), type=rng.choice(["bf16", "bf16", "fp16"]))
            if rng.random() < 0.8:
                c["rows"], c["cols"] = (c["rows"] + 7) // 8 * 8, (c["cols"] + 7) // 8 * 8
        else:
            c.update(tokens=_log_uniform(rng, 1, 65536), cols=_log_uniform(rng, 48, 14000),
                     type=rng.choice(["bf16", "bf16", "fp16", "fp32"]))
            if rng.random() < 0.7:
                c["cols"] = (c["cols"] + 7) // 8 * 8
            if op == "gate8":
                c["kind"] = rng.choice(["silu", "gelu", "gelu_tanh"])
                if rng.random() < 0.7:
                    c["gated"] = True
                    c[rng.choice(["halves", "apart"])] = True
        if op == "head":
            c["grad"] = c["type"]
        elif op == "linear8":
            c["grad"] = rng.choice([c["type"], "fp32"])
        if op == "head" and c["type"] == "fp16":  # a loss scale that the batch's gradients stand
            c["scale"] = float(min(65536, 512 * c["tokens"]))
        if _cost(c) <= most:
            return c


def _gen(seed, k):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 7919 + 104729 * k + 17)
    return gen


def _normal(shape, dtype, sigma, seed, k):
    gen, out = _gen(seed, k), torch.empty(shape, dtype=DTYPES[dtype], device="cuda")
    step = max(1, (1 << 27) // shape[1])
    for a in range(0, shape[0], step):
        part = out[a:a + step]
        part.copy_(torch.empty(part.shape, device="cuda").normal_(0.0, sigma, generator=gen))
    return out


def _activations(shape, dtype, seed, k):
    """N(0, 1) with some columns ten times as large, as layers' inputs have them."""
    x = _normal(shape, dtype, 1.0, seed, k)
    large = torch.rand(shape[1], generator=_gen(seed, k + 50), device="cuda") < 0.01
    return x.mul_(torch.where(large, 10.0, 1.0).to(x.dtype))


class _State:
    pass


def _inputs(case, seed):
    st = _State()
    st.case = case
    t = case["type"]
    if case["op"] in ("head", "score"):
        tokens, vocab, dim = case["tokens"], case["vocab"], case["dim"]
        st.factor = case.get("factor", 1.0)
        st.table = _normal((vocab, dim), t, 0.02, seed, 1)
        # text's law over a vocabulary sorted by frequency
        p = np.cumsum(1.0 / (np.arange(vocab) + 2.7))
        u = torch.rand(tokens, generator=_gen(seed, 2), device="cuda", dtype=torch.float64)
        want = torch.searchsorted(torch.from_numpy(p / p[-1]).cuda(), u).clamp_(max=vocab - 1)
        # hidden states that know the next token more or less: its logit is up to 12 above the others'
        st.hidden = _normal((tokens, dim), t, 1.0, seed, 3)
        known = 12.0 * torch.rand(tokens, 1, generator=_gen(seed, 4), device="cuda") / (4e-4 * dim)
        for a in range(0, tokens, 4096):
            st.hidden[a:a + 4096] += (known[a:a + 4096] * st.table[want[a:a + 4096]].float()).to(DTYPES[t])
        st.targets = want.view(-1, case["length"])
        if case.get("masked"):  # the ends of the sequences, as -1
            batch, length = st.targets.shape
            kept = 1.0 - 2.0 * case["masked"] * torch.rand(batch, 1, generator=_gen(seed, 5), device="cuda")
            if length == 1:
                gone = kept < 1.0 - case["masked"]
            else:
                gone = torch.arange(length, device="cuda")[None] >= kept * length
            st.targets = torch.where(gone, torch.full_like(st.targets, -1), st.targets)
        st.hidden = st.hidden.view(*st.targets.shape, dim)
        st.up = torch.full((), case.get("scale", 1.0), device="cuda")
    elif case["op"] == "linear8":
        st.x = _activations((case["tokens"], case["cols"]), t, seed, 1)
        st.weight = _normal((case["rows"], case["cols"]), t, 0.02, seed, 2)
        st.grad_out = _normal((case["tokens"], case["rows"]), t, 1e-3, seed, 3)
    else:
        n = case["cols"]
        if case.get("halves"):  # one buffer, the gate's columns before the other factor's
            both = _activations((case["tokens"], 2 * n), t, seed, 1)
            st.x, st.factor = both[:, :n], both[:, n:]
        else:
            st.x = _activations((case["tokens"], n), t, seed, 1)
            st.factor = _activations((case["tokens"], n), t, seed, 2) if case.get("gated") else None
        if case["op"] == "gate8":
            st.grad_out = _normal((case["tokens"], n), t, 1e-3, seed, 3)
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    if case["op"] == "head":  # the table's part of the flat gradient buffer
        st.grad_weight = torch.zeros(case["vocab"], case["dim"], dtype=DTYPES[case["grad"]], device="cuda")
    elif case["op"] == "linear8":
        st.grad_weight = torch.zeros(case["rows"], case["cols"], dtype=DTYPES[case["grad"]], device="cuda")
    if own:
        import paper_2511_07035_amd as gockpt
        st.lib = gockpt
    torch.cuda.synchronize()
    return st


# ---- plain forms -----------------------------------------------------------------


def _restored(x):
    """x as its 8-bit form stands for it: in blocks of 32 columns, whole
    multiples (at most 127) of a power of two, the least that will do."""
    rows, cols = x.shape
    wide = (cols + BLOCK - 1) // BLOCK * BLOCK
    v = torch.zeros(rows, wide, dtype=x.dtype, device=x.device)
    v[:, :cols] = x
    v = v.view(rows, wide // BLOCK, BLOCK)
    most = v.abs().amax(2, keepdim=True)
    half, e = torch.frexp(most)  # most = half * 2^e, half in [0.5, 1)
    e = torch.where(half * 128.0 > 127.0, e - 6, e - 7).clamp(min=-126)
    step = torch.ldexp(torch.ones_like(most), e)
    return (torch.round(v / step) * step).view(rows, wide)[:, :cols]


def _activation(x, kind):
    """The activation and its derivative."""
    if kind == "silu":
        s = torch.sigmoid(x)
        return x * s, s * (1.0 + x * (1.0 - s))
    if kind == "gelu":
        c = 0.5 * (1.0 + torch.erf(x * math.sqrt(0.5)))
        return x * c, c + x * torch.exp(-0.5 * x * x) / math.sqrt(2.0 * math.pi)
    a, b = math.sqrt(2.0 / math.pi), 0.044715
    th = torch.tanh(a * (x + b * x * x * x))
    return 0.5 * x * (1.0 + th), 0.5 * (1.0 + th) + 0.5 * x * (1.0 - th * th) * a * (1.0 + 3.0 * b * x * x)


def _linear8(x, w, dy):
    """x w^T, its gradient by x, and by w with x as kept."""
    return x @ w.t(), dy @ w, dy.t() @ _restored(x)


def _gate8(x, factor, dy, kind):
    """act(x) * factor, and the gradients with both as kept."""
    y = _activation(x, kind)[0]
    a, d = _activation(_restored(x), kind)
    if factor is None:
        return y, dy * d, None
    return y * factor, dy * d * _restored(factor), dy * a


def run(st):
    case = st.case
    if own:
        return _run_own(st)
    t = DTYPES[case["type"]]
    if case["op"] in ("head", "score"):
        hidden, table = st.hidden.reshape(-1, case["dim"]).float(), st.table.float()
        targets = st.targets.reshape(-1)
        there = targets >= 0
        at = targets.clamp(min=0)
        logits = (hidden @ table.t()).mul_(st.factor)
        most = logits.amax(1, keepdim=True)
        own_logit = logits.gather(1, at[:, None])
        p = logits.sub_(most).exp_()
        total = p.sum(1, keepdim=True)
        loss = torch.where(there, (most + total.log() - own_logit)[:, 0], torch.zeros_like(total[:, 0]))
        if case["op"] == "score":
            return loss.view(st.targets.shape)
        count = there.sum().clamp(min=1)
        p.div_(total)
        p.scatter_add_(1, at[:, None], torch.full_like(own_logit, -1.0))
        p.mul_((there * (st.up * st.factor / count))[:, None])
        grad_hidden = (p @ table).to(t).view(st.hidden.shape)
        st.grad_weight.copy_(p.t() @ hidden)
        return {"loss": loss.sum() / count, "grad_hidden": grad_hidden, "grad_weight": st.grad_weight}
    if case["op"] == "linear8":
        y, dx, dw = _linear8(st.x.float(), st.weight.float(), st.grad_out.float())
        st.grad_weight.copy_(dw)
        return {"out": y.to(t), "grad_x": dx.to(t), "grad_weight": st.grad_weight}
    if case["op"] == "gate8":
        y, dx, df = _gate8(st.x.float(), None if st.factor is None else st.factor.float(), st.grad_out.float(),
                           case["kind"])
        out = {"out": y.to(t), "grad_x": dx.to(t)}
        return out if df is None else {**out, "grad_factor": df.to(t)}
    return _restored(st.x.float()).to(t)


def _run_own(st):
    case, lib = st.case, st.lib
    if case["op"] == "score":
        return lib.linear_cross_entropy(st.hidden, st.table, st.targets, scale=st.factor, reduction="none")
    if case["op"] == "head":
        hidden, table = st.hidden.detach().requires_grad_(), st.table.detach().requires_grad_()
        loss = lib.linear_cross_entropy(hidden, table, st.targets, scale=st.factor, grad_weight=st.grad_weight)
        loss.backward(st.up)
        return {"loss": loss.detach(), "grad_hidden": hidden.grad, "grad_weight": st.grad_weight}
    if case["op"] == "linear8":
        x, weight = st.x.detach().requires_grad_(), st.weight.detach().requires_grad_()
        y = lib.linear8(x, weight, grad_weight=st.grad_weight)
        y.backward(st.grad_out)
        return {"out": y.detach(), "grad_x": x.grad, "grad_weight": st.grad_weight}
    if case["op"] == "gate8":
        x = st.x.detach().requires_grad_()
        factor = None if st.factor is None else st.factor.detach().requires_grad_()
        y = lib.gate8(x, factor, kind=case["kind"])
        y.backward(st.grad_out)
        out = {"out": y.detach(), "grad_x": x.grad}
        return out if factor is None else {**out, "grad_factor": factor.grad}
    return lib.act8_pack(st.x).unpack()


# ---- definitions in float64 --------------------------------------------------------


def _kept64(x):
    """The 8-bit form's values in float64: codes and steps found with exact logarithms."""
    rows, cols = x.shape
    out = torch.zeros(rows, cols, dtype=torch.float64, device=x.device)
    for a in range(0, cols, BLOCK):
        v = x[:, a:a + BLOCK].double()
        most = v.abs().amax(1, keepdim=True)
        e = torch.floor(torch.log2(torch.clamp(most, min=2.0 ** -120))) - 7.0
        for _ in range(3):  # up to the least step that reaches: one or two of these raise it
            e = torch.where(most > 127.0 * torch.exp2(e), e + 1.0, e)
        e = torch.clamp(e, min=-126.0)
        out[:, a:a + BLOCK] = torch.round(v * torch.exp2(-e)) * torch.exp2(e)
    return out


def _slope64(x, kind):
    if kind == "silu":
        e = torch.exp(-x.abs())
        s = torch.where(x >= 0, 1.0 / (1.0 + e), e / (1.0 + e))
        return x * s, s + x * s * (1.0 - s)
    if kind == "gelu":
        c = 0.5 * torch.erfc(-x / math.sqrt(2.0))
        return x * c, c + x * torch.exp(-x * x / 2.0) / math.sqrt(2.0 * math.pi)
    u = 2.0 * math.sqrt(2.0 / math.pi) * (x + 0.044715 * x ** 3)
    s = torch.sigmoid(u)  # (1 + tanh(u / 2)) / 2
    return x * s, s + x * s * (1.0 - s) * 2.0 * math.sqrt(2.0 / math.pi) * (1.0 + 3.0 * 0.044715 * x * x)


def exact(case, seed):
    st = _inputs(case, seed)
    if case["op"] in ("head", "score"):
        hidden, targets = st.hidden.reshape(-1, case["dim"]), st.targets.reshape(-1)
        table = st.table.double()
        loss = torch.zeros(targets.numel(), dtype=torch.float64, device="cuda")
        kept = (targets >= 0).nonzero()[:, 0]
        grad_hidden, grad_weight = torch.zeros(hidden.shape, dtype=torch.float64, device="cuda"), None
        if case["op"] == "head":
            grad_weight = torch.zeros_like(table)
        for a in range(0, kept.numel(), 2048):
            k = kept[a:a + 2048]
            x = hidden[k].double()
            logits = st.factor * torch.mm(x, table.t())
            lse = torch.logsumexp(logits, 1)
            loss[k] = lse - logits[torch.arange(k.numel(), device="cuda"), targets[k]]
            if case["op"] == "head":
                z = torch.exp(logits - lse[:, None])
                z[torch.arange(k.numel(), device="cuda"), targets[k]] -= 1.0
                z *= st.factor * float(st.up) / kept.numel()
                grad_hidden[k] = torch.mm(z, table)
                grad_weight += torch.mm(z.t(), x)
        if case["op"] == "score":
            return loss.view(st.targets.shape)
        return {"loss": loss.sum() / max(1, kept.numel()), "grad_hidden": grad_hidden.view(st.hidden.shape),
                "grad_weight": grad_weight}
    if case["op"] == "linear8":
        x, w, dy = st.x.double(), st.weight.double(), st.grad_out.double()
        return {"out": torch.mm(x, w.t()), "grad_x": torch.mm(dy, w), "grad_weight": torch.mm(dy.t(), _kept64(st.x))}
    if case["op"] == "gate8":
        y = _slope64(st.x.double(), case["kind"])[0]
        a, d = _slope64(_kept64(st.x), case["kind"])
        dy = st.grad_out.double()
        if st.factor is None:
            return {"out": y, "grad_x": dy * d}
        return {"out": y * st.factor.double(), "grad_x": dy * d * _kept64(st.factor), "grad_factor": dy * a}
    return _kept64(st.x)


def work(case):
    size = SIZE[case["type"]]
    if case["op"] in ("head", "score"):
        tokens, vocab, dim = case["tokens"], case["vocab"], case["dim"]
        kept = tokens * (1.0 - case.get("masked", 0.0))
        read = 8 * tokens + (kept + vocab) * dim * size
        if case["op"] == "score":  # the logits; one loss a token
            return {"bytes": read + 4 * tokens, "flops": 2 * kept * vocab * dim}
        # the logits, the hidden states' gradient, the table's
        return {"bytes": read + 4 + tokens * dim * size + vocab * dim * SIZE[case["grad"]],
                "flops": 6 * kept * vocab * dim}
    n = case["tokens"] * case["cols"]
    kept = n * (1.0 + 1.0 / BLOCK)  # the 8-bit form: a byte each, and one for each block's step
    if case["op"] == "linear8":
        out = case["tokens"] * case["rows"]
        # forward: input and weight read, output and 8-bit form written; backward: the output's gradient, weight
        # and 8-bit form read, both gradients written
        return {"bytes": n * size + out * size + kept + out * size + kept + n * size
                + case["rows"] * case["cols"] * (2 * size + SIZE[case["grad"]]), "flops": 6 * n * case["rows"]}
    if case["op"] == "gate8":
        k = 2 if case.get("gated") else 1
        # forward: k factors read, the product and k 8-bit forms written; backward: these and the gradient read,
        # k gradients written
        return {"bytes": 2 * (k + 1) * n * size + 2 * k * kept, "flops": 20 * k * n}
    return {"bytes": 2 * n * size + 2 * kept, "flops": 4 * n}  # read, kept; read again, restored
