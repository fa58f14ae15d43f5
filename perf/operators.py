"""The training operators beside the PSO-PS synchronisation, as cases that can be timed and checked.

Between two synchronisations a worker takes optimiser steps, and at a synchronisation its loss is its
fitness.  Three operators cover that for a model with a vocabulary (or a set of classes) at its end:

  xent    softmax cross entropy of a linear head, logits = h w^T, without keeping the logits: the loss alone
          (a worker's fitness), or the loss with the gradients of h and w (a training step)
  adamw   one AdamW step over many tensors at once, its two moments held in 32 or in 8 bits
  norm    the 2-norm of all gradients together, and the factor that clips it

``own`` selects the form: False computes the plain form (elementary torch operations in 32 bits), True makes
the calls of paper_2009_03816_b200.training.
"""
import math

import numpy as np
import torch

own = False

BLOCK = 256                       # elements that share one scale of an 8-bit moment
BETA1, BETA2, EPS, DECAY, LR = 0.9, 0.999, 1e-8, 0.01, 1e-3
STEPS_DONE = 100                  # the optimiser's state is that of a run under way
MAX_NORM = 1.0
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def listed():
    return [
        # The classifier head of the LeNet-sized model with the paper's batch of 256: launch latency is all there is.
        # 84 features are no multiple of 16 bytes.
        {"name": "xent head 256x84x10", "op": "xent", "tokens": 256, "dim": 84, "vocab": 10, "type": "bf16",
         "train": True, "masked": 0.0},
        # One token scored against a whole vocabulary: the weights are read once, nothing else matters.
        {"name": "xent one token", "op": "xent", "tokens": 1, "dim": 4096, "vocab": 32768, "type": "bf16",
         "train": False, "masked": 0.0},
        # A worker's fitness at a synchronisation: the loss of a held-out batch, no gradients; an odd vocabulary.
        {"name": "xent fitness", "op": "xent", "tokens": 2048, "dim": 2048, "vocab": 50001, "type": "fp16",
         "train": False, "masked": 0.1},
        # A small model's training step with odd sizes, a good part of the tokens being prompts without a loss.
        {"name": "xent train ragged", "op": "xent", "tokens": 3001, "dim": 1000, "vocab": 32003, "type": "fp16",
         "train": True, "masked": 0.35},
        # The training step of a large model: matrix products bound by the tensor cores.
        {"name": "xent train large", "op": "xent", "tokens": 8192, "dim": 4096, "vocab": 131072, "type": "bf16",
         "train": True, "masked": 0.0},
        # One worker's LeNet-sized weights, tensors packed tightly in the worker's fp32 row: latency.
        {"name": "adamw32 lenet row", "op": "adamw", "elements": 61706, "tensors": 10, "bits": 32, "grad": "fp32",
         "copy": "none", "packed": True},
        # A ResNet-18-sized model trained in bf16 with fp32 master weights in the row.
        {"name": "adamw32 resnet18", "op": "adamw", "elements": 11173962, "tensors": 62, "bits": 32, "grad": "bf16",
         "copy": "bf16", "packed": False},
        # The same with moments of 8 bits and fp16 training.
        {"name": "adamw8 resnet18", "op": "adamw", "elements": 11173962, "tensors": 62, "bits": 8, "grad": "fp16",
         "copy": "fp16", "packed": False},
        # Eight workers' ResNet-50-sized rows in one step, tightly packed.
        {"name": "adamw32 8 rows", "op": "adamw", "elements": 204456256, "tensors": 1288, "bits": 32, "grad": "fp32",
         "copy": "none", "packed": True},
        # A model whose optimiser state is what fills the memory: 8 bits, bf16 training; an odd total.
        {"name": "adamw8 large", "op": "adamw", "elements": 268000001, "tensors": 291, "bits": 8, "grad": "bf16",
         "copy": "bf16", "packed": False},
        # Clipping, at the smallest and the largest of the models above.
        {"name": "norm lenet row", "op": "norm", "elements": 61706, "tensors": 10, "grad": "fp32", "packed": True},
        {"name": "norm large", "op": "norm", "elements": 268000001, "tensors": 291, "grad": "bf16", "packed": False},
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["xent", "xent", "adamw", "adamw", "norm"])
    if op == "xent":
        tokens = _log_int(rng, 1, 8192)
        dim = _log_int(rng, 64, 4096)
        if rng.random() < 0.6:                      # mostly what an aligned model has, else any number
            dim = max(64, dim // 64 * 64)
        vocab = _log_int(rng, 10, 131072)
        return {"op": "xent", "tokens": tokens, "dim": dim, "vocab": vocab, "type": rng.choice(["bf16", "fp16"]),
                "train": rng.random() < 0.6, "masked": rng.choice([0.0, 0.0, round(rng.uniform(0.05, 0.9), 3)])}
    elements = _log_int(rng, 50_000, 180_000_000)
    tensors = min(_log_int(rng, 2, 1000), elements // 1000)
    grad = rng.choice(["fp32", "bf16", "fp16"])
    if op == "norm":
        return {"op": "norm", "elements": elements, "tensors": tensors, "grad": grad, "packed": rng.random() < 0.5}
    bits = rng.choice([32, 8])
    return {"op": "adamw", "elements": elements, "tensors": tensors, "bits": bits, "grad": grad,
            "copy": rng.choice(["none", grad if grad != "fp32" else "bf16"]),
            "packed": bits == 32 and rng.random() < 0.5}


# ---- inputs ---------------------------------------------------------------------------------------

def _valid_count(case):
    return case["tokens"] - int(case["tokens"] * case["masked"])


def _sizes(case):
    """Element counts of the tensors: a few large ones and many small ones, as in a model; odd sizes among them."""
    n, count = case["elements"], case["tensors"]
    share = np.random.RandomState(count).lognormal(0.0, 2.0, count)
    size = np.maximum(1, np.floor(share / share.sum() * (n - count)).astype(np.int64))
    size[int(np.argmax(size))] += n - int(size.sum())
    return [int(s) for s in size]


def _arena(case):
    """(first element of each tensor, its size, elements in all) of the flat buffers: tightly packed, or every
    tensor on a multiple of 256 elements, so that a scale's block lies within one tensor."""
    sizes, at, first = _sizes(case), 0, []
    for s in sizes:
        first.append(at)
        at += s if case["packed"] else -(-s // BLOCK) * BLOCK
    return first, sizes, at


def _flat(case, gen, total, first, sizes, scale):
    """One flat fp32 buffer of normal numbers whose spread differs from place to place; zero between the tensors."""
    x = torch.empty(total, device="cuda").normal_(generator=gen)
    spread = torch.empty(-(-total // BLOCK), 1, device="cuda").uniform_(-2.0, 0.5, generator=gen)
    full = total // BLOCK * BLOCK
    x[:full].view(-1, BLOCK).mul_(torch.pow(10.0, spread[: total // BLOCK]) * scale)
    x[full:].mul_(scale)
    if not case["packed"]:
        ends = torch.tensor([f + s for f, s in zip(first, sizes)])
        pads = torch.tensor([-(-s // BLOCK) * BLOCK - s for s in sizes])
        at = torch.repeat_interleave(ends - torch.cumsum(pads, 0) + pads, pads) + torch.arange(int(pads.sum()))
        x[at.cuda()] = 0.0
    return x


def _views(flat, first, sizes):
    return [flat[f:f + s] for f, s in zip(first, sizes)]


def _quantise(x):
    """8 bits a value: e4m3 numbers and one fp32 scale for each 256 (zero where all of them are next to nothing)."""
    x = x.view(-1, BLOCK)
    top = x.abs().amax(1, keepdim=True)
    some = top >= 2.0 ** -100
    scale = torch.where(some, top / torch.full_like(top, 448.0), torch.zeros_like(top))
    inverse = torch.where(some, torch.full_like(top, 448.0) / top, torch.zeros_like(top))
    return (x * inverse).to(torch.float8_e4m3fn).view(-1), scale.view(-1)


def _quantise_root(x):
    """The same for the roots, which are not negative: one that is not zero never becomes zero."""
    q, scale = _quantise(x)
    code = q.view(torch.uint8)
    code = torch.where(x > 0, code.clamp(min=1), code)
    return code.view(torch.float8_e4m3fn), scale


def _values(q, scale):
    return (q.float().view(-1, BLOCK) * scale.view(-1, 1)).view(-1)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    if case["op"] == "xent":
        T, D, V, kind = case["tokens"], case["dim"], case["vocab"], TYPES[case["type"]]
        w = torch.empty(V, D, device="cuda", dtype=kind).normal_(0.0, 0.02, generator=gen)
        targets = torch.randint(0, V, (T,), device="cuda", generator=gen)
        # hidden states as behind a norm, leaning to their target by more or less
        lean = torch.empty(T, 1, device="cuda").uniform_(0.0, 16.0, generator=gen) / (D * 0.02)
        h = torch.empty(T, D, device="cuda").normal_(generator=gen)
        h = (h + lean * w[targets].float() / 0.02).to(kind)
        out = torch.randperm(T, device="cuda", generator=gen)[_valid_count(case):]
        targets[out] = -100
        # the upstream gradient: fp16 training scales its loss, or the gradients would vanish in fp16
        scale = 4096.0 if case["type"] == "fp16" else 1.0
        state = {"case": case, "h": h, "w": w, "targets": targets,
                 "grad": torch.empty((), device="cuda").uniform_(0.5 * scale, 2.0 * scale, generator=gen)}
        if own:
            from paper_2009_03816_b200 import training
            state["op"] = training.LinearXent(T, D, V, dtype=kind, device="cuda")
        return state
    first, sizes, total = _arena(case)
    g = _flat(case, gen, total, first, sizes, 1e-2).to(TYPES[case["grad"]])
    if case["op"] == "norm":
        state = {"case": case, "g": g}
        if own:
            from paper_2009_03816_b200 import training
            state["op"] = training.GradNorm(_views(g, first, sizes))
        return state
    state = {"case": case, "g": g, "p": _flat(case, gen, total, first, sizes, 0.1), "steps": STEPS_DONE,
             "scale": torch.empty((), device="cuda").uniform_(0.25, 1.0, generator=gen)}
    m = _flat(case, gen, total, first, sizes, 1e-3)
    root = _flat(case, gen, total, first, sizes, 1e-2).abs()
    if case["bits"] == 32:
        state["m"], state["v"] = m, root * root
    else:
        state["m"], state["m_scale"] = _quantise(m)
        state["root"], state["root_scale"] = _quantise_root(root)
    del m, root
    if case["copy"] != "none":
        state["copy"] = state["p"].to(TYPES[case["copy"]])
    if own:
        from paper_2009_03816_b200 import training
        views = {k: _views(state[k], first, sizes) for k in ("p", "g", "m", "v", "root", "copy") if k in state}
        scales = {k: _views(state[k], [f // BLOCK for f in first], [-(-s // BLOCK) for s in sizes])
                  for k in ("m_scale", "root_scale") if k in state}
        moments = (views["m"], views["v"]) if case["bits"] == 32 else \
            (views["m"], scales["m_scale"], views["root"], scales["root_scale"])
        state["op"] = training.AdamW(views["p"], views["g"], moments=moments, bits=case["bits"],
                                     copies=views.get("copy"), betas=(BETA1, BETA2), eps=EPS, weight_decay=DECAY,
                                     steps_done=STEPS_DONE)
    return state


# ---- the operators --------------------------------------------------------------------------------

def _xent_plain(s):
    h, w, targets = s["h"].float(), s["w"].float(), s["targets"]
    valid = (targets >= 0) & (targets < w.shape[0])
    at = torch.where(valid, targets, torch.zeros_like(targets))[:, None]
    logits = h @ w.T
    top = logits.amax(1, keepdim=True)
    e = torch.exp(logits - top)
    z = e.sum(1, keepdim=True)
    lse = (top + torch.log(z))[:, 0]
    zero = torch.zeros_like(lse)
    rows = torch.where(valid, lse - logits.gather(1, at)[:, 0], zero)
    count = valid.sum().clamp(min=1).float()
    out = {"loss": rows.sum() / count, "rows": rows, "lse": torch.where(valid, lse, zero)}
    del logits
    if s["case"]["train"]:
        d = e.div_(z)
        d.scatter_add_(1, at, torch.full_like(lse, -1.0)[:, None])
        d.mul_(torch.where(valid, s["grad"] / count, zero)[:, None])
        out["dh"] = (d @ w).to(s["h"].dtype)
        out["dw"] = (d.T @ h).to(s["w"].dtype)
    return out


def _adamw_plain(s):
    case = s["case"]
    s["steps"] += 1
    decay = float(np.float32(1.0 - LR * DECAY))
    rate = float(np.float32(LR * (1.0 / (1.0 - BETA1 ** s["steps"]))))
    spread = float(np.float32(1.0 / math.sqrt(1.0 - BETA2 ** s["steps"])))
    g = s["g"].float() * s["scale"]
    if case["bits"] == 32:
        m, v = s["m"], s["v"]
    else:
        m, v = _values(s["m"], s["m_scale"]), _values(s["root"], s["root_scale"])
        v = v * v
    m = m * float(np.float32(BETA1)) + g * float(np.float32(1.0 - BETA1))
    v = v * float(np.float32(BETA2)) + g * g * float(np.float32(1.0 - BETA2))
    root = v.sqrt()
    p = s["p"] * decay - (m * rate) / (root * spread + float(np.float32(EPS)))
    s["p"].copy_(p)
    if case["bits"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
    else:
        s["m"], s["m_scale"] = _quantise(m)
        s["root"], s["root_scale"] = _quantise_root(root)
    if "copy" in s:
        s["copy"].copy_(p)
    return _adamw_out(s)


def _adamw_out(s):
    return {k: s[k] for k in ("p", "m", "v", "m_scale", "root", "root_scale", "copy") if k in s}


def _norm_plain(s):
    norm = torch.sqrt((s["g"].float() ** 2).sum())
    return {"norm": norm, "factor": torch.clamp(MAX_NORM / (norm + 1e-6), max=1.0)}


def run(state):
    op = state["case"]["op"]
    if op == "xent":
        if not own:
            return _xent_plain(state)
        x, h, w, targets = state["op"], state["h"], state["w"], state["targets"]
        loss, rows, lse = x.forward(h, w, targets)
        out = {"loss": loss, "rows": rows, "lse": lse}
        if state["case"]["train"]:
            out["dh"], out["dw"] = x.backward(h, w, targets, lse, state["grad"])
        return out
    if op == "adamw":
        if not own:
            return _adamw_plain(state)
        state["op"].step(LR, state["scale"])
        return _adamw_out(state)
    if not own:
        return _norm_plain(state)
    norm, factor = state["op"].norm(MAX_NORM)
    return {"norm": norm, "factor": factor}


def work(case):
    if case["op"] == "xent":
        T, D, V, n = case["tokens"], case["dim"], case["vocab"], _valid_count(case)
        read = 2 * D * (n + V) + 8 * T
        if not case["train"]:
            return {"bytes": read + 8 * T + 4, "flops": 2.0 * n * D * V}
        return {"bytes": read + 8 * T + 4 + 2 * D * (T + V), "flops": 6.0 * n * D * V}
    n = case["elements"]
    grad = 4 if case["grad"] == "fp32" else 2
    if case["op"] == "norm":
        return {"bytes": grad * n + 8, "flops": 2.0 * n}
    copy = 2 if case["copy"] != "none" else 0
    moments = 16 if case["bits"] == 32 else 4 + 16 / BLOCK
    return {"bytes": n * (8 + grad + copy + moments), "flops": 15.0 * n}


# ---- the same in 64 bits, from the definitions ----------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        norm = torch.linalg.vector_norm(s["g"].double())
        return {"norm": norm, "factor": torch.minimum(torch.ones_like(norm), MAX_NORM / (norm + 1e-6))}
    if case["op"] == "adamw":
        return _adamw_exact(case, s)
    # d loss / d logits[t, v] = (softmax - one-hot) * grad / count for the tokens that count; a piece of the tokens at a time
    h, w, targets = s["h"].double(), s["w"].double(), s["targets"]
    keep = torch.nonzero(targets >= 0)[:, 0]
    T, count = case["tokens"], max(1, keep.numel())
    rows, lse = (torch.zeros(T, dtype=torch.float64, device="cuda") for _ in range(2))
    dh, dw = torch.zeros_like(h), torch.zeros_like(w)
    for part in keep.split(1024):
        logits = h[part] @ w.T
        lse[part] = torch.logsumexp(logits, 1)
        right = targets[part]
        rows[part] = lse[part] - logits[torch.arange(part.numel(), device="cuda"), right]
        if case["train"]:
            d = torch.exp(logits - lse[part][:, None])
            d[torch.arange(part.numel(), device="cuda"), right] -= 1.0
            d *= s["grad"].double() / count
            dh[part] = d @ w
            dw += d.T @ h[part]
    out = {"loss": rows.sum() / count, "rows": rows, "lse": lse}
    if case["train"]:
        out["dh"], out["dw"] = dh, dw
    return out


def _adamw_exact(case, s):
    t = STEPS_DONE + 1
    g = s["g"].double() * s["scale"].double()
    if case["bits"] == 32:
        m, v = s["m"].double(), s["v"].double()
    else:
        m = s["m"].double() * s["m_scale"].double().repeat_interleave(BLOCK)
        v = (s["root"].double() * s["root_scale"].double().repeat_interleave(BLOCK)) ** 2
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g ** 2
    p = s["p"].double()
    p = p - LR * DECAY * p - LR * (m / (1 - BETA1 ** t)) / (torch.sqrt(v / (1 - BETA2 ** t)) + EPS)
    out = {"p": p}
    if case["bits"] == 32:
        out["m"], out["v"] = m, v
    else:
        for name, x in (("m", m), ("root", torch.sqrt(v))):
            top = x.view(-1, BLOCK).abs().amax(1)
            held = x * torch.where(top > 0, 448.0 / top, 0.0).repeat_interleave(BLOCK)
            # the nearest number of three fraction bits, of fixed steps below 2^-6
            step = torch.exp2(torch.floor(torch.log2(held.abs().clamp(min=2.0 ** -6))) - 3)
            held = torch.round(held / step) * step
            if name == "root":
                held = torch.where(x > 0, held.clamp(min=2.0 ** -9), held)
            out[name], out[name + "_scale"] = held, top / 448.0
    if "copy" in s:
        out["copy"] = p
    return out
