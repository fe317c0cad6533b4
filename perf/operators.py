"""The operators around a network's head, as cases that can be timed and compared.

Three kinds of work, each through the package's public entry points (torch.autograd):
  norm     layer norm over the last axis: y, and in training the gradients of x, weight and bias
  head     softmax cross entropy of a linear head over a vocabulary, from the features in front of it: the rows' losses, and in
           training the gradients of features, weight and bias
  distil   the same head taught by a teacher's top logits: the rows' divergences and the same gradients
Weights are shared by all rows, or there is one set per Monte-Carlo weight sample (samples > 0).  Sizes are those of the package's
workloads (ViT width 192 with 256 x 65 tokens and 10 classes, Swin widths 540 and 2160 with 7260 tokens) and generic ones.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
NORM_EPS = 1e-5
IGNORED = -100

LARGEST_HEAD = 8192 * 4096 * 131072        # rows x width x vocabulary of the largest head
LARGEST_NORM = 32768 * 8192


def listed():
    return [
        # the norm in front of the head for one token of a generated text: nothing but latency
        {"name": "norm_one_token", "kind": "norm", "type": "bf16", "samples": 0, "rows": 1, "width": 4096, "train": False},
        # a ViT block's norm over 256 images x 65 tokens, two weight samples with weights of their own
        {"name": "norm_vit_two_samples", "kind": "norm", "type": "f32", "samples": 2, "rows": 16640, "width": 192, "train": True},
        # an odd number of rows of an odd width, as pruned models have them
        {"name": "norm_odd", "kind": "norm", "type": "f16", "samples": 0, "rows": 5003, "width": 777, "train": True},
        # the largest: a language model's hidden states, 16 sequences of 2048 tokens
        {"name": "norm_large", "kind": "norm", "type": "bf16", "samples": 0, "rows": 32768, "width": 8192, "train": True},
        # the ViT's classifier on 64 images with 16 weight samples: ten classes, launches count
        {"name": "head_ten_classes", "kind": "head", "type": "f32", "samples": 16, "rows": 64, "width": 192, "vocab": 10, "bias": True, "ignored": 0.0, "train": True},
        # one token scored under a large vocabulary: every weight read once
        {"name": "head_score_one_token", "kind": "head", "type": "bf16", "samples": 0, "rows": 1, "width": 4096, "vocab": 131072, "bias": False, "ignored": 0.0, "train": False},
        # fine-tuning on answers: two fifths of the tokens are prompt or padding and carry no label; an odd vocabulary
        {"name": "head_answers_only", "kind": "head", "type": "bf16", "samples": 0, "rows": 4096, "width": 2048, "vocab": 50001, "bias": False, "ignored": 0.4, "train": True},
        # full precision, a bias, a number of rows that fills no tile
        {"name": "head_f32", "kind": "head", "type": "f32", "samples": 0, "rows": 1000, "width": 768, "vocab": 32768, "bias": True, "ignored": 0.1, "train": True},
        # the largest: pre-training, four sequences of 2048 tokens, 131072 words
        {"name": "head_large", "kind": "head", "type": "bf16", "samples": 0, "rows": 8192, "width": 4096, "vocab": 131072, "bias": False, "ignored": 0.0, "train": True},
        # a small student with four weight samples learns the ensemble's eight likeliest classes
        {"name": "distil_small", "kind": "distil", "type": "f32", "samples": 4, "rows": 48, "width": 192, "vocab": 1000, "bias": True, "top": 8, "temperature": 2.0, "train": True},
        # a batch of 2048 tokens in half precision, 64 words a token, softened
        {"name": "distil_f16", "kind": "distil", "type": "f16", "samples": 0, "rows": 2048, "width": 1024, "vocab": 65537, "bias": False, "top": 64, "temperature": 2.0, "train": True},
        # two sequences of 2048 tokens, up to 128 words a token
        {"name": "distil_wide", "kind": "distil", "type": "bf16", "samples": 0, "rows": 4096, "width": 2048, "vocab": 100003, "bias": False, "top": 128, "temperature": 1.0, "train": True},
    ]


def _log_uniform(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _size(rng, low, high):
    n = _log_uniform(rng, low, high)
    return max(low, n // 8 * 8) if rng.random() < 0.5 else n


def draw(rng):
    kind = rng.choice(["norm", "head", "head", "distil", "distil"])
    kind_type = rng.choice(["f32", "bf16", "bf16", "f16"])
    samples = rng.randint(1, 8) if kind_type == "f32" and rng.random() < 0.5 else 0
    train = rng.random() < 0.8
    case = {"kind": kind, "type": kind_type, "samples": samples, "train": train}
    if kind == "norm":
        rows, width = _log_uniform(rng, 1, 32768), _size(rng, 16, 8192)
        rows = max(1, min(rows, LARGEST_NORM // 2 // (width * max(1, samples))))
        return {**case, "rows": rows, "width": width}
    rows, width, vocab = _log_uniform(rng, 1, 8192), _size(rng, 16, 4096), _size(rng, 10, 131072)
    most = LARGEST_HEAD // (8 if kind_type == "f32" else 2)
    rows = max(1, min(rows, most // (width * vocab * max(1, samples))))
    case |= {"rows": rows, "width": width, "vocab": vocab, "bias": rng.random() < 0.4}
    if kind == "head":
        return {**case, "ignored": rng.choice([0.0, 0.0, round(rng.uniform(0.05, 0.7), 2)])}
    return {**case, "top": min(vocab, _log_uniform(rng, 1, 256)), "temperature": rng.choice([1.0, 2.0, round(rng.uniform(0.7, 4.0), 2)])}


def _labelled(case):
    """How many rows (of each sample) carry a label."""
    return max(1, case["rows"] - int(case.get("ignored", 0.0) * case["rows"]))


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    kind, dtype, rows, width = case["kind"], TYPES[case["type"]], case["rows"], case["width"]
    sets = (case["samples"],) if case["samples"] else ()
    state = {"case": case}

    def normal(*shape):
        return torch.randn(*shape, device=DEV, generator=g)

    if kind == "norm":
        # hidden states: a few loud channels, a mean per row
        loud = 1 + 4 * (torch.rand(width, device=DEV, generator=g) < 0.02)
        state["x"] = (normal(*sets, rows, width) * loud + 0.3 * normal(*sets, rows, 1)).to(dtype)
        state["w"] = (1 + 0.2 * normal(*sets, width)).to(dtype)
        state["b"] = (0.1 * normal(*sets, width)).to(dtype)
        if case["train"]:
            state["dy"] = normal(*sets, rows, width).to(dtype)
        return state

    vocab = case["vocab"]
    w = normal(*sets, vocab, width) * (2 / math.sqrt(width))       # logits of standard deviation 2
    x = normal(*sets, rows, width)
    first = torch.randint(vocab, (rows,), device=DEV, generator=g)
    # a trained model: the right word's logit stands out, on some rows clearly
    known = torch.rand(rows, 1, device=DEV, generator=g) * 1.5
    x = (x + known * w.index_select(-2, first)).to(dtype)
    state["x"], state["w"] = x, w.to(dtype)
    state["b"] = (0.5 * normal(*sets, vocab)).to(dtype) if case["bias"] else None
    if kind == "head":
        target = first.clone()
        labelled = _labelled(case)
        if labelled < rows:
            target[torch.randperm(rows, device=DEV, generator=g)[labelled:]] = IGNORED
        state["target"], used = target, labelled
    else:
        top = case["top"]
        # the right word and top - 1 others, all different, likeliest first; one row in eight lists fewer of them
        stride = 1 + (torch.rand(rows, 1, device=DEV, generator=g) * (vocab // top - 1)).long()
        index = (first[:, None] + stride * torch.arange(top, device=DEV)) % vocab
        falls = torch.rand(rows, top, device=DEV, generator=g).log().neg()
        state["logit"] = 12 - falls.cumsum(1)
        short = torch.rand(rows, 1, device=DEV, generator=g) < 0.125
        listed_words = 1 + (torch.rand(rows, 1, device=DEV, generator=g) * top).long()
        index[short & (torch.arange(top, device=DEV) >= listed_words)] = -1
        state["index"], used = index, rows
    if case["train"]:
        # what a loss that is the mean over rows (and samples) hands back; half precision is trained with a scaled loss
        scale = 8192.0 if case["type"] == "f16" else 1.0
        state["g"] = torch.full((*sets, rows), scale / (used * max(1, case["samples"])), device=DEV)
    return state


# --------------------------------------------------------------------------- the plain forms

def _plain_norm(s):
    x, w, b = s["x"].float(), s["w"].float().unsqueeze(-2), s["b"].float().unsqueeze(-2)
    centred = x - x.mean(-1, keepdim=True)
    r = torch.rsqrt((centred * centred).mean(-1, keepdim=True) + NORM_EPS)
    h = centred * r
    y = (h * w + b).to(s["x"].dtype)
    if "dy" not in s:
        return {"y": y}
    dy = s["dy"].float()
    u = dy * w
    dx = r * (u - u.mean(-1, keepdim=True) - h * (u * h).mean(-1, keepdim=True))
    return {"y": y, "dx": dx.to(s["x"].dtype), "dw": (dy * h).sum(-2).to(s["w"].dtype),
            "db": dy.sum(-2).to(s["b"].dtype)}


def _plain_targets(s):
    """(indices, weights, sum of weights times their logarithms, rows that count) and the temperature."""
    if "target" in s:
        counts = s["target"] != IGNORED
        return s["target"].clamp(min=0)[:, None], counts.float()[:, None], torch.zeros_like(counts, dtype=torch.float32), counts, 1.0
    t = s["case"]["temperature"]
    there = s["index"] >= 0
    scaled = torch.where(there, s["logit"] / t, torch.full_like(s["logit"], -math.inf))
    e = torch.exp(scaled - scaled.amax(1, keepdim=True))
    total = e.sum(1, keepdim=True)
    p = e / total
    log_p = torch.where(there, scaled - scaled.amax(1, keepdim=True) - torch.log(total), torch.zeros_like(scaled))
    return s["index"].clamp(min=0), p, (p * log_p).sum(1), there.any(1), t


def _plain_head(s):
    index, p, p_log_p, counts, t = _plain_targets(s)
    x, w = s["x"].float(), s["w"].float()
    z = torch.matmul(x, w.transpose(-1, -2))
    if s["b"] is not None:
        z = z + s["b"].float().unsqueeze(-2)
    z = z / t
    top = z.amax(-1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(-1, keepdim=True)
    lse = (top + torch.log(total)).squeeze(-1)
    wide = index.expand(*z.shape[:-1], index.shape[-1])
    loss = t * t * (p_log_p - (p * z.gather(-1, wide)).sum(-1) + lse) * counts
    if "g" not in s:
        return {"loss": loss}
    del z
    dz = (e / total).scatter_add(-1, wide, -p.expand(wide.shape)) * (s["g"] * counts * t).unsqueeze(-1)
    del e
    dx = torch.matmul(dz, w).to(s["x"].dtype)
    dw = torch.matmul(dz.transpose(-1, -2), x).to(s["w"].dtype)
    out = {"loss": loss, "dx": dx, "dw": dw}
    if s["b"] is not None:
        out["db"] = dz.sum(-2).to(s["b"].dtype)
    return out


# --------------------------------------------------------------------------- the package's operators

def _own(s):
    from paper_2604_04736_amd import autograd as ops
    train = s["case"]["train"]
    leaves = {n: s[n].detach().requires_grad_(train) for n in ("x", "w", "b") if s[n] is not None}
    if s["case"]["kind"] == "norm":
        out = ops.layer_norm(leaves["x"], leaves["w"], leaves["b"], eps=NORM_EPS)
        name, upstream = "y", s.get("dy")
    elif s["case"]["kind"] == "head":
        out = ops.head_cross_entropy(leaves["x"], leaves["w"], s["target"], bias=leaves.get("b"), ignore_index=IGNORED)
        name, upstream = "loss", s.get("g")
    else:
        out = ops.head_distillation(leaves["x"], leaves["w"], s["index"], s["logit"], bias=leaves.get("b"), temperature=s["case"]["temperature"])
        name, upstream = "loss", s.get("g")
    got = {name: out.detach()}
    if train:
        grads = torch.autograd.grad(out, list(leaves.values()), upstream)
        got |= {"d" + n: d for n, d in zip(leaves, grads)}
    return got


def run(state):
    if own:
        return _own(state)
    return _plain_norm(state) if state["case"]["kind"] == "norm" else _plain_head(state)


# --------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    size = 4 if case["type"] == "f32" else 2
    sets, rows, width = max(1, case["samples"]), case["rows"], case["width"]
    n = sets * rows * width
    if case["kind"] == "norm":
        moved = 2 * n + 2 * sets * width + ((2 * n + 2 * sets * width) if case["train"] else 0)     # x, y, w, b; dy, dx, dw, db
        return {"bytes": moved * size, "flops": n * (22 if case["train"] else 8)}
    weights = sets * case["vocab"] * (width + (1 if case["bias"] else 0))
    moved = (n + weights) * size * (2 if case["train"] else 1) + sets * rows * (8 if case["train"] else 4)
    moved += rows * 8 if case["kind"] == "head" else rows * case["top"] * 12
    products = sets * _labelled(case) * width * case["vocab"]
    return {"bytes": moved, "flops": products * (6 if case["train"] else 2)}


# --------------------------------------------------------------------------- in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    d = {n: s[n].double() if s.get(n) is not None else None for n in ("x", "w", "b", "dy", "g", "logit")}
    if case["kind"] == "norm":
        leaf = [d[n].requires_grad_(case["train"]) for n in ("x", "w", "b")]
        var, mean = torch.var_mean(leaf[0], -1, correction=0, keepdim=True)
        y = (leaf[0] - mean) / (var + NORM_EPS).sqrt() * leaf[1].unsqueeze(-2) + leaf[2].unsqueeze(-2)
        out = {"y": y.detach()}
        if case["train"]:
            out |= dict(zip(("dx", "dw", "db"), torch.autograd.grad(y, leaf, d["dy"])))
        return out
    rows, sets = case["rows"], case["samples"]
    out = {"loss": torch.zeros(*((sets,) if sets else ()), rows, dtype=torch.float64, device=DEV)}
    if case["train"]:
        out |= {"d" + n: torch.zeros_like(d[n]) for n in ("x", "w", "b") if d[n] is not None}
    temperature = case.get("temperature", 1.0)
    step = max(1, 2 ** 28 // case["vocab"])
    for k in range(max(1, sets)):
        of = (lambda v: v[k]) if sets else (lambda v: v)
        w = of(d["w"])
        for at in range(0, rows, step):
            to = min(rows, at + step)
            here = torch.arange(to - at, device=DEV)
            teach = torch.zeros(to - at, case["vocab"], dtype=torch.float64, device=DEV)
            if case["kind"] == "head":
                label = s["target"][at:to]
                keep = label != IGNORED
                teach[here[keep], label[keep]] = 1.0
                entropy = 0.0
            else:
                index = s["index"][at:to]
                p = torch.softmax((d["logit"][at:to] / temperature).masked_fill(index < 0, -math.inf), 1)
                teach[here[:, None].expand_as(index)[index >= 0], index[index >= 0]] = p[index >= 0]
                keep = (index >= 0).any(1)
                entropy = torch.special.entr(p).sum(1)
            z = of(d["x"])[at:to] @ w.T
            if d["b"] is not None:
                z += of(d["b"])
            log_q = torch.log_softmax(z / temperature, 1)
            of(out["loss"])[at:to] = torch.where(keep, -temperature ** 2 * ((teach * log_q).sum(1) + entropy), 0.0)
            if not case["train"]:
                continue
            del z
            dz = (log_q.exp_() - teach) * (of(d["g"])[at:to] * keep * temperature)[:, None]
            of(out["dx"])[at:to] = dz @ w
            of(out["dw"]).addmm_(dz.T, of(d["x"])[at:to])
            if d["b"] is not None:
                of(out["db"]).add_(dz.sum(0))
    return out
