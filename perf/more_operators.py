"""The operators of a transformer block around its matrix products, as cases that can be timed and compared.

Three kinds of work, each through the package's public entry points (torch.autograd):
  dropout   keeps elements by a counter-based generator, no mask in memory: y, and in training the gradient of x
  block     h = x + scale gate dropout(norm'(branch)), y = norm(h): the end of one block and the norm that begins the next;
            in training the gradients of x, branch, gate and of the norms' weights and biases
  attention softmax(scale q k^T + table[bucket of the two positions]) v, where groups (and causal order) allow; in training the
            gradients of q, k, v and of the table
Tables, gates and norm weights are shared, or there is one set per Monte-Carlo weight sample (samples > 0).  Sizes are those of the
package's workloads (ViT width 192 with 3 heads and 65 tokens an image, Swin width 540 over 7260 tokens, an MLP of width 128) and generic ones.

A kept element is one whose sixteen bits are below round(65536 keep): element c of row r of a sample takes bits 16 (c mod 2) .. of word
(c mod 8) / 2 of Philox-4x32-10 at counter (i, sample, step), i = 2^63 + offset + r ceil(width / 8) + c div 8, under the seed as its key.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5
STEP, FIRST, OFFSET = 7, 3, 4096

LARGEST_ROWS = 32768 * 8192                # elements of the largest block
LARGEST_PAIRS = 16 * 8192 * 8192 * 128     # heads x queries x keys x head width of the largest attention


def listed():
    return [
        # a hidden layer of the package's MLP under MC dropout, 16 passes at once: launches count
        {"name": "dropout_mlp", "kind": "dropout", "type": "f32", "samples": 16, "rows": 64, "width": 128, "keep": 0.9, "train": True},
        # an odd number of rows of an odd width
        {"name": "dropout_odd", "kind": "dropout", "type": "f16", "samples": 0, "rows": 10007, "width": 1531, "keep": 0.85, "train": True},
        # hidden states of 16 sequences of 2048 tokens
        {"name": "dropout_large", "kind": "dropout", "type": "bf16", "samples": 0, "rows": 32768, "width": 4096, "keep": 0.9, "train": True},
        # one token of a generated text: nothing but latency
        {"name": "block_one_token", "kind": "block", "type": "bf16", "samples": 0, "rows": 1, "width": 4096, "norm": "rms", "branch_norm": "", "gate": "", "scale": 1.0, "keep": 1.0, "train": False},
        # a ViT block over 256 images x 65 tokens, two weight samples with gates and norms of their own, MC dropout
        {"name": "block_vit_two_samples", "kind": "block", "type": "f32", "samples": 2, "rows": 16640, "width": 192, "norm": "layer", "branch_norm": "", "gate": "own", "scale": 1.0, "keep": 0.9, "train": True},
        # a norm on either side of the block, an odd number of rows of an odd width
        {"name": "block_odd", "kind": "block", "type": "f16", "samples": 0, "rows": 5003, "width": 777, "norm": "rms", "branch_norm": "rms", "gate": "", "scale": 0.5, "keep": 1.0, "train": True},
        # the largest: 16 sequences of 2048 tokens
        {"name": "block_large", "kind": "block", "type": "bf16", "samples": 0, "rows": 32768, "width": 8192, "norm": "rms", "branch_norm": "", "gate": "shared", "scale": 1.0, "keep": 0.9, "train": True},
        # Swin attention over 121 windows of 6 x 10 tokens, 6 heads of 90, a table for each of two weight samples; some windows hold pieces that are no neighbours
        {"name": "attention_swin", "kind": "attention", "type": "f32", "samples": 2, "batch": 121, "heads": 6, "kv_heads": 6, "queries": 60, "keys": 60, "width": 90, "positions": "6x10", "groups": "shifted", "causal": False, "train": True},
        # ViT attention over 256 images x 65 tokens
        {"name": "attention_vit", "kind": "attention", "type": "bf16", "samples": 0, "batch": 256, "heads": 3, "kv_heads": 3, "queries": 65, "keys": 65, "width": 64, "positions": "line 32 128", "groups": "", "causal": False, "train": True},
        # one new token of each of eight sequences over caches of up to 16384 tokens, four query heads to a key head
        {"name": "attention_one_token", "kind": "attention", "type": "bf16", "samples": 0, "batch": 8, "heads": 32, "kv_heads": 8, "queries": 1, "keys": 16384, "width": 128, "positions": "past 32 128", "groups": "cache", "causal": True, "train": False},
        # several texts packed into one row of an odd number of tokens
        {"name": "attention_packed", "kind": "attention", "type": "f16", "samples": 0, "batch": 2, "heads": 8, "kv_heads": 8, "queries": 3001, "keys": 3001, "width": 80, "positions": "line 64 512", "groups": "packed", "causal": True, "train": True},
        # the largest: a text of 8192 tokens, four query heads to a key head
        {"name": "attention_long", "kind": "attention", "type": "bf16", "samples": 0, "batch": 1, "heads": 16, "kv_heads": 4, "queries": 8192, "keys": 8192, "width": 128, "positions": "past 32 128", "groups": "", "causal": True, "train": True},
    ]


def _log_uniform(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _size(rng, low, high, step=8):
    n = _log_uniform(rng, low, high)
    return max(low, n // step * step) if rng.random() < 0.5 else n


def draw(rng):
    kind = rng.choice(["dropout", "block", "block", "attention", "attention", "attention"])
    kind_type = rng.choice(["f32", "bf16", "bf16", "f16"])
    samples = rng.randint(1, 8) if kind_type == "f32" and rng.random() < 0.5 else 0
    train = rng.random() < 0.8
    case = {"kind": kind, "type": kind_type, "samples": samples, "train": train}
    if kind != "attention":
        rows, width = _log_uniform(rng, 1, 32768), _size(rng, 8, 8192)
        rows = max(1, min(rows, LARGEST_ROWS // 4 // (width * max(1, samples))))
        case |= {"rows": rows, "width": width, "keep": rng.choice([1.0, 0.9, round(rng.uniform(0.5, 0.99), 3)]) if kind == "block" else round(rng.uniform(0.5, 0.99), 3)}
        if kind == "dropout":
            return case
        return {**case, "norm": rng.choice(["layer", "rms"]), "branch_norm": rng.choice(["", "", "layer", "rms"]), "gate": rng.choice(["", "shared", "own"]), "scale": rng.choice([1.0, 0.5, round(rng.uniform(0.1, 2.0), 2)])}
    width = rng.choice([16, 32, 64, 64, 80, 96, 128, 128, rng.randint(8, 128)])
    kv = rng.choice([1, 2, 3, 4, 6, 8])
    heads = kv * rng.choice([1, 1, 1, 2, 4])
    form = rng.choice(["window", "line", "line", "past", "token"])
    if form == "window":
        a, b = rng.randint(3, 12), rng.randint(3, 12)
        queries = keys = a * b
        case |= {"positions": "%dx%d" % (a, b), "groups": rng.choice(["", "shifted"]), "causal": False, "batch": _log_uniform(rng, 8, 512)}
    elif form == "token":
        case["train"] = False
        queries, keys = 1, _size(rng, 16, 16384)
        case |= {"positions": "past 32 128", "groups": rng.choice(["", "cache"]), "causal": True, "batch": _log_uniform(rng, 1, 32)}
    else:
        queries = keys = _size(rng, 16, 4096)
        if rng.random() < 0.25:
            queries = max(1, keys // rng.randint(2, 5))
        groups = rng.choice(["", "packed"]) if queries == keys else ""
        case |= {"positions": rng.choice(["line 32 128", "line 64 512"]) if form == "line" else "past 32 128", "groups": groups, "causal": form == "past" or rng.random() < 0.3, "batch": _log_uniform(rng, 1, 16)}
    most = LARGEST_PAIRS // (16 if kind_type == "f32" else 2)
    case["batch"] = max(1, min(case["batch"], most // (max(1, samples) * heads * queries * keys * width)))
    return {**case, "heads": heads, "kv_heads": kv, "queries": queries, "keys": keys, "width": width}


# --------------------------------------------------------------------------- inputs

def _line_buckets(distance, buckets, most, both):
    """Buckets of distances query - key: half of them one to a distance, the others wider and wider up to `most` and beyond."""
    if both:
        buckets //= 2
        side, away = (distance < 0).long() * buckets, distance.abs()
    else:
        side, away = torch.zeros_like(distance), distance.clamp(min=0)
    near = buckets // 2
    far = near + (torch.log(away.clamp(min=1).double() / near) / math.log(most / near) * (buckets - near)).long()
    return side + torch.where(away < near, away, far.clamp(max=buckets - 1))


def _positions(case):
    """(code of each query, of each key, bucket of every difference of codes from the smallest on, number of buckets): on the host."""
    text = case["positions"]
    if "x" in text:
        a, b = (int(n) for n in text.split("x"))
        code = (torch.arange(a)[:, None] * (2 * b - 1) + torch.arange(b)).reshape(-1)
        span = int(code[-1])
        return code, code, torch.arange(2 * span + 1), 2 * span + 1
    form, buckets, most = text.split()
    key = torch.arange(case["keys"])
    query = torch.arange(case["queries"]) + (case["keys"] - case["queries"] if case["causal"] else 0)
    distance = torch.arange(int(query[0]) - int(key[-1]), int(query[-1]) + 1)
    return query, key, _line_buckets(distance, int(buckets), int(most), form == "line"), int(buckets)


def _groups(case, g):
    """(group of each query, of each key), int32 [batch or windows, n], or None: pairs of one group see each other, negative ones nobody."""
    batch, nq, nk = case["batch"], case["queries"], case["keys"]
    if not case["groups"]:
        return None, None
    if case["groups"] == "shifted":         # the last windows of a row hold two pieces of the image
        piece = (torch.arange(nq, device=DEV) % max(1, nq // 4) >= max(1, nq // 8)).int()
        edge = (torch.arange(batch, device=DEV) % 11 == 10).int()
        both = piece * edge[:, None]
        return both, both
    if case["groups"] == "cache":           # texts of different lengths, padded in front: the new token's own entry is the last of each
        padding = (torch.rand(batch, 1, device=DEV, generator=g) * 0.75 * nk).long()
        keys = torch.where(torch.arange(nk, device=DEV) >= padding, 0, -1).int()
        return torch.zeros(batch, nq, dtype=torch.int32, device=DEV), keys
    # texts of different lengths one behind the other, the end of the row left over
    ends = torch.rand(batch, 7, device=DEV, generator=g).sort(1).values * 0.97 * nk
    at = torch.arange(nk, device=DEV).expand(batch, nk)
    group = torch.searchsorted(ends.contiguous(), at.float().contiguous(), right=True).int()
    group = torch.where(at < int(0.97 * nk) + 1, group, -1).int()
    return group, group


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    kind, dtype = case["kind"], TYPES[case["type"]]
    sets = (case["samples"],) if case["samples"] else ()
    state = {"case": case, "seed": (seed * 0x9E3779B97F4A7C15 + 12345) % 2 ** 64}

    def normal(*shape):
        return torch.randn(*shape, device=DEV, generator=g)

    if kind != "attention":
        rows, width = case["rows"], case["width"]
        # hidden states: a few loud channels, a mean per row
        loud = 1 + 4 * (torch.rand(width, device=DEV, generator=g) < 0.02)
        state["x"] = (normal(*sets, rows, width) * loud + 0.3 * normal(*sets, rows, 1)).to(dtype)
        if kind == "block":
            state["branch"] = (0.7 * normal(*sets, rows, width) + 0.1 * normal(width)).to(dtype)
            state["w"] = (1 + 0.2 * normal(*sets, width)).to(dtype)
            state["b"] = (0.1 * normal(*sets, width)).to(dtype) if case["norm"] == "layer" else None
            state["gate"] = (0.5 + 0.3 * normal(*(sets if case["gate"] == "own" else ()), width)).to(dtype) if case["gate"] else None
            state["bw"] = (1 + 0.2 * normal(*sets, width)).to(dtype) if case["branch_norm"] else None
            state["bb"] = (0.1 * normal(*sets, width)).to(dtype) if case["branch_norm"] == "layer" else None
            if case["train"]:
                state["dh"] = normal(*sets, rows, width).to(dtype)
        if case["train"]:
            state["dy"] = normal(*sets, rows, width).to(dtype)
        return state

    lead, width = (*sets, case["batch"]), case["width"]

    def heads(count, n, mean):
        """Heads side by side in a token's row, as a projection leaves them."""
        return (normal(*lead, n, count, width) + mean * normal(count, width)).to(dtype).transpose(-3, -2)

    state["q"], state["k"], state["v"] = heads(case["heads"], case["queries"], 0.5), heads(case["kv_heads"], case["keys"], 0.5), heads(case["kv_heads"], case["keys"], 0.3)
    if case["queries"] == 1:                # a cache: a head's keys behind one another
        state["k"], state["v"] = state["k"].contiguous(), state["v"].contiguous()
    query, key, bucket, buckets = _positions(case)
    state["table"] = (0.7 * normal(*sets, buckets, case["heads"])).to(dtype)
    state["query_groups"], state["key_groups"] = _groups(case, g)
    state["codes"] = (query.to(DEV), key.to(DEV), bucket.to(DEV), buckets)
    if own:
        from paper_2604_04736_amd import autograd as ops
        state["positions"] = ops.RelativePositions(query, key, bucket, buckets, DEV)
    if case["train"]:
        state["do"] = normal(*lead, case["queries"], case["heads"], width).to(dtype).transpose(-3, -2)
    return state


# --------------------------------------------------------------------------- the plain forms

def _mul_words(a, b):
    """High and low 32 bits of products of 32-bit numbers that int64 holds (the product's bits are right though its sign is not)."""
    p = a * b
    return (p >> 32) & 0xFFFFFFFF, p & 0xFFFFFFFF


def _philox(c0, c1, c2, c3, seed):
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for r in range(10):
        h0, l0 = _mul_words(c0, 0xD2511F53)
        h1, l1 = _mul_words(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ ((k0 + r * 0x9E3779B9) & 0xFFFFFFFF), l1, h0 ^ c3 ^ ((k1 + r * 0xBB67AE85) & 0xFFFFFFFF), l0
    return c0, c1, c2, c3


def _threshold(keep):
    return max(1, round(65536 * keep))


def _kept(case, seed):
    """Which elements stay: [samples or 1, rows, width]."""
    octets = -(-case["width"] // 8)
    at = OFFSET + torch.arange(case["rows"] * octets, device=DEV)[None]
    sample = FIRST + torch.arange(max(1, case["samples"]), device=DEV)[:, None]
    words = _philox(at & 0xFFFFFFFF, (at >> 32) | 0x80000000, sample, torch.full_like(sample, STEP), seed)
    halves = torch.stack([h for w in words for h in (w & 0xFFFF, w >> 16)], -1)
    kept = halves < _threshold(case["keep"])
    kept = kept.reshape(max(1, case["samples"]), case["rows"], octets * 8)[..., :case["width"]]
    return kept if case["samples"] else kept[0]


def _plain_dropout(s):
    case, dtype = s["case"], s["x"].dtype
    kept, up = _kept(case, s["seed"]), 65536 / _threshold(case["keep"])
    out = {"y": torch.where(kept, s["x"].float() * up, 0.0).to(dtype)}
    if case["train"]:
        out["dx"] = torch.where(kept, s["dy"].float() * up, 0.0).to(dtype)
    return out


def _normed(v, kind, w, b):
    """(result, normalised rows, 1 / scale of each row) of a norm."""
    centred = v - v.mean(-1, keepdim=True) if kind == "layer" else v
    r = torch.rsqrt((centred * centred).mean(-1, keepdim=True) + EPS)
    n = centred * r
    y = n * w.float().unsqueeze(-2)
    return (y if b is None else y + b.float().unsqueeze(-2)), n, r


def _normed_back(dy, kind, w, n, r):
    u = dy * w.float().unsqueeze(-2)
    c = (u * n).mean(-1, keepdim=True)
    return r * (u - n * c - u.mean(-1, keepdim=True)) if kind == "layer" else r * (u - n * c)


def _plain_block(s):
    case, dtype = s["case"], s["x"].dtype
    x, t = s["x"].float(), s["branch"].float()
    if case["branch_norm"]:
        t, tn, tr = _normed(t, case["branch_norm"], s["bw"], s["bb"])
    dropped = case["keep"] < 1
    if dropped:
        kept, up = _kept(case, s["seed"]), 65536 / _threshold(case["keep"])
        t = torch.where(kept, t * up, 0.0)
    gate = case["scale"] * (s["gate"].float().unsqueeze(-2) if s["gate"] is not None else torch.ones((), device=DEV))
    h = x + gate * t
    y, n, r = _normed(h, case["norm"], s["w"], s["b"])
    out = {"h": h.to(dtype), "y": y.to(dtype)}
    if not case["train"]:
        return out
    dy = s["dy"].float()
    out["dw"] = (dy * n).sum(-2).to(dtype)
    if s["b"] is not None:
        out["db"] = dy.sum(-2).to(dtype)
    dh = s["dh"].float() + _normed_back(dy, case["norm"], s["w"], n, r)
    out["dx"] = dh.to(dtype)
    if s["gate"] is not None:
        dgate = case["scale"] * (dh * t).sum(-2)
        out["dgate"] = (dgate.sum(0) if case["samples"] and case["gate"] == "shared" else dgate).to(dtype)
    dt = dh * gate
    if dropped:
        dt = torch.where(kept, dt * up, 0.0)
    if case["branch_norm"]:
        out["dbw"] = (dt * tn).sum(-2).to(dtype)
        if s["bb"] is not None:
            out["dbb"] = dt.sum(-2).to(dtype)
        dt = _normed_back(dt, case["branch_norm"], s["bw"], tn, tr)
    out["dbranch"] = dt.to(dtype)
    return out


def _visible(s):
    """Which keys a query may see: broadcastable to [samples, batch, 1, 1, queries, keys], or None."""
    case, may = s["case"], None
    if s["query_groups"] is not None:
        a, b = s["query_groups"], s["key_groups"]
        may = ((a[:, :, None] == b[:, None, :]) & (a >= 0)[:, :, None])[:, None, None]
    if case["causal"] and case["queries"] > 1:
        i, j = torch.arange(case["queries"], device=DEV)[:, None], torch.arange(case["keys"], device=DEV)
        before = j <= i + (case["keys"] - case["queries"])
        may = before if may is None else may & before
    return may


def _plain_attention(s):
    case, dtype = s["case"], s["q"].dtype
    kv, per = case["kv_heads"], case["heads"] // case["kv_heads"]
    scale = 1 / math.sqrt(case["width"])
    # [..., batch, kv heads, query heads of each, tokens, width]
    q, k, v = s["q"].float().unflatten(-3, (kv, per)), s["k"].float().unsqueeze(-3), s["v"].float().unsqueeze(-3)
    query, key, bucket, buckets = s["codes"]
    code = query[:, None] - key - (query.min() - key.max())
    wide = s["table"].float().movedim(-1, -2)[..., bucket]                         # [..., heads, codes]
    z = torch.matmul(q * scale, k.transpose(-1, -2))
    bias = wide[..., code].unflatten(-3, (kv, per))
    z += bias.unsqueeze(1) if case["samples"] else bias
    del bias
    may = _visible(s)
    if may is not None:
        z = z.masked_fill(~may, -math.inf)
    top = z.amax(-1, keepdim=True)
    p = torch.exp(z - torch.where(torch.isinf(top), 0.0, top))
    del z
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total > 0, total, 1.0)
    o = torch.matmul(p, v)
    out = {"o": o.flatten(-4, -3).to(dtype)}
    if not case["train"]:
        return out
    do = s["do"].float().unflatten(-3, (kv, per))
    out["dv"] = torch.matmul(p.transpose(-1, -2), do).sum(-3).to(dtype)
    ds = torch.matmul(do, v.transpose(-1, -2))
    ds -= (do * o).sum(-1, keepdim=True)
    ds *= p
    del p
    out["dq"] = (torch.matmul(ds, k) * scale).flatten(-4, -3).to(dtype)
    out["dk"] = (torch.matmul(ds.transpose(-1, -2), q).sum(-3) * scale).to(dtype)
    # over batch, then over pairs of one difference, then over differences of one bucket: long sums, in 64 bits
    db = ds.sum(-5, dtype=torch.float64).flatten(-4, -3).flatten(-2)               # [..., heads, pairs]
    del ds
    by_code = torch.zeros(*db.shape[:-1], bucket.numel(), dtype=torch.float64, device=DEV).index_add_(-1, code.reshape(-1), db)
    by_bucket = torch.zeros(*db.shape[:-1], buckets, dtype=torch.float64, device=DEV).index_add_(-1, bucket, by_code)
    out["dtable"] = by_bucket.movedim(-1, -2).to(dtype)
    return out


# --------------------------------------------------------------------------- the package's operators

def _own(s):
    from paper_2604_04736_amd import autograd as ops, binding
    case, train = s["case"], s["case"]["train"]
    rng = binding.hot_rng(seed=s["seed"], step=STEP, first_sample=FIRST) if case["kind"] != "attention" else None

    def leaves(*names):
        return {n: s[n].detach().requires_grad_(train) for n in names if s[n] is not None}

    if case["kind"] == "dropout":
        ins = leaves("x")
        outs, ups = {"y": ops.dropout(ins["x"], case["keep"], rng, samples=case["samples"], offset=OFFSET)}, [s.get("dy")]
    elif case["kind"] == "block":
        ins = leaves("x", "branch", "w", "b", "gate", "bw", "bb")
        h, y = ops.residual_norm(ins["x"], ins["branch"], ins["w"], ins.get("b"), norm=case["norm"], gate=ins.get("gate"), scale=case["scale"],
                                 branch_norm=case["branch_norm"] or None, branch_weight=ins.get("bw"), branch_bias=ins.get("bb"),
                                 keep=case["keep"], rng=rng, samples=case["samples"], offset=OFFSET, eps=EPS)
        outs, ups = {"h": h, "y": y}, [s.get("dh"), s.get("dy")]
    else:
        ins = leaves("q", "k", "v", "table")
        outs = {"o": ops.attention(ins["q"], ins["k"], ins["v"], ins["table"], s["positions"], causal=case["causal"],
                                   query_groups=s["query_groups"], key_groups=s["key_groups"])}
        ups = [s.get("do")]
    got = {n: t.detach() for n, t in outs.items()}
    if train:
        got |= {"d" + n: d for n, d in zip(ins, torch.autograd.grad(list(outs.values()), list(ins.values()), ups))}
    return got


def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    return _plain_dropout(state) if kind == "dropout" else _plain_block(state) if kind == "block" else _plain_attention(state)


# --------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    size = 4 if case["type"] == "f32" else 2
    sets, train = max(1, case["samples"]), case["train"]
    if case["kind"] == "dropout":
        n = sets * case["rows"] * case["width"]
        return {"bytes": n * size * (4 if train else 2), "flops": n * (4 if train else 2)}
    if case["kind"] == "block":
        n = sets * case["rows"] * case["width"]
        vectors = sets * case["width"] * sum([1, case["norm"] == "layer", bool(case["branch_norm"]), case["branch_norm"] == "layer"])
        vectors += (sets if case["gate"] == "own" else 1) * case["width"] if case["gate"] else 0
        # x, branch, h, y; dh, dy, dx, dbranch; the vectors and their gradients
        return {"bytes": (n * (8 if train else 4) + vectors * (2 if train else 1)) * size, "flops": n * (34 if train else 12)}
    batch, nq, nk, width = sets * case["batch"], case["queries"], case["keys"], case["width"]
    q, kv = batch * case["heads"] * nq * width, batch * case["kv_heads"] * nk * width
    buckets = _positions(case)[3]
    moved = (2 * q + 2 * kv) + (2 * q + 2 * kv if train else 0) + sets * buckets * case["heads"] * (2 if train else 1)
    first = nk - nq
    seen = nq * (first + 1 + nk) // 2 if case["causal"] and nq > 1 else nq * nk
    if case["groups"] == "cache":
        seen, moved = int(seen * 0.625), moved - int(2 * kv * 0.375)
    elif case["groups"] == "packed":
        seen //= 4
    return {"bytes": moved * size + (4 * case["batch"] * (nq + nk) if case["groups"] else 0), "flops": batch * case["heads"] * seen * width * (14 if train else 4)}


# --------------------------------------------------------------------------- in 64 bits

def _high_product(a, b):
    """(high, low) 32 bits of a times b from products of sixteen bits."""
    a1, a0, b1, b0 = a >> 16, a & 0xFFFF, b >> 16, b & 0xFFFF
    middle = a1 * b0 + ((a0 * b0) >> 16)
    other = a0 * b1 + (middle & 0xFFFF)
    return a1 * b1 + (middle >> 16) + (other >> 16), ((other & 0xFFFF) << 16) | ((a0 * b0) & 0xFFFF)


def _exact_kept(case, seed, sample):
    """Which elements of a sample stay, from the generator's definition."""
    octets = (case["width"] + 7) // 8
    i = torch.arange(case["rows"] * octets, device=DEV, dtype=torch.int64) + OFFSET
    x = [i % 2 ** 32, i // 2 ** 32 + 2 ** 31, torch.full_like(i, FIRST + sample), torch.full_like(i, STEP)]
    key = [seed % 2 ** 32, seed // 2 ** 32]
    for _ in range(10):
        (h0, l0), (h1, l1) = _high_product(x[0], 0xD2511F53), _high_product(x[2], 0xCD9E8D57)
        x = [h1 ^ x[1] ^ key[0], l1, h0 ^ x[3] ^ key[1], l0]
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    bits = torch.empty(case["rows"], octets * 8, dtype=torch.bool, device=DEV)
    most = max(1, round(65536 * case["keep"]))
    for c in range(8):
        bits[:, c::8] = ((x[c // 2] >> (16 * (c % 2))) % 65536 < most).reshape(case["rows"], octets)
    return bits[:, :case["width"]], 65536 / most


def _exact_norm(v, kind, w, b):
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    y = v / (v.square().mean(-1, keepdim=True) + EPS).sqrt() * w
    return y if b is None else y + b


def _exact_rows(case, s):
    sets = case["samples"]
    names = [n for n in ("x", "branch", "w", "b", "gate", "bw", "bb") if s.get(n) is not None]
    out, step = {}, max(1, 2 ** 25 // case["width"])
    vectors = [n for n in names if n not in ("x", "branch")]
    sums = {n: torch.zeros(s[n].shape, dtype=torch.float64, device=DEV) for n in vectors}
    wide = ["y"] + (["h"] if case["kind"] == "block" else []) + (["d" + n for n in names if n not in vectors] if case["train"] else [])
    for n in wide:
        out[n] = torch.empty(s["x"].shape, dtype=torch.float64, device=DEV)
    for k in range(max(1, sets)):
        mine = (lambda t: t[k]) if sets else (lambda t: t)
        kept, up = _exact_kept(case, s["seed"], k) if case["keep"] < 1 else (None, 1.0)
        for at in range(0, case["rows"], step):
            part = slice(at, at + step)
            ins = {n: (mine(s[n])[part] if n in ("x", "branch") else (s[n][k] if s[n].dim() == 2 else s[n])).double().requires_grad_(case["train"]) for n in names}
            drop = (lambda t: torch.where(kept[part], t * up, torch.zeros_like(t))) if kept is not None else (lambda t: t)
            if case["kind"] == "dropout":
                made = [("y", drop(ins["x"]), "dy")]
            else:
                t = _exact_norm(ins["branch"], case["branch_norm"], ins["bw"], ins.get("bb")) if case["branch_norm"] else ins["branch"]
                h = ins["x"] + drop(t) * case["scale"] * (ins["gate"] if "gate" in ins else 1.0)
                made = [("h", h, "dh"), ("y", _exact_norm(h, case["norm"], ins["w"], ins.get("b")), "dy")]
            for n, t, _ in made:
                mine(out[n])[part] = t.detach()
            if not case["train"]:
                continue
            grads = torch.autograd.grad([t for _, t, _ in made], list(ins.values()), [mine(s[d])[part].double() for _, _, d in made])
            for n, d in zip(ins, grads):
                if n in vectors:
                    (sums[n][k] if sums[n].dim() == 2 else sums[n]).add_(d)
                else:
                    mine(out["d" + n])[part] = d
    if case["train"]:
        out |= {"d" + n: v for n, v in sums.items()}
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] != "attention":
        return _exact_rows(case, s)
    heads, per, train = case["heads"], case["heads"] // case["kv_heads"], case["train"]
    lead = s["q"].shape[:-3]
    q, k, v = (s[n].reshape(-1, *s[n].shape[-3:]) for n in ("q", "k", "v"))
    table = s["table"] if case["samples"] else s["table"][None]
    query, key, bucket, buckets = s["codes"]
    which = bucket[(query[:, None] - key) - int(query.min() - key.max())]
    causal = torch.ones(case["queries"], case["keys"], dtype=torch.bool, device=DEV).tril(case["keys"] - case["queries"]) if case["causal"] else None
    o = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    if train:
        do = s["do"].reshape(q.shape)
        dq, dk, dv, dtable = (torch.zeros(t.shape, dtype=torch.float64, device=DEV) for t in (q, k, v, table))
        flat = which.reshape(-1)
    few = max(1, 2 ** 26 // (case["queries"] * case["keys"]))        # entries of the batch at once
    for first, last in [(at, min(at + few, end)) for end in range(case["batch"], q.shape[0] + 1, case["batch"]) for at in range(end - case["batch"], end, few)]:
        sample = first // case["batch"]
        entries = torch.arange(first, last, device=DEV)
        hidden = None
        if s["query_groups"] is not None:
            a, b = (s[n][entries % s[n].shape[0]] for n in ("query_groups", "key_groups"))
            hidden = (a[:, :, None] != b[:, None, :]) | (a < 0)[:, :, None]
        if causal is not None:
            hidden = ~causal if hidden is None else hidden | ~causal
        for head in range(heads):
            a, b, c = q[first:last, head].double(), k[first:last, head // per].double(), v[first:last, head // per].double()
            z = torch.matmul(a, b.transpose(1, 2)) / math.sqrt(case["width"]) + table[sample][:, head].double()[which]
            if hidden is not None:
                z = z.masked_fill(hidden, -math.inf)
            p = torch.softmax(z, -1).nan_to_num_(nan=0.0)
            del z
            o[first:last, head] = torch.matmul(p, c)
            if not train:
                continue
            up = do[first:last, head].double()
            dv[first:last, head // per] += torch.matmul(p.transpose(1, 2), up)
            dz = torch.matmul(up, c.transpose(1, 2))
            dz = p * (dz - (p * dz).sum(-1, keepdim=True))
            del p
            dq[first:last, head] = torch.matmul(dz, b) / math.sqrt(case["width"])
            dk[first:last, head // per] += torch.matmul(dz.transpose(1, 2), a) / math.sqrt(case["width"])
            dtable[sample][:, head] += torch.bincount(flat, weights=dz.sum(0).reshape(-1), minlength=buckets)
    out = {"o": o.reshape(*lead, *o.shape[1:])}
    if train:
        out |= {"dq": dq.reshape(s["q"].shape), "dk": dk.reshape(s["k"].shape), "dv": dv.reshape(s["v"].shape), "dtable": dtable if case["samples"] else dtable[0]}
    return out
