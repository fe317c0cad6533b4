"""How exact attention's results are where plain bounds, which add up every rounding with one sign, say little: long float32 texts, scores that lie far from zero together, small values in fp16."""
import math

import pytest
import torch

import block_util as U

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _ops():
    from paper_2604_04736_amd import autograd
    return autograd


@pytest.mark.parametrize("causal", [False, True])
def test_float32_tables_of_long_texts(causal):
    """The gradient of a float32 table over 4096 tokens whose values have a common part: what is off is D = do . o of each row, alike for all of its keys, so o's own roundings count.

    An addition is off by at most half a step of its result S, evenly spread: a variance of at most (2^-24 S)^2 / 3.  o is 128 sums of 32 keys added up, S growing in proportion: (2^-24 o)^2 times
    128 / 9, with 1/3 each for its scaling and its rounding.  D adds width terms of either sign in twelve steps: as much as 12 / 3 of the terms' squares.  A row's error goes to each bucket with the
    sum of p that the row has there; rows' errors are independent.  (dp's own roundings average out over a bucket's keys.)  The norm over 16 heads and 32 buckets varies by some tenth; half as much
    again is allowed.  One chain of all keys, four at a time, has 1024 / 9 in the place of 128 / 9: 2.5 times this."""
    n, heads, width, buckets = 4096, 16, 32, 32
    g = torch.Generator(device=DEV).manual_seed(11)
    q, k, do = (torch.randn(1, heads, n, width, device=DEV, generator=g) for _ in range(3))
    v = 3 + 0.1 * torch.randn(1, heads, n, width, device=DEV, generator=g)
    table = (0.5 * torch.randn(buckets, heads, device=DEV, generator=g)).requires_grad_()
    p = _ops().RelativePositions.distances(n, n, buckets, 512, DEV, both_sides=not causal)
    got, = torch.autograd.grad(_ops().attention(q, k, v, table, p, causal=causal), table, do)
    which = U.buckets_of(p, n, n)
    off = variance = size = 0.0
    for h in range(heads):
        qd, kd, vd, dod = (t[0, h].double() for t in (q, k, v, do))
        z = qd @ kd.T / math.sqrt(width) + table.detach()[:, h].double()[which]
        if causal:
            z = z.masked_fill(torch.ones(n, n, dtype=torch.bool, device=DEV).triu(1), -math.inf)
        w = torch.softmax(z, -1)
        o = w @ vd
        dp = dod @ vd.T
        dz = w * (dp - (w * dp).sum(-1, keepdim=True))
        want, shares = torch.zeros(buckets, dtype=torch.float64, device=DEV), torch.zeros(n, buckets, dtype=torch.float64, device=DEV)
        for b in range(buckets):
            there = which == b
            want[b], shares[:, b] = (dz * there).sum(), (w * there).sum(-1)
        d_variance = U.U32 ** 2 * (128 / 9 + 2 / 3 + 12 / 3) * (dod * o).square().sum(-1)
        variance += float((shares.square() * d_variance[:, None]).sum())
        off += float((got[:, h].double() - want).square().sum())
        size += float(want.square().sum())
    assert math.sqrt(off) <= 1.5 * math.sqrt(variance), (math.sqrt(off), math.sqrt(variance), math.sqrt(size))


def test_float32_keys_and_values_of_long_texts():
    """The gradients of keys and values that two heads of 4096 queries read, where what is added up has one sign: do and q have common parts, so that p do and (dp - D) q of a key do.

    As above: T = 2 x 4096 / 32 sums of 32 queries, growing in proportion, give a variance of (2^-24 dk)^2 T / 9; scaling and rounding at most a third each, and as much again for what p and dz are off,
    which is another number in every query and averages out.  Thousands of elements leave their norm no room; a fifth is allowed.  One chain, four queries at a time, has 2048 / 9 in the place of 256 / 9:
    2.7 times this."""
    n, batch, heads, kv, width = 4096, 2, 16, 8, 32
    g = torch.Generator(device=DEV).manual_seed(12)
    q, do = (3 + 0.1 * torch.randn(batch, heads, n, width, device=DEV, generator=g) for _ in range(2))
    k, v = (torch.randn(batch, kv, n, width, device=DEV, generator=g).requires_grad_() for _ in range(2))
    got = torch.autograd.grad(_ops().attention(q, k, v), (k, v), do)
    off, size = [0.0, 0.0], [0.0, 0.0]
    for b in range(batch):
        for h in range(kv):
            kd, vd, want = k.detach()[b, h].double(), v.detach()[b, h].double(), [0.0, 0.0]
            for i in (2 * h, 2 * h + 1):
                qd, dod = q[b, i].double(), do[b, i].double()
                w = torch.softmax(qd @ kd.T / math.sqrt(width), -1)
                dp = dod @ vd.T
                want[0] = want[0] + (w * (dp - (w * dp).sum(-1, keepdim=True))).T @ qd / math.sqrt(width)
                want[1] = want[1] + w.T @ dod
            for m in range(2):
                off[m] += float((got[m][b, h].double() - want[m]).square().sum())
                size[m] += float(want[m].square().sum())
    for m in range(2):
        assert math.sqrt(off[m] / size[m]) <= 1.2 * U.U32 * math.sqrt(2 * n / 32 / 9 + 4 / 3), (m, math.sqrt(off[m] / size[m]) / U.U32)


# ------------------------------------------------------------------ scores that lie far from zero together

SIZES = [(2, 80), (2, 300), (130, 129)]          # the last: enough tiles for the larger ones


def _inputs(kind, batch, n, width=32, heads=4, kv=2):
    g = torch.Generator(device=DEV).manual_seed(7 * n + width)
    return [torch.randn(batch, h, n, width, device=DEV, generator=g).to(U.TYPES[kind]) for h in (heads, kv, kv, heads)]


def _whole(kind, batch, n, width=16, heads=4, kv=2):
    """Queries and keys of small whole numbers: with SCALE scores are eighths in units of ln 2, and no sum of them or with a number of few bits is rounded."""
    g = torch.Generator(device=DEV).manual_seed(5 * n)
    q, k = (torch.randint(-2, 3, (batch, h, n, width), device=DEV, generator=g).to(U.TYPES[kind]) for h in (heads, kv))
    return [q, k] + [torch.randn(batch, h, n, width, device=DEV, generator=g).to(U.TYPES[kind]) for h in (kv, heads)]


SCALE = math.log(2) / 8


def _positions(form, n):
    ops = _ops()
    if form == "line":
        return ops.RelativePositions.distances(n, n, 8, 30, DEV)
    if form == "one":                            # a bucket for all
        return ops.RelativePositions(torch.arange(n), torch.arange(n), torch.zeros(2 * n - 1, dtype=torch.long), 8, DEV)
    g = torch.Generator().manual_seed(n)         # thousands of differences in a tile
    query, key = torch.randint(0, 60000, (n,), generator=g), torch.randint(0, 60000, (n,), generator=g)
    codes = int(query.max() - key.min() - (query.min() - key.max())) + 1
    return ops.RelativePositions(query, key, torch.randint(0, 8, (codes,), generator=g), 8, DEV)


def _pass(q, k, v, do, table=None, positions=None, **more):
    leaves = {"q": q, "k": k, "v": v, **({"table": table} if table is not None else {})}
    leaves = {n: t.detach().requires_grad_() for n, t in leaves.items()}
    o = _ops().attention(leaves["q"], leaves["k"], leaves["v"], leaves.get("table"), positions, **more)
    return {"o": o.detach(), **{"d" + n: t for n, t in zip(leaves, torch.autograd.grad(o, list(leaves.values()), do))}}


def _within(got, want):
    for name, t in got.items():
        t = t[None] if name == "dtable" else t
        U.within(t, *want[name], f"{name} {tuple(t.shape)} {t.dtype}")


def _alike(q, k, v, do, table, which, **more):
    """All scores that a row sees alike: the plain form with q = 0, and dk, which q itself goes into, with k = 0."""
    none = torch.zeros_like(table)[None]
    want = U.attention_plain(q * 0, k, v, do, none, which, **more)
    want["dk"] = U.attention_plain(q, k * 0, v, do, none, which, **more)["dk"]
    return want


@pytest.mark.parametrize("kind,table_kind,value", [("f32", "f32", -1e9), ("f32", "f32", None), ("bf16", "bf16", -1e9), ("bf16", "bf16", None), ("bf16", "f32", -1e9), ("bf16", "f32", None),
                                                   ("f16", "f32", -1e9), ("f16", "f32", None)])
@pytest.mark.parametrize("batch,n", SIZES)
@pytest.mark.parametrize("form", ["line", "one", "any"])
def test_rows_that_see_masked_keys_alone(kind, table_kind, value, batch, n, form):
    """A bias of -1e9, or of the type's lowest value, for every key that a row sees: float32 scores are then alike whatever q and k are, and so are the weights, forward and backward."""
    q, k, v, do = _inputs(kind, batch, n)
    p = _positions(form, n)
    value = torch.finfo(U.TYPES[table_kind]).min if value is None else value
    table = torch.full((8, 4), value, device=DEV, dtype=U.TYPES[table_kind])
    # half a step at 1.44e9 is 64 in units of ln 2
    assert float((q.float() @ k.repeat_interleave(2, 1).float().transpose(-1, -2)).abs().max()) / math.sqrt(32) * 1.4427 < 60
    which = U.buckets_of(p, n, n)
    group = (torch.arange(n, device=DEV) // 37).int()
    group[5:9] = -1
    for more in ({}, {"causal": True}, {"causal": True, "query_groups": group[None], "key_groups": group[None]}):
        _within(_pass(q, k, v, do, table, p, **more), _alike(q, k, v, do, table, which, **more))


@pytest.mark.parametrize("kind,table_kind", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f32")])
@pytest.mark.parametrize("batch,n", SIZES)
def test_rows_that_see_masked_keys_alone_beside_others(kind, table_kind, batch, n):
    """Causal order and distances 0 to 4 masked by the lowest value: rows 0 to 4 see masked keys alone, all others have some that are not."""
    q, k, v, do = _inputs(kind, batch, n)
    do[:, :, :5] *= 0.5                          # (fp16's pieces are in units of the largest row, which is then one of the others)
    p = _ops().RelativePositions(torch.arange(n), torch.arange(n), (torch.arange(2 * n - 1) - (n - 1) > 4).long(), 2, DEV)
    which = U.buckets_of(p, n, n)
    g = torch.Generator(device=DEV).manual_seed(n)
    table = torch.randn(2, 4, device=DEV, generator=g).to(U.TYPES[table_kind])
    table[0] = torch.finfo(table.dtype).min
    got = _pass(q, k, v, do, table, p, causal=True)
    masked = table.clone()
    masked[0] = -math.inf
    first, others = do.clone(), do.clone()
    first[:, :, 5:], others[:, :, :5] = 0, 0
    one = _alike(q, k, v, first, table, which, causal=True)
    two = U.attention_plain(q, k, v, others, masked[None], which, causal=True)
    want = {m: tuple(a + b for a, b in zip(one[m], two[m])) for m in ("dk", "dv", "dtable")}
    for m in ("o", "dq"):
        want[m] = tuple(torch.cat([a[:, :, :5], b[:, :, 5:]], 2) for a, b in zip(one[m], two[m]))
    _within(got, want)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("batch,n", SIZES)
@pytest.mark.parametrize("form", ["line", "one", "any"])
def test_a_bias_that_all_keys_share(kind, batch, n, form):
    """Scores of eighths and one bias for all: no score is rounded, so results are as near to 64 bits as without the bias, whatever its size."""
    q, k, v, do = _whole(kind, batch, n)
    p = _positions(form, n)
    which = U.buckets_of(p, n, n)
    want = U.attention_plain(q, k, v, do, torch.zeros(1, 8, 4, device=DEV), which, scale=SCALE)
    for value in (3000.0, -1e4, -65504.0, 1e5):
        _within(_pass(q, k, v, do, torch.full((8, 4), value, device=DEV), p, scale=SCALE), want)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("batch,n", SIZES)
@pytest.mark.parametrize("sign", [1, -1])
def test_products_that_all_keys_share(kind, batch, n, sign):
    """No bias, and one element of queries and keys that adds 8192 to every score (in units of ln 2): weights, and the gradients of everything else, are as without it."""
    q, k, v, do = _whole(kind, batch, n)
    q[..., 0], k[..., 0] = 256, 256 * sign
    plain_q, plain_k = q.clone(), k.clone()
    plain_q[..., 0], plain_k[..., 0] = 0, 0
    for causal in (False, True):
        want = U.attention_plain(plain_q, k, v, do, scale=SCALE, causal=causal)
        want["dk"] = U.attention_plain(q, plain_k, v, do, scale=SCALE, causal=causal)["dk"]
        _within(_pass(q, k, v, do, scale=SCALE, causal=causal), want)


@pytest.mark.parametrize("batch,n", SIZES)
@pytest.mark.parametrize("power", [11, 14])
def test_small_values_in_fp16(batch, n, power):
    """Values 2^power times smaller, few bits each so that all are there in fp16, under gradients 2^8 times as large: every gradient is 2^(8 - power) times that of the values as they were, and as near to it,
    though o and what its rounding leaves over end in steps of 2^-24.  A float32 table, whose gradient D's error goes into."""
    q, k, v, do = _inputs("f16", batch, n)
    v = (v * 8).round() / 8
    p = _positions("line", n)
    g = torch.Generator(device=DEV).manual_seed(n)
    table = torch.randn(8, 4, device=DEV, generator=g)
    want = U.attention_plain(q, k, v, do, table[None], U.buckets_of(p, n, n))
    got = _pass(q, k, v * 2.0 ** -power, do * 2.0 ** 8, table, p)
    for name in ("dq", "dk", "dtable"):
        # (fp16 results end in steps of 2^-24 too)
        value, bound = want[name]
        step = 0.0 if name == "dtable" else 2.0 ** (-25 + power - 8)
        U.within((got[name][None] if name == "dtable" else got[name]).double() * 2.0 ** (power - 8), value, bound + step, name)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("width", [8, 33, 64, 96, 128])
@pytest.mark.parametrize("batch,n", [(4, 3), *SIZES])
def test_weights_of_the_backward_pass_add_up_to_one(kind, width, batch, n):
    """Scores that a shared bias rounds to steps of 128 (in units of ln 2), steps up to 2^128 in a weight: every kernel forms the same ones.  The sum of dv over the keys is that of do over the queries."""
    nk = max(n, 300)
    g = torch.Generator(device=DEV).manual_seed(width + n)
    q, k, v, do = (s * torch.randn(batch, h, m, width, device=DEV, generator=g) for s, h, m in ((4, 4, n), (1, 2, nk), (1, 2, nk), (1, 4, n)))
    q, k, v, do = (t.to(U.TYPES[kind]) for t in (q, k, v, do))
    p = _ops().RelativePositions.distances(n, nk, 8, 30, DEV)
    held = {"f32": 0.0, "bf16": 2.0 ** -16, "f16": 2.0 ** -21}[kind]
    for bias in (-1e9, -1e6, 3e5):
        got = _pass(q, k, v, do, torch.full((8, 4), bias, device=DEV), p, scale=1.0)
        assert all(torch.isfinite(t).all() for t in got.values())
        up = do.double().unflatten(1, (2, 2))
        dv = got["dv"].double()
        # dv's own roundings, those of p (its pieces, 2^x, and the sum of all keys), and the additions
        bound = 1.01 * U.HALF_UNIT[U.TYPES[kind]] * dv.abs().sum(2) + nk * U.TINY[U.TYPES[kind]] + (held + (nk + 72 + 2 * n + 64) * U.U32) * up.abs().sum((2, 3))
        U.within(dv.sum(2), up.sum((2, 3)), bound, f"{kind} {bias}")
