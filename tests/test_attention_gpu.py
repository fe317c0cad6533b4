"""Attention with a learned position bias (autograd.attention, hot_attention_*) against the plain form in 64 bits: types, widths, lengths around every tile's limits, heads that
share keys, causal order, groups that leave rows empty, layouts, single tokens, streams and graphs, and gradients against differences."""
import math

import pytest
import torch

import block_util as U

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _ops():
    from paper_2604_04736_amd import autograd
    return autograd


def _inputs(kind, batch, heads, kv, nq, nk, width, seed=0, mean=0.5):
    g = torch.Generator(device=DEV).manual_seed(seed + 31 * nq + 7 * nk + width)

    def one(h, n):
        return (torch.randn(batch, h, n, width, device=DEV, generator=g) + mean * torch.randn(h, 1, width, device=DEV, generator=g)).to(U.TYPES[kind])
    return one(heads, nq), one(kv, nk), one(kv, nk), torch.randn(batch, heads, nq, width, device=DEV, generator=g).to(U.TYPES[kind])


def _table(kind, tables, buckets, heads, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed + buckets)
    return (0.7 * torch.randn(tables, buckets, heads, device=DEV, generator=g)).to(U.TYPES[kind])


def _pass(q, k, v, do, table=None, positions=None, **more):
    leaves = {"q": q, "k": k, "v": v, **({"table": table} if table is not None else {})}
    leaves = {n: t.detach().requires_grad_(do is not None) for n, t in leaves.items()}
    o = _ops().attention(leaves["q"], leaves["k"], leaves["v"], leaves.get("table"), positions, **more)
    got = {"o": o.detach()}
    if do is not None:
        got |= {"d" + n: t for n, t in zip(leaves, torch.autograd.grad(o, list(leaves.values()), do))}
    return got


def _check(q, k, v, do, table=None, positions=None, which=None, first_query=0, **more):
    if table is not None and which is None:
        which = U.buckets_of(positions, q.shape[2], k.shape[2], first_query)
    given = {**more, **({"first_query": first_query} if first_query else {})}
    samples = table is not None and table.shape[0] > 1
    if samples:                                             # (one table for each entry of the first axis)
        lead = (table.shape[0], q.shape[0] // table.shape[0])
        own = [t.unflatten(0, lead) if t is not None else None for t in (q, k, v, do)]
        got = _pass(*own, table, positions, **given)
        got = {n: t if n == "dtable" else t.flatten(0, 1) for n, t in got.items()}
    else:
        got = _pass(q, k, v, do, table[0] if table is not None else None, positions, **given)
        if "dtable" in got:
            got["dtable"] = got["dtable"][None]
    groups = {n: (t if t.dim() == 2 else t[None]) for n, t in more.items() if n.endswith("groups") and t is not None}
    want = U.attention_plain(q, k, v, do, table, which, more.get("scale"), more.get("causal", False), **groups)
    for name, t in got.items():
        U.within(t, want[name][0], want[name][1], f"{name} {tuple(q.shape)} {tuple(k.shape)} {q.dtype}")
    return got


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("width", [8, 9, 13, 16, 31, 32, 33, 48, 63, 64, 65, 80, 90, 96, 97, 104, 127, 128])
def test_widths(kind, width):
    p = _ops().RelativePositions.distances(70, 70, 16, 40, DEV)
    _check(*_inputs(kind, 2, 2, 2, 70, 70, width), _table(kind, 1, 16, 2), p)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("nq,nk", [(1, 1), (1, 2), (2, 1), (1, 31), (1, 32), (1, 33), (3, 64), (15, 65), (16, 16), (17, 17), (33, 100), (63, 63), (64, 64), (65, 65), (64, 129), (127, 127),
                                   (128, 128), (129, 130), (130, 64), (200, 7), (257, 300), (5, 700), (700, 5)])
def test_lengths(kind, nq, nk):
    for causal in (False, True):
        p = _ops().RelativePositions.distances(nq, nk, 12, 20, DEV, first_query=nk - nq)
        _check(*_inputs(kind, 2, 3, 3, nq, nk, 40), _table(kind, 1, 12, 3), p, causal=causal)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("heads,kv", [(1, 1), (4, 1), (6, 2), (8, 4), (12, 3)])
@pytest.mark.parametrize("nq,nk", [(1, 150), (4, 90), (70, 70), (140, 140)])
def test_heads_that_share_keys(kind, heads, kv, nq, nk):
    p = _ops().RelativePositions.distances(nq, nk, 8, 30, DEV, both_sides=False, first_query=nk - nq)
    _check(*_inputs(kind, 2, heads, kv, nq, nk, 64), _table(kind, 1, 8, heads), p, causal=True)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("table_kind", ["own", "f32"])
def test_a_table_for_every_weight_sample(kind, table_kind):
    for extent in ((3, 4), (6, 10), (12, 12), (2, 5, 7)):
        n = math.prod(extent)
        p = _ops().RelativePositions.windows(*extent, device=DEV)
        assert p.buckets == math.prod(2 * e - 1 for e in extent)
        _check(*_inputs(kind, 6, 2, 2, n, n, 30), _table(kind if table_kind == "own" else "f32", 3, p.buckets, 2), p)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("width", [16, 33, 64, 80, 96, 128])
@pytest.mark.parametrize("heads,kv,nq,nk", [(2, 2, 70, 70), (4, 2, 65, 200), (2, 1, 129, 129), (2, 2, 200, 150)])
def test_many_entries(kind, width, heads, kv, nq, nk):
    """Enough tiles for the larger ones (128 queries), whole and in part, with and without a table, order and groups."""
    batch = 264
    p = _ops().RelativePositions.distances(nq, nk, 16, 60, DEV, first_query=nk - nq if nk > nq else 0)
    inputs = _inputs(kind, batch, heads, kv, nq, nk, width)
    _check(*inputs, _table(kind, 2, 16, heads), p, causal=True)
    g = torch.Generator(device=DEV).manual_seed(nq)
    qg, kg = (torch.randint(-1, 3, (12, n), device=DEV, generator=g, dtype=torch.int32).sort(1).values for n in (nq, nk))
    _check(*inputs, query_groups=qg, key_groups=kg)
    window = _ops().RelativePositions.windows(10, 7, device=DEV) if nq == nk == 70 else None
    if window is not None:
        _check(*inputs, _table(kind, 1, window.buckets, heads), window)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_no_bias_and_other_scales(kind):
    for scale in (None, 0.0, -0.3, 1.0):
        _check(*_inputs(kind, 2, 2, 1, 66, 70, 24), **({"scale": scale} if scale is not None else {}))


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("spread", [1, 7, 40, 3000])
def test_codes_of_any_order(kind, spread):
    """Positions that are no line and no window: differences of few codes, of some hundred and of many thousand in a tile, and tokens that share a position."""
    g = torch.Generator().manual_seed(spread)
    nq, nk, buckets = 90, 150, 37
    query, key = torch.randint(0, 20 * spread, (nq,), generator=g), torch.randint(0, 20 * spread, (nk,), generator=g)
    codes = int(query.max() - key.min() - (query.min() - key.max())) + 1
    p = _ops().RelativePositions(query, key, torch.randint(0, buckets, (codes,), generator=g), buckets, DEV)
    _check(*_inputs(kind, 2, 2, 2, nq, nk, 32), _table(kind, 1, buckets, 2), p)
    ordered, _ = query.sort()
    p = _ops().RelativePositions(ordered, key.sort()[0], (torch.arange(codes) * buckets) // codes, buckets, DEV)
    _check(*_inputs(kind, 2, 2, 2, nq, nk, 32), _table(kind, 1, buckets, 2), p)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("buckets", [1, 2, 63, 65, 1023, 4096])
def test_few_and_many_buckets(kind, buckets):
    """As many as are allowed: the waves' own sums of them lie in LDS beside the tiles, of the widest rows too."""
    for nq, nk, width in ((60, 60, 24), (140, 200, 128)):
        codes = nq + nk - 1
        p = _ops().RelativePositions(torch.arange(nq), torch.arange(nk), (torch.arange(codes) * 67) % buckets, buckets, DEV)
        _check(*_inputs(kind, 2, 2, 1, nq, nk, width), _table(kind, 2, buckets, 2), p)


def _packed(batch, n, seed, holes=True):
    g = torch.Generator(device=DEV).manual_seed(seed)
    ends = torch.rand(batch, 4, device=DEV, generator=g).sort(1).values * n
    group = torch.searchsorted(ends.contiguous(), torch.arange(n, device=DEV).float().expand(batch, n).contiguous(), right=True).int()
    return torch.where(torch.rand(batch, n, device=DEV, generator=g) < 0.1, -1, group).int() if holes else group


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n", [20, 64, 90, 200, 450])
@pytest.mark.parametrize("causal", [False, True])
def test_groups(kind, n, causal):
    p = _ops().RelativePositions.distances(n, n, 16, 60, DEV)
    for holes in (False, True):
        group = _packed(3, n, n, holes)
        _check(*_inputs(kind, 6, 2, 2, n, n, 32), _table(kind, 2, 16, 2), p, causal=causal, query_groups=group, key_groups=group)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_rows_that_see_nothing_and_padding_that_is_no_number(kind):
    n, batch = 150, 3
    q, k, v, do = _inputs(kind, batch, 4, 2, n, n, 40)
    qg = torch.zeros(batch, n, dtype=torch.int32, device=DEV)
    kg = qg.clone()
    kg[0, 40:] = -1                       # padding behind
    kg[1, :130] = -5                      # padding in front: with causal order the first queries see nothing
    kg[2] = 9                             # keys of a group that no query has
    qg[0, 100:], qg[1, 7] = -1, -2
    for t, g in ((q, qg), (k, kg), (v, kg), (do, qg)):
        bad = (g < 0)[:, None, :, None].expand_as(t)
        t[bad] = float("nan")
        t[..., 1][bad[..., 1]] = float("inf")
    p = _ops().RelativePositions.distances(n, n, 8, 30, DEV)
    for causal in (False, True):
        got = _check(q, k, v, do, _table(kind, 1, 8, 4), p, causal=causal, query_groups=qg, key_groups=kg)
        for name in ("o", "dq"):
            assert not got[name][2].any() and not got[name][0][:, 100:].any() and not got[name][1][:, 7].any()
        for name in ("dk", "dv"):
            assert not got[name][2].any() and not got[name][0][:, 40:].any() and not got[name][1][:, :130].any()
    # key groups alone: every query is of group 0
    alone = _pass(*_inputs(kind, batch, 4, 2, n, n, 40), key_groups=kg.clamp(max=0))
    both = _pass(*_inputs(kind, batch, 4, 2, n, n, 40), key_groups=kg.clamp(max=0), query_groups=torch.zeros_like(qg))
    assert all(torch.equal(alone[n], both[n]) for n in alone)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_biases_that_mask(kind):
    """A bucket of -inf takes its keys out, one of the type's lowest value only where there are others; scores far from zero together keep their distances."""
    n = 80
    p = _ops().RelativePositions.distances(n, n, 8, 30, DEV)
    low = torch.finfo(U.TYPES[kind]).min
    for value in (-math.inf, low):
        table = _table(kind, 1, 8, 2)
        table[0, 4:, 0], table[0, 2, 1] = value, value                 # head 0: nothing ahead; head 1: some distances
        _check(*_inputs(kind, 2, 2, 2, n, n, 32), table, p)
    table = torch.full((1, 8, 2), low, device=DEV, dtype=U.TYPES[kind])   # all keys alike: the same as none
    got = _pass(*_inputs(kind, 2, 2, 2, n, n, 32), table[0], p)
    assert torch.isfinite(got["o"]).all() and torch.isfinite(got["dq"]).all() and torch.isfinite(got["dtable"]).all()
    table = torch.full((1, 8, 2), -math.inf, device=DEV, dtype=U.TYPES[kind])
    got = _pass(*_inputs(kind, 2, 2, 2, n, n, 32), table[0], p)
    assert all(not t.any() for t in got.values())
    table = _table(kind, 1, 8, 2) + 3000
    _check(*_inputs(kind, 2, 2, 2, n, n, 32), table, p)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_gradients_of_very_different_size(kind):
    """One row's gradient 2^20 times the others': sums of the others keep what float32 sums of them have."""
    n = 100
    q, k, v, do = _inputs(kind, 2, 2, 2, n, n, 32)
    do[:, :, 3] *= 2.0 ** (8 if kind == "f16" else 20)
    do[:, :, 4] *= 2.0 ** -12
    p = _ops().RelativePositions.distances(n, n, 8, 30, DEV)
    _check(q, k, v, do, _table(kind, 1, 8, 2), p)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("width", [40, 33])
def test_layouts(kind, width):
    """Heads side by side in a packed row, keys that all entries share, rows of odd pitch, elements that are not adjacent, tensors off their 16-byte and 4-byte grids."""
    n, batch, heads = 70, 3, 2
    q, k, v, do = _inputs(kind, batch, heads, heads, n, n, width)
    p = _ops().RelativePositions.distances(n, n, 8, 30, DEV)
    table = _table(kind, 1, 8, heads)
    want = _pass(q, k, v, do, table[0], p)

    def same(*tensors, reduce=lambda name, t: t):
        got = _pass(*tensors, table[0], p)
        for name in want:
            assert torch.equal(got[name], want[name]), name

    packed = torch.stack([q, k, v], 2).permute(0, 3, 2, 1, 4).contiguous()          # [batch, tokens, 3, heads, width]
    same(*(packed[:, :, i].transpose(1, 2) for i in range(3)), do.transpose(1, 2).contiguous().transpose(1, 2))
    leaf = packed.clone().requires_grad_()
    o = _ops().attention(*(leaf[:, :, i].transpose(1, 2) for i in range(3)), table[0], p)
    grad, = torch.autograd.grad(o, leaf, do)
    assert all(torch.equal(grad[:, :, i].transpose(1, 2), want["d" + m]) for i, m in enumerate("qkv"))

    def put(t, pitch, start, along=3):
        room = torch.full((batch, heads, n, pitch), float("nan"), device=DEV, dtype=t.dtype).flatten()
        room = torch.cat([room, room[:64]])[start:start + batch * heads * n * pitch].view(batch, heads, n, pitch)[..., :width]
        room.copy_(t)
        return room
    for pitch, start in ((width + 1, 0), (width + 2, 1), (64, 1), (64, 4), (64, 8), (41, 3)):
        same(put(q, pitch, start), put(k, pitch, start), put(v, pitch, start), put(do, pitch, start))
    for pitch, start in ((64, 1), (width + 1, 0)):                                  # one of them alone
        same(put(q, pitch, start), k, v, do)
        same(q, put(k, pitch, start), v, do)
        same(q, k, put(v, pitch, start), do)
        same(q, k, v, put(do, pitch, start))
    same(*(t.transpose(2, 3).contiguous().transpose(2, 3) for t in (q, k, v, do)))   # elements a row apart: copied
    # one set of keys for all entries: its gradient is the entries' sum
    got = _pass(q, k[:1].expand_as(k), v[:1].expand_as(v), do, table[0], p)
    each = _pass(q, k[:1].repeat(batch, 1, 1, 1), v[:1].repeat(batch, 1, 1, 1), do, table[0], p)
    assert all(torch.equal(got[m], each[m]) for m in got)
    leaf = k[:1].clone().requires_grad_()
    o = _ops().attention(q, leaf.expand_as(k), v, table[0], p)
    grad, = torch.autograd.grad(o, leaf, do)
    assert grad.shape == leaf.shape and torch.allclose(grad.float(), _pass(q, k[:1].repeat(batch, 1, 1, 1), v, do, table[0], p)["dk"].float().sum(0, keepdim=True), rtol=0.05, atol=0.05)
    # three axes, and five
    three = _ops().attention(q[0], k[0], v[0], table[0], p)
    assert torch.equal(three, want["o"][0])
    five = _ops().attention(*(t.unsqueeze(1) for t in (q, k, v)), table[0], p)
    assert torch.equal(five[:, 0], want["o"])
    # an upstream gradient of one number for all
    leaf = q.clone().requires_grad_()
    grad, = torch.autograd.grad(_ops().attention(leaf, k, v, table[0], p).sum(), leaf)
    assert torch.equal(grad, _pass(q, k, v, torch.ones_like(q), table[0], p)["dq"])


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_single_tokens_are_rows_of_the_whole(kind):
    """A text's tokens one by one over its keys so far, with one object of positions, against the rows of the whole causal call."""
    n, heads, kv = 100, 4, 2
    q, k, v, _ = _inputs(kind, 2, heads, kv, n, n, 64)
    p = _ops().RelativePositions.distances(n, n, 8, 30, DEV, both_sides=False)
    table = _table(kind, 1, 8, heads)
    which = U.buckets_of(p, n, n)
    whole = U.attention_plain(q, k, v, None, table, which, causal=True)["o"]
    for i in (0, 1, 30, 31, 32, 63, 64, 65, 99):
        o = _ops().attention(q[:, :, i:i + 1], k[:, :, :i + 1], v[:, :, :i + 1], table[0], p, first_query=i, causal=True)
        U.within(o, whole[0][:, :, i:i + 1], whole[1][:, :, i:i + 1], f"token {i}")
    for i in (10, 64, 90):                                  # several at once, from any one on
        o = _ops().attention(q[:, :, i:i + 10], k[:, :, :i + 10], v[:, :, :i + 10], table[0], p, first_query=i, causal=True)
        U.within(o, whole[0][:, :, i:i + 10], whole[1][:, :, i:i + 10], f"tokens from {i}")


def test_long_caches_are_split_and_joined():
    for kind, nk, heads, kv, rows in (("bf16", 9000, 8, 2, 1), ("f32", 5000, 2, 1, 3), ("f16", 4099, 3, 3, 40)):
        p = _ops().RelativePositions.distances(rows, nk, 32, 500, DEV, both_sides=False, first_query=nk - rows)
        kg = torch.zeros(2, nk, dtype=torch.int32, device=DEV)
        kg[1, :nk // 2 + 5] = -1
        _check(*_inputs(kind, 2, heads, kv, rows, nk, 128), _table(kind, 1, 32, heads), p, causal=True, key_groups=kg, query_groups=torch.zeros(2, rows, dtype=torch.int32, device=DEV))
        _check(*_inputs(kind, 1, heads, kv, rows, nk, 128), _table(kind, 1, 32, heads), p)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_long_texts_with_gradients(kind):
    """Far fields of one bucket, tiles along the diagonal and many tiles of 128 queries; packed texts too."""
    n, heads, kv = 2100, 32, 8
    p = _ops().RelativePositions.distances(n, n, 32, 128, DEV, both_sides=False)
    inputs = _inputs(kind, 1, heads, kv, n, n, 128)
    _check(*inputs, _table(kind, 1, 32, heads), p, causal=True)
    group = (torch.arange(n, device=DEV) // 700).int()
    _check(*inputs, _table(kind, 1, 32, heads), p, causal=True, query_groups=group[None], key_groups=group[None])


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_one_tensor_for_all_and_calls_at_once(kind):
    """q, k and v one tensor of three axes: its gradient is the sum of the three; and calls on several streams at the same time."""
    q, _, _, do = _inputs(kind, 1, 3, 3, 150, 150, 48)
    apart = _pass(q, q, q, do)
    leaf = q[0].clone().requires_grad_()
    grad, = torch.autograd.grad(_ops().attention(leaf, leaf, leaf), leaf, do[0])
    sizes = sum(apart[m].double().abs() for m in ("dq", "dk", "dv"))[0]
    assert ((grad.double() - (apart["dq"].double() + apart["dk"].double() + apart["dv"].double())[0]).abs() <= 2.02 * U.HALF_UNIT[grad.dtype] * sizes + U.TINY[grad.dtype]).all()      # (two additions)
    streams, results = [torch.cuda.Stream() for _ in range(3)], []
    torch.cuda.synchronize()
    for _ in range(5):
        for stream in streams:
            with torch.cuda.stream(stream):
                results.append(_pass(q, q, q, do))
    torch.cuda.synchronize()
    assert all(torch.equal(r[m], apart[m]) for r in results for m in apart)


def test_offsets_beyond_32_bits():
    """A cache of more than 2^32 bytes and 2^31 elements, of which only the last tokens are no padding."""
    nk, width = (1 << 24) + 77, 128
    k = torch.empty(1, 1, nk, width, dtype=torch.bfloat16, device=DEV)
    v = torch.empty_like(k)
    g = torch.Generator(device=DEV).manual_seed(1)
    last = 200
    k[:, :, :-last], v[:, :, :-last] = float("nan"), float("nan")
    k[:, :, -last:] = torch.randn(1, 1, last, width, device=DEV, generator=g).to(k.dtype)
    v[:, :, -last:] = torch.randn(1, 1, last, width, device=DEV, generator=g).to(k.dtype)
    q = torch.randn(1, 2, 1, width, device=DEV, generator=g).to(k.dtype)
    groups = torch.full((1, nk), -1, dtype=torch.int32, device=DEV)
    groups[:, -last:] = 0
    o = _ops().attention(q, k, v, key_groups=groups)
    want = U.attention_plain(q, k[:, :, -last:], v[:, :, -last:])["o"]
    U.within(o, want[0], want[1], "o")


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_nothing_to_do(kind):
    ops, dt = _ops(), U.TYPES[kind]
    p = ops.RelativePositions.distances(4, 4, 4, 8, DEV)
    for batch, nq, nk in ((2, 0, 4), (2, 4, 0), (0, 4, 4), (2, 0, 0)):
        q, k, v = (torch.randn(batch, 2, n, 16, device=DEV, dtype=dt, requires_grad=True) for n in (nq, nk, nk))
        table = torch.randn(4, 2, device=DEV, dtype=dt, requires_grad=True)
        o = ops.attention(q, k, v, table, p)
        assert o.shape == q.shape and not o.any()
        for t, grad in zip((q, k, v, table), torch.autograd.grad(o.sum(), (q, k, v, table))):
            assert grad.shape == t.shape and not grad.any()


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_the_same_twice_and_only_what_is_asked_for(kind):
    n = 300
    q, k, v, do = _inputs(kind, 2, 4, 2, n, n, 64)
    group = _packed(2, n, 3)
    p = _ops().RelativePositions.distances(n, n, 16, 60, DEV)
    table = _table(kind, 1, 16, 4)[0]
    more = dict(causal=True, query_groups=group, key_groups=group)
    first = _pass(q, k, v, do, table, p, **more)
    for _ in range(3):
        again = _pass(q, k, v, do, table, p, **more)
        assert all(torch.equal(first[m], again[m]) for m in first)
    with torch.no_grad():
        assert torch.equal(_ops().attention(q, k, v, table, p, **more), first["o"])
    for name in "qkv":
        leaves = {m: t.detach().requires_grad_(m == name) for m, t in zip("qkv", (q, k, v))}
        o = _ops().attention(leaves["q"], leaves["k"], leaves["v"], table, p, **more)
        assert torch.equal(torch.autograd.grad(o, leaves[name], do)[0], first["d" + name])
    leaf = table.detach().requires_grad_()
    assert torch.equal(torch.autograd.grad(_ops().attention(q, k, v, leaf, p, **more), leaf, do)[0], first["dtable"])
    leaf = q.detach().requires_grad_()
    grad, = torch.autograd.grad(_ops().attention(leaf, k, v, table, p, **more), leaf, do, create_graph=True)
    with pytest.raises(RuntimeError, match="differentiable once"):
        grad.sum().backward()


def test_gradients_against_differences():
    """float32, a window: central differences of sum(o do) along random directions, formed in 64 bits from the plain form's value at both ends."""
    p = _ops().RelativePositions.windows(4, 5, device=DEV)
    q, k, v, do = _inputs("f32", 2, 2, 1, 20, 20, 16)
    table = _table("f32", 1, p.buckets, 2)
    got = _pass(q, k, v, do, table[0], p)
    which = U.buckets_of(p, 20, 20)
    g = torch.Generator(device=DEV).manual_seed(5)
    for name, t in (("q", q), ("k", k), ("v", v), ("table", table)):
        way = torch.randn(t.shape, device=DEV, generator=g).double()
        step = 1e-5

        def value(s):
            moved = {"q": q.double(), "k": k.double(), "v": v.double(), "table": table.double()}
            moved[name] = moved[name] + s * way
            z = moved["q"] @ moved["k"].repeat_interleave(2, 1).transpose(-1, -2) / 4 + moved["table"][0][which].permute(2, 0, 1)
            return (torch.softmax(z, -1) @ moved["v"].repeat_interleave(2, 1) * do.double()).sum()
        slope = float((value(step) - value(-step)) / (2 * step))
        grad = got["d" + name].double().reshape(way.shape)
        # float32 gradients: some hundred roundings of terms of this size; the differences themselves are good to 1e-9 of it
        assert abs(float((grad * way).sum()) - slope) < 200 * 2.0 ** -24 * float((grad * way).abs().sum()) + 1e-7


def test_other_streams_and_a_captured_pass():
    ops = _ops()
    n = 200
    q, k, v, do = _inputs("bf16", 2, 4, 2, n, n, 64)
    p = ops.RelativePositions.distances(n, n, 16, 60, DEV)
    table = _table("bf16", 1, 16, 4)[0]
    want = _pass(q, k, v, do, table, p, causal=True)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        got = _pass(q, k, v, do, table, p, causal=True)
    torch.cuda.current_stream().wait_stream(stream)
    assert all(torch.equal(got[m], want[m]) for m in want)

    # two graphs of the same leaves, replayed in turn with new inputs and eager work between
    leaves = [t.detach().clone().requires_grad_() for t in (q, k, v, table)]
    up = do.clone()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for _ in range(2):
            torch.autograd.grad(ops.attention(*leaves[:3], leaves[3], p, causal=True), leaves, up)
    torch.cuda.current_stream().wait_stream(stream)
    graphs = []
    for causal in (True, False):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            o = ops.attention(*leaves[:3], leaves[3], p, causal=causal)
            grads = torch.autograd.grad(o, leaves, up)
        graphs.append((graph, causal, [o.detach(), *grads]))
        del o, grads
    for turn in range(4):
        with torch.no_grad():
            for t in leaves:
                t.add_(0.01 * turn)
        results = []
        for graph, causal, held in graphs:
            graph.replay()
            results.append([t.clone() for t in held])
        torch.cuda.synchronize()
        for (graph, causal, held), result in zip(graphs, results):
            fresh = _pass(*(t.detach() for t in leaves[:3]), up, leaves[3].detach(), p, causal=causal)
            for m, t in zip(("o", "dq", "dk", "dv", "dtable"), result):
                assert torch.equal(t, fresh[m]), (turn, causal, m)


def test_a_captured_pass_beside_a_graph_of_the_same_leaves_is_refused():
    ops = _ops()
    q, k, v, do = _inputs("bf16", 2, 4, 2, 70, 70, 64)
    leaves = [t.detach().requires_grad_() for t in (q, k, v)]
    eager = ops.attention(*leaves)
    with pytest.raises(RuntimeError, match="drop that graph first"), torch.cuda.graph(torch.cuda.CUDAGraph()):
        torch.autograd.grad(ops.attention(*leaves), leaves, do)
    with pytest.raises(RuntimeError, match="drop that graph first"), torch.cuda.graph(torch.cuda.CUDAGraph()):       # leaves further away
        torch.autograd.grad(ops.attention(leaves[0] * 2, k, v), leaves[0], do)
    want = _pass(q, k, v, do)
    assert torch.equal(torch.autograd.grad(eager, leaves, do)[1], want["dk"])
    del eager
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        grads = torch.autograd.grad(ops.attention(*leaves), leaves, do)
    for _ in range(2):
        graph.replay()
        assert torch.equal(grads[0], want["dq"]) and torch.equal(grads[1], want["dk"]) and torch.equal(grads[2], want["dv"])


def test_the_binding_is_what_autograd_calls():
    from paper_2604_04736_amd import binding as hot
    n = 130
    for kind in ("f32", "bf16"):
        q, k, v, do = _inputs(kind, 2, 4, 2, n, n, 40)
        p = _ops().RelativePositions.distances(n, n, 16, 60, DEV)
        table = _table(kind, 1, 16, 4)
        group = _packed(2, n, 1)
        want = _pass(q, k, v, do, table[0], p, query_groups=group, key_groups=group)
        codes = (p.query_code, p.key_code, p.query_range, p.key_range, p.bucket)
        o, rest = torch.empty_like(q), torch.empty_like(q) if kind != "f32" else None
        stats = torch.empty(2, 4, n, 2, device=DEV)
        rule = dict(scale=40 ** -0.5, query_groups=group, key_groups=group)
        hot.hot_attention_forward(q, k, v, o, table, codes, rest=rest, stats=stats, **rule)
        grads = {"grad_" + m: torch.full_like(t, 7.0) for m, t in (("q", q), ("k", k), ("v", v), ("table", table))}
        hot.hot_attention_backward(q, k, v, o, do, stats, rest, table, codes, **rule, **grads)
        assert torch.equal(o, want["o"])
        for m in ("q", "k", "v"):
            assert torch.equal(grads["grad_" + m], want["d" + m]), m
        assert torch.equal(grads["grad_table"][0], want["dtable"])
        with pytest.raises(ValueError):
            hot.hot_attention_forward(q, k[:, :, :5], v, o, scale=1.0)
        with pytest.raises(TypeError):
            hot.hot_attention_forward(q, k.double(), v, o, scale=1.0)


def test_refusals():
    ops = _ops()
    q, k, v, _ = _inputs("bf16", 2, 4, 2, 10, 12, 16)
    p = ops.RelativePositions.distances(10, 12, 4, 8, DEV)
    table = _table("bf16", 1, 4, 4)[0]
    groups = torch.zeros(2, 10, dtype=torch.int32, device=DEV), torch.zeros(2, 12, dtype=torch.int32, device=DEV)
    for error, call in ((TypeError, lambda: ops.attention(q, k.float(), v)), (TypeError, lambda: ops.attention(q.double(), k.double(), v.double())), (TypeError, lambda: ops.attention(q, k.cpu(), v)),
                        (TypeError, lambda: ops.attention(q, k, v, table)), (TypeError, lambda: ops.attention(q, k, v, table.half(), p)), (TypeError, lambda: ops.attention(q, k, v, table, "line")),
                        (TypeError, lambda: ops.attention(q, k, v, key_groups=groups[1].long())), (ValueError, lambda: ops.attention(q, k, v[:, :, :11])), (ValueError, lambda: ops.attention(q, k[:, :, :, :8], v)),
                        (ValueError, lambda: ops.attention(q[:1], k, v)), (ValueError, lambda: ops.attention(q[:, :3], k, v)), (ValueError, lambda: ops.attention(q[..., :7], k[..., :7], v[..., :7])),
                        (ValueError, lambda: ops.attention(*(torch.zeros(1, 1, 2, 129, device=DEV),) * 3)), (ValueError, lambda: ops.attention(q, k, v, table[:3], p)), (ValueError, lambda: ops.attention(q, k, v, table[:, :2], p)),
                        (ValueError, lambda: ops.attention(q, k, v, table.expand(3, 4, 4), p)), (ValueError, lambda: ops.attention(q, k, v, table, p, first_query=1)), (ValueError, lambda: ops.attention(q, k, v, table, p, first_query=-1)),
                        (ValueError, lambda: ops.attention(q, torch.cat([k, k], 2), torch.cat([v, v], 2), table, p)), (ValueError, lambda: ops.attention(q, k, v, query_groups=groups[0])),
                        (ValueError, lambda: ops.attention(q, k, v, key_groups=groups[0])), (ValueError, lambda: ops.attention(q, k, v, key_groups=torch.zeros(3, 12, dtype=torch.int32, device=DEV))),
                        (ValueError, lambda: ops.attention(q, k, v, scale=math.inf)), (ValueError, lambda: ops.attention(q, k, v, scale=math.nan)), (ValueError, lambda: ops.attention(q[0, 0], k[0, 0], v[0, 0]))):
        with pytest.raises(error):
            call()
