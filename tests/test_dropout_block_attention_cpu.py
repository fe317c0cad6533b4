"""No-GPU checks of dropout's, the block's end's and attention's entry points: structures as the header lays them out, refusals before anything is launched, scratch queries of many
shapes, what an object of positions holds, and the plain generator against published values."""
import ctypes
import os
import random
import subprocess

import pytest
import torch

import block_util as U

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ONE = 4096                       # (an address that nothing reads: every call below is refused)


@pytest.fixture(scope="module")
def hot():
    from paper_2604_04736_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2604_04736_amd import build
        build.build_libhot()
    return binding


def test_structures_are_the_headers(tmp_path, hot):
    src = tmp_path / "sizes.c"
    names = ("hot_dropout_desc", "hot_block_desc", "hot_pitch", "hot_attention_desc")
    fields = [(n, f) for n in names for f, _ in getattr(hot, n)._fields_]
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "hot.h"\nint main(void) {\n' + "".join(f'printf("%zu\\n", sizeof({n}));\n' for n in names) +
                   "".join(f'printf("%zu\\n", offsetof({n}, {f}));\n' for n, f in fields) + "return 0;\n}\n")
    exe = str(tmp_path / "sizes")
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), "-o", exe, str(src)], check=True)
    got = [int(v) for v in subprocess.run([exe], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [ctypes.sizeof(getattr(hot, n)) for n in names] + [getattr(getattr(hot, n), f).offset for n, f in fields]


def test_the_plain_generator(hot):
    """Ten rounds of Philox 4x32 against its authors' known answers, through the octets' counters."""
    # counter and key all ones: the words 408f276d 41c83b0e a20bc7c6 6d5451fd
    ones = (1 << 32) - 1
    mask, up = U.kept(1, 8, 0.5, (1 << 64) - 1, ones, ones, 1, (1 << 63) - 1, device="cpu")
    words = (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)
    halves = [h for w in words for h in (w & 0xFFFF, w >> 16)]
    assert mask.flatten().tolist() == [h < 32768 for h in halves] and up == 2.0


def _block(hot, **more):
    d = hot.hot_block_desc(rows=4, width=8, scale=1.0, keep=1.0, eps=1e-5, samples=1, dtype=1, vector_dtype=1, norm=1, branch_norm=0)
    for k, v in more.items():
        setattr(d, k, v)
    return d


def _attention(hot, batch=2, heads=4, kv=2, queries=10, keys=12, width=16, dtype=1, **more):
    d = hot.hot_attention_desc()
    p = lambda h, n: hot.hot_pitch(h * n * width, n * width, width)      # noqa: E731
    d.batch, d.heads, d.kv_heads, d.queries, d.keys, d.width, d.dtype, d.table_dtype, d.scale = batch, heads, kv, queries, keys, width, dtype, dtype, 0.25
    for name in ("q", "o", "grad_o", "grad_q"):
        setattr(d, name, p(heads, queries))
    for name in ("k", "v", "grad_k", "grad_v"):
        setattr(d, name, p(kv, keys))
    for k, v in more.items():
        setattr(d, k, v)
    return d


def test_refusals_before_anything_is_launched(hot):
    lib = hot.lib()
    rng = hot.hot_rng(seed=1, step=0, first_sample=0)
    good = dict(rows=3, width=8, offset=0, keep=0.5, samples=1, dtype=0)
    for more in (dict(rows=-1), dict(width=0), dict(offset=-1), dict(keep=0.0), dict(keep=1.5), dict(keep=float("nan")), dict(samples=0), dict(dtype=3)):
        d = hot.hot_dropout_desc(**{**good, **more})
        assert lib.hot_dropout(ctypes.byref(d), ctypes.byref(rng), ONE, ONE, None) == hot.HOT_EINVAL, more
    d = hot.hot_dropout_desc(**good)
    for args in ((None, ctypes.byref(rng), ONE, ONE), (ctypes.byref(d), None, ONE, ONE), (ctypes.byref(d), ctypes.byref(rng), None, ONE), (ctypes.byref(d), ctypes.byref(rng), ONE, None),
                 (ctypes.byref(d), ctypes.byref(rng), ONE + 2, ONE)):
        assert lib.hot_dropout(*args, None) == hot.HOT_EINVAL

    def forward(d, **a):
        a = {**dict(x=ONE, b=ONE, w=None, bias=None, g=None, bw=None, bb=None, h=ONE, y=ONE, stats=ONE, rng=None), **a}
        return lib.hot_block_forward(ctypes.byref(d), a["rng"], a["x"], a["b"], a["w"], a["bias"], a["g"], a["bw"], a["bb"], a["h"], a["y"], a["stats"], None)
    for more in (dict(rows=-1), dict(width=0), dict(width=16385), dict(samples=0), dict(dtype=3), dict(vector_dtype=2), dict(norm=3), dict(norm=-1), dict(branch_norm=5), dict(keep=0.0), dict(keep=2.0),
                 dict(eps=-1.0), dict(eps=float("nan")), dict(scale=float("inf")), dict(weight_sample=-1), dict(offset=-1), dict(keep=0.5)):
        assert forward(_block(hot, **more)) == hot.HOT_EINVAL, more
        if "keep" not in more and "scale" not in more and "offset" not in more:
            assert lib.hot_block_backward_workspace_bytes(ctypes.byref(_block(hot, **more))) == hot.HOT_EINVAL or "eps" in more, more
    for more in (dict(x=None), dict(b=None), dict(h=None), dict(y=None), dict(x=ONE + 1), dict(stats=ONE + 2)):
        assert forward(_block(hot), **more) == hot.HOT_EINVAL, more
    d = _block(hot)
    need = lib.hot_block_backward_workspace_bytes(ctypes.byref(d))
    assert need > 0
    for stats, dw, ws, size in ((None, None, None, 0), (ONE, ONE, None, need), (ONE, ONE, ONE, need - 1), (ONE + 2, None, None, 0)):
        assert lib.hot_block_backward(ctypes.byref(d), None, ONE, ONE, ONE, None, None, None, stats, ONE, ONE, ONE, ONE, dw, None, None, None, None, ws, size, None) == hot.HOT_EINVAL

    for more in (dict(batch=-1), dict(heads=0), dict(kv_heads=0), dict(kv_heads=3), dict(width=7), dict(width=129), dict(dtype=3), dict(queries=-1), dict(keys=-1), dict(scale=float("nan")),
                 dict(groups=-1), dict(tables=3, buckets=4, codes=21), dict(tables=1, buckets=0, codes=21), dict(tables=1, buckets=4097, codes=21),
                 dict(tables=1, buckets=4, codes=0), dict(tables=1, buckets=4, codes=(1 << 22) + 1), dict(first_query=-1, tables=1, buckets=4, codes=21), dict(queries=1 << 31)):
        d = _attention(hot, **more)
        extra = (ONE,) * 6 if more.get("tables") else (None,) * 6
        groups = (ONE, ONE) if more.get("groups") else (None, None)
        assert lib.hot_attention_forward(ctypes.byref(d), ONE, ONE, ONE, *extra, *groups, ONE, None, None, ONE, 1 << 40, None) == hot.HOT_EINVAL, more
        assert lib.hot_attention_workspace_bytes(ctypes.byref(d), 0) == hot.HOT_EINVAL, more
    d = _attention(hot)
    assert lib.hot_attention_workspace_bytes(ctypes.byref(d), 2) == hot.HOT_EINVAL and lib.hot_attention_workspace_bytes(None, 0) == hot.HOT_EINVAL
    need = lib.hot_attention_workspace_bytes(ctypes.byref(d), 0)
    for q, k, v, o, ws, size in ((None, ONE, ONE, ONE, ONE, need), (ONE, None, ONE, ONE, ONE, need), (ONE, ONE, None, ONE, ONE, need), (ONE, ONE, ONE, None, ONE, need), (ONE + 1, ONE, ONE, ONE, ONE, need)):
        assert lib.hot_attention_forward(ctypes.byref(d), q, k, v, *(None,) * 8, o, None, None, ws, size, None) == hot.HOT_EINVAL
    with_table = _attention(hot, tables=2, buckets=4, codes=21)
    need = lib.hot_attention_workspace_bytes(ctypes.byref(with_table), 0)
    for ws, size, codes in ((None, need, (ONE,) * 5), (ONE, need - 1, (ONE,) * 5), (ONE + 8, need, (ONE,) * 5), *((ONE, need, (ONE,) * i + (None,) + (ONE,) * (4 - i)) for i in range(5)),
                            (ONE, need, (ONE + 2,) + (ONE,) * 4), (ONE, need, (ONE, ONE, ONE + 4, ONE, ONE)), (ONE, need, (ONE,) * 4 + (ONE + 4,))):
        assert lib.hot_attention_forward(ctypes.byref(with_table), ONE, ONE, ONE, ONE, *codes, None, None, ONE, None, None, ws, size, None) == hot.HOT_EINVAL, (ws, size, codes)
    need = lib.hot_attention_workspace_bytes(ctypes.byref(d), 1)
    assert need > 0
    for rest, stats, up, ws, size in ((ONE, None, ONE, ONE, need), (ONE, ONE, None, ONE, need), (ONE, ONE, ONE, None, need), (ONE, ONE, ONE, ONE, need - 1), (ONE, ONE + 2, ONE, ONE, need)):
        assert lib.hot_attention_backward(ctypes.byref(d), ONE, ONE, ONE, *(None,) * 8, ONE, rest, stats, up, ONE, ONE, ONE, None, ws, size, None) == hot.HOT_EINVAL


def test_scratch_of_many_shapes(hot):
    """Never negative for what the calls take, a multiple of 16, and no matrix of scores."""
    r = random.Random(5)
    for _ in range(3000):
        batch, kv, per = r.choice([1, 1, 2, 7, 64]), r.choice([1, 2, 8]), r.choice([1, 1, 4, 16])
        queries, keys, width, dtype = int(2 ** r.uniform(0, 14)), int(2 ** r.uniform(0, 18)), r.randint(8, 128), r.choice([0, 1, 2])
        heads = kv * per
        d = _attention(hot, batch, heads, kv, queries, keys, width, dtype)
        if r.random() < 0.5:
            d.tables, d.buckets, d.codes = 1, 32, min(queries + keys - 1, 1 << 22)
        d.causal = r.random() < 0.5
        rows = batch * heads * queries
        both = [hot.lib().hot_attention_workspace_bytes(ctypes.byref(d), which) for which in (0, 1)]
        assert all(n >= 0 and n % 16 == 0 for n in both), (batch, heads, kv, queries, keys, width, both)
        # the splits' parts: of so few rows that they fill the card a few times over; and what is kept for each row, key, bucket, difference and tile
        tiles, key_tiles = (queries + 15) // 16, (keys + 15) // 16
        small = 4 * (rows + batch * heads * keys) + 32 * (batch * (tiles + key_tiles)) + (d.codes * 8 * heads + 4096 * 8 * heads * (batch + 2048) if d.tables else 0) + 65536
        copies = 2 * 2 * batch * (2 * heads * queries + 2 * kv * keys) * (width + 8)
        parts = 4 * 2048 * 64 * 2 * (width + 2) * 4 + 4 * rows * (width + 2) * 16 + 8 * batch * heads * keys * width * 4 * 2
        assert all(n <= small + copies + parts for n in both), (batch, heads, kv, queries, keys, width, dtype, both)
    for _ in range(2000):
        d = _block(hot, rows=int(2 ** r.uniform(0, 20)), width=int(2 ** r.uniform(0, 14)), samples=r.choice([1, 3, 16]))
        n = hot.lib().hot_block_backward_workspace_bytes(ctypes.byref(d))
        assert 0 < n <= max(4 * 1024, d.samples * 2) * 5 * d.width * 4 * 2


def test_positions_hold_what_they_say():
    from paper_2604_04736_amd.autograd import RelativePositions
    for nq, nk, first, sides in ((5, 9, 4, True), (1, 200, 199, False), (130, 70, 0, True), (64, 64, 0, False)):
        p = RelativePositions.distances(nq, nk, 8, 30, "cpu", both_sides=sides, first_query=first)
        which = U.buckets_of(p, nq, nk)
        distance = torch.arange(nq)[:, None] + first - torch.arange(nk)
        assert which.shape == (nq, nk) and 0 <= int(which.min()) and int(which.max()) < 8
        side = 4 if sides else 8
        away = distance.abs() if sides else distance.clamp(min=0)
        near = side // 2
        assert torch.equal((which % side)[away < near], away[away < near]) and ((which % side)[away >= 30] == side - 1).all()
        if sides:
            assert torch.equal(which >= side, distance < 0)
        order = away.flatten().argsort()
        assert ((which % side).flatten()[order].diff() >= 0).all()                 # further away is never an earlier bucket
        # the last difference of every run, and whether a tile's codes are a line
        runs = p.bucket
        for c in range(0, len(runs), 7):
            end = int(runs[c, 1])
            assert (runs[c:end + 1, 0] == runs[c, 0]).all() and (end + 1 == len(runs) or runs[end + 1, 0] != runs[c, 0])
        assert p.query_range.shape == ((nq + 63) // 64, 4) and p.query_range[:, 2].all() and p.key_range[:, 2].all()
    p = RelativePositions.windows(3, 4, device="cpu")
    which = U.buckets_of(p, 12, 12)
    for i in range(12):
        for j in range(12):
            assert int(which[i, j]) == int(which[0, 0]) + (i // 4 - j // 4) * 7 + (i % 4 - j % 4)
    assert p.buckets == 35 and len(which.unique()) == 35
    shuffled = RelativePositions([5, 3, 9, 3], [2, 2], torch.arange(7) % 3, 3, "cpu")
    assert not shuffled.query_range[0, 2] and shuffled.query_range[0, :2].tolist() == [0, 6]


def test_refused_positions_and_tensors_off_the_gpu(hot):
    from paper_2604_04736_amd import autograd
    P = autograd.RelativePositions
    for call in (lambda: P([0, 1], [0], [0, 0, 0], 1, "cpu"), lambda: P([0, 1], [0], [0, 5], 5, "cpu"), lambda: P([0, 1], [0], [0, -1], 5, "cpu"), lambda: P([], [0], [0], 1, "cpu"),
                 lambda: P([0.5], [0], [0], 1, "cpu"), lambda: P([[0]], [0], [0], 1, "cpu"), lambda: P([0], [0, 1 << 40], [0], 1, "cpu"), lambda: P([0, 1], [0], [0, 0], 0, "cpu"),
                 lambda: P([0, 1], [0], [0, 0], 5000, "cpu"), lambda: P.distances(0, 3, 8, 30, "cpu"), lambda: P.distances(3, 3, 7, 30, "cpu"), lambda: P.distances(3, 3, 8, 2, "cpu"),
                 lambda: P.distances(3, 3, 2, 30, "cpu"), lambda: P.windows(device="cpu"), lambda: P.windows(0, 3, device="cpu"), lambda: P.windows(40, 60, device="cpu")):
        with pytest.raises(ValueError):
            call()
    x = torch.zeros(2, 3, 8)
    rng = hot.hot_rng(seed=1, step=0, first_sample=0)
    for call in (lambda: autograd.dropout(x, 0.5, rng), lambda: autograd.residual_norm(x, x), lambda: autograd.attention(x, x, x), lambda: autograd.attention(None, x, x),
                 lambda: autograd.attention(x, x, x, torch.zeros(3, 2), P.distances(3, 3, 4, 8, "cpu"))):
        with pytest.raises(TypeError):
            call()
