"""No-GPU checks of the norm's and the head's entry points: scratch queries, refusals before anything is launched, structures as the header lays them
out, and that the product loops wait for memory once per tile."""
import ctypes
import os
import random
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def hot():
    from paper_2604_04736_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2604_04736_amd import build
        build.build_libhot()
    return binding


def _norm(hot, rows=4, width=8, samples=1, **more):
    d = hot.hot_norm_desc(rows, width, width, rows * width, width, rows * width, 0, 1e-5, samples, 0, 0, 0)
    for k, v in more.items():
        setattr(d, k, v)
    return d


def _head(hot, rows=4, width=8, vocab=16, samples=1, top=0, dtype=1, **more):
    own = samples > 1
    d = hot.hot_head_desc(rows, width, vocab, width, rows * width if own else 0, width, vocab * width if own else 0, vocab if own else 0, max(top, 1), 0, top, 0, -100, 1.0, top, samples,
                          dtype, 0, 1, 0)
    for k, v in more.items():
        setattr(d, k, v)
    return d


def test_structures_are_the_headers(tmp_path):
    from paper_2604_04736_amd import binding as hot
    src = tmp_path / "sizes.c"
    names = ("hot_norm_desc", "hot_head_desc")
    fields = [(n, f) for n in names for f, _ in getattr(hot, n)._fields_]
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "hot.h"\nint main(void) {\n' + "".join(f'printf("%zu\\n", sizeof({n}));\n' for n in names) +
                   "".join(f'printf("%zu\\n", offsetof({n}, {f}));\n' for n, f in fields) + "return 0;\n}\n")
    exe = str(tmp_path / "sizes")
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), "-o", exe, str(src)], check=True)
    got = [int(v) for v in subprocess.run([exe], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [ctypes.sizeof(getattr(hot, n)) for n in names] + [getattr(getattr(hot, n), f).offset for n, f in fields]


def test_scratch_of_many_shapes(hot):
    """Never negative for what the calls take, a multiple of 16, and of the size that the arrays in it need: the pieces of the vocabulary keep it
    from growing with the product of rows and words."""
    r = random.Random(3)
    for _ in range(3000):
        rows, width, vocab = int(2 ** r.uniform(0, 17)), int(2 ** r.uniform(0, 14)), int(2 ** r.uniform(0, 18))
        samples, top, dtype = r.choice([1, 1, 2, 16]), r.choice([0, 0, 1, 64, 1024]), r.choice([0, 1, 2])
        d = _head(hot, rows, width, vocab, samples, top, dtype)
        got = [hot.lib().hot_head_workspace_bytes(ctypes.byref(d), which) for which in (0, 1, 2)]
        assert all(n > 0 and n % 16 == 0 for n in got), (rows, width, vocab, samples, top, dtype, got)
        assert got[1] >= got[2] + samples * rows * width * 4
        pieces = 3 if dtype == 0 else 1
        places = (rows + 255) // 256 * 256
        fixed = samples * places * (width + 64) * 2 * pieces + samples * rows * (40 + top * 12) + samples * rows * (vocab // 64 + 8) * 2 + 65536
        least_piece = samples * 1280 * (places * 4 * max(2, pieces) + (width + 64) * 2 * pieces)
        runs = 1024 * 256 * 256 * 4                 # partial sums of the weights' gradients: at most two rounds of tiles, each four times over where they are cut
        assert got[2] <= fixed + max(least_piece, 300 << 20) + runs + samples * vocab * 4 * (places // 32 + 1), (rows, width, vocab, samples, top, dtype, got)
    for _ in range(2000):
        d = _norm(hot, int(2 ** r.uniform(0, 20)), int(2 ** r.uniform(0, 17)), r.choice([1, 3, 16]))
        n = hot.lib().hot_norm_backward_workspace_bytes(ctypes.byref(d))
        assert 0 < n <= max(4 * 256, d.samples) * 2 * d.width * 4 * 16 and n % (8 * d.width) == 0


def test_refusals_before_anything_is_launched(hot):
    lib, one = hot.lib(), 4096                       # (an address that nothing reads: every call below is refused)
    bad_norms = [dict(rows=-1), dict(width=0), dict(samples=0), dict(dtype=3), dict(weight_dtype=-1), dict(eps=-1.0), dict(eps=float("nan")), dict(w_sample=4), dict(ldx=-8)]
    for more in bad_norms:
        d = _norm(hot, **more)
        assert lib.hot_norm_forward(ctypes.byref(d), one, None, None, one, None, None, None) == hot.HOT_EINVAL, more
        assert lib.hot_norm_backward_workspace_bytes(ctypes.byref(d)) == hot.HOT_EINVAL
        assert lib.hot_norm_backward(ctypes.byref(d), one, None, one, one, one, one, None, None, None, 0, None) == hot.HOT_EINVAL
    d = _norm(hot)
    need = lib.hot_norm_backward_workspace_bytes(ctypes.byref(d))
    assert lib.hot_norm_forward(None, one, None, None, one, None, None, None) == hot.HOT_EINVAL
    for args in ((None, None, None, one, None, None), (one, None, None, None, None, None), (one + 2, None, None, one, None, None), (one, one + 1, None, one, None, None), (one, None, None, one, one, None)):
        assert lib.hot_norm_forward(ctypes.byref(d), *args, None) == hot.HOT_EINVAL, args
    for x, dw, ws, size in ((None, one, one, need), (one, one, None, need), (one, one, one, need - 1), (one, one, one + 2, need)):
        assert lib.hot_norm_backward(ctypes.byref(d), x, None, one, one, one, one, dw, None, ws, size, None) == hot.HOT_EINVAL

    bad_heads = [dict(rows=-1), dict(width=0), dict(vocab=0), dict(samples=0), dict(dtype=5), dict(ldw=4), dict(top=1025), dict(top=-1), dict(temperature=2.0), dict(rows=(1 << 20) + 1),
                 dict(width=(1 << 19) + 1), dict(vocab=(1 << 24) + 1), dict(rows=1 << 20, vocab=1 << 20), dict(top=2, temperature=0.0), dict(top=2, temperature=float("nan")),
                 dict(top=2, temperature=float("inf")), dict(top=2, logit_dtype=9), dict(ldx=-1), dict(samples=2, w_sample=0), dict(samples=2, w_sample=100), dict(samples=2, bias_sample=7)]
    for more in bad_heads:
        d = _head(hot, **{k: v for k, v in more.items() if k in ("rows", "width", "vocab", "samples", "top", "dtype")})
        for k, v in more.items():
            setattr(d, k, v)
        assert lib.hot_head_workspace_bytes(ctypes.byref(d), 0) == hot.HOT_EINVAL, more
        assert lib.hot_head_forward(ctypes.byref(d), one, one, None, one, one, one, one, one, 1 << 40, None) == hot.HOT_EINVAL, more
        assert lib.hot_head_backward(ctypes.byref(d), one, one, None, one, one, one, one, 0, 0, one, one, None, one, 1 << 40, None) == hot.HOT_EINVAL, more
    d = _head(hot)
    assert lib.hot_head_workspace_bytes(ctypes.byref(d), 3) == hot.HOT_EINVAL
    need = lib.hot_head_workspace_bytes(ctypes.byref(d), 0)
    good = dict(x=one, w=one, b=None, i=one, t=None, loss=one, lse=one, ws=one, size=need)
    for more in (dict(x=None), dict(w=None), dict(i=None), dict(loss=None), dict(ws=None), dict(size=need - 1), dict(x=one + 1), dict(w=one + 2), dict(b=one + 1), dict(i=one + 4), dict(loss=one + 2),
                 dict(lse=one + 4), dict(ws=one + 8)):
        a = {**good, **more}
        assert lib.hot_head_forward(ctypes.byref(d), a["x"], a["w"], a["b"], a["i"], a["t"], a["loss"], a["lse"], a["ws"], a["size"], None) == hot.HOT_EINVAL, more
    need = lib.hot_head_workspace_bytes(ctypes.byref(d), 1)
    good = dict(lse=one, g=one, gs=0, gr=1, dx=one, ws=one, size=need)
    for more in (dict(lse=None), dict(g=None), dict(g=one + 2), dict(gs=-1), dict(gr=-1), dict(dx=one + 1), dict(ws=None), dict(size=need - 1)):
        a = {**good, **more}
        assert lib.hot_head_backward(ctypes.byref(d), one, one, None, one, None, a["lse"], a["g"], a["gs"], a["gr"], a["dx"], None, None, a["ws"], a["size"], None) == hot.HOT_EINVAL, more
    # samples with one bias for all, lists without a teacher's logits
    d = _head(hot, samples=2)
    d.bias_sample = 0
    assert lib.hot_head_forward(ctypes.byref(d), one, one, one, one, None, one, one, one, 1 << 40, None) == hot.HOT_EINVAL
    d = _head(hot, top=2)
    assert lib.hot_head_forward(ctypes.byref(d), one, one, None, one, None, one, one, one, 1 << 40, None) == hot.HOT_EINVAL


def test_tensors_off_the_gpu_are_refused(hot):
    import torch
    from paper_2604_04736_amd import autograd
    x, w, t = torch.zeros(3, 4), torch.zeros(5, 4), torch.zeros(3, dtype=torch.long)
    for call in (lambda: autograd.layer_norm(x), lambda: autograd.head_cross_entropy(x, w, t), lambda: autograd.head_distillation(x, w, t[:, None], x[:, :1])):
        with pytest.raises(TypeError):
            call()


def test_product_loops_wait_once_for_a_tile(tmp_path):
    """The loop of every head kernel's product waits for memory once per tile, at its barrier: with the operands' arrays seen as possibly the same
    memory as the tile on its way, the compiler waited for that before every read of LDS (forward of 8192 x 4096 x 131072 6.4 -> 8.5 ms), and with
    registers spilled inside the loop it waits for those."""
    from paper_2604_04736_amd import build
    out = tmp_path / "head.s"
    src = [s for s in build.SRCS if s.endswith("head.hip")][0]
    subprocess.run([build.HIPCC] + build.FLAGS + ["-S", "--cuda-device-only", "-o", str(out), src], check=True, capture_output=True)
    text, loops = out.read_text(), 0
    for m in re.finditer(r"^(_Z\w+):[^\n]*\n(.*?)\.Lfunc_end", text, re.S | re.M):
        if "v_mfma" not in m.group(2) or re.search(r"ELi\d+ELi\d+ELi1ELb[01]ELb[01]EEE", m.group(1)):       # (one tile: no loop)
            continue
        blocks = re.split(r"^\.LBB\S+:", m.group(2), flags=re.M)
        at = [i for i, b in enumerate(blocks) if "v_mfma" in b]         # (where some waves load and others do not, the loop has branches)
        loop = "".join(blocks[at[0]:at[-1] + 1])
        waits = re.findall(r"s_waitcnt[^\n]*vmcnt\((\d+)\)", loop)
        assert len(waits) == 1 and len(re.findall(r"s_barrier", loop)) == 1 and "scratch_" not in loop, (m.group(1), waits)
        loops += 1
    assert loops >= 40
