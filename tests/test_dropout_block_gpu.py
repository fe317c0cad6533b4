"""Dropout by the counter generator and a block's end (autograd.dropout, autograd.residual_norm, hot_dropout, hot_block_*) against plain forms in 64 bits, and a transformer block
of all of them."""
import math

import pytest
import torch

import block_util as U

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _ops():
    from paper_2604_04736_amd import autograd
    return autograd


def _rng(seed=11, step=3, first_sample=0):
    from paper_2604_04736_amd import binding as hot
    return hot.hot_rng(seed=seed, step=step, first_sample=first_sample)


def _randn(shape, kind, seed=0, mean=0.3):
    g = torch.Generator(device=DEV).manual_seed(seed + 13 * math.prod(shape) + len(shape))
    return (torch.randn(shape, device=DEV, generator=g) + mean).to(U.TYPES[kind])


# ------------------------------------------------------------------ dropout

@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape,samples", [((1, 1), 0), ((3, 7), 0), ((5, 8), 0), ((4, 9), 0), ((2, 3, 31), 2), ((3, 5, 64), 3), ((2, 2, 3, 257), 2), ((1, 4097), 0), ((300, 24), 0), ((2, 129, 1000), 2)])
def test_dropout_keeps_what_the_generator_says(kind, shape, samples):
    x = _randn(shape, kind)
    sets, width = samples or 1, shape[-1]
    rows = x.numel() // width // sets
    for keep, offset, rng in ((0.9, 0, _rng()), (0.25, 12345, _rng((1 << 63) + 5, (1 << 32) - 1, 7)), (1.0, 1 << 40, _rng()), (1e-9, 0, _rng())):
        mask, up = U.kept(rows, width, keep, rng.seed, rng.step, rng.first_sample, sets, offset)
        leaf = x.clone().requires_grad_()
        y = _ops().dropout(leaf, keep, rng, samples, offset)
        want = torch.where(mask.view(shape), x.double() * up, 0.0)
        if kind == "f16":                        # (half a step above 65504 and more is an infinity: keep of 2^-16 takes a 1.0 there)
            want = torch.where(want.abs() >= 65520, want.sign() * math.inf, want)
        U.within(y, want, U.rounded(want, x.dtype) + 2 * U.U32 * want.abs(), "y")            # (the factor and the product, and the result's own rounding)
        assert torch.equal(y == 0, ~mask.view(shape) | (x == 0))
        g = _randn(shape, kind, 5, 0.0)
        grad, = torch.autograd.grad(y, leaf, g, create_graph=True)
        assert torch.equal(grad, _ops().dropout(g, keep, rng, samples, offset))
    if keep == 1.0:
        assert torch.equal(y, x)


def test_dropout_of_gradients_of_gradients():
    x = _randn((6, 40), "f32").requires_grad_()
    y = _ops().dropout(x, 0.5, _rng())
    grad, = torch.autograd.grad((y ** 3).sum(), x, create_graph=True)
    second, = torch.autograd.grad(grad.sum(), x)
    up = (y / x).detach()
    torch.testing.assert_close(second, 6 * y.detach() * up ** 2, rtol=1e-5, atol=1e-6)


def test_dropout_is_one_mask_for_shards_and_layers():
    """The samples of two GPUs are those of one, layers that follow each other take disjoint parts of the generator's range, and how often elements stay is as asked."""
    ops = _ops()
    x = torch.ones(8, 50, 77, device=DEV)
    whole = ops.dropout(x, 0.7, _rng(), 8)
    halves = [ops.dropout(x[4 * i:4 * i + 4], 0.7, _rng(first_sample=4 * i), 4) for i in range(2)]
    assert torch.equal(torch.cat(halves), whole)
    calls = ops.dropout_calls(x, 8)
    assert calls == 50 * 10
    second = ops.dropout(x, 0.7, _rng(), 8, calls)
    both = torch.cat([x, x], 1)
    assert torch.equal(ops.dropout(both, 0.7, _rng(), 8)[:, 50:], second)
    assert not torch.equal(second, whole)
    n = 1 << 22
    share = float((ops.dropout(torch.ones(1024, n // 1024, device=DEV), 0.7, _rng()) != 0).double().mean())
    assert abs(share - round(65536 * 0.7) / 65536) < 6 * math.sqrt(0.21 / n)


def test_dropout_of_strange_tensors():
    ops = _ops()
    x = _randn((6, 10, 24), "bf16")
    assert torch.equal(ops.dropout(x.transpose(0, 1), 0.5, _rng()), ops.dropout(x.transpose(0, 1).contiguous(), 0.5, _rng()))
    assert torch.equal(ops.dropout(x[..., 1:18], 0.5, _rng()), ops.dropout(x[..., 1:18].contiguous(), 0.5, _rng()))
    flat = _randn((1 + 6 * 17,), "f16")
    for start in (0, 1):
        view = flat[start:start + 6 * 17].view(6, 17)
        assert torch.equal(ops.dropout(view, 0.5, _rng()), ops.dropout(view.clone(), 0.5, _rng()))
    assert ops.dropout(x[:0], 0.5, _rng()).shape == x[:0].shape
    y = torch.full((4, 9), math.nan, device=DEV)
    y[:, 0] = math.inf
    mask = U.kept(4, 9, 0.5, 11, 3)[0][0]
    out = ops.dropout(y, 0.5, _rng())
    assert not out[~mask].any() and torch.isnan(out[mask & torch.isnan(y)]).all()           # what is left out is a zero whatever it was
    single = _randn((9,), "f32")
    assert ops.dropout(single, 0.5, _rng()).shape == single.shape


def test_dropout_of_more_than_two_to_the_32_bytes():
    rows, width = 1 << 21, 1032                    # 2.16e9 elements, 4.3e9 bytes
    x = torch.ones(rows, width, device=DEV, dtype=torch.bfloat16)
    y = _ops().dropout(x, 0.5, _rng())
    for first in (0, rows // 2 + 3, rows - 5):
        mask, up = U.kept(5, width, 0.5, 11, 3, offset=first * (width // 8))
        assert torch.equal(y[first:first + 5], mask[0].to(torch.bfloat16) * up)


# ------------------------------------------------------------------ a block's end

def _block(x, branch, dh, dy, vectors, **rule):
    given = {n: t for n, t in vectors.items() if t is not None}
    leaves = {"x": x, "branch": branch, **given}
    leaves = {n: t.detach().clone().requires_grad_() for n, t in leaves.items()}
    h, y = _ops().residual_norm(leaves["x"], leaves["branch"], **{n: leaves[n] for n in given}, **rule)
    outs, ups = [h], [dh]
    if y is not None:
        outs.append(y)
        ups.append(dy)
    pairs = [(o, u) for o, u in zip(outs, ups) if u is not None]
    grads = torch.autograd.grad([o for o, _ in pairs], list(leaves.values()), [u for _, u in pairs], allow_unused=True)
    got = {"h": h.detach(), **({"y": y.detach()} if y is not None else {})}
    return got | {"d" + n: g for n, g in zip(leaves, grads)}


def _block_check(kind, samples, rows, width, norm, branch_norm=None, gate=False, vectors="own", shared=False, keep=1.0, scale=1.0, dh=True, dy=True, offset=0, seed=0):
    x, branch = _randn((samples, rows, width), kind, seed), _randn((samples, rows, width), kind, seed + 1, -0.2)
    vt = kind if vectors == "own" else "f32"
    shape = (width,) if shared else (samples, width)
    v = {"weight": _randn(shape, vt, 2, 1.0) if norm else None, "bias": _randn(shape, vt, 3) if norm == "layer" else None, "gate": _randn(shape, vt, 4, 0.5) if gate else None,
         "branch_weight": _randn(shape, vt, 5, 1.0) if branch_norm else None, "branch_bias": _randn(shape, vt, 6) if branch_norm == "layer" else None}
    if vectors == "none":
        v = dict.fromkeys(v)
    up_h = _randn(x.shape, kind, 7, 0.0) if dh else None
    up_y = _randn(x.shape, kind, 8, 0.0) if dy and norm else None
    rng = _rng()
    mask, up = U.kept(rows, width, keep, rng.seed, rng.step, 0, samples, offset) if keep < 1 else (None, 1.0)
    got = _block(x, branch, up_h, up_y, v, norm=norm, branch_norm=branch_norm, scale=scale, keep=keep, rng=rng if keep < 1 else None, samples=samples, offset=offset)
    want = U.block_plain(x, branch, up_h, up_y, norm, branch_norm, scale=scale, mask=mask, up=up, **v)
    for name, t in got.items():
        if t is not None:
            U.within(t, want[name][0], want[name][1], f"{name} {tuple(x.shape)} {kind} {norm} {branch_norm}")
        else:
            assert not want[name][0].any(), name
    return got


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("width", [1, 2, 7, 8, 9, 31, 64, 65, 127, 255, 256, 513, 768, 1000, 1023, 2048, 2049, 4096, 5001, 8191, 8192, 8193, 12345, 16384])
def test_block_widths(kind, width):
    for norm, branch_norm in (("layer", None), ("rms", "rms")):
        _block_check(kind, 1, 5, width, norm, branch_norm, gate=True)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("samples,rows", [(1, 1), (1, 3), (2, 1), (3, 17), (16, 2), (2, 700), (1, 5000)])
def test_block_rows_and_samples(kind, samples, rows):
    for shared in (False, True):
        _block_check(kind, samples, rows, 72, "layer", gate=True, shared=shared, keep=0.8)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("norm", ["layer", "rms", None])
@pytest.mark.parametrize("branch_norm", ["layer", "rms", None])
@pytest.mark.parametrize("vectors", ["own", "f32", "none"])
def test_block_forms(kind, norm, branch_norm, vectors):
    for keep, scale, gate, dh, dy in ((1.0, 1.0, False, True, True), (0.6, -0.5, True, True, True), (0.9, 2.0, True, False, True), (1.0, 0.25, False, True, False), (0.5, 0.0, True, True, True)):
        if not dh and not (dy and norm):
            continue
        _block_check(kind, 2, 9, 136, norm, branch_norm, gate, vectors, keep=keep, scale=scale, dh=dh, dy=dy, offset=1000)
        _block_check(kind, 2, 3, 100, norm, branch_norm, gate, vectors, keep=keep, scale=scale, dh=dh, dy=dy)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_block_rows_far_from_zero_and_alike(kind):
    """A row whose mean is far larger than its spread, and rows of one number: their norm is the bias."""
    x = torch.full((1, 3, 96), 5.0, device=DEV, dtype=U.TYPES[kind])
    h, y = _ops().residual_norm(x, torch.zeros_like(x))
    assert torch.equal(h, x) and not y.any()
    zero = torch.zeros_like(x, requires_grad=True)
    h, y = _ops().residual_norm(zero, zero, norm="rms", branch_norm="rms")
    grad, = torch.autograd.grad(y.sum(), zero)
    slope = 1e5 + 1e5 ** 0.5                 # (x's: 1 / sqrt(eps); the branch's: that squared; beyond fp16's largest number, 65504)
    assert not y.any() and (torch.isposinf(grad).all() if kind == "f16" else ((grad.double() - slope).abs() <= slope * (2 * U.HALF_UNIT[grad.dtype] + 16 * U.U32)).all())
    x = _randn((1, 4, 200), kind, 3, 100.0)
    v = dict.fromkeys(("weight", "bias", "gate", "branch_weight", "branch_bias"))
    branch, up = _randn(x.shape, kind, 4), _randn(x.shape, kind, 5)
    got, want = _block(x, branch, up, up, v, norm="layer"), U.block_plain(x, branch, up, up, "layer")
    for name, t in got.items():
        U.within(t, want[name][0], want[name][1], name)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_block_nothing_to_do_and_strange_tensors(kind):
    ops = _ops()
    x = torch.zeros(0, 24, device=DEV, dtype=U.TYPES[kind], requires_grad=True)
    w = torch.ones(24, device=DEV, dtype=U.TYPES[kind], requires_grad=True)
    h, y = ops.residual_norm(x, x, w)
    assert h.shape == y.shape == x.shape
    gx, gw = torch.autograd.grad(y.sum(), (x, w))
    assert gx.shape == x.shape and not gw.any()
    a, b, up = (_randn((10, 6, 25), kind, i) for i in range(3))
    w = _randn((24,), kind, 9)

    def run(a, b, up):
        leaf, wl = a.detach().requires_grad_(), w.clone().requires_grad_()
        h, y = ops.residual_norm(leaf, b, wl, keep=0.5, rng=_rng())
        return (h.detach(), y.detach(), *torch.autograd.grad(y, (leaf, wl), up))
    views = [t[..., 1:].transpose(0, 1) for t in (a, b, up)]                       # (strided, off their grid)
    for p, q in zip(run(*views), run(*(t.contiguous() for t in views))):
        assert torch.equal(p, q)
    flat = _randn((1 + 3 * 24,), kind)
    off = flat[1:].view(3, 24)                                                     # dense, but off the 16-byte grid
    for p, q in zip(run(off, off, off), run(off.clone(), off.clone(), off.clone())):
        assert torch.equal(p, q)
    leaf = _randn((4, 24), kind).requires_grad_()                                  # the same tensor twice: its gradient is the sum
    h, _ = ops.residual_norm(leaf, leaf, norm=None)
    assert torch.equal(torch.autograd.grad(h.sum(), leaf)[0], torch.full_like(leaf, 2.0))
    grad, = torch.autograd.grad(ops.residual_norm(leaf, leaf.detach())[1].sum(), leaf, create_graph=True)
    with pytest.raises(RuntimeError, match="differentiable once"):
        grad.sum().backward()


def test_block_gradients_against_differences():
    x, branch, dh, dy = (_randn((1, 3, 20), "f32", i) for i in range(4))
    v = {"weight": _randn((20,), "f32", 5, 1.0), "bias": _randn((20,), "f32", 6), "gate": _randn((20,), "f32", 7), "branch_weight": _randn((20,), "f32", 8, 1.0), "branch_bias": _randn((20,), "f32", 9)}
    got = _block(x, branch, dh, dy, v, norm="layer", branch_norm="rms", scale=0.7, keep=0.5, rng=_rng(), samples=1)
    mask, up = U.kept(3, 20, 0.5, 11, 3)

    def value(a):
        t = a["branch"] * (a["branch"].square().mean(-1, keepdim=True) + 1e-5).rsqrt() * a["branch_weight"] + a["branch_bias"]
        h = a["x"] + 0.7 * a["gate"] * torch.where(mask, t * up, 0.0)
        c = h - h.mean(-1, keepdim=True)
        y = c * (c.square().mean(-1, keepdim=True) + 1e-5).rsqrt() * a["weight"] + a["bias"]
        return (h * dh.double() + y * dy.double()).sum()
    base = {n: t.double() for n, t in {"x": x, "branch": branch, **v}.items()}
    g = torch.Generator(device=DEV).manual_seed(1)
    for name in base:
        way, step = torch.randn(base[name].shape, device=DEV, generator=g).double(), 1e-5
        slope = float((value({**base, name: base[name] + step * way}) - value({**base, name: base[name] - step * way})) / (2 * step))
        grad = got["d" + name].double()
        assert abs(float((grad * way).sum()) - slope) < 200 * U.U32 * float((grad * way).abs().sum()) + 1e-7, name


def test_block_is_the_same_twice_and_takes_a_capture():
    ops = _ops()
    x, branch, dh, dy = (_randn((4, 600, 200), "bf16", i) for i in range(4))
    v = {"weight": _randn((4, 200), "f32", 5, 1.0), "bias": _randn((4, 200), "f32", 6), "gate": _randn((200,), "f32", 7), "branch_weight": None, "branch_bias": None}
    rule = dict(norm="layer", scale=0.5, keep=0.9, rng=_rng(), samples=4)
    first = _block(x, branch, dh, dy, v, **rule)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        second = _block(x, branch, dh, dy, v, **rule)
    torch.cuda.current_stream().wait_stream(stream)
    assert all(torch.equal(first[n], second[n]) for n in first)
    leaves = {n: t.clone().requires_grad_() for n, t in {"x": x, "branch": branch, **v}.items() if t is not None}

    def step():
        h, y = ops.residual_norm(**leaves, **rule)
        z = ops.dropout(y, 0.5, _rng(), 4, 10 ** 6)
        return [h.detach(), z.detach(), *torch.autograd.grad([h, z], list(leaves.values()), [dh, dy])]
    with torch.cuda.stream(stream):
        step()
    torch.cuda.current_stream().wait_stream(stream)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = step()
        graphs.append((graph, held))
    for turn in range(4):
        with torch.no_grad():
            for t in leaves.values():
                t.mul_(1 + 0.01 * turn)
        for graph, _ in graphs:
            graph.replay()
        with torch.cuda.stream(stream):
            stream.wait_stream(torch.cuda.default_stream())
            fresh = step()
        torch.cuda.synchronize()
        for _, held in graphs:
            assert all(torch.equal(a, b) for a, b in zip(held, fresh))
    eager = ops.residual_norm(**leaves, **rule)
    with pytest.raises(RuntimeError, match="drop that graph first"), torch.cuda.graph(torch.cuda.CUDAGraph()):
        step()
    del eager


def test_the_binding_is_what_autograd_calls():
    from paper_2604_04736_amd import binding as hot
    x, branch, dh, dy = (_randn((2, 9, 40), "bf16", i) for i in range(4))
    w = _randn((2, 40), "f32", 5, 1.0)
    want = _block(x, branch, dh, dy, {"weight": w}, norm="rms", keep=0.5, rng=_rng(), samples=2)
    h, y, dx, dbranch = (torch.empty_like(x) for _ in range(4))
    stats, dw = torch.empty(2, 9, 4, device=DEV), torch.empty_like(w)
    rule = dict(weight=w, norm="rms", keep=0.5, rng=_rng())
    hot.hot_block_forward(x, branch, h, y, stats=stats, **rule)
    hot.hot_block_backward(x, branch, stats, dh, dy, dx, dbranch, {"weight": dw}, **rule)
    for name, t in (("h", h), ("y", y), ("dx", dx), ("dbranch", dbranch), ("dweight", dw)):
        assert torch.equal(t, want[name]), name
    out = torch.empty_like(x)
    hot.hot_dropout(_rng(), 0.5, x, out)
    assert torch.equal(out, _ops().dropout(x, 0.5, _rng(), 2))
    again = x.clone()
    hot.hot_dropout(_rng(), 0.5, again, again)                   # (y may be x)
    assert torch.equal(again, out)
    with pytest.raises(ValueError):
        hot.hot_dropout(_rng(), 0.5, x[0], out[0])
    with pytest.raises(TypeError):
        hot.hot_block_forward(x, branch[:, :4], h, y)


def test_refusals():
    ops, rng = _ops(), _rng()
    x = _randn((4, 6, 16), "bf16")
    w = torch.ones(16, device=DEV)
    for error, call in ((TypeError, lambda: ops.dropout(x, 0.5, None)), (TypeError, lambda: ops.dropout(x.double(), 0.5, rng)), (TypeError, lambda: ops.dropout(x.long(), 0.5, rng)),
                        (ValueError, lambda: ops.dropout(x, 0.0, rng)), (ValueError, lambda: ops.dropout(x, 1.1, rng)), (ValueError, lambda: ops.dropout(x, math.nan, rng)), (ValueError, lambda: ops.dropout(x, 0.5, rng, 3)),
                        (ValueError, lambda: ops.dropout(x, 0.5, rng, -1)), (ValueError, lambda: ops.dropout(x, 0.5, rng, 0, -1)), (ValueError, lambda: ops.dropout(x[..., :0], 0.5, rng)),
                        (ValueError, lambda: ops.dropout(x.view(-1)[0], 0.5, rng)),
                        (TypeError, lambda: ops.residual_norm(x, x.float())), (TypeError, lambda: ops.residual_norm(x, x.cpu())), (TypeError, lambda: ops.residual_norm(x, x, w.half())),
                        (TypeError, lambda: ops.residual_norm(x, x, w, w.bfloat16())), (ValueError, lambda: ops.residual_norm(x, x[:3])), (ValueError, lambda: ops.residual_norm(x, x, w[:8])),
                        (ValueError, lambda: ops.residual_norm(x, x, w.expand(4, 16))), (ValueError, lambda: ops.residual_norm(x, x, w.expand(3, 16), samples=4)), (ValueError, lambda: ops.residual_norm(x, x, norm="batch")),
                        (ValueError, lambda: ops.residual_norm(x, x, w, norm=None)), (ValueError, lambda: ops.residual_norm(x, x, branch_weight=w)), (ValueError, lambda: ops.residual_norm(x, x, keep=0.5)),
                        (TypeError, lambda: ops.residual_norm(x, x, keep=0.5, rng=3)), (ValueError, lambda: ops.residual_norm(x, x, scale=math.inf)), (ValueError, lambda: ops.residual_norm(x, x, eps=-1.0)),
                        (ValueError, lambda: ops.residual_norm(x, x, eps=math.nan)), (ValueError, lambda: ops.residual_norm(*(torch.zeros(1, 16385, device=DEV),) * 2)), (ValueError, lambda: ops.residual_norm(x, x, samples=3))):
        with pytest.raises(error):
            call()


# ------------------------------------------------------------------ together

@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_a_transformer_block_of_all_of_them(kind):
    """A pre-norm block over a few weight samples, with packed texts: attention, its projection, the block's end with dropout, two products, the end of the second half and dropout of what
    leaves it.  Every operator's results and gradients are compared with its plain form in 64 bits at the values that it was given."""
    ops, dt = _ops(), U.TYPES[kind]
    s, n, heads, kv, width = 2, 75, 4, 2, 16
    dim = heads * width
    g = torch.Generator(device=DEV).manual_seed(3)

    def weight(*shape):
        return (torch.randn(*shape, device=DEV, generator=g) / shape[-1] ** 0.5).to(dt).requires_grad_()
    x = torch.randn(s, n, dim, device=DEV, generator=g).to(dt).requires_grad_()
    wqkv, wo, wi, wj = weight(s, dim, (heads + 2 * kv) * width), weight(s, dim, dim), weight(s, dim, 2 * dim), weight(s, 2 * dim, dim)
    norms = [torch.ones(s, dim, device=DEV).requires_grad_(), torch.zeros(s, dim, device=DEV).requires_grad_()]
    p = ops.RelativePositions.distances(n, n, 8, 32, DEV)
    table = (0.5 * torch.randn(s, 8, heads, device=DEV, generator=g)).requires_grad_()
    group = (torch.arange(n, device=DEV) // 30).int()
    rng = _rng()
    leaves = [x, wqkv, wo, wi, wj, *norms, table]
    seen = {}

    def watch(name, inputs, outputs):
        seen[name] = (inputs, outputs, {})
        for kept, group_ in ((seen[name][2], inputs), (seen[name][2], outputs)):
            for m, t in group_.items():
                if t.requires_grad and not t.is_leaf:
                    t.register_hook(lambda grad, m=m, kept=kept: kept.__setitem__(m, grad))
        return list(outputs.values())

    def mine(t):
        return t.clone()                               # (a node of its own, so that its gradient is this operator's alone)
    # torch's batched product with weights as they lie: its backward forms transposed views of them, which stays in float32 here
    def product(a, w):
        return torch.stack([(a[i].float() @ w[i].float()).to(dt) for i in range(s)])
    y0, = [ops.residual_norm(x, torch.zeros_like(x), norms[0], norms[1], samples=s)[1]]
    qkv = product(y0, wqkv).view(s, n, heads + 2 * kv, width)
    q, k, v = mine(qkv[:, :, :heads].transpose(1, 2)), mine(qkv[:, :, heads:heads + kv].transpose(1, 2)), mine(qkv[:, :, heads + kv:].transpose(1, 2))
    table_in = mine(table)
    # one entry for each sample: [S, 1, heads, tokens, width] would do as well
    o, = watch("attention", {"q": q, "k": k, "v": v, "table": table_in}, {"o": ops.attention(q, k, v, table_in, p, causal=True, query_groups=group, key_groups=group)})
    a = mine(product(o.transpose(1, 2).reshape(s, n, dim), wo))
    x_in, vectors = mine(x), [mine(t) for t in norms]
    h, y = ops.residual_norm(x_in, a, *vectors, keep=0.9, rng=rng, samples=s)
    watch("block", {"x": x_in, "branch": a, "weight": vectors[0], "bias": vectors[1]}, {"h": h, "y": y})
    b = product(torch.nn.functional.gelu(product(y, wi)), wj)
    end, none = ops.residual_norm(h, b, norm=None, keep=0.9, rng=rng, samples=s, offset=ops.dropout_calls(x, s))
    assert none is None
    out = ops.dropout(end, 0.9, rng, s, 2 * ops.dropout_calls(x, s))
    up = torch.randn(out.shape, device=DEV, generator=g).to(dt)
    grads = torch.autograd.grad(out, leaves, up)
    assert all(t.shape == leaf.shape and torch.isfinite(t).all() and t.any() for t, leaf in zip(grads, leaves))

    (inputs, outputs, got) = seen["attention"]
    want = U.attention_plain(inputs["q"].detach(), inputs["k"].detach(), inputs["v"].detach(), got["o"], table.detach(), U.buckets_of(p, n, n), causal=True, query_groups=group[None], key_groups=group[None])
    for m, t in (("o", outputs["o"]), ("dq", got["q"]), ("dk", got["k"]), ("dv", got["v"]), ("dtable", got["table"])):
        U.within(t, want[m][0], want[m][1], m)
    (inputs, outputs, got) = seen["block"]
    mask, upby = U.kept(n, dim, 0.9, rng.seed, rng.step, 0, s)
    want = U.block_plain(inputs["x"].detach(), inputs["branch"].detach(), got["h"], got["y"], "layer", weight=norms[0].detach(), bias=norms[1].detach(), mask=mask, up=upby)
    for m, t in (("h", outputs["h"]), ("y", outputs["y"]), ("dx", got["x"]), ("dbranch", got["branch"]), ("dweight", got["weight"]), ("dbias", got["bias"])):
        U.within(t, want[m][0], want[m][1], m)
    # the last of a text alone, over the keys so far, is the whole call's row
    last = ops.attention(q[:, :, -1:], k, v, table_in, p, causal=True, first_query=n - 1, query_groups=group[-1:], key_groups=group)
    whole = U.attention_plain(q.detach(), k.detach(), v.detach(), None, table.detach(), U.buckets_of(p, n, n), causal=True, query_groups=group[None], key_groups=group[None])["o"]
    U.within(last, whole[0][:, :, -1:], whole[1][:, :, -1:], "last token")
