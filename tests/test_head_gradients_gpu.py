"""Gradients of the head's losses where operands share memory and where 16 bits are few: features expanded over weight samples, logits' gradients of
16-bit heads of many rows, rows of very different weights."""
import math

import pytest
import torch

import head_norm_util as U

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _ops():
    from paper_2604_04736_amd import autograd
    return autograd


def _loss(x, w, b, targets):
    if isinstance(targets, tuple):
        return _ops().head_distillation(x, w, *targets, bias=b, temperature=2.0)
    return _ops().head_cross_entropy(x, w, targets, bias=b)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("lists", [False, True])
@pytest.mark.parametrize("lead,width,vocab", [((12,), 8, 17), ((5, 14), 40, 300), ((3, 2, 50), 64, 2000)])
def test_features_expanded_over_samples(kind, lists, lead, width, vocab):
    """x.expand(S, ...) gives every sample's own gradient, and their sum where it was expanded from, as a copy of it does."""
    samples, dt = 3, U.TYPES[kind]
    g = torch.Generator(device=DEV).manual_seed(width + vocab)
    x = torch.randn(*lead, width, device=DEV, generator=g).to(dt)
    w = (torch.randn(samples, vocab, width, device=DEV, generator=g) * (2 / math.sqrt(width))).to(dt)
    b = torch.randn(samples, vocab, device=DEV, generator=g).to(dt)
    up = torch.rand(samples, *lead, device=DEV, generator=g) + 0.5
    if lists:
        targets = (torch.randint(-1, vocab, (*lead, 4), device=DEV, generator=g), torch.randn(*lead, 4, device=DEV, generator=g))
    else:
        targets = torch.randint(vocab, lead, device=DEV, generator=g)
    got = {}
    for name in ("expanded", "copied"):
        leaves = [t.detach().requires_grad_() for t in (x, w, b)]
        each = leaves[0].expand(samples, *lead, width)
        each = each.contiguous() if name == "copied" else each
        loss = _loss(each, leaves[1], leaves[2], targets)
        torch.empty(samples, *lead, width, dtype=dt, device=DEV).fill_(float("nan"))         # (what a gradient that is not written would hold)
        got[name] = [loss.detach(), *torch.autograd.grad(loss, [each, *leaves], up)]
    for n, a, c in zip(("loss", "dx of each sample", "dx", "dw", "db"), got["expanded"], got["copied"]):
        assert torch.equal(a, c), n
    teach = U.labels(targets.reshape(1, -1), vocab) if not lists else U.teacher(*(t.reshape(1, -1, 4) for t in targets), 2.0, vocab)
    x3 = x.reshape(1, -1, width).expand(samples, -1, -1)
    want = U.head_plain(x3, w, b, teach, up.reshape(samples, -1), 2.0 if lists else 1.0)["dx"]
    U.within(got["expanded"][1].reshape(x3.shape), *want, "dx of each sample")


def test_one_memory_for_all_samples_has_one_gradient():
    from paper_2604_04736_amd import binding as hot
    x, w = torch.randn(1, 6, 8, device=DEV), torch.randn(2, 9, 8, device=DEV)
    index, up = torch.zeros(1, 6, dtype=torch.long, device=DEV), torch.ones(2, 6, device=DEV)
    loss, lse = torch.empty(2, 6, device=DEV), torch.empty(2, 6, device=DEV, dtype=torch.float64)
    each = x.expand(2, 6, 8)
    hot.hot_head_forward(each, w, None, index, None, loss, lse)
    with pytest.raises(ValueError):
        hot.hot_head_backward(each, w, None, index, None, lse, up, dx=torch.empty(2, 6, 8, device=DEV))
    dw, again, dx = torch.empty_like(w), torch.empty_like(w), torch.empty_like(x)
    hot.hot_head_backward(each, w, None, index, None, lse, up, grad_weight=dw)          # (the weights' gradients need no copy)
    hot.hot_head_backward(x, w, None, index, None, lse, up, dx=dx, grad_weight=again)
    assert torch.equal(dw, again) and torch.isfinite(dx).all()


def _sixteen_bits(kind, rows, width, vocab, top, share, samples=0):
    """A case of which `share` of the rows count: x, w, b, targets, upstream gradients."""
    dt, g = U.TYPES[kind], torch.Generator(device=DEV).manual_seed(rows + vocab + top)
    sets = (samples,) if samples else ()
    x = torch.randn(*sets, rows, width, device=DEV, generator=g).to(dt)
    w = (torch.randn(*sets, vocab, width, device=DEV, generator=g) * (2 / math.sqrt(width))).to(dt)
    b = torch.randn(*sets, vocab, device=DEV, generator=g).to(dt)
    up = (torch.rand(*sets, rows, device=DEV, generator=g) + 0.5) * (64.0 if kind == "f16" else 1.0) / rows
    out = torch.randperm(rows, device=DEV, generator=g)[max(1, int(share * rows)):]
    if top:
        index = torch.randint(vocab, (rows, top), device=DEV, generator=g)
        index[out] = -1
        return x, w, b, (index, torch.randn(rows, top, device=DEV, generator=g) * 3), up
    target = torch.randint(vocab, (rows,), device=DEV, generator=g)
    target[out] = -100
    return x, w, b, target, up


# (rows, width, vocabulary, words listed, share of the rows that count, samples): small, middle and large tiles, runs of rows and of words, ten rows of many
MANY = [(40, 48, 900, 0, 1.0, 0), (64, 96, 2000, 16, 1.0, 2), (300, 64, 20000, 0, 1.0, 0), (520, 128, 9000, 40, 1.0, 0), (1100, 72, 3001, 5, 0.6, 3), (4096, 64, 3000, 0, 0.0025, 0),
        (2100, 264, 33001, 64, 1.0, 0), (3000, 40, 1200, 0, 1.0, 0)]


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("rows,width,vocab,top,share,samples", MANY)
def test_sixteen_bit_gradients_are_rounded_once(kind, rows, width, vocab, top, share, samples):
    """As far from 64 bits as what is rounded once at the end: what else goes into a gradient, dz's residual of 2^-16 (bf16) or 2^-22 and float32 logits, is
    below a tenth of that rounding, 1.005 of it in the root of a sum of squares; a rounding of dz to 16 bits would be 1.2 to 1.5."""
    x, w, b, targets, up = _sixteen_bits(kind, rows, width, vocab, top, share, samples)
    leaves = [t.detach().requires_grad_() for t in (x, w, b)]
    got = torch.autograd.grad(_loss(*leaves, targets), leaves, up)
    temperature = 2.0 if top else 1.0
    x3, w3, b2, up2 = (t if samples else t[None] for t in (x, w, b, up))
    spread, _, counts = U.teacher(*(t[None] for t in targets), temperature, vocab) if top else U.labels(targets[None], vocab)
    z = (x3.double() @ w3.double().transpose(1, 2).contiguous() + b2.double().unsqueeze(1)) / temperature
    dz = (torch.softmax(z, -1) - spread) * (up2.double() * counts * temperature).unsqueeze(-1)
    del z
    want = (dz @ w3.double(), dz.transpose(1, 2).contiguous() @ x3.double(), dz.sum(1))
    for n, a, c in zip(("dx", "dw", "db"), got, want):
        a, c = a.reshape(c.shape), c
        off, least = (a.double() - c).norm(), (c.to(a.dtype).double() - c).norm()
        assert off <= 1.02 * least, (n, float(off / least))


def test_rows_of_very_different_weights():
    """fp16 holds dz in steps of 2^-39 of the largest gradient: a row of a millionth of it keeps its likely words' bits, and no word is further off than half
    a step."""
    rows, width, vocab = 40, 32, 700
    x, w, b, target, up = _sixteen_bits("f16", rows, width, vocab, 0, 1.0)
    up = 64.0 * 10.0 ** torch.linspace(-6, 0, rows, device=DEV)
    leaf = x.detach().requires_grad_()
    (got,) = torch.autograd.grad(_loss(leaf, w, b, target), leaf, up)
    step = float(up.max()) * 2.0 ** -39
    for r in range(rows):
        want, bound = U.head_plain(x[r:r + 1][None], w[None], b[None], U.labels(target[r:r + 1][None], vocab), up[r:r + 1][None])["dx"]
        U.within(got[r:r + 1], want[0], bound[0] + 1.01 * step / 2 * w.double().abs().sum(0), f"row {r}")


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_weights_that_lie_between_each_other(kind):
    """Samples whose rows alternate in memory, and rows that are one row, give what copies of them give."""
    g = torch.Generator(device=DEV).manual_seed(1)
    x, target = torch.randn(2, 40, 32, device=DEV, generator=g).to(U.TYPES[kind]), torch.randint(90, (40,), device=DEV, generator=g)
    alternate = torch.randn(90, 2, 32, device=DEV, generator=g).to(U.TYPES[kind])
    one = alternate[:1, 0]
    for x, base, view in ((x, alternate, lambda t: t.permute(1, 0, 2)), (x[0], one, lambda t: t.expand(90, 32))):
        got = {}
        for name in ("as they lie", "copied"):
            leaves = [t.detach().requires_grad_() for t in (x, base)]
            w = view(leaves[1])
            loss = _loss(leaves[0], w if name == "as they lie" else w.contiguous(), None, target)
            got[name] = [loss.detach(), *torch.autograd.grad(loss.sum(), leaves)]
        assert all(torch.equal(a, c) for a, c in zip(*got.values()))


def test_no_rows_expanded_over_samples():
    base, drawn = torch.zeros(0, 8, device=DEV, requires_grad=True), torch.randn(2, 100, device=DEV, requires_grad=True)
    loss = _loss(base.expand(2, 0, 8), drawn[:, 3:75].unflatten(1, (9, 8)), None, torch.zeros(0, dtype=torch.long, device=DEV))
    dx, dw = torch.autograd.grad(loss.sum(), (base, drawn))
    assert loss.shape == (2, 0) and dx.shape == (0, 8) and not dw.any()
