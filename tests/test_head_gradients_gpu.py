"""Gradients of the head's losses where operands share memory and where 16 bits are few: features expanded over weight samples."""
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
