"""Calls near the limits of the head's and the norm's sizes, where a launch of one workgroup to everything would pass a grid's 2^32 threads."""
import pytest
import torch

import head_norm_util as U

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _ops():
    from paper_2604_04736_amd import autograd
    return autograd


def test_lists_of_many_rows_of_many_samples():
    """2^26 lists, one for each of 64 samples' 2^20 rows."""
    samples, rows = 64, 1 << 20
    g = torch.Generator(device=DEV).manual_seed(3)
    x = torch.randn(rows, 1, device=DEV, generator=g).bfloat16()
    w = torch.randn(samples, 3, 1, device=DEV, generator=g).bfloat16()
    index = torch.randint(-1, 3, (samples, rows, 1), device=DEV, generator=g)
    got = _ops().head_distillation(x, w, index, torch.ones(1, device=DEV).expand(samples, rows, 1).contiguous())
    for s in (0, 1, 31, 62, 63):
        z = x.double() * w[s, :, 0].double()
        at = index[s]
        want = torch.where(at[:, 0] >= 0, (torch.logsumexp(z, 1, keepdim=True) - z.gather(1, at.clamp(min=0)))[:, 0], 0.0)
        # |z| below 2^5; a loss of a few additions of numbers of that size
        assert z.abs().max() < 32 and (got[s].double() - want).abs().max() < 16 * 32 * U.U32, s


def test_as_many_logits_as_a_call_takes():
    """float32, 2^20 rows and 2^18 words: more tiles than one launch holds."""
    rows, vocab = 1 << 20, 1 << 18
    g = torch.Generator(device=DEV).manual_seed(4)
    few = torch.randn(8, 1, device=DEV, generator=g)
    w = torch.randn(vocab, 1, device=DEV, generator=g)
    which = torch.randint(8, (rows,), device=DEV, generator=g)
    target = torch.randint(vocab, (rows,), device=DEV, generator=g)
    got = _ops().head_cross_entropy(few[which], w, target)
    z = few.double() @ w.double().T
    want = torch.logsumexp(z, 1)[which] - few.double()[which, 0] * w.double()[target, 0]
    # |z| below 2^5, logarithms of sums below 2^5: a few roundings of numbers of that size
    assert z.abs().max() < 32 and (got.double() - want).abs().max() < 32 * 32 * U.U32


def test_weights_gradients_of_the_widest_rows():
    """Two rows of 2^28 + 65 elements: more blocks of columns than one launch of a workgroup each holds."""
    width = (1 << 28) + 65
    g = torch.Generator(device=DEV).manual_seed(5)
    x = torch.randn(2, width, device=DEV, generator=g)
    w, b = torch.ones(width, device=DEV, requires_grad=True), torch.zeros(width, device=DEV, requires_grad=True)
    dy = torch.randn(2, width, device=DEV, generator=g)
    dw, db = torch.autograd.grad(_ops().layer_norm(x, w, b), (w, b), dy)
    stats = [(float(x[r].double().mean()), float((x[r].double().var(correction=0) + 1e-5).rsqrt())) for r in range(2)]
    for at in (slice(0, 1 << 20), slice((1 << 26) - 500, (1 << 26) + 500), slice(width - (1 << 20), width)):
        d = dy[:, at].double()
        h = torch.stack([(x[r, at].double() - stats[r][0]) * stats[r][1] for r in range(2)])
        # sums of 2^28 elements over 1024 threads, each a chain of 2^18: mean and variance good for 2^18 U32 of their terms at worst, and two rows
        off = (1 << 18) * U.U32
        U.within(dw[at], (d * h).sum(0), (d.abs() * (off * (1 + h.abs()) + 8 * U.U32 * h.abs())).sum(0) + 1e-30, "dw")
        U.within(db[at], d.sum(0), 4 * U.U32 * d.abs().sum(0) + 1e-30, "db")
