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
