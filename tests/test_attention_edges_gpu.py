"""Attention where other tests do not go: sides without tokens in groups."""
import pytest
import torch

import block_util as U

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _ops():
    from paper_2604_04736_amd import autograd
    return autograd


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("batch,nq,nk", [(2, 0, 4), (2, 4, 0), (0, 4, 4), (2, 0, 0), (2, 1, 0), (2, 0, 130), (2, 130, 0)])
@pytest.mark.parametrize("alone", [False, True])
def test_groups_of_nothing(kind, batch, nq, nk, alone):
    """A cache that is still empty, padding and all: zeros, and gradients of zeros."""
    ops, dt = _ops(), U.TYPES[kind]
    p = ops.RelativePositions.distances(130, 130, 4, 8, DEV)
    rows = max(batch, 1)
    q, k, v = (torch.randn(batch, h, n, 16, device=DEV, dtype=dt, requires_grad=True) for h, n in ((4, nq), (2, nk), (2, nk)))
    table = torch.randn(4, 4, device=DEV, dtype=dt, requires_grad=True)
    groups = {"key_groups": torch.zeros(rows, nk, dtype=torch.int32, device=DEV)}
    if not alone:
        groups["query_groups"] = torch.zeros(rows, nq, dtype=torch.int32, device=DEV)
    for causal in (False, True):
        o = ops.attention(q, k, v, table, p, causal=causal, **groups)
        assert o.shape == q.shape and not o.any()
        for t, grad in zip((q, k, v, table), torch.autograd.grad(o.sum(), (q, k, v, table))):
            assert grad.shape == t.shape and not grad.any()
        assert not ops.attention(q, k, v, causal=causal, **groups).any()
