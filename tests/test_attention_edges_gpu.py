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


def _positions(form, n):
    ops = _ops()
    if form == "window":
        return ops.RelativePositions.windows(n // 10, 10, device=DEV)
    if form == "line":
        return ops.RelativePositions.distances(n, n, 8, 30, DEV)
    if form == "one":                            # one bucket ahead, one behind
        return ops.RelativePositions(torch.arange(n), torch.arange(n), (torch.arange(2 * n - 1) >= n).long(), 8, DEV)
    g = torch.Generator().manual_seed(n)         # thousands of differences in a tile
    query, key = torch.randint(0, 60000, (n,), generator=g), torch.randint(0, 60000, (n,), generator=g)
    codes = int(query.max() - key.min() - (query.min() - key.max())) + 1
    return ops.RelativePositions(query, key, torch.randint(0, 8, (codes,), generator=g), 8, DEV)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("form", ["window", "line", "one", "any"])
@pytest.mark.parametrize("entries,heads,n", [(601, 8, 20), (514, 16, 20), (643, 4, 130)])
def test_workgroups_of_several_entries(kind, form, entries, heads, n):
    """More than 8192 tiles of queries: two or three entries one after the other in a workgroup, the last workgroup of each of two tables with fewer."""
    g = torch.Generator(device=DEV).manual_seed(entries + n)
    batch, width = 2 * entries, 24
    q, k, v, do = (torch.randn(batch, heads, n, width, device=DEV, generator=g).to(U.TYPES[kind]) for _ in range(4))
    p = _positions(form, n)
    which = U.buckets_of(p, n, n)
    table = (0.7 * torch.randn(2, p.buckets, heads, device=DEV, generator=g)).to(U.TYPES[kind])
    group = torch.randint(-1, 2, (entries, n), device=DEV, generator=g, dtype=torch.int32).sort(1).values
    for groups in ({}, {"query_groups": group, "key_groups": group}):
        leaves = [t.unflatten(0, (2, entries)).detach().requires_grad_() for t in (q, k, v)] + [table.detach().requires_grad_()]
        o = _ops().attention(*leaves, p, causal=n == 130, **groups)
        grads = torch.autograd.grad(o, leaves, do.unflatten(0, (2, entries)))
        want = U.attention_plain(q, k, v, do, table, which, causal=n == 130, **groups)
        for name, t in zip(("o", "dq", "dk", "dv", "dtable"), (o, *grads)):
            U.within(t if name == "dtable" else t.flatten(0, 1), *want[name], f"{name} {form} {kind}")
