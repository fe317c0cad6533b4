"""How exact attention's results are where plain bounds, which add up every rounding with one sign, say little: long float32 texts."""
import math

import pytest
import torch

import block_util as U

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _ops():
    from paper_2604_04736_amd import autograd
    return autograd


@pytest.mark.parametrize("causal", [False, True])
def test_float32_tables_of_long_texts(causal):
    """The gradient of a float32 table over 4096 tokens whose values have a common part: what is off is D = do . o of each row, alike for all of its keys, so o's own roundings count.

    An addition is off by at most half a step of its result S, evenly spread: a variance of at most (2^-24 S)^2 / 3.  o is 128 sums of 32 keys added up, S growing in proportion: (2^-24 o)^2 times
    128 / 9, with 1/3 each for its scaling and its rounding.  D adds width terms of either sign in twelve steps: as much as 12 / 3 of the terms' squares.  A row's error goes to each bucket with the
    sum of p that the row has there; rows' errors are independent.  (dp's own roundings average out over a bucket's keys.)  The norm over 16 heads and 32 buckets varies by some tenth; half as much
    again is allowed.  One chain of all keys, four at a time, has 1024 / 9 in the place of 128 / 9: 2.5 times this."""
    n, heads, width, buckets = 4096, 16, 32, 32
    g = torch.Generator(device=DEV).manual_seed(11)
    q, k, do = (torch.randn(1, heads, n, width, device=DEV, generator=g) for _ in range(3))
    v = 3 + 0.1 * torch.randn(1, heads, n, width, device=DEV, generator=g)
    table = (0.5 * torch.randn(buckets, heads, device=DEV, generator=g)).requires_grad_()
    p = _ops().RelativePositions.distances(n, n, buckets, 512, DEV, both_sides=not causal)
    got, = torch.autograd.grad(_ops().attention(q, k, v, table, p, causal=causal), table, do)
    which = U.buckets_of(p, n, n)
    off = variance = size = 0.0
    for h in range(heads):
        qd, kd, vd, dod = (t[0, h].double() for t in (q, k, v, do))
        z = qd @ kd.T / math.sqrt(width) + table.detach()[:, h].double()[which]
        if causal:
            z = z.masked_fill(torch.ones(n, n, dtype=torch.bool, device=DEV).triu(1), -math.inf)
        w = torch.softmax(z, -1)
        o = w @ vd
        dp = dod @ vd.T
        dz = w * (dp - (w * dp).sum(-1, keepdim=True))
        want, shares = torch.zeros(buckets, dtype=torch.float64, device=DEV), torch.zeros(n, buckets, dtype=torch.float64, device=DEV)
        for b in range(buckets):
            there = which == b
            want[b], shares[:, b] = (dz * there).sum(), (w * there).sum(-1)
        d_variance = U.U32 ** 2 * (128 / 9 + 2 / 3 + 12 / 3) * (dod * o).square().sum(-1)
        variance += float((shares.square() * d_variance[:, None]).sum())
        off += float((got[:, h].double() - want).square().sum())
        size += float(want.square().sum())
    assert math.sqrt(off) <= 1.5 * math.sqrt(variance), (math.sqrt(off), math.sqrt(variance), math.sqrt(size))
