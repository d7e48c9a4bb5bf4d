"""GPU: many tokens of small weights beside one of a large weight (a first token
that draws most of the attention).  Each weight is far below the largest, their
sum is not; rounding them to the cache's type must not lose it."""
import pytest
import torch

import kv_ref
from paper_2607_21686_gb300 import pcs
from test_gpu_attend import TYPES, attend

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("new", [1, 17])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("below", [14.2, 17.6])
def test_small_weights_count(ctx, dtype, new, dim, below):
    # As many sessions and heads as leave one block all tokens of a row.
    n, sessions = 3000, 10
    p = kv_ref.Population(new, [n] * sessions, [new] * sessions, 16, 16, dim, page_rows=64, dtype=dtype)
    p.k.zero_()
    p.q.zero_()
    p.q[..., 0] = 8.0
    p.v = (1.0 + p.v.float().abs() / 8).to(dtype)
    first = p.table[:, 0].long()
    p.k[first, 17, :, 0] = below / 8  # the others' scores are 0
    p.v[first, 17] = 0.0
    keep, memo = p.seen, {}
    p.seen = lambda s, at, w: memo.setdefault((s, at), keep(s, at, w))
    out, lse, _, ltol = p.reference(scale=1.0)
    # Values are not negative, so a relative error of the weights is one of the
    # result: of a score's sum of `dim` products (es, for weight and total), of the
    # sums, of the rounding to the type.  In float16 a weight is held at 2^7 and
    # more for the largest one, to 2^-25: 2^-32 of the total at most.
    u = kv_ref.ROUND[dtype]
    es = (dim + 8) * 2.0 ** -24 * (below + 1.0) + 2.0 ** -20
    tol = (2.01 * u + 3 * es + n * 2.0 ** -23) * out + 2.0 ** -24
    if dtype == torch.float16:
        tol = tol + 2.0 ** -32 * n * p.v.float().max().item()
    got, got_lse = attend(ctx, p, scale=1.0)
    off = (got.cpu().double() - out).abs() - tol
    assert (off <= 0).all(), off.max()
    assert ((got_lse.cpu().double() - lse).abs() <= ltol).all()
