"""GPU: results in place of the queries, of every form of attention over 8-bit caches and of
trees, have the bits of results in a tensor of their own."""
import pytest
import torch

import kv8_ref as ref
from paper_2607_21686_gb300 import pcs

pytestmark = pytest.mark.gpu

# One token (alone, in parts joined by their warps, by a second launch), a few, a block, a
# block in parts, several blocks widened ahead; pages that no box divides.
SHAPES = [([70, 400], [1, 1], 4, 16), ([5000], [1], 4, 16), ([9000], [2], 32, 32), ([300, 200], [5, 3], 4, 16),
          ([300, 200], [90, 40], 4, 16), ([2500], [60], 4, 16), ([400, 300], [300, 150], 8, 16), ([900, 90], [2, 2], 4, 25),
          ([400, 90], [60, 40], 4, 25)]


@pytest.mark.parametrize("codes", [ref.E4M3, ref.I8])
@pytest.mark.parametrize("lens,new,hq,rows", SHAPES)
def test_attention(ctx, codes, lens, new, hq, rows):
    p = ref.Population8(21, lens, new, hq, 2, 128, codes, page_rows=rows)
    cache, batch, q = ref.on_gpu(pcs, p)
    out, lse = ctx.attend(cache, batch, q, return_lse=True)
    _, lse2 = ctx.attend(cache, batch, q, out=q, return_lse=True)
    ctx.sync()
    assert torch.equal(q, out) and torch.equal(lse, lse2)


@pytest.mark.parametrize("codes", [None, ref.E4M3, ref.I8])
@pytest.mark.parametrize("lens,new,hq,rows", [([70, 400], [7, 5], 4, 16), ([5000], [6], 4, 16), ([300, 200], [60, 40], 8, 16),
                                              ([2500], [40], 8, 16), ([300, 200], [64, 40], 32, 16), ([90, 200], [9, 9], 4, 25)])
def test_trees(ctx, codes, lens, new, hq, rows):
    p = ref.trees(codes, 22, lens, new, hq, 2, 64, page_rows=rows)
    cache, batch, q = ref.on_gpu(pcs, p)
    parent = ref.parents_on(p)
    out, lse = ctx.attend_tree(cache, batch, parent, q, return_lse=True)
    _, lse2 = ctx.attend_tree(cache, batch, parent, q, out=q, return_lse=True)
    ctx.sync()
    assert torch.equal(q, out) and torch.equal(lse, lse2)
