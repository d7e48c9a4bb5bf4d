"""GPU: what a node of a tree does not see changes no bit of its result: infinities and NaN
in other nodes' values, caches of 16 and of 8 bits."""
import math

import pytest
import torch

import kv8_ref as ref
from paper_2607_21686_gb300 import pcs

pytestmark = pytest.mark.gpu


def attend(ctx, p, window):
    cache, batch, q = ref.on_gpu(pcs, p)
    out = ctx.attend_tree(cache, batch, ref.parents_on(p), q, window=window)
    ctx.sync()
    return out.cpu()


@pytest.mark.parametrize("codes", [None, ref.E4M3])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("hq,hk,dim,nodes", [(2, 2, 64, 9), (4, 1, 128, 7), (2, 2, 80, 16), (2, 1, 64, 12)])
@pytest.mark.parametrize("window", [0, 40])
def test_others_rows_change_no_bit(ctx, codes, dtype, hq, hk, dim, nodes, window):
    n = 24
    lens = [nodes + 5 * i for i in range(n)]
    p = ref.trees(codes, dim + nodes, lens, [nodes] * n, hq, hk, dim, chain=0.4, dtype=dtype)
    out = attend(ctx, p, window)
    for i in range(n):  # node i mod nodes of session i
        at = lens[i] - nodes + i % nodes
        page, r = int(p.table[i, at // 16]), at % 16
        if codes is None:
            p.v[page, r] = math.nan if i % 2 else math.inf
        else:
            p.v_rows[page, r, :hk * dim] = 0x7F
    again = attend(ctx, p, window)
    for i in range(n):
        parents = p.parents[i * nodes:(i + 1) * nodes]
        for j in range(nodes):
            t = i * nodes + j
            if i % nodes in ref.line_of(parents, j)[:window or None]:
                assert not torch.isfinite(again[t]).any()
            else:
                assert torch.equal(out[t], again[t]), (i, j)
