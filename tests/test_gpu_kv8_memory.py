"""GPU: several blocks of query rows over 8-bit codes that are not widened ahead -- tables with
room for more tokens than there is working memory for -- against the definition in 64 bits
and beside the same calls over tables that fit."""
import pytest
import torch

import kv8_ref as ref
import kv_ref
from paper_2607_21686_gb300 import pcs

pytestmark = pytest.mark.gpu


def attend(ctx, p, window, vast, hint=True):
    cache, batch, q = ref.on_gpu(pcs, p, hint=hint)
    if vast:  # beyond 1 GiB as 16-bit elements
        pages = max(p.pages, (1 << 29) // (p.rows * p.hk * p.dim * 2 * len(p.lens)) + 1)
        wide = torch.full((len(p.lens), pages), -1, dtype=torch.int32, device=q.device)
        wide[:, :p.pages] = p.dt
        cache = pcs.KvCache(p.dk, p.dv, wide, sinks=p.sinks, ring=p.ring, codes=p.codes, heads=p.hk, head_dim=p.dim)
    if getattr(p, "parents", None) is not None:
        out, lse = ctx.attend_tree(cache, batch, ref.parents_on(p), q, window=window, return_lse=True)
    else:
        out, lse = ctx.attend(cache, batch, q, window=window, return_lse=True)
    ctx.sync()
    return out, lse


def check(ctx, p, window=0):
    before = ctx.stats().kernel_launches
    fits = attend(ctx, p, window, False)
    widened = ctx.stats().kernel_launches - before
    got = attend(ctx, p, window, True)
    assert ctx.stats().kernel_launches - before == 2 * widened - 1  # (without k_widen)
    for out, lse in (fits, got):
        kv_ref.check_attend(p, out, lse, window)


@pytest.mark.parametrize("codes", [ref.E4M3, ref.I8])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("hq,hk,dim", [(4, 1, 64), (8, 2, 128), (4, 1, 80)])
def test_blocks_over_codes(ctx, codes, dtype, hq, hk, dim):
    for rows in (16, 25):
        check(ctx, ref.Population8(dim + rows, [200, 150, 90, 1], [140, 66, 70, 1], hq, hk, dim, codes, dtype=dtype, page_rows=rows))


@pytest.mark.parametrize("sinks,ring,window", [(4, 0, 50), (0, 200, 0), (5, 201, 90), (16, 230, 40)])
def test_blocks_over_codes_of_rings(ctx, sinks, ring, window):
    for codes in (ref.E4M3, ref.I8):
        check(ctx, ref.Population8(ring, [130, 200, 310, 471], [70, 65, 130, 80], 8, 2, 64, codes, sinks=sinks, ring=ring), window)


@pytest.mark.parametrize("codes", [ref.E4M3, ref.I8])
def test_trees_over_codes(ctx, codes):
    check(ctx, ref.trees(codes, 8, [300, 64, 90], [64, 64, 40], 16, 2, 64), 70)


@pytest.mark.parametrize("codes", [ref.E4M3, ref.I8])
def test_parts_over_codes(ctx, codes):
    # One session of two blocks in parts, with and without a hint of its length.
    p = ref.Population8(2, [1300], [140], 4, 2, 64, codes)
    for hint in (True, False):
        out, lse = attend(ctx, p, 0, True, hint)
        kv_ref.check_attend(p, out, lse)
        again, lse2 = attend(ctx, p, 0, True, hint)
        assert torch.equal(out, again) and torch.equal(lse, lse2)
