"""GPU: attention of blocks of new tokens over a paged cache (more rows of a
key head than the token kernel takes) against the definition in 64 bits."""
import math

import pytest
import torch

import kv_ref
from paper_2607_21686_gb300 import pcs
from test_gpu_attend import TYPES, attend, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hq,hk,dim", [(2, 2, 64), (1, 1, 128), (4, 1, 128), (3, 1, 80), (2, 1, 96), (1, 1, 8)])
def test_prompts(ctx, dtype, hq, hk, dim):
    lens = [1, 33, 64, 127, 128, 129, 300]
    check(ctx, kv_ref.Population(dim + hq, lens, lens, hq, hk, dim, dtype=dtype))


@pytest.mark.parametrize("new", [33, 128, 129, 256, 257, 400])
def test_blocks_after_a_context(ctx, new):
    check(ctx, kv_ref.Population(new, [new, new + 1, new + 200], [new] * 3, 1, 1, 64))


@pytest.mark.parametrize("rows", [1, 7, 24, 64, 200])
def test_page_sizes(ctx, rows):
    check(ctx, kv_ref.Population(rows, [50, 333], [50, 90], 2, 1, 128, page_rows=rows, dtype=torch.float16))


@pytest.mark.parametrize("sinks,ring,window", [
    (0, 0, 1), (0, 0, 100), (4, 0, 50), (130, 0, 33), (0, 300, 0), (5, 200, 0), (16, 300, 40), (200, 150, 20)])
def test_windows_sinks_rings(ctx, sinks, ring, window):
    p = kv_ref.Population(sinks + ring + window, [40, 300, 500, 700], [40, 150, 40, 140], 2, 1, 64,
                          sinks=sinks, ring=ring)
    check(ctx, p, window)


def test_ragged_with_nothing_new(ctx):
    check(ctx, kv_ref.Population(1, [300, 20, 0, 77, 40], [100, 0, 0, 77, 1], 2, 2, 64), window=60)


def test_many_query_heads(ctx):
    check(ctx, kv_ref.Population(2, [40, 90], [2, 7], 40, 1, 64))


@pytest.mark.parametrize("hint", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
def test_long_sessions_are_split_and_joined(ctx, hint, dim):
    p = kv_ref.Population(3, [2500, 60], [70, 40], 2, 1, dim, page_rows=32)
    out, lse = check(ctx, p, hint=hint)
    again, lse2 = attend(ctx, p, hint=hint)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


def test_large_scores(ctx):
    p = kv_ref.Population(4, [500], [100], 2, 2, 64, spread=4.0)
    for j in range(500):
        page, row = int(p.table[0, j // 16]), j % 16
        p.k[page, row] = (p.k[page, row].double() * (0.2 + j / 125)).to(p.dtype)
    check(ctx, p)
    check(ctx, p, scale=1.0)


def test_empty_pages(ctx):
    for dead in ([0], [5, 6, 7], list(range(19))):
        p = kv_ref.Population(5, [300, 300], [100, 40], 2, 1, 64)
        p.table[0, dead] = -1
        check(ctx, p, window=150)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("new", [3, 100])  # a few tokens, a block
def test_what_a_row_does_not_see_does_not_matter(ctx, dtype, new):
    # Infinities and NaN in tokens that some rows see and others do not: only
    # those that see them change.
    p = kv_ref.Population(6, [300], [new], 2, 1, 64, dtype=dtype)
    out, lse = check(ctx, p, window=120)
    j = 300 - new + 1  # the second new token
    page, row = int(p.table[0, j // 16]), j % 16
    old = 300 - new - 119  # only the first new token's window reaches it
    page2, row2 = int(p.table[0, old // 16]), old % 16
    p.v[page, row, 0, 3] = math.inf
    p.v[page, row, 0, 9] = math.nan
    p.v[page2, row2, 0, 50] = -math.inf
    got, lse2 = attend(ctx, p, window=120)
    assert torch.equal(lse, lse2)
    assert (got[1:, :, 3] == math.inf).all() and torch.isnan(got[1:, :, 9]).all()
    assert (got[0, :, 50] == -math.inf).all()
    same = torch.ones(new, 2, 64, dtype=torch.bool)
    same[1:, :, 3] = same[1:, :, 9] = False
    same[0, :, 50] = False
    assert torch.equal(got.cpu()[same], out.cpu()[same])
    # A key that is NaN spoils the rows that see it, and no other.
    p.v[page, row] = 1.0
    p.v[page2, row2] = 1.0
    p.k[page, row, 0, 0] = math.nan
    got, _ = attend(ctx, p, window=120)
    assert torch.isnan(got[1:]).all() and torch.isfinite(got[0]).all()


def test_junk_outside_the_sessions(ctx):
    p = kv_ref.Population(8, [200, 90], [60, 33], 2, 1, 128)
    out, lse = check(ctx, p)
    used = {(int(p.table[s, j // 16]), j % 16) for s in range(2) for j in range(p.lens[s])}
    for page in range(p.n_pages):
        for r in range(16):
            if (page, r) not in used:
                p.k[page, r] = math.nan
                p.v[page, r] = math.inf
    again, lse2 = attend(ctx, p)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


def test_layouts(ctx, dev):
    p = kv_ref.Population(9, [190, 131], [50, 50], 4, 2, 64, v_table=True)
    out, _ = check(ctx, p)
    dk, dv = (x.to(dev).transpose(1, 2).contiguous().transpose(1, 2) for x in (p.k, p.v))
    cache = pcs.KvCache(dk, dv, p.table.to(dev), v_table=p.v_table.to(dev))
    batch = pcs.KvBatch(torch.tensor(p.lens, dtype=torch.int32, device=dev), 100)
    wide = torch.randn(100, 9, 64, device=dev).to(p.dtype)
    wide[:, 3:7] = p.q.to(dev)
    got = torch.zeros(4, 100, 64, dtype=p.dtype, device=dev).transpose(0, 1)
    ctx.attend(cache, batch, wide[:, 3:7], out=got)
    assert torch.equal(got, out)


def test_block_and_token_kernels_agree(ctx):
    # The same rows through both: within twice their bounds of one another.
    p = kv_ref.Population(10, [400], [40], 1, 1, 64)
    out, lse = check(ctx, p)
    ref = p.reference()
    q = p.q
    for i in range(0, 40, 13):
        one = kv_ref.Population(10, [400], [40], 1, 1, 64)
        one.lens, one.new, one.tokens, one.q_off, one.q = [361 + i], [1], 1, [0, 1], q[i:i + 1]
        a, b = attend(ctx, one)
        assert ((a.cpu().double() - out[i:i + 1].cpu().double()).abs() <= 2 * ref[2][i:i + 1]).all()
        assert ((b - lse[i:i + 1]).abs().cpu() <= 2 * ref[3][i:i + 1]).all()


def test_more_new_tokens_than_said_are_reported(ctx, dev):
    p = kv_ref.Population(11, [60, 100], [40, 70], 1, 1, 64)
    cache, batch, q = kv_ref.on_gpu(pcs, p)
    batch.struct.max_new = 50
    out = torch.full_like(q, 7.0)
    ctx.attend(cache, batch, q, out=out)
    with pytest.raises(pcs.PcsError) as e:
        ctx.sync()
    assert e.value.status == pcs.PCS_E_RANGE
    assert (out[40:] == 7.0).all()
    want = p.reference()
    assert ((out.cpu().double() - want[0]).abs() <= want[2])[:40].all()


def test_bad_ids_and_short_sessions(ctx, dev):
    p = kv_ref.Population(12, [160, 60], [50, 50], 1, 1, 64)
    p.table[0, 2] = 10 ** 7
    p.lens[1] = 20
    cache, batch, q = kv_ref.on_gpu(pcs, p)
    out, lse = ctx.attend(cache, batch, q, return_lse=True)
    with pytest.raises(pcs.PcsError) as e:
        ctx.sync()
    assert e.value.status == pcs.PCS_E_RANGE
    kv_ref.check_attend(p, out, lse)
    assert (out[50:80] == 0).all() and (lse[50:80] == -math.inf).all()


@pytest.mark.parametrize("sinks,ring", [(0, 301), (0, 200), (5, 200), (16, 333), (7, 129), (130, 190), (3, 500)])
@pytest.mark.parametrize("rows", [8, 16, 24, 64])
def test_rings_that_wrap_anywhere(ctx, sinks, ring, rows):
    # Lengths that put the ring's end at every place of a box and a tile.
    lens = [ring + sinks + d for d in (-1, 0, 1, 7, 40, 100, ring // 2)]
    new = [40, 100, 120, 33, 128, 90, 50]
    p = kv_ref.Population(ring + rows, lens, new, 1, 1, 64, page_rows=rows, sinks=sinks, ring=ring, dtype=torch.float16)
    check(ctx, p)
    check(ctx, p, window=77)


def test_junk_past_the_end_of_a_ring(ctx):
    # Rows of the last page behind the ring, and of the page of the first tokens.
    p = kv_ref.Population(20, [400], [60], 1, 1, 64, page_rows=16, sinks=5, ring=203)
    out, lse = check(ctx, p)
    for at in range(208, 16 * p.pages):
        p.k[int(p.table[0, at // 16]), at % 16] = math.nan
        p.v[int(p.table[0, at // 16]), at % 16] = math.inf
    again, lse2 = attend(ctx, p)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dim,new,page_rows", [(128, 2, 16), (128, 40, 16), (64, 40, 8), (128, 40, 13), (64, 300, 24)])
def test_again_and_again(ctx, dev, dim, new, page_rows):
    # Many ragged sessions whose keys and values come from far and near, over and
    # over: every pass gives the same bits, and no wait runs out.
    n = 48
    g = torch.Generator().manual_seed(dim + new)
    lens = torch.randint(new, 3000, (n,), generator=g, dtype=torch.int32)
    pages = -(-3000 // page_rows)
    dk, dv = (torch.randn(n * pages + 5, page_rows, 4, dim, device=dev, dtype=torch.bfloat16) for _ in range(2))
    table = torch.randperm(n * pages + 5, generator=g)[:n * pages].reshape(n, pages).int().to(dev)
    cache = pcs.KvCache(dk, dv, table)
    batch = pcs.KvBatch(lens.to(dev), n * new)
    q = torch.randn(n * new, 72 if new == 2 else 4, dim, device=dev, dtype=torch.bfloat16)
    far = torch.empty(64 << 20, dtype=torch.int32, device=dev)
    first = None
    for i in range(60):
        if i % 3 == 0:
            far.fill_(i)  # the pools leave the cache
        out, lse = ctx.attend(cache, batch, q, window=1000, return_lse=True)
        if first is None:
            first = (out, lse)
        else:
            assert torch.equal(out, first[0]) and torch.equal(lse, first[1]), i
    ctx.sync()


@pytest.mark.parametrize("lens,new,hq", [([70, 400], [1, 1], 2), ([5000], [2], 8), ([300, 200], [90, 40], 2), ([2500], [60], 2)])
def test_results_in_place_of_the_queries(ctx, dev, lens, new, hq):
    p = kv_ref.Population(21, lens, new, hq, 2, 128)
    out, lse = check(ctx, p)
    cache, batch, q = kv_ref.on_gpu(pcs, p)
    ctx.attend(cache, batch, q, out=q)
    assert torch.equal(q, out)
