"""GPU: attention over a paged cache against the definition in 64 bits
(tests/kv_ref.py), each value within a bound that its own rounding gives."""
import math

import pytest
import torch

import kv_ref
from paper_2607_21686_gb300 import pcs

pytestmark = pytest.mark.gpu


def attend(ctx, p, window=0, scale=0.0, hint=True, even=None):
    cache, batch, q = kv_ref.on_gpu(pcs, p, hint=hint, even=even)
    out, lse = ctx.attend(cache, batch, q, window=window, scale=scale, return_lse=True)
    ctx.sync()
    return out, lse


def check(ctx, p, window=0, scale=None, **kw):
    out, lse = attend(ctx, p, window, scale or 0.0, **kw)
    kv_ref.check_attend(p, out, lse, window, scale)
    return out, lse


TYPES = [torch.bfloat16, torch.float16]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hq,hk,dim", [(16, 16, 64), (8, 1, 128), (12, 4, 128), (2, 2, 8), (10, 2, 80),
                                       (6, 2, 96), (32, 2, 64), (25, 1, 40), (4, 4, 120)])
def test_one_token(ctx, dtype, hq, hk, dim):
    lens = [1, 2, 15, 16, 17, 64, 65, 200, 333]
    check(ctx, kv_ref.Population(dim + hq, lens, [1] * len(lens), hq, hk, dim, dtype=dtype))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [1, 5, 16, 24, 64, 1000])
def test_page_sizes(ctx, dtype, rows):
    check(ctx, kv_ref.Population(rows, [1, 77, 300], [1, 1, 1], 4, 2, 64, page_rows=rows, dtype=dtype))


@pytest.mark.parametrize("sinks,ring,window", [
    (0, 0, 1), (0, 0, 50), (4, 0, 50), (100, 0, 50), (0, 64, 0), (5, 64, 0), (16, 96, 40), (3, 50, 200),
    (300, 0, 7), (17, 33, 33)])
def test_windows_sinks_rings(ctx, sinks, ring, window):
    lens = [1, 4, 30, 64, 65, 70, 131, 290]
    for new in (1, 3):
        p = kv_ref.Population(sinks + ring + window, [max(n, new) for n in lens], [new] * len(lens), 4, 2, 64,
                              sinks=sinks, ring=ring)
        check(ctx, p, window)


@pytest.mark.parametrize("dtype", TYPES)
def test_a_few_ragged_tokens(ctx, dtype):
    check(ctx, kv_ref.Population(9, [5, 40, 100, 12, 3, 8], [5, 0, 7, 1, 3, 2], 8, 2, 128, dtype=dtype),
          window=6)


def test_sessions_of_no_tokens(ctx, dev):
    p = kv_ref.Population(2, [0, 9, 0], [0, 2, 0], 2, 2, 64)
    check(ctx, p)
    p = kv_ref.Population(2, [0, 0], [0, 0], 2, 2, 64)
    out, lse = attend(ctx, p, even=True)
    assert out.shape == (0, 2, 64) and lse.shape == (0, 2)


@pytest.mark.parametrize("hint", [False, True])
def test_long_sessions_are_split_and_joined(ctx, hint):
    p = kv_ref.Population(3, [5000, 3], [1, 1], 4, 2, 128, page_rows=32)
    out, lse = check(ctx, p, hint=hint)
    again, lse2 = attend(ctx, p, hint=hint)
    assert torch.equal(out, again) and torch.equal(lse, lse2)  # the parts join in a fixed order


def test_large_scores(ctx):
    # Running maxima that rise late, and scores whose exponential overflows.
    p = kv_ref.Population(4, [600, 600], [1, 1], 4, 4, 64, spread=4.0)
    ramp = torch.linspace(0.2, 4, 600)
    for s in range(2):
        for j in range(600):
            page, row = int(p.table[s, j // 16]), j % 16
            p.k[page, row] = (p.k[page, row].double() * ramp[j if s else 599 - j]).to(p.dtype)
    check(ctx, p)
    check(ctx, p, scale=1.0)
    check(ctx, p, scale=1e-3)


def test_empty_pages(ctx):
    for dead in ([0], [1, 2], [0, 1, 2, 3, 4, 5, 6]):
        p = kv_ref.Population(5, [100, 100], [1, 2], 4, 2, 64)
        p.table[0, dead] = -1
        check(ctx, p, window=70)


def test_what_is_not_seen_does_not_matter(ctx, dev):
    p = kv_ref.Population(6, [100, 37], [1, 1], 4, 2, 64, sinks=5)
    seen = {(k, r) for s in range(2) for _, k, _, r in p.seen(s, p.lens[s] - 1, 40)}
    out, lse = check(ctx, p, window=40)
    for junk in (math.nan, math.inf, -math.inf):
        for page in range(p.n_pages):
            for r in range(16):
                if (page, r) not in seen:
                    p.k[page, r] = junk
                    p.v[page, r] = junk
        again, lse2 = attend(ctx, p, window=40)
        assert torch.equal(out, again) and torch.equal(lse, lse2)


def test_infinities_and_nan_that_are_seen(ctx, dev):
    p = kv_ref.Population(7, [50, 50, 50], [1, 1, 1], 2, 2, 64)
    p.v[int(p.table[0, 1]), 3, 0, 5] = math.inf
    p.k[int(p.table[1, 2]), 3, 1] = math.nan
    cache, batch, q = kv_ref.on_gpu(pcs, p)
    out = ctx.attend(cache, batch, q).cpu()
    assert out[0, 0, 5] == math.inf and torch.isfinite(out[0, 1]).all()
    assert torch.isfinite(out[0, 0, :5]).all() and torch.isfinite(out[0, 0, 6:]).all()
    assert torch.isnan(out[1, 1]).all() and torch.isfinite(out[1, 0]).all()
    assert torch.isfinite(out[2]).all()


def test_layouts(ctx, dev):
    p = kv_ref.Population(8, [90, 31], [1, 1], 8, 4, 64, v_table=True)
    out, lse = check(ctx, p)
    # Heads before rows in a page, queries and results out of wider tensors.
    dk, dv = (x.to(dev).transpose(1, 2).contiguous().transpose(1, 2) for x in (p.k, p.v))
    wide = torch.full((2, p.pages + 3), -9, dtype=torch.int32, device=dev)
    vwide = wide.clone()
    wide[:, :p.pages], vwide[:, :p.pages] = p.table.to(dev), p.v_table.to(dev)
    cache = pcs.KvCache(dk, dv, wide[:, :p.pages], v_table=vwide[:, :p.pages])
    batch = pcs.KvBatch(torch.tensor(p.lens, dtype=torch.int32, device=dev), 2)
    qkv = torch.randn(2, 16, 64, device=dev).to(p.dtype)
    qkv[:, 3:11] = p.q.to(dev)
    got = torch.zeros(8, 2, 64, dtype=p.dtype, device=dev).transpose(0, 1)
    ctx.attend(cache, batch, qkv[:, 3:11], out=got)
    assert torch.equal(got, out)


def test_streams_side_by_side(ctx, dev):
    ps = [kv_ref.Population(20 + i, [3000], [1], 4, 2, 64) for i in range(4)]
    want = [attend(ctx, p)[0] for p in ps]
    made = [kv_ref.on_gpu(pcs, p) for p in ps]
    streams = [torch.cuda.Stream() for _ in ps]
    torch.cuda.synchronize()
    got = [[] for _ in ps]
    for _ in range(5):
        for i, (cache, batch, q) in enumerate(made):
            with torch.cuda.stream(streams[i]):
                got[i].append(ctx.attend(cache, batch, q))
    torch.cuda.synchronize()
    assert all(torch.equal(x, w) for g, w in zip(got, want) for x in g)


def test_offsets_past_32_bits(ctx, dev):
    # 5 GB a pool; the session's pages are its last ones.
    p = kv_ref.Population(30, [200], [1], 4, 8 // 2, 128, page_rows=64, spare=0)
    pages = 80000
    dk = torch.empty(pages, 64, 4, 128, dtype=p.dtype, device=dev)
    dv = torch.empty_like(dk)
    table = torch.arange(pages - p.n_pages, pages, dtype=torch.int32)
    dk[-p.n_pages:], dv[-p.n_pages:] = p.k.to(dev), p.v.to(dev)
    cache = pcs.KvCache(dk, dv, table[p.table.long()].to(dev))
    batch = pcs.KvBatch(torch.tensor(p.lens, dtype=torch.int32, device=dev), 1)
    out, lse = ctx.attend(cache, batch, p.q.to(dev), return_lse=True)
    kv_ref.check_attend(p, out, lse)
    nk = torch.randn(1, 4, 128, dtype=p.dtype, device=dev)
    ctx.kv_append(cache, batch, nk, nk)
    page = int(table[int(p.table[0, 3])])
    assert torch.equal(dk[page, 199 - 192], nk[0]) and torch.equal(dv[page, 199 - 192], nk[0])


def test_bad_ids_are_reported_and_unseen(ctx, dev):
    for bad in (10 ** 6, -3):
        p = kv_ref.Population(31, [60, 60], [1, 1], 2, 2, 64)
        p.table[1, 2] = bad
        cache, batch, q = kv_ref.on_gpu(pcs, p)
        out, lse = ctx.attend(cache, batch, q, return_lse=True)
        with pytest.raises(pcs.PcsError) as e:
            ctx.sync()
        assert e.value.status == pcs.PCS_E_RANGE
        kv_ref.check_attend(p, out, lse)


def test_more_new_tokens_than_said_are_reported(ctx, dev):
    p = kv_ref.Population(32, [60, 60, 60], [1, 5, 2], 2, 2, 64)
    cache, batch, q = kv_ref.on_gpu(pcs, p)
    batch.struct.max_new = 3
    out = torch.full_like(q, 7.0)
    ctx.attend(cache, batch, q, out=out)
    with pytest.raises(pcs.PcsError) as e:
        ctx.sync()
    assert e.value.status == pcs.PCS_E_RANGE
    assert (out[1:6] == 7.0).all()
    want = p.reference()
    assert ((out.cpu().double() - want[0]).abs() <= want[2])[[0, 6, 7]].all()


def test_a_session_shorter_than_its_new_tokens(ctx, dev):
    p = kv_ref.Population(33, [60, 8], [4, 4], 2, 2, 64)
    p.lens[1] = 2  # two of the four have no position
    cache, batch, q = kv_ref.on_gpu(pcs, p)
    out, lse = ctx.attend(cache, batch, q, return_lse=True)
    with pytest.raises(pcs.PcsError) as e:
        ctx.sync()
    assert e.value.status == pcs.PCS_E_RANGE
    kv_ref.check_attend(p, out, lse)
    assert (out[4:6] == 0).all() and (lse[4:6] == -math.inf).all()
