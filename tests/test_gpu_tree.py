"""GPU: attention of trees of drafted tokens, over 16- and 8-bit caches, against the
definition in 64 bits (tests/kv8_ref.py); kept tokens; and a run of them together."""
import math

import pytest
import torch

import kv8_ref as ref
import kv_ref
from paper_2607_21686_gb300 import pcs

pytestmark = pytest.mark.gpu

KINDS = [None, ref.E4M3, ref.I8]
TYPES = [torch.bfloat16, torch.float16]


def attend(ctx, p, window=0, scale=0.0, hint=True, even=None):
    cache, batch, q = ref.on_gpu(pcs, p, hint=hint, even=even)
    out, lse = ctx.attend_tree(cache, batch, ref.parents_on(p), q, window=window, scale=scale, return_lse=True)
    ctx.sync()
    return out, lse


def check(ctx, p, window=0, scale=None, **kw):
    out, lse = attend(ctx, p, window, scale or 0.0, **kw)
    kv_ref.check_attend(p, out, lse, window, scale)
    return out, lse


@pytest.mark.parametrize("codes", KINDS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hq,hk,dim,nodes", [(2, 2, 64, 7), (4, 4, 128, 32), (4, 1, 128, 8), (8, 2, 64, 64), (2, 2, 16, 33),
                                             (10, 2, 80, 12), (16, 2, 128, 64), (3, 1, 96, 2), (1, 1, 64, 1)])
def test_trees(ctx, codes, dtype, hq, hk, dim, nodes):
    lens = [nodes, nodes + 1, nodes + 200, nodes + 131]
    check(ctx, ref.trees(codes, dim + nodes, lens, [nodes] * 4, hq, hk, dim, dtype=dtype))


@pytest.mark.parametrize("codes", KINDS)
@pytest.mark.parametrize("group", [1, 8])
def test_ragged_trees(ctx, codes, group):
    lens, new = [300, 64, 5, 40, 33, 190], [64, 64, 0, 1, 33, 17]
    for chain in (0.0, 0.6, 1.0):
        check(ctx, ref.trees(codes, 3, lens, new, 2 * group, 2, 64, chain=chain))


@pytest.mark.parametrize("codes", KINDS)
@pytest.mark.parametrize("sinks,ring,window", [(0, 0, 1), (0, 0, 5), (0, 0, 50), (4, 0, 50), (100, 0, 3), (0, 64, 0), (5, 64, 0),
                                               (16, 96, 40), (3, 80, 200), (300, 0, 7), (17, 64, 33), (0, 200, 130)])
@pytest.mark.parametrize("group", [1, 5])
def test_windows_sinks_rings(ctx, codes, sinks, ring, window, group):
    lens, new = [30, 64, 65, 70, 131, 290], [30, 60, 64, 9, 64, 50]
    check(ctx, ref.trees(codes, sinks + ring + window, lens, new, 2 * group, 2, 64, sinks=sinks, ring=ring), window)


@pytest.mark.parametrize("rows", [1, 5, 8, 24, 64, 1000])
@pytest.mark.parametrize("codes", [None, ref.I8])
def test_page_sizes(ctx, codes, rows):
    for group in (1, 6):
        check(ctx, ref.trees(codes, rows, [150, 277], [50, 20], 2 * group, 2, 128, page_rows=rows))


@pytest.mark.parametrize("codes", [None, ref.E4M3])
def test_rings_whose_end_lies_in_a_tree(ctx, codes):
    # The nodes' slots go over the end of the ring, at every distance.
    for group in (1, 8):
        for beyond in (1, 7, 16, 30):
            p = ref.trees(codes, beyond, [96 + beyond, 4 + 2 * 96 + beyond], [31, 32], 2 * group, 2, 64, sinks=4, ring=96)
            check(ctx, p, 50)
            check(ctx, p, 0)


@pytest.mark.parametrize("codes", KINDS)
def test_long_contexts_are_split_and_joined(ctx, codes):
    for hq, nodes in ((2, 6), (8, 50)):
        p = ref.trees(codes, 3, [2500, 60], [nodes, nodes], hq, 2, 64, page_rows=32)
        out, lse = check(ctx, p)
        again, lse2 = attend(ctx, p, hint=False)
        if hq == 2:
            kv_ref.check_attend(p, again, lse2)
        again, lse2 = attend(ctx, p)
        assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("codes", KINDS)
def test_a_chain_is_what_attend_computes(ctx, codes):
    for group, nodes in ((1, 5), (1, 30), (4, 60)):
        p = ref.trees(codes, 5, [400, 77], [nodes, nodes], 2 * group, 2, 128, sinks=3, ring=150, chain=1.0)
        cache, batch, q = ref.on_gpu(pcs, p)
        for window in (0, 64):
            out, lse = ctx.attend_tree(cache, batch, ref.parents_on(p), q, window=window, return_lse=True)
            want, wlse = ctx.attend(cache, batch, q, window=window, return_lse=True)
            ctx.sync()
            assert torch.equal(out, want) and torch.equal(lse, wlse)


@pytest.mark.parametrize("codes", KINDS)
@pytest.mark.parametrize("hq,nodes", [(2, 20), (8, 40)])
def test_what_some_nodes_do_not_see(ctx, dev, codes, hq, nodes):
    # NaN and infinities in a node's row reach its descendants alone, in a context row beyond
    # some windows those that see it, in empty places nobody.
    p = ref.trees(codes, 8, [110, 45], [nodes, 9], hq, 2, 64, sinks=2, chain=0.3)
    out, lse = check(ctx, p, window=60)
    bad_at = nodes // 3
    first = p.lens[0] - nodes
    page, r = int(p.table[0, (first + bad_at) // 16]), (first + bad_at) % 16
    low = first - 60 + 2                                        # beyond the windows of deeper nodes
    lpage, lr = int(p.table[0, low // 16]), low % 16
    if codes is None:
        for junk in (math.nan, math.inf):
            p.v[page, r, 0, 5] = junk
            p.v[lpage, lr, 1, 7] = junk
    else:
        p.v_rows[page, r, 128] = 255
        p.v_rows[lpage, lr, 129] = 255
    again, _ = attend(ctx, p, window=60)
    again, out = again.cpu(), out.cpu()
    group = hq // 2
    for i in range(nodes):
        see = [j for j, *_ in p.seen(0, first + i, 60)]
        for where, head, d in ((first + bad_at, 0, 5), (low, 1, 7)):
            got = again[i, head * group:(head + 1) * group]
            if where in see:
                assert not torch.isfinite(got[:, d]).any()
            else:
                assert torch.equal(got, out[i, head * group:(head + 1) * group])
    assert torch.equal(again[nodes:], out[nodes:])


def test_bad_parents_count_as_the_context(ctx, dev):
    for hq in (2, 8):
        for bad in (5, 64, 10 ** 9, -2, -(2 ** 31)):
            p = ref.trees(None, 9, [90, 40], [12, 12], hq, 2, 64)
            cache, batch, q = ref.on_gpu(pcs, p)
            p.parents[5] = bad
            out, lse = ctx.attend_tree(cache, batch, ref.parents_on(p), q, return_lse=True)
            with pytest.raises(pcs.PcsError) as e:
                ctx.sync()
            assert e.value.status == pcs.PCS_E_RANGE
            p.parents[5] = -1
            kv_ref.check_attend(p, out, lse)


@pytest.mark.parametrize("codes", KINDS)
def test_short_and_long_sessions_are_bounded(ctx, dev, codes):
    # Lengths that the new tokens exceed, that exceed the table, offsets outside the call.
    for hq in (2, 8):
        p = ref.trees(codes, 10, [60, 8], [20, 20], hq, 2, 64)
        p.lens[1] = 3
        cache, batch, q = ref.on_gpu(pcs, p)
        out, lse = ctx.attend_tree(cache, batch, ref.parents_on(p), q, return_lse=True)
        with pytest.raises(pcs.PcsError) as e:
            ctx.sync()
        assert e.value.status == pcs.PCS_E_RANGE
        kv_ref.check_attend(p, out, lse)
        want = p.reference()
        lens = torch.tensor([60, 2 ** 31 - 1], dtype=torch.int32, device=dev)
        out = ctx.attend_tree(cache, pcs.KvBatch(lens, 40), ref.parents_on(p), q)
        with pytest.raises(pcs.PcsError):
            ctx.sync()
        assert ((out.cpu().double() - want[0]).abs() <= want[2])[:20].all()
        for off in ([-5, 15, 40], [0, 20, 47], [10 ** 9, 10 ** 9 + 1, 40]):
            o = torch.tensor(off, dtype=torch.int32, device=dev)
            ctx.attend_tree(cache, pcs.KvBatch(torch.tensor(p.lens, dtype=torch.int32, device=dev), 40, o, 25),
                            ref.parents_on(p), q)
            with pytest.raises(pcs.PcsError) as e:
                ctx.sync()
            assert e.value.status == pcs.PCS_E_RANGE


# ---------------------------------------------------------------------------
# Keep
# ---------------------------------------------------------------------------

def kept(ctx, dev, p, chosen, wide=0, lens_out=None):
    """The pools and lengths after keeping chosen[s] of session s's new tokens."""
    cache, batch, _ = ref.on_gpu(pcs, p)
    most = max([len(c) for c in chosen] + [1])
    index = torch.full((len(chosen), most + wide), -7, dtype=torch.int32)
    for s, c in enumerate(chosen):
        index[s, :len(c)] = torch.tensor(c, dtype=torch.int32)
    count = torch.tensor([len(c) for c in chosen], dtype=torch.int32, device=dev)
    lens = ctx.kv_keep(cache, batch, index.to(dev)[:, :most], count, lens_out=lens_out)
    return lens, p.dk.cpu(), p.dv.cpu()


def kept_expected(p, chosen):
    vt = p.table if p.v_table is None else p.v_table
    pools = (p.k_rows.clone(), p.v_rows.clone()) if hasattr(p, "codes") else (p.k.clone(), p.v.clone())
    old = [x.clone() for x in pools]
    lens = []
    for s, c in enumerate(chosen):
        first = p.lens[s] - p.new[s]
        for i, x in enumerate(c):
            a, b = (kv_ref.slot_of(first + j, p.sinks, p.ring) for j in (x, i))
            for pool, was, t in ((pools[0], old[0], p.table), (pools[1], old[1], vt)):
                ta, tb = int(t[s, a // p.rows]), int(t[s, b // p.rows])
                if ta < 0 or tb < 0:
                    continue
                row = was[ta, a % p.rows].clone()
                if hasattr(p, "codes"):  # what lies behind the scales stays
                    n = p.hk * (p.dim + 1)
                    row[n:] = pool[tb, b % p.rows][n:]
                pool[tb, b % p.rows] = row
        lens.append(first + len(c))
    return pools, lens


@pytest.mark.parametrize("codes", KINDS)
@pytest.mark.parametrize("hk,dim,sinks,ring,rows", [(2, 64, 0, 0, 16), (1, 128, 4, 80, 24), (5, 80, 100, 0, 5), (16, 128, 0, 64, 32)])
def test_kept_tokens_move(ctx, dev, codes, hk, dim, sinks, ring, rows):
    g = torch.Generator().manual_seed(dim)
    lens, new = [64, 200, 333, 70, 5, 90, 30], [64, 64, 40, 1, 0, 33, 30]
    p = ref.trees(codes, 1, lens, new, hk, hk, dim, sinks=sinks, ring=ring, page_rows=rows, v_table=True)
    chosen = [sorted(torch.randperm(m, generator=g)[:int(torch.randint(0, m + 1, (1,), generator=g))].tolist()) for m in new]
    chosen[1] = list(range(64))                 # all stay where they are
    chosen[2] = [39]
    pools, want = kept_expected(p, chosen)
    got, dk, dv = kept(ctx, dev, p, chosen, wide=3)
    ctx.sync()
    assert got.tolist() == want
    assert torch.equal(dk, pools[0]) and torch.equal(dv, pools[1])


def test_many_kept_tokens(ctx, dev):
    # More of them than are looked up at a time, each behind the one that it replaces.
    for codes in (None, ref.E4M3):
        p = ref.trees(codes, 2, [400], [300], 2, 2, 64) if codes else kv_ref.Population(2, [400], [300], 2, 2, 64)
        chosen = [[i + 1 for i in range(150)] + list(range(160, 290))]
        pools, want = kept_expected(p, chosen)
        got, dk, dv = kept(ctx, dev, p, chosen)
        assert got.tolist() == want and torch.equal(dk, pools[0]) and torch.equal(dv, pools[1])


def test_lengths_are_replaced_in_place(ctx, dev):
    p = kv_ref.Population(3, [50, 60], [9, 9], 2, 2, 64)
    cache, batch, _ = ref.on_gpu(pcs, p)
    lens = batch.keep[0]
    index = torch.tensor([[1, 3], [0, 8]], dtype=torch.int32, device=dev)
    count = torch.tensor([2, 1], dtype=torch.int32, device=dev)
    assert ctx.kv_keep(cache, batch, index, count, lens_out=lens) is lens
    ctx.sync()
    assert lens.tolist() == [43, 52]


@pytest.mark.parametrize("chosen", [[2, 2], [3, 1], [9], [-1, 2], [0, 1, 2, 3, 4, 5, 6, 7, 8, 9], [2 ** 31 - 1]])
def test_bad_indices_are_reported_and_leave_the_session(ctx, dev, chosen):
    p = kv_ref.Population(4, [50, 60], [9, 9], 2, 2, 64)
    pools, want = kept_expected(p, [[], [1, 4]])
    got, dk, dv = kept(ctx, dev, p, [chosen, [1, 4]])
    with pytest.raises(pcs.PcsError) as e:
        ctx.sync()
    assert e.value.status == pcs.PCS_E_RANGE
    assert got.tolist() == [50, 53]
    assert torch.equal(dk, pools[0]) and torch.equal(dv, pools[1])


def test_bad_counts_and_pages(ctx, dev):
    p = kv_ref.Population(4, [50, 60], [9, 9], 2, 2, 64)
    cache, batch, _ = ref.on_gpu(pcs, p)
    index = torch.tensor([[1, 3], [0, 8]], dtype=torch.int32, device=dev)
    for count in ([3, 0], [-1, 0], [2 ** 31 - 1, 0]):
        lens = ctx.kv_keep(cache, batch, index, torch.tensor(count, dtype=torch.int32, device=dev))
        with pytest.raises(pcs.PcsError) as e:
            ctx.sync()
        assert e.value.status == pcs.PCS_E_RANGE
        assert lens.tolist() == [50, 51]
    assert torch.equal(p.dk.cpu(), p.k) and torch.equal(p.dv.cpu(), p.v)
    # The page of a kept token is empty, that of its place is not: reported, not moved.
    for bad, fine in ((-1, False), (10 ** 6, False)):
        q = kv_ref.Population(4, [50, 60], [9, 9], 2, 2, 64)
        q.table[1, 3] = bad                        # positions 48 ..; the first new token is 51
        q.table[0, 2] = -1                         # where the first session's go
        cache, batch, _ = ref.on_gpu(pcs, q)
        ctx.kv_keep(cache, batch, index, torch.tensor([2, 2], dtype=torch.int32, device=dev))
        if bad == -1:
            ctx.sync()                             # both ends in the empty page: nothing is lost
        else:
            with pytest.raises(pcs.PcsError):
                ctx.sync()
        assert torch.equal(q.dk.cpu(), q.k) and torch.equal(q.dv.cpu(), q.v)
    q = kv_ref.Population(4, [50, 65], [9, 9], 2, 2, 64)
    q.table[1, 4] = -1                             # position 64, kept as 57
    cache, batch, _ = ref.on_gpu(pcs, q)
    ctx.kv_keep(cache, batch, index, torch.tensor([0, 2], dtype=torch.int32, device=dev))
    with pytest.raises(pcs.PcsError) as e:
        ctx.sync()
    assert e.value.status == pcs.PCS_E_RANGE
    assert torch.equal(q.dk.cpu(), q.k)


# ---------------------------------------------------------------------------
# Together
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("codes", [ref.E4M3, ref.I8])
def test_draft_check_keep_checkpoint(ctx, dev, codes):
    """Prompt, tree, keep, next token over an 8-bit cache, with a checkpoint and a restore of
    its pages in between: the same as the same tokens appended one after the other."""
    heads, dim, rows, ring, n = 2, 64, 16, 128, 100
    bytes_ = pcs.kv_row_bytes(heads, dim)
    g = torch.Generator().manual_seed(1)

    def session(seed):
        k, v = (torch.zeros(12, rows, bytes_, dtype=torch.uint8, device=dev) for _ in range(2))
        table = torch.randperm(12, generator=torch.Generator().manual_seed(seed))[:8].int()[None].to(dev)
        return k, v, table, pcs.KvCache(k, v, table, ring=ring, codes=codes, heads=heads, head_dim=dim)

    def rotary(pos):
        freq = torch.exp(torch.arange(32) * -0.25).to(dev)
        return pcs.Rotary(torch.tensor(pos, dtype=torch.int32, device=dev)[:, None].contiguous(), freq, (32,))

    def batch(length, new):
        return pcs.KvBatch(torch.tensor([length], dtype=torch.int32, device=dev), new)

    q, k, v = (torch.randn(n + 9, h, dim, generator=g).bfloat16().to(dev) for h in (4, heads, heads))
    parents = [-1, 0, 0, 1, 3, 2]
    depth = [0, 1, 1, 2, 3, 2]
    path = [0, 1, 3, 4]
    # With a tree: prompt, six drafted tokens, four of them kept, and the next one.
    kp, vp, table, cache = session(1)
    ctx.kv_append(cache, batch(n, n), k[:n], v[:n], q[:n], rotary(range(n)))
    b = batch(n + 6, 6)
    draft = slice(n, n + 6)
    turned = ctx.kv_append(cache, b, k[draft], v[draft], q[draft], rotary([n + d for d in depth]))
    tree = ctx.attend_tree(cache, b, torch.tensor(parents, dtype=torch.int32, device=dev), turned, window=90)
    lens = ctx.kv_keep(cache, b, torch.tensor([path], dtype=torch.int32, device=dev),
                       torch.tensor([4], dtype=torch.int32, device=dev))
    ctx.sync()
    assert lens.tolist() == [n + 4]
    # Its pages through a checkpoint and a verified restore into other pages.
    start = (n + 4) % ring
    meta = torch.tensor([n + 4], dtype=torch.int64, device=dev)

    def state(kp, vp, table):
        return pcs.kv_session(7, meta, kp, vp, table, start, ring)

    snap = ctx.checkpoint([state(kp, vp, table)])[0]
    k2, v2, table2, cache2 = session(2)
    ctx.restore([snap], [state(k2, v2, table2)], verify=True)
    ctx.delete(snap)
    last = slice(n + 6, n + 7)
    b = pcs.KvBatch(lens + 1, 1)
    turned = ctx.kv_append(cache2, b, k[last], v[last], q[last], rotary([n + 4]))
    out = ctx.attend(cache2, b, turned, window=90)
    # One after the other.
    k3, v3, _, cache3 = session(3)
    ctx.kv_append(cache3, batch(n, n), k[:n], v[:n], q[:n], rotary(range(n)))
    for i, x in enumerate(path):
        one = slice(n + x, n + x + 1)
        turned = ctx.kv_append(cache3, batch(n + i + 1, 1), k[one], v[one], q[one], rotary([n + i]))
        want = ctx.attend(cache3, batch(n + i + 1, 1), turned, window=90)
        assert torch.allclose(tree[x].float(), want[0].float(), atol=2.0 ** -7, rtol=2.0 ** -7)
    got, want = ctx.kv_read(cache2, batch(n + 4, n + 4)), ctx.kv_read(cache3, batch(n + 4, n + 4))
    assert torch.equal(got[0][6:], want[0][6:]) and torch.equal(got[1][6:], want[1][6:])
    turned = ctx.kv_append(cache3, batch(n + 5, 1), k[last], v[last], q[last], rotary([n + 4]))
    want = ctx.attend(cache3, batch(n + 5, 1), turned, window=90)
    ctx.sync()
    assert torch.allclose(out.float(), want.float(), atol=2.0 ** -8, rtol=2.0 ** -7)


@pytest.mark.parametrize("codes", [None, ref.E4M3])
def test_a_step_in_a_graph(ctx, dev, codes):
    """Append, tree attention and keep captured once and run again on other data."""
    p = ref.trees(codes, 6, [300, 90], [20, 20], 4, 2, 64)
    cache, batch, q = ref.on_gpu(pcs, p)
    parent = ref.parents_on(p)
    k, v = (torch.randn(40, 2, 64, device=dev).to(p.dtype) for _ in range(2))
    index = torch.tensor([[1, 3, 7], [0, 2, 2]], dtype=torch.int32, device=dev)
    count = torch.tensor([3, 2], dtype=torch.int32, device=dev)
    out, lens = torch.empty_like(q), torch.empty(2, dtype=torch.int32, device=dev)

    def step():
        ctx.kv_append(cache, batch, k, v)
        ctx.attend_tree(cache, batch, parent, q, out=out)
        ctx.kv_keep(cache, batch, index, count, lens_out=lens)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for seed in range(3):
        torch.manual_seed(seed)
        k.normal_(), v.normal_(), q.normal_()
        pools = p.dk.clone(), p.dv.clone()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), lens.clone(), p.dk.clone(), p.dv.clone()
        p.dk.copy_(pools[0]), p.dv.copy_(pools[1])
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (out, lens, p.dk, p.dv)))
