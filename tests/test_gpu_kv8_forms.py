"""GPU: the forms that attention over 8-bit caches takes -- key heads of a block, parts and
their joins, sessions by length, codes widened ahead -- against the definition in 64 bits;
what the binding refuses; captured calls beside others."""
import math

import pytest
import torch

import kv8_ref as ref
import kv_ref
from paper_2607_21686_gb300 import pcs

pytestmark = pytest.mark.gpu

KINDS = [ref.E4M3, ref.I8]
TYPES = [torch.bfloat16, torch.float16]


def attend(ctx, p, window=0, hint=True, even=None):
    cache, batch, q = ref.on_gpu(pcs, p, hint=hint, even=even)
    if getattr(p, "parents", None) is not None:
        return ctx.attend_tree(cache, batch, ref.parents_on(p), q, window=window, return_lse=True)
    return ctx.attend(cache, batch, q, window=window, return_lse=True)


def check(ctx, p, window=0, **kw):
    out, lse = attend(ctx, p, window, **kw)
    ctx.sync()
    kv_ref.check_attend(p, out, lse, window)
    return out, lse


@pytest.mark.parametrize("hk", [1, 2, 3, 4, 5, 6, 8, 12, 20])
@pytest.mark.parametrize("new", [1, 2])
def test_key_heads(ctx, hk, new):
    # Blocks of four heads, of two, of one; scale bytes of more than sixteen heads.
    for dim in (64, 80):
        check(ctx, ref.Population8(hk, [40, 130, 77], [new] * 3, 2 * hk, hk, dim, KINDS[hk % 2], sinks=3, ring=100), 60)


@pytest.mark.parametrize("hq,hk", [(4, 4), (8, 2), (32, 2), (4, 1), (24, 1)])
@pytest.mark.parametrize("dim", [64, 128])
def test_parts_are_joined(ctx, hq, hk, dim):
    # One session: parts of turns, joined by their warps or by a launch of its own.
    for n in (600, 2500):
        p = ref.Population8(n + dim, [n], [1], hq, hk, dim, KINDS[dim == 64], dtype=TYPES[hk % 2])
        out, lse = check(ctx, p)
        again, lse2 = attend(ctx, p)
        assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("rows", [8, 32, 25])
def test_sessions_by_length(ctx, rows):
    # Lengths in no order, equal ones among them, most of them short.
    g = torch.Generator().manual_seed(rows)
    lens = torch.randint(1, 60, (40,), generator=g).tolist() + [2300, 60, 60, 2300, 1500, 1]
    check(ctx, ref.Population8(rows, lens, [1] * len(lens), 4, 4, 64, ref.E4M3, page_rows=rows))
    lens[44] = 2500
    p = ref.Population8(rows, lens, [1] * len(lens), 2, 1, 128, ref.I8, page_rows=rows)
    check(ctx, p)
    new = [min(n, 20 + i % 30) for i, n in enumerate(lens[:12])]
    check(ctx, ref.Population8(rows, lens[:12], new, 4, 2, 64, ref.I8, page_rows=rows))


def test_many_sessions(ctx):
    # More than are ranked by length.
    lens = [1 + i * 7 % 23 for i in range(530)]
    for n in (512, 530):
        p = ref.Population8(n, lens[:n], [1] * n, 2, 2, 64, page_rows=8)
        cache, batch, q = ref.on_gpu(pcs, p)
        batch.struct.max_len = 0
        wide = torch.full((n, 300), -1, dtype=torch.int32, device=q.device)  # (2,400 slots each)
        wide[:, :p.pages] = p.dt
        cache = pcs.KvCache(p.dk, p.dv, wide, codes=p.codes, heads=2, head_dim=64)
        out, lse = ctx.attend(cache, batch, q, return_lse=True)
        ctx.sync()
        kv_ref.check_attend(p, out, lse)


# ---------------------------------------------------------------------------
# Codes that are widened ahead of several blocks of rows
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("codes", KINDS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [64, 128, 80, 16])
def test_several_blocks(ctx, codes, dtype, dim):
    check(ctx, ref.Population8(dim, [300, 90, 150, 1], [300, 70, 66, 1], 4, 1, dim, codes, dtype=dtype, v_table=True))


@pytest.mark.parametrize("sinks,ring,window", [(0, 0, 1), (4, 0, 50), (100, 0, 30), (0, 200, 0), (5, 200, 90), (16, 230, 40),
                                               (17, 140, 33), (300, 0, 7)])
def test_several_blocks_over_windows_and_rings(ctx, sinks, ring, window):
    lens = [130, 90, 200, 310, 471]
    for rows in (16, 24, 25, 128):
        p = ref.Population8(sinks + ring, lens, [70, 90, 65, 130, 80], 8, 2, 64, KINDS[rows % 2], sinks=sinks, ring=ring,
                            page_rows=rows)
        check(ctx, p, window)


@pytest.mark.parametrize("codes", KINDS)
def test_several_blocks_and_empty_pages(ctx, codes):
    for dead in ([0], [1, 4], list(range(13))):
        p = ref.Population8(5, [200, 200], [90, 130], 8, 2, 64, codes)
        p.table[0, dead] = -1
        check(ctx, p, window=70)
        p.table[0, dead] = 10 ** 6
        cache, batch, q = ref.on_gpu(pcs, p)
        out, lse = ctx.attend(cache, batch, q, window=70, return_lse=True)
        if dead == [0]:
            ctx.sync()  # nobody's window reaches back to it
        else:
            with pytest.raises(pcs.PcsError) as e:
                ctx.sync()
            assert e.value.status == pcs.PCS_E_RANGE
        kv_ref.check_attend(p, out, lse, 70)


@pytest.mark.parametrize("codes", KINDS)
def test_what_was_in_the_working_memory_does_not_matter(ctx, dev, codes):
    # Calls over other data, with NaN among it, before: the widened pages hold it still.
    p = ref.Population8(6, [250, 157], [140, 100], 8, 2, 64, codes, sinks=5, ring=220)
    out, lse = check(ctx, p, window=60)
    bad = ref.Population8(7, [250, 250], [140, 140], 8, 2, 64, codes)
    bad.k_rows[:, :, 128:130] = 255
    bad.v_rows[:, :, 128:130] = 255
    for _ in range(2):
        junk, _ = attend(ctx, bad)
        assert torch.isnan(junk).all()
        again, lse2 = attend(ctx, p, window=60)
        assert torch.equal(out, again) and torch.equal(lse, lse2)
    # NaN and codes of it in rows that only some new tokens see.
    j = p.lens[0] - 1
    page, r = int(p.table[0, kv_ref.slot_of(j, 5, 220) // 16]), kv_ref.slot_of(j, 5, 220) % 16
    p.v_rows[page, r, 128] = 255
    again, _ = attend(ctx, p, window=60)
    assert torch.equal(again[:139], out[:139]) and torch.isnan(again[139, :4]).all()
    assert torch.equal(again[139, 4:], out[139, 4:]) and torch.equal(again[140:], out[140:])


@pytest.mark.parametrize("codes", KINDS)
@pytest.mark.parametrize("sinks,ring,window", [(0, 0, 0), (6, 150, 70), (30, 0, 5)])
def test_trees_of_several_blocks(ctx, codes, sinks, ring, window):
    p = ref.trees(codes, 8, [300, 64, 90], [64, 64, 40], 16, 2, 64, sinks=sinks, ring=ring)
    check(ctx, p, window)


# ---------------------------------------------------------------------------
# The binding, graphs
# ---------------------------------------------------------------------------

def test_the_binding_refuses(ctx, dev):
    k = torch.zeros(4, 16, 160, dtype=torch.uint8, device=dev)
    t = torch.zeros(2, 2, dtype=torch.int32, device=dev)
    ok = dict(codes=torch.int8, heads=2, head_dim=64)
    for args, kw in (((k, k[:3], t), ok), ((k.char(), k.char(), t), ok), ((k[..., ::2], k[..., ::2], t), ok),
                     ((k, k, t), dict(ok, codes=torch.uint8)), ((k, k, t), dict(ok, heads=None)),
                     ((k, k, t), dict(ok, head_dim=None)), ((k, k, t), dict(ok, heads=3)), ((k, k, t), dict(ok, heads=0)),
                     ((k, k, t), dict(heads=2)), ((k[0], k[0], t), ok), ((k, k, t), {}),
                     ((k.bfloat16()[..., None], k.bfloat16()[..., None], t), dict(ok))):
        with pytest.raises(ValueError):
            pcs.KvCache(*args, **kw)
    cache = pcs.KvCache(k, k, t, **ok)
    batch = pcs.KvBatch(torch.tensor([5, 6], dtype=torch.int32, device=dev), 4)
    q = torch.zeros(4, 2, 64, dtype=torch.bfloat16, device=dev)
    up = torch.tensor([-1, 0, -1, 0], dtype=torch.int32, device=dev)
    before = ctx.stats().kernel_launches
    for bad in (up[:3], up.long(), up.cpu(), up[None]):
        with pytest.raises(ValueError):
            ctx.attend_tree(cache, batch, bad, q)
    for args in ((up[None], up[:2]), (up.reshape(2, 2), up[:1]), (up.reshape(2, 2).long(), up[:2]), (up.reshape(2, 2), up[:2].cpu()),
                 (up, up[:2])):
        with pytest.raises(ValueError):
            ctx.kv_keep(cache, batch, *args)
    with pytest.raises(ValueError):
        ctx.kv_keep(cache, batch, up.reshape(2, 2), up[:2], lens_out=up)
    with pytest.raises(pcs.PcsError) as e:  # rows of index that overlap
        ctx.kv_keep(cache, batch, up.as_strided((2, 2), (1, 1)), up[:2])
    assert e.value.status == pcs.PCS_E_INVAL
    for kw in (dict(k_out=q[:3]), dict(v_out=q.half()), dict(dtype=torch.float64), dict(k_out=q[0])):
        with pytest.raises((ValueError, pcs.PcsError)):
            ctx.kv_read(cache, batch, **kw)
    assert ctx.stats().kernel_launches == before
    ctx.sync()


def test_two_graphs_and_calls_between_them(ctx, dev):
    """Each captured call has working memory of its own: two graphs run at once beside a
    plain call on a third stream give what each gives alone."""
    ps = [ref.Population8(40, [1800], [1], 8, 2, 128, ref.E4M3), ref.Population8(41, [700, 300], [130, 90], 8, 2, 64, ref.I8),
          kv_ref.Population(42, [2000], [1], 4, 2, 64)]
    made = [ref.on_gpu(pcs, p) for p in ps]
    want = [ctx.attend(*m) for m in made]
    ctx.sync()
    graphs, outs, streams = [], [], [torch.cuda.Stream() for _ in ps]
    for (cache, batch, q), stream in zip(made, streams):
        out = torch.empty_like(q)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            ctx.attend(cache, batch, q, out=out)
        graphs.append(graph)
        outs.append(out)
    for _ in range(3):
        for out in outs:
            out.fill_(7.0)
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        plain = [ctx.attend(*m) for m in made]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
        assert all(torch.equal(a, b) for a, b in zip(plain, want))


def test_calls_on_a_given_stream(ctx, dev):
    p = ref.trees(ref.E4M3, 50, [300, 90], [20, 20], 4, 2, 64)
    cache, batch, q = ref.on_gpu(pcs, p)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    out, lse = ctx.attend_tree(cache, batch, ref.parents_on(p), q, return_lse=True, stream=side)
    k, v = ctx.kv_read(cache, batch, stream=side)
    count = torch.full((2,), 2, dtype=torch.int32, device=dev)
    index = torch.tensor([[0, 3], [1, 2]], dtype=torch.int32, device=dev)
    torch.cuda.synchronize()
    lens = ctx.kv_keep(cache, batch, index, count, stream=side)
    side.synchronize()
    kv_ref.check_attend(p, out, lse)
    assert lens.tolist() == [282, 72]
    assert torch.isfinite(k).all() and math.isfinite(float(v.float().sum()))
