"""GPU: rotary positions with several axes and the append to a paged cache,
against their definitions in 64 bits (tests/kv_ref.py)."""
import math

import pytest
import torch

import kv_ref
from paper_2607_21686_gb300 import pcs

pytestmark = pytest.mark.gpu


def freqs(pairs, dev):
    return torch.cat([torch.exp(torch.arange(n) * (-math.log(10000.0) / max(n, 1))) for n in pairs]
                     ).float().to(dev)


def positions(g, tokens, axes, hi=4000):
    return torch.randint(-hi, hi, (tokens, axes), generator=g, dtype=torch.int32)


def off_by(got, want, dtype):
    """One rounding of the result, and of angles, cosines and products in 32
    bits a few units of the largest element of a pair (at most 8 here)."""
    tol = kv_ref.ROUND[dtype] * want.abs() * 1.0001 + 8 * 8 * 2.0 ** -24 \
        + (2.0 ** -24 if dtype == torch.float16 else 0.0)
    return ((got.cpu().double() - want).abs() - tol).max().item()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens,heads,dim,pairs", [
    (1, (1, 1), 64, (8, 12, 12)), (7, (3, 1), 128, (16, 24, 24)), (33, (2,), 64, (5, 4, 3)),
    (1000, (4, 2), 80, (16, 8, 8)), (5, (1,), 7, (1, 0, 1)), (3, (2,), 256, (128,)),
    (300, (16, 16, 16), 96, (8, 8, 8, 8)), (9, (1,), 2, (1,)), (2, (5,), 64, (0,))])
def test_rotate(ctx, dev, dtype, inverse, interleaved, tokens, heads, dim, pairs):
    g = torch.Generator().manual_seed(tokens * 131 + dim)
    pos, freq = positions(g, tokens, len(pairs)), freqs(pairs, "cpu")
    xs = [torch.randn(tokens, h, dim, generator=g).clamp(-5, 5).to(dtype) for h in heads]
    rot = pcs.Rotary(pos.to(dev), freq.to(dev), pairs, interleaved)
    got = ctx.rotate([x.to(dev) for x in xs], rot, inverse=inverse)
    for x, y in zip(xs, got):
        want = kv_ref.turned(x, pos, freq, pairs, interleaved, inverse)
        assert off_by(y, want, dtype) <= 0
        assert torch.equal(y[..., 2 * sum(pairs):].cpu(), x[..., 2 * sum(pairs):])


def test_far_positions_keep_their_angles(ctx, dev):
    pos = torch.tensor([[2 ** 31 - 1], [-2 ** 31], [123456789], [16777217], [105616]], dtype=torch.int32)
    freq = freqs((32,), "cpu")
    x = torch.randn(5, 3, 64, generator=torch.Generator().manual_seed(1)).clamp(-5, 5)
    got = ctx.rotate([x.to(dev)], pcs.Rotary(pos.to(dev), freq.to(dev), (32,)))[0]
    want = kv_ref.turned(x, pos, freq, (32,))
    # A position of 31 bits times a frequency of 24 in two floats: 2^-47 of
    # 2^31, so 2^-16 of a turn's radian on elements up to 8.
    assert (got.cpu().double() - want).abs().max() <= 8 * 2.0 ** -16
    near = (pos.abs() < 2 ** 27)[:, 0]
    assert off_by(got[near], want[near], torch.float32) <= 0


@pytest.mark.parametrize("interleaved", [False, True])
def test_strides_offsets_and_in_place(ctx, dev, interleaved):
    g = torch.Generator().manual_seed(5)
    pairs, tokens = (8, 8, 8), 41
    pos, freq = positions(g, tokens, 3), freqs(pairs, "cpu")
    rot = pcs.Rotary(pos.to(dev), freq.to(dev), pairs, interleaved)
    base = torch.randn(tokens, 9, 64, generator=g).to(torch.bfloat16)
    for a, b in ((0, 64), (1, 61), (8, 64)):  # heads that start anywhere
        whole = base.to(dev)
        x = whole[:, 2:7, a:b]
        want = kv_ref.turned(base[:, 2:7, a:b], pos, freq, pairs, interleaved)
        got = ctx.rotate([x], rot)[0]
        assert off_by(got, want, torch.bfloat16) <= 0
        # Heads before tokens.
        y = torch.empty(5, tokens, b - a, dtype=torch.bfloat16, device=dev).transpose(0, 1)
        ctx.rotate([x], rot, out=[y])
        assert torch.equal(y, got)
        ctx.rotate([x], rot, out=[x])
        assert torch.equal(x, got)
        kept = whole.cpu()
        kept[:, 2:7, a:b] = base[:, 2:7, a:b]
        assert torch.equal(kept, base)


@pytest.mark.parametrize("interleaved", [False, True])
def test_inverse_is_the_gradient(ctx, dev, interleaved):
    # L = <w, R x>: dL/dx = R^T w by the formula, and by differences.
    g = torch.Generator().manual_seed(11)
    pairs = (2, 3, 1)
    pos, freq = positions(g, 3, 3, 50).to(dev), freqs(pairs, dev)
    rot = pcs.Rotary(pos, freq, pairs, interleaved)
    x = torch.randn(3, 2, 14, generator=g).to(dev)
    w = torch.randn(3, 2, 14, generator=g).to(dev)
    grad = ctx.rotate([w], rot, inverse=True)[0]
    step = 0.5  # the rotation is linear: any step does
    for i in range(x.numel()):
        e = torch.zeros_like(x).reshape(-1)
        e[i] = step
        e = e.reshape(x.shape)
        up, down = ctx.rotate([x + e, x - e], rot)
        d = ((up - down).double() * w.double()).sum() / (2 * step)
        # Differences of 28 values of at most 6, rounded at 2^-24 a few times.
        assert abs(d - grad.reshape(-1)[i].double()) <= 28 * 6 * 6 * 2.0 ** -22


def append_case(seed, lens, new, hk, dim, rows, sinks, ring, dtype, hq=0):
    p = kv_ref.Population(seed, lens, new, max(hq, hk), hk, dim, rows, sinks, ring, dtype)
    p.nk = torch.randn(p.tokens, hk, dim, generator=p.g).clamp(-5, 5).to(dtype)
    p.nv = torch.randn(p.tokens, hk, dim, generator=p.g).clamp(-5, 5).to(dtype)
    return p


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("lens,new,hk,dim,rows,sinks,ring,pairs", [
    ([1], [1], 16, 64, 16, 0, 0, (8, 12, 12)),
    ([1030, 5, 1024, 40], [1, 1, 1, 1], 16, 64, 16, 0, 1024, (8, 12, 12)),
    ([100, 7, 64, 33], [90, 7, 1, 20], 2, 128, 24, 5, 60, (16, 24, 24)),
    ([500, 90], [400, 90], 3, 80, 7, 3, 50, (5, 3, 9)),     # laps of the ring in one call
    ([50, 0, 9], [50, 0, 3], 1, 8, 1, 0, 0, (1, 1, 2)),
    ([40, 41], [10, 10], 2, 64, 16, 0, 0, None)])
def test_append(ctx, dev, dtype, lens, new, hk, dim, rows, sinks, ring, pairs):
    p = append_case(sum(lens) + dim, lens, new, hk, dim, rows, sinks, ring, dtype, hq=2 * hk)
    cache, batch, q = kv_ref.on_gpu(pcs, p)
    rot = None
    wk, wq = p.nk.double(), p.q.double()
    if pairs:
        pos, freq = positions(p.g, p.tokens, 3), freqs(pairs, "cpu")
        rot = pcs.Rotary(pos.to(dev), freq.to(dev), pairs)
        wk, wq = kv_ref.turned(p.nk, pos, freq, pairs), kv_ref.turned(p.q, pos, freq, pairs)
    got = ctx.kv_append(cache, batch, p.nk.to(dev), p.nv.to(dev), q, rot)
    ctx.sync()
    assert off_by(got, wq, dtype) <= 0
    k, v = p.k.double(), p.v.clone()
    written = torch.zeros(p.k.shape[:2], dtype=torch.bool)
    for s, m in enumerate(new):
        for i in range(m):  # in order: the last token of a slot stays
            at = kv_ref.slot_of(lens[s] - m + i, sinks, ring)
            page, row = int(p.table[s, at // rows]), at % rows
            k[page, row], v[page, row] = wk[p.q_off[s] + i], p.nv[p.q_off[s] + i]
            written[page, row] = True
    assert torch.equal(p.dv.cpu(), v)
    assert torch.equal(p.dk.cpu()[~written], p.k[~written])
    assert off_by(p.dk, k, dtype) <= 0


def test_append_of_unaligned_tensors_and_other_layouts(ctx, dev):
    p = append_case(3, [20, 33], [4, 9], 4, 64, 8, 0, 0, torch.bfloat16)
    cache, batch, _ = kv_ref.on_gpu(pcs, p)
    # Pools with heads before rows, values' pages of their own, tensors off 16 bytes.
    dk = p.k.to(dev).transpose(1, 2).contiguous().transpose(1, 2)
    dv = p.v.to(dev).transpose(1, 2).contiguous().transpose(1, 2)
    vt = torch.flip(p.table, (1,)).contiguous()
    cache = pcs.KvCache(dk, dv, p.dt, v_table=vt.to(dev))
    wide = torch.zeros(p.tokens, 4, 70, dtype=torch.bfloat16, device=dev)
    nk, nv = wide[:, :, 3:67], torch.clone(wide)[:, :, 1:65]
    nk.copy_(p.nk)
    nv.copy_(p.nv)
    ctx.kv_append(cache, batch, nk, nv)
    ctx.sync()
    k, v = p.k.clone(), p.v.clone()
    for s, m in enumerate(p.new):
        for i in range(m):
            at = p.lens[s] - m + i
            k[int(p.table[s, at // 8]), at % 8] = p.nk[p.q_off[s] + i]
            v[int(vt[s, at // 8]), at % 8] = p.nv[p.q_off[s] + i]
    assert torch.equal(dk.cpu(), k) and torch.equal(dv.cpu(), v)


def test_append_skips_empty_pages_and_reports_bad_ones(ctx, dev):
    for bad, status in ((-1, None), (10 ** 6, pcs.PCS_E_RANGE), (-7, pcs.PCS_E_RANGE)):
        p = append_case(4, [20, 20], [3, 3], 2, 64, 16, 0, 0, torch.float16)
        p.table[1, 1] = bad
        cache, batch, _ = kv_ref.on_gpu(pcs, p)
        ctx.kv_append(cache, batch, p.nk.to(dev), p.nv.to(dev))
        if status is None:
            ctx.sync()
        else:
            with pytest.raises(pcs.PcsError) as e:
                ctx.sync()
            assert e.value.status == status
        k = p.k.clone()
        k[int(p.table[0, 1]), 1:4] = p.nk[:3]
        assert torch.equal(p.dk.cpu(), k)


def test_append_reports_slots_and_positions_out_of_range(ctx, dev):
    for lens in ([100], [2]):  # beyond the table; more new tokens than the session has
        p = append_case(4, [20], [3], 2, 64, 16, 0, 0, torch.float16)
        cache, _, _ = kv_ref.on_gpu(pcs, p)
        batch = pcs.KvBatch(torch.tensor(lens, dtype=torch.int32, device=dev), 3)
        ctx.kv_append(cache, batch, p.nk.to(dev), p.nv.to(dev))
        with pytest.raises(pcs.PcsError) as e:
            ctx.sync()
        assert e.value.status == pcs.PCS_E_RANGE
        k = p.k.clone()
        if lens == [2]:
            k[int(p.table[0, 0]), 0:2] = p.nk[1:]
        assert torch.equal(p.dk.cpu(), k)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,pairs", [(128, (15, 24, 24)), (64, (9, 10, 10)), (80, (3, 3, 3)), (96, (13, 16, 16)),
                                       (64, (10, 10, 10)), (8, (1, 1, 1)), (256, (41, 43, 42)), (16, (2, 3, 3))])
def test_pairs_that_are_no_whole_vectors(ctx, dev, dtype, interleaved, dim, pairs):
    g = torch.Generator().manual_seed(dim + sum(pairs))
    pos, freq = positions(g, 37, 3), freqs(pairs, "cpu")
    x = torch.randn(37, 5, dim, generator=g).clamp(-5, 5).to(dtype)
    x[3, 2, 2 * sum(pairs):] = math.inf  # what stays does not meet a product
    rot = pcs.Rotary(pos.to(dev), freq.to(dev), pairs, interleaved)
    y = x.to(dev)
    got = ctx.rotate([y], rot)[0]
    want = kv_ref.turned(x, pos, freq, pairs, interleaved)
    m = 2 * sum(pairs)
    assert off_by(got[..., :m], want[..., :m], dtype) <= 0
    assert torch.equal(got[..., m:].cpu(), x[..., m:])
    ctx.rotate([y], rot, out=[y])
    assert torch.equal(y, got)
