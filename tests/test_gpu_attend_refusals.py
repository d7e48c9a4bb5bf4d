"""GPU: what the operators over a paged cache refuse, and with which status.
Nothing is enqueued by a refused call."""
import ctypes
import math

import pytest
import torch

import kv_ref
from paper_2607_21686_gb300 import pcs

pytestmark = pytest.mark.gpu

INVAL, ALIGN = pcs.PCS_E_INVAL, pcs.PCS_E_ALIGN


def refused(status, call, *args, **kw):
    with pytest.raises(pcs.PcsError) as e:
        call(*args, **kw)
    assert e.value.status == status, str(e.value)


@pytest.fixture()
def world(ctx, dev):
    p = kv_ref.Population(1, [40, 40], [2, 2], 4, 2, 64)
    cache, batch, q = kv_ref.on_gpu(pcs, p)
    before = ctx.stats().kernel_launches
    yield p, cache, batch, q
    assert ctx.stats().kernel_launches == before


@pytest.mark.parametrize("field,value,status", [
    ("heads", 0, INVAL), ("heads", 3, INVAL), ("head_dim", 12, INVAL), ("head_dim", 256, INVAL),
    ("head_dim", 0, INVAL), ("head_dim", 128, INVAL), ("n_pages", 0, INVAL), ("page_rows", 0, INVAL),
    ("table_pages", -1, INVAL), ("page_rows", 2 ** 30, INVAL), ("table_stride", 1, INVAL), ("sinks", -1, INVAL),
    ("ring", -1, INVAL), ("ring", 10 ** 6, INVAL), ("page_stride", -8, INVAL), ("row_stride", 100, ALIGN),
    ("head_stride", 4, ALIGN), ("dtype", pcs.PCS_DT_F32, INVAL), ("dtype", pcs.PCS_DT_F16, INVAL), ("k", None, INVAL),
    ("v", None, INVAL), ("table", None, INVAL)])
def test_caches(ctx, world, field, value, status):
    p, cache, batch, q = world
    setattr(cache.struct, field, value)
    refused(status, ctx.attend, cache, batch, q)


def test_pools_off_16_bytes(ctx, world):
    p, cache, batch, q = world
    cache.struct.k += 2
    refused(ALIGN, ctx.attend, cache, batch, q)


@pytest.mark.parametrize("field,value", [("tokens", -1), ("tokens", 2 ** 31), ("tokens", 5), ("sessions", -1),
                                         ("sessions", 0), ("max_len", -1), ("lens", None)])
def test_batches(ctx, world, field, value):
    p, cache, batch, q = world
    setattr(batch.struct, field, value)
    refused(INVAL, ctx.attend, cache, batch, q)


def test_ragged_batches_say_their_most_new_tokens(ctx, dev, world):
    p, cache, _, q = world
    off = torch.tensor([0, 1, 4], dtype=torch.int32, device=dev)
    refused(INVAL, ctx.attend, cache, pcs.KvBatch(torch.tensor(p.lens, dtype=torch.int32, device=dev), 4, off), q)


def test_attend_arguments(ctx, dev, world):
    p, cache, batch, q = world
    for scale in (-1.0, math.nan, math.inf):
        refused(INVAL, ctx.attend, cache, batch, q, scale=scale)
    refused(INVAL, ctx.attend, cache, batch, q, window=-1)
    refused(INVAL, ctx.attend, cache, batch, q[:, :3].contiguous())      # 3 heads over 2
    refused(INVAL, ctx.attend, cache, batch, q.half())
    refused(INVAL, ctx.attend, cache, batch, q[..., :32].contiguous())
    refused(INVAL, ctx.attend, cache, batch, q, out=torch.empty(4, 2, 64, dtype=q.dtype, device=dev))
    wide = torch.zeros(4, 4, 68, dtype=q.dtype, device=dev)
    refused(ALIGN, ctx.attend, cache, batch, wide[..., :64])
    refused(ALIGN, ctx.attend, cache, batch, q, out=wide[..., 4:])
    for bad in (q[:3], q[0], q.cpu(), q.transpose(1, 2)):
        with pytest.raises(ValueError):
            ctx.attend(cache, batch, bad)
    with pytest.raises(ValueError):
        ctx.attend(cache, batch, q, lse=torch.empty(4, 4, dtype=torch.float64, device=dev))
    with pytest.raises(ValueError):
        ctx.attend(cache, pcs.KvBatch(torch.zeros(3, dtype=torch.int32, device=dev), 3), q[:3])
    lib = ctx.lib
    h = pcs._heads(q, "q", 4)
    par = pcs.pcs_attend_params(0.0, 0, 0, 0)
    for args in ((None, cache.struct, batch.struct, par, h, h), (ctx.h, None, batch.struct, par, h, h),
                 (ctx.h, cache.struct, None, par, h, h), (ctx.h, cache.struct, batch.struct, None, h, h),
                 (ctx.h, cache.struct, batch.struct, par, None, h), (ctx.h, cache.struct, batch.struct, par, h, None)):
        assert lib.pcs_attend(*args, None, None) == INVAL
        assert lib.pcs_last_error()


def test_append_arguments(ctx, dev, world):
    p, cache, batch, q = world
    k = q[:, :2].contiguous()
    refused(INVAL, ctx.kv_append, cache, batch, q, k)                     # 4 heads into 2
    refused(INVAL, ctx.kv_append, cache, batch, k, k.half())
    lib = ctx.lib
    hk, hq = pcs._heads(k, "k", 4), pcs._heads(q, "q", 4)
    assert lib.pcs_kv_append(ctx.h, cache.struct, batch.struct, None, hk, hk, hq, None, None) == INVAL
    assert lib.pcs_kv_append(ctx.h, cache.struct, batch.struct, None, hk, None, None, None, None) == INVAL
    with pytest.raises(ValueError):
        ctx.kv_append(cache, batch, k, k, q_out=q)
    pos = torch.zeros(3, 1, dtype=torch.int32, device=dev)
    with pytest.raises(ValueError):
        ctx.kv_append(cache, batch, k, k, rotary=pcs.Rotary(pos, torch.ones(4, device=dev), (4,)))


def test_rotary_arguments(ctx, dev, world):
    x = torch.zeros(3, 2, 16, device=dev)
    pos, freq = torch.zeros(3, 2, dtype=torch.int32, device=dev), torch.ones(9, device=dev)
    refused(INVAL, ctx.rotate, [x], pcs.Rotary(pos, freq, (4, 5)))        # 9 pairs in 16 elements
    ok = pcs.Rotary(pos, freq[:8], (4, 4))
    refused(INVAL, ctx.rotate, [x.double().float()[..., :0]], ok)
    refused(INVAL, ctx.rotate, [x, x.half()], ok)
    refused(INVAL, ctx.rotate, [x] * 9, ok)
    for field, value in (("axes", 0), ("axes", 5), ("flags", 4), ("pos", None), ("freq", None)):
        bad = pcs.Rotary(pos, freq[:8], (4, 4))
        setattr(bad.forward, field, value)
        refused(INVAL, ctx.rotate, [x], bad)
    bad = pcs.Rotary(pos, freq[:8], (4, 4))
    bad.forward.pairs[3] = 1
    refused(INVAL, ctx.rotate, [x], bad)
    for args in ((pos[:, :1], freq[:8], (4, 4)), (pos.long(), freq[:8], (4, 4)), (pos, freq, (4, 4)), (pos, freq[:8], ())):
        with pytest.raises(ValueError):
            pcs.Rotary(*args)
    with pytest.raises(ValueError):
        ctx.rotate([x[:2]], ok)
    assert ctx.rotate([], ok) == []
    assert ctx.lib.pcs_rotate(None, ok.forward, None, None, 0, 0, None) == INVAL
    assert ctx.lib.pcs_rotate(ctx.h, None, None, None, 0, 0, None) == INVAL


def test_pools_of_a_cache_agree(ctx, dev, world):
    k = torch.zeros(4, 16, 2, 64, dtype=torch.float16, device=dev)
    t = torch.zeros(2, 2, dtype=torch.int32, device=dev)
    for args in ((k, k[:3], t), (k, k.float(), t), (k, k.bfloat16(), t), (k, k.transpose(1, 2), t), (k, k, t.long()),
                 (k.cpu(), k.cpu(), t), (k[..., ::2], k[..., ::2], t), (k, k, t[0])):
        with pytest.raises(ValueError):
            pcs.KvCache(*args)


def test_long_and_out_of_place_sessions_are_bounded(ctx, dev):
    # Lengths far beyond the table and offsets outside the call's tensors, from
    # device memory: reported, skipped, and over at once.
    for new in (1, 40):
        p = kv_ref.Population(3, [64, 64], [new, new], 2, 2, 64)
        cache, _, q = kv_ref.on_gpu(pcs, p)
        lens = torch.tensor([2 ** 31 - 1, 64], dtype=torch.int32, device=dev)
        out = ctx.attend(cache, pcs.KvBatch(lens, 2 * new), q)
        with pytest.raises(pcs.PcsError) as e:
            ctx.sync()
        assert e.value.status == pcs.PCS_E_RANGE
        want = p.reference()
        assert ((out.cpu().double() - want[0]).abs() <= want[2])[new:].all()
        for off in ([-5, new - 5, 2 * new], [0, new, 2 * new + 7], [10 ** 9, 10 ** 9 + 1, 2 * new]):
            o = torch.tensor(off, dtype=torch.int32, device=dev)
            ctx.attend(cache, pcs.KvBatch(torch.tensor(p.lens, dtype=torch.int32, device=dev), 2 * new, o, new + 9), q)
            with pytest.raises(pcs.PcsError) as e:
                ctx.sync()
            assert e.value.status == pcs.PCS_E_RANGE
