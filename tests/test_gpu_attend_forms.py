"""GPU: forms of the operators over a paged cache that belong together and are
reached by no other test: keys appended as neighbouring pairs, rings with first
tokens under heads of 128, and blocks over them whose tokens are split."""
import pytest
import torch

import kv_ref
from paper_2607_21686_gb300 import pcs
from test_gpu_attend import TYPES, attend, check
from test_gpu_rotary import append_case, freqs, off_by, positions

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim,pairs,shift", [(64, (8, 12, 12), 0), (64, (9, 10, 10), 0), (80, (5, 3, 9), 0), (8, (1, 1, 2), 0),
                                             (128, (16, 24, 24), 0), (64, (8, 12, 12), 1)])
def test_append_of_neighbouring_pairs(ctx, dev, dtype, dim, pairs, shift):
    p = append_case(dim + sum(pairs), [100, 7, 90], [70, 1, 33], 2, dim, 24, 5, 60, dtype, hq=4)
    cache, batch, q = kv_ref.on_gpu(pcs, p)
    pos, freq = positions(p.g, p.tokens, 3), freqs(pairs, "cpu")
    rot = pcs.Rotary(pos.to(dev), freq.to(dev), pairs, interleaved=True)
    wide = torch.zeros(p.tokens, 2, dim + 8, dtype=dtype, device=dev)
    nk = wide[..., shift:shift + dim]  # (shift: off 16 bytes)
    nk.copy_(p.nk)
    got = ctx.kv_append(cache, batch, nk, p.nv.to(dev), q, rot)
    ctx.sync()
    assert off_by(got, kv_ref.turned(p.q, pos, freq, pairs, True), dtype) <= 0
    wk = kv_ref.turned(p.nk, pos, freq, pairs, True)
    k, v = p.k.double(), p.v.clone()
    for s, m in enumerate(p.new):
        for i in range(m):  # in order: the last token of a slot stays
            at = kv_ref.slot_of(p.lens[s] - m + i, p.sinks, p.ring)
            page, row = int(p.table[s, at // 24]), at % 24
            k[page, row], v[page, row] = wk[p.q_off[s] + i], p.nv[p.q_off[s] + i]
    assert torch.equal(p.dv.cpu(), v)
    assert off_by(p.dk, k, dtype) <= 0


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [8, 13, 32])
@pytest.mark.parametrize("sinks,ring", [(0, 301), (16, 333), (130, 190)])
def test_rings_and_first_tokens_of_wide_heads(ctx, dtype, rows, sinks, ring):
    lens = [ring + sinks + d for d in (-1, 40, ring // 2)]
    p = kv_ref.Population(ring + rows, lens, [40, 150, 50], 2, 1, 128, page_rows=rows, sinks=sinks, ring=ring, dtype=dtype)
    check(ctx, p)
    check(ctx, p, window=77)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("rows", [8, 17, 64])
@pytest.mark.parametrize("sinks,ring,over", [(0, 1500, 700), (20, 1701, 33), (300, 1400, 1390), (7, 2000, -300)])
def test_split_tokens_of_rings(ctx, dim, rows, sinks, ring, over):
    p = kv_ref.Population(dim + over, [sinks + ring + over], [60], 1, 1, dim, page_rows=rows, sinks=sinks, ring=ring)
    out, lse = check(ctx, p)
    again, lse2 = attend(ctx, p)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    check(ctx, p, window=1100)


@pytest.mark.parametrize("bad,status", [(-1, None), (10 ** 6, pcs.PCS_E_RANGE), (-7, pcs.PCS_E_RANGE)])
@pytest.mark.parametrize("of_values", [False, True])
def test_append_writes_keys_and_values_or_neither(ctx, dev, bad, status, of_values):
    p = append_case(4, [20, 20], [3, 3], 2, 64, 16, 0, 0, torch.float16)
    vt = torch.flip(p.table, (1,)).contiguous()
    (vt if of_values else p.table)[1, 1] = bad
    dk, dv = p.k.to(dev), p.v.to(dev)
    cache = pcs.KvCache(dk, dv, p.table.to(dev), v_table=vt.to(dev))
    batch = pcs.KvBatch(torch.tensor(p.lens, dtype=torch.int32, device=dev), 6)
    ctx.kv_append(cache, batch, p.nk.to(dev), p.nv.to(dev))
    if status is None:
        ctx.sync()
    else:
        with pytest.raises(pcs.PcsError) as e:
            ctx.sync()
        assert e.value.status == status
    k, v = p.k.clone(), p.v.clone()
    k[int(p.table[0, 1]), 1:4] = p.nk[:3]
    v[int(vt[0, 1]), 1:4] = p.nv[:3]
    assert torch.equal(dk.cpu(), k) and torch.equal(dv.cpu(), v)
