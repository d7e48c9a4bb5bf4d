"""GPU: rows of a call's tensors behind the last session's, as a batch that is filled up to a
fixed size has them, are nobody's: what is read, appended and attended leaves them alone."""
import pytest
import torch

import kv8_ref as ref
import kv_ref
from paper_2607_21686_gb300 import pcs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("codes", [None, ref.E4M3, ref.I8])
@pytest.mark.parametrize("new,more", [([5, 0, 9], 7), ([70, 130, 3], 300), ([1, 1], 1), ([0, 0], 40)])
def test_rows_behind_the_last_session(ctx, dev, codes, new, more):
    cls = kv_ref.Population if codes is None else ref.Population8
    p = cls(len(new) + more, [n + 40 for n in new], new, 4, 2, 64, **({} if codes is None else {"codes": codes}))
    n = p.tokens
    cache, batch, q = ref.on_gpu(pcs, p, even=False)
    padded = pcs.KvBatch(batch.keep[0], n + more, batch.keep[1], max(new + [1]))
    for dtype in [p.dtype] if codes is None else [p.dtype, torch.float16, torch.float32]:
        k, v = ctx.kv_read(cache, batch, dtype=dtype) if n else (torch.empty(0, 2, 64, dtype=dtype, device=dev),) * 2
        k_out, v_out = (torch.full((n + more, 2, 64), 7.0, dtype=dtype, device=dev) for _ in range(2))
        ctx.kv_read(cache, padded, dtype=dtype, k_out=k_out, v_out=v_out)
        ctx.sync()
        assert torch.equal(k_out[:n], k) and torch.equal(v_out[:n], v)
        assert (k_out[n:] == 7).all() and (v_out[n:] == 7).all()
    # Attention, and an append, whose own rows are in the cache alone.
    wide = torch.cat([q, torch.full((more, 4, 64), float("nan"), dtype=p.dtype, device=dev)])
    out = torch.full_like(wide, 7.0)
    ctx.attend(cache, padded, wide, out=out)
    parent = torch.full((n + more,), -1, dtype=torch.int32, device=dev)
    if max(new) <= pcs.PCS_TREE_MAX:
        ctx.attend_tree(cache, padded, parent, wide, out=wide)
        assert torch.isnan(wide[n:]).all()
    ctx.sync()
    assert (out[n:] == 7).all()
    if n:
        assert torch.equal(out[:n], ctx.attend(cache, batch, q))
    pools = [x.clone() for x in cache.keep[:2]]
    k = torch.randn(n + more, 2, 64, device=dev).to(p.dtype)
    ctx.kv_append(cache, padded, k, k)
    got = [x.clone() for x in cache.keep[:2]]
    for x, y in zip(cache.keep[:2], pools):
        x.copy_(y)
    if n:
        ctx.kv_append(cache, batch, k[:n], k[:n])
    ctx.sync()
    assert all(torch.equal(x, y) for x, y in zip(got, cache.keep[:2]))
