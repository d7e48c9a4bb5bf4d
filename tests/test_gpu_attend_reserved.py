"""GPU: fields of the operators' structs that have no meaning yet are refused
unless they are 0, so that they can be given one."""
import pytest
import torch

import kv_ref
from paper_2607_21686_gb300 import pcs

pytestmark = pytest.mark.gpu


def test_reserved_fields_are_refused(ctx, dev):
    p = kv_ref.Population(1, [40, 40], [2, 2], 4, 2, 64)
    cache, batch, q = kv_ref.on_gpu(pcs, p)
    lib, before = ctx.lib, ctx.stats().kernel_launches
    k = q[:, :2].contiguous()
    hq, hk = pcs._heads(q, "q", 4), pcs._heads(k, "k", 4)
    pos = torch.zeros(4, 1, dtype=torch.int32, device=dev)
    rotary = pcs.Rotary(pos, torch.ones(4, device=dev), (4,)).forward

    def attend(b=batch.struct, par=pcs.pcs_attend_params(0.0, 0, 0, 0), x=hq, y=hq):
        return lib.pcs_attend(ctx.h, cache.struct, b, par, x, y, None, None)

    def heads(h):
        return pcs.pcs_heads(h.data, h.token_stride, h.head_stride, h.heads, h.head_dim, h.dtype, 1)

    b = batch.struct
    other = pcs.pcs_kv_batch(b.lens, b.q_off, b.tokens, b.sessions, b.max_new, b.max_len, 7)
    refused = [
        attend(par=pcs.pcs_attend_params(0.0, 0, 1, 0)), attend(par=pcs.pcs_attend_params(0.0, 0, 0, 1)),
        attend(b=other), attend(x=heads(hq)), attend(y=heads(hq)),
        lib.pcs_kv_append(ctx.h, cache.struct, other, None, hk, hk, None, None, None),
        lib.pcs_kv_append(ctx.h, cache.struct, b, None, heads(hk), hk, None, None, None),
        lib.pcs_kv_append(ctx.h, cache.struct, b, None, hk, heads(hk), None, None, None),
        lib.pcs_kv_append(ctx.h, cache.struct, b, None, hk, hk, heads(hq), hq, None),
        lib.pcs_kv_append(ctx.h, cache.struct, b, None, hk, hk, hq, heads(hq), None),
        lib.pcs_rotate(ctx.h, rotary, heads(hq), hq, 1, 4, None), lib.pcs_rotate(ctx.h, rotary, hq, heads(hq), 1, 4, None)]
    assert refused == [pcs.PCS_E_INVAL] * len(refused)
    assert b"0" in lib.pcs_last_error()
    assert ctx.stats().kernel_launches == before
    assert attend() == pcs.PCS_OK
    ctx.sync()
