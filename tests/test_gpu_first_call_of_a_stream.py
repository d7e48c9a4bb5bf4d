"""GPU: a stream's first call puts its workspace's words to zero on that stream,
whatever torch's default stream is busy with."""
import pytest
import torch

import kv_ref
from paper_2607_21686_gb300 import pcs

pytestmark = pytest.mark.gpu


def test_calls_on_a_fresh_stream_beside_a_busy_one(ctx, dev):
    # Parts whose blocks count themselves in the workspace's words: words put to
    # zero late, behind the default stream's work, would lose count of some.
    p = kv_ref.Population(3, [1900], [1], 4, 2, 64)
    cache, batch, q = kv_ref.on_gpu(pcs, p)
    want, want_lse = ctx.attend(cache, batch, q, return_lse=True)
    torch.cuda.synchronize()
    for _ in range(60):
        with pcs.Context(0) as own:
            side = torch.cuda.Stream()
            with torch.cuda.stream(side):
                outs = [(torch.full_like(want, 7.0), torch.full_like(want_lse, 7.0)) for _ in range(300)]
            torch.cuda.synchronize()
            torch.cuda._sleep(4_000_000)  # the default stream
            for out, lse in outs:
                own.attend(cache, batch, q, out=out, lse=lse, stream=side)
            torch.cuda.synchronize()
            assert all(torch.equal(out, want) and torch.equal(lse, want_lse) for out, lse in outs)
            own.sync()


def test_an_error_beside_a_busy_default_stream_is_kept(ctx, dev):
    # A context made while the default stream is busy, and an error of another
    # stream before that one's work is over.
    p = kv_ref.Population(31, [60, 60], [1, 1], 2, 2, 64)
    p.table[1, 2] = 10 ** 6
    cache, batch, q = kv_ref.on_gpu(pcs, p)
    out = torch.empty_like(q)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)  # the default stream
    with pcs.Context(0) as own:
        own.attend(cache, batch, q, out=out, stream=side)
        with pytest.raises(pcs.PcsError) as e:
            own.sync(side)
        assert e.value.status == pcs.PCS_E_RANGE
        own.sync(side)  # reported once
    torch.cuda.synchronize()
