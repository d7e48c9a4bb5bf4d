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
