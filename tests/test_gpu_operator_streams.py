"""GPU: results that the operators' calls make on a stream given to them."""
import pytest
import torch

import kv_ref
from paper_2607_21686_gb300 import pcs

pytestmark = pytest.mark.gpu


def population():
    return kv_ref.Population(3, [90, 33], [20, 20], 8, 2, 64)


def pending(like):
    """A tensor of this size that the current stream is still to write, given back."""
    x = torch.empty_like(like, memory_format=torch.contiguous_format)
    torch.cuda._sleep(40_000_000)
    x.fill_(7.0)


@pytest.mark.parametrize("handle", [False, True])
def test_results_on_another_stream(ctx, dev, handle):
    # A result must not lie in memory that another stream is still to write.
    p = population()
    cache, batch, q = kv_ref.on_gpu(pcs, p)
    k, v = q[:, :2].contiguous(), q[:, 2:4].contiguous()
    pos = torch.arange(40, dtype=torch.int32, device=dev)[:, None].contiguous()
    rot = pcs.Rotary(pos, torch.rand(32, device=dev), (32,))
    side = torch.cuda.Stream()
    given = side.cuda_stream if handle else side
    calls = {
        "attend": lambda s: ctx.attend(cache, batch, q, stream=s, return_lse=True),
        "rotate": lambda s: ctx.rotate([q, k], rot, stream=s),
        "kv_append": lambda s: ctx.kv_append(cache, batch, k, v, q, rot, stream=s),
    }
    for name, call in calls.items():
        want = call(None)
        want = [x.clone() for x in (want if isinstance(want, (list, tuple)) else [want])]
        torch.cuda.synchronize()
        for x in want:
            pending(x)
        got = call(given)
        torch.cuda.synchronize()
        got = got if isinstance(got, (list, tuple)) else [got]
        assert all(torch.equal(a, b) for a, b in zip(got, want)), name
    ctx.sync()
