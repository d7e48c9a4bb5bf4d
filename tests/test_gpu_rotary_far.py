"""GPU: rotary positions keep the accuracy of a float's angle at every position
that 32 bits hold, against angles whose product of position (31 bits) and frequency (24) is exact."""
import numpy as np
import pytest
import torch

from paper_2607_21686_gb300 import pcs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("top", [1.0, 0.9999, 3.7])
def test_far_positions(ctx, dev, interleaved, top):
    g = torch.Generator().manual_seed(int(1000 * top))
    n = 400
    far = torch.randint(2 ** 24, 2 ** 31, (n, 1), generator=g)
    near = torch.randint(0, 2 ** 20, (n, 1), generator=g)
    pos = torch.cat([far, -far, near, torch.tensor([[2 ** 31 - 1], [-2 ** 31], [0], [2 ** 24 + 1], [4095], [4096]])]).int()
    pairs = 24
    freq = (top * torch.exp(torch.rand(pairs, generator=g, dtype=torch.float64) * -3)).float()
    freq[0] = top
    x = torch.randn(pos.shape[0], 2, 48, generator=g).clamp(-5, 5)
    rot = pcs.Rotary(pos.to(dev), freq.to(dev), (pairs,), interleaved)
    got = ctx.rotate([x.to(dev)], rot)[0].cpu().double()
    angle = pos.numpy().astype(np.longdouble) * freq.numpy().astype(np.longdouble)  # 55 bits: exact
    c, t = (torch.from_numpy(f(angle).astype(np.float64))[:, None] for f in (np.cos, np.sin))
    want = x.double().clone()
    a, b = (slice(0, None, 2), slice(1, None, 2)) if interleaved else (slice(0, pairs), slice(pairs, None))
    u, v = x[..., a].double(), x[..., b].double()
    want[..., a], want[..., b] = u * c - v * t, u * t + v * c
    # One rounding of the result; angles, cosines and products in 32 bits are off
    # by a few units of the largest element of a pair (at most 8 here).
    tol = 2.0 ** -24 * 1.0001 * want.abs() + 8 * 8 * 2.0 ** -24
    off = (got - want).abs() - tol
    assert (off <= 0).all(), off.max()
