"""GPU: blocks of the kernels over 8-bit caches rank sessions by their lengths in memory that
their copies then fill: over and over, with the cache warm and cold, every pass of a call
gives the bits of the first, and those are right."""
import pytest
import torch

import kv8_ref as ref
from paper_2607_21686_gb300 import pcs

pytestmark = pytest.mark.gpu

U = torch.finfo(torch.bfloat16).eps / 2


@pytest.mark.parametrize("hk,dim,codes", [(4, 64, ref.E4M3), (2, 128, ref.I8), (1, 64, ref.I8)])
@pytest.mark.parametrize("new", [1, 2, 40])
def test_ranked_sessions_again_and_again(ctx, dev, hk, dim, codes, new):
    # Far more blocks than an SM holds, most of them of short sessions; one is long enough
    # that sessions are ranked.
    g = torch.Generator(device=dev).manual_seed(dim + new)
    lens = torch.randint(new, 90 + new, (150,), generator=g, device=dev).tolist() + [2500, 2500, 700, new]
    n, rows, pages = len(lens), 32, -(-2500 // 32)
    row = pcs.kv_row_bytes(hk, dim)
    k, v = (torch.randint(0, 0x7F, (n * pages, rows, row), generator=g, device=dev).to(torch.uint8) for _ in range(2))
    for pool in (k, v):  # codes of either sign and no NaN; scales near 1/64
        pool |= torch.randint(0, 2, pool.shape, generator=g, device=dev).to(torch.uint8) << 7
        pool[..., hk * dim:] = 119 + pool[..., hk * dim:] % 3
    table = torch.randperm(n * pages, generator=g, device=dev).reshape(n, pages).int()
    cache = pcs.KvCache(k, v, table, codes=codes, heads=hk, head_dim=dim)
    lens_on = torch.tensor(lens, dtype=torch.int32, device=dev)
    batch = pcs.KvBatch(lens_on, n * new, max_len=max(lens))
    q = torch.randn(n * new, 2 * hk, dim, generator=g, device=dev, dtype=torch.bfloat16) / 64
    first = ctx.attend(cache, batch, q, return_lse=True)
    off = torch.tensor([sum(lens[:i]) for i in range(n + 1)], dtype=torch.int32, device=dev)
    kk, vv = ctx.kv_read(cache, pcs.KvBatch(lens_on, sum(lens), off, max(lens)), dtype=torch.float32)
    ctx.sync()
    for s, m in enumerate(lens):
        at = slice(sum(lens[:s]), sum(lens[:s + 1]))
        ks, vs = (x[at].double().repeat_interleave(2, 1) for x in (kk, vv))
        x = torch.einsum("qhd,khd->hqk", q[s * new:(s + 1) * new].double(), ks) / dim ** 0.5
        x = x.masked_fill(~torch.ones(new, m, dtype=torch.bool, device=dev).tril(m - new), float("-inf"))
        w = x.softmax(-1)
        want, mass = (torch.einsum("hqk,khd->qhd", w, y) for y in (vs, vs.abs()))
        # The result and each weight are rounded once to bfloat16 or better; scores, sums of
        # dim exact products of at most `size` together, are off by dim roundings in 32 bits,
        # which a weight takes twice, as it takes those of m sums.  In float16 a small weight is
        # off by 2^-32 of the largest weight times scale, and meets codes of at most 2 max|v| / scale.
        size = torch.einsum("qhd,khd->hqk", q[s * new:(s + 1) * new].double().abs(), ks.abs()).max() / dim ** 0.5
        rel = 1.01 * U + 3 * ((dim + 8) * 2.0 ** -24 * (size + 1) + 2.0 ** -20) + m * 2.0 ** -23
        d = (first[0][s * new:(s + 1) * new].double() - want).abs()
        assert (d <= U * want.abs() + rel * mass + m * 2.0 ** -31 * vs.abs().max() + 2.0 ** -24).all(), s
    far = torch.empty(64 << 20, dtype=torch.int32, device=dev)
    for i in range(60):
        if i % 4 == 0:
            far.fill_(i)  # the pools leave the cache
        out, lse = ctx.attend(cache, batch, q, return_lse=True)
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1]), i
    ctx.sync()
