"""Rotary positions, append and attention over a paged cache in 64 bits, and
how far a result in 16 bits may be from them.

The definitions are restated here token by token: a position's slot, what a
token sees, a softmax over it.
"""
import math

import torch

# Unit roundoff of the types: half the distance of 1 from the next number.
ROUND = {t: torch.finfo(t).eps / 2 for t in (torch.bfloat16, torch.float16, torch.float32)}


def slot_of(p, sinks, ring):
    return p if ring == 0 or p < sinks else sinks + (p - sinks) % ring


def turned(x, pos, freq, pairs, interleaved=False, inverse=False):
    """x [tokens, heads, dim] rotated, in float64."""
    y = x.detach().cpu().double().clone()
    pos, freq = pos.cpu().double(), freq.cpu().double()
    n, i = sum(pairs), 0
    for axis, m in enumerate(pairs):
        for j in range(i, i + m):
            ang = pos[:, axis] * freq[j] * (-1.0 if inverse else 1.0)
            c, s = torch.cos(ang)[:, None], torch.sin(ang)[:, None]
            a, b = (2 * j, 2 * j + 1) if interleaved else (j, n + j)
            u, v = y[:, :, a].clone(), y[:, :, b].clone()
            y[:, :, a], y[:, :, b] = u * c - v * s, u * s + v * c
        i += m
    return y


class Population:
    """Sessions over a pool: lens and new tokens per session, pages anywhere."""

    def __init__(self, seed, lens, new, q_heads, kv_heads, dim, page_rows=16, sinks=0, ring=0,
                 dtype=torch.bfloat16, spare=3, v_table=False, spread=1.0):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.new = list(lens), list(new)
        self.hq, self.hk, self.dim, self.rows = q_heads, kv_heads, dim, page_rows
        self.sinks, self.ring, self.dtype = sinks, ring, dtype
        slots = max([1, sinks + ring if ring else max(lens)])
        self.pages = -(-slots // page_rows)
        n = len(self.lens) * self.pages
        self.n_pages = n + spare
        self.k = (torch.randn(self.n_pages, page_rows, kv_heads, dim, generator=g) * spread).to(dtype)
        self.v = torch.randn(self.n_pages, page_rows, kv_heads, dim, generator=g).to(dtype)
        self.table = torch.randperm(self.n_pages, generator=g)[:n].reshape(-1, self.pages).int()
        self.v_table = None
        if v_table:
            self.v_table = torch.randperm(self.n_pages, generator=g)[:n].reshape(-1, self.pages).int()
        self.q_off = [0]
        for m in self.new:
            self.q_off.append(self.q_off[-1] + m)
        self.tokens = self.q_off[-1]
        self.q = (torch.randn(self.tokens, q_heads, dim, generator=g) * spread).to(dtype)
        self.g = g

    def seen(self, s, p, window):
        """Positions that the token at p of session s sees and their places."""
        out = []
        n = self.lens[s]
        vt = self.table if self.v_table is None else self.v_table
        for j in range(0, min(p + 1, n)):
            if self.ring and j >= self.sinks and j < n - self.ring:
                continue
            if window and j >= self.sinks and j <= p - window:
                continue
            at = slot_of(j, self.sinks, self.ring)
            if at // self.rows >= self.pages:
                continue
            kp, vp = int(self.table[s, at // self.rows]), int(vt[s, at // self.rows])
            if 0 <= kp < self.n_pages and 0 <= vp < self.n_pages:
                out.append((j, kp, vp, at % self.rows))
        return out

    def reference(self, window=0, scale=None):
        """out, lse in float64 and each value's bound."""
        scale = 1.0 / math.sqrt(self.dim) if scale is None else scale
        group = self.hq // self.hk
        u = ROUND[self.dtype]
        out = torch.zeros(self.tokens, self.hq, self.dim, dtype=torch.float64)
        lse = torch.full((self.tokens, self.hq), -math.inf, dtype=torch.float64)
        tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
        for s, m in enumerate(self.new):
            for i in range(m):
                t, p = self.q_off[s] + i, self.lens[s] - m + i
                see = self.seen(s, p, window)
                if not see:
                    continue
                _, kp, vp, r = (torch.tensor(x) for x in zip(*see))
                k = self.k[kp, r].double().repeat_interleave(group, 1)  # [n, hq, d]
                v = self.v[vp, r].double().repeat_interleave(group, 1)
                q = self.q[t].double()
                x = torch.einsum("hd,nhd->hn", q, k) * scale
                lse[t] = torch.logsumexp(x, 1)
                w = torch.exp(x - lse[t][:, None])
                out[t] = torch.einsum("hn,nhd->hd", w, v)
                # A score is a sum of dim exact products in 32 bits: off by at
                # most dim roundings of the sum of their sizes (es).  A weight
                # takes that twice (itself and the total) and is rounded to the
                # type; small float16 weights are rounded to 2^-25 of the
                # largest.  The result is rounded once more.
                size = torch.einsum("hd,nhd->hn", q.abs(), k.abs()).amax(1) * scale
                es = (self.dim + 8) * 2.0 ** -24 * (size + 1.0) + 2.0 ** -20
                n = len(see)
                mass = torch.einsum("hn,nhd->hd", w, v.abs())
                tol[t] = u * out[t].abs() + (1.01 * u + 3 * es[:, None] + n * 2.0 ** -23) * mass \
                    + 2.0 ** -25 * v.abs().sum(0) + 2.0 ** -24
                ltol[t] = 2 * es + n * 2.0 ** -23 + 2.0 ** -21 * lse[t].abs()
        return out, lse, tol, ltol


def on_gpu(pcs, p, dev="cuda:0", hint=True, even=None):
    """Cache, batch and queries of a population on the GPU."""
    even = (len(set(p.new)) == 1) if even is None else even
    p.dk, p.dv, p.dt = p.k.to(dev), p.v.to(dev), p.table.to(dev)
    cache = pcs.KvCache(p.dk, p.dv, p.dt, sinks=p.sinks, ring=p.ring,
                        v_table=None if p.v_table is None else p.v_table.to(dev))
    lens = torch.tensor(p.lens, dtype=torch.int32, device=dev)
    off = torch.tensor(p.q_off, dtype=torch.int32, device=dev)
    batch = pcs.KvBatch(lens, p.tokens, None if even else off, max(p.new + [1]),
                        max(p.lens + [0]) if hint else 0)
    return cache, batch, p.q.to(dev)


def check_attend(p, got, lse, window=0, scale=None):
    out, ref_lse, tol, ltol = p.reference(window, scale)
    got, lse = got.cpu().double(), lse.cpu().double()
    assert torch.isfinite(got).all()
    off = (got - out).abs() - tol
    assert (off <= 0).all(), "value off by %g more than its bound" % off.max()
    empty = torch.isinf(ref_lse)
    assert torch.equal(torch.isinf(lse) & (lse < 0), empty)
    d = ((lse - ref_lse).abs() - ltol)[~empty]
    assert d.numel() == 0 or (d <= 0).all(), "lse off by %g more than its bound" % d.max()
