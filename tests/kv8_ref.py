"""Caches in 8 bits and trees of drafted tokens for the tests: what codes stand
for, how they are made and what a node sees, restated in 64 bits element by
element, and populations of sessions over them (on top of kv_ref)."""
import math

import torch

import kv_ref

E4M3, I8 = torch.float8_e4m3fn, torch.int8
MOST = {E4M3: 448.0, I8: 127.0}


def _e4m3_values():
    """What the 256 codes stand for."""
    out = []
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        x = (8 + m) * 2.0 ** (e - 10) if e else m * 2.0 ** -9
        x = math.nan if e == 15 and m == 7 else x
        out.append(-x if c > 127 else x)
    return torch.tensor(out, dtype=torch.float64)


VALUES = {E4M3: _e4m3_values(),
          I8: torch.tensor([c if c < 128 else c - 256 for c in range(256)], dtype=torch.float64)}


def scale_byte(top, codes):
    """The byte of a head whose largest magnitude is `top` (255: not finite)."""
    if not math.isfinite(top):
        return 255
    e = -126
    while top > MOST[codes] * 2.0 ** e:
        e += 1
    return e + 127


def coded(x, codes):
    """Codes uint8 and scale bytes uint8 of heads x [.., dim] (any float type)."""
    y = x.double()
    tops = y.abs().amax(-1)
    tops = torch.where(torch.isfinite(y).all(-1), tops, math.inf)
    memo = {}
    b = torch.tensor([memo.setdefault(t, scale_byte(t, codes)) for t in tops.flatten().tolist()],
                     dtype=torch.int64).reshape(tops.shape)
    y = torch.where((b < 255)[..., None], y * 2.0 ** (127.0 - b.double())[..., None], 0.0)
    if codes == I8:
        c = torch.round(y).long() % 256
    else:
        # The nearest of the numbers that a code stands for, the even code of two.
        grid = VALUES[E4M3][:127]
        a = y.abs()
        hi = torch.searchsorted(grid, a.contiguous()).clamp(max=126)
        lo = (hi - 1).clamp(min=0)
        dl, dh = a - grid[lo], grid[hi] - a
        c = torch.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
        c = c + 128 * (torch.signbit(y)).long()
    return c.to(torch.uint8), b.to(torch.uint8)


def valued(c, b, codes):
    """What codes [.., dim] with scale bytes [..] stand for, in 64 bits."""
    scale = torch.where(b == 255, math.nan, 2.0 ** (b.double() - 127))
    return VALUES[codes][c.long()] * scale[..., None]


def rows_of(values, codes, row_bytes):
    """Rows [.., row bytes] of heads [.., heads, dim]."""
    c, b = coded(values, codes)
    h, d = values.shape[-2:]
    rows = torch.full(values.shape[:-2] + (row_bytes,), 0xA5, dtype=torch.uint8)
    rows[..., :h * d] = c.flatten(-2)
    rows[..., h * d:h * d + h] = b
    return rows


def heads_of(rows, codes, h, d):
    """What rows [.., row bytes] stand for [.., heads, dim], in 64 bits."""
    return valued(rows[..., :h * d].unflatten(-1, (h, d)), rows[..., h * d:h * d + h], codes)


class Population8(kv_ref.Population):
    """Sessions over pools of codes; k and v are what those stand for."""

    def __init__(self, seed, lens, new, q_heads, kv_heads, dim, codes=E4M3, row_bytes=None, sizes=0.7, **kw):
        super().__init__(seed, lens, new, q_heads, kv_heads, dim, **kw)
        self.codes = codes
        self.row_bytes = row_bytes or -(-kv_heads * (dim + 1) // 32) * 32
        for name in ("k", "v"):
            x = getattr(self, name).double()
            x = x * torch.exp(sizes * torch.randn(*x.shape[:3], 1, generator=self.g).double())
            self.set(name, x.to(self.dtype))

    def set(self, name, x):
        rows = rows_of(x, self.codes, self.row_bytes)
        setattr(self, name + "_rows", rows)
        setattr(self, name, heads_of(rows, self.codes, self.hk, self.dim))

    def refresh(self):
        """k and v after a change of the rows."""
        self.k, self.v = (heads_of(r, self.codes, self.hk, self.dim) for r in (self.k_rows, self.v_rows))

    def reference(self, window=0, scale=None):
        """As kv_ref's.  Few rows take weights with their values' scales: in float16 they
        are off by 2^-11 of themselves or 2^-32 of the largest weight times scale (2^7 of
        them are a number's last bit, 2^-25), and meet codes of at most 2 max|v| / scale
        (a scale is less than twice what the largest code needs)."""
        out, lse, tol, ltol = super().reference(window, scale)
        largest = torch.nan_to_num(self.v.abs(), 0.0, 0.0, 0.0).amax()
        return out, lse, tol + max(self.lens + [1]) * 2.0 ** -31 * largest, ltol


def on_gpu(pcs, p, dev="cuda:0", hint=True, even=None):
    """Cache, batch and queries of a population, in 8 bits or 16, on the GPU."""
    if not hasattr(p, "codes"):
        return kv_ref.on_gpu(pcs, p, dev, hint, even)
    even = (len(set(p.new)) == 1) if even is None else even
    p.dk, p.dv, p.dt = p.k_rows.to(dev), p.v_rows.to(dev), p.table.to(dev)
    cache = pcs.KvCache(p.dk, p.dv, p.dt, sinks=p.sinks, ring=p.ring,
                        v_table=None if p.v_table is None else p.v_table.to(dev),
                        codes=p.codes, heads=p.hk, head_dim=p.dim)
    lens = torch.tensor(p.lens, dtype=torch.int32, device=dev)
    off = torch.tensor(p.q_off, dtype=torch.int32, device=dev)
    batch = pcs.KvBatch(lens, p.tokens, None if even else off, max(p.new + [1]),
                        max(p.lens + [0]) if hint else 0)
    return cache, batch, p.q.to(dev)


# ---------------------------------------------------------------------------
# Trees
# ---------------------------------------------------------------------------

def random_parents(g, new, chain=0.5):
    """A parent for each new token: the one before it, or any before it, or -1."""
    out = []
    for m in new:
        for i in range(m):
            r = float(torch.rand(1, generator=g))
            out.append(i - 1 if r < chain else int(torch.randint(-1, i, (1,), generator=g)) if i else -1)
    return out


def line_of(parents, i):
    """Node i and its ancestors, the nearest first."""
    out = [i]
    while parents[out[-1]] >= 0:
        out.append(parents[out[-1]])
    return out


class Trees:
    """Mixed into a population: its new tokens are nodes of trees."""

    parents = None

    def seen(self, s, p, window):
        at, m, n = self.q_off[s], self.new[s], self.lens[s]
        first = n - m
        i = p - first
        line = line_of(self.parents[at:at + m], i)
        pos = first + len(line) - 1
        keep = []
        for j, kp, vp, r in super().seen(s, n - 1, 0):  # all that is there
            if j < first:
                where = j
            elif j - first in line:
                where = first + len(line) - 1 - line.index(j - first)
            else:
                continue
            if p >= 0 and (window == 0 or where > pos - window or where < self.sinks):
                keep.append((j, kp, vp, r))
        return keep


class TreePopulation(Trees, kv_ref.Population):
    pass


class TreePopulation8(Trees, Population8):
    pass


def trees(codes, seed, *args, chain=0.5, **kw):
    """A population of trees over 16 bits (codes None) or codes."""
    p = TreePopulation(seed, *args, **kw) if codes is None else TreePopulation8(seed, *args, codes=codes, **kw)
    p.parents = random_parents(p.g, p.new, chain)
    return p


def parents_on(p, dev="cuda:0"):
    return torch.tensor(p.parents, dtype=torch.int32, device=dev)
