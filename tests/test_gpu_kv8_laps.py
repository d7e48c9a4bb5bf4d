"""GPU: 8-bit caches and trees at the ends of rings: prompts that lap the ring they are written
to, rings that wrap anywhere in a box, sessions of two billion tokens, against the definition
in 64 bits."""
import pytest
import torch

import kv8_ref as ref
import kv_ref
from test_gpu_kv8_forms import attend, check

pytestmark = pytest.mark.gpu

KINDS = [ref.E4M3, ref.I8]


@pytest.mark.parametrize("dim,hq,codes", [(64, 1, ref.I8), (128, 4, ref.E4M3)])
@pytest.mark.parametrize("sinks,ring,rows", [(4, 64, 16), (16, 203, 8), (64, 128, 128), (100, 64, 16), (130, 150, 32),
                                             (5, 90, 17)])
def test_prompts_that_lap_their_ring(ctx, dim, hq, codes, sinks, ring, rows):
    lens = [sinks + ring + d for d in (1, 7, rows, rows + 1)]
    p = ref.Population8(sinks + rows, lens, lens, hq, 1, dim, codes, page_rows=rows, sinks=sinks, ring=ring)
    check(ctx, p)
    check(ctx, p, window=50)


@pytest.mark.parametrize("codes", KINDS)
@pytest.mark.parametrize("sinks,ring", [(0, 101), (5, 64), (16, 203), (130, 190), (7, 129)])
@pytest.mark.parametrize("rows", [8, 24, 64])
@pytest.mark.parametrize("new", [1, 9])
def test_rings_that_wrap_anywhere(ctx, codes, sinks, ring, rows, new):
    lens = [ring + sinks + d for d in (-1, 0, 1, 7, 40, 100, ring // 2)]
    p = ref.Population8(ring + rows, lens, [new] * len(lens), 1, 1, 64, codes, page_rows=rows, sinks=sinks, ring=ring)
    check(ctx, p)
    check(ctx, p, window=77)
    p = ref.trees(codes, ring + rows, lens, [new] * len(lens), 3, 1, 64, page_rows=rows, sinks=sinks, ring=ring)
    check(ctx, p, window=77)


class Far:
    """Sessions too long to be walked from their first token."""

    def seen(self, s, p, window):
        n = self.lens[s]
        low = max(n - self.ring, p - window + 1 if window else 0)
        assert low >= self.sinks
        out = []
        for j in list(range(self.sinks)) + list(range(low, p + 1)):
            at = kv_ref.slot_of(j, self.sinks, self.ring)
            page = int(self.table[s, at // self.rows])
            out.append((j, page, page, at % self.rows))
        return out


class Far8(Far, ref.Population8):
    def reference(self, window=0, scale=None):
        """As Population8's, by the tokens that are there."""
        out, lse, tol, ltol = kv_ref.Population.reference(self, window, scale)
        largest = torch.nan_to_num(self.v.abs(), 0.0, 0.0, 0.0).amax()
        return out, lse, tol + (self.sinks + self.ring) * 2.0 ** -31 * largest, ltol


class FarTree8(ref.Trees, Far8):
    pass


class FarTree(ref.Trees, Far, kv_ref.Population):
    pass


@pytest.mark.parametrize("codes", KINDS)
@pytest.mark.parametrize("new,hq", [(1, 2), (2, 2), (40, 2), (150, 2), (150, 8)])
@pytest.mark.parametrize("rows", [16, 13])
def test_sessions_of_two_billion_tokens(ctx, codes, new, hq, rows):
    lens = [2 ** 31 - 1, 2 ** 31 - 60, 2 ** 31 - 301]
    p = Far8(new + rows, lens, [new] * 3, hq, 1, 64, codes, page_rows=rows, sinks=9, ring=260)
    out, lse = attend(ctx, p)
    ctx.sync()
    kv_ref.check_attend(p, out, lse)


@pytest.mark.parametrize("codes", KINDS + [None])
@pytest.mark.parametrize("new,hq", [(7, 2), (40, 2), (64, 8)])
@pytest.mark.parametrize("rows", [16, 13])
def test_trees_of_two_billion_tokens(ctx, codes, new, hq, rows):
    lens = [2 ** 31 - 1, 2 ** 31 - 60, 2 ** 31 - 301]
    args = (new + rows, lens, [new] * 3, hq, 1, 64)
    kw = dict(page_rows=rows, sinks=9, ring=260)
    p = FarTree(*args, **kw) if codes is None else FarTree8(*args, codes=codes, **kw)
    p.parents = ref.random_parents(p.g, p.new)
    out, lse = attend(ctx, p)
    ctx.sync()
    kv_ref.check_attend(p, out, lse)
