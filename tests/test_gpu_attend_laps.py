"""GPU: attention of blocks of new tokens that lap the ring they are written to
(more new tokens than it has slots), with first tokens that stay, against the
definition in 64 bits."""
import pytest
import torch

import kv_ref
from paper_2607_21686_gb300 import pcs
from test_gpu_attend import TYPES, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim,dtype", [(64, TYPES[0]), (128, TYPES[1])])
@pytest.mark.parametrize("sinks,ring,rows", [(4, 64, 16), (16, 203, 8), (64, 128, 128), (100, 64, 16), (130, 150, 32),
                                             (5, 90, 17)])
def test_prompts_that_lap_their_ring(ctx, dim, dtype, sinks, ring, rows):
    # Lengths a little over sinks + ring: the run behind the first tokens begins
    # in a box that it shares with them.
    lens = [sinks + ring + d for d in (1, 7, rows, rows + 1)]
    p = kv_ref.Population(sinks + rows, lens, lens, 2, 1, dim, page_rows=rows, sinks=sinks, ring=ring, dtype=dtype)
    check(ctx, p)
    check(ctx, p, window=50)


def test_a_prompt_of_a_wide_page(ctx):
    p = kv_ref.Population(1, [700], [700], 1, 1, 64, page_rows=128, sinks=4, ring=600)
    check(ctx, p)


@pytest.mark.parametrize("dim,rows", [(64, 16), (128, 8), (128, 13)])
def test_blocks_of_first_tokens_alone(ctx, dim, rows):
    # Blocks of rows that see nothing of the ring, which begins behind them.
    p = kv_ref.Population(dim + rows, [600, 570], [600, 490], 1, 1, dim, page_rows=rows, sinks=300, ring=300)
    check(ctx, p)
    p = kv_ref.Population(rows, [24, 20], [24, 9], 64, 1, dim, page_rows=rows, sinks=8, ring=16)
    check(ctx, p)


class Far(kv_ref.Population):
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


@pytest.mark.parametrize("new", [2, 150])
@pytest.mark.parametrize("rows", [16, 13])
def test_sessions_of_two_billion_tokens(ctx, new, rows):
    lens = [2 ** 31 - 1, 2 ** 31 - 60, 2 ** 31 - 301]
    p = Far(new + rows, lens, [new] * 3, 2, 1, 64, page_rows=rows, sinks=9, ring=260)
    check(ctx, p)
    check(ctx, p, window=77)
