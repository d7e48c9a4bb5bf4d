"""GPU: attention over 8-bit caches whose boxes of rows reach over the end of a ring, or
begin before a window: codes that stand for NaN and scales that do, in slots that no new
token sees, change no bit of a result."""
import pytest
import torch

import kv8_ref as ref
import kv_ref
from paper_2607_21686_gb300 import pcs

pytestmark = pytest.mark.gpu

JUNK = {"7f": (0x7F, 127), "ff": (0xFF, 120), "scale": (0x11, 255)}


def attend(ctx, p, window=0):
    cache, batch, q = ref.on_gpu(pcs, p)
    if getattr(p, "parents", None) is not None:
        out, lse = ctx.attend_tree(cache, batch, ref.parents_on(p), q, window=window, return_lse=True)
    else:
        out, lse = ctx.attend(cache, batch, q, window=window, return_lse=True)
    ctx.sync()
    return out, lse


def unseen(p, window):
    """Rows of the pools that no new token of any session sees."""
    seen = {(k, r) for s, m in enumerate(p.new) for i in range(m) for _, k, _, r in p.seen(s, p.lens[s] - m + i, window)}
    return [(page, r) for page in range(p.n_pages) for r in range(p.rows) if (page, r) not in seen]


def fill(p, places, kind):
    code, scale = JUNK[kind]
    n = p.hk * p.dim
    for page, r in places:
        for rows in (p.k_rows, p.v_rows):
            rows[page, r, :n] = code
            rows[page, r, n:n + p.hk] = scale


def same(ctx, p, window=0):
    """Junk wherever nobody looks; what came out before and with the last of it."""
    out, lse = attend(ctx, p, window)
    kv_ref.check_attend(p, out, lse, window)
    places = unseen(p, window)
    for kind in JUNK:
        fill(p, places, kind)
        again, lse2 = attend(ctx, p, window)
        assert torch.equal(out, again) and torch.equal(lse, lse2), kind
    return out


def lengths(sinks, ring, new):
    """The ring's end at many places of a tile, with many tokens or few behind it."""
    return [max(new, sinks + ring + d) for d in (-1, 0, 1, 9, ring // 3, ring // 2, 3 * ring + 45)]


@pytest.mark.parametrize("codes", [ref.E4M3, ref.I8])
@pytest.mark.parametrize("sinks,ring", [(0, 100), (0, 203), (5, 199), (16, 134), (17, 90), (40, 333)])
@pytest.mark.parametrize("rows,new", [(8, 1), (16, 1), (32, 1), (8, 3), (16, 3), (32, 3), (16, 40)])
def test_slots_behind_the_end_of_a_ring(ctx, codes, sinks, ring, rows, new):
    lens = lengths(sinks, ring, new)
    same(ctx, ref.Population8(ring + rows, lens, [new] * len(lens), 4, 2, 64, codes, sinks=sinks, ring=ring, page_rows=rows))


@pytest.mark.parametrize("hq,hk,dim", [(4, 4, 64), (3, 3, 128), (8, 1, 128), (24, 1, 64), (8, 2, 80)])
@pytest.mark.parametrize("window", [0, 70])
def test_forms_and_windows(ctx, hq, hk, dim, window):
    # Blocks of four heads, of two, of one; one, two and four tiles of query rows.
    for rows in (16, 24):
        lens = lengths(6, 187, 1)
        same(ctx, ref.Population8(hq + dim, lens, [1] * len(lens), hq, hk, dim, sinks=6, ring=187, page_rows=rows), window)


def test_long_rings(ctx):
    # Parts of a session; a tile of the gap deep inside one of them.
    for sinks, ring, n in ((16, 1000, 5000), (0, 1001, 1500), (5, 2043, 9000)):
        same(ctx, ref.Population8(ring, [n], [1], 4, 2, 64, sinks=sinks, ring=ring))
        same(ctx, ref.Population8(ring, [n, 60], [2, 2], 4, 4, 128, sinks=sinks, ring=ring, page_rows=32))


@pytest.mark.parametrize("codes", [ref.E4M3, ref.I8])
@pytest.mark.parametrize("sinks,ring", [(0, 100), (5, 199), (16, 134)])
@pytest.mark.parametrize("window", [0, 50])
@pytest.mark.parametrize("hq", [2, 32])
def test_trees(ctx, codes, sinks, ring, window, hq):
    for rows in (8, 16, 32):
        lens = lengths(sinks, ring, 7)
        same(ctx, ref.trees(codes, ring + rows, lens, [7] * len(lens), hq, 2, 64, sinks=sinks, ring=ring, page_rows=rows), window)


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("codes", [ref.E4M3, ref.I8])
@pytest.mark.parametrize("ring", [100, 134, 199])
def test_junk_behind_the_ring_beside_a_token_that_some_see(ctx, codes, ring, tree):
    # The last new token's values stand for NaN: in the tiles where rows are told apart, and
    # those of the gap among them, nobody else takes them.
    m = 4
    lens = lengths(3, ring, m)
    if tree:
        p = ref.trees(codes, ring, lens, [m] * len(lens), 4, 2, 64, sinks=3, ring=ring)
    else:
        p = ref.Population8(ring, lens, [m] * len(lens), 4, 2, 64, codes, sinks=3, ring=ring)
    out = same(ctx, p)
    for s, n in enumerate(lens):
        at = kv_ref.slot_of(n - 1, 3, ring)
        fill(p, [(int(p.table[s, at // 16]), at % 16)], "7f")
        p.k_rows[int(p.table[s, at // 16]), at % 16, 128:130] = 100  # (scores of next to nothing)
    again, _ = attend(ctx, p)
    for s in range(len(lens)):
        at = p.q_off[s + 1] - 1
        assert torch.equal(out[at - m + 1:at], again[at - m + 1:at])
        if codes == ref.E4M3:
            assert torch.isnan(again[at]).all()
        else:
            assert torch.isfinite(again[at]).all()
