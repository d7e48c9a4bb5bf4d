"""GPU: caches in 8 bits against their definition in 64 bits (tests/kv8_ref.py):
append, read back, attention of single tokens, of a few and of blocks."""
import math

import pytest
import torch

import kv8_ref as ref
import kv_ref
from paper_2607_21686_gb300 import pcs

pytestmark = pytest.mark.gpu

KINDS = [ref.E4M3, ref.I8]
TYPES = [torch.bfloat16, torch.float16]


# ---------------------------------------------------------------------------
# Append
# ---------------------------------------------------------------------------

def appended(ctx, dev, p, k, v, rotary=None, q=None):
    """The pools' rows after an append into pools of 0xA5."""
    p.k_rows.fill_(0xA5)
    p.v_rows.fill_(0xA5)
    cache, batch, _ = ref.on_gpu(pcs, p)
    out = ctx.kv_append(cache, batch, k.to(dev), v.to(dev), None if q is None else q.to(dev), rotary)
    ctx.sync()
    return p.dk.cpu(), p.dv.cpu(), out


def places(p):
    """(token, pages of key and value, row) of the new tokens that stay."""
    out = {}
    for s, m in enumerate(p.new):
        for i in range(m):
            pos = p.lens[s] - m + i
            at = kv_ref.slot_of(pos, p.sinks, p.ring)
            if p.ring and pos >= p.sinks and pos < p.lens[s] - p.ring:
                continue
            vt = p.table if p.v_table is None else p.v_table
            out[(s, at)] = (p.q_off[s] + i, int(p.table[s, at // p.rows]), int(vt[s, at // p.rows]), at % p.rows)
    return list(out.values())


def expected(p, k, v):
    """Rows of the pools after an append of k and v into rows of 0xA5."""
    want = [torch.full_like(p.k_rows, 0xA5) for _ in range(2)]
    n = p.hk * p.dim
    for x, w, which in ((k, want[0], 1), (v, want[1], 2)):
        c, b = ref.coded(x, p.codes)
        for at in places(p):
            if at[1] < 0 or at[2] < 0:
                continue
            w[at[which], at[3], :n] = c[at[0]].flatten()
            w[at[which], at[3], n:n + p.hk] = b[at[0]]
    return want


@pytest.mark.parametrize("codes", KINDS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hk,dim", [(16, 64), (1, 128), (3, 16), (2, 80), (5, 96), (4, 48), (1, 112)])
def test_append_writes_the_codes_of_the_definition(ctx, dev, codes, dtype, hk, dim):
    p = ref.Population8(dim + hk, [40, 3, 90], [17, 1, 60], hk, hk, dim, codes, dtype=dtype)
    g = torch.Generator().manual_seed(dim)
    k, v = ((torch.randn(p.tokens, hk, dim, generator=g) * torch.exp(3 * torch.randn(p.tokens, hk, 1, generator=g)))
            .to(dtype) for _ in range(2))
    got = appended(ctx, dev, p, k, v)
    for x, w in zip(got, expected(p, k, v)):
        assert torch.equal(x, w)


@pytest.mark.parametrize("codes", KINDS)
@pytest.mark.parametrize("dtype", TYPES)
def test_append_at_the_borders(ctx, dev, codes, dtype):
    # Largest elements at and around the codes' ends, ties, zeros, the smallest numbers of
    # the type, infinities and NaN.
    most = ref.MOST[codes]
    info = torch.finfo(dtype)
    rows = []
    for e in (-10, 0, 5):
        for t in (most, most * 1.0078125, most * 0.99609375, most / 2, most * 1.25):
            x = torch.linspace(-1, 1, 32) * t * 2.0 ** e
            x[0] = t * 2.0 ** e
            rows.append(x)
    x = torch.zeros(32)
    rows += [x, torch.full((32,), info.tiny), torch.full((32,), info.smallest_normal * info.eps),
             torch.full((32,), info.max), torch.full((32,), -info.max)]
    tie = torch.arange(32) + 0.5
    tie[0] = most
    rows += [tie, -tie, torch.arange(32) * 2.0 ** -9]
    for bad in (math.inf, -math.inf, math.nan):
        x = torch.randn(32, generator=torch.Generator().manual_seed(1))
        x[7] = bad
        rows.append(x)
    k = torch.stack(rows)[:, None].to(dtype)
    v = k.flip(0)
    p = ref.Population8(1, [len(rows) + 5], [len(rows)], 1, 1, 32, codes, dtype=dtype)
    got = appended(ctx, dev, p, k, v)
    for x, w in zip(got, expected(p, k, v)):
        assert torch.equal(x, w)


@pytest.mark.parametrize("codes", KINDS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pairs,interleaved", [((32,), False), ((8, 12, 12), False), ((20,), False), ((18,), False),
                                               ((15,), False), ((0,), False), ((32,), True), ((15,), True), ((3, 4), True)])
def test_append_rotates_first(ctx, dev, codes, dtype, pairs, interleaved):
    # What is written is what pcs_rotate would give, in codes; queries come out rotated.
    p = ref.Population8(sum(pairs), [500, 90], [70, 33], 4, 2, 64, codes, dtype=dtype)
    g = torch.Generator().manual_seed(9)
    k, v = (torch.randn(p.tokens, 2, 64, generator=g).to(dtype) for _ in range(2))
    pos = torch.randint(-50, 100000, (p.tokens, len(pairs)), generator=g).int().to(dev)
    freq = torch.rand(sum(pairs), generator=g).to(dev)
    rotary = pcs.Rotary(pos, freq, pairs, interleaved)
    kr, qr = ctx.rotate([k.to(dev), p.q.to(dev)], rotary)
    dk, dv, q = appended(ctx, dev, p, k, v, rotary, p.q)
    want = expected(p, kr.cpu(), v)
    assert torch.equal(q, qr)
    assert torch.equal(dk, want[0]) and torch.equal(dv, want[1])
    # Any alignment, in place.
    wide = torch.zeros(p.tokens, 7, 67, dtype=dtype, device=dev)
    wide[:, :4, 1:65], wide[:, 4:6, 2:66] = p.q.to(dev), k.to(dev)
    cache, batch, _ = ref.on_gpu(pcs, p)
    qw = wide[:, :4, 1:65]
    ctx.kv_append(cache, batch, wide[:, 4:6, 2:66], v.to(dev), qw, rotary, q_out=qw)
    assert torch.equal(qw, qr)
    assert torch.equal(p.dk.cpu(), want[0]) and torch.equal(p.dv.cpu(), want[1])


@pytest.mark.parametrize("sinks,ring", [(0, 64), (5, 64), (16, 20), (100, 40)])
@pytest.mark.parametrize("codes", KINDS)
def test_append_into_rings(ctx, dev, sinks, ring, codes):
    p = ref.Population8(ring, [30, 100, 300, 64, 1], [30, 90, 5, 64, 1], 4, 4, 64, codes, sinks=sinks, ring=ring,
                        page_rows=24, v_table=True)
    p.table[2, 0] = -1
    k, v = (torch.randn(p.tokens, 4, 64, generator=p.g).bfloat16() for _ in range(2))
    got = appended(ctx, dev, p, k, v)
    for x, w in zip(got, expected(p, k, v)):
        assert torch.equal(x, w)


# ---------------------------------------------------------------------------
# Read back
# ---------------------------------------------------------------------------

def read_expected(p, pool, table, dtype):
    out = torch.zeros(p.tokens, p.hk, p.dim, dtype=torch.float64)
    for t, kp, vp, r in places(p):
        if 0 <= kp < p.n_pages and 0 <= vp < p.n_pages:
            out[t] = pool[kp if table == "k" else vp, r].double()
    # (Exact in bfloat16 but for numbers below its normal ones.)
    return out.to(dtype)


@pytest.mark.parametrize("codes", KINDS + [None])
@pytest.mark.parametrize("hk,dim,rows", [(16, 64, 16), (1, 128, 24), (3, 80, 5), (8, 128, 32), (2, 16, 1)])
def test_read_back(ctx, dev, codes, hk, dim, rows):
    lens, new = [500, 7, 60, 33], [300, 7, 0, 32]
    cls = kv_ref.Population if codes is None else ref.Population8
    kw = {} if codes is None else {"codes": codes}
    p = cls(dim, lens, new, hk, hk, dim, page_rows=rows, v_table=True, sinks=6, ring=130, **kw)
    p.table[0, 1] = -1
    cache, batch, _ = ref.on_gpu(pcs, p)
    types = [p.dtype] if codes is None else [torch.bfloat16, torch.float16, torch.float32]
    for dtype in types:
        k, v = ctx.kv_read(cache, batch, dtype=dtype)
        ctx.sync()
        assert k.dtype == dtype
        assert torch.equal(k.cpu(), read_expected(p, p.k, "k", dtype))
        assert torch.equal(v.cpu(), read_expected(p, p.v, "v", dtype))
    k, v = ctx.kv_read(cache, batch)
    assert k.dtype == torch.bfloat16
    # One of the two, and into wider tensors.
    wide = torch.full((p.tokens, 2 * hk + 1, dim + 16), 7.0, dtype=k.dtype, device=dev)
    ctx.kv_read(cache, batch, dtype=k.dtype, k_out=wide[:, 1:1 + hk, :dim], v_out=wide[:, 1 + hk:, 16:])
    assert torch.equal(wide[:, 1:1 + hk, :dim], k) and torch.equal(wide[:, 1 + hk:, 16:], v)
    assert (wide[:, 0] == 7).all() and (wide[:, 1:1 + hk, dim:] == 7).all() and (wide[:, 1 + hk:, :16] == 7).all()
    alone = torch.zeros_like(v)
    assert ctx.lib.pcs_kv_read(ctx.h, cache.struct, batch.struct, None, pcs._heads(alone, "v", p.tokens),
                               pcs._stream_ptr(None)) == pcs.PCS_OK
    assert torch.equal(alone, v)


@pytest.mark.parametrize("codes", KINDS)
def test_every_code_and_scale_reads_as_what_it_stands_for(ctx, dev, codes):
    # All codes at all scales: 16 heads of 16 codes, 256 rows of the scale byte.
    p = ref.Population8(1, [256], [256], 16, 16, 16, codes)
    for j in range(256):
        row = p.k_rows[int(p.table[0, j // 16]), j % 16]
        row[:256] = torch.arange(256, dtype=torch.uint8)
        row[256:272] = j
    p.refresh()
    cache, batch, _ = ref.on_gpu(pcs, p)
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        k, _ = ctx.kv_read(cache, batch, dtype=dtype)
        want = read_expected(p, p.k, "k", torch.float64)
        if dtype == torch.float16:
            want = want.clamp(-65504, 65504)
        # (Overflow of 448 * 2^127 in 32 bits.)
        want = torch.where(want.abs() > torch.finfo(torch.float32).max, torch.sign(want) * math.inf, want).to(dtype)
        got = k.cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(got, 0.0, math.inf, -math.inf), torch.nan_to_num(want, 0.0, math.inf, -math.inf))


# ---------------------------------------------------------------------------
# Attention
# ---------------------------------------------------------------------------

def attend(ctx, p, window=0, scale=0.0, hint=True, even=None):
    cache, batch, q = ref.on_gpu(pcs, p, hint=hint, even=even)
    out, lse = ctx.attend(cache, batch, q, window=window, scale=scale, return_lse=True)
    ctx.sync()
    return out, lse


def check(ctx, p, window=0, scale=None, **kw):
    out, lse = attend(ctx, p, window, scale or 0.0, **kw)
    kv_ref.check_attend(p, out, lse, window, scale)
    return out, lse


@pytest.mark.parametrize("codes", KINDS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hq,hk,dim", [(16, 16, 64), (8, 1, 128), (12, 4, 128), (2, 2, 16), (10, 2, 80), (6, 2, 96),
                                       (32, 2, 64), (25, 1, 48), (4, 4, 112), (32, 1, 128)])
def test_one_token(ctx, codes, dtype, hq, hk, dim):
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 64, 65, 200, 333]
    check(ctx, ref.Population8(dim + hq, lens, [1] * len(lens), hq, hk, dim, codes, dtype=dtype))


@pytest.mark.parametrize("codes", KINDS)
@pytest.mark.parametrize("rows", [1, 5, 16, 24, 64, 1000])
def test_page_sizes(ctx, codes, rows):
    check(ctx, ref.Population8(rows, [1, 77, 300], [1, 1, 1], 4, 2, 64, codes, page_rows=rows))
    check(ctx, ref.Population8(rows, [50, 77, 300], [50, 44, 60], 4, 2, 64, codes, page_rows=rows))


@pytest.mark.parametrize("sinks,ring,window", [
    (0, 0, 1), (0, 0, 50), (4, 0, 50), (100, 0, 50), (0, 64, 0), (5, 64, 0), (16, 96, 40), (3, 50, 200),
    (300, 0, 7), (17, 33, 33)])
@pytest.mark.parametrize("new", [1, 3, 40])
def test_windows_sinks_rings(ctx, sinks, ring, window, new):
    lens = [1, 4, 30, 64, 65, 70, 131, 290]
    p = ref.Population8(sinks + ring + window, [max(n, new) for n in lens], [new] * len(lens), 4, 2, 64,
                        KINDS[new % 2], sinks=sinks, ring=ring)
    check(ctx, p, window)


@pytest.mark.parametrize("codes", KINDS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hq,hk,dim", [(2, 2, 64), (4, 1, 128), (4, 2, 80), (1, 1, 16), (8, 1, 112)])
def test_blocks_of_tokens(ctx, codes, dtype, hq, hk, dim):
    check(ctx, ref.Population8(dim + hq, [40, 200, 300, 513, 70], [40, 130, 257, 33, 0], hq, hk, dim, codes, dtype=dtype))


@pytest.mark.parametrize("codes", KINDS)
def test_few_ragged_tokens(ctx, codes):
    check(ctx, ref.Population8(9, [5, 40, 100, 12, 3, 8], [5, 0, 7, 1, 3, 2], 8, 2, 128, codes, dtype=torch.float16), window=6)


@pytest.mark.parametrize("hint", [False, True])
@pytest.mark.parametrize("new,dim", [(1, 128), (1, 64), (40, 128), (40, 64)])
def test_long_sessions_are_split_and_joined(ctx, hint, new, dim):
    p = ref.Population8(3, [3000, max(3, new)], [new, new], 4, 2, dim, KINDS[dim == 64], page_rows=32)
    out, lse = check(ctx, p, hint=hint)
    again, lse2 = attend(ctx, p, hint=hint)
    assert torch.equal(out, again) and torch.equal(lse, lse2)  # the parts join in a fixed order


@pytest.mark.parametrize("new", [1, 60])
@pytest.mark.parametrize("codes", KINDS)
def test_large_scores(ctx, codes, new):
    # Running maxima that rise late, and scores whose exponential overflows.
    p = ref.Population8(4, [600, 600], [new, new], 4, 4, 64, codes, spread=4.0)
    ramp = torch.linspace(0.2, 4, 600).double()
    k = p.k.clone()
    for s in range(2):
        for j in range(600):
            page, row = int(p.table[s, j // 16]), j % 16
            k[page, row] *= ramp[j if s else 599 - j]
    p.set("k", k.bfloat16())
    check(ctx, p)
    check(ctx, p, scale=1.0)
    check(ctx, p, scale=1e-3)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("late", [False, True])
def test_values_of_very_different_sizes(ctx, dtype, late):
    # One token with nearly all of the weight and tiny values, many with tiny weights and
    # large values, in either order: neither may push the other out of the sums.
    p = ref.Population8(5, [300], [1], 1, 1, 64, ref.E4M3, dtype=dtype, sizes=0.0)
    q = p.q[0, 0].double()
    k, v = p.k.clone(), p.v.clone()
    size = 2.0 ** -10 if dtype == torch.float16 else 2.0 ** -40
    for j in range(300):
        page, row = int(p.table[0, j // 16]), j % 16
        k[page, row, 0] *= 0.05
        if j == (280 if late else 3):
            k[page, row, 0] = q * 40.0 * 8.0 / (q @ q)  # a score some 40 above the others'
            v[page, row] *= size
    p.set("k", k.to(dtype))
    p.set("v", v.to(dtype))
    out, lse = attend(ctx, p)
    want, ref_lse, _, _ = p.reference()
    w = torch.exp(torch.tensor(0.0))
    # Against the values' own sizes: the large one's, and what the others' weights leave.
    u = kv_ref.ROUND[dtype]
    scores = [(p.q[0, 0].double() @ p.k[kp, r, 0]) / 8.0 for _, kp, _, r in p.seen(0, 299, 0)]
    values = [p.v[vp, r, 0] for _, _, vp, r in p.seen(0, 299, 0)]
    w = torch.softmax(torch.stack(scores), 0)
    mass = sum(x * y.abs() for x, y in zip(w, values))
    assert ((out[0, 0].cpu().double() - want[0, 0]).abs() <= 4 * u * mass + 2.0 ** -24 * (dtype == torch.float16)).all()
    assert mass.max() < 1e-2  # (no larger than the token's own values are)


def test_empty_pages(ctx):
    for dead in ([0], [1, 2], [0, 1, 2, 3, 4, 5, 6]):
        for new in ([1, 2], [40, 60]):
            p = ref.Population8(5, [100, 100], new, 4, 2, 64)
            p.table[0, dead] = -1
            check(ctx, p, window=70)


@pytest.mark.parametrize("codes", KINDS)
@pytest.mark.parametrize("new", [1, 2, 50])
def test_what_is_not_seen_does_not_matter(ctx, dev, codes, new):
    # Codes that stand for NaN and scales that do, in rows that no new token sees, and in
    # rows that only some of them do.
    p = ref.Population8(6, [100, 57], [new, new], 4, 2, 64, codes, sinks=5)
    out, lse = check(ctx, p, window=40)
    seen = {(k, r) for s in range(2) for i in range(new) for _, k, _, r in p.seen(s, p.lens[s] - new + i, 40)}
    for junk in ("codes", "scales"):
        for page in range(p.n_pages):
            for r in range(16):
                if (page, r) not in seen:
                    for rows in (p.k_rows, p.v_rows):
                        rows[page, r, :128] = 0x7F if junk == "codes" else 0x55
                        rows[page, r, 128:130] = 255 if junk == "scales" else 120
        again, lse2 = attend(ctx, p, window=40)
        assert torch.equal(out, again) and torch.equal(lse, lse2)
    if new == 1:
        return
    # The last token's own row: those before it do not see it.
    for junk in ("codes", "scales"):
        for s in range(2):
            j = p.lens[s] - 1
            page, r = int(p.table[s, j // 16]), j % 16
            p.v_rows[page, r, :128] = 0x7F if junk == "codes" else 0x11
            p.v_rows[page, r, 128:130] = 255 if junk == "scales" else 120
            p.k_rows[page, r, 128:130] = 255 if junk == "scales" else 120
        again, lse2 = attend(ctx, p, window=40)
        for s in range(2):
            at = slice(p.q_off[s], p.q_off[s + 1] - 1)
            assert torch.equal(out[at], again[at]) and torch.equal(lse[at], lse2[at])
            bad = again[p.q_off[s + 1] - 1]
            assert torch.isnan(bad).all() if junk == "scales" or codes == ref.E4M3 else torch.isfinite(bad).all()


def test_nan_that_is_seen(ctx, dev):
    for new in (1, 60):
        p = ref.Population8(7, [70, 70, 70], [new] * 3, 2, 2, 64)
        p.v_rows[int(p.table[0, 0]), 3, 5] = 0x7F                 # one dim of one head
        p.k_rows[int(p.table[1, 0]), 3, 128 + 1] = 255            # a key's head
        cache, batch, q = ref.on_gpu(pcs, p)
        out = ctx.attend(cache, batch, q).cpu()
        a, b, c = (out[p.q_off[s]:p.q_off[s + 1]][-1] for s in range(3))
        assert torch.isnan(a[0, 5]) and torch.isfinite(a[1]).all()
        assert torch.isfinite(a[0, :5]).all() and torch.isfinite(a[0, 6:]).all()
        assert torch.isnan(b[1]).all() and torch.isfinite(b[0]).all()
        assert torch.isfinite(c).all()


def test_queries_beyond_float16(ctx, dev):
    # bfloat16 queries of any size: rows are scaled to float16's range and back.
    for new in (1, 3):
        p = ref.Population8(8, [90, 31], [new, new], 8, 4, 64, sizes=0.0)
        q = p.q.double()
        q[:, 0] *= 2.0 ** 60
        q[:, 1] *= 2.0 ** -70
        q[:, 2] = 0
        p.q = q.bfloat16()
        k = p.k.clone()
        k[:, :, 0] *= 2.0 ** -60
        p.set("k", k.bfloat16())
        check(ctx, p)


def test_layouts(ctx, dev):
    for new in (1, 40):
        p = ref.Population8(8, [90, 61], [new, new], 8, 4, 64, v_table=True)
        out, lse = check(ctx, p)
        # Rows apart, tables and queries out of wider tensors.
        wide = torch.full((p.n_pages, 16, p.row_bytes + 48), 0xEE, dtype=torch.uint8, device=dev)
        vw = wide.clone()
        wide[:, :, 16:16 + p.row_bytes], vw[:, :, 16:16 + p.row_bytes] = p.k_rows.to(dev), p.v_rows.to(dev)
        tables = torch.full((2, 2, p.pages + 3), -9, dtype=torch.int32, device=dev)
        tables[0, :, :p.pages], tables[1, :, :p.pages] = p.table.to(dev), p.v_table.to(dev)
        cut = slice(16, 16 + p.row_bytes)
        cache = pcs.KvCache(wide[:, :, cut], vw[:, :, cut], tables[0, :, :p.pages], v_table=tables[1, :, :p.pages],
                            codes=ref.E4M3, heads=4, head_dim=64)
        batch = pcs.KvBatch(torch.tensor(p.lens, dtype=torch.int32, device=dev), 2 * new)
        qkv = torch.randn(2 * new, 16, 64, device=dev).to(p.dtype)
        qkv[:, 3:11] = p.q.to(dev)
        got = torch.zeros(8, 2 * new, 64, dtype=p.dtype, device=dev).transpose(0, 1)
        ctx.attend(cache, batch, qkv[:, 3:11], out=got)
        assert torch.equal(got, out)


def test_offsets_past_32_bits(ctx, dev):
    # 5 GB a pool; the session's pages are its last ones.
    for new in (1, 50):
        p = ref.Population8(30, [200], [new], 4, 4, 128, page_rows=64, spare=0)
        pages = 5 * 2 ** 30 // (64 * p.row_bytes)
        dk = torch.empty(pages, 64, p.row_bytes, dtype=torch.uint8, device=dev)
        dv = torch.empty_like(dk)
        table = torch.arange(pages - p.n_pages, pages, dtype=torch.int32)
        dk[-p.n_pages:], dv[-p.n_pages:] = p.k_rows.to(dev), p.v_rows.to(dev)
        cache = pcs.KvCache(dk, dv, table[p.table.long()].to(dev), codes=ref.E4M3, heads=4, head_dim=128)
        batch = pcs.KvBatch(torch.tensor(p.lens, dtype=torch.int32, device=dev), new)
        out, lse = ctx.attend(cache, batch, p.q.to(dev), return_lse=True)
        kv_ref.check_attend(p, out, lse)
        k, v = ctx.kv_read(cache, batch, dtype=torch.float32)
        assert torch.equal(k.cpu(), read_expected(p, p.k, "k", torch.float32))
        assert torch.equal(v.cpu(), read_expected(p, p.v, "v", torch.float32))
        nk = torch.randn(new, 4, 128, dtype=p.dtype)
        ctx.kv_append(cache, batch, nk.to(dev), nk.to(dev))
        page = int(table[int(p.table[0, 3])])
        want = ref.rows_of(nk[-1:], ref.E4M3, p.row_bytes)[0, :4 * 129]
        assert torch.equal(dk[page, 199 - 192, :4 * 129].cpu(), want) and torch.equal(dv[page, 199 - 192, :4 * 129].cpu(), want)


def test_bad_ids_are_reported_and_unseen(ctx, dev):
    for bad in (10 ** 6, -3):
        for new in (1, 50):
            p = ref.Population8(31, [60, 60], [new, new], 2, 2, 64)
            p.table[1, 2] = bad
            cache, batch, q = ref.on_gpu(pcs, p)
            for call in (lambda: ctx.attend(cache, batch, q, return_lse=True), lambda: ctx.kv_read(cache, batch),
                         lambda: ctx.kv_append(cache, batch, q, q)):
                got = call()
                if new == 1 and not (isinstance(got, tuple) and got[1].dtype == torch.float32):
                    ctx.sync()  # the last token alone is in the page behind it
                    continue
                with pytest.raises(pcs.PcsError) as e:
                    ctx.sync()
                assert e.value.status == pcs.PCS_E_RANGE
                if isinstance(got, tuple) and got[1].dtype == torch.float32:
                    kv_ref.check_attend(p, *got)


def test_streams_side_by_side(ctx, dev):
    ps = [ref.Population8(20 + i, [1500], [1 if i % 2 else 40], 4, 2, 64, KINDS[i // 2]) for i in range(4)]
    want = [attend(ctx, p)[0] for p in ps]
    made = [ref.on_gpu(pcs, p) for p in ps]
    streams = [torch.cuda.Stream() for _ in ps]
    torch.cuda.synchronize()
    got = [[] for _ in ps]
    for _ in range(5):
        for i, (cache, batch, q) in enumerate(made):
            with torch.cuda.stream(streams[i]):
                got[i].append(ctx.attend(cache, batch, q))
    torch.cuda.synchronize()
    assert all(torch.equal(x, w) for g, w in zip(got, want) for x in g)
