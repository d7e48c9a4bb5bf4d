"""Operators over a paged cache of 8-bit keys and values, and over trees of
drafted tokens, that are measured, with their plain forms.

A case is a dict of plain values.  `op` names the operator:

  store    new tokens rotated and written to a cache in 8 bits, and read back:
           queries, and the values that the written keys and values stand for
  read     tokens of many sessions read out of an 8-bit cache
  attend   attention of new tokens over an 8-bit cache
  tree     attention of a tree of drafted tokens of each session: a node sees
           the context, its ancestors and itself
  keep     the accepted nodes of the trees moved next to their contexts

`cache` is what the pages hold: bf16, f16 (an element each), e4m3 or i8 (a head
is its codes, and one byte behind the row's codes gives its scale, a power of
two).  Where `own` is false, `run` computes the operators from elementary torch
operations in 32 bits; where it is true, through the public binding.  Lengths
inside a population come from the case alone, so every seed of a case has the
same shapes; contents, page tables, trees and positions' order in the pool come
from the seed.
"""
import math

import torch

own = False

_DEV = "cuda:0"
_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
_CODES = {"e4m3": torch.float8_e4m3fn, "i8": torch.int8}
_FRAME = (22, 40)  # tokens of one frame: height, width
_ctx = None


def _context():
    """The one context a program keeps for its lifetime."""
    global _ctx
    if _ctx is None:
        from paper_2607_21686_gb300 import pcs
        _ctx = pcs.Context(0)
    return _ctx


# ---------------------------------------------------------------------------
# The cases
# ---------------------------------------------------------------------------

def _case(name, op, cache, sessions, length, new, q_heads, kv_heads, head_dim, page_rows=16,
          sinks=0, ring=0, window=0, dtype="bf16"):
    return dict(name=name, op=op, cache=cache, sessions=sessions, len_lo=length[0],
                len_hi=length[1], new_lo=new[0], new_hi=new[1], q_heads=q_heads,
                kv_heads=kv_heads, head_dim=head_dim, page_rows=page_rows, sinks=sinks, ring=ring,
                window=window, dtype=dtype)


def listed():
    return [
        # One new token of each of 64 sessions in their 1,024-token ring windows.
        _case("store_token", "store", "e4m3", 64, (1025, 9000), (1, 1), 16, 16, 64, ring=1024),
        # A few frames of each of 24 sessions behind their 16 first tokens.
        _case("store_frames", "store", "i8", 24, (900, 6000), (131, 1760), 16, 16, 64, sinks=16,
              ring=2048, dtype="f16"),
        # One frame of one session, for a model part that wants 16 bits.
        _case("read_frame", "read", "e4m3", 1, (5000, 5000), (880, 880), 16, 16, 64, sinks=16,
              ring=2944),
        # Whole ragged contexts of many sessions, grouped heads, pages of 32 tokens.
        _case("read_contexts", "read", "i8", 48, (1, 12000), (1, 12000), 32, 8, 128, page_rows=32,
              dtype="f16"),
        # The next token of every session a server holds.
        _case("token_256", "attend", "e4m3", 256, (1024, 5000), (1, 1), 16, 16, 64, ring=1024),
        # Ragged contexts, grouped heads, pages of 32 tokens.
        _case("token_ragged", "attend", "i8", 48, (1, 12000), (1, 1), 32, 8, 128, page_rows=32,
              dtype="f16"),
        # One frame of one session over its window and first tokens.
        _case("block_frame", "attend", "e4m3", 1, (5000, 5000), (880, 880), 16, 16, 64, sinks=16,
              ring=2944, window=2048),
        # A prompt from its first token, grouped heads.
        _case("block_prompt", "attend", "i8", 1, (8000, 8000), (8000, 8000), 32, 8, 128),
        # A small tree of one session over its window: latency.
        _case("tree_one", "tree", "bf16", 1, (1500, 1500), (26, 26), 16, 16, 64, ring=1088,
              window=1024),
        # Trees of many sessions, ragged contexts, grouped heads.
        _case("tree_sessions", "tree", "e4m3", 32, (500, 9000), (60, 60), 32, 8, 128,
              page_rows=32),
        # The accepted path of one session's tree.
        _case("keep_one", "keep", "bf16", 1, (1500, 1500), (26, 26), 16, 16, 64, ring=1088),
        # Those of all sessions a server holds.
        _case("keep_sessions", "keep", "e4m3", 256, (600, 3000), (60, 64), 32, 8, 128,
              page_rows=32, dtype="f16"),
    ]


def draw(rng):
    """One more case of the ranges that the listed ones stand for."""
    top = max(_cost(c) for c in listed())
    while True:
        c = _draw(rng)
        scores = c["sessions"] * c["q_heads"] * c["new_hi"] * c["len_hi"]
        places = c["sessions"] * c["len_hi"] * c["kv_heads"] * c["head_dim"]
        if _cost(c) <= top and places <= 1_000_000_000 \
                and (c["op"] not in ("attend", "tree") or scores <= 2_000_000_000):
            return c


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw(rng):
    op = rng.choice(["store", "read", "token", "token", "block", "tree", "tree", "keep"])
    head_dim = rng.choice([64, 128, 128, 64, 96, 80])
    kv_heads = rng.choice([1, 2, 4, 8, 16]) if head_dim > 64 else rng.choice([4, 8, 16])
    q_heads = kv_heads * rng.choice([1, 1, 2, 4, 5, 8])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    cache = rng.choice(["e4m3", "i8"])
    if op in ("tree", "keep"):
        cache = rng.choice([cache, dtype])
    page_rows = rng.choice([8, 16, 16, 24, 32, 64])
    sinks = rng.choice([0, 0, rng.randint(1, 128)])
    if op == "token":
        sessions, new = _log(rng, 1, 300), rng.choice([1, 1, 1, 2, 4])
    elif op == "block":
        sessions, new = _log(rng, 1, 32), _log(rng, 33, 9000)
    elif op in ("tree", "keep"):
        sessions, new = _log(rng, 1, 256), rng.randint(2, 64)
    else:
        sessions, new = _log(rng, 1, 200), _log(rng, 1, 2500)
    hi = max(new, _log(rng, 100, 150000 if op in ("token", "tree") else 9000))
    lo = hi if sessions == 1 else rng.randint(1, hi)
    window = rng.choice([0, 0, rng.randint(100, 4000)])
    ring = rng.choice([0, new + max(window, rng.randint(200, 2500))])
    new_lo = new if op == "token" or sessions == 1 else rng.randint(1, new)
    c = _case("", "attend" if op in ("token", "block") else op, cache, sessions, (lo, hi),
              (new_lo, new), q_heads, kv_heads, head_dim, page_rows, sinks, ring, window, dtype)
    del c["name"]
    return c


def _spread(lo, hi, i, n):
    """The i-th of n whole numbers spread over [lo, hi]; a single one is hi."""
    return hi if n == 1 else lo + int((hi - lo + 1) * ((i + 1) * 0.6180339887498949 % 1.0))


def _lengths(c):
    """New tokens of each session and its length with them."""
    n = c["sessions"]
    new = [_spread(c["new_lo"], c["new_hi"], i, n) for i in range(n)]
    lens = [max(new[i], _spread(c["len_lo"], c["len_hi"], 7 * i + 3, n)) for i in range(n)]
    # Whole contexts are read up to their last token.
    return (lens, lens) if c["op"] == "read" and n > 1 else (new, lens)


def _kept(c, new):
    """Nodes of each session's tree that are accepted: few of them."""
    return [1 + int(7 * (0.3 + i * 0.6180339887498949) % 7) % m for i, m in enumerate(new)]


def _capacity(c, lens):
    """Slots of one session's page table."""
    rows = c["sinks"] + c["ring"] if c["ring"] else max(lens)
    return -(-rows // c["page_rows"])


def _row_bytes(c):
    """A row of an 8-bit cache: codes of all heads, then a scale byte a head,
    filled up to a multiple of 32."""
    return -(-c["kv_heads"] * (c["head_dim"] + 1) // 32) * 32


def _head_bytes(c):
    """Bytes of one head of a row that mean something."""
    return c["head_dim"] + 1 if c["cache"] in _CODES else 2 * c["head_dim"]


def _there(c, m, n):
    """How many of a session's last m tokens are in the cache, of n."""
    early = max(0, min(c["sinks"], n - c["ring"]) - (n - m)) if c["ring"] else 0
    return min(m, c["ring"]) + early if c["ring"] else m


def _visible(c, p, n):
    """Tokens that the token at position p sees of n in the cache."""
    low = max(n - c["ring"] if c["ring"] else 0, p - c["window"] + 1 if c["window"] else 0)
    return min(c["sinks"], p + 1) + max(0, p + 1 - max(low, c["sinks"])) if low > 0 else p + 1


def work(case):
    c = case
    d, hq, hk, op = c["head_dim"], c["q_heads"], c["kv_heads"], c["op"]
    new, lens = _lengths(c)
    tokens, head = sum(new), _head_bytes(c)
    if op == "store":
        n = tokens * (hq + hk) * d
        cached = 2 * sum(_there(c, m, length) for m, length in zip(new, lens)) * hk * head
        return {"bytes": 4 * n + 2 * tokens * hk * d + 12 * tokens + 2 * cached
                + 4 * tokens * hk * d, "flops": 3 * n + 4 * tokens * hk * d}
    if op == "read":
        rows = sum(_there(c, m, length) for m, length in zip(new, lens))
        return {"bytes": 2 * hk * (rows * head + tokens * 2 * d), "flops": 2 * rows * hk * d}
    if op == "keep":
        rows = sum(_kept(c, new))
        return {"bytes": 4 * rows * hk * head + 4 * rows + 12 * len(new), "flops": rows}
    rows = pairs = 0
    for m, length in zip(new, lens):
        # Rows of the cache that some new token sees, and (token, row) pairs.
        first = length - m
        low = max(length - c["ring"] if c["ring"] else 0,
                  first - c["window"] + 1 if c["window"] else 0)
        rows += min(length, c["sinks"] + length - max(low, c["sinks"])) if low > 0 else length
        if op == "tree":  # (a handful of ancestors each)
            pairs += m * (_visible(c, first, length) + 4)
        else:
            pairs += sum(_visible(c, p, length) for p in range(first, length))
    return {"bytes": 2 * rows * hk * head + 4 * tokens * hq * d + 4 * tokens * hq
            + (4 * tokens if op == "tree" else 0), "flops": 4 * hq * d * pairs}


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 6.7e12, w["flops"] / 1.9e15)


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _positions(token):
    """(time, height, width) of tokens by their number in the session."""
    h, w = _FRAME
    return torch.stack([token // (h * w), token // w % h, token % w], -1).to(torch.int32)


def _frequencies(pairs):
    """Angle per unit position: each axis from 1 downwards to 1 / 10,000."""
    return torch.cat([torch.exp(torch.arange(n, device=_DEV, dtype=torch.float32)
                                * (-math.log(10000.0) / n)) for n in pairs])


def _pool(c, pages, g):
    """Pages full of keys or values: heads of different sizes."""
    rows, hk, d = c["page_rows"], c["kv_heads"], c["head_dim"]

    def values(n):
        x = torch.randn(n, rows, hk, d, generator=g, device=_DEV)
        size = torch.exp(0.5 * torch.randn(n, rows, hk, 1, generator=g, device=_DEV))
        return (x * size).to(_TYPES[c["dtype"]])

    if c["cache"] not in _CODES:
        return values(pages)
    pool = torch.zeros(pages, rows, _row_bytes(c), dtype=torch.uint8, device=_DEV)
    step = max(1, (1 << 27) // (rows * hk * d))
    for i in range(0, pages, step):
        _write_rows(c, pool[i:i + step], values(min(step, pages - i)))
    return pool


def prepare(case, seed):
    c = case
    g = torch.Generator(device=_DEV)
    g.manual_seed(0x8B17 + seed)
    dt = _TYPES[c["dtype"]]
    d = c["head_dim"]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=_DEV, dtype=dt)

    s = {"case": c, "ctx": _context() if own else None}
    new, lens = _lengths(c)
    n, pages = c["sessions"], _capacity(c, lens)
    total = n * pages
    pool = total + total // 8 + 1
    s["k_pool"], s["v_pool"] = _pool(c, pool, g), _pool(c, pool, g)
    # Sessions' pages lie anywhere in the pool, in any order.
    ids = torch.randperm(pool, generator=g, device=_DEV)[:total].to(torch.int32)
    s["table"] = ids.reshape(n, pages)
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device=_DEV)
    off = [0]
    for m in new:
        off.append(off[-1] + m)
    s["q_off"] = torch.tensor(off, dtype=torch.int32, device=_DEV)
    s["tokens"], s["max_new"], s["max_len"] = off[-1], max(new), max(lens)
    s["even"] = min(new) == max(new)
    if c["op"] in ("store", "attend", "tree"):
        s["q"] = normal(off[-1], c["q_heads"], d)
    if c["op"] == "store":
        s["k"] = normal(off[-1], c["kv_heads"], d)
        s["v"] = normal(off[-1], c["kv_heads"], d)
        number = torch.cat([torch.arange(a - m, a, device=_DEV) for m, a in zip(new, lens)])
        s["pos"] = _positions(number)
        third = d // 8
        s["pairs"] = (d // 2 - 2 * (d // 6), d // 6, d // 6) if d % 3 else (third, third, third)
        s["freq"] = _frequencies(s["pairs"])
    if c["op"] == "tree":
        # A drafted token's parent is one of those before it, most often a late one.
        at = torch.cat([torch.arange(m, device=_DEV) for m in new])
        back = torch.rand(off[-1], generator=g, device=_DEV).square() * (at + 1)
        s["parent"] = (at - 1 - back.long().minimum(at)).to(torch.int32)
    if c["op"] == "keep":
        kept = _kept(c, new)
        order = torch.rand(n, max(new), generator=g, device=_DEV)
        order[torch.arange(max(new), device=_DEV)[None] >= torch.tensor(new, device=_DEV)[:, None]] = 2.0
        low = order.argsort(1)[:, :max(kept)]
        late = torch.arange(max(kept), device=_DEV)[None] >= torch.tensor(kept, device=_DEV)[:, None]
        low = low.masked_fill(late, max(new) + 1).sort(1).values
        s["index"] = low.masked_fill(late, -1).to(torch.int32)
        s["count"] = torch.tensor(kept, dtype=torch.int32, device=_DEV)
    if own:
        from paper_2607_21686_gb300 import pcs
        if c["cache"] in _CODES:
            s["cache"] = pcs.KvCache(s["k_pool"], s["v_pool"], s["table"], sinks=c["sinks"],
                                     ring=c["ring"], codes=_CODES[c["cache"]],
                                     heads=c["kv_heads"], head_dim=d)
        else:
            s["cache"] = pcs.KvCache(s["k_pool"], s["v_pool"], s["table"], sinks=c["sinks"],
                                     ring=c["ring"])
        s["batch"] = pcs.KvBatch(s["lens"], s["tokens"], None if s["even"] else s["q_off"],
                                 s["max_new"], s["max_len"])
        if c["op"] == "store":
            s["rotary"] = pcs.Rotary(s["pos"], s["freq"], s["pairs"])
    return s


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(state):
    s = state
    c = s["case"]
    op, dt = c["op"], _TYPES[c["dtype"]]
    if op == "store":
        if own:
            q = s["ctx"].kv_append(s["cache"], s["batch"], s["k"], s["v"], s["q"], s["rotary"])
            k, v = s["ctx"].kv_read(s["cache"], s["batch"], dtype=dt)
        else:
            q = _append(s)
            k, v = _read(s)
        return {"q": q, "k": k, "v": v}
    if op == "read":
        if own:
            k, v = s["ctx"].kv_read(s["cache"], s["batch"], dtype=dt)
        else:
            k, v = _read(s)
        return {"k": k, "v": v}
    if op == "keep":  # (pages come as their bytes: moved, not computed)
        if own:
            lens = s["ctx"].kv_keep(s["cache"], s["batch"], s["index"], s["count"])
        else:
            lens = _keep(s)
        return {"lens": lens, "k_pool": s["k_pool"], "v_pool": s["v_pool"]}
    if own and op == "tree":
        out, lse = s["ctx"].attend_tree(s["cache"], s["batch"], s["parent"], s["q"],
                                        window=c["window"], return_lse=True)
    elif own:
        out, lse = s["ctx"].attend(s["cache"], s["batch"], s["q"], window=c["window"],
                                   return_lse=True)
    else:
        out, lse = _attend(s)
    return {"out": out, "lse": lse}


def _angles(pos, freq, pairs):
    """cos and sin of position times frequency [tokens, pairs], in 64 bits: a
    key's last digit decides codes next to a border."""
    axis = torch.cat([torch.full((n,), a, device=pos.device) for a, n in enumerate(pairs)])
    a = pos.double()[:, axis] * freq.double()[None]
    return torch.cos(a).float(), torch.sin(a).float()


def _turned(x, cos, sin):
    n = cos.shape[1]
    y = x.float()
    cos, sin = cos[:, None], sin[:, None]
    a, b = y[..., :n], y[..., n:2 * n]
    return torch.cat([a * cos - b * sin, a * sin + b * cos, y[..., 2 * n:]], -1).to(x.dtype)


def _power(e):
    """2^e of whole numbers from -126 to 127, from its bits: exact."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _codes(x, kind):
    """Codes and scale bytes of heads x [..., head_dim]: the least power of two
    from 2^-126 on by which the largest element fits the codes' range."""
    y = x.float()
    top = y.abs().amax(-1)
    fine = torch.isfinite(top)
    m, e = torch.frexp(top.masked_fill(~fine, 1.0))
    if kind == "e4m3":  # up to 448 = 0.875 * 2^9
        e = e - 9 + (m > 0.875).int()
    else:               # up to 127 = 127 / 128 * 2^7
        e = e - 7 + (m > 127 / 128).int()
    e = torch.where(m == 0, -126, e).clamp_min(-126)
    y = torch.where(fine[..., None], y * _power(-e)[..., None], 0.0)
    if kind == "e4m3":
        codes = y.to(torch.float8_e4m3fn).view(torch.uint8)
    else:
        codes = torch.round(y).to(torch.int8).view(torch.uint8)
    return codes, torch.where(fine, e + 127, 255).to(torch.uint8)


def _write_rows(c, rows, x):
    """x [.., kv_heads, head_dim] into rows [.., row bytes]."""
    codes, scale = _codes(x, c["cache"])
    n = c["kv_heads"] * c["head_dim"]
    rows[..., :n] = codes.flatten(-2)
    rows[..., n:n + c["kv_heads"]] = scale


def _values(c, rows):
    """What rows of the cache stand for, in 32 bits [.., kv_heads, head_dim]."""
    if c["cache"] not in _CODES:
        return rows.float()
    n = c["kv_heads"] * c["head_dim"]
    codes = rows[..., :n].contiguous().view(_CODES[c["cache"]]).float()
    b = rows[..., n:n + c["kv_heads"]].int()
    scale = torch.where(b == 255, math.nan, _power((b - 127).clamp_max(127)))
    return codes.unflatten(-1, (c["kv_heads"], c["head_dim"])) * scale[..., None]


def _slots(c, j):
    """The slot of the token at position j."""
    if not c["ring"]:
        return j
    return torch.where(j < c["sinks"], j, c["sinks"] + (j - c["sinks"]) % c["ring"])


def _sessions_of(s):
    """Session and position of every new token."""
    t = torch.arange(s["tokens"], device=_DEV, dtype=torch.int32)
    session = torch.searchsorted(s["q_off"][1:], t, right=True)
    return session, (s["lens"][session] - s["q_off"][session + 1] + t).long()


def _rows_of(s, session, p):
    """Rows of the pools (flat) of positions p of sessions, and whether they are
    in the cache."""
    c = s["case"]
    slot = _slots(c, p)
    row = s["table"][session, slot // c["page_rows"]].long() * c["page_rows"] + slot % c["page_rows"]
    there = torch.ones_like(p, dtype=torch.bool)
    if c["ring"]:  # of tokens that share a slot the last one stays
        there = (p < c["sinks"]) | (p >= s["lens"][session] - c["ring"])
    return row, there


def _append(s):
    c = s["case"]
    cos, sin = _angles(s["pos"], s["freq"], s["pairs"])
    session, p = _sessions_of(s)
    row, there = _rows_of(s, session, p)
    row = row[there]
    for pool, x in ((s["k_pool"], _turned(s["k"], cos, sin)), (s["v_pool"], s["v"])):
        codes, scale = _codes(x[there], c["cache"])
        n = c["kv_heads"] * c["head_dim"]
        pool.flatten(0, 1)[row, :n] = codes.flatten(-2)
        pool.flatten(0, 1)[row, n:n + c["kv_heads"]] = scale
    return _turned(s["q"], cos, sin)


def _read(s):
    c = s["case"]
    row, there = _rows_of(s, *_sessions_of(s))
    return [torch.where(there[:, None, None], _values(c, pool.flatten(0, 1)[row]), 0.0)
            .to(_TYPES[c["dtype"]]) for pool in (s["k_pool"], s["v_pool"])]


def _keep(s):
    new = s["q_off"][1:] - s["q_off"][:-1]
    first = s["lens"] - new
    i = torch.arange(s["index"].shape[1], device=_DEV)
    session, i = torch.nonzero(i[None] < s["count"][:, None], as_tuple=True)
    p = first[session].long()
    src, _ = _rows_of(s, session, p + s["index"][session, i].long())
    dst, _ = _rows_of(s, session, p + i)
    for pool in (s["k_pool"], s["v_pool"]):
        flat = pool.flatten(0, 1)
        flat[dst] = flat[src]
    return first + s["count"]


def _attend(s):
    c = s["case"]
    n, d, hk = c["sessions"], c["head_dim"], c["kv_heads"]
    group = c["q_heads"] // hk
    j = torch.arange(s["max_len"], device=_DEV)
    lens = s["lens"].long()
    slot = _slots(c, j)
    page = s["table"][:, slot // c["page_rows"]].long()
    there = j[None] < lens[:, None]
    if c["ring"]:
        there = there & ((j < c["sinks"])[None] | (j[None] >= lens[:, None] - c["ring"]))
    row = slot % c["page_rows"]
    hide = ~there[..., None, None]
    k = _values(c, s["k_pool"][page, row]).masked_fill(hide, 0.0)
    v = _values(c, s["v_pool"][page, row]).masked_fill(hide, 0.0)
    session, p = _sessions_of(s)
    m = s["max_new"]
    place = torch.arange(s["tokens"], device=_DEV) - s["q_off"][session]
    q = torch.zeros(n, m, hk, group, d, device=_DEV)
    q[session, place] = s["q"].float().reshape(-1, hk, group, d)
    if c["op"] == "tree":
        sees = _tree(s, session, place, j)
    else:
        pos = torch.full((n, m), -1, device=_DEV)
        pos[session, place] = p
        sees = j[None, None] <= pos[..., None]
        if c["window"]:
            near = j[None, None] > pos[..., None] - c["window"]
            sees = sees & ((j < c["sinks"])[None, None] | near)
    sees = (sees & there[:, None])[:, None, None]
    x = torch.matmul(q.permute(0, 2, 3, 1, 4).reshape(n, hk, group * m, d), k.permute(0, 2, 3, 1))
    x = (x * (1.0 / math.sqrt(d))).reshape(n, hk, group, m, -1).masked_fill(~sees, -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    x = torch.exp(x - top)
    total = x.sum(-1, keepdim=True)
    out = torch.matmul(x.reshape(n, hk, group * m, -1), v.permute(0, 2, 1, 3))
    out = out.reshape(n, hk, group, m, d) / torch.where(total == 0.0, 1.0, total)
    lse = (top + torch.log(total))[..., 0]
    out = out.permute(0, 3, 1, 2, 4)[session, place].reshape(-1, c["q_heads"], d)
    return out.to(s["q"].dtype), lse.permute(0, 3, 1, 2)[session, place].reshape(-1, c["q_heads"])


def _tree(s, session, place, j):
    """What the nodes see of positions j: [sessions, nodes, positions]."""
    c = s["case"]
    n, m = c["sessions"], s["max_new"]
    # Paths of up to 64 steps: powers of "is itself or its parent".
    step = torch.zeros(n, m, m + 1, device=_DEV)
    up = s["parent"].long()
    step[session, place, torch.where(up < 0, m, up)] = 1.0
    step = step[..., :m] + torch.eye(m, device=_DEV)
    line = torch.linalg.matrix_power(step, 64) > 0.5          # [n, node, ancestor or itself]
    depth = line.sum(-1) - 1
    first = s["lens"].long() - (s["q_off"][1:] - s["q_off"][:-1])
    pos = first[:, None] + depth                              # [n, m]
    at = j[None] - first[:, None]                             # a node's number, at its slot's position
    node = at.clamp(0, m - 1)
    own_pos = torch.where(at < 0, j[None], torch.gather(pos, 1, node))
    sees = (at < 0)[:, None] | torch.gather(line, 2, node[:, None].expand(-1, m, -1))
    if c["window"]:
        near = own_pos[:, None] > pos[..., None] - c["window"]
        sees = sees & ((own_pos < c["sinks"])[:, None] | near)
    return sees


# ---------------------------------------------------------------------------
# The definition in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    c = case
    if c["op"] == "keep":  # rows are moved, nothing is computed
        return None
    s = prepare(case, seed)
    new, lens = _lengths(c)
    if c["op"] == "store":
        return _store_64(s, c, new, lens)
    if c["op"] == "read":
        k, v = (_read_64(s, c, pool, new, lens) for pool in (s["k_pool"], s["v_pool"]))
        return {"k": k, "v": v}
    return _attend_64(s, c, new, lens)


def _turned_64(x, s):
    """Each pair as a complex number, multiplied by exp(i angle)."""
    out = x.double().clone()
    i, count = 0, sum(s["pairs"])
    for axis, n in enumerate(s["pairs"]):
        angle = s["pos"][:, axis].double()[:, None] * s["freq"][i:i + n].double()
        turn = torch.polar(torch.ones_like(angle), angle)[:, None]
        a, b = slice(i, i + n), slice(count + i, count + i + n)
        z = torch.complex(out[..., a], out[..., b]) * turn
        out[..., a], out[..., b] = z.real.clone(), z.imag.clone()
        i += n
    return out


def _power_64(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _stored_64(x, kind):
    """What heads x (in 64 bits) stand for once they are in 8 bits."""
    most = 448.0 if kind == "e4m3" else 127.0
    top = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(top / most)).clamp(-126, 127)
    # (A logarithm next to a whole number may be off.)
    e = torch.where(top > most * _power_64(e), e + 1, e)
    e = torch.where(top <= most * _power_64(e - 1), e - 1, e).clamp_min(-126)
    y = x * _power_64(-e)
    if kind == "i8":
        return torch.round(y) * _power_64(e)
    # Four digits from 2^-6 on, multiples of 2^-9 below.
    _, digit = torch.frexp(y.abs().clamp_min(2.0 ** -6))
    return torch.round(y * _power_64(4 - digit)) * _power_64(digit - 4) * _power_64(e)


def _store_64(s, c, new, lens):
    dt = s["q"].dtype
    k = _stored_64(_turned_64(s["k"], s).to(dt).double(), c["cache"])
    v = _stored_64(s["v"].double(), c["cache"])
    at = 0
    for m, length in zip(new, lens):
        if c["ring"]:  # overwritten by later new tokens
            p = torch.arange(length - m, length, device=_DEV)
            gone = (p >= c["sinks"]) & (p < length - c["ring"])
            k[at:at + m][gone] = 0.0
            v[at:at + m][gone] = 0.0
        at += m
    return {"q": _turned_64(s["q"], s), "k": k, "v": v}


def _value_64(c, pool, page, row, h):
    """One head of rows of the pool."""
    d = c["head_dim"]
    if c["cache"] not in _CODES:
        return pool[page, row, h].double()
    x = pool[page, row]
    codes = x[:, h * d:(h + 1) * d].int()
    if c["cache"] == "i8":
        y = ((codes + 128) % 256 - 128).double()
    else:
        e, m = (codes >> 3) & 15, (codes & 7).double()
        y = torch.where(e > 0, (8.0 + m) * _power_64(e - 10), m * 2.0 ** -9)
        y = torch.where(codes > 127, -y, y)
    return y * _power_64(x[:, c["kv_heads"] * d + h].long() - 127)[:, None]


def _slots_64(c, p):
    slot = p.clone()
    if c["ring"]:
        late = p >= c["sinks"]
        slot[late] = (p[late] - c["sinks"]).remainder(c["ring"]) + c["sinks"]
    return slot


def _read_64(s, c, pool, new, lens):
    out = torch.zeros(s["tokens"], c["kv_heads"], c["head_dim"], device=_DEV, dtype=torch.float64)
    at = 0
    for i, (m, length) in enumerate(zip(new, lens)):
        p = torch.arange(length - m, length, device=_DEV)
        if c["ring"]:
            p = p[(p < c["sinks"]) | (p >= length - c["ring"])]
        slot = _slots_64(c, p)
        page = s["table"][i].long()[torch.div(slot, c["page_rows"], rounding_mode="floor")]
        for h in range(c["kv_heads"]):
            out[at + p - (length - m), h] = _value_64(c, pool, page, slot.remainder(c["page_rows"]), h)
        at += m
    return out


def _lines_64(parent):
    """Every node's ancestors and itself, and its depth."""
    m = len(parent)
    line = torch.zeros(m, m, dtype=torch.bool)
    depth = torch.zeros(m, dtype=torch.long)
    for i, up in enumerate(parent):
        if up >= 0:
            line[i] = line[up]
            depth[i] = depth[up] + 1
        line[i, i] = True
    return line.to(_DEV), depth.to(_DEV)


def _attend_64(s, c, new, lens):
    d, hk = c["head_dim"], c["kv_heads"]
    group = c["q_heads"] // hk
    out = torch.zeros(s["tokens"], c["q_heads"], d, device=_DEV, dtype=torch.float64)
    lse = torch.full((s["tokens"], c["q_heads"]), -math.inf, device=_DEV, dtype=torch.float64)
    parents = s["parent"].tolist() if c["op"] == "tree" else None
    at = 0
    for i, (m, length) in enumerate(zip(new, lens)):
        first = length - m
        oldest = max(0, length - c["ring"]) if c["ring"] else 0
        if c["window"]:
            oldest = max(oldest, first - c["window"] + 1)
        kept = torch.arange(length, device=_DEV)
        kept = kept[(kept < c["sinks"]) | (kept >= oldest)]
        # Positions of the new tokens and of the kept ones.
        pos, own_pos = torch.arange(first, length, device=_DEV), kept.clone()
        if parents:
            line, depth = _lines_64(parents[at:at + m])
            pos = first + depth
            drafted = kept >= first
            own_pos[drafted] = pos[kept[drafted] - first]
        slot = _slots_64(c, kept)
        page = s["table"][i].long()[torch.div(slot, c["page_rows"], rounding_mode="floor")]
        row = slot.remainder(c["page_rows"])
        for h in range(hk):
            k = _value_64(c, s["k_pool"], page, row, h)
            v = _value_64(c, s["v_pool"], page, row, h)
            for t in range(0, m, 1024):
                e = min(m, t + 1024)
                p = pos[t:e, None]
                q = s["q"][at + t:at + e, h * group:(h + 1) * group].double().transpose(0, 1)
                x = q @ k.T / math.sqrt(d)
                if parents:
                    far = torch.zeros(e - t, len(kept), dtype=torch.bool, device=_DEV)
                    far[:, drafted] = ~line[t:e][:, kept[drafted] - first]
                else:
                    far = kept[None] > p
                if c["window"]:
                    far |= (p - own_pos[None] >= c["window"]) & (own_pos[None] >= c["sinks"])
                x[far.expand_as(x)] = -math.inf
                part = torch.logsumexp(x, -1)
                y = torch.exp(x - part[..., None].clamp_min(-1e300)) @ v
                out[at + t:at + e, h * group:(h + 1) * group] = y.transpose(0, 1)
                lse[at + t:at + e, h * group:(h + 1) * group] = part.transpose(0, 1)
        at += m
    return {"out": out, "lse": lse}
