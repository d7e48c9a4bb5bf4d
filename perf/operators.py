"""Operators over a paged cache of keys and values that are measured, with their
plain forms.

A case is a dict of plain values.  `op` names the operator:

  rotate   rotary positions with several axes (time, height, width) applied to
           query and key heads, or with `inverse` taken back (its gradient)
  append   the new tokens of many sessions: queries and keys rotated, keys and
           values written to the pages of each session's window
  attend   attention of the new tokens over the paged cache: one token or a few
           of each session, or whole blocks and prompts, with a sliding window
           and the first tokens (sinks) always visible

Where `own` is false, `run` computes the operators from elementary torch
operations in 32 bits; where it is true, through the public binding.  Lengths
inside a population come from the case alone, so every seed of a case has the
same shapes; contents, page tables and positions' order in the pool come from
the seed.
"""
import math

import torch

own = False

_DEV = "cuda:0"
_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f16": 2, "f32": 4}
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

def _rotate(name, tokens, q_heads, kv_heads, head_dim, pairs, dtype="bf16", interleaved=False,
            inverse=False):
    return dict(name=name, op="rotate", tokens=tokens, q_heads=q_heads, kv_heads=kv_heads,
                head_dim=head_dim, pairs_t=pairs[0], pairs_h=pairs[1], pairs_w=pairs[2],
                dtype=dtype, interleaved=interleaved, inverse=inverse)


def _cached(name, op, sessions, length, new, q_heads, kv_heads, head_dim, page_rows=16, sinks=0,
            ring=0, window=0, dtype="bf16"):
    return dict(name=name, op=op, sessions=sessions, len_lo=length[0], len_hi=length[1],
                new_lo=new[0], new_hi=new[1], q_heads=q_heads, kv_heads=kv_heads,
                head_dim=head_dim, page_rows=page_rows, sinks=sinks, ring=ring, window=window,
                dtype=dtype)


def listed():
    return [
        # One frame's queries and keys, 16 heads of 64: a step's first kernel.
        _rotate("rotate_frame", 880, 16, 16, 64, (8, 12, 12)),
        # The gradient of a long clip's rotation, grouped heads, pairs side by side.
        _rotate("rotate_gradient", 49153, 32, 8, 128, (16, 24, 24), "f16", True, True),
        # One new token of each of 64 sessions in their 1,024-token ring windows.
        _cached("append_token", "append", 64, (1025, 9000), (1, 1), 16, 16, 64, ring=1024),
        # A few frames of each of 24 sessions behind their 16 first tokens.
        _cached("append_frames", "append", 24, (900, 6000), (131, 1760), 16, 16, 64, sinks=16,
                ring=2048, dtype="f16"),
        # One session's next token over its window: latency.
        _cached("token_one", "attend", 1, (1500, 1500), (1, 1), 16, 16, 64, ring=1024),
        # The next token of every session a server holds.
        _cached("token_256", "attend", 256, (1024, 5000), (1, 1), 16, 16, 64, ring=1024),
        # Ragged contexts, grouped heads, pages of 32 tokens.
        _cached("token_ragged", "attend", 48, (1, 12000), (1, 1), 32, 8, 128, page_rows=32,
                dtype="f16"),
        # One very long context, four drafted tokens checked at once.
        _cached("token_long", "attend", 1, (200001, 200001), (4, 4), 32, 8, 128, page_rows=64),
        # One frame of one session over its window and first tokens.
        _cached("block_frame", "attend", 1, (5000, 5000), (880, 880), 16, 16, 64, sinks=16,
                ring=2944, window=2048),
        # A few frames of many sessions, ragged, odd lengths.
        _cached("block_sessions", "attend", 24, (700, 3000), (65, 700), 16, 16, 64, sinks=16,
                window=1024, dtype="f16"),
        # A prompt from its first token, grouped heads.
        _cached("block_prompt", "attend", 1, (8000, 8000), (8000, 8000), 32, 8, 128),
        # A long clip under a window with many first tokens visible.
        _cached("block_window", "attend", 1, (12345, 12345), (12345, 12345), 16, 4, 128,
                page_rows=24, sinks=100, window=1500, dtype="f16"),
    ]


def draw(rng):
    """One more case of the ranges that the listed ones stand for."""
    top = max(_cost(c) for c in listed())
    while True:
        c = _draw(rng)
        scores = c.get("sessions", 0) * c.get("q_heads", 0) * c.get("new_hi", 0) * c.get("len_hi", 0)
        if _cost(c) <= top and (c["op"] != "attend" or scores <= 2_000_000_000):
            return c


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw(rng):
    op = rng.choice(["rotate", "append", "token", "token", "block", "block"])
    head_dim = rng.choice([64, 128, 128, 64, 96, 80])
    kv_heads = rng.choice([1, 2, 4, 8, 16]) if head_dim > 64 else rng.choice([4, 8, 16])
    q_heads = kv_heads * rng.choice([1, 1, 2, 4, 5, 8])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    if op == "rotate":
        third = head_dim // 6
        pairs = (rng.randint(4, third), rng.randint(4, third), rng.randint(4, third))
        c = _rotate("", _log(rng, 1, 60000), q_heads, kv_heads, head_dim, pairs,
                    rng.choice([dtype, "f32"]), rng.random() < 0.5, rng.random() < 0.5)
    else:
        page_rows = rng.choice([8, 16, 16, 24, 32, 64])
        sinks = rng.choice([0, 0, rng.randint(1, 128)])
        if op == "append":
            sessions, new = _log(rng, 1, 200), _log(rng, 1, 2500)
        elif op == "token":
            sessions, new = _log(rng, 1, 300), rng.choice([1, 1, 1, 2, 4])
        else:
            sessions, new = _log(rng, 1, 32), _log(rng, 33, 9000)
        hi = max(new, _log(rng, 100, 150000 if op == "token" else 9000))
        lo = hi if sessions == 1 else rng.randint(1, hi)
        window = rng.choice([0, 0, rng.randint(100, 4000)])
        ring = rng.choice([0, new + max(window, rng.randint(200, 2500))])
        new_lo = new if op == "token" or sessions == 1 else rng.randint(1, new)
        c = _cached("", "append" if op == "append" else "attend", sessions, (lo, hi),
                    (new_lo, new), q_heads, kv_heads, head_dim, page_rows, sinks, ring, window,
                    dtype)
    del c["name"]
    return c


def _spread(lo, hi, i, n):
    """The i-th of n whole numbers spread over [lo, hi]; a single one is hi."""
    return hi if n == 1 else lo + int((hi - lo + 1) * ((i + 1) * 0.6180339887498949 % 1.0))


def _lengths(c):
    """New tokens of each session and its length with them."""
    n = c["sessions"]
    new = [_spread(c["new_lo"], c["new_hi"], i, n) for i in range(n)]
    return new, [max(new[i], _spread(c["len_lo"], c["len_hi"], 7 * i + 3, n)) for i in range(n)]


def _capacity(c, lens):
    """Slots of one session's page table."""
    rows = c["sinks"] + c["ring"] if c["ring"] else max(lens)
    return -(-rows // c["page_rows"])


def _visible(c, p, n):
    """Tokens that the token at position p sees of n in the cache."""
    low = max(n - c["ring"] if c["ring"] else 0, p - c["window"] + 1 if c["window"] else 0)
    return min(c["sinks"], p + 1) + max(0, p + 1 - max(low, c["sinks"])) if low > 0 else p + 1


def work(case):
    c = case
    size = _BYTES[c["dtype"]]
    if c["op"] == "rotate":
        n = c["tokens"] * (c["q_heads"] + c["kv_heads"]) * c["head_dim"]
        pairs = c["pairs_t"] + c["pairs_h"] + c["pairs_w"]
        return {"bytes": 2 * n * size + 12 * c["tokens"] + 4 * pairs, "flops": 3 * n}
    new, lens = _lengths(c)
    d, hq, hk = c["head_dim"], c["q_heads"], c["kv_heads"]
    tokens = sum(new)
    if c["op"] == "append":
        n = tokens * (hq + hk) * d
        return {"bytes": 2 * size * (n + tokens * hk * d) + 12 * tokens, "flops": 3 * n}
    rows = pairs = 0
    for m, length in zip(new, lens):
        # Rows of the cache that some new token sees, and (token, row) pairs.
        first = length - m
        low = max(length - c["ring"] if c["ring"] else 0,
                  first - c["window"] + 1 if c["window"] else 0)
        rows += min(length, c["sinks"] + length - max(low, c["sinks"])) if low > 0 else length
        pairs += sum(_visible(c, p, length) for p in range(first, length))
    return {"bytes": 2 * size * (rows * hk * d + tokens * hq * d) + 4 * tokens * hq,
            "flops": 4 * hq * d * pairs}


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


def prepare(case, seed):
    c = case
    g = torch.Generator(device=_DEV)
    g.manual_seed(0x0DD5EED + seed)
    dt = _TYPES[c["dtype"]]
    d = c["head_dim"]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=_DEV, dtype=dt)

    s = {"case": c, "ctx": _context() if own else None}
    if c["op"] == "rotate":
        t = c["tokens"]
        start = int(torch.randint(0, 200000, (1,), generator=g, device=_DEV))
        s["pos"] = _positions(start + torch.arange(t, device=_DEV))
        s["pairs"] = (c["pairs_t"], c["pairs_h"], c["pairs_w"])
        s["freq"] = _frequencies(s["pairs"])
        # Queries and keys side by side, as one projection writes them.
        x = normal(t, c["q_heads"] + c["kv_heads"], d)
        s["q"], s["k"] = x[:, :c["q_heads"]], x[:, c["q_heads"]:]
        if own:
            from paper_2607_21686_gb300 import pcs
            s["rotary"] = pcs.Rotary(s["pos"], s["freq"], s["pairs"], c["interleaved"])
        return s
    new, lens = _lengths(c)
    n, pages = c["sessions"], _capacity(c, lens)
    total = n * pages
    pool = total + total // 8 + 1
    s["k_pool"] = normal(pool, c["page_rows"], c["kv_heads"], d)
    s["v_pool"] = normal(pool, c["page_rows"], c["kv_heads"], d)
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
    s["q"] = normal(off[-1], c["q_heads"], d)
    if c["op"] == "append":
        s["k"] = normal(off[-1], c["kv_heads"], d)
        s["v"] = normal(off[-1], c["kv_heads"], d)
        number = torch.cat([torch.arange(a - m, a, device=_DEV) for m, a in zip(new, lens)])
        s["pos"] = _positions(number)
        third = d // 8
        s["pairs"] = (d // 2 - 2 * (d // 6), d // 6, d // 6) if d % 3 else (third, third, third)
        s["freq"] = _frequencies(s["pairs"])
    if own:
        from paper_2607_21686_gb300 import pcs
        s["cache"] = pcs.KvCache(s["k_pool"], s["v_pool"], s["table"], sinks=c["sinks"],
                                 ring=c["ring"])
        s["batch"] = pcs.KvBatch(s["lens"], s["tokens"], None if s["even"] else s["q_off"],
                                 s["max_new"], s["max_len"])
        if c["op"] == "append":
            s["rotary"] = pcs.Rotary(s["pos"], s["freq"], s["pairs"])
    return s


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(state):
    s = state
    c = s["case"]
    if c["op"] == "rotate":
        if own:
            q, k = s["ctx"].rotate([s["q"], s["k"]], s["rotary"], inverse=c["inverse"])
        else:
            cos, sin = _angles(s["pos"], s["freq"], s["pairs"])
            sin = -sin if c["inverse"] else sin
            q = _turned(s["q"], cos, sin, c["interleaved"])
            k = _turned(s["k"], cos, sin, c["interleaved"])
        return {"q": q, "k": k}
    if c["op"] == "append":
        if own:
            q = s["ctx"].kv_append(s["cache"], s["batch"], s["k"], s["v"], s["q"], s["rotary"])
        else:
            q = _append(s)
        return {"q": q, "k_pool": s["k_pool"], "v_pool": s["v_pool"]}
    if own:
        out, lse = s["ctx"].attend(s["cache"], s["batch"], s["q"], window=c["window"],
                                   return_lse=True)
    else:
        out, lse = _attend(s)
    return {"out": out, "lse": lse}


def _angles(pos, freq, pairs):
    """cos and sin of position times frequency [tokens, pairs].  The product is
    carried in two parts, so that far positions keep their last digits."""
    axis = torch.cat([torch.full((n,), a, device=pos.device) for a, n in enumerate(pairs)])
    p = pos.float()[:, axis]
    f = freq[None, :].expand_as(p)

    def halves(x):
        big = x * 4097.0
        high = big - (big - x)
        return high, x - high

    a = p * f
    ph, pl = halves(p)
    fh, fl = halves(f)
    rest = ((ph * fh - a) + ph * fl + pl * fh) + pl * fl
    cos, sin = torch.cos(a), torch.sin(a)
    return cos - sin * rest, sin + cos * rest


def _turned(x, cos, sin, interleaved):
    n = cos.shape[1]
    y = x.float()
    cos, sin = cos[:, None], sin[:, None]
    if interleaved:
        a, b = y[..., 0:2 * n:2], y[..., 1:2 * n:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = y[..., :n], y[..., n:2 * n]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([turned, y[..., 2 * n:]], -1).to(x.dtype)


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


def _append(s):
    c = s["case"]
    cos, sin = _angles(s["pos"], s["freq"], s["pairs"])
    session, p = _sessions_of(s)
    slot = _slots(c, p)
    row = s["table"][session, slot // c["page_rows"]].long() * c["page_rows"] + slot % c["page_rows"]
    k = _turned(s["k"], cos, sin, False)
    v = s["v"]
    if c["ring"]:  # of new tokens that share a slot the last one stays
        keep = (p < c["sinks"]) | (p >= s["lens"][session] - c["ring"])
        row, k, v = row[keep], k[keep], v[keep]
    s["k_pool"].flatten(0, 1)[row] = k
    s["v_pool"].flatten(0, 1)[row] = v
    return _turned(s["q"], cos, sin, False)


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
    k = s["k_pool"][page, row].float().masked_fill(hide, 0.0)
    v = s["v_pool"][page, row].float().masked_fill(hide, 0.0)
    session, p = _sessions_of(s)
    m = s["max_new"]
    place = torch.arange(s["tokens"], device=_DEV) - s["q_off"][session]
    q = torch.zeros(n, m, hk, group, d, device=_DEV)
    q[session, place] = s["q"].float().reshape(-1, hk, group, d)
    pos = torch.full((n, m), -1, device=_DEV)
    pos[session, place] = p
    sees = j[None, None] <= pos[..., None]
    if c["window"]:
        sees = sees & ((j < c["sinks"])[None, None] | (j[None, None] > pos[..., None] - c["window"]))
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


# ---------------------------------------------------------------------------
# The definition in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    c = case
    if c["op"] == "rotate":
        return {x: _turned_64(s[x], s, c["interleaved"], c["inverse"]) for x in ("q", "k")}
    new, lens = _lengths(c)
    if c["op"] == "append":
        return _append_64(s, c, new, lens)
    return _attend_64(s, c, new, lens)


def _turned_64(x, s, interleaved, inverse):
    """Each pair as a complex number, multiplied by exp(i angle)."""
    out = x.double().clone()
    i = 0
    count = sum(s["pairs"])
    for axis, n in enumerate(s["pairs"]):
        angle = s["pos"][:, axis].double()[:, None] * s["freq"][i:i + n].double()
        turn = torch.polar(torch.ones_like(angle), -angle if inverse else angle)[:, None]
        if interleaved:
            a, b = slice(2 * i, 2 * (i + n), 2), slice(2 * i + 1, 2 * (i + n), 2)
        else:
            a, b = slice(i, i + n), slice(count + i, count + i + n)
        z = torch.complex(out[..., a], out[..., b]) * turn
        out[..., a], out[..., b] = z.real.clone(), z.imag.clone()
        i += n
    return out


def _place_64(c, table, p):
    """Page and row of position p (a whole number) in a session's table."""
    if c["ring"] and p >= c["sinks"]:
        p = c["sinks"] + (p - c["sinks"]) % c["ring"]
    return int(table[p // c["page_rows"]]), p % c["page_rows"]


def _append_64(s, c, new, lens):
    kp, vp = s["k_pool"].double(), s["v_pool"].double()
    k, v = _turned_64(s["k"], s, False, False), s["v"].double()
    tables = s["table"].cpu().numpy()
    at, pages, rows, tokens = 0, [], [], []
    for i, (m, length) in enumerate(zip(new, lens)):
        last = {}
        for t in range(m):  # the last token of a slot stays
            last[_place_64(c, tables[i], length - m + t)] = at + t
        pages += [x[0] for x in last]
        rows += [x[1] for x in last]
        tokens += list(last.values())
        at += m
    pages, rows, tokens = (torch.tensor(x, device=_DEV) for x in (pages, rows, tokens))
    kp[pages, rows] = k[tokens]
    vp[pages, rows] = v[tokens]
    return {"q": _turned_64(s["q"], s, False, False), "k_pool": kp, "v_pool": vp}


def _attend_64(s, c, new, lens):
    d, hk = c["head_dim"], c["kv_heads"]
    group = c["q_heads"] // hk
    out = torch.zeros(s["tokens"], c["q_heads"], d, device=_DEV, dtype=torch.float64)
    lse = torch.full((s["tokens"], c["q_heads"]), -math.inf, device=_DEV, dtype=torch.float64)
    at = 0
    for i, (m, length) in enumerate(zip(new, lens)):
        oldest = max(0, length - c["ring"]) if c["ring"] else 0
        if c["window"]:
            oldest = max(oldest, length - m - c["window"] + 1)
        kept = torch.arange(length, device=_DEV)
        kept = kept[(kept < c["sinks"]) | (kept >= oldest)]
        slot = kept.clone()
        if c["ring"]:
            late = kept >= c["sinks"]
            slot[late] = (kept[late] - c["sinks"]).remainder(c["ring"]) + c["sinks"]
        page = s["table"][i].long()[torch.div(slot, c["page_rows"], rounding_mode="floor")]
        row = slot.remainder(c["page_rows"])
        for h in range(hk):
            k = s["k_pool"][page, row, h].double()
            v = s["v_pool"][page, row, h].double()
            for t in range(0, m, 1024):
                e = min(m, t + 1024)
                p = torch.arange(length - m + t, length - m + e, device=_DEV)[:, None]
                q = s["q"][at + t:at + e, h * group:(h + 1) * group].double().transpose(0, 1)
                x = q @ k.T / math.sqrt(d)
                far = kept[None] > p
                if c["window"]:
                    far |= (p - kept[None] >= c["window"]) & (kept[None] >= c["sinks"])
                x[far.expand_as(x)] = -math.inf
                part = torch.logsumexp(x, -1)
                y = torch.exp(x - part[..., None].clamp_min(-1e300)) @ v
                out[at + t:at + e, h * group:(h + 1) * group] = y.transpose(0, 1)
                lse[at + t:at + e, h * group:(h + 1) * group] = part.transpose(0, 1)
        at += m
    return {"out": out, "lse": lse}
