"""A generative session on a windowed key/value cache, suspended, resumed and
forked, with the library's operators doing what its model would do on the cache.

    python examples/window_session.py

A small model (random projections instead of weights) generates a clip frame by
frame: every layer gives queries and keys their place in time, height and width,
appends keys and values to the pages of a 1,024-token ring window and attends
over it.  After a few frames the session is checkpointed; it goes on, is
restored into other pages and goes on again from there: both continuations are
the same to the bit.  Then it is forked by sharing its pages: two branches write
different tokens, each into a page of its own, and do not see one another.
"""
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2607_21686_gb300 import pcs  # noqa: E402

LAYERS, HEADS, DIM, WINDOW, PAGE = 2, 16, 64, 1024, 16
FRAME = (20, 22)  # height, width: tokens of a frame
PAIRS = (8, 12, 12)


class Model:
    """Random projections per layer: what a real model would have trained."""

    def __init__(self, dev):
        g = torch.Generator(device=dev).manual_seed(7)
        n = HEADS * DIM
        self.qkv = [torch.randn(n, 3 * n, generator=g, device=dev, dtype=torch.bfloat16) / n ** 0.5 for _ in range(LAYERS)]
        self.freq = torch.cat([10000.0 ** (-torch.arange(p, device=dev) / p) for p in PAIRS]).float()


class Session:
    """Page tables per layer over shared pools, and the length so far."""

    def __init__(self, pools, tables, length=0):
        self.k_pool, self.v_pool = pools
        self.k_table, self.v_table = tables  # int32 [LAYERS, pages of a window]
        self.length = length

    def caches(self):
        return [pcs.KvCache(self.k_pool, self.v_pool, self.k_table[l:l + 1], ring=WINDOW, v_table=self.v_table[l:l + 1])
                for l in range(LAYERS)]

    def records(self):
        """The window as a session to checkpoint or to restore into."""
        meta = torch.tensor([self.length], dtype=torch.int64, device=self.k_pool.device)
        return pcs.kv_session(0, meta, self.k_pool, self.v_pool, self.k_table, self.length % WINDOW, WINDOW,
                              v_page_table=self.v_table)


def step(ctx, model, session, x):
    """One pass of the model over new tokens x [tokens, HEADS * DIM]."""
    n, dev = x.shape[0], x.device
    at = session.length + torch.arange(n, device=dev)
    h, w = FRAME
    pos = torch.stack([at // (h * w), at // w % h, at % w], -1).int()
    rotary = pcs.Rotary(pos, model.freq, PAIRS)
    session.length += n
    lens = torch.tensor([session.length], dtype=torch.int32, device=dev)
    batch = pcs.KvBatch(lens, n, max_len=session.length)
    for layer, cache in enumerate(session.caches()):
        q, k, v = (x @ model.qkv[layer]).view(n, 3, HEADS, DIM).unbind(1)
        q = ctx.kv_append(cache, batch, k, v, q, rotary)
        x = x + ctx.attend(cache, batch, q).reshape(n, -1)
        x = x / x.float().square().mean(-1, keepdim=True).sqrt().to(x.dtype)
    return x


def main():
    dev = torch.device("cuda:0")
    pages = WINDOW // PAGE
    with pcs.Context(0) as ctx:
        model = Model(dev)
        total = 4 * LAYERS * pages
        pools = [torch.zeros(total, PAGE, HEADS, DIM, dtype=torch.bfloat16, device=dev) for _ in range(2)]
        alloc = [pcs.Pool(ctx, p) for p in pools]

        def fresh():
            return [a.alloc(LAYERS * pages).view(LAYERS, pages) for a in alloc]

        g = torch.Generator(device=dev).manual_seed(1)

        def noise(n):
            return torch.randn(n, HEADS * DIM, generator=g, device=dev, dtype=torch.bfloat16)

        s = Session(pools, fresh())
        for _ in range(3):  # frames: blocks of tokens
            x = step(ctx, model, s, noise(FRAME[0] * FRAME[1]))
        x = x[-1:]
        for _ in range(4):  # token by token
            x = step(ctx, model, s, x)

        # Suspend, go on; resume in other pages, go on from there.
        snap, = ctx.checkpoint([s.records()])
        length = s.length
        ahead = step(ctx, model, s, step(ctx, model, s, x))
        back = Session(pools, fresh(), length)
        ctx.restore([snap], [back.records()], verify=True)
        again = step(ctx, model, back, step(ctx, model, back, x))
        assert torch.equal(ahead, again), "the resumed session went another way"

        # Fork: the child shares the pages; a branch makes the page that it
        # writes its own first.
        child = Session(pools, [a.share(t) for a, t in zip(alloc, (back.k_table, back.v_table))], back.length)
        page = torch.tensor([l * pages + back.length % WINDOW // PAGE for l in range(LAYERS)], dtype=torch.int32, device=dev)
        for a, t in zip(alloc, (child.k_table, child.v_table)):
            a.prepare_write(t, page)
        other = step(ctx, model, child, noise(1))
        same = step(ctx, model, back, again)
        alone = step(ctx, model, s, ahead)
        assert torch.equal(same, alone), "the branches saw one another"
        assert not torch.equal(other, same)
        ctx.delete(snap)
        ctx.sync()
        print("%d tokens, window %d, resumed and forked to the bit" % (s.length, WINDOW))
    return s.length


if __name__ == "__main__":
    main()
