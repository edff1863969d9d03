"""The operators on sequences of tokens from their definitions, in 64 bits, and how far a computation in 32 bits may be from them.

Errors are bounded by the usual model: every operation has a relative error of at most U = 2^-24.
"""
import math

import numpy as np
import torch

from block_ops_reference import ROUND, U, ckpt8, f64  # noqa: F401

# ------------------------------------------------------------------------------------------------- rotary positions ----

def rope(x, pos, freqs, pairs, scale=1.0, inverse=False):
    """x [N, H, D], pos [N] -> (y, bound without the output's rounding).  Cosine and sine: the argument, at most pi / 4 after the reduction, has three
    roundings, the series two more and what they leave out (2e-9 < U / 8), the scale one: 6 U in all, absolute; the angle itself is off by its size times 2^-51 (product, turns
    and their difference in 64 bits).  The sum of two products has two more."""
    x = f64(x)
    f = f64(freqs)
    half = f.numel()
    angle = torch.outer(pos.cpu().double(), f)[:, None]
    a, b = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if pairs else (x[..., :half], x[..., half:2 * half])
    c, s = torch.cos(angle) * scale, torch.sin(-angle if inverse else angle) * scale
    y, e = x.clone(), torch.zeros_like(x)
    u, v = a * c - b * s, b * c + a * s
    off = (8 * U + angle.abs() * 2.0 ** -51) * abs(scale) * (a.abs() + b.abs()) * 1.01
    for t, p, q in ((y, u, v), (e, off, off)):
        if pairs:
            t[..., 0:2 * half:2], t[..., 1:2 * half:2] = p, q
        else:
            t[..., :half], t[..., half:2 * half] = p, q
    return y, e


# ------------------------------------------------------------------------------------------------------- the cache ----

class Batch:
    """A scheduler's view: tokens of every sequence before the call (past), new ones, pages in random order, everything that nobody owns
    filled with what must not be seen."""

    def __init__(self, tj, past, new, heads, D, page, bits8=False, prefix=0, seed=0, spare=3, one_each=False, extra_width=0):
        B = tj.binding
        g = torch.Generator().manual_seed(seed)
        self.past, self.new, self.heads, self.D, self.page, self.prefix, self.bits8 = past, new, heads, D, page, prefix, bits8
        self.lens = [a + n for a, n in zip(past, new)]
        counts = [-(-n // page) for n in self.lens]
        ppages = -(-prefix // page)
        total = sum(counts) + ppages + spare
        order = torch.randperm(total, generator=g).tolist()
        width = max([1] + counts) + extra_width
        self.prefix_pages, at = order[:ppages], ppages
        self.tables = []
        for n in counts:
            self.tables.append(order[at:at + n] + [-1] * (width - n))
            at += n
        self.starts = [0]
        for n in new:
            self.starts.append(self.starts[-1] + n)
        self.N = self.starts[-1]
        ints = lambda v: torch.tensor(v, dtype=torch.int32).cuda()
        table = ints(self.tables) if past else torch.zeros(0, width, dtype=torch.int32, device="cuda")
        self.kv = tj.KVBatch(table, ints(self.lens), None if one_each else ints(self.starts), ints(self.prefix_pages) if prefix else None, prefix)
        self.cache = tj.alloc_kv_cache(total, heads, page, D, B.KV_8 if bits8 else B.KV_BF16)
        if bits8:
            for t in (self.cache.k, self.cache.v):
                t.fill_(0x7F)
            for t in (self.cache.k_exps, self.cache.v_exps):
                t.fill_(200)
        else:
            for t in (self.cache.k, self.cache.v):
                t.fill_(float("nan"))
        self.rows = [(b, i) for b, n in enumerate(new) for i in range(n)]

    def place(self, b, t):
        """(page, slot) of own token t of sequence b; b None: of the prefix."""
        pages = self.prefix_pages if b is None else self.tables[b]
        return pages[t // self.page], t % self.page

    def tokens(self):
        return [(None, t) for t in range(self.prefix)] + [(b, t) for b, n in enumerate(self.lens) for t in range(n)]

    def fill(self, k, v):
        """Keys and values [tokens(), heads, D] into the cache; returns them as the cache holds them, in 64 bits."""
        at = self.tokens()
        where = torch.tensor([self.place(b, t) for b, t in at]).reshape(-1, 2).cuda()
        held = []
        for x, name in ((k, "k"), (v, "v")):
            if self.bits8:
                codes, exps, values = ckpt8(x.reshape(-1, self.D))
                getattr(self.cache, name)[where[:, 0], :, where[:, 1]] = torch.from_numpy(codes).view(-1, self.heads, self.D).cuda()
                getattr(self.cache, name + "_exps")[where[:, 0], :, where[:, 1]] = torch.from_numpy(exps).view(len(at), self.heads, -1).cuda()
                held.append(values.view(-1, self.heads, self.D))
            else:
                x = x.to(torch.bfloat16)
                getattr(self.cache, name)[where[:, 0], :, where[:, 1]] = x.cuda()
                held.append(x.double())
        self.index = {p: i for i, p in enumerate(at)}
        return held

    def seen(self, b, i):
        """Indices of the tokens that new token i of sequence b sees."""
        last = self.past[b] + i
        return [self.index[(None, t)] for t in range(self.prefix)] + [self.index[(b, t)] for t in range(last + 1)]


def attn(q, k, v, batch, scale, Hq):
    """q [N, Hq, D] -> (out, bound).  Scores: exact products, sums of D in 32 bits, two roundings for the scale; the exponential is off by the score's error and
    two units; the weight's rounding to 8 bits is 2^-8 of it, which the sum of the weights does not have; the joins' and the sums' additions."""
    q = f64(q)
    N, _, D = q.shape
    G = Hq // batch.heads
    out, bound = torch.zeros_like(q), torch.zeros_like(q)
    for n, (b, i) in enumerate(batch.rows):
        at = batch.seen(b, i)
        if not at:
            continue
        ks, vs = k[at], v[at]
        for h in range(Hq):
            kk, vv = ks[:, h // G], vs[:, h // G]
            s = (kk @ q[n, h]) * scale
            e = (abs(scale) * (kk.abs() @ q[n, h].abs()) * (D + 4) + 4 * s.abs()) * U
            p = torch.softmax(s, 0)
            y = p @ vv
            rel = 2 * e.max() + (len(at) + 64) * U + 2.0 ** -8
            out[n, h] = y
            bound[n, h] = (p @ vv.abs()) * rel * 1.01 + ROUND[torch.bfloat16] * y.abs() + 1e-37
    return out, bound


# -------------------------------------------------------------------------------------------------------- sampling ----

def sample(x, u, T=None, k=None, p=None, m=None):
    """Tokens, row by row, in 64 bits."""
    x = f64(x).numpy()
    got = []
    for n in range(x.shape[0]):
        row = np.where(np.isnan(x[n]), -np.inf, x[n])
        top = row.max()
        if top == -np.inf:
            got.append(-1)
            continue
        order = np.lexsort((np.arange(row.size), -row))
        t = 1.0 if T is None else float(T[n])
        if not t > 0:
            got.append(int(order[0]))
            continue
        if top == np.inf:
            w = (row == np.inf).astype(float)
        else:
            w = np.exp((row - top) / t)
        w = np.where(row == -np.inf, 0.0, w)[order]
        keep = w.size
        if k is not None and 1 <= int(k[n]) < keep:
            keep = int(k[n])
        sums = np.cumsum(w[:keep])
        share = float(p[n]) if p is not None else 1.0
        many = keep
        if share < 1.0:
            before = sums - w[:keep]
            many = max(1, int((before < max(share, 0.0) * sums[-1]).sum()))
        least = float(m[n]) if m is not None else 0.0
        if least > 0.0:
            many = max(1, min(many, int((w[:keep] >= min(least, 1.0)).sum())))
        uu = min(max(float(u[n]), 0.0), 1 - 2.0 ** -24) if u[n] == u[n] else 0.0
        got.append(int(order[min(int(np.searchsorted(sums[:many], uu * sums[many - 1], side="right")), many - 1)]))
    return got
