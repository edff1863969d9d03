"""A small decoder on the library's calls, answering several prompts at once: packed weights, a paged cache of keys and values, a token for each sequence per step.

    block:  x  ->  norm  ->  queries, keys, values  ->  rotated, into the cache  ->  attention over the cache  ->  out  ->  + x
            x  ->  norm  ->  up  ->  SwiGLU  ->  down  ->  + x

All prompts may begin with the same tokens: these lie in the cache once, and every step reads them once for the whole batch.  Pages are handed out as sequences grow.  The weights
are random: what comes out is no text, but what every call gives can be followed.

    python examples/decoder.py [--hidden 512] [--layers 2] [--sequences 5] [--shared 300] [--steps 20] [--bits8]
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2510_27527_amd as tj  # noqa: E402
from paper_2510_27527_amd import binding as B  # noqa: E402

PAGE = 16


class Sequences:
    """The scheduler's side: which pages hold which tokens.  The same for all layers, each of which has a cache of its own."""

    def __init__(self, pages, count, most, device="cuda"):
        self.free = list(range(pages))
        self.device = device
        self.prefix, self.prefix_pages = 0, []
        self.lens = [0] * count
        self.pages = [[] for _ in range(count)]
        self.width = -(-most // PAGE)

    def _ints(self, v):
        return torch.tensor(v, dtype=torch.int32, device=self.device)

    def share(self, n):
        """The batch of one sequence that writes the shared tokens."""
        self.prefix_pages = [self.free.pop() for _ in range(-(-n // PAGE))]
        self.prefix = n
        return tj.KVBatch(self._ints([self.prefix_pages]), self._ints([n]), self._ints([0, n]))

    def grow(self, new):
        """`new[b]` more tokens for every sequence: the batch of the call that appends and attends to them."""
        starts = [0]
        for b, n in enumerate(new):
            self.lens[b] += n
            while len(self.pages[b]) * PAGE < self.lens[b]:
                self.pages[b].append(self.free.pop())
            starts.append(starts[-1] + n)
        table = [p + [-1] * (self.width - len(p)) for p in self.pages]
        return tj.KVBatch(self._ints(table), self._ints(self.lens), None if all(n == 1 for n in new) else self._ints(starts),
                          self._ints(self.prefix_pages) if self.prefix else None, self.prefix)


class Decoder:
    def __init__(self, hidden=512, heads=8, kv_heads=2, layers=2, mlp=1024, vocabulary=1000, pages=256, bits8=False, seed=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        draw = lambda *s: torch.randn(s, generator=g, device=device)
        pack = lambda rows, cols: tj.quantize((draw(rows, cols) * cols ** -0.5).bfloat16(), 0, B.ROUND_RTN)
        self.heads, self.kv_heads, self.D = heads, kv_heads, hidden // heads
        self.widths = [heads * self.D, kv_heads * self.D, kv_heads * self.D]
        self.turn = tj.Rope(tj.rope_frequencies(self.D, device=device))
        self.embedding = draw(vocabulary, hidden).bfloat16()
        self.head = pack(vocabulary, hidden)
        self.layers = [{"qkv": pack(sum(self.widths), hidden), "out": pack(hidden, hidden), "up": pack(2 * mlp, hidden), "down": pack(hidden, mlp),
                        "gamma1": 1 + 0.1 * draw(hidden), "gamma2": 1 + 0.1 * draw(hidden),
                        "cache": tj.alloc_kv_cache(pages, kv_heads, PAGE, self.D, B.KV_8 if bits8 else B.KV_BF16, device)} for _ in range(layers)]

    def attention(self, layer, x, batch):
        y = tj.norm_fwd(x, layer["gamma1"], norm=B.NORM_RMS)
        q, k, v = tj.gemv(y, layer["qkv"]).split(self.widths, 1)
        q = tj.kv_append(k, v, layer["cache"], batch, self.turn, Q=q)
        return tj.gemv(tj.attn(q, layer["cache"], batch, self.heads), layer["out"]).add_(x)

    def mlp(self, layer, x):
        y = tj.norm_fwd(x, layer["gamma2"], norm=B.NORM_RMS)
        return tj.gemv(tj.act_fwd(tj.gemv(y, layer["up"]), B.ACT_SWIGLU), layer["down"]).add_(x)

    def forward(self, tokens, batch):
        """tokens [N] of the batch's rows -> their hidden states; keys and values are in the caches afterwards."""
        x = self.embedding[tokens]
        for layer in self.layers:
            x = self.mlp(layer, self.attention(layer, x, batch))
        return x

    def choose(self, x, u, **how):
        return tj.sample(tj.gemv(tj.norm_fwd(x, norm=B.NORM_RMS), self.head, B.OUT_F32), u, **how)


def answer(model, shared, prompts, steps, seed=0, **how):
    """`steps` tokens for each of the prompts (lists of tokens), which all follow the tokens of `shared`; [steps, prompts]."""
    assert all(prompts), "prompts: one token each at least, whose hidden state the answer begins with"
    device = model.embedding.device
    g = torch.Generator(device=device).manual_seed(seed)
    pages = model.layers[0]["cache"].k.shape[0]
    seqs = Sequences(pages, len(prompts), max(map(len, prompts)) + steps, device)
    ints = lambda v: torch.tensor(v, dtype=torch.int64, device=device)
    if shared:
        model.forward(ints(shared), seqs.share(len(shared)))
    batch = seqs.grow([len(p) for p in prompts])
    x = model.forward(ints([t for p in prompts for t in p]), batch)
    last = ints([len(p) for p in prompts]).cumsum(0) - 1
    x = x[last]
    out = []
    for step in range(steps):
        out.append(model.choose(x, torch.rand(len(prompts), generator=g, device=device), **how))
        if step + 1 < steps:
            x = model.forward(out[-1], seqs.grow([1] * len(prompts)))
    return torch.stack(out)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--hidden", type=int, default=512)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--sequences", type=int, default=5)
    ap.add_argument("--shared", type=int, default=300)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--bits8", action="store_true")
    a = ap.parse_args()
    model = Decoder(a.hidden, layers=a.layers, mlp=2 * a.hidden, bits8=a.bits8)
    g = torch.Generator().manual_seed(1)
    words = lambda n: torch.randint(0, 1000, (n,), generator=g).tolist()
    shared, prompts = words(a.shared), [words(3 + 7 * i) for i in range(a.sequences)]
    full = lambda v: torch.full((a.sequences,), v, device="cuda")
    how = dict(temperature=full(0.8), top_p=full(0.9), top_k=torch.full((a.sequences,), 40, dtype=torch.int32, device="cuda"))
    answer(model, shared, prompts, 2, **how)
    torch.cuda.synchronize()
    began = time.perf_counter()
    tokens = answer(model, shared, prompts, a.steps, **how)
    torch.cuda.synchronize()
    took = time.perf_counter() - began
    for b in range(a.sequences):
        print("after %d + %d tokens:" % (a.shared, len(prompts[b])), *tokens[:, b].tolist())
    print("%d tokens for each of %d sequences in %.1f ms" % (a.steps, a.sequences, 1e3 * took))
    cache = model.layers[0]["cache"]
    print("a token's keys and values: %.0f bytes a layer" % (sum(t.numel() * t.element_size() for t in vars(cache).values() if t is not None) / (cache.k.shape[0] * PAGE)))


if __name__ == "__main__":
    main()
