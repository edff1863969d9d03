"""The operators with which a model attends to what came before and chooses what comes next, as cases that can be prepared, run, checked and timed.

  rope     rotary positions on the heads of N tokens, forward and backward (the gradient is rotated back); the first R of a head's D
           elements, as two halves ("half") or as neighbours ("pairs"); angle = position * frequency
  append   keys (rotated) and values of new tokens into a paged cache, their queries rotated; "bf16" cache: the queries and the whole
           cache come back; "bits8": E4M3 codes and a power of two per token and head, and the new tokens are read back from it
  attend   queries against the paged cache: every token sees the shared prefix (if there is one), its own sequence's past and itself
  sample   one token per row of logits: temperature, the k largest, the smallest set of probability p, the least share of the
           largest probability, then the one that a given random number falls on, from the largest down

A batch is B sequences; sequence b has past_b tokens in the cache and n_b new ones, whose rows follow each other.  The pages of its own tokens
are listed in row b of a table, those of the prefix in a table of their own; position = prefix length + place in the sequence.  Where
`own` is false the operators are computed in their plain form, elementary torch operations in 32 bits (angles and what sampling adds up in 64);
where it is true by the library's calls.
"""
import math
import random

import torch

own = False

GROUP = 128                                   # elements of a head that share a power of two in an 8-bit cache
DEVICE = "cuda"


# ------------------------------------------------------------------------------------------------------ the cases ----

def listed():
    return [
        # a training step of the 1024-hidden model: queries and keys of 8 sequences of 2048 tokens, in one row of 16 + 16 heads
        dict(name="rope_16384x32x64", kind="rope", N=16384, H=32, D=64, R=64, form="half", type="bf16", far=2048, stretch=1.0),
        # a binary32 stream with odd sizes, half of each head turned, positions far beyond the trained ones, frequencies stretched for them
        dict(name="rope_1001x5x80_far_f32", kind="rope", N=1001, H=5, D=80, R=40, form="pairs", type="f32", far=1 << 20, stretch=32.0),
        # one answer of the 1024-hidden model: latency
        dict(name="append_1x16x64", kind="append", B=1, past=1000, new=1, Hq=16, Hkv=16, D=64, R=64, form="half", page=16, cache="bf16", prefix=0, lens=1),
        # 256 answers, each with its first tokens in two pages
        dict(name="append_256x8x128", kind="append", B=256, past=100, new=1, Hq=32, Hkv=8, D=128, R=128, form="half", page=64, cache="bf16", prefix=0, lens=2),
        # seven ragged prompts after a shared prefix into an 8-bit cache
        dict(name="append_prompts_bits8", kind="append", B=7, past=0, new=1200, Hq=32, Hkv=8, D=128, R=64, form="pairs", page=16, cache="bits8", prefix=777, lens=3),
        # one answer of the 1024-hidden model after a thousand tokens: latency
        dict(name="answer_1x1000", kind="attend", B=1, past=1000, new=1, Hq=16, Hkv=16, D=64, page=16, cache="bf16", prefix=0, lens=4),
        # 64 answers of ragged lengths: what a server does most
        dict(name="answer_64x8192", kind="attend", B=64, past=8192, new=1, Hq=32, Hkv=8, D=128, page=64, cache="bf16", prefix=0, lens=5),
        # one answer far into a long text, 8-bit cache
        dict(name="answer_1x200000_bits8", kind="attend", B=1, past=200000, new=1, Hq=32, Hkv=8, D=128, page=64, cache="bits8", prefix=0, lens=6),
        # 48 answers to questions on one long text
        dict(name="prefix_48x16384", kind="attend", B=48, past=500, new=1, Hq=32, Hkv=8, D=128, page=32, cache="bf16", prefix=16384, lens=7),
        # four ragged prompts at once
        dict(name="prompts_4x4096", kind="attend", B=4, past=0, new=4096, Hq=32, Hkv=8, D=128, page=64, cache="bf16", prefix=0, lens=8),
        # one answer, 16-bit logits over an odd vocabulary: latency
        dict(name="sample_1x50021", kind="sample", N=1, V=50021, type="bf16", k=50, p=0.9, m=0.0, greedy=False),
        # 64 answers over a large vocabulary, a wide set to draw from
        dict(name="sample_64x131072", kind="sample", N=64, V=131072, type="f32", k=0, p=0.95, m=0.0, greedy=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    D = rng.choice([32, 64, 64, 80, 96, 128, 128, 128, 192, 256])
    Hkv = _log(rng, 1, 16)
    return D, Hkv, Hkv * rng.choice([1, 1, 2, 4, 8])


def draw(rng):
    kind = rng.choice(["rope", "append", "append", "attend", "attend", "attend", "attend", "sample", "sample"])
    if kind == "rope":
        D = rng.choice([32, 64, 80, 96, 128, 256])
        H, type_ = _log(rng, 1, 64), rng.choice(["bf16", "bf16", "f32"])
        N = min(_log(rng, 1, 16384), (1 << (25 if type_ == "bf16" else 24)) // (H * D))
        return dict(kind="rope", N=N, H=H, D=D, R=D if rng.random() < 0.6 else 2 * rng.randint(1, D // 2), form=rng.choice(["half", "pairs"]), type=type_, far=_log(rng, 1000, 1 << 20),
                    stretch=rng.choice([1.0, 1.0, 8.0]))
    if kind == "sample":
        V = _log(rng, 1000, 200000)
        return dict(kind="sample", N=min(_log(rng, 1, 128), (1 << 23) // V), V=V, type=rng.choice(["bf16", "f32"]), k=0 if rng.random() < 0.4 else min(V, _log(rng, 1, 4000)),
                    p=rng.choice([1.0, 0.5, 0.9, 0.99]), m=rng.choice([0.0, 0.0, 0.02, 0.3]), greedy=rng.random() < 0.3)
    D, Hkv, Hq = _heads(rng)
    case = dict(kind=kind, Hq=Hq, Hkv=Hkv, D=D, page=rng.choice([16, 32, 64, 128]), cache=rng.choice(["bf16", "bf16", "bits8"]), lens=rng.randrange(1 << 30))
    if kind == "append":
        B = _log(rng, 1, 256)
        new = 1 if rng.random() < 0.5 else _log(rng, 2, max(2, min(2048, 8192 // B)))
        past = rng.choice([0, _log(rng, 1, 200)])
        return dict(case, B=B, past=past, new=new, R=D if rng.random() < 0.6 else 2 * rng.randint(1, D // 2), form=rng.choice(["half", "pairs"]), prefix=rng.choice([0, 777]))
    if rng.random() < 0.25:                   # prompts, or pieces of prompts after what is there already
        B = _log(rng, 1, 8)
        new = _log(rng, 2, min(4096, 12000 // B, int(math.sqrt(2.0 ** 30 / (B * Hq)))))
        past = rng.choice([0, _log(rng, 1, new)])
        return dict(case, B=B, past=past, new=new, prefix=0 if rng.random() < 0.7 else _log(rng, 100, new + 100))
    B = _log(rng, 1, 64)
    most = (1 << 27) // (B * Hkv * D)
    prefix = 0 if rng.random() < 0.6 else _log(rng, 100, max(200, min(16384, (1 << 25) // (Hkv * D), (1 << 26) // (B * Hq))))
    return dict(case, B=B, past=_log(rng, 1, max(2, min(100000, most, (1 << 29) // (B * Hq)))), new=1 if rng.random() < 0.8 else rng.randint(2, 5), prefix=prefix)


def _lengths(case):
    """Tokens in the cache and new tokens of each sequence: the longest as the case says, the others anywhere up to that."""
    r = random.Random(case["lens"])
    past = [r.randint(case["past"] // 8, case["past"]) for _ in range(case["B"])]
    new = [r.randint((case["new"] + 7) // 8, case["new"]) for _ in range(case["B"])]
    past[-1], new[-1] = case["past"], case["new"]
    return past, new


# ----------------------------------------------------------------------------------------------------- the inputs ----

def _type(case):
    return torch.bfloat16 if case["type"] == "bf16" else torch.float32


def _draws(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g, lambda *shape: torch.randn(shape, generator=g, device=DEVICE, dtype=torch.float32)


def _frequencies(R, stretch):
    """One per turned pair, base 10000; `stretch` divides them, for contexts that much longer than the trained ones."""
    j = torch.arange(R // 2, dtype=torch.float64)
    return (10000.0 ** (-2.0 * j / R) / stretch).float().to(DEVICE)


def _pages(case, seed, past, new):
    """The batch: tables and lengths on the GPU, and what the scheduler that made them knows of them."""
    B, page = case["B"], case["page"]
    own_pages = [-(-(a + n) // page) for a, n in zip(past, new)]
    prefix_pages = -(-case["prefix"] // page)
    total = sum(own_pages) + prefix_pages + 2                 # two that nobody has
    order = list(range(total))
    random.Random(seed).shuffle(order)
    width = max(1, max(own_pages))
    table, at = [], prefix_pages
    for n in own_pages:
        table.append(order[at:at + n] + [-1] * (width - n))
        at += n
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    ints = lambda v, t=torch.int32: torch.tensor(v, dtype=t, device=DEVICE)
    s = {"table": ints(table), "lens": ints([a + n for a, n in zip(past, new)]), "starts": ints(starts), "pages": total,
         "prefix_table": ints(order[:prefix_pages]) if prefix_pages else None}
    # of each row: its sequence and which of the sequence's new tokens it is
    s["row_seq"] = ints([b for b, n in enumerate(new) for _ in range(n)], torch.int64)
    s["row_at"] = ints([i for n in new for i in range(n)], torch.int64)
    s["most_new"], s["N"] = max(new), starts[-1]
    return s


def _bits8(x):
    """Codes and exponent bytes of values [..., D] for an 8-bit cache."""
    lead, D = x.shape[:-1], x.shape[-1]
    g = x.reshape(-1, D).split(GROUP, 1)
    m, e = torch.frexp(torch.stack([v.abs().amax(1) for v in g], 1))
    e = (e - 9 + (m > 0.875).int()).clamp(-126, 120)
    e = torch.where(m == 0, torch.full_like(e, -126), e)
    codes = torch.ldexp(x.reshape(-1, D), -e.repeat_interleave(GROUP, 1)[:, :D]).to(torch.float8_e4m3fn)
    return codes.view(torch.uint8).reshape(*lead, D), (e + 127).to(torch.uint8).reshape(*lead, len(g))


def _cache(case, pages, normal):
    """Pages of keys and values with something in every place: [pages, heads, tokens of a page, D]."""
    shape = (pages, case["Hkv"], case["page"], case["D"])
    k, v = normal(*shape), normal(*shape)
    if case["cache"] == "bf16":
        return {"k": k.to(torch.bfloat16), "v": v.to(torch.bfloat16), "k_exps": None, "v_exps": None}
    (kc, ke), (vc, ve) = _bits8(k), _bits8(v)
    return {"k": kc, "v": vc, "k_exps": ke, "v_exps": ve}


def prepare(case, seed):
    g, normal = _draws(seed)
    s = {"case": case}
    if case["kind"] == "rope":
        N, width, t = case["N"], case["H"] * case["D"], _type(case)
        s["x"], s["dy"] = normal(N, width).to(t), (1e-3 * normal(N, width)).to(t)
        s["pos"] = torch.randint(0, case["far"], (N,), generator=g, device=DEVICE, dtype=torch.int32)
        s["freqs"] = _frequencies(case["R"], case["stretch"])
        return s
    if case["kind"] == "sample":
        N, V = case["N"], case["V"]
        s["logits"] = (2.5 * normal(N, V)).to(_type(case))
        s["u"] = torch.rand(N, generator=g, device=DEVICE)
        full = lambda v, t=torch.float32: torch.full((N,), v, dtype=t, device=DEVICE)
        s["temperature"] = full(0.8)
        if case["greedy"]:
            s["temperature"][::4] = 0.0       # one answer in four takes the largest
        s["top_k"] = full(case["k"], torch.int32) if case["k"] else None
        s["top_p"] = full(case["p"]) if case["p"] < 1.0 else None
        s["min_p"] = full(case["m"]) if case["m"] > 0.0 else None
        return s
    past, new = _lengths(case)
    s |= _pages(case, seed, past, new)
    s |= _cache(case, s["pages"], normal)
    N, D = s["N"], case["D"]
    if case["kind"] == "attend":
        s["q"] = (2.0 * normal(N, case["Hq"] * D)).to(torch.bfloat16)
        return s
    # queries, keys and values in one row each, as one product gives them
    s["qkv"] = normal(N, (case["Hq"] + 2 * case["Hkv"]) * D).to(torch.bfloat16)
    s["freqs"] = _frequencies(case["R"], 1.0)
    return s


# ------------------------------------------------------------------------------------------------------ one pass ----

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2510_27527_amd as tj
    B = tj.binding
    case = s["case"]
    if case["kind"] == "sample":
        return {"tokens": tj.sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])}
    if case["kind"] == "rope":
        out = B.OUT_BF16 if case["type"] == "bf16" else B.OUT_F32
        turn = tj.Rope(s["freqs"], B.ROPE_HALF if case["form"] == "half" else B.ROPE_PAIRS)
        return {"y": tj.rope(s["x"], s["pos"], turn, case["H"], out), "dx": tj.rope(s["dy"], s["pos"], turn, case["H"], out, inverse=True)}
    cache = tj.KVCache(s["k"], s["v"], s["k_exps"], s["v_exps"])
    batch = tj.KVBatch(s["table"], s["lens"], None if case["new"] == 1 else s["starts"], s["prefix_table"], case["prefix"])
    if case["kind"] == "attend":
        return {"out": tj.attn(s["q"], cache, batch, case["Hq"])}
    turn = tj.Rope(s["freqs"], B.ROPE_HALF if case["form"] == "half" else B.ROPE_PAIRS)
    q, k, v = s["qkv"].split([case["Hq"] * case["D"], case["Hkv"] * case["D"], case["Hkv"] * case["D"]], 1)
    out = {"q": tj.kv_append(k, v, cache, batch, turn, Q=q)}
    if case["cache"] == "bf16":
        return dict(out, k=s["k"], v=s["v"])
    out["k"], out["v"] = tj.kv_load(cache, batch, s["N"])
    return out


def _turn(x, pos, freqs, form, back=False):
    """x [N, H, D] in 32 bits, turned by the angles of pos [N]."""
    R = 2 * freqs.numel()
    angle = pos.double()[:, None] * freqs.double()
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(-angle if back else angle).float()[:, None]
    t = x[..., :R]
    a, b = (t[..., :R // 2], t[..., R // 2:]) if form == "half" else (t[..., 0::2], t[..., 1::2])
    a, b = a * cos - b * sin, b * cos + a * sin
    t = torch.cat((a, b), -1) if form == "half" else torch.stack((a, b), -1).flatten(-2)
    return torch.cat((t, x[..., R:]), -1)


def _values(codes, exps):
    """Cache contents in 32 bits."""
    if exps is None:
        return codes.float()
    return torch.ldexp(codes.view(torch.float8_e4m3fn).float(), (exps.int() - 127).repeat_interleave(GROUP, -1)[..., :codes.shape[-1]])


def _plain_append(s):
    case = s["case"]
    D, Hq, Hkv, N = case["D"], case["Hq"], case["Hkv"], s["N"]
    q, k, v = s["qkv"].float().view(N, Hq + 2 * Hkv, D).split([Hq, Hkv, Hkv], 1)
    place = (s["lens"] - s["starts"].diff())[s["row_seq"]] + s["row_at"]
    q, k = (_turn(x, place + case["prefix"], s["freqs"], case["form"]) for x in (q, k))
    page, slot = s["table"][s["row_seq"], place // case["page"]].long(), place % case["page"]
    out = {"q": q.to(torch.bfloat16).view(N, Hq * D)}
    if case["cache"] == "bf16":
        s["k"][page, :, slot] = k.to(torch.bfloat16)
        s["v"][page, :, slot] = v.to(torch.bfloat16)
        return dict(out, k=s["k"], v=s["v"])
    (s["k"][page, :, slot], s["k_exps"][page, :, slot]), (s["v"][page, :, slot], s["v_exps"][page, :, slot]) = _bits8(k), _bits8(v)
    out["k"] = _values(s["k"][page, :, slot], s["k_exps"][page, :, slot]).to(torch.bfloat16).view(N, Hkv * D)
    out["v"] = _values(s["v"][page, :, slot], s["v_exps"][page, :, slot]).to(torch.bfloat16).view(N, Hkv * D)
    return out


def _plain_attend(s):
    case = s["case"]
    B, D, Hq, Hkv, most = case["B"], case["D"], case["Hq"], case["Hkv"], s["most_new"]
    G = Hq // Hkv

    def pages(codes, exps, table):            # [..., pages of a row] -> [..., heads, tokens, D]
        table = table.clamp_min(0).long()
        t = _values(codes[table], exps[table] if exps is not None else None)
        return t.transpose(-4, -3).reshape(*table.shape[:-1], Hkv, -1, D)

    q = torch.zeros(B, most, Hq, D, device=s["q"].device)
    q[s["row_seq"], s["row_at"]] = s["q"].float().view(-1, Hq, D)
    q = q.view(B, most, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, most * G, D)
    k, v = pages(s["k"], s["k_exps"], s["table"]), pages(s["v"], s["v_exps"], s["table"])
    scores = torch.matmul(q, k.transpose(-1, -2)) * D ** -0.5
    last = (s["lens"] - s["starts"].diff())[:, None] + torch.arange(most, device=q.device)       # the last place that a new token sees
    seen = torch.arange(k.shape[2], device=q.device) <= last[..., None]                          # [B, most, tokens]
    scores = scores.masked_fill(~seen.repeat_interleave(G, 1)[:, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    if case["prefix"]:
        pk, pv = (pages(c, e, s["prefix_table"])[:, :case["prefix"]] for c, e in ((s["k"], s["k_exps"]), (s["v"], s["v_exps"])))
        rows = q.transpose(0, 1).reshape(Hkv, -1, D)
        before = torch.matmul(rows, pk.transpose(-1, -2)) * D ** -0.5
        back = lambda t: t.view(Hkv, B, most * G, -1).transpose(0, 1)
        top = torch.maximum(top, back(before.amax(-1, keepdim=True)))
        before = torch.exp(before - top.transpose(0, 1).reshape(Hkv, -1, 1))
    weights = torch.exp(scores - top)
    total, out = weights.sum(-1, keepdim=True), torch.matmul(weights, v)
    if case["prefix"]:
        total = total + back(before.sum(-1, keepdim=True))
        out = out + back(torch.matmul(before, pv))
    out = (out / total).view(B, Hkv, most, G, D).permute(0, 2, 1, 3, 4).reshape(B, most, Hq * D)
    return {"out": out[s["row_seq"], s["row_at"]].to(torch.bfloat16)}


def _plain_sample(s):
    x, u = s["logits"].double(), s["u"].double()[:, None]
    N, V = x.shape
    warm = s["temperature"].double()[:, None]
    greedy = warm <= 0
    x, order = torch.sort(x, dim=1, descending=True, stable=True)
    w = torch.exp((x - x[:, :1]) / torch.where(greedy, torch.ones_like(warm), warm))
    rank = torch.arange(V, device=x.device)
    keep = torch.ones_like(w, dtype=torch.bool)
    if s["top_k"] is not None:
        keep &= rank < s["top_k"][:, None]
    if s["min_p"] is not None:
        least = w >= s["min_p"].double()[:, None]
    w = w * keep
    if s["top_p"] is not None:
        before = torch.cumsum(w, 1) - w
        keep &= (before < s["top_p"].double()[:, None] * w.sum(1, keepdim=True))
    if s["min_p"] is not None:
        keep &= least
    keep = torch.where(greedy, rank == 0, keep)
    sums = torch.cumsum(w * keep, 1)
    at = (sums <= u * sums[:, -1:]).sum(1, keepdim=True)
    return {"tokens": order.gather(1, at)[:, 0]}


def _run_plain(s):
    case = s["case"]
    if case["kind"] == "append":
        return _plain_append(s)
    if case["kind"] == "attend":
        return _plain_attend(s)
    if case["kind"] == "sample":
        return _plain_sample(s)
    t, shape = _type(case), (case["N"], case["H"], case["D"])
    y, dx = (_turn(x.float().view(shape), s["pos"], s["freqs"], case["form"], back).to(t).flatten(1) for x, back in ((s["x"], False), (s["dy"], True)))
    return {"y": y, "dx": dx}


# ------------------------------------------------------------------------------------- the definition in 64 bits ----

def _exact_turn(x, pos, freqs, form, back=False):
    """Pair j of a head as a complex number times e^(i angle)."""
    x = x.double().clone()
    half = freqs.numel()
    angle = torch.outer(pos.double(), freqs.double())[:, None]
    w = torch.polar(torch.ones_like(angle), -angle if back else angle)
    at = (slice(0, half), slice(half, 2 * half)) if form == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    z = torch.complex(x[..., at[0]], x[..., at[1]]) * w
    x[..., at[0]], x[..., at[1]] = z.real, z.imag
    return x


def _exact_kept(x):
    """What an 8-bit cache holds of x [..., D]: E4M3 times the least power of two that holds the largest of up to 128 elements."""
    out = torch.empty_like(x)
    for at in range(0, x.shape[-1], GROUP):
        v = x[..., at:at + GROUP]
        a = v.abs().amax(-1, keepdim=True)
        e = torch.ceil(torch.log2(a.clamp_min(2.0 ** -140) / 448.0))
        e = torch.where(a > 448.0 * torch.exp2(e), e + 1, e)
        e = torch.where(a <= 448.0 * torch.exp2(e - 1), e - 1, e).clamp(-126.0, 120.0)
        v = v * torch.exp2(-e)
        unit = torch.exp2((torch.frexp(v).exponent.double() - 4.0).clamp_min(-9.0))
        out[..., at:at + GROUP] = torch.round(v / unit) * unit * torch.exp2(e)
    return out


def _exact_sample(s):
    """Row by row: the kept tokens are a list, from the largest weight down."""
    import numpy as np
    x, u = s["logits"].double().cpu().numpy(), s["u"].double().cpu().numpy()
    got = []
    at = lambda name, n: None if s[name] is None else float(s[name][n])
    for n in range(x.shape[0]):
        order = np.lexsort((np.arange(x.shape[1]), -x[n]))
        if at("temperature", n) <= 0.0:
            got.append(int(order[0]))
            continue
        w = np.exp((x[n] - x[n].max()) / at("temperature", n))
        if s["top_k"] is not None:
            order = order[:int(at("top_k", n))]
        sums = np.cumsum(w[order])
        many = order.size
        if s["top_p"] is not None:
            many = min(many, 1 + int((sums[:-1] < at("top_p", n) * sums[-1]).sum()))
        if s["min_p"] is not None:
            many = min(many, int((w[order] >= at("min_p", n)).sum()))
        got.append(int(order[np.searchsorted(sums[:many], u[n] * sums[many - 1], side="right")]))
    return {"tokens": torch.tensor(got, dtype=torch.int64)}


def _exact_cache(codes, exps):
    if exps is None:
        return codes.double()
    b = codes.long() & 127
    size = torch.where(b < 8, b * 2.0 ** -9, (8.0 + b % 8) * torch.exp2((b // 8 - 10).double()))
    return torch.where(codes > 127, -size, size) * torch.exp2(exps.double() - 127.0).repeat_interleave(GROUP, -1)[..., :codes.shape[-1]]


def _exact_attend(s):
    case = s["case"]
    D, Hq, Hkv, page = case["D"], case["Hq"], case["Hkv"], case["page"]
    past, new = _lengths(case)
    out = torch.empty(s["N"], Hq, D, dtype=torch.float64, device=s["q"].device)

    def tokens(name, table, count):
        some = table[:-(-count // page)].long()
        t = _exact_cache(s[name][some], None if s[name + "_exps"] is None else s[name + "_exps"][some])
        return torch.cat(list(t.unbind(0)), 1)[:, :count]                   # [heads, tokens, D]

    before = [tokens(n, s["prefix_table"], case["prefix"]) for n in ("k", "v")] if case["prefix"] else None
    at = 0
    for b, (a, n) in enumerate(zip(past, new)):
        k, v = (tokens(name, s["table"][b], a + n) for name in ("k", "v"))
        if before is not None:
            k, v = torch.cat((before[0], k), 1), torch.cat((before[1], v), 1)
        hidden = torch.arange(k.shape[1], device=k.device)[None] > torch.arange(n, device=k.device)[:, None] + (case["prefix"] + a)
        q = s["q"][at:at + n].double().view(n, Hq, D)
        for h in range(Hkv):
            for j in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                p = torch.softmax((torch.matmul(q[:, j], k[h].t()) / math.sqrt(D)).masked_fill(hidden, -math.inf), 1)
                out[at:at + n, j] = torch.matmul(p, v[h])
        at += n
    return {"out": out.flatten(1)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "sample":
        return _exact_sample(s)
    if case["kind"] == "attend":
        return _exact_attend(s)
    if case["kind"] == "rope":
        shape = (case["N"], case["H"], case["D"])
        return {"y": _exact_turn(s["x"].view(shape), s["pos"], s["freqs"], case["form"]).flatten(1), "dx": _exact_turn(s["dy"].view(shape), s["pos"], s["freqs"], case["form"], True).flatten(1)}
    past, new = _lengths(case)
    D, Hq, Hkv, page, bits8 = case["D"], case["Hq"], case["Hkv"], case["page"], case["cache"] == "bits8"
    heads = s["qkv"].view(s["N"], -1, D)
    place = torch.tensor([a + i for a, n in zip(past, new) for i in range(n)], device=heads.device)
    q, k = (_exact_turn(x, place + case["prefix"], s["freqs"], case["form"]) for x in (heads[:, :Hq], heads[:, Hq:Hq + Hkv]))
    v = heads[:, Hq + Hkv:].double()
    out = {"q": q.flatten(1)}
    if bits8:
        return dict(out, k=_exact_kept(k).flatten(1), v=_exact_kept(v).flatten(1))
    out["k"], out["v"] = s["k"].double(), s["v"].double()
    where = s["table"].long()[s["row_seq"], place // page] * page + place % page            # tokens of the cache, in order
    for name, new_rows in (("k", k), ("v", v)):
        flat = out[name].transpose(1, 2).reshape(-1, Hkv, D)
        flat[where] = new_rows
        out[name] = flat.view(s["pages"], page, Hkv, D).transpose(1, 2).contiguous()
    return out


# ----------------------------------------------------------------------------------------- what a pass must cost ----

def work(case):
    """Bytes: each input read once, each output written once, the tokens that a batch sees read once per sequence, the prefix once for all."""
    if case["kind"] == "rope":
        n, e = float(case["N"] * case["H"] * case["D"]), 2.0 if case["type"] == "bf16" else 4.0
        return {"bytes": 4 * n * e + 8.0 * case["N"] + 4.0 * case["R"], "flops": 6.0 * n * case["R"] / case["D"]}
    if case["kind"] == "sample":
        n = float(case["N"] * case["V"])
        return {"bytes": n * (2.0 if case["type"] == "bf16" else 4.0) + 28.0 * case["N"], "flops": 20.0 * n}
    past, new = _lengths(case)
    D, Hq, Hkv = case["D"], case["Hq"], case["Hkv"]
    head = D * 2.0 if case["cache"] == "bf16" else D + float(-(-D // GROUP))
    N = float(sum(new))
    if case["kind"] == "append":
        bytes_ = N * (2 * Hq + 2 * Hkv) * D * 2.0 + N * 2 * Hkv * head + (N * 2 * Hkv * (head + 2.0 * D) if case["cache"] == "bits8" else 0.0)
        return {"bytes": bytes_, "flops": 3.0 * N * (Hq + Hkv) * case["R"]}
    seen = sum(a + n for a, n in zip(past, new)) + case["prefix"]
    pairs = sum(n * (a + case["prefix"]) + n * (n + 1) / 2.0 for a, n in zip(past, new))
    return {"bytes": seen * 2 * Hkv * head + N * 2 * Hq * D * 2.0, "flops": 4.0 * D * Hq * pairs}
