"""GPU tests of the operators on sequences of tokens (rotary positions, the paged cache, attention over it, sampling) against their definitions
in 64 bits (seq_ops_reference.py)."""
import math

import numpy as np
import pytest
import torch

import seq_ops_reference as ref
from block_ops_reference import within
from test_gpu_block_ops import BF, F32, draws, out_of, spread, tj, untouched  # noqa: F401  (tj: the fixture)

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------- rotary positions ----

# heads of every shape: whole and ragged runs of eight pairs, parts of heads, nothing turned, single pairs, odd lengths
HEADS = [(1, 2, 2), (3, 5, 4), (2, 16, 16), (16, 64, 64), (5, 80, 40), (3, 96, 26), (2, 128, 128), (4, 128, 2), (7, 33, 30), (1, 256, 256), (2, 300, 298), (9, 40, 0), (1, 4096, 4096)]


@pytest.mark.parametrize("H,D,R", HEADS)
@pytest.mark.parametrize("pairs", [False, True])
def test_rope(tj, H, D, R, pairs):  # noqa: F811
    B = tj.binding
    normal = draws(H * D + R)
    for N, tx, ty, far, scale in ((1, BF, BF, 100, 1.0), (37, F32, BF, 1 << 20, 0.7), (5, BF, F32, 1 << 14, 1.0), (67, F32, F32, 2 ** 31 - 1, 1.25)):
        print("rope", N, H, D, R, pairs, tx, ty, flush=True)
        x = normal(N, H * D).to(tx).cuda()
        pos = torch.randint(-far if N == 5 else 0, far, (N,), generator=torch.Generator().manual_seed(N)).to(torch.int32).cuda()
        freqs = tj.rope_frequencies(R)
        turn = tj.Rope(freqs, B.ROPE_PAIRS if pairs else B.ROPE_HALF, scale)
        for inverse in (False, True):
            want, e = ref.rope(x.view(N, H, D), pos, freqs, pairs, np.float32(scale).item(), inverse)
            y = tj.rope(x, pos, turn, H, out_of(tj, ty), inverse=inverse)
            within(y.view(N, H, D), want, e + ref.ROUND[ty] * want.abs() + 1e-38, "y")
            if R < D:
                assert torch.equal(y.view(N, H, D)[..., R:], x.view(N, H, D)[..., R:].to(ty))
        # strided, off any alignment, and in place
        buf, v = spread(x, 3, 5)
        out, z = spread(torch.zeros(N, H * D, dtype=ty, device="cuda"), 1, 7)
        tj.rope(v, pos, turn, H, out_of(tj, ty), inverse=True, Y=z)
        assert torch.equal(z, y) and untouched(out, z)
        if tx == ty:
            tj.rope(v, pos, turn, H, out_of(tj, ty), inverse=True, Y=v)
            assert torch.equal(v, y) and untouched(buf, v)


def test_rope_gradient(tj):  # noqa: F811
    """<dy, f(x + h) - f(x)> = <f'(dy), h>: the rotation is linear, so the difference is the derivative at any step; the bound adds the errors of both sides."""
    B = tj.binding
    normal = draws(3)
    N, H, D = 33, 3, 48
    for form in (B.ROPE_HALF, B.ROPE_PAIRS):
        turn = tj.Rope(tj.rope_frequencies(32, scaling=B.ROPE_PARTS, factor=4.0, trained=512.0), form, 1.1)
        pos = torch.arange(N, dtype=torch.int32).cuda() * 1000
        x, h, dy = (normal(N, H * D).cuda() for _ in range(3))
        a, b = (tj.rope(t, pos, turn, H, B.OUT_F32).double() for t in (x + h, x))
        dx = tj.rope(dy, pos, turn, H, B.OUT_F32, inverse=True).double()
        left, right = (dy.double() * (a - b)).sum(), (dx * ((x + h).double() - x.double())).sum()
        size = (dy.double().abs() * (a.abs() + b.abs())).sum() + (dx.abs() * h.double().abs()).sum()
        assert float((left - right).abs()) <= 16 * ref.U * 1.1 * float(size)


def test_rope_of_many_tokens(tj):  # noqa: F811
    """More tokens and wider rows than one workgroup has, and the same bits for a token whatever the size of the call."""
    B = tj.binding
    g = torch.Generator(device="cuda").manual_seed(1)
    for N, H, D in ((5000, 1, 16), (300, 40, 128), (2, 4000, 64)):
        x = torch.randn(N, H * D, generator=g, device="cuda").to(BF)
        pos = torch.randint(0, 1 << 20, (N,), generator=g, device="cuda", dtype=torch.int32)
        turn = tj.Rope(tj.rope_frequencies(D))
        y = tj.rope(x, pos, turn, H)
        for n in (0, 1, N // 2, N - 1):
            assert torch.equal(tj.rope(x[n:n + 1], pos[n:n + 1], turn, H), y[n:n + 1])
        rows = slice(max(0, N - 3), N)
        want, e = ref.rope(x[rows].view(-1, H, D), pos[rows], turn.freqs, False)
        within(y[rows].view(-1, H, D), want, e + ref.ROUND[BF] * want.abs() + 1e-38, "y")


# -------------------------------------------------------------------------------------------------------- appending ----

# (past, new, heads of queries, heads, D, R, page, prefix)
APPENDS = [([0], [1], 1, 1, 16, 16, 16, 0), ([5, 0, 31, 100], [1, 1, 1, 1], 8, 2, 64, 64, 16, 0), ([0, 17, 3], [40, 0, 7], 6, 3, 80, 40, 32, 33), ([15, 16, 0], [2, 1, 16], 4, 4, 128, 26, 16, 0),
           ([0, 9], [70, 65], 2, 1, 256, 256, 64, 5), ([3], [12], 5, 5, 192, 0, 16, 0), ([1000, 2], [3, 2], 32, 8, 128, 128, 128, 300), ([0], [19], 40, 20, 144, 144, 16, 7)]


@pytest.mark.parametrize("case", APPENDS, ids=lambda c: "x".join(str(v) for v in c[2:]))
@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("pairs", [False, True])
def test_append_and_load(tj, case, bits8, pairs):  # noqa: F811
    B = tj.binding
    past, new, Hq, H, D, R, page, prefix = case
    normal = draws(D + page)
    for t in (BF, F32):
        one = all(n == 1 for n in new) and t == BF
        print("append", case, bits8, pairs, t, flush=True)
        bt = ref.Batch(tj, past, new, H, D, page, bits8, prefix, one_each=one)
        before = [x.clone() for x in (bt.cache.k, bt.cache.v, bt.cache.k_exps, bt.cache.v_exps) if x is not None]
        N = bt.N
        # queries, keys and values are columns of one matrix that starts off any alignment
        _, qkv = spread(normal(N, (Hq + 2 * H) * D).to(t).cuda(), 3, 1)
        q, k, v = qkv.split([Hq * D, H * D, H * D], 1)
        freqs = tj.rope_frequencies(R)
        turn = tj.Rope(freqs, B.ROPE_PAIRS if pairs else B.ROPE_HALF)
        out, qo = spread(torch.zeros(N, Hq * D, dtype=t, device="cuda"), 1, 2)
        tj.kv_append(k, v, bt.cache, bt.kv, turn, Q=q, Qo=qo, out_dtype=out_of(tj, t))
        pos = torch.tensor([prefix + past[b] + i for b, i in bt.rows], dtype=torch.int32)
        want, e = ref.rope(q.view(N, Hq, D) if q.is_contiguous() else q.reshape(N, Hq, D), pos, freqs, pairs)
        within(qo.reshape(N, Hq, D), want, e + ref.ROUND[t] * want.abs() + 1e-38, "q")
        assert untouched(out, qo)
        want, e = ref.rope(k.reshape(N, H, D), pos, freqs, pairs)
        lk, lv = tj.kv_load(bt.cache, bt.kv, N, B.OUT_F32)
        if bits8:
            # half a step of E4M3 (2^-4 of the value, 2^-10 of the group's power of two below the smallest ordinary one), a power of two at most one larger at the border
            top = torch.stack([g.abs().amax(-1) for g in want.split(128, -1)], -1).repeat_interleave(128, -1)[..., :D]
            power = torch.exp2(torch.ceil(torch.log2(top.clamp_min(1e-30) * (1 + 16 * ref.U) / 448)))
            within(lk.view(N, H, D), want, e * 1.1 + want.abs() * 2.0 ** -4 + power * 2.0 ** -10, "k")
            codes, exps, values = ref.ckpt8(v.reshape(-1, D).float())
            assert torch.equal(lv.view(-1, D).cpu().double(), values)
            at = torch.tensor([bt.place(b, past[b] + i) for b, i in bt.rows]).cuda()
            assert np.array_equal(bt.cache.v[at[:, 0], :, at[:, 1]].cpu().numpy().reshape(-1, D), codes)
            assert np.array_equal(bt.cache.v_exps[at[:, 0], :, at[:, 1]].cpu().numpy().reshape(exps.shape), exps)
        else:
            within(lk.view(N, H, D), want, e + ref.ROUND[BF] * want.abs() + 1e-38, "k")
            assert torch.equal(lv, v.to(BF).float())
        # nothing else in the cache has changed
        at = torch.tensor([bt.place(b, past[b] + i) for b, i in bt.rows]).cuda()
        for x, old in zip([x for x in (bt.cache.k, bt.cache.v, bt.cache.k_exps, bt.cache.v_exps) if x is not None], before):
            x[at[:, 0], :, at[:, 1]] = old[at[:, 0], :, at[:, 1]]
            raw = torch.int16 if x.dtype == BF else torch.uint8
            assert torch.equal(x.view(raw), old.view(raw))


def test_append_without_rotation_or_queries(tj):  # noqa: F811
    normal = draws(8)
    bt = ref.Batch(tj, [4, 0], [3, 20], 2, 64, 16)
    k, v = normal(bt.N, 128).to(BF).cuda(), normal(bt.N, 128).to(BF).cuda()
    assert tj.kv_append(k, v, bt.cache, bt.kv) is None
    lk, lv = tj.kv_load(bt.cache, bt.kv, bt.N)
    assert torch.equal(lk, k) and torch.equal(lv, v)


# -------------------------------------------------------------------------------------------------------- attention ----

# (past, new, heads of queries, heads, D, page, prefix): single tokens, lengths around blocks, units and pages, pieces of prompts, more rows than a tile, a prefix alone and with own tokens
ATTNS = [([0], [1], 1, 1, 16, 16, 0), ([0, 1, 14, 15, 16, 31, 32, 33], [1] * 8, 4, 2, 64, 16, 0), ([62, 63, 64, 127, 128, 129, 255], [1] * 7, 8, 1, 128, 32, 0), ([300, 5], [1, 1], 16, 16, 80, 64, 0),
         ([700, 90, 0], [1, 1, 1], 6, 2, 96, 128, 0), ([40, 333], [1, 1], 4, 1, 256, 16, 0), ([500], [1], 3, 3, 192, 32, 0), ([0], [70], 2, 1, 64, 16, 0), ([0, 10, 33], [33, 5, 64], 6, 2, 128, 32, 0),
         ([7, 0], [3, 0], 24, 1, 64, 16, 0), ([0, 0, 0], [1, 1, 1], 4, 2, 64, 16, 100), ([20, 3], [1, 1], 8, 2, 128, 16, 513), ([0, 31], [17, 20], 4, 4, 48, 64, 65), ([2, 100], [2, 1], 40, 1, 128, 16, 31)]
# and enough rows of a sequence, or of all against the prefix, for the kernel with tiles of 128: whole and ragged tiles, parts, tokens in front of the call's
ATTNS += [([0, 30], [64, 50], 4, 2, 64, 16, 0), ([300], [33], 4, 1, 128, 16, 0), ([0, 5], [200, 100], 1, 1, 128, 32, 0), ([0], [300], 2, 2, 64, 64, 0), ([129, 0], [200, 190], 2, 1, 80, 16, 0), ([1500], [100], 1, 1, 112, 128, 0),
          ([0] * 33, [1] * 33, 4, 2, 128, 16, 700), ([3] * 40, [2] * 40, 6, 2, 64, 32, 333), ([0, 7], [130, 150], 3, 1, 128, 16, 100), ([2] * 18, [1] * 18, 12, 1, 96, 16, 1200), ([0, 40], [70, 90], 2, 1, 256, 16, 0), ([300], [70], 3, 1, 192, 32, 60), ([0], [150], 1, 1, 144, 64, 0)]


def run_attn(tj, case, bits8, seed, one=False, spice=None):  # noqa: F811
    past, new, Hq, H, D, page, prefix = case
    normal = draws(seed)
    bt = ref.Batch(tj, past, new, H, D, page, bits8, prefix, seed=seed, one_each=one, extra_width=seed % 3)
    T = len(bt.tokens())
    k, v = normal(T, H, D), normal(T, H, D)
    if spice:
        spice(bt, k, v)
    k, v = bt.fill(k, v)
    q = normal(bt.N, Hq * D, std=2.0).to(BF).cuda()
    scale = D ** -0.5
    out, o = spread(torch.zeros(bt.N, Hq * D, dtype=BF, device="cuda"), 1, 3)
    _, qv = spread(q, 5, 2)
    tj.attn(qv, bt.cache, bt.kv, Hq, Out=o)
    assert untouched(out, o)
    return bt, q, k, v, o, scale


@pytest.mark.parametrize("case", ATTNS, ids=lambda c: "-".join(str(v) for v in (max(c[0]), max(c[1])) + c[2:]))
@pytest.mark.parametrize("bits8", [False, True])
def test_attention(tj, case, bits8):  # noqa: F811
    past, new, Hq, H, D, page, prefix = case
    for one in ([False, True] if all(n == 1 for n in new) else [False]):
        print("attn", case, bits8, one, flush=True)
        bt, q, k, v, o, scale = run_attn(tj, case, bits8, 7, one)
        want, bound = ref.attn(q.view(bt.N, Hq, D), k, v, bt, scale, Hq)
        within(o.reshape(bt.N, Hq, D), want, bound, "out")
        assert float((o.reshape(bt.N, Hq, D).double().cpu() - want).norm()) <= 2.0 ** -7 * float(want.norm())
        assert torch.equal(tj.attn(q, bt.cache, bt.kv, Hq), o)                      # the same bits again


# ---------------------------------------------------------------------------------------------------------- sampling ----

def rows(*v, t=F32):
    return torch.tensor(v, dtype=t).cuda()


@pytest.mark.parametrize("V", [1, 2, 7, 8, 63, 64, 1000, 1023, 4097, 8192, 16385, 50021, 131072, 200003])
@pytest.mark.parametrize("t", [BF, F32])
def test_sample(tj, V, t):  # noqa: F811
    g = torch.Generator().manual_seed(V)
    N = 24 if V < 100000 else 12
    x = (2.5 * torch.randn(N, V, generator=g)).to(t)
    u = torch.rand(N, generator=g)
    u[0], u[1] = 0.0, 1 - 2.0 ** -24
    T = torch.tensor([1.0, 0.8, 0.1, 3.0, 0.0, 1.5])[torch.arange(N) % 6]
    k = torch.tensor([0, 1, 5, 50, 4000, -3], dtype=torch.int32)[torch.arange(N) % 6 if N < 13 else (torch.arange(N) // 4) % 6]
    p = torch.tensor([0.9, 0.5, 1.0, 0.99, 0.1])[torch.arange(N) % 5]
    m = torch.tensor([0.0, 0.02, 0.3, 0.0])[torch.arange(N) % 4]
    # rows that are strided and start anywhere
    buf, v = spread(x.cuda(), 3, 5)
    for kw in ({}, dict(T=T), dict(k=k), dict(p=p), dict(m=m), dict(T=T, k=k, p=p, m=m)):
        print("sample", V, t, sorted(kw), flush=True)
        names = dict(T="temperature", k="top_k", p="top_p", m="min_p")
        got = tj.sample(v, u.cuda(), **{names[n]: a.cuda() for n, a in kw.items()})
        assert got.tolist() == ref.sample(x, u, **kw), sorted(kw)
    assert untouched(buf, v)


def test_sample_ties_go_by_index(tj):  # noqa: F811
    """Rows of equal logits, and of a few values: every border lies among equal weights, which are exact."""
    V = 20000
    flat = torch.zeros(1, V)
    steps = torch.arange(V).remainder(7).float()[None] * 0.5
    for x in (flat, steps):
        x = x.expand(16, V).contiguous()
        u = (torch.arange(16) + 0.37) / 16
        p = torch.full((16,), 0.5)
        k = torch.full((16,), 1234, dtype=torch.int32)
        for kw in ({}, dict(p=p), dict(k=k), dict(k=k, p=p)):
            names = dict(k="top_k", p="top_p")
            for t in (BF, F32):
                got = tj.sample(x.to(t).cuda(), u.cuda(), **{names[n]: a.cuda() for n, a in kw.items()})
                assert got.tolist() == ref.sample(x, u, **kw), sorted(kw)


def test_sample_of_odd_rows(tj):  # noqa: F811
    """NaN, infinities, nothing to draw from, one value far above the others, parameters that are no numbers."""
    inf, nan = math.inf, math.nan
    x = torch.full((10, 300), -1.0)
    x[0] = -inf
    x[1] = nan
    x[2, 5] = inf
    x[3, 7], x[3, 200] = inf, inf
    x[4, ::2] = nan
    x[5, 11] = 1e30
    x[6] = -3e38
    x[7, 1:] = -inf
    x[8, 100] = 0.0
    x[9] = torch.linspace(-40, 40, 300)
    u = torch.tensor([0.5, 0.5, 0.9, 0.75, 0.999, 0.999, 0.999, 0.3, 0.5, 0.2])
    assert tj.sample(x.cuda(), u.cuda()).tolist() == ref.sample(x, u)
    bad = torch.full((10,), nan)
    far = torch.full((10,), inf)
    assert tj.sample(x.cuda(), u.cuda(), temperature=bad.cuda()).tolist() == ref.sample(x, u, T=bad)
    assert tj.sample(x.cuda(), u.cuda(), top_p=bad.cuda(), min_p=bad.cuda()).tolist() == ref.sample(x, u)
    assert tj.sample(x.cuda(), u.cuda(), top_p=-far.cuda(), min_p=bad.cuda()).tolist() == ref.sample(x, u, p=-far)
    assert tj.sample(x.cuda(), u.cuda(), min_p=far.cuda()).tolist() == ref.sample(x, u, m=far)
    for T in (1e-3, 1e-30, 1e6):
        t = torch.full((10,), T)
        assert tj.sample(x.cuda(), u.cuda(), temperature=t.cuda()).tolist() == ref.sample(x, u, T=t), T
    for v in (-1.0, nan, -inf):
        assert tj.sample(x.cuda(), torch.full((10,), v).cuda()).tolist() == ref.sample(x, torch.zeros(10))
    assert tj.sample(x.cuda(), torch.full((10,), 5.0).cuda()).tolist() == ref.sample(x, torch.full((10,), 1 - 2.0 ** -24))
