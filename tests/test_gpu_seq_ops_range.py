"""GPU tests of the operators on sequences of tokens at the ends of their ranges: values that are not finite, tables and lengths that are not what they should be, rows of no
sequence, many sequences, caches beyond 32-bit offsets, streams, graphs, and a step of all of them together."""
import math

import pytest
import torch

import seq_ops_reference as ref
from block_ops_reference import within
from test_gpu_block_ops import BF, F32, draws, spread, tj, untouched  # noqa: F401  (tj: the fixture)
from test_gpu_seq_ops import run_attn

pytestmark = pytest.mark.gpu


def check_attn(bt, q, k, v, o, scale, Hq):
    want, bound = ref.attn(q.view(bt.N, Hq, bt.D), k, v, bt, scale, Hq)
    within(o.reshape(bt.N, Hq, bt.D), want, bound, "out")
    return want


# ------------------------------------------------------------------------------------------- values that are not finite ----

# prompts and pieces of prompts on both kinds of tiles, whole and ragged heads, one answer, a prefix
@pytest.mark.parametrize("case", [([0], [20], 2, 2, 64, 16, 0), ([5], [9], 8, 1, 128, 16, 0), ([40], [1], 4, 2, 96, 32, 0), ([0], [150], 1, 1, 64, 16, 0), ([70, 0], [90, 64], 2, 1, 128, 32, 0), ([3], [40], 4, 1, 256, 16, 0),
                                  ([0, 3], [3, 2], 4, 2, 64, 16, 70), ([0], [70], 2, 1, 80, 16, 100), ([0, 20], [80, 70], 1, 1, 208, 16, 0)], ids=lambda c: "-".join(str(v) for v in (max(c[0]), max(c[1])) + c[2:]))
@pytest.mark.parametrize("bits8", [False, True])
def test_what_is_not_finite_stays_with_the_rows_that_see_it(tj, case, bits8):  # noqa: F811
    """NaN and infinities in keys and values of new tokens: the rows in front of them must not know.  An 8-bit cache holds NaN in their place."""
    past, new, Hq, H, D, page, prefix = case

    def spice(bt, k, v):
        at = {p: i for i, p in enumerate(bt.tokens())}
        for b, n in enumerate(new):
            v[at[(b, past[b] + n - 1)], 0, 3] = math.nan
            if n > 2:
                v[at[(b, past[b] + n // 2)], H - 1, D - 1] = math.inf
                k[at[(b, past[b] + 2 * n // 3)], 0, 5] = math.nan
            if n > 30:
                v[at[(b, past[b] + 17)], 0, 8:12] = -math.inf
    bt, q, k, v, o, scale = run_attn(tj, case, bits8, 11, spice=spice)
    want = check_attn(bt, q, k, v, o, scale, Hq)
    assert torch.isnan(want).any() and (sum(new) == len(new) or torch.isfinite(want).any())


def test_scores_of_every_size(tj):  # noqa: F811
    """Scores far apart, growing from token to token, and all equal: the running maximum is moved often, and never."""
    normal = draws(2)
    Hq = H = 2
    D = 64
    for past, new in (([600], [1]), ([0], [200])):
        for kind in ("grow", "shrink", "equal", "huge"):
            bt = ref.Batch(tj, past, new, H, D, 32, seed=3)
            T = len(bt.tokens())
            ramp = torch.linspace(0, 1, T)
            k, v = normal(T, H, D), normal(T, H, D)
            k[:, :, 0] = {"grow": 400 * ramp, "shrink": 400 * (1 - ramp), "equal": 0 * ramp, "huge": 1e30 * (ramp - 0.5)}[kind][:, None]
            if kind == "equal":
                k[:] = 1.0
            k, v = bt.fill(k, v)
            q = normal(bt.N, Hq * D)
            q[:, ::D] = 1.0
            q = q.to(BF).cuda()
            o = tj.attn(q, bt.cache, bt.kv, Hq, scale=0.5)
            check_attn(bt, q, k, v, o, 0.5, Hq)


# ------------------------------------------------------------------------------ tables and lengths that are not in order ----

def test_pages_that_the_cache_does_not_have(tj):  # noqa: F811
    """Appending writes nothing there, attention sees no token there, loading gives zeros."""
    B = tj.binding
    normal = draws(4)
    Hq, H, D, page = 4, 2, 64, 16
    for bits8 in (False, True):
        for past, new in (([70, 40], [1, 1]), ([20, 0], [100, 90])):
            bt = ref.Batch(tj, past, new, H, D, page, bits8, seed=5)
            T = len(bt.tokens())
            k, v = bt.fill(normal(T, H, D), normal(T, H, D))
            table = bt.kv.table.clone()
            gone = {(0, 1): 1 << 30, (0, 3): -1, (1, 0): bt.cache.k.shape[0], (1, 2): -(1 << 31)}
            for (b, i), p in gone.items():
                table[b, i] = p
            kv = tj.KVBatch(table, bt.kv.lens, bt.kv.starts)
            q = normal(bt.N, Hq * D).to(BF).cuda()
            o = tj.attn(q, bt.cache, kv, Hq)
            seen = bt.seen
            bt.seen = lambda b, i: [j for j in seen(b, i) if (bt.tokens()[j][0], bt.tokens()[j][1] // page) not in gone]
            check_attn(bt, q, k, v, o, D ** -0.5, Hq)
            before = [t.clone() for t in (bt.cache.k, bt.cache.v)]
            x = normal(bt.N, H * D).to(BF).cuda()
            tj.kv_append(x, x, bt.cache, kv)
            lk, lv = tj.kv_load(bt.cache, kv, bt.N, B.OUT_F32)
            lost = torch.tensor([(b, (past[b] + i) // page) in gone for b, i in bt.rows]).cuda()
            assert not lk[lost].any() and not lv[lost].any() and (lk[~lost].any(1)).all()
            kept = torch.ones(bt.cache.k.shape[0], page, dtype=torch.bool, device="cuda")
            for (b, i), there in zip(bt.rows, (~lost).tolist()):
                if there:
                    kept[bt.place(b, past[b] + i)] = False
            raw = torch.uint8 if bits8 else torch.int16
            for t, old in zip((bt.cache.k, bt.cache.v), before):
                assert torch.equal(t.view(raw).transpose(1, 2)[kept], old.view(raw).transpose(1, 2)[kept])


def test_lengths_and_starts_out_of_order(tj):  # noqa: F811
    """Whatever lengths and starts hold, nothing outside the arrays is read or written; rows with nothing to see give zeros; sequences longer than their table end where it does."""
    normal = draws(6)
    Hq, H, D, page = 2, 1, 64, 16
    bt = ref.Batch(tj, [30, 20, 10], [1, 1, 1], H, D, page, seed=1)
    T = len(bt.tokens())
    bt.fill(normal(T, H, D), normal(T, H, D))
    q = normal(3, Hq * D).to(BF).cuda()
    good = tj.attn(q, bt.cache, bt.kv, Hq)
    ints = lambda *v: torch.tensor(v, dtype=torch.int32).cuda()
    width = bt.kv.table.shape[1]
    # lengths: none, below zero, beyond the table (whose last pages are not filled: those tokens are NaN and seen)
    o = tj.attn(q, bt.cache, tj.KVBatch(bt.kv.table, ints(0, -5, 11)), Hq)
    assert not o[:2].any() and torch.equal(o[2], good[2])
    table = bt.kv.table.clone()
    table[0] = table[0, 0]
    a, b = (tj.attn(q[:1], bt.cache, tj.KVBatch(table[:1].contiguous(), ints(n)), Hq) for n in (2 ** 31 - 1, width * page))
    assert torch.equal(a, b) and torch.isfinite(a.float()).all()
    # fewer tokens than rows: the first rows have nothing
    o = tj.attn(q, bt.cache, tj.KVBatch(bt.kv.table[:1].contiguous(), ints(1), ints(0, 3)), Hq)
    assert not o[:2].any() and torch.isfinite(o[2].float()).all() and o[2].any()
    # starts that descend, leave gaps, name rows twice, lie outside: every row is its own sequence's or left as it was
    for starts in ((0, 3, 0, 3), (2, 1, 0, 3), (-7, 1, 900, 3), (0, 0, 0, 0), (3, 3, 3, 3), (5, 9, 12, 70), (2 ** 31 - 1, -(2 ** 31), 2 ** 31 - 1, 0), (1, 2, 2, 3)):
        kv = tj.KVBatch(bt.kv.table, ints(4, 5, 6), ints(*starts))
        out, o = spread(torch.zeros(3, Hq * D, dtype=BF, device="cuda"), 1, 3)
        tj.attn(q, bt.cache, kv, Hq, Out=o)
        x = normal(3, H * D).to(BF).cuda()
        kout, ko = spread(torch.zeros(3, H * D, dtype=BF, device="cuda"), 1, 3)
        vout, vo = spread(torch.zeros(3, H * D, dtype=BF, device="cuda"), 1, 3)
        tj.kv_append(x, x, bt.cache, kv, Q=x)
        tj.kv_load(bt.cache, kv, 3, K=ko, V=vo)
        torch.cuda.synchronize()
        assert untouched(out, o) and untouched(kout, ko) and untouched(vout, vo)


def test_rows_of_no_sequence_are_left_as_they_were(tj):  # noqa: F811
    """A batch padded to a fixed number of rows, rows in front of the first sequence too, sequences without rows."""
    normal = draws(7)
    Hq, H, D = 4, 2, 64
    for prefix in (0, 50):
        for new in ([1, 0, 3], [70, 0, 65]):
            bt = ref.Batch(tj, [20, 9, 33], new, H, D, 16, prefix=prefix, seed=2)
            T = len(bt.tokens())
            k, v = bt.fill(normal(T, H, D), normal(T, H, D))
            n = bt.N
            q = normal(n + 7, Hq * D).to(BF).cuda()
            starts = bt.kv.starts + 3
            o = torch.full((n + 7, Hq * D), -7.0, dtype=BF, device="cuda")
            tj.attn(q, bt.cache, tj.KVBatch(bt.kv.table, bt.kv.lens, starts, bt.kv.prefix_table, prefix), Hq, Out=o)
            assert (o[:3] == -7.0).all() and (o[n + 3:] == -7.0).all()
            check_attn(bt, q[3:n + 3], k, v, o[3:n + 3], D ** -0.5, Hq)
            x = normal(n + 7, H * D).to(BF).cuda()
            qo = torch.full((n + 7, Hq * D), -7.0, dtype=BF, device="cuda")
            kv = tj.KVBatch(bt.kv.table, bt.kv.lens, starts, bt.kv.prefix_table, prefix)
            tj.kv_append(x, x, bt.cache, kv, tj.Rope(tj.rope_frequencies(D)), Q=q, Qo=qo)
            assert (qo[:3] == -7.0).all() and (qo[n + 3:] == -7.0).all() and (qo[3:n + 3] != -7.0).any(1).all()
            lk = torch.full((n + 7, H * D), -7.0, dtype=BF, device="cuda")
            lv = lk.clone()
            tj.kv_load(bt.cache, kv, n + 7, K=lk, V=lv)
            assert (lk[:3] == -7.0).all() and (lv[n + 3:] == -7.0).all() and torch.equal(lv[3:n + 3], x[3:n + 3])


def test_empty_calls(tj):  # noqa: F811
    e = lambda *s, dtype=BF: torch.zeros(s, dtype=dtype, device="cuda")
    i32 = lambda *s: e(*s, dtype=torch.int32)
    cache = tj.alloc_kv_cache(0, 2, 16, 64)
    for B, N, starts in ((0, 0, None), (0, 4, i32(1)), (2, 0, i32(3)), (2, 2, None)):
        kv = tj.KVBatch(i32(B, 0), i32(B), starts)
        o = tj.attn(e(N, 128), cache, kv, 2, Out=torch.full((N, 128), 3.0, dtype=BF, device="cuda"))
        assert (o == (0.0 if N == B else 3.0)).all()
        tj.kv_append(e(N, 128), e(N, 128), cache, kv)
        k, v = tj.kv_load(cache, kv, N, K=torch.full((N, 128), 3.0, dtype=BF, device="cuda"))
        assert (k == 3.0).all()              # no token has a place: nothing is loaded
    assert tj.rope(e(0, 128), i32(0), tj.Rope(tj.rope_frequencies(64)), 2).shape == (0, 128)
    assert tj.sample(e(0, 50), e(0, dtype=F32)).shape == (0,)
    torch.cuda.synchronize()


# ------------------------------------------------------------------------------------------------------ large and many ----

def test_many_sequences(tj):  # noqa: F811
    """More sequences than a workgroup has threads: every one with its own length, and the same bits as alone."""
    Hq, H, D, page = 4, 1, 64, 16
    for count in (300, 1111):
        g = torch.Generator().manual_seed(count)
        past = torch.randint(0, 200, (count,), generator=g).tolist()
        bt = ref.Batch(tj, past, [1] * count, H, D, page, seed=count, one_each=count == 1111)
        bt.cache.k.copy_(torch.randn(bt.cache.k.shape, generator=g))
        bt.cache.v.copy_(torch.randn(bt.cache.v.shape, generator=g))
        q = torch.randn(count, Hq * D, generator=g).to(BF).cuda()
        o = tj.attn(q, bt.cache, bt.kv, Hq)
        K, V = bt.cache.k.double().cpu(), bt.cache.v.double().cpu()
        for b in list(range(0, count, 37)) + [count - 1]:
            n = bt.lens[b]
            pages = bt.tables[b][:-(-n // page)]
            k, v = (t[pages].transpose(1, 2).reshape(-1, H, D)[:n] for t in (K, V))
            for h in range(Hq):
                s = k[:, 0] @ q[b].cpu().double().view(Hq, D)[h] * D ** -0.5
                p = torch.softmax(s, 0)
                want = p @ v[:, 0]
                bound = (p @ v[:, 0].abs()) * (2.0 ** -8 + 2.0 ** -14) + 2.0 ** -8 * want.abs() + 1e-37
                assert ((o[b].view(Hq, D)[h].double().cpu() - want).abs() <= bound).all()
        assert torch.equal(tj.attn(q, bt.cache, bt.kv, Hq), o)


@pytest.mark.parametrize("bits8", [False, True])
def test_a_cache_beyond_32_bit_offsets(tj, bits8):  # noqa: F811
    """More than 2^32 elements: the pages in use are the first and the last ones."""
    B = tj.binding
    H, D, page, Hq = 8, 128, 64, 8
    pages = (1 << 32) // (H * D * page) + 700
    cache = tj.alloc_kv_cache(pages, H, page, D, B.KV_8 if bits8 else B.KV_BF16)
    small = tj.alloc_kv_cache(4, H, page, D, B.KV_8 if bits8 else B.KV_BF16)
    g = torch.Generator(device="cuda").manual_seed(1)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32).cuda()
    n = 100
    x, y, q = (torch.randn(2 * n, H * D, generator=g, device="cuda").to(BF) for _ in range(3))
    outs = []
    for c, table in ((cache, [[pages - 1, 0], [pages - 2, pages - 650]]), (small, [[3, 0], [1, 2]])):
        kv = tj.KVBatch(i32(table), i32([n, n]), i32([0, n, 2 * n]))
        tj.kv_append(x, y, c, kv, tj.Rope(tj.rope_frequencies(D)))
        step = tj.KVBatch(i32(table), i32([n, n - 3]))
        outs.append(tj.kv_load(c, kv, 2 * n) + (tj.attn(q, c, kv, Hq), tj.attn(q[:2], c, step, Hq)))
    for a, b in zip(*outs):
        assert torch.equal(a, b)


def test_the_same_bits_whatever_the_size_of_a_call(tj):  # noqa: F811
    """A workspace for more is one for less, and a call's outputs do not depend on what it held."""
    Hq, H, D = 8, 2, 128
    bt = ref.Batch(tj, [700, 30, 1500], [1, 1, 1], H, D, 32, seed=4)
    g = torch.Generator().manual_seed(4)
    bt.cache.k.copy_(torch.randn(bt.cache.k.shape, generator=g))
    bt.cache.v.copy_(torch.randn(bt.cache.v.shape, generator=g))
    q = torch.randn(3, Hq * D, generator=g).to(BF).cuda()
    need = tj.attn_workspace_bytes(3, Hq, bt.cache, bt.kv)
    want = tj.attn(q, bt.cache, bt.kv, Hq)
    for fill in (0, 255):
        ws = torch.full((need + 5000,), fill, dtype=torch.uint8, device="cuda")
        assert torch.equal(tj.attn(q, bt.cache, bt.kv, Hq, ws=ws), want)
        assert (ws[need:] == fill).all()
    with pytest.raises(tj.NVFP4Error):
        tj.attn(q, bt.cache, bt.kv, Hq, ws=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))


# ------------------------------------------------------------------------------------------- streams, devices and graphs ----

def test_the_stream_of_a_call(tj):  # noqa: F811
    """Everything is enqueued on the current stream: work in front of it there is waited for."""
    side = torch.cuda.Stream()
    H, D, Hq, V = 2, 64, 4, 1000
    bt = ref.Batch(tj, [40], [1], H, D, 16, seed=1)
    bt.cache.k.zero_(), bt.cache.v.zero_()
    x = torch.randn(1, Hq * D, device="cuda").to(BF)
    logits = torch.randn(1, V, device="cuda")
    u = torch.full((1,), 0.4, device="cuda")
    turn = tj.Rope(tj.rope_frequencies(D))
    kv = x[:, :H * D]
    pos = torch.full((1,), 40, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()

    def step(x, kv, logits):
        q = tj.kv_append(kv, kv, bt.cache, bt.kv, turn, Q=x)
        return q, tj.attn(q, bt.cache, bt.kv, Hq), tj.rope(x, pos, turn, Hq), tj.sample(logits, u), *tj.kv_load(bt.cache, bt.kv, 1)
    want = step(x, kv, logits)
    torch.cuda.synchronize()
    a, b = torch.zeros_like(x), torch.zeros_like(logits)
    big = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            big = big @ big * 1e-3
        a.copy_(x), b.copy_(logits)
        got = step(a, a[:, :H * D], b)
    side.synchronize()
    for g, w in zip(got, want):
        assert torch.equal(g, w)


def test_refuses_tensors_of_another_device(tj, monkeypatch):  # noqa: F811
    B = tj.binding
    e = lambda *s, dtype=BF: torch.zeros(s, dtype=dtype, device="cuda")
    i32 = lambda *s: e(*s, dtype=torch.int32)
    cache, kv, turn = tj.alloc_kv_cache(2, 2, 16, 64), tj.KVBatch(i32(1, 2), i32(1)), tj.Rope(tj.rope_frequencies(64))
    calls = [lambda: tj.rope(e(1, 128), i32(1), turn, 2), lambda: tj.kv_append(e(1, 128), e(1, 128), cache, kv, turn), lambda: tj.kv_load(cache, kv, 1), lambda: tj.attn(e(1, 128), cache, kv, 2),
             lambda: tj.sample(e(1, 9), e(1, dtype=F32))]
    for call in calls:
        call()
    torch.cuda.synchronize()
    elsewhere = B._current_device() + 1
    monkeypatch.setattr(B, "_current_device", lambda: elsewhere)
    for call in calls:
        with pytest.raises(AssertionError, match="current device"):
            call()


def test_captured_steps(tj):  # noqa: F811
    """Two graphs with workspaces of their own, replayed in turn with eager work between: lengths, tables, logits and random numbers change between the replays, the sizes do not."""
    H, D, Hq, page, V = 2, 64, 8, 16, 5000
    normal = draws(9)
    turn = tj.Rope(tj.rope_frequencies(D))
    batches = [ref.Batch(tj, [100, 3, 47], [1, 1, 1], H, D, page, prefix=40, seed=1, one_each=True, extra_width=30), ref.Batch(tj, [0, 60], [70, 65], H, D, page, seed=2, extra_width=5)]
    graphs = []
    for bt in batches:
        bt.cache.k.copy_(normal(*bt.cache.k.shape)), bt.cache.v.copy_(normal(*bt.cache.v.shape))
        s = {"q": normal(bt.N, Hq * D).to(BF).cuda(), "kv": normal(bt.N, H * D).to(BF).cuda(), "logits": normal(bt.N, V).cuda(), "u": torch.rand(bt.N).cuda(),
             "ws": torch.empty(tj.attn_workspace_bytes(bt.N, Hq, bt.cache, bt.kv) + 16, dtype=torch.uint8, device="cuda")}

        def step(bt=bt, s=s):
            q = tj.kv_append(s["kv"], s["kv"], bt.cache, bt.kv, turn, Q=s["q"])
            return q, tj.attn(q, bt.cache, bt.kv, Hq, ws=s["ws"]), tj.sample(s["logits"], s["u"], top_p=s["u"])
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step()
        graphs.append((bt, s, step, graph, out))
    for turn_no in range(4):
        for bt, s, step, graph, out in graphs:
            s["q"].copy_(normal(bt.N, Hq * D)), s["kv"].copy_(normal(bt.N, H * D)), s["logits"].copy_(normal(bt.N, V)), s["u"].copy_(torch.rand(bt.N))
            if turn_no and bt.kv.starts is None:
                # what the tables have room for: other lengths, pages dealt anew
                g = torch.Generator().manual_seed(turn_no)
                width = bt.kv.table.shape[1]
                bt.kv.table.copy_(torch.randint(0, bt.cache.k.shape[0], (3, width), generator=g))
                for i in range(3):          # no page in two sequences: every place has one writer
                    bt.kv.table[i, 0::1] = torch.arange(i, 3 * width, 3)[:width].remainder(bt.cache.k.shape[0]).to(torch.int32).cuda()
                bt.kv.lens.copy_(torch.tensor([1, 16 * turn_no, 30]))
        for bt, s, step, graph, out in graphs:
            graph.replay()
        torch.cuda.synchronize()
        got = [[t.clone() for t in out] for *_, out in graphs]
        for (bt, s, step, graph, out), kept in zip(graphs, got):
            for a, b in zip(kept, step()):
                assert torch.equal(a, b), turn_no
        torch.cuda.synchronize()


@pytest.mark.parametrize("V", [8193, 50021, 1 << 20])
@pytest.mark.parametrize("values", ["equal", "near", "masked"])
def test_sample_of_crowded_rows(tj, V, values):  # noqa: F811
    """More tokens around the borders than the list holds: equal logits, different ones closer together than a bin is wide, and the larger half of a row equal above the others."""
    N = 4
    g = torch.Generator().manual_seed(V)
    if values == "equal":
        x = torch.full((N, V), -2.5)
    elif values == "near":
        x = 1.0 + 0.01 * torch.rand(N, V, generator=g)
    else:
        x = torch.where(torch.rand(N, V, generator=g) < 0.5, torch.tensor(3.0), torch.tensor(-1e30))
    u = torch.tensor([0.0, 0.2513, 0.7031, 1 - 2.0 ** -24])
    p = torch.tensor([0.9, 0.35, 0.6, 0.77])
    k = torch.tensor([V // 3, 0, 8192, V // 2 - 5], dtype=torch.int32)
    for t in (BF, F32):
        y = x.to(t)
        for kw in ({}, dict(p=p), dict(k=k, p=p)):
            print("sample", V, values, t, sorted(kw), flush=True)
            names = dict(p="top_p", k="top_k")
            got = tj.sample(y.cuda(), u.cuda(), **{names[n]: a.cuda() for n, a in kw.items()})
            assert got.tolist() == ref.sample(y, u, **kw), sorted(kw)


@pytest.mark.parametrize("rows", [47, 48, 49, 63, 64])
@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("shared", [False, True])
def test_attention_between_the_kinds_of_tiles(tj, rows, bits8, shared):  # noqa: F811
    """Rows on either side of where a call takes tiles of 128: new tokens of a sequence after others, and single tokens after a prefix."""
    case = ([5] * rows, [1] * rows, 2, 2, 128, 16, 333) if shared else ([200, 3], [rows, rows], 2, 2, 64, 32, 0)
    bt, q, k, v, o, scale = run_attn(tj, case, bits8, 3)
    check_attn(bt, q, k, v, o, scale, 2)


@pytest.mark.parametrize("N,starts,past,prefix", [(100, [0, 100] * 5 + [0], 40, 200), (40, [0, 40] * 9 + [0], 500, 0), (300, [0, 300, 7] * 6 + [300], 100, 777), (64, [0, 64, 0, 64], 300, 0)])
@pytest.mark.parametrize("bits8", [False, True])
def test_starts_that_name_rows_often_stay_in_the_workspace(tj, N, starts, past, prefix, bits8):  # noqa: F811
    """More tiles than the sizes of the call allow for: nothing behind the workspace or beside the output is written."""
    Hq, H, D, page = 2, 1, 64, 16
    B = len(starts) - 1
    bt = ref.Batch(tj, [past] * B, [1] * B, H, D, page, bits8, prefix, seed=4)
    normal = draws(9)
    T = len(bt.tokens())
    bt.fill(normal(T, H, D), normal(T, H, D))
    kv = tj.KVBatch(bt.kv.table, bt.kv.lens, torch.tensor(starts, dtype=torch.int32).cuda(), bt.kv.prefix_table, prefix)
    q = normal(N, Hq * D).to(BF).cuda()
    need = tj.attn_workspace_bytes(N, Hq, bt.cache, kv)
    whole = torch.full((need + (1 << 20),), 0xA5, dtype=torch.uint8, device="cuda")
    out, o = spread(torch.zeros(N, Hq * D, dtype=BF, device="cuda"), 1, 3)
    print("attn", N, starts, past, prefix, bits8, flush=True)
    tj.attn(q, bt.cache, kv, Hq, Out=o, ws=whole[:need])
    torch.cuda.synchronize()
    assert bool((whole[need:] == 0xA5).all()) and untouched(out, o)
