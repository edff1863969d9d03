"""GPU tests of the operators on sequences of tokens: calls at the edges of what a cache and a batch can be."""
import pytest
import torch

import seq_ops_reference as ref
from block_ops_reference import within
from test_gpu_block_ops import BF, draws, tj  # noqa: F401  (tj: the fixture)
from test_gpu_seq_ops import run_attn

pytestmark = pytest.mark.gpu


# single tokens and prompts, tables whose tokens would be cut into parts or not, a prefix in front of few rows and of many
@pytest.mark.parametrize("new,width,prefix", [([1, 1], 1, 0), ([1, 1], 500, 0), ([1, 3], 40, 3000), ([0, 70], 5, 0), ([150, 20], 300, 0), ([300, 300], 10, 1000), ([200], 2, 64)])
@pytest.mark.parametrize("bits8", [False, True])
def test_a_cache_of_no_pages_has_no_tokens(tj, new, width, prefix, bits8):  # noqa: F811
    """Whatever tables and lengths hold: attention gives zeros, loading gives zeros, appending turns the queries and writes nothing else."""
    B = tj.binding
    H, D, Hq, page = 2, 64, 4, 16
    cache = tj.alloc_kv_cache(0, H, page, D, B.KV_8 if bits8 else B.KV_BF16)
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    N = starts[-1]
    ints = lambda v: torch.tensor(v, dtype=torch.int32).cuda()
    table = torch.arange(len(new) * width, dtype=torch.int32).view(len(new), width).cuda()
    batch = tj.KVBatch(table, ints([width * page] * len(new)), ints(starts), ints(list(range(-(-prefix // page)))) if prefix else None, prefix)
    normal = draws(N)
    q, kv = normal(N, Hq * D).to(BF).cuda(), normal(N, H * D).to(BF).cuda()
    print("no pages", new, width, prefix, bits8, flush=True)
    o = tj.attn(q, cache, batch, Hq, Out=torch.full((N, Hq * D), 3.0, dtype=BF, device="cuda"))
    assert not o.any()
    # rows that are more than their table has room for have no place: they stay as they were
    pos = torch.cat([torch.arange(width * page - n, width * page) for n in new]).to(torch.int32).cuda()
    placed = pos >= 0
    k, v = tj.kv_load(cache, batch, N, K=torch.full((N, H * D), 3.0, dtype=BF, device="cuda"), V=torch.full((N, H * D), 3.0, dtype=BF, device="cuda"))
    for t in (k, v):
        assert not t[placed].any() and (t[~placed] == 3.0).all()
    turn = tj.Rope(tj.rope_frequencies(D))
    qo = tj.kv_append(kv, kv, cache, batch, turn, Q=q, Qo=torch.full((N, Hq * D), 3.0, device="cuda"), out_dtype=B.OUT_F32)
    want = tj.rope(q, pos + prefix, turn, Hq, B.OUT_F32)
    assert (qo[~placed] == 3.0).all()
    # beside keys for 8 bits cosines and sines are made in 64 bits: 8 U of each of a pair's two elements on either side, and U of the sum
    off = 0.0 if not bits8 else 2.0 ** -24 * (2 * 8 * 2 + 2) * float(q.abs().max())
    assert float((qo - want)[placed].abs().max()) <= off


# On either side of who takes the prefix: a short one, and many tiles, in front of their own tokens; a long one in parts.
@pytest.mark.parametrize("case", [([0], [140], 4, 1, 64, 16, 300), ([0], [140], 4, 1, 64, 16, 420), ([0], [100], 2, 1, 128, 64, 1500), ([0, 30], [70, 65], 4, 2, 128, 32, 1111), ([3], [130], 1, 1, 208, 16, 700),
                                  ([0] * 4, [64, 1, 63, 129], 2, 1, 64, 16, 900)], ids=lambda c: "-".join(str(v) for v in (len(c[0]), max(c[1])) + c[2:]))
@pytest.mark.parametrize("bits8", [False, True])
def test_prompts_after_prefixes_of_every_length(tj, case, bits8):  # noqa: F811
    past, new, Hq, H, D, page, prefix = case
    print("attn", case, bits8, flush=True)
    bt, q, k, v, o, scale = run_attn(tj, case, bits8, 5)
    want, bound = ref.attn(q.view(bt.N, Hq, D), k, v, bt, scale, Hq)
    within(o.reshape(bt.N, Hq, D), want, bound, "out")
    assert torch.equal(tj.attn(q, bt.cache, bt.kv, Hq), o)


# Ascending starts that begin below the first row, end behind the last one, leave rows out at either end, or give sequences none; few rows and tiles of 128, one part and several
@pytest.mark.parametrize("N,starts", [(3, (-7, 1, 2, 900)), (3, (0, 0, 2, 3)), (3, (1, 1, 1, 2)), (3, (-5, -1, 0, 2)), (3, (3, 3, 3, 3)), (3, (2, 7, 9, 70)), (3, (-(2 ** 31), -9, 1, 2 ** 31 - 1)), (3, (5, 9, 12, 70)),
                                      (3, (-3, -2, -1, 0)), (150, (-50, 70, 4000, 4000)), (150, (10, 80, 80, 140)), (300, (-1, 299, 299, 2 ** 31 - 1))])
@pytest.mark.parametrize("prefix,extra", [(0, 0), (0, 40), (50, 0), (700, 40)])
def test_starts_that_reach_outside_the_rows(tj, N, starts, prefix, extra):  # noqa: F811
    """Every sequence has the rows between its starts that there are, the last tokens of it; rows between no two starts are left as they were."""
    B = tj.binding
    Hq, H, D = 4, 2, 64
    inside = [min(max(s, 0), N) for s in starts]
    new = [b - a for a, b in zip(inside, inside[1:])]
    bt = ref.Batch(tj, [30, 20, 10], new, H, D, 16, prefix=prefix, seed=3, extra_width=extra)
    normal = draws(N + prefix)
    T = len(bt.tokens())
    k, v = bt.fill(normal(T, H, D), normal(T, H, D))
    kv = tj.KVBatch(bt.kv.table, bt.kv.lens, torch.tensor(starts, dtype=torch.int32).cuda(), bt.kv.prefix_table, prefix)
    print("starts", N, starts, prefix, extra, flush=True)
    mine = torch.zeros(N, dtype=torch.bool)
    mine[inside[0]:inside[-1]] = True
    fresh = lambda width, dtype=BF: torch.full((N, width), -7.0, dtype=dtype, device="cuda")
    q = normal(N, Hq * D).to(BF).cuda()
    o = tj.attn(q, bt.cache, kv, Hq, Out=fresh(Hq * D))
    assert (o[~mine] == -7.0).all()
    want, bound = ref.attn(q[mine].view(-1, Hq, D), k, v, bt, D ** -0.5, Hq)
    within(o[mine].view(-1, Hq, D), want, bound, "out")
    lk, lv = tj.kv_load(bt.cache, kv, N, K=fresh(H * D), V=fresh(H * D))
    at = [bt.index[(b, bt.past[b] + i)] for b, i in bt.rows]
    for got, held in ((lk, k), (lv, v)):
        assert (got[~mine] == -7.0).all() and torch.equal(got[mine].double().cpu(), held[at].reshape(-1, H * D))
    x = normal(N, H * D).to(BF).cuda()
    turn = tj.Rope(tj.rope_frequencies(D))
    qo = tj.kv_append(x, x, bt.cache, kv, turn, Q=q, Qo=fresh(Hq * D, torch.float32), out_dtype=B.OUT_F32)
    pos = torch.zeros(N, dtype=torch.int32)
    pos[mine] = torch.tensor([prefix + bt.past[b] + i for b, i in bt.rows], dtype=torch.int32)
    assert (qo[~mine] == -7.0).all() and torch.equal(qo[mine], tj.rope(q, pos.cuda(), turn, Hq, B.OUT_F32)[mine])
    _, lv = tj.kv_load(bt.cache, kv, N, K=fresh(H * D), V=fresh(H * D))
    assert (lv[~mine] == -7.0).all() and torch.equal(lv[mine], x[mine])
