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
