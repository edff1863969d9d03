"""GPU tests of sampling from rows whose masks leave little: -infinity and NaN beside logits so low, or a temperature so small, that all of a row lies where logits are no longer told apart by
their distance; and a top_k between what is left and the size of the vocabulary."""
import math

import pytest
import torch

import seq_ops_reference as ref
from test_gpu_block_ops import BF, F32, tj  # noqa: F401  (tj: the fixture)

pytestmark = pytest.mark.gpu

# (value of the logits that are left, temperature): far below zero at ordinary temperatures, ordinary ones at temperatures near zero, the types' lowest, and one of every kind that is not
LOW = [(-2000.0, 1e-5), (-4e5, 0.01), (-3.5e7, 1.0), (-33554422.0, 1.0), (-1e9, 1.0), (-1e30, 1.0), (-3.3e38, 1.0), (-1e9, 50.0), (-2.5, 1.0), (-2.5, 1e-30), (3e38, 1.0)]


@pytest.mark.parametrize("V,left", [(100, 3), (100, 100), (8192, 5), (20011, 7), (50021, 1)])
@pytest.mark.parametrize("t", [BF, F32])
@pytest.mark.parametrize("hidden", [-math.inf, math.nan])
def test_top_k_counts_what_can_be_drawn(tj, V, left, t, hidden):  # noqa: F811
    """`left` equal logits, anywhere in the row, and nothing else that could be drawn: every k from `left` on keeps them all."""
    g = torch.Generator().manual_seed(V + left)
    where = torch.randperm(V, generator=g)[:left]
    N = len(LOW)
    x = torch.full((N, V), hidden)
    for n, (value, _) in enumerate(LOW):
        x[n, where] = value
    x = x.to(t)
    assert torch.isfinite(x[:, where]).all()
    T = torch.tensor([temperature for _, temperature in LOW])
    for k in (1, 2, left, left + 1, V - 1, V, V + 5, 1 << 30):
        top_k = torch.full((N,), k, dtype=torch.int32)
        for share in (0.0, 0.4, 0.9999):
            u, p, m = torch.full((N,), share), torch.full((N,), 0.75), torch.full((N,), 0.5)
            for kw in (dict(T=T, k=top_k), dict(T=T, k=top_k, p=p), dict(T=T, k=top_k, m=m)):
                print("sample", V, left, t, hidden, k, share, sorted(kw), flush=True)
                names = dict(T="temperature", k="top_k", p="top_p", m="min_p")
                got = tj.sample(x.cuda(), u.cuda(), **{names[n]: a.cuda() for n, a in kw.items()})
                assert got.tolist() == ref.sample(x, u, **kw), (k, share, sorted(kw))


@pytest.mark.parametrize("T", [0.9, 1.0, 2.0, 8.0])
def test_low_logits_of_different_weight(tj, T):  # noqa: F811
    """Logits from -2^25 down in binary32's steps of 4, so that weights differ by e^(-4 / T) a step, half of the row masked, and k on either side of what is left.  The random numbers keep away from
    the borders, which are off by the weights' rounding at most: 2^-43 of the largest for each of 300 tokens."""
    V, N = 600, 6
    steps = torch.randperm(V, generator=torch.Generator().manual_seed(5)).float()
    x = (-(2.0 ** 25) - 4.0 * (steps % 10)).expand(N, V).clone()
    x[:, ::2] = -math.inf
    warm = torch.full((N,), T)
    top_k = torch.tensor([1, 7, 299, 300, 301, 600], dtype=torch.int32)
    for share in (0.0, 0.1237, 0.6181, 0.98):
        u = torch.full((N,), share)
        for kw in (dict(T=warm, k=top_k), dict(T=warm, k=top_k, p=torch.full((N,), 0.8123)), dict(T=warm)):
            print("sample", T, share, sorted(kw), flush=True)
            names = dict(T="temperature", k="top_k", p="top_p")
            got = tj.sample(x.cuda(), u.cuda(), **{names[n]: a.cuda() for n, a in kw.items()})
            assert got.tolist() == ref.sample(x, u, **kw), (share, sorted(kw))
