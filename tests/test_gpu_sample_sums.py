"""GPU tests of sampling where a target lies between two bins of a row to the last unit: more weight than a double holds to the unit, and none in the bins that follow the border."""
import numpy as np
import pytest
import torch

from sample_weights import weight
from test_gpu_block_ops import tj  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


def at(number, part):
    """A logit in bin `number` below 0 at temperature 1: bins are 1 / 32 wide."""
    x = float(np.float32(-(number - 1 + part) / 32))
    assert -np.floor(np.float32(x) * np.float32(32)) == number
    return x


def row_halved_behind_bin_2():
    """2048 tokens of 2^43, one each in bins 1 and 2, then as much as these have together in bins from 20 on, within a few units: half of the sum is at the end of bin 2.  The weights are so chosen
    that 2^54 + a + b comes to different doubles as (a + b) + 2^54 and a + (b + 2^54)."""
    for x1 in (at(1, 0.01 + 0.0021 * j) for j in range(450)):
        if weight(-x1) % 4 != 3:
            continue
        for x2 in (at(2, 0.01 + 0.0021 * j) for j in range(450)):
            b, c = weight(-x1), weight(-x2)
            if c % 4 == 3 and (float(c) + float(b)) + 2.0 ** 54 < float(c) + (float(b) + 2.0 ** 54):
                row = [0.0] * 2048 + [x1, x2]
                need = int((float(c) + float(b)) + 2.0 ** 54) + int(float(c) + (float(b) + 2.0 ** 54)) - (2 ** 54 + b + c)
                for number in range(20, 1000, 7):
                    x = at(number, 0.5)
                    row += [x] * (need // weight(-x))
                    need %= weight(-x)
                    if weight(-x) == 1:
                        return row
    raise AssertionError("no such weights")


def first_beyond(sums, target):
    return next(i for i, s in enumerate(sums) if float(s) > target)


@pytest.mark.parametrize("seed", [0, 1])
def test_a_target_between_two_bins_finds_a_token(tj, seed):  # noqa: F811
    """The definition in whole numbers; sums become doubles where they are compared with a share of the whole."""
    x = torch.tensor(row_halved_behind_bin_2())
    x = x[torch.randperm(x.numel(), generator=torch.Generator().manual_seed(seed))]
    order = np.lexsort((np.arange(x.numel()), -x.numpy()))
    w = [weight(-float(v)) for v in x.numpy()[order]]
    sums = np.cumsum(np.array(w, dtype=object))
    total = float(sums[-1])
    tops = torch.tensor([0.5, 0.25, 0.75, float(np.nextafter(np.float32(0.5), np.float32(0))), float(np.nextafter(np.float32(0.5), np.float32(1)))])
    u = torch.tensor([0.0, 0.3, 0.5, 0.99, 1 - 2.0 ** -24])
    rows = lambda n: x[None].expand(n, -1).contiguous().cuda()
    print("sample", x.numel(), flush=True)
    assert tj.sample(rows(5), tops.cuda()).tolist() == [int(order[first_beyond(sums, float(t) * total)]) for t in tops]
    for p in tops.tolist():
        many = 1 + sum(1 for s in sums[:-1] if float(s) < p * total)
        kept = float(sums[many - 1])
        want = [int(order[first_beyond(sums[:many], float(t) * kept)]) for t in u]
        assert tj.sample(rows(5), u.cuda(), top_p=torch.full((5,), p).cuda()).tolist() == want, p
