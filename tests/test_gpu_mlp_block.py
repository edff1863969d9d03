"""GPU tests of the MLP block that examples/mlp_block.py builds from the library's calls."""
import os
import sys

import pytest
import torch

import block_ops_reference as ref

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module")
def ex():
    import mlp_block
    return mlp_block


def inputs(ex, hidden, tokens=256):
    g = torch.Generator().manual_seed(5)
    return torch.randn(tokens, hidden, generator=g).bfloat16().cuda(), (torch.randn(tokens, hidden, generator=g) * 1e-3).bfloat16().cuda()


@pytest.mark.parametrize("swiglu", [True, False])
@pytest.mark.parametrize("layer", [True, False])
@pytest.mark.parametrize("outer", [0, 1])
def test_a_step(ex, swiglu, layer, outer):
    """Every stage from what the stage before it gave: the linears bit for bit (same seeds), the operators around them within their bounds, with
    the gradients taken at the values that the 8-bit checkpoints hold."""
    tj, B = ex.tj, ex.B
    act, norm = B.ACT_SWIGLU if swiglu else B.ACT_GELU, B.NORM_LAYER if layer else B.NORM_RMS
    block = ex.MLPBlock(256, 384, act, norm, outer=outer)
    p = block.params
    x, do = inputs(ex, 256)
    out, saved = block.forward(x)
    dx, grads = block.backward(do, saved, seed=3)
    y = tj.norm_fwd(x, p["gamma"], p.get("beta"), norm=norm)
    (wy, _, _), (ey, _, _) = ref.norm_fwd(x, p["gamma"], p.get("beta"), 1e-5, layer, torch.bfloat16)
    ref.within(y, wy, ey, "norm")
    h, Xq, Wq = tj.linear_fwd(y, p["up"].bfloat16(), outer=outer)
    assert torch.equal(Xq.codes, saved.up[0].codes) and torch.equal(Wq.codes, saved.up[1].codes)
    a = tj.act_fwd(h, act)
    ref.within(a, *ref.act_fwd(h, swiglu, torch.bfloat16), "nonlinearity")
    o, *down = tj.linear_fwd(a, p["down"].bfloat16(), outer=outer)
    assert torch.equal(down[0].codes, saved.down[0].codes) and torch.equal(out, o + x)

    da, d_down = tj.linear_bwd(do, *down, 3, 1)
    assert torch.equal(grads["down"], d_down)
    dh = tj.act_bwd(da, saved.h, act)
    ref.within(dh, *ref.act_bwd(da, ref.ckpt8(h.reshape(-1, 384))[2].reshape(h.shape), swiglu, torch.bfloat16), "dh")
    dy, d_up = tj.linear_bwd(dh, Xq, Wq, 3, 0)
    assert torch.equal(grads["up"], d_up)
    wants, bounds = ref.norm_bwd(dy, ref.ckpt8(x)[2], saved.stats, p["gamma"], layer, torch.bfloat16)
    ref.within(grads["gamma"], wants[1], bounds[1], "dgamma")
    if layer:
        ref.within(grads["beta"], wants[2], bounds[2], "dbeta")
    assert set(grads) == set(p)
    inner, _, _ = tj.norm_bwd(dy, saved.x, saved.stats, p["gamma"], norm=norm)
    ref.within(inner, wants[0], bounds[0], "dx")
    assert torch.equal(dx, inner + do)


def test_what_8_bits_change(ex):
    """Same draws of the stochastic rounding, checkpoints on and off: the output and the last linear's gradient do not see the checkpoints, the
    others do.  Of bf16 inputs a checkpoint holds half; the 4-bit contexts of the linears are there either way."""
    x, do = inputs(ex, 256)
    runs = {}
    for bits8 in (True, False):
        block = ex.MLPBlock(256, 384, bits8=bits8)
        out, saved = block.forward(x)
        runs[bits8] = (out, *block.backward(do, saved, seed=3), saved.bytes())
    (o8, dx8, g8, m8), (o, dx, g, m) = runs[True], runs[False]
    assert torch.equal(o8, o) and torch.equal(g8["down"], g["down"])
    assert not torch.equal(dx8, dx) and not torch.equal(g8["up"], g["up"]) and not torch.equal(g8["gamma"], g["gamma"])
    inputs_bytes = x.numel() * 2 + 256 * 2 * 384 * 2
    assert m - m8 == inputs_bytes // 2 - (256 * 2 + 512 * 3)       # the exponents: one byte per 128 elements


def test_training_and_answers(ex):
    """The loss falls; answers are the block's definition on the packed weights, within the roundings of its five calls."""
    block = ex.MLPBlock(512, 1024)
    x, _ = inputs(ex, 512, 2048)
    target = x.float() + 0.5 * torch.roll(x.float(), 1, 1)
    losses = ex.train(block, x, target, 30, 3e-3)
    assert losses[-1] < 0.5 * losses[0]
    up, down = (ref.unpack(w.codes, w.scales, w.gscale, False) for w in block.packed)
    xd = x.double().cpu()
    bf = lambda t: t.bfloat16().double()
    for M in (1, 2, 5, 20):
        v = xd[:M]
        y = bf(v * (v.square().mean(1, keepdim=True) + 1e-5).rsqrt() * block.params["gamma"].double().cpu())
        g, u = bf(y @ up.t()).chunk(2, 1)
        want = bf(bf(g * torch.sigmoid(g) * u) @ down.t()) + v
        got = block.answer(x[:M])
        assert float((got.double().cpu() - want).norm() / want.norm()) < 2.0 ** -7       # five roundings of 2^-9 each
