"""GPU tests of the decoder that examples/decoder.py builds from the library's calls, and of the rotation between a quantized linear and its gradients."""
import os
import sys

import pytest
import torch

import block_ops_reference as block
import seq_ops_reference as ref

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

BF = torch.bfloat16


@pytest.fixture(scope="module")
def ex():
    import decoder
    return decoder


class Seen:
    """The part of a batch that the reference of attention asks for: token j of sequence b is row index[b][j] of the keys and values read back."""

    def __init__(self, heads, rows, index, past):
        self.heads, self.rows, self.index, self.past = heads, rows, index, past

    def seen(self, b, i):
        return self.index[b][:self.past[b] + i + 1]


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("shared", [0, 37])
def test_the_stages_of_a_step(ex, bits8, shared):
    """Prompts and then steps of one token each: every stage from what the stage before it gave, attention over what the cache then holds."""
    tj, B = ex.tj, ex.B
    model = ex.Decoder(256, heads=4, kv_heads=2, layers=1, mlp=256, vocabulary=300, pages=40, bits8=bits8)
    layer, D = model.layers[0], model.D
    g = torch.Generator().manual_seed(1)
    prompts = [5, 1, 40]
    seqs = ex.Sequences(40, 3, 60)
    words = lambda n: torch.randint(0, 300, (n,), generator=g).cuda()
    everything = None
    if shared:
        everything = seqs.share(shared)
        model.forward(words(shared), everything)
    past = [0, 0, 0]
    for new in (prompts, [1, 1, 1], [1, 1, 1], [2, 0, 3]):
        batch = seqs.grow(new)
        rows = [(b, i) for b, n in enumerate(new) for i in range(n)]
        x = model.embedding[words(len(rows))]
        out = model.attention(layer, x, batch)
        y = tj.norm_fwd(x, layer["gamma1"], norm=B.NORM_RMS)
        qkv = tj.gemv(y, layer["qkv"])
        block.within(qkv, *block.gemv(y, block.unpack(layer["qkv"].codes, layer["qkv"].scales, layer["qkv"].gscale, False), BF), "qkv")
        q, k, v = qkv.split(model.widths, 1)
        pos = torch.tensor([shared + past[b] + i for b, i in rows])
        want, e = ref.rope(q.reshape(-1, 4, D), pos, model.turn.freqs, False)
        q = tj.kv_append(k, v, layer["cache"], batch, model.turn, Q=q)         # writes what is there already
        block.within(q.view(-1, 4, D), want, e + ref.ROUND[BF] * want.abs() + 1e-38, "q")
        # the cache as attention sees it: all tokens of the prefix and of every sequence, read back
        total = sum(seqs.lens)
        starts = torch.tensor([0] + seqs.lens, dtype=torch.int32).cumsum(0).to(torch.int32).cuda()
        held = [tj.kv_load(layer["cache"], tj.KVBatch(batch.table, batch.lens, starts), total, B.OUT_F32)]
        if shared:
            held.insert(0, tj.kv_load(layer["cache"], everything, shared, B.OUT_F32))
        k, v = (torch.cat([h[j] for h in held]).view(-1, 2, D).double().cpu() for j in (0, 1))
        index, at = [], shared
        for n in seqs.lens:
            index.append(list(range(shared)) + list(range(at, at + n)))
            at += n
        a = tj.attn(q, layer["cache"], batch, 4)
        want, bound = ref.attn(q.view(-1, 4, D), k, v, Seen(2, rows, index, [shared + p for p in past]), D ** -0.5, 4)
        block.within(a.view(-1, 4, D), want, bound, "attention")
        assert torch.equal(out, tj.gemv(a, layer["out"]).add_(x))
        past = [p + n for p, n in zip(past, new)]


def test_answers(ex):
    """The same tokens on every run and for every number in the batch; greedy ones are the largest logits'; a shared beginning in pages of its own gives what it gives in front of each prompt."""
    tj = ex.tj
    model = ex.Decoder(256, heads=4, kv_heads=2, layers=2, mlp=256, vocabulary=300, pages=80)
    g = torch.Generator().manual_seed(2)
    words = lambda n: torch.randint(0, 300, (n,), generator=g).tolist()
    prompts = [words(n) for n in (4, 19, 33)]
    full = lambda v: torch.full((3,), v, device="cuda")
    a = ex.answer(model, [], prompts, 6, temperature=full(0.7), top_p=full(0.8))
    b = ex.answer(model, [], prompts, 6, temperature=full(0.7), top_p=full(0.8))
    assert a.shape == (6, 3) and torch.equal(a, b) and (a >= 0).all() and (a < 300).all()
    shared = words(50)
    seqs = [ex.Sequences(80, 3, 100) for _ in range(2)]
    ints = lambda v: torch.tensor(v).cuda()
    model.forward(ints(shared), seqs[0].share(50))
    x = model.forward(ints(sum(prompts, [])), seqs[0].grow([len(p) for p in prompts]))
    last = ints([len(p) for p in prompts]).cumsum(0) - 1
    # the same tokens without a prefix: the shared ones in front of every prompt
    y = model.forward(ints(sum([shared + p for p in prompts], [])), seqs[1].grow([50 + len(p) for p in prompts]))
    at = ints([50 + len(p) for p in prompts]).cumsum(0) - 1
    logits = [tj.gemv(tj.norm_fwd(h, norm=ex.B.NORM_RMS), model.head, ex.B.OUT_F32) for h in (x[last], y[at])]
    # two computations with some 13 roundings to bf16 a layer that fall differently, each at most 2^-8 of its value and in no common direction: 2 sqrt(26) of them, with a half as much for the values that
    # a residual's addition outgrows
    assert float((logits[0] - logits[1]).norm()) <= 16 * 2.0 ** -8 * float(logits[1].norm())
    greedy = tj.sample(logits[0], full(0.5), temperature=full(0.0))
    assert torch.equal(greedy, logits[0].argmax(1))


def test_a_linear_with_rotated_outputs_is_trained(ex):
    """Y = turn(X W^T): the gradient goes back through the transposed rotation into the linear's backward call."""
    tj, B = ex.tj, ex.B
    N, hidden, H, D = 256, 256, 6, 64
    g = torch.Generator().manual_seed(3)
    X, W = torch.randn(N, hidden, generator=g).to(BF).cuda(), (torch.randn(H * D, hidden, generator=g) * hidden ** -0.5).to(BF).cuda()
    dR = (torch.randn(N, H * D, generator=g) * 1e-3).to(BF).cuda()
    turn = tj.Rope(tj.rope_frequencies(D))
    pos = torch.arange(N, dtype=torch.int32).cuda() % 100
    Y, Xq, Wq = tj.linear_fwd(X, W)
    R = tj.rope(Y, pos, turn, H)
    want, e = ref.rope(Y.view(N, H, D), pos, turn.freqs, False)
    block.within(R.view(N, H, D), want, e + ref.ROUND[BF] * want.abs() + 1e-38, "rotated")
    dY = tj.rope(dR, pos, turn, H, inverse=True)
    want, e = ref.rope(dR.view(N, H, D), pos, turn.freqs, False, inverse=True)
    block.within(dY.view(N, H, D), want, e + ref.ROUND[BF] * want.abs() + 1e-38, "gradient")
    in_place = dR.clone()
    tj.rope(in_place, pos, turn, H, inverse=True, Y=in_place)
    assert torch.equal(in_place, dY)
    dX, dW = tj.linear_bwd(dY, Xq, Wq, 5, 1)
    assert torch.equal(dX, tj.linear_bwd_dx(in_place, Wq, 5, 1)) and torch.equal(dW, tj.linear_bwd_dw(in_place, Xq, 5, 1))
