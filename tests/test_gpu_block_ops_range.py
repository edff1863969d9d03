"""GPU tests of the operators around the quantized linears at the ends of their ranges, against their definitions in 64 bits
(block_ops_reference.py): more rows than workgroups, values whose products in another order would overflow, wide outputs."""
import pytest
import torch

import block_ops_reference as ref
from test_gpu_block_ops import BF, EPS, operand, spread, tj, untouched  # noqa: F401  (tj: the fixture)

pytestmark = pytest.mark.gpu


# Rows that a workgroup of several waves holds, and rows that it reads again: whole and ragged, each beyond the workgroups of a launch (1024, 512, 256
# and 8192 of them), so that a workgroup sums one row after another.
@pytest.mark.parametrize("N,D", [(2600, 2056), (2500, 4096), (1300, 4104), (1200, 8191), (700, 8200), (900, 16384), (16500, 3), (8300, 16390)])
@pytest.mark.parametrize("layer", [True, False])
def test_norm_of_more_rows_than_workgroups(tj, N, D, layer):  # noqa: F811
    B = tj.binding
    kind = B.NORM_LAYER if layer else B.NORM_RMS
    g = torch.Generator(device="cuda").manual_seed(D)
    # rows of very different size: another row's sum in the place of a row's own would show at once
    x = (torch.randn(N, D, generator=g, device="cuda") * torch.exp2(torch.randint(-8, 9, (N, 1), generator=g, device="cuda").float())).to(BF)
    gamma = 1 + 0.1 * torch.randn(D, generator=g, device="cuda")
    stats, kept = tj.alloc_stats(N), tj.alloc_ckpt8(N, D)
    print("norm", N, D, layer, flush=True)
    y = tj.norm_fwd(x, gamma, eps=EPS, norm=kind, stats=stats, ckpt=kept)
    alone = tj.norm_fwd(x, gamma, eps=EPS, norm=kind)
    assert torch.equal(alone, y)
    step = 200
    for at in range(0, N, step):
        rows = slice(at, min(at + step, N))
        n = rows.stop - at
        s, k = tj.alloc_stats(n), tj.alloc_ckpt8(n, D)
        assert torch.equal(tj.norm_fwd(x[rows], gamma, eps=EPS, norm=kind, stats=s, ckpt=k), y[rows]), at
        assert torch.equal(s, stats[rows]) and torch.equal(k.codes, kept.codes[rows]) and torch.equal(k.exps, kept.exps[rows]), at
    last = slice(N - 20, N)
    (wy, wm, wr), (ey, em, er) = ref.norm_fwd(x[last], gamma, None, EPS, layer, BF)
    ref.within(y[last], wy, ey, "y")
    ref.within(stats[last, :1], wm, em + 1e-38, "mean")
    ref.within(stats[last, 1:], wr, er, "rstd")


# Widths of which no kernel has all columns, D * (1 / D) = 1 in binary32; and rows that end in the middle of what a workgroup takes at once
@pytest.mark.parametrize("N,D", [(4, 9), (4, 100), (4, 520), (4, 1100), (4, 1600), (4, 3000), (4, 5000), (4, 9000), (4, 20000), (1025, 4096), (600, 8192), (300, 3000), (300, 1000)])
def test_norm_backward_of_rows_far_from_zero(tj, N, D):  # noqa: F811
    """Rows of one large power of two: the mean is exact, the deviation zero, and mean / deviation overflows.  No term of a gradient has it."""
    B = tj.binding
    import numpy as np
    assert np.float32(D) * (np.float32(1) / np.float32(D)) == 1
    g = torch.Generator(device="cuda").manual_seed(D)
    x = torch.full((N, D), 2.0 ** 110, device="cuda")
    dy = torch.randn(N, D, generator=g, device="cuda")
    gamma = 1 + 0.1 * torch.randn(D, generator=g, device="cuda")
    stats = tj.alloc_stats(N)
    y = tj.norm_fwd(x, gamma, eps=1e-12, out_dtype=B.OUT_F32, stats=stats)
    assert not y.any() and (stats[:, 0] == 2.0 ** 110).all() and ((stats[:, 1] - 1e6).abs() <= 1).all()
    for src in (x, x.to(BF), tj.ckpt8_save(x)):
        got = tj.norm_bwd(dy, src, stats, gamma, out_dtype=B.OUT_F32)
        want, bound = ref.norm_bwd(dy, x, stats, gamma, True, torch.float32)
        for a, w, b, what in zip(got, want, bound, ("dx", "dgamma", "dbeta")):
            ref.within(a, w, b, what)


@pytest.mark.parametrize("size", [1.0, 1e9, 1e30])
@pytest.mark.parametrize("t", [BF, torch.float32])
def test_nonlinearity_backward_of_large_gradients(tj, t, size):  # noqa: F811
    """Gates of any size with large gradients and up values: wherever a gradient is a binary32 number it comes out, whatever its factors' other products are."""
    B = tj.binding
    gates = torch.tensor([-3e38, -1e30, -1e13, -300.0, -100.0, -50.0, -17.0, -1.0, 0.0, 1.0, 17.0, 300.0, 1e6])
    ups = torch.tensor([-1e9, -1e5, 1.0, 1e12])
    g, u = (v.flatten() for v in torch.meshgrid(gates, ups, indexing="ij"))
    h = torch.cat((g, u))[None].to(t).cuda()
    da = torch.full((1, g.numel()), size, device="cuda")
    for act, x in ((B.ACT_SWIGLU, h), (B.ACT_GELU, h[:, :g.numel()].contiguous())):
        want, bound = ref.act_bwd(da, x, act == B.ACT_SWIGLU, torch.float32)
        got = tj.act_bwd(da, x, act, B.OUT_F32)
        fits = (want.abs() < 3e38) & torch.isfinite(want)      # in 64 bits the cube of GELU's argument overflows far out
        ref.within(got.cpu()[fits], want[fits], bound[fits], "dh")


def test_the_stream_of_a_call(tj):  # noqa: F811
    """The one that is current, on the default stream and beside it."""
    assert tj.binding._stream() == torch.cuda.current_stream().cuda_stream
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        assert tj.binding._stream() == side.cuda_stream != 0
    assert tj.binding._stream() == torch.cuda.current_stream().cuda_stream


def calls(tj, t):  # noqa: F811
    """Every call on the tensors of `t`, by what it reads and writes."""
    B = tj.binding
    return {
        "x y gamma beta stats kept": lambda: tj.norm_fwd(t["x"], t["gamma"], t["beta"], Y=t["y"], stats=t["stats"], ckpt=t["kept"]),
        "y x gamma stats dx dg db ws": lambda: tj.norm_bwd(t["y"], t["x"], t["stats"], t["gamma"], dX=t["dx"], dgamma=t["dg"], dbeta=t["db"], ws=t["ws"]),
        "y kept stats": lambda: tj.norm_bwd(t["y"], t["kept"], t["stats"]),
        "x y kept": lambda: tj.act_fwd(t["x"], B.ACT_GELU, A=t["y"], ckpt=t["kept"]),
        "y x dx": lambda: tj.act_bwd(t["y"], t["x"], B.ACT_GELU, dH=t["dx"]),
        "y kept dx": lambda: tj.act_bwd(t["y"], t["kept"], B.ACT_GELU, dH=t["dx"]),
        "x kept ": lambda: tj.ckpt8_save(t["x"], t["kept"]),
        "kept y": lambda: tj.ckpt8_load(t["kept"], Y=t["y"]),
        "x W z": lambda: tj.gemv(t["x"], t["W"], Y=t["z"]),
    }


def test_refuses_tensors_of_another_device(tj, monkeypatch):  # noqa: F811
    """Every tensor of every call has to be where the call is enqueued; one in the host's memory stands for those that are not."""
    B = tj.binding
    N, D, Co = 6, 256, 40
    e = lambda *s, dtype=BF: torch.zeros(s, dtype=dtype, device="cuda")
    t = dict(x=e(N, D), y=e(N, D), dx=e(N, D), z=e(N, Co), gamma=e(D, dtype=torch.float32), beta=e(D, dtype=torch.float32), dg=e(D, dtype=torch.float32), db=e(D, dtype=torch.float32),
             stats=tj.alloc_stats(N), kept=tj.alloc_ckpt8(N, D), ws=tj.alloc_workspace(1 << 20), W=tj.alloc_nvfp4(Co, D))
    t["kept"].codes.zero_(), t["kept"].exps.fill_(127), t["W"].codes.zero_(), t["W"].scales.zero_(), t["W"].gscale.zero_(), t["stats"].zero_()
    for call in calls(tj, t).values():
        call()
    torch.cuda.synchronize()
    for names in calls(tj, t):
        for name in names.split():
            v = t[name]
            if isinstance(v, torch.Tensor):
                moved = [v.cpu()]
            else:
                fields = [f for f in ("codes", "exps", "scales", "gscale") if hasattr(v, f)]
                moved = [type(v)(**{**vars(v), f: getattr(v, f).cpu()}) for f in fields]
            for m in moved:
                with pytest.raises(AssertionError, match="current device"):
                    calls(tj, {**t, name: m})[names]()
    elsewhere = B._current_device() + 1
    monkeypatch.setattr(B, "_current_device", lambda: elsewhere)
    for call in calls(tj, t).values():
        with pytest.raises(AssertionError, match="current device"):
            call()


# Products where a lane takes four rows (one or two tokens; 8192, 16384 or 32768 outputs on by the length of the reduction) and where a workgroup takes two tiles of rows (more
# tokens; 8177 outputs on), whole and ragged, with every number of waves that shares a reduction; and the borders below them.
@pytest.mark.parametrize("block", [False, True])
@pytest.mark.parametrize("C", [4096, 4097, 8176, 8177, 8192, 8193, 16387, 32771])
def test_gemv_of_wide_outputs(tj, C, block):  # noqa: F811
    B = tj.binding
    outer = B.OUTER_BLOCK128 if block else B.OUTER_TENSOR
    for K in (128, 384, 640, 1024, 1280, 2176) + (() if block else (16, 400, 2064)):
        W = operand(tj, C, K, outer, C + K, exact=True)
        w = ref.unpack(W.codes, W.scales, W.gscale, block).cuda().t().contiguous()
        for M in (1, 2, 3, 16, 17, 33):
            print("gemv", M, C, K, block, flush=True)
            # small integers times weights of few bits: nothing is rounded, so every product is there exactly once
            x = torch.randint(-3, 4, (M, K), generator=torch.Generator().manual_seed(M * K)).to(BF).cuda()
            buf, y = spread(torch.zeros(M, C, device="cuda"), 3, 5)
            tj.gemv(x, W, B.OUT_F32, Y=y)
            want = x.double() @ w
            assert torch.equal(y.double(), want) and untouched(buf, y)
            assert torch.equal(tj.gemv(x, W), want.to(BF))


@pytest.mark.parametrize("M", [1, 2, 3, 20])
def test_gemv_of_long_reductions(tj, M):  # noqa: F811
    """Reductions of every length modulo the waves that share one, a rest of 16 at the end among them."""
    B = tj.binding
    for C, K in ((70, 4112), (70, 8208), (8200, 4112), (33, 16400)):
        W = operand(tj, C, K, B.OUTER_TENSOR, C + K, exact=True)
        x = torch.randint(-3, 4, (M, K), generator=torch.Generator().manual_seed(K)).to(BF).cuda()
        want = x.double() @ ref.unpack(W.codes, W.scales, W.gscale, False).cuda().t().contiguous()
        print("gemv", M, C, K, flush=True)
        assert torch.equal(tj.gemv(x, W, B.OUT_F32).double(), want)


@pytest.mark.parametrize("parts", [1, 2])
def test_more_rows_than_a_launch_has(tj, parts):  # noqa: F811
    """Narrow rows by the million: a workgroup walks over several lots of them (beyond 65535 x 16 rows, twice that where a thread takes two)."""
    B = tj.binding
    act = B.ACT_SWIGLU if parts == 2 else B.ACT_GELU
    N, F = 2 * 65535 * 16 + 1001, 8
    g = torch.Generator(device="cuda").manual_seed(parts)
    H = torch.randn(N, parts * F, generator=g, device="cuda").to(BF)
    dA = torch.randn(N, F, generator=g, device="cuda").to(BF)
    kept = tj.alloc_act_ckpt8(N, F, act)
    A = tj.act_fwd(H, act, ckpt=kept)
    dH, dH8 = tj.act_bwd(dA, H, act), tj.act_bwd(dA, kept, act)
    saved = tj.ckpt8_save(H)
    loaded = tj.ckpt8_load(saved)
    for at in list(range(0, N, 100000)) + [N - 3]:
        rows = slice(at, min(at + 100000, N))
        n = rows.stop - at
        h, da, both = H[rows], dA[rows], slice(at * parts, rows.stop * parts)
        k = tj.alloc_act_ckpt8(n, F, act)
        assert torch.equal(tj.act_fwd(h, act, ckpt=k), A[rows]), at
        assert torch.equal(k.codes, kept.codes[both]) and torch.equal(k.exps, kept.exps[both]), at
        assert torch.equal(tj.act_bwd(da, h, act), dH[rows]) and torch.equal(tj.act_bwd(da, k, act), dH8[rows]), at
        s = tj.ckpt8_save(h)
        assert torch.equal(s.codes, saved.codes[rows]) and torch.equal(s.exps, saved.exps[rows]) and torch.equal(tj.ckpt8_load(s), loaded[rows]), at
    last = slice(N - 50, N)
    ref.within(A[last], *ref.act_fwd(H[last], parts == 2, BF), "a")
    ref.within(dH[last], *ref.act_bwd(dA[last], H[last], parts == 2, BF), "dh")
