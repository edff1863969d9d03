"""GPU tests of the operators around the quantized linears (norms, nonlinearities, 8-bit checkpoints, products of single tokens)
against their definitions in 64 bits (block_ops_reference.py)."""
import numpy as np
import pytest
import torch

import block_ops_reference as ref

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
EPS = 1e-5


@pytest.fixture(scope="module")
def tj():
    import paper_2510_27527_amd as tj
    tj.binding.lib()
    return tj


def out_of(tj, t):
    return tj.binding.OUT_BF16 if t == BF else tj.binding.OUT_F32


def draws(seed):
    g = torch.Generator().manual_seed(seed)
    return lambda *shape, std=1.0: torch.randn(shape, generator=g) * std


def activations(normal, rows, cols, t):
    """On the GPU: N(0, 1), some entries 50 times as large, zeros among them."""
    x = normal(rows, cols)
    x = torch.where(normal(rows, cols) > 2.5, x * 50, x)
    return torch.where(normal(rows, cols) > 2.5, torch.zeros(()), x).to(t).cuda()


def spread(t, at, gap):
    """The same matrix in a larger buffer: it starts `at` elements in, its rows are `gap` elements further apart than they are long.  Everything around is
    a sentinel."""
    rows, cols = t.shape
    buf = torch.full((at + rows * (cols + gap) + 64,), -77.0, dtype=t.dtype, device=t.device)
    v = torch.as_strided(buf, (rows, cols), (cols + gap, 1), at)
    v.copy_(t)
    return buf, v


def untouched(buf, v):
    b = buf.clone()
    torch.as_strided(b, v.shape, v.stride(), v.storage_offset()).fill_(-77.0)
    return bool((b == -77.0).all())


# rows that a wave holds, that a workgroup holds, that nothing holds; whole and ragged; the borders between the kernels
ROWS = [1, 7, 8, 120, 128, 129, 511, 512, 513, 768, 1023, 1024, 1025, 2048, 2051, 4096, 4100, 8191, 8192, 8200, 16384, 16391, 20001]


# ------------------------------------------------------------------------------------------------------------ norms ----

@pytest.mark.parametrize("D", ROWS)
@pytest.mark.parametrize("layer", [True, False])
def test_norm(tj, D, layer):
    B = tj.binding
    normal = draws(D * 2 + layer)
    for N, tx, ty, tg in ((1, BF, BF, BF), (9, F32, BF, F32), (70, BF, F32, BF), (33, F32, F32, F32)):
        print("norm", N, D, layer, tx, ty, tg, flush=True)
        x = activations(normal, N, D, tx) + (3.0 if N == 33 else 0.0)
        gamma = (1 + normal(D, std=0.1)).cuda() if N != 9 else None
        beta = normal(D, std=0.1).cuda() if layer and N != 70 else None
        kind = B.NORM_LAYER if layer else B.NORM_RMS
        stats, kept = tj.alloc_stats(N), tj.alloc_ckpt8(N, D)
        y = tj.norm_fwd(x, gamma, beta, eps=EPS, norm=kind, out_dtype=out_of(tj, ty), stats=stats, ckpt=kept)
        (wy, wm, wr), (ey, em, er) = ref.norm_fwd(x, gamma, beta, EPS, layer, ty)
        ref.within(y, wy, ey, "y")
        ref.within(stats[:, :1], wm, em + 1e-38, "mean")
        ref.within(stats[:, 1:], wr, er, "rstd")
        codes, exps, values = ref.ckpt8(x)
        assert np.array_equal(kept.codes.cpu().numpy(), codes) and np.array_equal(kept.exps.cpu().numpy(), exps)
        # without the extras the same bytes
        assert torch.equal(tj.norm_fwd(x, gamma, beta, eps=EPS, norm=kind, out_dtype=out_of(tj, ty)), y)
        dy = normal(N, D, std=1e-3).to(tg).cuda()
        for src, xr in ((x, x), (kept, values)):
            dx, dg, db = tj.norm_bwd(dy, src, stats, gamma, norm=kind, out_dtype=out_of(tj, ty))
            want, bound = ref.norm_bwd(dy, xr, stats, gamma, layer, ty)
            for got, w, b, what in zip((dx, dg, db), want, bound, ("dx", "dgamma", "dbeta")):
                if what == "dbeta" and not layer:
                    assert got is None
                else:
                    ref.within(got, w, b, what)
            alone, _, _ = tj.norm_bwd(dy, src, stats, gamma, norm=kind, out_dtype=out_of(tj, ty), params=False)
            assert torch.equal(alone, dx)


@pytest.mark.parametrize("N,D", [(5000, 1024), (3000, 640), (2500, 2048), (1300, 4096), (1100, 8192), (600, 16384), (530, 17000)])
def test_norm_parameter_gradients_of_many_rows(tj, N, D):
    """More rows than workgroups: every one walks over several, and their partial sums are added in a fixed order."""
    normal = draws(N)
    x = activations(normal, N, D, BF)
    gamma = (1 + normal(D, std=0.1)).cuda()
    dy = normal(N, D, std=1e-3).to(BF).cuda()
    stats = tj.alloc_stats(N)
    tj.norm_fwd(x, gamma, stats=stats)
    dx, dg, db = tj.norm_bwd(dy, x, stats, gamma)
    xd, st, dd = x.double(), stats.double(), dy.double()
    h = (xd - st[:, :1]) * st[:, 1:]
    for got, terms in ((dg, dd * h), (db, dd)):
        ref.within(got, terms.sum(0).cpu(), ((N / 64 + 128) * ref.U * terms.abs().sum(0)).cpu())
    g = dd * gamma.double()
    want = st[:, 1:] * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
    assert float((dx.double() - want).norm() / want.norm()) < 2.0 ** -8
    again = tj.norm_bwd(dy, x, stats, gamma)
    assert all(torch.equal(a, b) for a, b in zip(again, (dx, dg, db)))


def test_norm_gradient_against_differences(tj):
    """The forward call's own differences along random directions, centred, in binary32 on inputs of one sign of curvature."""
    B = tj.binding
    normal = draws(5)
    N, D, t = 6, 200, 2.0 ** -6
    x, gamma, beta = normal(N, D).cuda(), (1 + normal(D, std=0.1)).cuda(), normal(D, std=0.1).cuda()
    dy = normal(N, D).cuda()
    for kind in (B.NORM_LAYER, B.NORM_RMS):
        f = lambda x, g, b: float((tj.norm_fwd(x, g, b, norm=kind, out_dtype=B.OUT_F32).double() * dy.double()).sum())
        stats = tj.alloc_stats(N)
        tj.norm_fwd(x, gamma, beta, norm=kind, out_dtype=B.OUT_F32, stats=stats)
        dx, dg, db = tj.norm_bwd(dy, x, stats, gamma, norm=kind, out_dtype=B.OUT_F32, dbeta=torch.empty(D, device="cuda"))
        vx, vg, vb = normal(N, D).cuda(), normal(D).cuda(), normal(D).cuda()
        for got, hi, lo in (((dx * vx).sum(), (x + t * vx, gamma, beta), (x - t * vx, gamma, beta)),
                            ((dg * vg).sum(), (x, gamma + t * vg, beta), (x, gamma - t * vg, beta)),
                            ((db * vb).sum(), (x, gamma, beta + t * vb), (x, gamma, beta - t * vb))):
            # truncation t^2 / 6 of a third derivative of the size of the sum's terms; rounding U / t of the same
            size = float(dy.norm()) * (1 + float(vx.abs().max()) ** 3)
            assert abs(float(got) - (f(*hi) - f(*lo)) / (2 * t)) <= (t * t + 64 * ref.U / t) * size


@pytest.mark.parametrize("D", [5, 300, 1500, 3000, 18000])
def test_norm_of_odd_values(tj, D):
    """Constant rows, zeros, and what is not finite: it stays in its row."""
    B = tj.binding
    x = torch.randn(6, D, generator=torch.Generator().manual_seed(D)).cuda()
    x[1] = 2.5
    x[2] = 0.0
    x[3, D // 2] = float("nan")
    x[4, D - 1] = float("inf")
    x[5] *= 1e-30
    stats, kept = tj.alloc_stats(6), tj.alloc_ckpt8(6, D)
    y = tj.norm_fwd(x, out_dtype=B.OUT_F32, stats=stats, ckpt=kept)
    assert torch.isnan(y[3]).all() and torch.isnan(y[4]).any() and torch.isfinite(y[[0, 1, 2, 5]]).all()
    (wy, _, _), (ey, _, _) = ref.norm_fwd(x[[0, 1, 2, 5]], None, None, EPS, True, F32)
    ref.within(y[[0, 1, 2, 5]], wy, ey)
    assert not y[2].any()
    codes, exps, _ = ref.ckpt8(x)
    assert np.array_equal(kept.codes.cpu().numpy(), codes) and np.array_equal(kept.exps.cpu().numpy(), exps)
    dy = torch.ones(6, D, device="cuda")
    dx, dg, _ = tj.norm_bwd(dy, kept, stats, out_dtype=B.OUT_F32)
    assert torch.isfinite(dx[[0, 1, 2, 5]]).all() and torch.isnan(dx[3]).all() and torch.isnan(dg).all()


# --------------------------------------------------------------------------------------------------- nonlinearities ----

@pytest.mark.parametrize("F", [1, 7, 8, 127, 128, 129, 768, 1000, 1365, 2752, 4096, 5001])
@pytest.mark.parametrize("swiglu", [True, False])
def test_nonlinearity(tj, F, swiglu):
    B = tj.binding
    act = B.ACT_SWIGLU if swiglu else B.ACT_GELU
    normal = draws(F * 2 + swiglu)
    for N, th, ta, tg in ((1, BF, BF, BF), (5, F32, BF, F32), (37, BF, F32, BF), (12, F32, F32, F32)):
        print("act", N, F, swiglu, th, ta, tg, flush=True)
        h = activations(normal, N, F * (2 if swiglu else 1), th)
        kept = tj.alloc_act_ckpt8(N, F, act)
        a = tj.act_fwd(h, act, out_of(tj, ta), ckpt=kept)
        ref.within(a, *ref.act_fwd(h, swiglu, ta), "a")
        codes, exps, values = ref.ckpt8(h.reshape(-1, F))
        assert np.array_equal(kept.codes.cpu().numpy(), codes) and np.array_equal(kept.exps.cpu().numpy(), exps)
        assert torch.equal(tj.act_fwd(h, act, out_of(tj, ta)), a)
        da = normal(N, F, std=1e-3).to(tg).cuda()
        for src, hr in ((h, h), (kept, values.reshape(h.shape))):
            ref.within(tj.act_bwd(da, src, act, out_of(tj, ta)), *ref.act_bwd(da, hr, swiglu, ta), "dh")


def test_nonlinearity_far_out_and_not_finite(tj):
    """Gates of any size: the limits 0 and x, never a NaN that the input did not have."""
    B = tj.binding
    big = torch.tensor([-3e38, -1e13, -1e4, -300.0, -88.0, -17.0, -16.0, -0.0, 0.0, 16.0, 17.0, 88.0, 300.0, 1e4, 1e13, 3e38]).cuda()
    one = torch.ones_like(big)
    for swiglu in (True, False):
        act = B.ACT_SWIGLU if swiglu else B.ACT_GELU
        h = (torch.cat((big, one)) if swiglu else big)[None]
        a = tj.act_fwd(h, act, B.OUT_F32)[0]
        dh = tj.act_bwd(one[None], h, act, B.OUT_F32)[0]
        assert torch.isfinite(a).all() and torch.isfinite(dh).all()
        assert torch.equal(a[big >= 300], big[big >= 300]) and not a[big <= -300].any()
        assert (dh[:16][big >= 300] == 1).all() and not dh[:16][big <= -300].any()
    for bad in (float("nan"), float("inf"), float("-inf")):
        h = torch.ones(2, 300, device="cuda")
        h[1, 40] = bad
        kept = tj.alloc_act_ckpt8(2, 300, B.ACT_GELU)
        a = tj.act_fwd(h, B.ACT_GELU, B.OUT_F32, ckpt=kept)
        dh = tj.act_bwd(torch.ones(2, 300, device="cuda"), kept, B.ACT_GELU, B.OUT_F32)
        assert torch.isfinite(a[0]).all() and torch.isfinite(dh[0]).all()
        hurt = torch.isnan(dh[1]).nonzero().flatten().tolist()
        assert hurt == [40] and torch.isfinite(a[1, :40]).all() and torch.isfinite(a[1, 41:]).all()


@pytest.mark.parametrize("swiglu", [True, False])
def test_nonlinearity_gradient_against_differences(tj, swiglu):
    B = tj.binding
    act = B.ACT_SWIGLU if swiglu else B.ACT_GELU
    normal = draws(17 + swiglu)
    h, da, v = normal(4, 256).cuda(), normal(4, 128 if swiglu else 256).cuda(), normal(4, 256).cuda()
    t = 2.0 ** -6
    f = lambda h: float((tj.act_fwd(h, act, B.OUT_F32).double() * da.double()).sum())
    got = float((tj.act_bwd(da, h, act, B.OUT_F32).double() * v.double()).sum())
    size = float(da.abs().sum()) * (1 + float(h.abs().max())) * float(v.abs().max()) ** 3
    assert abs(got - (f(h + t * v) - f(h - t * v)) / (2 * t)) <= (t * t / 6 + 64 * ref.U / t) * size


# ---------------------------------------------------------------------------------------------- 8-bit checkpoints ----

@pytest.mark.parametrize("D", [1, 5, 8, 127, 128, 130, 1000, 4099])
@pytest.mark.parametrize("t", [BF, F32])
def test_checkpoint(tj, D, t):
    normal = draws(D)
    x = activations(normal, 11, D, t)
    x[3] *= 2.0 ** -90
    x[4] *= 2.0 ** 90
    x[5] = 0
    x[6] = float("nan")
    x[7, D // 2] = float("-inf")
    kept = tj.ckpt8_save(x)
    codes, exps, values = ref.ckpt8(x)
    assert np.array_equal(kept.codes.cpu().numpy(), codes) and np.array_equal(kept.exps.cpu().numpy(), exps)
    for out in (F32, BF):
        y = tj.ckpt8_load(kept, out_of(tj, out))
        want = values.to(F32).to(out).double()      # exact but in the last bits of subnormal numbers
        got = ref.f64(y)
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))


def test_checkpoint_of_every_rounding(tj):
    """Every code value, every midpoint and the neighbours of both, both signs, at several powers of two; and the extremes of the exponent."""
    table = ref.e4m3_table()
    mid = (table[1:] + table[:-1]) / 2
    v = np.concatenate([table, mid, np.nextafter(mid.astype(np.float32), np.float32(0)), np.nextafter(mid.astype(np.float32), np.float32(1e9))])
    v = np.concatenate([v, -v]).astype(np.float32)
    rows = []
    for i in range(0, len(v), 127):
        part = np.zeros(127, np.float32)
        part[:len(v[i:i + 127])] = v[i:i + 127]
        rows += [np.append(part, np.float32(448.0)) * np.float32(s) for s in (1.0, 2.0 ** -100, 2.0 ** 100, 1.75)]
    rows += [np.full(128, s, np.float32) for s in (3.4028235e38, 2.0 ** -126, 2.0 ** -149, 448.0, 448.0000305, 0.0)]
    x = torch.from_numpy(np.stack(rows)).cuda()
    kept = tj.ckpt8_save(x)
    codes, exps, _ = ref.ckpt8(x)
    assert np.array_equal(kept.exps.cpu().numpy(), exps)
    assert np.array_equal(kept.codes.cpu().numpy(), codes)


# ------------------------------------------------------------------------------------------------------- products ----

def operand(tj, C, K, outer, seed, exact=False):
    """Packed weights made of random bytes; exact: scales that are powers of two, so that sums of products with small integers are exact."""
    B = tj.binding
    g = torch.Generator().manual_seed(seed)
    codes = torch.randint(0, 256, (C, K // 2), generator=g, dtype=torch.uint8).cuda()
    if exact:
        scales = (torch.randint(6, 9, (C, K // 16), generator=g) * 8).to(torch.uint8).cuda()
    else:
        scales = torch.randint(0, 127, (C, K // 16), generator=g, dtype=torch.uint8).cuda()
    shape = (1,) if outer == B.OUTER_TENSOR else (C, K // 128)
    gscale = torch.pow(2.0, torch.randint(-2, 3, shape, generator=g).float()).cuda() if exact else (torch.rand(shape, generator=g) + 0.5).cuda() * 1e-3
    return tj.NVFP4Tensor(codes, scales, gscale, None, C, K, outer)


TOKENS = [1, 2, 3, 4, 5, 8, 9, 16, 17, 31, 32, 33, 48, 64, 65, 130]


@pytest.mark.parametrize("block", [False, True])
@pytest.mark.parametrize("M", TOKENS)
def test_gemv(tj, M, block):
    B = tj.binding
    outer = B.OUTER_BLOCK128 if block else B.OUTER_TENSOR
    normal = draws(M)
    for C, K in ((1, 128), (15, 256), (16, 1024), (77, 640), (200, 2176)) + (() if block else ((33, 16), (18, 48), (130, 1040), (19, 2064))):
        for out in (BF, F32):
            print("gemv", M, C, K, block, out, flush=True)
            W = operand(tj, C, K, outer, C * 7 + K)
            x = activations(normal, M, K, BF)
            y = tj.gemv(x, W, out_of(tj, out))
            ref.within(y, *ref.gemv(x, ref.unpack(W.codes, W.scales, W.gscale, block), out), "y")
            # small integers times weights of few bits: nothing is rounded, so every product is there exactly once
            W = operand(tj, C, K, outer, C * 11 + K, exact=True)
            xi = torch.randint(-3, 4, (M, K), generator=torch.Generator().manual_seed(K)).to(BF).cuda()
            y = tj.gemv(xi, W, B.OUT_F32)
            assert torch.equal(ref.f64(y), ref.f64(xi) @ ref.unpack(W.codes, W.scales, W.gscale, block).t())


def test_gemv_of_the_layers_own_weights(tj):
    """The context that the training layer's forward call leaves, in both outer modes; bit for bit again on a second call."""
    B = tj.binding
    normal = draws(3)
    X, W = normal(256, 512).to(BF).cuda(), normal(384, 512, std=0.02).to(BF).cuda()
    for outer in (B.OUTER_TENSOR, B.OUTER_BLOCK128):
        _, _, Wq = tj.linear_fwd(X, W, outer=outer)
        for M in (1, 3, 20):
            y = tj.gemv(X[:M], Wq, B.OUT_F32)
            ref.within(y, *ref.gemv(X[:M], ref.unpack(Wq.codes, Wq.scales, Wq.gscale, outer == B.OUTER_BLOCK128), F32))
            assert torch.equal(y, tj.gemv(X[:M], Wq, B.OUT_F32))


def test_gemv_keeps_what_is_not_finite_in_its_token(tj):
    B = tj.binding
    W = operand(tj, 40, 512, B.OUTER_TENSOR, 1)
    for M in (2, 6, 40):
        x = torch.ones(M, 512, dtype=BF, device="cuda")
        x[1, 300] = float("nan")
        y = tj.gemv(x, W, B.OUT_F32)
        assert torch.isnan(y[1]).all() and torch.isfinite(y[0]).all() and torch.isfinite(y[2:]).all()


# ------------------------------------------------------------------------------ strides, empties, streams, graphs, size ----

@pytest.mark.parametrize("at,gap", [(0, 8), (1, 0), (3, 5), (8, 1), (2, 30)])
def test_strided_and_unaligned(tj, at, gap):
    """Rows that start anywhere give the bytes that contiguous ones give, and nothing around the outputs is written."""
    B = tj.binding
    normal = draws(at * 31 + gap)
    for N, D in ((5, 200), (3, 1023), (4, 3001)):
        print("strided", at, gap, N, D, flush=True)
        for t in (BF, F32):
            o = out_of(tj, t)
            x, dy, gamma = activations(normal, N, D, t), normal(N, D, std=1e-3).to(t).cuda(), normal(D).cuda()
            xs, dys = spread(x, at, gap)[1], spread(dy, at, gap)[1]
            stats, kept, kept2 = tj.alloc_stats(N), tj.alloc_ckpt8(N, D), tj.alloc_ckpt8(N, D)
            y = tj.norm_fwd(x, gamma, out_dtype=o, stats=stats, ckpt=kept)
            buf, ys = spread(torch.zeros_like(y), at, gap)
            tj.norm_fwd(xs, gamma, out_dtype=o, Y=ys, ckpt=kept2)
            assert torch.equal(ys, y) and untouched(buf, ys) and torch.equal(kept.codes, kept2.codes) and torch.equal(kept.exps, kept2.exps)
            dx, dg, db = tj.norm_bwd(dy, x, stats, gamma, out_dtype=o)
            buf, dxs = spread(torch.zeros_like(dx), at, gap)
            _, dg2, db2 = tj.norm_bwd(dys, xs, stats, gamma, out_dtype=o, dX=dxs)
            assert torch.equal(dxs, dx) and untouched(buf, dxs) and torch.equal(dg, dg2) and torch.equal(db, db2)
            for act in (B.ACT_SWIGLU, B.ACT_GELU):
                h = activations(normal, N, D * (2 if act == B.ACT_SWIGLU else 1), t)
                hs = spread(h, at, gap)[1]
                a = tj.act_fwd(h, act, o)
                buf, as_ = spread(torch.zeros_like(a), at, gap)
                tj.act_fwd(hs, act, o, A=as_)
                assert torch.equal(as_, a) and untouched(buf, as_)
                dh = tj.act_bwd(dy, h, act, o)
                buf, dhs = spread(torch.zeros_like(dh), at, gap)
                tj.act_bwd(dys, hs, act, o, dH=dhs)
                assert torch.equal(dhs, dh) and untouched(buf, dhs)
            k1, k2 = tj.ckpt8_save(x), tj.ckpt8_save(xs)
            assert torch.equal(k1.codes, k2.codes) and torch.equal(k1.exps, k2.exps)
            buf, ys = spread(torch.zeros_like(x), at, gap)
            tj.ckpt8_load(k1, o, Y=ys)
            assert torch.equal(ys, tj.ckpt8_load(k1, o)) and untouched(buf, ys)
    for M in (1, 3, 9, 33):
        W = operand(tj, 51, 400, B.OUTER_TENSOR, M)
        x = activations(normal, M, 400, BF)
        xs = spread(x, at, gap)[1]
        for t in (BF, F32):
            y = tj.gemv(x, W, out_of(tj, t))
            buf, ys = spread(torch.zeros_like(y), at, gap)
            tj.gemv(xs, W, out_of(tj, t), Y=ys)
            assert torch.equal(ys, y) and untouched(buf, ys)


# calls of under 8 MB, of more, of more than half the last-level cache: what a row gives does not depend on the rows around it
@pytest.mark.parametrize("N,F", [(1601, 1999), (30011, 1543)])
@pytest.mark.parametrize("swiglu", [True, False])
def test_rows_do_not_depend_on_the_size_of_a_call(tj, N, F, swiglu):
    B = tj.binding
    act, parts = (B.ACT_SWIGLU, 2) if swiglu else (B.ACT_GELU, 1)
    g = torch.Generator(device="cuda").manual_seed(N)
    H = torch.randn(N, parts * F, generator=g, device="cuda").to(BF)
    dA = torch.randn(N, F, generator=g, device="cuda").to(BF)
    kept = tj.alloc_act_ckpt8(N, F, act)
    A = tj.act_fwd(H, act, ckpt=kept)
    dH, dH8 = tj.act_bwd(dA, H, act), tj.act_bwd(dA, kept, act)
    saved = tj.ckpt8_save(H)
    loaded = tj.ckpt8_load(saved)
    for at in (0, N // 2, N - 200):
        rows = slice(at, at + 200)
        h, da = H[rows].contiguous(), dA[rows].contiguous()
        k = tj.alloc_act_ckpt8(200, F, act)
        assert torch.equal(tj.act_fwd(h, act, ckpt=k), A[rows])
        both = slice(at * parts, (at + 200) * parts)
        assert torch.equal(k.codes, kept.codes[both]) and torch.equal(k.exps, kept.exps[both])
        assert torch.equal(tj.act_bwd(da, h, act), dH[rows]) and torch.equal(tj.act_bwd(da, k, act), dH8[rows])
        s = tj.ckpt8_save(h)
        assert torch.equal(s.codes, saved.codes[rows]) and torch.equal(s.exps, saved.exps[rows])
        assert torch.equal(tj.ckpt8_load(s), loaded[rows])


@pytest.mark.parametrize("D", [500, 1023, 2047, 4096, 8191, 16384])
def test_norm_rows_do_not_depend_on_the_size_of_a_call(tj, D):
    N = (144 << 20) // (5 * D)
    g = torch.Generator(device="cuda").manual_seed(D)
    x, dy = torch.randn(N, D, generator=g, device="cuda").to(BF), torch.randn(N, D, generator=g, device="cuda").to(BF)
    gamma, beta = torch.randn(D, generator=g, device="cuda"), torch.randn(D, generator=g, device="cuda")
    stats, kept = tj.alloc_stats(N), tj.alloc_ckpt8(N, D)
    y = tj.norm_fwd(x, gamma, beta, stats=stats, ckpt=kept)
    dx, dx8 = tj.norm_bwd(dy, x, stats, gamma)[0], tj.norm_bwd(dy, kept, stats, gamma)[0]
    for at in (0, N // 2, N - 100):
        rows = slice(at, at + 100)
        s, k = tj.alloc_stats(100), tj.alloc_ckpt8(100, D)
        h, d = x[rows].contiguous(), dy[rows].contiguous()
        assert torch.equal(tj.norm_fwd(h, gamma, beta, stats=s, ckpt=k), y[rows])
        assert torch.equal(s, stats[rows]) and torch.equal(k.codes, kept.codes[rows]) and torch.equal(k.exps, kept.exps[rows])
        assert torch.equal(tj.norm_bwd(d, h, s, gamma)[0], dx[rows]) and torch.equal(tj.norm_bwd(d, k, s, gamma)[0], dx8[rows])


def test_checkpoints_write_nothing_past_their_ends(tj):
    """Buffers cut out of larger ones: every byte around stays."""
    for N, D in ((3, 130), (2, 7), (5, 1023)):
        groups = -(-D // 128)
        big = torch.full((N * D + N * groups + 96,), 0xA5, dtype=torch.uint8, device="cuda")
        codes, exps = big[33:33 + N * D].view(N, D), big[33 + N * D + 30:33 + N * D + 30 + N * groups].view(N, groups)
        kept = tj.Ckpt8(codes, exps, N, D)
        x = torch.randn(N, D, device="cuda")
        tj.ckpt8_save(x, kept)
        want = tj.ckpt8_save(x)
        assert torch.equal(codes, want.codes) and torch.equal(exps, want.exps)
        assert (big[:33] == 0xA5).all() and (big[33 + N * D:63 + N * D] == 0xA5).all() and (big[63 + N * D + N * groups:] == 0xA5).all()


def test_empty(tj):
    B = tj.binding
    for N, D in ((0, 64), (3, 0), (0, 0)):
        x = torch.empty(N, D, dtype=BF, device="cuda")
        stats, kept = tj.alloc_stats(N), tj.alloc_ckpt8(N, D)
        assert tj.norm_fwd(x, stats=stats, ckpt=kept).shape == (N, D)
        dx, dg, db = tj.norm_bwd(x, x, stats, dgamma=torch.ones(D, device="cuda"), dbeta=torch.ones(D, device="cuda"))
        assert dx.shape == (N, D) and not dg.any() and not db.any()
        assert tj.act_fwd(x, B.ACT_GELU).shape == (N, D) and tj.act_bwd(x, x, B.ACT_GELU).shape == (N, D)
        assert tj.ckpt8_load(tj.ckpt8_save(x)).shape == (N, D)
    W = operand(tj, 9, 32, B.OUTER_TENSOR, 0)
    assert tj.gemv(torch.empty(0, 32, dtype=BF, device="cuda"), W).shape == (0, 9)
    y = tj.gemv(torch.empty(2, 0, dtype=BF, device="cuda"), tj.alloc_nvfp4(5, 0), B.OUT_F32, Y=torch.ones(2, 5, device="cuda"))
    assert not y.any()
    assert tj.gemv(torch.ones(2, 32, dtype=BF, device="cuda"), tj.alloc_nvfp4(0, 32)).shape == (2, 0)
    torch.cuda.synchronize()


def step(tj, t):
    """One pass through every operator on the tensors of `t`, into its own outputs."""
    B = tj.binding
    tj.norm_fwd(t["x"], t["gamma"], Y=t["y"], stats=t["stats"], ckpt=t["kept"])
    tj.norm_bwd(t["dy"], t["kept"], t["stats"], t["gamma"], dX=t["dx"], dgamma=t["dg"], dbeta=t["db"], ws=t["ws"])
    tj.act_fwd(t["y"], B.ACT_SWIGLU, A=t["a"], ckpt=t["hkept"])
    tj.act_bwd(t["a"], t["hkept"], B.ACT_SWIGLU, dH=t["dh"])
    tj.gemv(t["y"][:3], t["W"], Y=t["z"])


def buffers(tj, seed):
    B = tj.binding
    N, D = 700, 1024
    normal = draws(seed)
    e = lambda *s, dtype=BF: torch.empty(s, dtype=dtype, device="cuda")
    return dict(x=activations(normal, N, D, BF), gamma=normal(D).cuda(), dy=normal(N, D).to(BF).cuda(), y=e(N, D), stats=tj.alloc_stats(N), kept=tj.alloc_ckpt8(N, D),
                dx=e(N, D), dg=e(D, dtype=F32), db=e(D, dtype=F32), ws=tj.alloc_workspace(B.lib().nvfp4_norm_workspace_bytes(N, D)), a=e(N, D // 2),
                hkept=tj.alloc_act_ckpt8(N, D // 2, B.ACT_SWIGLU), dh=e(N, D), W=operand(tj, 600, D, B.OUTER_TENSOR, seed), z=e(3, 600))


OUTPUTS = ("y", "dx", "dg", "db", "a", "dh", "z")


def test_on_another_stream_and_in_a_graph(tj):
    t = buffers(tj, 1)
    step(tj, t)
    torch.cuda.synchronize()
    want = {k: t[k].clone() for k in OUTPUTS}
    s = torch.cuda.Stream()
    for k in OUTPUTS:
        t[k].zero_()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step(tj, t)
    s.synchronize()
    assert all(torch.equal(t[k], want[k]) for k in OUTPUTS)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(tj, t)
    other = buffers(tj, 2)
    first = t["x"].clone()
    for i in range(4):                 # inputs change between the replays, and eager work runs there
        src = first if i % 2 else other["x"]
        t["x"].copy_(src)
        for k in OUTPUTS:
            t[k].zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = {k: t[k].clone() for k in OUTPUTS}
        step(tj, t)
        torch.cuda.synchronize()
        assert all(torch.equal(t[k], got[k]) for k in OUTPUTS), i
        if i % 2:
            assert all(torch.equal(got[k], want[k]) for k in OUTPUTS), i


def test_offsets_past_32_bits(tj):
    """Rows 2^30 elements apart, and contiguous arrays of more than 2^32 elements: the last rows are as right as the first."""
    B = tj.binding
    normal = draws(9)
    N, D, ld = 5, 300, 1 << 30
    buf = torch.empty((N - 1) * ld + D, dtype=BF, device="cuda")
    out = torch.empty((N - 1) * ld + 2 * D, dtype=BF, device="cuda")
    x = activations(normal, N, D, BF)
    xs, ys = torch.as_strided(buf, (N, D), (ld, 1)), torch.as_strided(out, (N, D), (ld, 1))
    xs.copy_(x)
    stats = tj.alloc_stats(N)
    want = tj.norm_fwd(x, stats=stats)
    tj.norm_fwd(xs, Y=ys)
    assert torch.equal(ys, want)
    tj.norm_bwd(xs, xs, stats, dX=ys)
    assert torch.equal(ys, tj.norm_bwd(x, x, stats)[0])
    tj.act_fwd(xs, B.ACT_GELU, A=ys)
    assert torch.equal(ys, tj.act_fwd(x, B.ACT_GELU))
    tj.act_bwd(xs, xs, B.ACT_GELU, dH=ys)
    assert torch.equal(ys, tj.act_bwd(x, x, B.ACT_GELU))
    W = operand(tj, 300, 288, B.OUTER_TENSOR, 4)
    tj.gemv(xs[:, :288], W, Y=ys)
    assert torch.equal(ys, tj.gemv(x[:, :288].contiguous(), W))
    del buf, out, xs, ys
    rows, K = 67000, 1 << 16                       # 4.4e9 elements: codes past 4 GiB
    x = torch.zeros(rows, K, dtype=BF, device="cuda")
    x[-3:] = activations(normal, 3, K, BF)
    kept = tj.ckpt8_save(x)
    tail = tj.ckpt8_save(x[-3:])
    assert torch.equal(kept.codes[-3:], tail.codes) and torch.equal(kept.exps[-3:], tail.exps) and not kept.codes[:-3].any()
    y = tj.ckpt8_load(kept)
    assert torch.equal(y[-3:], tj.ckpt8_load(tail)) and not y[:-3].any()
    del y, kept
    W = tj.NVFP4Tensor(torch.zeros(131072, K // 2, dtype=torch.uint8, device="cuda"), torch.full((131072, K // 16), 56, dtype=torch.uint8, device="cuda"),
                       torch.ones(1, device="cuda"), None, 131072, K, B.OUTER_TENSOR)      # 2^33 elements, as many as an operand may have: 4 GiB of codes
    small = operand(tj, 20, K, B.OUTER_TENSOR, 6)
    W.codes[-20:] = small.codes
    W.scales[-20:] = small.scales
    small.gscale.fill_(1.0)
    for M in (1, 3):
        got, want = tj.gemv(x[-M:], W), tj.gemv(x[-M:], small)
        assert torch.equal(got[:, -20:], want) and not got[:, :-20].any()
