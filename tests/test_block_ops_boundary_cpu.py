"""What the operators around the quantized linears refuse, on the host and before anything is enqueued: no GPU is needed."""
import ctypes as C
import os

import pytest

from paper_2510_27527_amd import binding as B

FAKE = 0x7F0000001000      # a 16-byte aligned, never dereferenced "device pointer"
NULL, SHAPE, ENUM, WORKSPACE, ALIGN, MISMATCH = -1, -2, -3, -4, -5, -6
BIG = 1 << 34              # more elements than an array may have


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2510_27527_amd import build
        build.build(force=True)
    return B.lib()


def ckpt(rows=8, K=64, codes=FAKE, exps=FAKE):
    return B.CCkpt8(codes, exps, rows, K)


def refuses(call, good, cases):
    for code, change in cases:
        assert call(**{**good, **change}) == code, change


def test_norm_fwd_refuses(lib):
    # N = 0 launches nothing, so the good call itself can be made here
    good = dict(X=FAKE, kind=0, ldx=64, N=0, D=64, gamma=FAKE, beta=FAKE, eps=1e-5, norm=0, Y=FAKE, out=0, ldy=64, stats=FAKE, kept=ckpt())

    def call(X, kind, ldx, N, D, gamma, beta, eps, norm, Y, out, ldy, stats, kept):
        return lib.nvfp4_norm_fwd(X, kind, ldx, N, D, gamma, beta, eps, norm, Y, out, ldy, stats, C.byref(kept) if kept else None, None)
    assert call(**good) == 0
    assert call(**{**good, "gamma": None, "beta": None, "stats": None, "kept": None, "eps": 0.0, "norm": 1}) == 0
    refuses(call, good, [
        (NULL, dict(X=None)), (NULL, dict(Y=None)), (NULL, dict(kept=ckpt(codes=None))), (NULL, dict(kept=ckpt(exps=None))),
        (SHAPE, dict(N=-1)), (SHAPE, dict(D=-1)), (SHAPE, dict(N=BIG)), (SHAPE, dict(N=1 << 20, D=1 << 20)), (SHAPE, dict(D=(1 << 22) + 1, ldx=1 << 23, ldy=1 << 23)),
        (SHAPE, dict(ldx=63)), (SHAPE, dict(ldy=0)), (SHAPE, dict(N=1 << 20, ldx=1 << 40)), (SHAPE, dict(ldx=-64)),
        (ENUM, dict(kind=1)), (ENUM, dict(kind=3)), (ENUM, dict(kind=9)), (ENUM, dict(out=2)), (ENUM, dict(norm=2)), (ENUM, dict(eps=-1.0)), (ENUM, dict(eps=float("nan"))),
        (ALIGN, dict(X=FAKE + 1)), (ALIGN, dict(X=FAKE + 2, kind=2)), (ALIGN, dict(Y=FAKE + 2, out=1)), (ALIGN, dict(gamma=FAKE + 4)), (ALIGN, dict(beta=FAKE + 8)), (ALIGN, dict(stats=FAKE + 4))])


def test_norm_bwd_refuses(lib):
    good = dict(dY=FAKE, dkind=0, lddy=64, X=FAKE, kind=0, ldx=64, stats=FAKE, gamma=FAKE, N=8, D=64, norm=0, dX=FAKE, out=0, lddx=64, dg=FAKE, db=FAKE, ws=FAKE, wsb=1 << 30)

    def call(dY, dkind, lddy, X, kind, ldx, stats, gamma, N, D, norm, dX, out, lddx, dg, db, ws, wsb):
        return lib.nvfp4_norm_bwd(dY, dkind, lddy, X if isinstance(X, int) or X is None else C.byref(X), kind, ldx, stats, gamma, N, D, norm, dX, out, lddx, dg, db, ws, wsb, None)
    assert lib.nvfp4_norm_workspace_bytes(8, 64) > 0
    assert call(**{**good, "N": 0, "D": 0, "ws": None, "wsb": 0}) == 0
    assert call(**{**good, "N": 0, "D": 0, "X": ckpt(0, 0), "kind": 3, "ldx": 0, "dg": None, "db": None, "ws": None, "gamma": None}) == 0
    refuses(call, good, [
        (NULL, dict(dY=None)), (NULL, dict(X=None)), (NULL, dict(stats=None)), (NULL, dict(dX=None)), (NULL, dict(X=ckpt(codes=None), kind=3)),
        (SHAPE, dict(N=-1)), (SHAPE, dict(D=-5)), (SHAPE, dict(N=BIG)), (SHAPE, dict(D=(1 << 22) + 1)), (SHAPE, dict(lddy=63)), (SHAPE, dict(ldx=63)), (SHAPE, dict(lddx=63)),
        (ENUM, dict(dkind=3)), (ENUM, dict(dkind=1)), (ENUM, dict(kind=1)), (ENUM, dict(out=5)), (ENUM, dict(norm=-1)),
        (MISMATCH, dict(X=ckpt(9, 64), kind=3)), (MISMATCH, dict(X=ckpt(8, 65), kind=3)),
        (WORKSPACE, dict(ws=None)), (WORKSPACE, dict(wsb=lib.nvfp4_norm_workspace_bytes(8, 64) - 1)),
        (ALIGN, dict(dY=FAKE + 1)), (ALIGN, dict(X=FAKE + 2, kind=2)), (ALIGN, dict(dX=FAKE + 2, out=1)), (ALIGN, dict(gamma=FAKE + 4)), (ALIGN, dict(dg=FAKE + 4)),
        (ALIGN, dict(db=FAKE + 8)), (ALIGN, dict(stats=FAKE + 4)), (ALIGN, dict(ws=FAKE + 8))])


def test_norm_workspace(lib):
    f = lib.nvfp4_norm_workspace_bytes
    assert f(-1, 64) == f(64, -1) == f(0, 64) == f(64, 0) == f(BIG, 2) == f(4, 1 << 23) == 0
    for D in (1, 64, 1000, 1024, 5000, 16384, 100000):
        sizes = [f(N, D) for N in (1, 2, 8, 100, 1000, 20000)]
        assert sizes == sorted(sizes) and sizes[-1] == f(60000, D) and sizes[-1] % (2 * D * 4) == 0


def test_nonlinearity_refuses(lib):
    good = dict(H=FAKE, kind=0, ldh=128, N=0, F=64, act=0, A=FAKE, out=0, lda=64, kept=None)

    def fwd(H, kind, ldh, N, F, act, A, out, lda, kept):
        return lib.nvfp4_act_fwd(H, kind, ldh, N, F, act, A, out, lda, C.byref(kept) if kept else None, None)
    assert fwd(**good) == 0 and fwd(**{**good, "kept": ckpt()}) == 0
    refuses(fwd, good, [
        (NULL, dict(H=None)), (NULL, dict(A=None)), (NULL, dict(kept=ckpt(codes=None))),
        (SHAPE, dict(N=-1)), (SHAPE, dict(F=-1)), (SHAPE, dict(F=1 << 62)), (SHAPE, dict(N=1 << 20, F=1 << 13, ldh=1 << 14, lda=1 << 13)), (SHAPE, dict(ldh=127)), (SHAPE, dict(lda=63)),
        (ENUM, dict(kind=1)), (ENUM, dict(kind=3)), (ENUM, dict(act=2)), (ENUM, dict(out=2)),
        (ALIGN, dict(H=FAKE + 1)), (ALIGN, dict(H=FAKE + 2, kind=2)), (ALIGN, dict(A=FAKE + 2, out=1))])
    good = dict(dA=FAKE, dkind=0, ldda=64, H=FAKE, kind=0, ldh=128, N=0, F=64, act=0, dH=FAKE, out=0, lddh=128)

    def bwd(dA, dkind, ldda, H, kind, ldh, N, F, act, dH, out, lddh):
        return lib.nvfp4_act_bwd(dA, dkind, ldda, H if isinstance(H, int) or H is None else C.byref(H), kind, ldh, N, F, act, dH, out, lddh, None)
    assert bwd(**good) == 0 and bwd(**{**good, "H": ckpt(0, 64), "kind": 3}) == 0
    refuses(bwd, good, [
        (NULL, dict(dA=None)), (NULL, dict(H=None)), (NULL, dict(dH=None)), (NULL, dict(H=ckpt(0, 64, exps=None), kind=3)),
        (SHAPE, dict(N=-1)), (SHAPE, dict(F=1 << 62)), (SHAPE, dict(ldda=63)), (SHAPE, dict(ldh=127)), (SHAPE, dict(lddh=127)),
        (ENUM, dict(dkind=3)), (ENUM, dict(kind=7)), (ENUM, dict(act=-1)), (ENUM, dict(out=3)),
        (MISMATCH, dict(N=4, H=ckpt(4, 64), kind=3)),       # SwiGLU's has two rows a token
        (MISMATCH, dict(N=4, H=ckpt(8, 128), kind=3)), (MISMATCH, dict(N=4, act=1, H=ckpt(8, 64), kind=3)),
        (ALIGN, dict(dA=FAKE + 1)), (ALIGN, dict(H=FAKE + 2, kind=2)), (ALIGN, dict(dH=FAKE + 2, out=1))])


def test_checkpoint_refuses(lib):
    save = lambda X=FAKE, kind=0, ldx=64, N=0, D=64, out=ckpt(): lib.nvfp4_ckpt8_save(X, kind, ldx, N, D, C.byref(out) if out else None, None)
    assert save() == 0
    assert save(X=None) == NULL and save(out=None) == NULL and save(out=ckpt(codes=None)) == NULL
    assert save(N=-1) == SHAPE and save(ldx=63) == SHAPE and save(N=BIG) == SHAPE
    assert save(kind=1) == ENUM and save(kind=3) == ENUM
    assert save(X=FAKE + 1) == ALIGN and save(X=FAKE + 2, kind=2) == ALIGN
    load = lambda src=None, Y=FAKE, out=0, ldy=64: lib.nvfp4_ckpt8_load(C.byref(src or ckpt(0, 64)), Y, out, ldy, None)
    assert load() == 0
    assert lib.nvfp4_ckpt8_load(None, FAKE, 0, 64, None) == NULL and load(Y=None) == NULL and load(src=ckpt(0, 64, exps=None)) == NULL
    assert load(src=ckpt(-1, 64)) == SHAPE and load(src=ckpt(BIG, 64)) == SHAPE and load(ldy=63) == SHAPE
    assert load(out=2) == ENUM and load(Y=FAKE + 1) == ALIGN
    out = ckpt(3, 3)                                        # a saving call states what it saved
    assert save(N=0, D=40, out=out) == 0 and (out.rows, out.K) == (0, 40)


def test_gemv_refuses(lib):
    def tensor(rows=32, K=256, outer=0, codes=FAKE, scales=FAKE, gscale=FAKE):
        return B.CTensor(codes, scales, gscale, None, rows, K, outer, 0)

    def call(X=FAKE, ldx=256, M=0, W=None, Y=FAKE, out=0, ldy=32, null=False):
        return lib.nvfp4_gemv(X, ldx, M, None if null else C.byref(W or tensor()), Y, out, ldy, None)
    assert call() == 0
    assert call(null=True) == NULL and call(X=None) == NULL and call(Y=None) == NULL
    assert call(W=tensor(codes=None)) == NULL and call(W=tensor(scales=None)) == NULL and call(W=tensor(gscale=None)) == NULL
    assert call(M=-1) == SHAPE and call(M=(1 << 20) + 1) == SHAPE and call(ldx=255) == SHAPE and call(ldy=31) == SHAPE
    assert call(W=tensor(K=200)) == SHAPE and call(W=tensor(K=272, outer=1), ldx=272) == SHAPE      # whole groups of 16, whole blocks of 128
    assert call(W=tensor(rows=-1)) == SHAPE and call(W=tensor(rows=(1 << 26) + 1, K=16)) == SHAPE and call(W=tensor(K=(1 << 22) + 16)) == SHAPE
    assert call(W=tensor(rows=1 << 20, K=1 << 14)) == SHAPE
    assert call(W=tensor(outer=2)) == ENUM and call(out=2) == ENUM
    assert call(X=FAKE + 1) == ALIGN and call(Y=FAKE + 2, out=1) == ALIGN
    assert call(W=tensor(codes=FAKE + 8)) == ALIGN and call(W=tensor(scales=FAKE + 1)) == ALIGN and call(W=tensor(gscale=FAKE + 2)) == ALIGN
