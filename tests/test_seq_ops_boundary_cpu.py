"""What the operators on sequences of tokens refuse, on the host and before anything is enqueued: no GPU is needed."""
import ctypes as C
import math
import os

import pytest
import torch

from paper_2510_27527_amd import binding as B

FAKE = 0x7F0000001000      # a 16-byte aligned, never dereferenced "device pointer"
NULL, SHAPE, ENUM, WORKSPACE, ALIGN, MISMATCH = -1, -2, -3, -4, -5, -6
BIG = 1 << 34


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2510_27527_amd import build
        build.build(force=True)
    return B.lib()


def rotation(freqs=FAKE, R=64, form=0, scale=1.0):
    return B._ROTATION.pack(freqs, R, form, scale)


def cache(k=FAKE, v=FAKE, ke=0, ve=0, pages=10, H=2, page=16, D=64, kind=0):
    return B._KVCACHE.pack(k, v, ke, ve, pages, H, page, D, kind, 0)


def batch(table=FAKE, lens=FAKE, starts=0, prefix_table=0, Bn=0, width=4, prefix=0):
    return B._KVBATCH.pack(table, lens, starts, prefix_table, Bn, width, prefix)


BAD_CACHES = [(NULL, dict(k=0)), (NULL, dict(v=0)), (NULL, dict(kind=1)), (NULL, dict(kind=1, ke=FAKE)), (ENUM, dict(kind=2)), (ENUM, dict(kind=-1)), (SHAPE, dict(page=8)), (SHAPE, dict(page=24)),
              (SHAPE, dict(page=1 << 17)), (SHAPE, dict(page=0)), (SHAPE, dict(D=8)), (SHAPE, dict(D=72)), (SHAPE, dict(D=272)), (SHAPE, dict(D=0)), (SHAPE, dict(H=0)), (SHAPE, dict(H=1 << 20)),
              (SHAPE, dict(pages=-1)), (SHAPE, dict(pages=1 << 31)), (SHAPE, dict(pages=1 << 30, H=16, page=256, D=128)), (ALIGN, dict(k=FAKE + 8)), (ALIGN, dict(v=FAKE + 2)),
              (ALIGN, dict(kind=1, ke=FAKE + 8, ve=FAKE)), (ALIGN, dict(kind=1, ke=FAKE, ve=FAKE + 1))]
BAD_BATCHES = [(NULL, dict(table=0)), (NULL, dict(lens=0)), (NULL, dict(prefix=5)), (SHAPE, dict(Bn=-1)), (SHAPE, dict(Bn=1 << 17)), (SHAPE, dict(width=-1)), (SHAPE, dict(width=1 << 28)),
               (SHAPE, dict(prefix=-1)), (SHAPE, dict(prefix=1 << 31, prefix_table=FAKE)), (SHAPE, dict(width=1 << 26, prefix=1 << 30, prefix_table=FAKE)), (ALIGN, dict(table=FAKE + 2)),
               (ALIGN, dict(lens=FAKE + 1)), (ALIGN, dict(starts=FAKE + 2)), (ALIGN, dict(prefix=5, prefix_table=FAKE + 2)), (MISMATCH, dict(Bn=3))]


def test_descriptors_are_the_header_s():
    assert (B._ROTATION.size, B._KVCACHE.size, B._KVBATCH.size) == (24, 72, 56)


def test_rope_refuses(lib):
    good = dict(X=FAKE, kind=0, ldx=128, pos=FAKE, N=0, H=2, D=64, r=rotation(), inverse=0, Y=FAKE, out=0, ldy=128)

    def call(X, kind, ldx, pos, N, H, D, r, inverse, Y, out, ldy):
        return lib.nvfp4_rope(X, kind, ldx, pos, N, H, D, r, inverse, Y, out, ldy, None)
    assert call(**good) == 0 and call(**{**good, "r": rotation(freqs=0, R=0), "N": 0}) == 0 and call(**{**good, "H": 0, "N": 5}) == 0
    for code, change in [(NULL, dict(X=None)), (NULL, dict(Y=None)), (NULL, dict(pos=None)), (NULL, dict(r=None)), (NULL, dict(r=rotation(freqs=0))), (SHAPE, dict(N=-1)), (SHAPE, dict(N=(1 << 24) + 1)),
                         (SHAPE, dict(H=-1)), (SHAPE, dict(D=-1)), (SHAPE, dict(D=4097, ldx=1 << 20, ldy=1 << 20)), (SHAPE, dict(H=1 << 20)), (SHAPE, dict(ldx=127)), (SHAPE, dict(ldy=127)),
                         (SHAPE, dict(r=rotation(R=66))), (SHAPE, dict(r=rotation(R=63))), (SHAPE, dict(r=rotation(R=-2))), (ENUM, dict(r=rotation(form=2))), (ENUM, dict(kind=1)), (ENUM, dict(kind=3)),
                         (ENUM, dict(out=2)), (ALIGN, dict(X=FAKE + 1)), (ALIGN, dict(Y=FAKE + 2, out=1)), (ALIGN, dict(pos=FAKE + 2)), (ALIGN, dict(r=rotation(freqs=FAKE + 2)))]:
        assert call(**{**good, **change}) == code, change


def test_append_and_load_refuse(lib):
    good = dict(Q=FAKE, ldq=256, Hq=4, K=FAKE, ldk=128, V=FAKE, ldv=128, kind=0, N=0, c=cache(), b=batch(), r=rotation(), Qo=FAKE, out=0, ldo=256)

    def call(Q, ldq, Hq, K, ldk, V, ldv, kind, N, c, b, r, Qo, out, ldo):
        return lib.nvfp4_kv_append(Q, ldq, Hq, K, ldk, V, ldv, kind, N, c, b, r, Qo, out, ldo, None)
    assert call(**good) == 0 and call(**{**good, "Q": None, "Qo": None, "r": None}) == 0 and call(**{**good, "c": cache(kind=1, ke=FAKE, ve=FAKE)}) == 0
    assert call(**{**good, "b": batch(starts=FAKE), "N": 9}) == 0          # rows that belong to no sequence
    bad = [(code, dict(c=cache(**ch))) for code, ch in BAD_CACHES] + [(code, dict(b=batch(**ch))) for code, ch in BAD_BATCHES]
    for code, change in bad + [(NULL, dict(c=None)), (NULL, dict(b=None)), (NULL, dict(K=None)), (NULL, dict(V=None)), (NULL, dict(Qo=None)), (SHAPE, dict(N=-1)), (SHAPE, dict(N=BIG)),
                               (SHAPE, dict(ldk=127)), (SHAPE, dict(ldv=127)), (SHAPE, dict(ldq=255)), (SHAPE, dict(ldo=255)), (SHAPE, dict(Hq=-1)), (SHAPE, dict(Hq=1 << 20)),
                               (SHAPE, dict(r=rotation(R=66))), (ENUM, dict(r=rotation(form=-1))), (ENUM, dict(kind=1)), (ENUM, dict(out=3)), (ALIGN, dict(K=FAKE + 1)), (ALIGN, dict(V=FAKE + 2, kind=2)),
                               (ALIGN, dict(Q=FAKE + 1)), (ALIGN, dict(Qo=FAKE + 1))]:
        assert call(**{**good, **change}) == code, change
    good = dict(c=cache(), b=batch(), N=0, K=FAKE, ldk=128, V=FAKE, ldv=128, out=0)

    def load(c, b, N, K, ldk, V, ldv, out):
        return lib.nvfp4_kv_load(c, b, N, K, ldk, V, ldv, out, None)
    assert load(**good) == 0
    bad = [(code, dict(c=cache(**ch))) for code, ch in BAD_CACHES] + [(code, dict(b=batch(**ch))) for code, ch in BAD_BATCHES]
    for code, change in bad + [(NULL, dict(K=None)), (NULL, dict(V=None)), (SHAPE, dict(N=-1)), (SHAPE, dict(ldk=127)), (SHAPE, dict(ldv=0)), (ENUM, dict(out=2)), (ALIGN, dict(K=FAKE + 1)),
                               (ALIGN, dict(V=FAKE + 2, out=1))]:
        assert load(**{**good, **change}) == code, change


def test_attention_refuses(lib):
    good = dict(Q=FAKE, ldq=256, N=0, Hq=4, c=cache(), b=batch(), scale=0.125, Out=FAKE, ldo=256, ws=None, wsb=0)

    def call(Q, ldq, N, Hq, c, b, scale, Out, ldo, ws, wsb):
        return lib.nvfp4_attn(Q, ldq, N, Hq, c, b, scale, Out, ldo, ws, wsb, None)
    assert call(**good) == 0 and call(**{**good, "N": 5, "b": batch(starts=FAKE)}) == 0
    bad = [(code, dict(c=cache(**ch))) for code, ch in BAD_CACHES] + [(code, dict(b=batch(**ch))) for code, ch in BAD_BATCHES]
    for code, change in bad + [(NULL, dict(Q=None)), (NULL, dict(Out=None)), (SHAPE, dict(N=-1)), (SHAPE, dict(N=BIG)), (SHAPE, dict(Hq=0)), (SHAPE, dict(Hq=5)), (SHAPE, dict(Hq=1 << 30)),
                               (SHAPE, dict(ldq=255)), (SHAPE, dict(ldo=255)), (ENUM, dict(scale=0.0)), (ENUM, dict(scale=-1.0)), (ENUM, dict(scale=math.inf)), (ENUM, dict(scale=math.nan)),
                               (ALIGN, dict(Q=FAKE + 1)), (ALIGN, dict(Out=FAKE + 1))]:
        assert call(**{**good, **change}) == code, change
    need = lib.nvfp4_attn_workspace_bytes(2, 4, 2, 64, 16, 2, 500, 0)
    assert need > 0
    two = {**good, "N": 2, "b": batch(Bn=2, width=500)}
    assert call(**two) == WORKSPACE and call(**{**two, "ws": FAKE, "wsb": need - 1}) == WORKSPACE and call(**{**two, "ws": FAKE + 8, "wsb": need}) == ALIGN


def test_attention_workspace(lib):
    f = lib.nvfp4_attn_workspace_bytes
    for bad in [(0, 4, 2, 64, 16, 1, 4, 0), (-1, 4, 2, 64, 16, 1, 4, 0), (1, 5, 2, 64, 16, 1, 4, 0), (1, 4, 0, 64, 16, 1, 4, 0), (1, 4, 2, 60, 16, 1, 4, 0), (1, 4, 2, 64, 15, 1, 4, 0), (1, 4, 2, 64, 16, 0, 4, 0),
                (1, 4, 2, 64, 16, 1, 1 << 28, 0), (1, 4, 2, 64, 16, 1, 4, -1), (1 << 24, 1 << 20, 1, 16, 16, 1, 4, 0)]:
        assert f(*bad) == 0, bad
    # tokens that one workgroup takes need none, and lengths play no part: the most that the table has room for
    assert f(1, 4, 2, 64, 16, 1, 1, 0) == 0 and f(1, 4, 2, 64, 16, 1, 100, 0) > 0
    assert f(8, 32, 8, 128, 64, 8, 100, 0) < f(8, 32, 8, 128, 64, 8, 100, 5000)
    # whatever the sizes: no overflow, and no more than binary32 rows for own tokens and prefix, and the parts that a few rows are cut into
    for N, Bn in ((1, 1), (1 << 16, 1 << 16), (1 << 20, 3), (1 << 22, 1 << 16)):
        for Hq, H, D in ((1, 1, 16), (64, 8, 128), (128, 128, 256)):
            if N * Hq <= 1 << 30:
                tiles = 2 * (N * Hq + 128 * H * (Bn + 1)) + 128 * (2048 + 512 + H)
                assert 0 <= f(N, Hq, H, D, 16, Bn, 1 << 20, 1 << 20) <= tiles * (4 * D + 8) + 16 * Bn, (N, Bn, Hq, H, D)


def test_sampling_refuses(lib):
    good = dict(x=FAKE, kind=0, ld=100, N=0, V=100, u=FAKE, T=FAKE, k=FAKE, p=FAKE, m=FAKE, tokens=FAKE, ws=None, wsb=0)

    def call(x, kind, ld, N, V, u, T, k, p, m, tokens, ws, wsb):
        return lib.nvfp4_sample(x, kind, ld, N, V, u, T, k, p, m, tokens, ws, wsb, None)
    assert call(**good) == 0 and call(**{**good, "T": None, "k": None, "p": None, "m": None}) == 0
    for code, change in [(NULL, dict(x=None)), (NULL, dict(u=None)), (NULL, dict(tokens=None)), (SHAPE, dict(N=-1)), (SHAPE, dict(N=BIG)), (SHAPE, dict(V=0)), (SHAPE, dict(V=-1)),
                         (SHAPE, dict(V=(1 << 20) + 1, ld=1 << 21)), (SHAPE, dict(ld=99)), (ENUM, dict(kind=1)), (ENUM, dict(kind=3)), (ALIGN, dict(x=FAKE + 1)), (ALIGN, dict(x=FAKE + 2, kind=2)),
                         (ALIGN, dict(u=FAKE + 2)), (ALIGN, dict(T=FAKE + 1)), (ALIGN, dict(k=FAKE + 2)), (ALIGN, dict(p=FAKE + 2)), (ALIGN, dict(m=FAKE + 1)), (ALIGN, dict(tokens=FAKE + 4))]:
        assert call(**{**good, **change}) == code, change
    need = lib.nvfp4_sample_workspace_bytes(3, 100)
    assert need > 0 and lib.nvfp4_sample_workspace_bytes(0, 100) == lib.nvfp4_sample_workspace_bytes(3, 0) == lib.nvfp4_sample_workspace_bytes(-1, 5) == lib.nvfp4_sample_workspace_bytes(3, BIG) == 0
    three = {**good, "N": 3}
    assert call(**three) == WORKSPACE and call(**{**three, "ws": FAKE, "wsb": need - 1}) == WORKSPACE and call(**{**three, "ws": FAKE + 8, "wsb": need}) == ALIGN


def test_frequencies(lib):
    """Against the formulas in 64 bits: a binary32 rounding each, and a unit of pow()."""
    def want(R, base, scaling, factor, trained, low, high):
        if scaling == B.ROPE_BASE:
            base *= factor ** (R / (R - 2))
        out = []
        for j in range(R // 2):
            f = base ** (-2.0 * j / R)
            if scaling == B.ROPE_LINEAR:
                f /= factor
            if scaling == B.ROPE_PARTS:
                share = min(1.0, max(0.0, (trained * f / (2 * math.pi) - low) / (high - low)))
                f = share * f + (1 - share) * f / factor
            out.append(f)
        return torch.tensor(out, dtype=torch.float64)
    for R in (0, 2, 4, 26, 64, 128, 512):
        for scaling in (B.ROPE_PLAIN, B.ROPE_LINEAR, B.ROPE_BASE, B.ROPE_PARTS):
            if scaling == B.ROPE_BASE and R == 2:
                continue
            got = B.rope_frequencies(R, 50000.0, scaling=scaling, factor=8.0, trained=4096.0, device="cpu").double()
            w = want(R, 50000.0, scaling, 8.0, 4096.0, 1.0, 32.0)
            assert got.shape == (R // 2,) and ((got - w).abs() <= w * (2.0 ** -24 + 1e-13)).all()
    # the ends of the scalings: the fastest frequency stays, the slowest is divided by the factor (BASE and PARTS)
    f = [B.rope_frequencies(128, scaling=s, factor=8.0, trained=2048.0, device="cpu").double() for s in (B.ROPE_PLAIN, B.ROPE_BASE, B.ROPE_PARTS)]
    for scaled in f[1:]:
        assert scaled[0] == 1.0 and abs(scaled[-1] * 8.0 / f[0][-1] - 1.0) < 1e-6
    buf = (C.c_float * 8)()
    for code, args in [(SHAPE, (3, 1e4, 0, 1.0, 0, 1, 32)), (SHAPE, (-2, 1e4, 0, 1.0, 0, 1, 32)), (SHAPE, ((1 << 20) + 2, 1e4, 0, 1.0, 0, 1, 32)), (SHAPE, (2, 1e4, 2, 1.0, 0, 1, 32)), (ENUM, (8, 1e4, 4, 1.0, 0, 1, 32)),
                       (ENUM, (8, 1e4, -1, 1.0, 0, 1, 32)), (ENUM, (8, 0.0, 0, 1.0, 0, 1, 32)), (ENUM, (8, math.inf, 0, 1.0, 0, 1, 32)), (ENUM, (8, 1e4, 1, 0.0, 0, 1, 32)), (ENUM, (8, 1e4, 1, math.nan, 0, 1, 32)),
                       (ENUM, (8, 1e4, 3, 2.0, 0.0, 1, 32)), (ENUM, (8, 1e4, 3, 2.0, 100.0, 5, 5)), (ENUM, (8, 1e4, 3, 2.0, 100.0, -1, 5))]:
        assert lib.nvfp4_rope_frequencies(*args, buf) == code, args
    assert lib.nvfp4_rope_frequencies(8, 1e4, 0, 1.0, 0, 1, 32, None) == NULL and lib.nvfp4_rope_frequencies(0, 1e4, 0, 1.0, 0, 1, 32, None) == 0


def test_binding_refuses(monkeypatch):
    """What the binding asserts, with tensors of the host in the place of the device's."""
    monkeypatch.setattr(B, "_current_device", lambda: -1)
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype)
    i32 = lambda *s: z(*s, dtype=torch.int32)
    c = B.KVCache(z(4, 2, 16, 64), z(4, 2, 16, 64))
    c8 = B.KVCache(z(4, 2, 16, 64, dtype=torch.uint8), z(4, 2, 16, 64, dtype=torch.uint8), z(4, 2, 16, 1, dtype=torch.uint8), z(4, 2, 16, 1, dtype=torch.uint8))
    b = B.KVBatch(i32(3, 2), i32(3))
    r = B.Rope(torch.zeros(32))
    assert len(c.packed(-1)) == len(c8.packed(-1)) == 72 and len(b.packed(-1, 16)) == 56 and len(r.packed(-1)) == 24
    for bad in (B.KVCache(z(4, 2, 16, 64), z(4, 2, 16, 32)), B.KVCache(z(4, 2, 64), z(4, 2, 64)), B.KVCache(z(4, 2, 16, 64).float(), z(4, 2, 16, 64).float()), B.KVCache(c.k, c8.v),
                B.KVCache(c.k.transpose(0, 1), c.v.transpose(0, 1)), B.KVCache(c.k, c.v, c8.k_exps, c8.v_exps), B.KVCache(c8.k, c8.v), B.KVCache(c8.k, c8.v, c8.k_exps, c8.v_exps[:3])):
        with pytest.raises(AssertionError):
            bad.packed(-1)
    for bad in (B.KVBatch(i32(3, 2), i32(2)), B.KVBatch(i32(3, 2).long(), i32(3)), B.KVBatch(i32(3), i32(3)), B.KVBatch(i32(3, 2), i32(3), i32(3)), B.KVBatch(i32(3, 2), i32(3), None, None, 5),
                B.KVBatch(i32(3, 2), i32(3), None, i32(1), 17), B.KVBatch(i32(3, 4)[:, ::2], i32(3)), B.KVBatch(i32(3, 2), i32(6)[::2])):
        with pytest.raises(AssertionError):
            bad.packed(-1, 16)
    for bad in (B.Rope(torch.zeros(32).double()), B.Rope(torch.zeros(64)[::2]), B.Rope(torch.zeros(4, 8))):
        with pytest.raises(AssertionError):
            bad.packed(-1)
    for call in (lambda: B.kv_append(z(3, 128), z(3, 64), c, b), lambda: B.kv_append(z(3, 64), z(3, 64), c, b), lambda: B.kv_append(z(3, 128), z(3, 128).float(), c, b),
                 lambda: B.kv_append(z(3, 128), z(3, 128), c, b, Q=z(2, 128)), lambda: B.kv_append(z(3, 128), z(3, 128), c, b, Q=z(3, 100)), lambda: B.kv_append(z(3, 128), z(3, 128), c, b, Q=z(3, 128).float()),
                 lambda: B.kv_append(z(3, 128), z(3, 128), c, b, Qo=z(3, 128)), lambda: B.attn(z(3, 128).float(), c, b, 2), lambda: B.attn(z(3, 128), c, b, 4), lambda: B.attn(z(3, 256), c, b, 4, Out=z(3, 128)),
                 lambda: B.kv_load(c, b, 3, K=z(3, 64)), lambda: B.rope(z(3, 128), i32(2), r, 2), lambda: B.rope(z(3, 128), i32(3).long(), r, 2), lambda: B.rope(z(3, 128), i32(3), r, 3),
                 lambda: B.rope(z(3, 128), i32(3), r, 0), lambda: B.sample(z(3, 9), torch.zeros(2)), lambda: B.sample(z(3, 9), torch.zeros(3).double()), lambda: B.sample(z(3, 9), torch.zeros(3), top_k=torch.zeros(3)),
                 lambda: B.sample(z(3, 9), torch.zeros(3), tokens=i32(3)), lambda: B.sample(z(3, 9).half(), torch.zeros(3))):
        with pytest.raises(AssertionError):
            call()


def test_more_workgroups_than_a_launch_has_are_refused(lib):
    """A launch has less than 2^32 threads: 2^24 workgroups of 256, 2^22 of 1024."""
    rope = lambda N: lib.nvfp4_rope(FAKE, 0, 0, FAKE, N, 0, 64, rotation(), 0, FAKE, 0, 0, None)
    assert rope((1 << 24) - 1) == 0 and rope(1 << 24) == SHAPE
    none = batch(starts=FAKE)
    append = lambda N: lib.nvfp4_kv_append(None, 0, 0, FAKE, 128, FAKE, 128, 0, N, cache(), none, None, None, 0, 0, None)
    load = lambda N: lib.nvfp4_kv_load(cache(), none, N, FAKE, 128, FAKE, 128, 0, None)
    for f in (append, load):
        assert f((1 << 24) - 1) == 0 and f(1 << 24) == SHAPE
    assert lib.nvfp4_sample_workspace_bytes((1 << 22) - 1, 100) > 0 and lib.nvfp4_sample_workspace_bytes(1 << 22, 100) == 0
    assert lib.nvfp4_sample(FAKE, 0, 100, 1 << 22, 100, FAKE, None, None, None, None, FAKE, FAKE, 1 << 60, None) == SHAPE
    f = lib.nvfp4_attn_workspace_bytes

    def attn(N, Hq, H, Bn, width, prefix):
        return lib.nvfp4_attn(FAKE, Hq * 16, N, Hq, cache(H=H, D=16), batch(starts=FAKE, Bn=Bn, width=width, prefix=prefix, prefix_table=FAKE), 0.25, FAKE, Hq * 16, None, 0, None)
    # rows to join: a token and query head each (64 rows a sequence: 128 would take the prefix themselves).  The size, which is the host's alone, comes first: a call that needs no
    # workspace would not be refused.
    assert f(65535, 256, 4, 16, 16, 65535, 1, 4096) > 0
    assert attn(65535, 256, 4, 65535, 1, 4096) == WORKSPACE
    assert f(65536, 256, 4, 16, 16, 65536, 1, 4096) == 0
    assert attn(65536, 256, 4, 65536, 1, 4096) == SHAPE
    # tiles of key heads: a tile for each sequence at least
    assert attn(65536, 512, 512, 65536, 1, 0) == SHAPE
    assert attn(1, 1 << 18, 1 << 18, 65536, 4, 0) == SHAPE
