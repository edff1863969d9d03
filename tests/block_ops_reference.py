"""The operators around the quantized linears from their definitions, in 64 bits, and how far a computation in 32 bits may be from them.

Errors are bounded by the usual model: every operation has a relative error of at most U = 2^-24, a sum of terms t taken in any
order of at most `steps` additions per term one of steps * U * sum |t|.
"""
import math

import numpy as np
import torch

U = 2.0 ** -24
GROUP = 128
ROUND = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -23}    # of a value rounded to nearest, twice over
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def f64(t):
    return t.detach().double().cpu()


# ---------------------------------------------------------------------------------------------- 8-bit checkpoints ----

def e4m3_table():
    """Values of the codes 0 .. 126 (the magnitudes; 127 is the NaN)."""
    c = np.arange(127)
    return np.where(c < 8, c * 2.0 ** -9, (8 + c % 8) * 2.0 ** (c // 8 - 10.0))


def ckpt8(x):
    """(codes, exps, values) of a [rows, K] array by a search among the code values, ties to the even code."""
    x = f64(x).numpy()
    rows, K = x.shape
    groups = -(-K // GROUP)
    table = e4m3_table()
    codes, exps, values = np.zeros((rows, K), np.uint8), np.zeros((rows, groups), np.uint8), np.zeros((rows, K))
    for r in range(rows):
        for g in range(groups):
            v = x[r, g * GROUP:(g + 1) * GROUP]
            fine = np.abs(v[np.isfinite(v)])
            a = fine.max() if fine.size else 0.0
            e = -126
            while a > 448.0 * 2.0 ** e:
                e += 1
            e = min(e, 120)
            m = np.where(np.isfinite(v), np.abs(v), 0.0) * 2.0 ** -e
            hi = np.searchsorted(table, m).clip(0, 126)
            lo = np.maximum(hi - 1, 0)
            up = (table[hi] - m < m - table[lo]) | ((table[hi] - m == m - table[lo]) & (hi % 2 == 0)) | (table[hi] == m)
            c = np.where(up, hi, lo)
            bad = ~np.isfinite(v)
            codes[r, g * GROUP:(g + 1) * GROUP] = np.where(bad, 127, c | np.where(np.signbit(v), 128, 0))
            exps[r, g] = e + 127
            values[r, g * GROUP:(g + 1) * GROUP] = np.where(bad, np.nan, np.copysign(table[c] * 2.0 ** e, v))
    return codes, exps, torch.from_numpy(values)


# ------------------------------------------------------------------------------------------------------------ norms ----

def steps_of_row(D):
    """Additions that a term of a row's sum meets at most: a thread's own elements, the exchange between 64 lanes, the waves of a row."""
    return 8 * -(-D // 512) + 6 + 16


def norm_fwd(x, gamma, beta, eps, layer, out):
    """(y, mean, rstd) and the bounds of y, mean and rstd."""
    x = f64(x)
    N, D = x.shape
    g = torch.ones(D, dtype=torch.float64) if gamma is None else f64(gamma)
    b = torch.zeros(D, dtype=torch.float64) if beta is None else f64(beta)
    s = steps_of_row(D) + 2
    mean = x.mean(1, keepdim=True) if layer else torch.zeros(N, 1, dtype=torch.float64)
    d = x - mean
    var = d.square().mean(1, keepdim=True)
    rstd = 1.0 / (var + eps).sqrt()
    e_mean = s * U * x.abs().mean(1, keepdim=True) if layer else torch.zeros_like(mean)
    # the variance about a mean that is e_mean off grows by e_mean^2; its own sum and its terms' roundings; 1/sqrt halves the relative error
    rel = 0.5 * ((s + 6) * U * var + e_mean.square() + 2 * U * e_mean * d.abs().mean(1, keepdim=True)) / (var + eps) + 4 * U
    y = d * rstd * g + b
    e_y = g.abs() * rstd * (e_mean + d.abs() * (rel + 4 * U)) * 1.01 + 2 * U * (y.abs() + b.abs()) + ROUND[out] * y.abs() + 1e-38
    return (y, mean, rstd), (e_y, e_mean + U * mean.abs(), rstd * rel * 1.01)


def norm_bwd(dy, x, stats, gamma, layer, out):
    """(dx, dgamma, dbeta) from the given statistics, and their bounds."""
    dy, x, st = f64(dy), f64(x), f64(stats)
    N, D = x.shape
    w = torch.ones(D, dtype=torch.float64) if gamma is None else f64(gamma)
    s = steps_of_row(D) + 8
    r = st[:, 1:]
    h = (x - st[:, :1]) * r
    g = dy * w
    m1 = g.mean(1, keepdim=True) if layer else torch.zeros(N, 1, dtype=torch.float64)
    m2 = (g * h).mean(1, keepdim=True)
    dx = r * (g - m1 - h * m2)
    e_sum = s * U * ((g.abs().mean(1, keepdim=True) if layer else 0.0) + h.abs() * (g * h).abs().mean(1, keepdim=True))
    e_dx = r.abs() * (e_sum + 8 * U * (g.abs() + m1.abs() + (h * m2).abs())) + ROUND[out] * dx.abs() + 1e-38
    n = (N + 8) * U
    return (dx, (dy * h).sum(0), dy.sum(0)), (e_dx, n * (dy * h).abs().sum(0) + 1e-38, n * dy.abs().sum(0) + 1e-38)


# ---------------------------------------------------------------------------------------------------- nonlinearities ----

C, A = 2.0 * math.sqrt(2.0 / math.pi), 0.044715


def _pair(z):
    """s(z), s(-z)."""
    return torch.sigmoid(z), torch.sigmoid(-z)


def _rel(z):
    """Relative error of s(z) or s(-z) in 32 bits: z itself (three roundings), the exponential of a rounded product, sum, quotient, product."""
    return (6.0 * z.abs() + 24.0) * U


def act_fwd(h, swiglu, out):
    h = f64(h)
    if swiglu:
        g, u = h.chunk(2, 1)
        s, _ = _pair(g)
        a = g * s * u
        e = _rel(g) * a.abs() + 1e-37 * (g * u).abs()
    else:
        z = C * (h + A * h ** 3)
        a = h * _pair(z)[0]
        e = _rel(z).clamp(max=1.0) * a.abs() + 1e-37 * h.abs()
    return a, e + ROUND[out] * a.abs() + 1e-38


def act_bwd(da, h, swiglu, out):
    da, h = f64(da), f64(h)
    if swiglu:
        g, u = h.chunk(2, 1)
        s, t = _pair(g)
        dh = torch.cat((da * u * s * (1 + g * t), da * g * s), 1)
        e = torch.cat(((da * u * s).abs() * (1 + (g * t).abs()) * _rel(g) + 1e-37 * (da * u).abs() * (1 + g.abs()), (da * g * s).abs() * _rel(g) + 1e-37 * (da * g).abs()), 1)
    else:
        z = C * (h + A * h ** 3)
        s, t = _pair(z)
        inner = h * s * t * C * (1 + 3 * A * h ** 2)
        dh = da * (s + inner)
        e = da.abs() * (s + inner.abs()) * _rel(z).clamp(max=1.0) + 1e-30 * da.abs()
    return dh, e + ROUND[out] * dh.abs() + 1e-38


# ---------------------------------------------------------------------------------------------------------- products ----

def unpack(codes, scales, gscale, outer_block):
    """Weights of a packed operand from its bytes."""
    c = codes.cpu().numpy()
    C_, K = c.shape[0], c.shape[1] * 2
    idx = np.stack((c & 15, c >> 4), 2).reshape(C_, K)
    v = E2M1[idx & 7] * np.where(idx & 8, -1.0, 1.0)
    w = v * np.append(e4m3_table(), np.nan)[scales.cpu().numpy()].repeat(16, 1)
    g = f64(gscale).numpy()
    return torch.from_numpy(w * (g.repeat(GROUP, 1) if outer_block else g.reshape(-1)[0]))


def gemv(x, w, out):
    """y and its bound: exact products; a term meets the additions of a quarter of the reduction at most (four waves share it) and a few more."""
    x = f64(x)
    y = x @ w.t()
    return y, (w.shape[1] / 4 + 64) * U * (x.abs() @ w.abs().t()) + ROUND[out] * y.abs() + 1e-38


def within(got, want, bound, what=""):
    """Every finite value within its bound; the same NaNs."""
    got = f64(got)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what + ": NaNs elsewhere"
    off = torch.nan_to_num((got - want).abs(), nan=0.0)
    over = off > torch.nan_to_num(bound, nan=0.0)
    assert not over.any(), "%s: %d of %d values off, worst %.3g times the bound" % (what, int(over.sum()), got.numel(), float((off / bound).nan_to_num(0).max()))
