"""Plain 64-bit forms of the group quantizer, the products on its codes, rotary positions, the 4-bit cache and its
attention, in numpy on the host, with the error bounds the GPU results are held to."""
import numpy as np

HALF = 2.0 ** -11            # largest relative error of one rounding to fp16
TINY = 2.0 ** -25            # largest absolute error of one below the normal range
EPS32 = 2.0 ** -24


def quantize(x):
    """fp16 [..., group] -> codes int [..., group], steps fp16 [...]: the step is max / 7 in fp32 (a division), rounded to
    fp16, 1 where that is zero; the codes come from 64 bits."""
    x = np.asarray(x, np.float16)
    steps = (np.abs(x.astype(np.float32)).max(-1) / np.float32(7)).astype(np.float16)
    steps[steps == 0] = 1
    codes = np.clip(np.floor(x.astype(np.float64) / steps.astype(np.float64)[..., None] + 0.5), -8, 7).astype(np.int64)
    return codes, steps


def pack(codes):
    c = np.asarray(codes) & 15
    return (c[..., 0::2] | (c[..., 1::2] << 4)).astype(np.uint8)


def product(X, codes, steps, group, scaled_weights=False):
    """Y in 64 bits and the bound on |gpu - Y|.

    The sums of a group run on nibbles plus 8 (16 |x| bounds a term), at most group / 32 steps of 32 products each; the
    K / group sums then add in fp32.  scaled_weights: the kernel for many tokens rounds code * step to fp16 first (half a
    step of fp16 on every product) and adds K / 16 steps of 16 products.  One rounding to fp16 at the end."""
    X64, w = X.astype(np.float64), codes.astype(np.float64)
    N, K = w.shape
    s = steps.astype(np.float64)
    ws = (w.reshape(N, K // group, group) * s[..., None]).reshape(N, K)
    Y = X64 @ ws.T
    mags = np.abs(X64) @ np.abs(ws).T
    if scaled_weights:
        slack = ((K // 16 + 18) * EPS32 + HALF) * mags + TINY * np.abs(X64).sum(1, keepdims=True)
    else:
        sums = np.abs(X64).reshape(-1, K // group, group).sum(-1) @ s.T
        slack = (group // 32 + 33) * EPS32 * 16 * sums + (K // group + 4) * EPS32 * mags
    return Y, HALF * (np.abs(Y) + slack) + slack + TINY


def frequencies(rot, base=10000.0, scaling=0, factor=1.0, trained=0.0, low=0.0, high=0.0):
    i = np.arange(rot // 2, dtype=np.float64)
    if scaling == 2:
        base = base * factor ** (rot / (rot - 2))
    f = base ** (-2 * i / rot)
    if scaling == 1:
        f = f / factor
    if scaling == 3:
        turns = trained * f / (2 * np.pi)
        keep = np.clip((turns - low) / (high - low), 0, 1)
        f = keep * f + (1 - keep) * f / factor
    return f


def rotary(X, positions, f, half, magnitude=1.0):
    """fp16 [T, H, D] -> 64-bit result and bound: angles within 2^-25 of a turn (2^-24 pi), sine, cosine, products and sums
    in fp32 (four roundings of terms up to m (|a| + |b|)), one rounding to fp16; copied channels exact.  The reference
    angle itself, position * f in 64 bits, is off by at most 2^-53 of it and 2^-53 position f of the table."""
    x = X.astype(np.float64)
    y, bound = x.copy(), np.zeros_like(x)
    n = len(f)
    i = np.arange(n)
    p, q = (i, i + n) if half else (2 * i, 2 * i + 1)
    angle = positions.astype(np.float64)[:, None, None] * f
    a, b = x[..., p], x[..., q]
    y[..., p] = magnitude * (a * np.cos(angle) - b * np.sin(angle))
    y[..., q] = magnitude * (a * np.sin(angle) + b * np.cos(angle))
    slack = magnitude * (np.abs(a) + np.abs(b)) * (np.pi * 2.0 ** -24 + 6 * EPS32 + np.abs(angle) * 2.0 ** -51)
    for place in (p, q):
        bound[..., place] = slack + HALF * (np.abs(y[..., place]) + slack) + TINY
    return y, bound


class Cache:
    """The cached rows as numbers, sequence by sequence (no pages): codes and steps of K and V."""

    def __init__(self, B):
        self.rows = [([], []) for _ in range(B)]          # per sequence: lists of (codes [Hk, D], steps [Hk])

    def append(self, b, k, v):
        self.rows[b][0].append(quantize(k))
        self.rows[b][1].append(quantize(v))

    def values(self, b, which, upto):
        """fp64 [rows, Hk, D] and the steps [rows, Hk]"""
        rows = self.rows[b][which][:upto]
        codes = np.stack([r[0] for r in rows]).astype(np.float64)
        steps = np.stack([r[1] for r in rows]).astype(np.float64)
        return codes * steps[..., None], steps


def attention(q, k, v, sk, sv, sees, scale):
    """One head: q fp16 [n, D], k, v fp64 [L, D] with their steps [L], sees bool [n, L] -> O fp64 [n, D] and its bound.

    Scores: products of fp16 and nibbles plus 8 (16 |q| bounds a term), D / 32 steps of 32, the offset taken off, then four
    fp32 roundings; delta is the largest error of a score in natural units, so that a weight is off by a factor within
    exp(+-2 delta) (its own and the normaliser's) beside 6 roundings.  A weight times the value's step is rounded to fp16:
    half a step of fp16, or 2^-25 below its normal range.  The largest such product P is at least 2^-1, and with l the
    normaliser on the same scale sum(p sv) >= P / l, so n keys of codes up to 8 are off by n 8 2^-25 / l <= n 2^-21 sum(p sv).
    The sums of weights and nibbles plus 8 (16 steps bound a term) take L / 32 steps of 32 per part and as many to add the
    parts.  One rounding to fp16 at the end."""
    n, D = q.shape
    L = k.shape[0]
    O, bound = np.zeros((n, D)), np.zeros((n, D))
    if L == 0:
        return O, bound
    q64 = q.astype(np.float64)
    s = np.where(sees, (q64 @ k.T) * scale, -np.inf)
    some = sees.any(1)
    s, see, qq = s[some], sees[some], q64[some]
    if not some.any():
        return O, bound
    top = s.max(1, keepdims=True)
    e = np.exp(s - top)
    l = e.sum(1, keepdims=True)
    p = e / l
    O[some] = p @ v
    delta = scale * (D // 32 + 33) * EPS32 * 16 * np.abs(qq).sum(1, keepdims=True) * np.where(see, sk, 0).max(1, keepdims=True) \
        + 6 * EPS32 * np.abs(np.where(see, s, 0)).max(1, keepdims=True)
    mags = p @ np.abs(v)
    slack = (2 * delta + HALF + 8 * EPS32) * mags + (L // 32 + 40) * EPS32 * 16 * (p @ sv)[:, None] \
        + see.sum(1, keepdims=True) * 2.0 ** -21 * (p @ sv)[:, None]
    bound[some] = slack + HALF * (np.abs(O[some]) + slack) + TINY
    return O, bound


def held(got, want, bound, what):
    """got (fp16 array) within bound of want, and finite."""
    g = np.asarray(got).astype(np.float64)
    assert g.shape == want.shape, what
    assert np.isfinite(g).all(), f"{what}: not finite"
    excess = np.abs(g - want) - bound
    assert excess.max(initial=-1.0) <= 0, f"{what}: {excess.max():.3e} over the bound at {np.unravel_index(excess.argmax(), g.shape)}"
