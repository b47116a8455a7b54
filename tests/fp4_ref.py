"""Plain forms, in 64 bits, of the operators in microscaled 4-bit floating point."""
import numpy as np

BLOCK = HEAD = 32
MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
VALUES = np.concatenate([MAGNITUDES, -MAGNITUDES])
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def quantise(x):
    """(codes 0 .. 15, scale bytes) of x [..., 32 m] by blocks along the last axis."""
    x = np.asarray(x, dtype=np.float64)
    shape = x.shape
    x = x.reshape(-1, BLOCK)
    with np.errstate(invalid="ignore", over="ignore"):
        top = np.abs(x).max(axis=1)
        bad = ~np.isfinite(x).all(axis=1)
        s = np.full(top.shape, -127)
        while True:                                # the smallest exponent with top <= 7 * 2^s
            up = ~bad & (top > 7.0 * 2.0 ** s.astype(np.float64))
            if not up.any():
                break
            s = s + up
        y = np.where(bad[:, None], 0.0, x * 2.0 ** -s.astype(np.float64)[:, None])
    a = np.abs(y)
    hi = np.clip(np.searchsorted(MAGNITUDES, a), 1, 7)
    lo = hi - 1
    d_lo, d_hi = a - MAGNITUDES[lo], MAGNITUDES[hi] - a
    code = np.where((d_lo < d_hi) | ((d_lo == d_hi) & (lo % 2 == 0)), lo, hi)
    code = np.where(bad[:, None], 0, code + 8 * np.signbit(y))
    return code.astype(np.uint8).reshape(shape), np.where(bad, 255, s + 127).astype(np.uint8).reshape(*shape[:-1], -1)


def numbers(code, byte):
    v = VALUES[code].reshape(*byte.shape, BLOCK)
    s = np.where(byte == 255, np.nan, 2.0 ** (byte.astype(np.float64) - 127))
    return (v * s[..., None]).reshape(code.shape)


def rounded(x):
    return numbers(*quantise(x))


def store(K, V):
    """(codes [n, d], scales [n, heads, 2]) of K and V rows: two codes to a byte, the first in the low half."""
    (k, kb), (v, vb) = quantise(K), quantise(V)
    c = np.concatenate([k, v], axis=1)
    return c[:, 0::2] | (c[:, 1::2] << 4), np.stack([kb, vb], axis=2)


def values(codes, scales):
    """(K, V) in 64 bits of store rows."""
    codes, scales = np.asarray(codes), np.asarray(scales)
    n, d = codes.shape
    c = np.stack([codes & 15, codes >> 4], axis=2).reshape(n, 2 * d)
    return numbers(c[:, :d], scales[:, :, 0]), numbers(c[:, d:], scales[:, :, 1])


def across(W):
    """A weight matrix [k, n] in blocks along k."""
    return rounded(np.ascontiguousarray(np.asarray(W, dtype=np.float64).T)).T


def proj(S, W, rounding):
    """(product, bound). A sum of k products of numbers with two bits, each exact: an addition is off by at most 2^-23 of what is
    summed (rounded or cut off), and every product takes part in at most k additions."""
    s, w = rounded(S), across(W)
    y = s @ w
    return y, rounding * np.abs(y) + s.shape[1] * 2.0 ** -23 * (np.abs(s) @ np.abs(w)) + 1e-37


def ffn(S, W1, W2, eps, rounding):
    """(LayerNorm(S + q(max(q(S) q(W1), 0)) q(W2)), bound), for inputs whose sums are exact in 32 bits (hidden values and with them
    their codes are then the same; see exact_sums).

    x = S + product is off by u |x|, u = 2^-24. The mean of d numbers in groups (16 in turn, then two halves and up to 8 groups,
    each addition rounded): 26 u of the mean magnitude, as is what the differences are taken from; x - mean: u of itself. With d_i the
    sum of these, the sum of squares is off by at most 2 |d| / |x - mean| relative (norms over the row) and 30 u, the reciprocal root by
    half of that and 4 u more. The last product and its rounding follow.
    """
    x64 = np.asarray(S, dtype=np.float64)
    h = np.maximum(rounded(x64) @ across(W1), 0)
    x = x64 + rounded(h) @ across(W2)
    u = 2.0 ** -24
    mean = x.mean(axis=1, keepdims=True)
    c = x - mean
    std = np.sqrt((c * c).mean(axis=1, keepdims=True) + eps)
    y = c / std
    d = u * np.abs(x) + 2 * 26 * u * np.abs(x).mean(axis=1, keepdims=True) + u * np.abs(c)
    rel = np.sqrt((d * d).mean(axis=1, keepdims=True)) / std + 20 * u
    return y, 1.01 * (d / std + np.abs(y) * rel) + rounding * np.abs(y) + 1e-37


def exact_sums(S, W):
    """Whether every partial sum of q(S) q(W) fits 24 bits: all products are multiples of the smallest step of theirs."""
    (_, sb), w = quantise(S), across(W)
    _, wb = quantise(np.ascontiguousarray(np.asarray(W, dtype=np.float64).T))
    step = 0.25 * 2.0 ** (sb.astype(int).min(axis=1)[:, None] + wb.astype(int).min(axis=1)[None, :] - 254.0)
    return (np.abs(rounded(S)) @ np.abs(w) < step * 2.0 ** 24).all()
