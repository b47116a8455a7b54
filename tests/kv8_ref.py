"""Plain forms, in 64 bits, of the operators on the K|V store in 8 bits."""
import numpy as np

HEAD = 32
LARGEST = {"e4m3": 448.0, "int8": 127.0}


def e4m3_values():
    """The number each of the 256 codes stands for (1 sign, 4 exponent, 3 mantissa bits, bias 7; 0x7F and 0xFF are NaN)."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e > 0, (1 + m / 8) * 2.0 ** (e - 7.0), m / 8 * 2.0 ** -6)
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c < 128, v, -v)


def int8_values():
    return np.arange(256, dtype=np.uint8).view(np.int8).astype(np.float64)


VALUES = {"e4m3": e4m3_values(), "int8": int8_values()}


def quantise(x, fmt):
    """(codes' numbers [rows, d], scale bytes [rows, d/32]) of rows x."""
    x = np.asarray(x, dtype=np.float64).reshape(len(x), -1, HEAD)
    with np.errstate(invalid="ignore", over="ignore"):
        top = np.abs(x).max(axis=2)
        bad = ~np.isfinite(x).all(axis=2)
        s = np.full(top.shape, -127)
        while True:                                # the smallest exponent with top <= largest * 2^s
            up = ~bad & (top > LARGEST[fmt] * 2.0 ** s.astype(np.float64))
            if not up.any():
                break
            s = s + up
        y = np.where(bad[..., None], 0.0, x * 2.0 ** -s.astype(np.float64)[..., None])
    if fmt == "int8":
        y = np.rint(y)
    else:
        grid = VALUES["e4m3"][:127]                # ascending, from 0 to 448
        a = np.abs(y)
        hi = np.clip(np.searchsorted(grid, a), 1, 126)
        lo = hi - 1
        d_lo, d_hi = a - grid[lo], grid[hi] - a
        pick = np.where((d_lo < d_hi) | ((d_lo == d_hi) & (lo % 2 == 0)), lo, hi)
        y = np.copysign(grid[pick], y)
    return y.reshape(len(x), -1), np.where(bad, 255, s + 127).astype(np.uint8)


def values(codes, scales, fmt):
    """(K, V) in 64 bits of store rows (codes [n, 2d], scales [n, heads, 2])."""
    codes, scales = np.asarray(codes), np.asarray(scales)
    n, d = codes.shape[0], codes.shape[1] // 2
    out = []
    for part in (0, 1):
        v = VALUES[fmt][codes[:, part * d:(part + 1) * d]].reshape(n, -1, HEAD)
        s = scales.reshape(n, -1, 2)[:, :, part].astype(np.float64)
        s = np.where(s == 255, np.nan, 2.0 ** (s - 127))
        out.append((v * s[..., None]).reshape(n, d))
    return out


def attention(nbr_ptr, nbr_idx, nbr_rel, gates, Q, K, V, bias, rounding):
    """(A, bound): dense attention of each listed gate over its row, and how far a computation in 32 bits may be from it.

    Sources of a relation with bias -inf are left out. The bound, per element: a head's score is a sum of 32 products and a
    bias, each step rounded (2^-24 relative to the magnitudes summed): 36 steps with slack. Subtracting the maximum and
    multiplying by log2 e rounds twice more, 2^-23 of |score - max|, and the power is within 2^-22. A weight is then off by at
    most e = 2 * (score error) + 2^-22 relative (numerator and denominator), the sum over n sources by another n 2^-24 twice,
    all relative to sum(alpha |v|). `rounding` is half a step of the output's type, relative.
    """
    Q, K, V, bias = (np.asarray(t, dtype=np.float64) for t in (Q, K, V, bias))
    heads = Q.shape[1] // HEAD
    out, bound = np.zeros((len(gates), Q.shape[1])), np.zeros((len(gates), Q.shape[1]))
    for i, v in enumerate(gates):
        lo, hi = nbr_ptr[v], nbr_ptr[v + 1]
        src, rel = nbr_idx[lo:hi], nbr_rel[lo:hi]
        for h in range(heads):
            keep = bias[h][rel] != -np.inf
            if not keep.any():
                continue
            sl = slice(h * HEAD, (h + 1) * HEAD)
            k, x, b = K[src[keep], sl], V[src[keep], sl], bias[h][rel[keep]]
            s = k @ Q[i, sl] / np.sqrt(HEAD) + b
            w = np.exp(s - s.max())
            w /= w.sum()
            out[i, sl] = w @ x
            size = (np.abs(k) @ np.abs(Q[i, sl])) / np.sqrt(HEAD) + np.abs(b)
            # (a source whose weight vanishes may be off as it likes: its error counts by its weight)
            e = 36 * 2.0 ** -24 * size + 2.0 ** -23 * np.abs(s - s.max()) + 2.0 ** -22
            e = np.where(w > 0, e, 0)
            bound[i, sl] = ((2 * e + 2 * len(src) * 2.0 ** -24) * w) @ np.abs(x) + (w @ (2 * e)) * (w @ np.abs(x)) + rounding * np.abs(out[i, sl])
    return out, bound + 1e-37
