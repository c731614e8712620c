"""Plain 64-bit reference of the paged window cache, on the CPU (numpy, one position at a time where that is
clearest): what a quantised row stands for, and the attention over visible tokens and bank."""

import numpy as np

LARGEST = {"fp8": 448.0, "fp4": 6.0}
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def e4m3_values():
    """Values of the codes 0..126 (127 is NaN), ascending."""
    c = np.arange(127)
    ex, fr = c >> 3, c & 7
    return np.where(ex == 0, fr / 8 * 2.0 ** -6, (1 + fr / 8) * 2.0 ** (ex - 7.0))


def nearest_codes(a, table):
    """Code of the table's nearest value to each a >= 0, a value half way between two taking the even code."""
    hi = np.clip(np.searchsorted(table, a), 0, len(table) - 1)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - table[lo], table[hi] - a
    up = (dh < dl) | ((dh == dl) & (hi % 2 == 0))
    return np.where(up, hi, lo)


def quantise(x, fmt):
    """float64 [..., d] -> (codes uint8 [..., row bytes], scale codes uint8 [..., d / 32])."""
    g = np.asarray(x, np.float64).reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    bad = ~np.isfinite(g).all(-1)
    g = np.where(bad[..., None], 0.0, g)
    top = np.abs(g).max(-1)
    e = np.full(top.shape, -100)
    for cand in range(-100, 128):  # the smallest exponent that fits
        e = np.where((e == cand) & (top > LARGEST[fmt] * 2.0 ** cand), cand + 1, e)
    y = g * 2.0 ** -e[..., None].astype(np.float64)
    neg = np.signbit(y)
    if fmt == "fp8":
        codes = (nearest_codes(np.abs(y), e4m3_values()) + 128 * neg).astype(np.uint8).reshape(x.shape)
    else:
        c = (nearest_codes(np.abs(y), E2M1) + 8 * neg).reshape(x.shape)
        codes = (c[..., 0::2] + 16 * c[..., 1::2]).astype(np.uint8)
    sc = np.where(bad, 255, e + 127).astype(np.uint8)
    codes_flat = codes
    if bad.any():  # the codes of such a group are not compared
        w = codes.shape[-1] // sc.shape[-1]
        codes_flat = np.where(np.repeat(bad, w, -1), 0, codes).astype(np.uint8)
    return codes_flat, sc


def values(codes, scale, fmt):
    if fmt == "fp8":
        t = np.concatenate([e4m3_values(), [np.nan]])
        y = np.where(codes >= 128, -1.0, 1.0) * t[codes & 127]
    else:
        c = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], 2 * codes.shape[-1])
        y = np.where(c >= 8, -1.0, 1.0) * E2M1[c & 7]
    f = np.where(scale == 255, np.nan, 2.0 ** (scale.astype(np.float64) - 127))
    return y * np.repeat(f, 32, -1)


def visible(p_len, n, i, window, sink, causal):
    """Positions that new token i of n sees in a sequence of p_len tokens."""
    at = p_len - n + i if causal else p_len - 1
    return [j for j in range(p_len) if j <= at and (window == 0 or j > at - window or j < sink)]


def attention(q, k, v, mask, scale):
    """q [n, d], k, v [m, d], mask [n, m] (True: seen), float64.  Returns (out, sum of weights x |v|, bound of
    sum |q k| scale): rows that see nothing are zeros; what is not seen is not touched."""
    n, d = q.shape
    out, av, big = np.zeros((n, d)), np.zeros((n, d)), np.zeros(n)
    for i in range(n):
        m = np.nonzero(mask[i])[0]
        if not m.size:
            continue
        km, vm = k[m], v[m]
        with np.errstate(invalid="ignore", over="ignore"):
            s = km @ q[i] * scale
            w = np.exp(s - s.max())
            w = w / w.sum()
            out[i], av[i] = w @ vm, w @ np.abs(vm)
            big[i] = (np.abs(km) @ np.abs(q[i])).max() * scale
    return out, av, big


def tolerance(out, av, big, d, m, dtype):
    """How far a kernel's row may be from `out`, from the roundings it makes.

    A score is a sum of d products in binary32 (error at most (d + 2) 2^-24 of sum |q k| scale, twice that with the
    conversion to log2 units), so a weight is off by eps = 2 (d + 4) 2^-24 big, and by 2^-20 for exp2 of arguments whose
    rounding is 2^-24 of at most big (in eps).  In bf16 each weight is rounded to 8 significant bits (2^-8), and its
    rounded value enters numerator and denominator alike; the output is rounded once (2^-8; 2^-23 in binary32, with its
    division).  Sums of m weights in binary32 add m 2^-24, and joining partial sums 2^-20."""
    w = 2 * (d + 4) * 2.0 ** -24 * big[:, None] + 2.0 ** -19 + m * 2.0 ** -24 + (2.0 ** -8 if dtype == "bf16" else 0.0)
    return w * (av + np.abs(out)) + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -23) * (np.abs(out) + w * av) + 1e-30
