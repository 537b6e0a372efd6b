"""Plain 64-bit forms of the MXFP4 cache and of attention of many rows with capped scores, distance bias and masks, and the bounds of their results
(those of token_path_ref.py where they are the same)."""
import numpy as np

import token_path_ref as ref

E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def mxfp4_exponent(most):
    """floor(log2 most) - 2 within -23..13, for a most of 0 the least."""
    with np.errstate(divide="ignore"):
        return np.clip(np.where(most > 0, np.floor(np.log2(np.where(most > 0, most, 1))) - 2, -23), -23, 13)


def mxfp4_codes(a):
    """The E2M1 code of |a|: nearest, halves to the even code, saturating."""
    middle = (E2M1[1:] + E2M1[:-1]) / 2
    below = np.searchsorted(middle, a, side="left")              # middles below a
    tie = (below < 7) & (a == middle[np.minimum(below, 6)])
    return below + (tie & (below % 2 == 1))


def mxfp4(v):
    """Rows [..., D] in 64 bits as (codes with sign [..., D], scale bytes [..., D/32])."""
    g = v.reshape(*v.shape[:-1], -1, 32)
    bad = ~np.isfinite(g).all(-1)
    g = np.where(bad[..., None], 0, g)
    e = mxfp4_exponent(np.abs(g).max(-1))
    codes = mxfp4_codes(np.abs(g) * 2.0 ** -e[..., None]) + 8 * (np.signbit(g))
    return codes.reshape(v.shape), np.where(bad, 255, e + 127).astype(np.int64)


def mxfp4_values(codes, scales):
    v = np.where(codes & 8, -1, 1) * E2M1[codes & 7]
    s = np.where(scales == 255, np.nan, 2.0 ** (np.minimum(scales, 254) - 127.0))
    return (v.reshape(*v.shape[:-1], -1, 32) * s[..., None]).reshape(v.shape)


def mxfp4_held(cache, slots):
    """(codes, scale bytes) of keys and of values [slots][heads][...]."""
    page, off = slots // cache.page, slots % cache.page
    out = []
    for x, s, keys in ((cache.k, cache.k_scale, True), (cache.v, cache.v_scale, False)):
        x, s = x.cpu().numpy(), s.cpu().numpy()
        b = x[page, :, :, off].reshape(len(slots), cache.kv_heads, -1) if keys else x[page, :, off]
        codes = np.stack((b & 15, b >> 4), -1).reshape(len(slots), cache.kv_heads, cache.head_dim).astype(np.int64)
        out.append((codes, s[page, :, :, off].astype(np.int64)))
    return out


def cache_rows(cache, slots):
    """(k, v) rows [slots][heads][D] in 64 bits of any cache."""
    if cache.format != "mxfp4":
        return ref.cache_rows(cache, slots)
    return tuple(mxfp4_values(*x) for x in mxfp4_held(cache, slots))


def attention(q, k, v, scale, lo, hi, p, cap=0.0, slopes=None, rounded=True):
    """One row: q [heads][D] at position p over tokens lo <= t < hi of k, v [tokens][kv heads][D] -> (o, lse, bound of o, bound of lse).
    rounded: the weights enter the product as fp16 numbers, with a factor of 2^10."""
    heads, D = q.shape
    g = heads // k.shape[1]
    o, lse, bo, bl = np.zeros((heads, D)), np.full(heads, -np.inf), np.full((heads, D), ref.TINY), np.zeros(heads)
    lo, hi = max(lo, 0), min(hi, len(k))
    if lo >= hi:
        return o, lse, bo, bl
    away = np.abs(p - np.arange(lo, hi))
    for h in range(heads):
        qq, kk, vv = q[h].astype(np.float64), k[lo:hi, h // g], v[lo:hi, h // g]
        x = kk @ qq * scale
        # a score: D products summed in fp32, then two factors; fma, difference and logarithms' unit: 2^-22 of the largest in sight
        score = (D + 4) * 2.0 ** -24 * (np.abs(kk) @ np.abs(qq)) * abs(scale)
        if cap:
            x = cap * np.tanh(x / cap)
            # 2^-22 of tanh, and the factor; (1 - e) / (1 + e) of an e that is off by 2^-23 of itself: half of that where e is 1
            score = score + 2.0 ** -21 * np.abs(x) + (2.0 ** -24 * cap if cap <= 64 else 0)
        if slopes is not None:
            x = x - float(slopes[h]) * away
            score = score + 2.0 ** -22 * float(abs(slopes[h])) * away
        m = x.max()
        if m == -np.inf:
            continue
        w = np.exp(x - m)
        total = w.sum()
        o[h], lse[h] = w @ vv / total, m + np.log(total)
        # a token's weight is off by its score's error, the sum by the mean of them; scores that are far below the largest weigh nothing
        far = (w * score).sum() / total
        each = score + far + 2.0 ** -20 + 2.0 ** -22 * np.abs(x).max(where=w > 2.0 ** -40, initial=0) + (2.0 ** -11 if rounded else 0)
        bo[h] = ref.F16 * np.abs(o[h]) + ref.TINY + (w * each) @ np.abs(vv) / total
        if rounded:                                          # weights below 2^-24 of the largest lose bits, and end at 2^-35 of it
            bo[h] += 2.0 ** -35 * np.abs(vv).sum(0) / total
        bl[h] = far + 2.0 ** -20 + 2.0 ** -22 * (abs(lse[h]) + abs(m))
    return o, lse, bo, bl


def interval(p, n, window=0, first=0, prefix=0):
    """The tokens lo <= t < hi that a row at position p of a sequence of n tokens attends to."""
    return max(0, p - window + 1 if window else 0, first), max(p + 1, min(prefix, n), 0)
