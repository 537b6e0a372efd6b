"""Plain 64-bit forms of the operators between the linears, and the bounds that a kernel's results are held to.

An fp16 result of fp32 arithmetic is off by half a unit in its last place, 2^-11 of its size (2^-25 where it is subnormal), plus what
the fp32 steps before it lose; every bound below is that sum, with the fp32 part written out at its place."""
import numpy as np

F16 = 2.0 ** -11 * (1 + 2.0 ** -6)                   # half a unit of fp16, and an fp32 error of some units before it
TINY = 2.0 ** -25 * (1 + 2.0 ** -6)


def e4m3_values():
    """The value of every E4M3 byte: 1 sign, 4 exponent (bias 7), 3 mantissa bits; 0x7f and 0xff are NaN."""
    b = np.arange(256)
    e, m = (b >> 3) & 15, b & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v[(b & 127) == 127] = np.nan
    return np.where(b & 128, -v, v)


def half_step(q):
    """Half the distance of E4M3's numbers around |q|."""
    e = np.floor(np.log2(np.maximum(np.abs(q), 2.0 ** -6)))
    return 2.0 ** (e - 4)


def rms_norm(x, r, w, eps):
    h = x.astype(np.float64) + (0 if r is None else r.astype(np.float64))
    return h, h / np.sqrt((h * h).mean(1, keepdims=True) + eps) * w.astype(np.float64)


def rotate(x, positions, inv_freq, layout, magnitude):
    """x [T][heads][D] in 64 bits."""
    y = x.astype(np.float64).copy()
    n = len(inv_freq)
    a = positions.astype(np.float64)[:, None] * inv_freq.astype(np.float64)
    c, s = np.cos(a)[:, None] * magnitude, np.sin(a)[:, None] * magnitude
    ia, ib = (np.arange(n), np.arange(n, 2 * n)) if layout == "halves" else (np.arange(0, 2 * n, 2), np.arange(1, 2 * n, 2))
    p, q = y[..., ia].copy(), y[..., ib].copy()
    y[..., ia], y[..., ib] = p * c - q * s, p * s + q * c
    return y


def rotate_bound(x, ref, inv_freq, layout, magnitude):
    """Half a unit of the result, and 2^-21 of what went into a channel for sine, cosine, products and sum in fp32."""
    n = len(inv_freq)
    into = np.abs(x.astype(np.float64)).copy()
    ia, ib = (np.arange(n), np.arange(n, 2 * n)) if layout == "halves" else (np.arange(0, 2 * n, 2), np.arange(1, 2 * n, 2))
    both = (into[..., ia] + into[..., ib]) * abs(magnitude)
    into[...] = 0
    into[..., ia] = into[..., ib] = both
    return F16 * np.abs(ref) + TINY + 2.0 ** -21 * into


def cache_rows(cache, slots):
    """(k, v) rows [slots][heads][D] in 64 bits, out of a cache's tensors."""
    page, off = slots // cache.page, slots % cache.page
    k = cache.k.cpu().numpy()[page, :, :, off].reshape(len(slots), cache.kv_heads, cache.head_dim)
    v = cache.v.cpu().numpy()[page, :, off]
    if cache.format == "fp16":
        return k.astype(np.float64), v.astype(np.float64)
    table = e4m3_values()
    ks, vs = (s.cpu().numpy()[page, :, off].astype(np.float64)[..., None] for s in (cache.k_scale, cache.v_scale))
    return table[k] * 2.0 ** (ks - 127), table[v] * 2.0 ** (vs - 127)


def attention(q, k, v, scale):
    """q [heads][D], k, v [tokens][kv heads][D] -> (o, lse, bound of o, bound of lse)."""
    heads, D = q.shape
    g = heads // k.shape[1]
    o, lse, bo, bl = np.zeros((heads, D)), np.full(heads, -np.inf), np.full((heads, D), TINY), np.zeros(heads)
    if not len(k):
        return o, lse, bo, bl
    for h in range(heads):
        qq, kk, vv = q[h].astype(np.float64), k[:, h // g], v[:, h // g]
        x = kk @ qq * scale
        m = x.max()
        if m == -np.inf:
            continue
        p = np.exp(x - m)
        total = p.sum()
        o[h], lse[h] = p @ vv / total, m + np.log(total)
        # a score: D products summed in fp32, then two factors; a weight: twice that (itself and the sum it is divided by)
        score = ((D + 4) * 2.0 ** -24 * (np.abs(kk) @ np.abs(qq)) * abs(scale)).max()
        each = 2 * score + 2.0 ** -20
        bo[h] = F16 * np.abs(o[h]) + TINY + 2 * each * (p @ np.abs(vv)) / total
        bl[h] = score + 2.0 ** -20 + 2.0 ** -22 * abs(lse[h])
    return o, lse, bo, bl
