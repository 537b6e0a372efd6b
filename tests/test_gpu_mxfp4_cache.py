"""The MXFP4 key-value cache (append and attention of one token) and the scores of attention, against 64-bit forms; bounds: more_attention_ref.py."""
import numpy as np
import pytest

import more_attention_ref as more
import token_path_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2511_10645_amd as paro
    return paro


def say(msg):
    print(msg, flush=True)


def cuda(x):
    import torch
    return torch.as_tensor(x).cuda()


def within(got, want, bound, what):
    err = np.abs(got.astype(np.float64) - want)
    worst = float(np.max(err / bound)) if err.size else 0.0
    say(f"  {what}: worst err/bound {worst:.3f}")
    assert worst <= 1.0


def awkward(rs, T, heads, D):
    """fp16 rows with zeros, numbers that lie between two codes, far ones, subnormal ones and the largest."""
    x = rs.standard_normal((T, heads, D)).astype(np.float16)
    x[0] = 0
    if T > 1:
        x[1, :, :32] = np.resize(np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6, 7, 7.9, -0.25, -5, -2.5, 0, -0.0, 4], np.float16), 32)
        x[1, :, 32:64] *= np.float16(2.0 ** -12)
    if T > 2:
        x[2, :, ::7] = 65504
        x[2, :, 32:64] = np.float16(2.0 ** -24)
    if T > 3:
        x[3] *= np.float16(2.0 ** -14)
        x[3, :, 5] = -65504
    return x


@pytest.mark.parametrize("T,hkv,D,page", [(1, 1, 64, 16), (3, 2, 128, 16), (37, 8, 128, 32), (5, 3, 256, 64), (1030, 2, 64, 128), (1027, 8, 128, 16)])
def test_append_holds_the_conversion(P, T, hkv, D, page):
    import torch
    say(f"append {T} x {hkv} x {D}, page {page}")
    rs = np.random.default_rng(T + D)
    k, v = awkward(rs, T, hkv, D), awkward(rs, T, hkv, D)[::-1].copy()
    n_pages = -(-T // page) + 3
    cache = P.KVCache(n_pages, hkv, D, page, "mxfp4")
    slots = rs.permutation(n_pages * page)[:T].astype(np.int64)
    before = [x.clone() for x in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    P.paro_kv_append(cache, cuda(k.reshape(T, -1)), cuda(v.reshape(T, -1)), cuda(slots))
    for (codes, scales), x in zip(more.mxfp4_held(cache, slots), (k, v)):
        want, s = more.mxfp4(x.astype(np.float64))
        assert np.array_equal(scales, s)
        assert np.array_equal(more.mxfp4_values(codes, scales), more.mxfp4_values(want, s))
        held = more.mxfp4_values(codes, scales)
        assert np.array_equal(held.astype(np.float16).astype(np.float64), held)        # all are fp16 values
    others = np.setdiff1d(np.arange(n_pages * page), slots)
    after = [x.cpu().numpy() for x in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    for x, y, at in zip(before, after, ((0, 3), (0, 2), (0, 3), (0, 3))):
        x, y = (np.moveaxis(z, at[1], 1).reshape(n_pages * page, -1) for z in (x.cpu().numpy(), y))
        assert np.array_equal(x[others], y[others])                     # and no other place is written
    torch.cuda.synchronize()


@pytest.mark.parametrize("D,rot,layout", [(128, 128, "halves"), (128, 48, "halves"), (64, 16, "halves"), (256, 256, "halves"), (256, 112, "halves"),
                                          (128, 128, "interleaved"), (64, 32, "interleaved")])
def test_append_rotates(P, D, rot, layout):
    say(f"append rotated {rot} of {D}, {layout}")
    T, hkv, hq = 19, 3, 6
    rs = np.random.default_rng(rot + D)
    k, v, q = (rs.standard_normal((T, h, D)).astype(np.float16) for h in (hkv, hkv, hq))
    f = (10000.0 ** (-np.arange(0, rot, 2) / rot)).astype(np.float32)
    pos = rs.integers(0, 100000, T).astype(np.int32)
    cache, rope = P.KVCache(4, hkv, D, 16, "mxfp4"), P.Rope(f, D, layout, 1.25)
    slots = rs.permutation(64)[:T].astype(np.int64)
    slots[3] = -1                                                       # padding
    qr = P.paro_kv_append(cache, cuda(k.reshape(T, -1)), cuda(v.reshape(T, -1)), cuda(slots), rope, cuda(pos), cuda(q.reshape(T, -1)))
    q_ref = ref.rotate(q, pos, f, layout, 1.25)
    within(qr.cpu().numpy().reshape(T, hq, D), q_ref, ref.rotate_bound(q, q_ref, f, layout, 1.25), "q")
    live = slots >= 0
    (kc, ks), (vc, vs) = more.mxfp4_held(cache, slots[live])
    want, s = more.mxfp4(v[live].astype(np.float64))
    assert np.array_equal(vs, s) and np.array_equal(more.mxfp4_values(vc, vs), more.mxfp4_values(want, s))
    # keys: the 64-bit value and the kernel's lie 2^-21 of what went into a channel apart, so the code is one of those that values so near have
    k_ref = ref.rotate(k, pos, f, layout, 1.25)[live]
    slack = ref.rotate_bound(k, ref.rotate(k, pos, f, layout, 1.25), f, layout, 1.25)[live] - ref.F16 * np.abs(k_ref) - ref.TINY
    most = np.abs(k_ref).reshape(*k_ref.shape[:-1], -1, 32).max(-1)
    assert (np.abs(ks - (more.mxfp4_exponent(most) + 127)) * (np.abs(np.log2(most) - np.round(np.log2(most))) > 1e-5) == 0).all()
    unit = np.repeat(2.0 ** (ks - 127.0), 32, -1)
    lo, hi = (more.mxfp4_codes(np.maximum(np.abs(k_ref) + sign * slack, 0) / unit) for sign in (-1, 1))
    assert ((lo <= (kc & 7)) & ((kc & 7) <= hi)).all()
    assert (((kc & 8) != 0) == (k_ref < 0))[(kc & 7) > 0].all()


def test_append_not_finite(P):
    say("NaN and infinities mark their 32 channels")
    T, hkv, D = 5, 2, 128
    rs = np.random.default_rng(3)
    k, v = (rs.standard_normal((T, hkv, D)).astype(np.float16) for _ in range(2))
    k[1, 0, 40], k[2, 1, 127], v[3, 1, 0], v[4, 0, 95] = np.nan, np.inf, -np.inf, np.nan
    cache = P.KVCache(2, hkv, D, 16, "mxfp4")
    slots = np.array([7, 3, 20, 31, 0])
    P.paro_kv_append(cache, cuda(k.reshape(T, -1)), cuda(v.reshape(T, -1)), cuda(slots))
    for (codes, scales), x in zip(more.mxfp4_held(cache, slots), (k, v)):
        want, s = more.mxfp4(x.astype(np.float64))
        assert np.array_equal(scales, s)
        got, want = more.mxfp4_values(codes, scales), more.mxfp4_values(want, s)
        assert np.array_equal(got, want, equal_nan=True) and np.isnan(got).sum() == 64


def filled(P, lengths, hkv, D, page, fmt, seed, spread=1.0):
    """A cache that holds sequences of these lengths on scattered pages: (cache, table, [(k, v) as held])."""
    rs = np.random.default_rng(seed)
    held = [max(0, -(-n // page)) for n in lengths]
    n_pages, width = sum(held) + 2, max(1, max(held))
    order = rs.permutation(n_pages)
    table = np.full((len(lengths), width), -1, np.int32)
    at, slots = 0, []
    for i, (n, h) in enumerate(zip(lengths, held)):
        table[i, :h] = order[at:at + h]
        at += h
        t = np.arange(n)
        slots.append(table[i, t // page].astype(np.int64) * page + t % page)
    cache = P.KVCache(n_pages, hkv, D, page, fmt)
    total = sum(lengths)
    if total:
        k, v = ((rs.standard_normal((total, hkv * D)) * spread).astype(np.float16) for _ in range(2))
        v += np.float16(0.25)
        P.paro_kv_append(cache, cuda(k), cuda(v), cuda(np.concatenate(slots)))
    rows = [more.cache_rows(cache, s) if len(s) else (np.zeros((0, hkv, D)),) * 2 for s in slots]
    return cache, table, rows


def check(P, cache, table, rows, lengths, hq, seed, window=0, cap=0.0, slopes=None, spread=1.0, scale=None):
    B, D = len(lengths), cache.head_dim
    scale = D ** -0.5 if scale is None else scale
    q = (np.random.default_rng(seed).standard_normal((B, hq * D)) * spread).astype(np.float16)
    ws = P.Workspace(P.paro_workspace_bytes_attention(cache, hq, B))
    o, lse = P.paro_paged_attention(cache, cuda(q), cuda(table), cuda(np.asarray(lengths, np.int32)), ws, scale, window, with_lse=True, cap=cap,
                                    slopes=None if slopes is None else cuda(slopes))
    want = [more.attention(q[i].reshape(hq, D), *rows[i], scale, *more.interval(n - 1, n, window), n - 1, cap, slopes, rounded=False) for i, n in enumerate(lengths)]
    within(o.cpu().numpy().reshape(B, hq, D), np.stack([w[0] for w in want]), np.stack([w[2] for w in want]), "o")
    l_ref, l_bound, got = np.stack([w[1] for w in want]), np.stack([w[3] for w in want]), lse.cpu().numpy()
    some = np.isfinite(l_ref)
    assert np.array_equal(got[~some], l_ref[~some])
    within(got[some], l_ref[some], l_bound[some], "lse")
    assert ws.partials_clean(P.paro_workspace_exchange_bytes_attention(cache, hq, B)) and ws.error_word() == 0


def slopes_of(hq):
    return (2.0 ** (-8 * np.arange(1, hq + 1) / hq)).astype(np.float32)


EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 64, 65, 127, 129, 257]


@pytest.mark.parametrize("hq,hkv,D,page", [(4, 1, 64, 16), (8, 2, 128, 16), (5, 5, 128, 64), (40, 8, 128, 32), (17, 1, 64, 128), (6, 2, 256, 16), (16, 1, 256, 1024)])
def test_attention_mxfp4_lengths(P, hq, hkv, D, page):
    say(f"mxfp4 {hq}/{hkv} x {D}, page {page}")
    check(P, *filled(P, EDGES, hkv, D, page, "mxfp4", hq + D), EDGES, hq, 1)


@pytest.mark.parametrize("n,hq,hkv,D,page", [(5003, 8, 2, 128, 16), (20011, 4, 1, 64, 32), (9001, 6, 2, 256, 16)])
def test_attention_mxfp4_long(P, n, hq, hkv, D, page):
    say(f"mxfp4 of {n} tokens, {hq}/{hkv} x {D}")
    check(P, *filled(P, [n, 3], hkv, D, page, "mxfp4", n), [n, 3], hq, 2, window=0)
    check(P, *filled(P, [n], hkv, D, page, "mxfp4", n + 1), [n], hq, 2, window=1000)


@pytest.mark.parametrize("fmt", ["fp16", "e4m3", "mxfp4"])
@pytest.mark.parametrize("D,hq,hkv", [(64, 6, 2), (128, 8, 2), (256, 4, 2)])
@pytest.mark.parametrize("cap,bias,window", [(30.0, False, 0), (0.0, True, 0), (5.0, True, 70), (1e6, False, 0), (0.5, False, 0)])
def test_attention_scores(P, fmt, D, hq, hkv, cap, bias, window):
    say(f"{fmt} {hq}/{hkv} x {D} cap {cap} bias {bias} window {window}")
    lengths = [1, 2, 33, 64, 700, 0, 1300]
    check(P, *filled(P, lengths, hkv, D, 16, fmt, D + hq), lengths, hq, 3, window, cap, slopes_of(hq) if bias else None, spread=4.0)


def test_attention_scores_signs(P):
    say("negative and zero scales, slopes of either sign and zero, scores far beyond the cap")
    case = filled(P, [50, 333], 2, 128, 16, "fp16", 9)
    for scale, cap, slopes in ((-0.1, 20.0, None), (0.0, 20.0, None), (0.1, 0.0, np.array([0, -0.01, 0.5, 1], np.float32)), (100.0, 3.0, slopes_of(4)),
                               (1e-8, 1e-6, None)):
        check(P, *case, [50, 333], 4, 4, 0, cap, slopes, scale=scale)


def test_attention_mxfp4_masked_places_hold_anything(P):
    import torch
    say("scale bytes of 255 behind the last token, before the window and on pages that are not there")
    hq, hkv, D, page = 8, 2, 128, 16
    for n, window in ((37, 0), (300, 100), (1, 0)):
        cache, table, rows = filled(P, [n], hkv, D, page, "mxfp4", n)
        q, ln = cuda(np.random.default_rng(n).standard_normal((1, hq * D)).astype(np.float16)), cuda(np.array([n], np.int32))
        ws = P.Workspace(P.paro_workspace_bytes_attention(cache, hq, 1))
        want = P.paro_paged_attention(cache, q, cuda(table), ln, ws, window=window, with_lse=True)
        keep = {int(table[0, t // page]) * page + t % page for t in range(max(0, n - window) if window else 0, n)}
        for s in range(cache.n_pages * page):
            if s not in keep:
                cache.k_scale[s // page, :, :, s % page] = 255
                cache.v_scale[s // page, :, :, s % page] = 255
        got = P.paro_paged_attention(cache, q, cuda(table), ln, ws, window=window, with_lse=True)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    bad = table.copy()
    bad[0, 0] = 2 ** 30
    o, lse = P.paro_paged_attention(cache, q, cuda(bad), ln, ws, with_lse=True)
    assert (o == 0).all() and (lse == -np.inf).all()


def test_attention_mxfp4_not_finite(P):
    say("a value of NaN spoils its 32 channels, a key of NaN its head's rows")
    hq, hkv, D, n = 4, 2, 128, 70
    cache, table, rows = filled(P, [n], hkv, D, 16, "mxfp4", 1)
    q, ln = cuda(np.random.default_rng(1).standard_normal((1, hq * D)).astype(np.float16)), cuda(np.array([n], np.int32))
    ws = P.Workspace(P.paro_workspace_bytes_attention(cache, hq, 1))
    clean = P.paro_paged_attention(cache, q, cuda(table), ln, ws).cpu().numpy().reshape(hq, D)
    cache.v_scale[int(table[0, 2]), 1, 3, 5] = 255
    o = P.paro_paged_attention(cache, q, cuda(table), ln, ws).cpu().numpy().reshape(hq, D)
    assert np.isnan(o[2:, 96:]).all() and np.array_equal(o[:2], clean[:2]) and np.array_equal(o[2:, :96], clean[2:, :96])
    cache.v_scale[int(table[0, 2]), 1, 3, 5] = 127
    cache.k_scale[int(table[0, 4]), 0, 1, 2] = 255
    o = P.paro_paged_attention(cache, q, cuda(table), ln, ws).cpu().numpy().reshape(hq, D)
    assert np.isnan(o[:2]).all() and np.isfinite(o[2:]).all()


def test_attention_mxfp4_far_pages(P):
    import torch
    say("pages behind 4 GiB of the cache")
    hq, hkv, D, page, n = 8, 8, 256, 1024, 1500
    n_pages = 5000                                                      # 1 MiB of codes and 64 KiB of scales a page, each
    cache = P.KVCache(n_pages, hkv, D, page, "mxfp4")
    rs = np.random.default_rng(2)
    table = np.array([[n_pages - 1, n_pages - 2]], np.int32)
    k, v = (rs.standard_normal((n, hkv * D)).astype(np.float16) for _ in range(2))
    t = np.arange(n)
    slots = table[0, t // page].astype(np.int64) * page + t % page
    P.paro_kv_append(cache, cuda(k), cuda(v), cuda(slots))
    small = P.KVCache.from_device(*(x[n_pages - 2:].clone() for x in (cache.k, cache.v, cache.k_scale, cache.v_scale)))
    want, s = more.mxfp4(k.reshape(n, hkv, D).astype(np.float64))
    codes, scales = more.mxfp4_held(small, slots - (n_pages - 2) * page)[0]
    assert np.array_equal(scales, s) and np.array_equal(more.mxfp4_values(codes, scales), more.mxfp4_values(want, s))
    q, ln = cuda(rs.standard_normal((1, hq * D)).astype(np.float16)), cuda(np.array([n], np.int32))
    ws = P.Workspace(max(P.paro_workspace_bytes_attention(cache, hq, 1), P.paro_workspace_bytes_prompt(cache, hq, 1, 1)))
    starts = cuda(np.array([0, 1], np.int32))
    for call in (lambda c, tb: P.paro_paged_attention(c, q, tb, ln, ws), lambda c, tb: P.paro_prompt_attention(c, q, starts, tb, ln, ws)):
        assert torch.equal(call(cache, cuda(table)), call(small, cuda(table - (n_pages - 2))))
