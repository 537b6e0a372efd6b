"""Places of the cache that hold what is not finite, pages that are not there, and documents, in calls of few and of many rows, split and whole; the 64-bit form
and bounds: more_attention_ref.py."""
import numpy as np
import pytest

import more_attention_ref as more
from test_gpu_mxfp4_cache import cuda, filled, say, slopes_of, within
from test_gpu_prompt_attention import P, check, starts_of, workspace  # noqa: F401

pytestmark = pytest.mark.gpu

FORMATS = ["fp16", "e4m3", "mxfp4"]
# few rows, of which the second sequence is cut into parts; many, cut and whole
ROWS = {"few": ([3, 5], [77, 1500]), "cut": ([150], [4000]), "whole": ([90, 200, 130], [120, 333, 130])}
SCORES = {"plain": {}, "cap": dict(cap=20.0), "bias": dict(slopes=slopes_of(4)), "both": dict(cap=20.0, slopes=slopes_of(4), window=100)}


def spoil(cache, table, b, t, head, keys=False):
    """A value (or key) of one token and head becomes infinite or NaN; returns what was there."""
    page, off = int(table[b, t // cache.page]), t % cache.page
    if cache.format == "fp16":
        place = cache.k[page, head, :, off] if keys else cache.v[page, head, off]
        old = place.clone()
        place[...] = float("nan")
        if not keys:
            place[::2] = float("inf")
    elif cache.format == "e4m3":
        place = cache.k[page, head, :, off] if keys else cache.v[page, head, off]
        old = place.clone()
        place[...] = 0x7f
    else:
        place = (cache.k_scale if keys else cache.v_scale)[page, head, :, off]
        old = place.clone()
        place[...] = 255
    return place, old


@pytest.mark.parametrize("rows", list(ROWS))
@pytest.mark.parametrize("scores", list(SCORES))
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D", [64, 128, 256])
def test_not_finite(P, rows, scores, fmt, D):
    """Rows that attend to such a token have no finite result in its head, all others what they had."""
    say(f"{rows} rows, {scores}, {fmt} x {D}")
    hq, hkv = 4, 4 if rows == "few" else 2
    new, lengths = ROWS[rows]
    cache, table, _ = filled(P, lengths, hkv, D, 16, fmt, 6)
    T, B = sum(new), len(new)
    q = cuda(np.random.default_rng(8).standard_normal((T, hq * D)).astype(np.float16))
    starts, tb, ln, ws = cuda(starts_of(new)), cuda(table), cuda(np.array(lengths, np.int32)), workspace(P, cache, hq, T, B)
    kw = {k: cuda(v) if isinstance(v, np.ndarray) else v for k, v in SCORES[scores].items()}
    window = kw.get("window", 0)
    call = lambda: [x.cpu().numpy() for x in P.paro_prompt_attention(cache, q, starts, tb, ln, ws, with_lse=True, **kw)]  # noqa: E731
    clean, clean_lse = call()
    assert np.isfinite(clean).all() and np.isfinite(clean_lse).all()
    b, n, m = B - 1, lengths[-1], new[-1]
    p = np.concatenate([np.full(k, -1) for k in new[:-1]] + [np.arange(n - m, n)])      # positions in the sequence that is spoiled
    for t in sorted({0, n // 3, n - m - 1, n - m, n - m + 1, n - m // 2, n - 2, n - 1} & set(range(n))):
        sees = (p >= t) & ((p < t + window) | (window == 0))
        for keys in (False, True):
            place, old = spoil(cache, table, b, t, 1, keys)
            o, lse = call()
            place[...] = old
            mine = np.zeros((T, hq), bool)
            mine[sees, hq // hkv:2 * (hq // hkv)] = True
            got, was = o.reshape(T, hq, D), clean.reshape(T, hq, D)
            assert not np.isfinite(got[mine]).any(), (t, keys)
            assert np.array_equal(got[~mine], was[~mine]), (t, keys)
            assert np.array_equal(lse[~mine], clean_lse[~mine]) and (np.isnan(lse[mine]).all() if keys else np.array_equal(lse, clean_lse)), (t, keys)
    assert all(np.array_equal(x, y) for x, y in zip(call(), (clean, clean_lse)))
    assert ws.partials_clean(P.paro_workspace_exchange_bytes_prompt(cache, hq, T, B))


@pytest.mark.parametrize("rows", list(ROWS))
@pytest.mark.parametrize("cap", [0.0, 15.0])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D,page", [(64, 16), (128, 64), (256, 16)])
def test_pages_that_are_not_there(P, rows, cap, fmt, D, page):
    say(f"{rows} rows, cap {cap}, {fmt} x {D}, page {page}")
    hq, hkv = 4, 4 if rows == "few" else 2
    new, lengths = ROWS[rows]
    cache, table, held = filled(P, lengths, hkv, D, page, fmt, 9)
    gone = [sorted({0, (n // page) // 2, (n // page) // 2 + 1, (n - 1) // page} & set(range((n - 1) // page + 1))) for n in lengths]
    for b, pages in enumerate(gone):
        table[b, pages] = [(-1, cache.n_pages, 2 ** 31 - 1, -2 ** 31)[i] for i in range(len(pages))]
    T = sum(new)
    q = np.random.default_rng(2).standard_normal((T, hq * D)).astype(np.float16)
    o, lse = P.paro_prompt_attention(cache, cuda(q), cuda(starts_of(new)), cuda(table), cuda(np.array(lengths, np.int32)), workspace(P, cache, hq, T, len(new)), cap=cap,
                                     with_lse=True)
    want, r = [], 0
    for b, (m, n) in enumerate(zip(new, lengths)):
        for p in range(n - m, n):
            t = np.flatnonzero(~np.isin(np.arange(p + 1) // page, gone[b]))
            want.append(more.attention(q[r].reshape(hq, D), held[b][0][t], held[b][1][t], D ** -0.5, 0, len(t), p, cap))
            r += 1
    o_ref, l_ref, o_bound, l_bound = (np.stack([w[i] for w in want]) for i in range(4))
    within(o.cpu().numpy().reshape(T, hq, D), o_ref, o_bound, "o")
    got, some = lse.cpu().numpy(), np.isfinite(l_ref)
    assert np.array_equal(got[~some], l_ref[~some])
    within(got[some], l_ref[some], l_bound[some], "lse")


@pytest.mark.parametrize("prefix,window", [(None, 0), ([3, 9, 200, 2 ** 31 - 1], 0), ([3, 9, 200, 70], 25)])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D,hq,hkv", [(64, 4, 4), (128, 6, 2), (256, 2, 2)])
def test_documents_of_few_rows(P, prefix, window, fmt, D, hq, hkv):
    say(f"documents of few rows, {fmt} {hq}/{hkv} x {D}, prefix {prefix}, window {window}")
    new, lengths = [1, 3, 7, 5], [1, 40, 300, 1500]
    first = np.array([0, 38, 40, 38, 0, 295, 120, 297, -5, 298, 1000, 1496, 0, 1499, 64, 1499], np.int32)     # 40: nothing of its own; 1000: beyond the row
    case = filled(P, lengths, hkv, D, 16, fmt, 4)
    check(P, *case, new, lengths, hq, 5, first=first, prefix=prefix, window=window)
    check(P, *case, new, lengths, hq, 6, first=first, prefix=prefix, window=window, cap=12.0, slopes=slopes_of(hq))
