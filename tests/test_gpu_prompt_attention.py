"""paro_prompt_attention against a 64-bit form; bounds: more_attention_ref.py."""
import numpy as np
import pytest

import more_attention_ref as more
from test_gpu_mxfp4_cache import cuda, filled, say, slopes_of, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2511_10645_amd as paro
    return paro


def starts_of(new):
    return np.concatenate(([0], np.cumsum(new))).astype(np.int32)


def workspace(P, cache, hq, T, B):
    return P.Workspace(P.paro_workspace_bytes_prompt(cache, hq, T, B))


def wanted(q, rows, new, lengths, hq, scale, window=0, cap=0.0, slopes=None, prefix=None, first=None):
    D = q.shape[1] // hq
    out, r = [], 0
    for b, (m, n) in enumerate(zip(new, lengths)):
        for i in range(m):
            p = n - m + i
            lo, hi = more.interval(p, n, window, 0 if first is None else int(first[r]), 0 if prefix is None else int(prefix[b]))
            out.append(more.attention(q[r].reshape(hq, D), *rows[b], scale, lo, hi, p, cap, slopes))
            r += 1
    return [np.stack([w[i] for w in out]) for i in range(4)]


def check(P, cache, table, rows, new, lengths, hq, seed=0, window=0, cap=0.0, slopes=None, prefix=None, first=None, spread=1.0, scale=None, q=None, ws=None):
    B, D, T = len(lengths), cache.head_dim, sum(new)
    scale = D ** -0.5 if scale is None else scale
    if q is None:
        q = (np.random.default_rng(seed).standard_normal((T, hq * D)) * spread).astype(np.float16)
    maybe = lambda x, kind: None if x is None else cuda(np.asarray(x, kind))  # noqa: E731
    ws = ws or workspace(P, cache, hq, T, B)
    o, lse = P.paro_prompt_attention(cache, cuda(q), cuda(starts_of(new)), cuda(table), cuda(np.asarray(lengths, np.int32)), ws, scale, window, cap,
                                     maybe(slopes, np.float32), maybe(prefix, np.int32), maybe(first, np.int32), with_lse=True)
    o_ref, l_ref, o_bound, l_bound = wanted(q, rows, new, lengths, hq, scale, window, cap, slopes, prefix, first)
    within(o.cpu().numpy().reshape(T, hq, D), o_ref, o_bound, "o")
    got = lse.cpu().numpy()
    some = np.isfinite(l_ref)
    assert np.array_equal(got[~some], l_ref[~some])
    within(got[some], l_ref[some], l_bound[some], "lse")
    assert ws.partials_clean(P.paro_workspace_exchange_bytes_prompt(cache, hq, T, B)) and ws.error_word() == 0
    return o, lse


@pytest.mark.parametrize("fmt", ["fp16", "e4m3", "mxfp4"])
@pytest.mark.parametrize("hq,hkv,D,page", [(4, 1, 64, 16), (8, 2, 128, 16), (3, 3, 128, 64), (10, 2, 128, 128), (7, 1, 64, 32), (6, 2, 256, 16), (20, 1, 256, 1024)])
def test_lengths(P, fmt, hq, hkv, D, page):
    say(f"{fmt} {hq}/{hkv} x {D}, page {page}")
    new = [1, 0, 2, 15, 16, 17, 33, 64, 1, 65]
    lengths = [1, 0, 2, 40, 16, 17, 33, 129, 300, 65]
    check(P, *filled(P, lengths, hkv, D, page, fmt, hq + D), new, lengths, hq)


@pytest.mark.parametrize("fmt", ["fp16", "e4m3", "mxfp4"])
@pytest.mark.parametrize("hq,hkv,D,page", [(2, 2, 64, 16), (5, 1, 128, 32), (8, 1, 256, 16)])
def test_few_rows(P, fmt, hq, hkv, D, page):
    say(f"few rows of many sequences, {fmt} {hq}/{hkv} x {D}, page {page}")
    new = [1, 3, 0, 7, 5, 2, 1, 4, 6, 1, 2, 3]
    lengths = [1, 3, 0, 7, 33, 64, 65, 127, 128, 129, 300, 1500]
    check(P, *filled(P, lengths, hkv, D, page, fmt, hq + D), new, lengths, hq)
    check(P, *filled(P, lengths, hkv, D, page, fmt, hq + D), new, lengths, hq, window=50, cap=9.0)


@pytest.mark.parametrize("fmt,D,hq,hkv,new,held", [("fp16", 128, 8, 2, 200, 0), ("fp16", 128, 8, 2, 5, 5003), ("mxfp4", 128, 4, 1, 3, 20011), ("e4m3", 64, 16, 1, 9, 9001),
                                                   ("fp16", 256, 4, 2, 67, 4000), ("mxfp4", 256, 4, 2, 1, 4001), ("fp16", 64, 2, 2, 513, 500)])
def test_long(P, fmt, D, hq, hkv, new, held):
    say(f"{new} rows behind {held} tokens, {fmt} {hq}/{hkv} x {D}")
    case = filled(P, [held + new], hkv, D, 16, fmt, held + D)
    a = check(P, *case, [new], [held + new], hq, 1)
    b = check(P, *case, [new], [held + new], hq, 1)
    assert all((x == y).all() for x, y in zip(a, b))


MASKS = [dict(window=1), dict(window=40), dict(prefix=[0, 30, 500, 2]), dict(prefix=[5, 1, 64, 2 ** 31 - 1], window=20), dict(documents=True), dict(documents=True, window=9),
         dict(documents=True, prefix=[9, 0, 100, 3])]


@pytest.mark.parametrize("mask", range(len(MASKS)))
@pytest.mark.parametrize("fmt,D,hq,hkv", [("fp16", 128, 4, 2), ("e4m3", 64, 5, 1), ("mxfp4", 128, 4, 4)])
def test_masks(P, mask, fmt, D, hq, hkv):
    say(f"{MASKS[mask]} {fmt}")
    m = dict(MASKS[mask])
    new, lengths = [70, 31, 150, 1], [70, 90, 333, 40]
    if m.pop("documents", False):
        rs = np.random.default_rng(mask)
        m["first"] = np.concatenate([np.maximum.accumulate(np.where(rs.random(k) < 0.1, np.arange(n - k, n), 0)) for k, n in zip(new, lengths)])
        m["first"][5] = 1000                                            # a row with nothing to attend to
        m["first"][100] = -7
    check(P, *filled(P, lengths, hkv, D, 16, fmt, mask), new, lengths, hq, 2, **m)


@pytest.mark.parametrize("fmt", ["fp16", "e4m3", "mxfp4"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("cap,bias,window", [(30.0, False, 0), (0.0, True, 0), (4.0, True, 50), (1e6, False, 0)])
def test_scores(P, fmt, D, cap, bias, window):
    say(f"{fmt} x {D} cap {cap} bias {bias} window {window}")
    new, lengths, hq = [50, 1, 70], [50, 400, 100], 4
    check(P, *filled(P, lengths, 2, D, 16, fmt, D), new, lengths, hq, 3, window, cap, slopes_of(hq) if bias else None, prefix=[20, 0, 90] if bias else None, spread=4.0)


def test_scales(P):
    say("negative, zero and large scales; scores beyond 2^16 and beyond 2^24")
    new, lengths = [40, 3], [100, 77]
    case = filled(P, lengths, 2, 128, 16, "fp16", 4)
    for scale in (-0.1, 0.0, 1.0, 30.0):
        check(P, *case, new, lengths, 4, 5, scale=scale)
    check(P, *case, new, lengths, 4, 5, scale=-0.1, cap=3.0)
    check(P, *case, new, lengths, 4, 5, scale=0.0, slopes=slopes_of(4))


def test_huge_scores(P):
    """Two keys whose scores are far apart or equal: weights 1 and 0, or even ones, at any finite size."""
    import torch
    D = 64
    for size, scale in ((2.0 ** 12, 1.0), (2.0 ** 15, 1.0), (2.0 ** 15, 2.0 ** 20), (2.0 ** 15, -2.0 ** 20)):
        say(f"scores of {size * size * scale:g}")
        k, v = torch.zeros((40, D), dtype=torch.float16, device="cuda"), torch.zeros((40, D), dtype=torch.float16, device="cuda")
        k[:, 0] = size
        k[20:, 0] = -size
        v[:20, 0], v[20:, 0] = 1, -3
        cache = P.KVCache(3, 1, D, 16)
        P.paro_kv_append(cache, k, v, torch.arange(40, device="cuda"))
        q = torch.zeros((40, D), dtype=torch.float16, device="cuda")
        q[:, 0] = size
        o, lse = P.paro_prompt_attention(cache, q, cuda(np.array([0, 40], np.int32)), cuda(np.array([[0, 1, 2]], np.int32)), cuda(np.array([40], np.int32)),
                                         workspace(P, cache, 1, 40, 1), scale, with_lse=True)
        p = np.arange(40)
        ones, threes = np.minimum(p + 1, 20), np.maximum(p - 19, 0)
        want = np.where(threes > 0, -3.0, 1.0) if scale < 0 else np.ones(40)
        n = np.where((threes > 0) & (scale < 0), threes, ones)
        assert np.array_equal(o[:, 0].cpu().numpy(), want.astype(np.float16))
        x = np.where((threes > 0) | (scale > 0), abs(size * size * scale), size * size * scale)
        l_ref = x + np.log(n)
        assert (np.abs(lse[:, 0].cpu().numpy() - l_ref) <= 2.0 ** -22 * np.abs(l_ref) + 2.0 ** -20).all()


def test_infinite_scores(P):
    import torch
    say("scores of -inf weigh nothing; a row of them gives zeros")
    D = 64
    k, v = torch.zeros((20, D), dtype=torch.float16, device="cuda"), torch.ones((20, D), dtype=torch.float16, device="cuda")
    k[:, 0] = -float("inf")
    k[7, 0] = 1
    cache = P.KVCache(2, 1, D, 16)
    P.paro_kv_append(cache, k, v, torch.arange(20, device="cuda"))
    q = torch.zeros((20, D), dtype=torch.float16, device="cuda")
    q[:, 0] = 1
    q[:, 1:] = 1
    o, lse = P.paro_prompt_attention(cache, q, cuda(np.array([0, 20], np.int32)), cuda(np.array([[0, 1]], np.int32)), cuda(np.array([20], np.int32)),
                                     workspace(P, cache, 1, 20, 1), 1.0, with_lse=True)
    assert (o[:7] == 0).all() and (lse[:7] == -np.inf).all() and (o[7:] == 1).all() and (lse[7:] - 1).abs().max() < 2.0 ** -19


@pytest.mark.parametrize("fmt", ["fp16", "e4m3", "mxfp4"])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_masked_places_hold_anything(P, fmt, D):
    import torch
    say(f"NaN behind the last token, after a row's own and before its window, {fmt} x {D}")
    hq, hkv, page = 4, 2, 16
    new, lengths = [50, 90], [77, 200]
    cache, table, rows = filled(P, lengths, hkv, D, page, fmt, 6)
    q = cuda(np.random.default_rng(8).standard_normal((140, hq * D)).astype(np.float16))
    starts, tb, ln, ws = cuda(starts_of(new)), cuda(table), cuda(np.array(lengths, np.int32)), workspace(P, cache, hq, 140, 2)
    call = lambda window=0: [x.cpu().numpy() for x in P.paro_prompt_attention(cache, q, starts, tb, ln, ws, window=window, with_lse=True)]  # noqa: E731
    clean, clean_w = call(), call(30)

    def spoil(slot, keys, values):
        page_, off = slot // page, slot % page
        if fmt == "fp16":
            if keys:
                cache.k[page_, :, :, off] = float("nan")
            if values:
                cache.v[page_, :, off, :D // 2] = float("inf")
                cache.v[page_, :, off, D // 2:] = float("nan")
        elif fmt == "e4m3":
            if keys:
                cache.k[page_, :, :, off] = 0x7f
            if values:
                cache.v[page_, :, off] = 0xff
        else:
            if keys:
                cache.k_scale[page_, :, :, off] = 255
            if values:
                cache.v_scale[page_, :, :, off] = 255

    used = {int(table[b, t // page]) * page + t % page for b, n in enumerate(lengths) for t in range(n)}
    for s in range(cache.n_pages * page):
        if s not in used:
            spoil(s, True, True)
    assert all(np.array_equal(a, b) for a, b in zip(call() + call(30), clean + clean_w))
    at = 150                                                            # of sequence 1, whose rows are positions 110 .. 199
    spoil(int(table[1, at // page]) * page + at % page, False, True)
    for (o, lse), (o0, l0), window in ((call(), clean, 0), (call(30), clean_w, 30)):
        p = np.arange(110, 200)
        sees = np.concatenate((np.zeros(50, bool), (p >= at) & ((p < at + window) | (window == 0))))
        assert not np.isfinite(o[sees]).any() and np.array_equal(o[~sees], o0[~sees]) and np.array_equal(lse, l0)
    at = 120
    spoil(int(table[1, at // page]) * page + at % page, True, False)
    o, lse = call(30)
    sees = np.concatenate((np.zeros(50, bool), (p >= at) & (p < at + 30)))
    touched = sees | np.concatenate((np.zeros(50, bool), (p >= 150) & (p < 180)))
    assert np.isnan(o[sees]).all() and np.isnan(lse[sees]).all() and np.array_equal(o[~touched], clean_w[0][~touched])


def test_pages_lengths_and_starts_that_are_not_there(P):
    import torch
    say("pages the cache does not have, lengths beyond the table, starts that fall or lie outside")
    hq, hkv, D, page = 4, 2, 128, 16
    lengths, new = [100, 200], [20, 30]
    cache, table, rows = filled(P, lengths, hkv, D, page, "fp16", 3)
    q = np.random.default_rng(1).standard_normal((50, hq * D)).astype(np.float16)
    bad = table.copy()
    bad[0, 2], bad[1, 0], bad[1, 12] = cache.n_pages, -5, 2 ** 31 - 1
    kept = []
    for b, gone in ((0, [2]), (1, [0, 12])):
        there = ~np.isin(np.arange(lengths[b]) // page, gone)
        kept.append(there)
    ws = workspace(P, cache, hq, 50, 2)
    run = lambda tb, st, ln, **kw: P.paro_prompt_attention(cache, cuda(q), cuda(np.array(st, np.int32)), cuda(tb), cuda(np.array(ln, np.int32)), ws, with_lse=True, **kw)  # noqa: E731
    o, lse = run(bad, [0, 20, 50], lengths)
    r = 0
    for b in (0, 1):
        for i in range(new[b]):
            p = lengths[b] - new[b] + i
            t = np.flatnonzero(kept[b][:p + 1])
            want = more.attention(q[r].reshape(hq, D), rows[b][0][t], rows[b][1][t], D ** -0.5, 0, len(t), p)
            assert (np.abs(o[r].cpu().numpy().reshape(hq, D) - want[0]) <= want[2]).all() and (np.abs(lse[r].cpu().numpy() - want[1]) <= want[3]).all()
            r += 1
    room = table.shape[1] * page
    a, b = run(table, [0, 20, 50], [100, 2 ** 31 - 1]), run(table, [0, 20, 50], [100, room])
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    o, lse = run(table, [0, 20, 50], [-3, 200])
    assert (o[:20] == 0).all() and (lse[:20] == -np.inf).all()
    o, lse = run(table, [0, 20, 50], [7, 200])                          # more rows than tokens: the first are at positions below 0
    assert (o[:13] == 0).all() and (lse[:13] == -np.inf).all() and torch.isfinite(lse[13:]).all()
    out = torch.full((50, hq * D), 7.0, dtype=torch.float16, device="cuda")
    for st in ([5, 20, 45], [0, 30, 10], [-9, 3, 3], [40, 60, 90], [50, 50, 50], [-2 ** 31, 2 ** 31 - 1, 0]):
        out.fill_(7)
        run(table, st, lengths, O=out)
        s0, s1 = (np.clip(st[i], 0, 50) for i in (0, 1))
        s2 = max(np.clip(st[2], 0, 50), s1)
        written = np.zeros(50, bool)
        written[s0:max(s0, s1)] = True
        written[s1:s2] = True
        assert (out[cuda(~written)] == 7).all() and (out[cuda(written)] != 7).any(1).all()
    torch.cuda.synchronize()


def test_strides_and_given_outputs(P):
    import torch
    say("queries as columns of a linear's output, results into columns of wider rows, one shared table row")
    hq, hkv, D = 4, 2, 128
    new, lengths = [33, 7], [60, 60]
    cache, table, rows = filled(P, [60], hkv, D, 16, "fp16", 5)
    wide = torch.full((40, hq * D + 2 * hkv * D + 8), float("nan"), dtype=torch.float16, device="cuda")
    q = np.random.default_rng(2).standard_normal((40, hq * D)).astype(np.float16)
    wide[:, 8:8 + hq * D] = cuda(q)
    out = torch.full((40, hq * D + 16), 7.0, dtype=torch.float16, device="cuda")
    tb = cuda(table).expand(2, -1)
    got = P.paro_prompt_attention(cache, wide[:, 8:8 + hq * D], cuda(starts_of(new)), tb, cuda(np.array(lengths, np.int32)), workspace(P, cache, hq, 40, 2),
                                  O=out[:, 8:8 + hq * D])
    assert got.data_ptr() == out[:, 8:].data_ptr() and (out[:, :8] == 7).all() and (out[:, 8 + hq * D:] == 7).all()
    o_ref, _, bound, _ = wanted(q, rows * 2, new, lengths, hq, D ** -0.5)
    within(got.cpu().numpy().reshape(40, hq, D), o_ref, bound, "o")


def test_one_row_each_is_a_step(P):
    import torch
    say("one row of every sequence: the single tokens' attention")
    hq, hkv, D = 8, 2, 128
    lengths = [1, 0, 17, 900, 64]
    for fmt in ("fp16", "mxfp4"):
        cache, table, rows = filled(P, lengths, hkv, D, 16, fmt, 7)
        q, ln = cuda(np.random.default_rng(3).standard_normal((5, hq * D)).astype(np.float16)), cuda(np.array(lengths, np.int32))
        ws = P.Workspace.shared([], attention=[(cache, hq, 5)], prompts=[(cache, hq, 5, 5)])
        a, la = P.paro_paged_attention(cache, q, cuda(table), ln, ws, with_lse=True, cap=9.0)
        b, lb = P.paro_prompt_attention(cache, q, cuda(np.arange(6, dtype=np.int32)), cuda(table), ln, ws, with_lse=True, cap=9.0)
        # each is within its bound of the exact result: 2 * 2^-11 of it and, of weights that round to fp16, 2^-11 of the sum of |p v|
        assert (a.float() - b.float()).abs().max() <= 3 * 2.0 ** -11 * 4 and torch.equal(la == -np.inf, lb == -np.inf)
        assert (la - lb)[la > -np.inf].abs().max() <= 2.0 ** -17


def test_many_sequences(P):
    say("300 sequences, some without rows")
    rs = np.random.default_rng(11)
    lengths = rs.integers(0, 40, 300).tolist()
    new = [int(rs.integers(0, n + 1)) if n else 0 for n in lengths]
    check(P, *filled(P, lengths, 1, 64, 16, "e4m3", 1), new, lengths, 2)


def test_graphs_streams_and_bindings(P):
    import torch
    say("two captured calls of one workspace, replayed in turn with other inputs and lengths; another stream; the same calls through ctypes")
    hq, hkv, D, page = 8, 2, 128, 16
    cache, table, rows = filled(P, [3000, 500], hkv, D, page, "mxfp4", 12)
    q = torch.zeros((9, hq * D), dtype=torch.float16, device="cuda")
    tb, ln, st = cuda(table), cuda(np.array([3000, 500], np.int32)), cuda(np.array([0, 4, 9], np.int32))
    slopes, first = cuda(slopes_of(hq)), torch.zeros(9, dtype=torch.int32, device="cuda")
    ws = P.Workspace.shared([], prompts=[(cache, hq, 9, 2)])
    calls = (lambda: P.paro_prompt_attention(cache, q, st, tb, ln, ws, with_lse=True), lambda: P.paro_prompt_attention(cache, q, st, tb, ln, ws, None, 700, 20.0, slopes,
                                                                                                                    ln, first, with_lse=True))
    graphs = []
    for call in calls:
        call()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = call()
        graphs.append((g, out))
    for k in range(4):
        q.copy_(cuda(np.random.default_rng(k).standard_normal(q.shape).astype(np.float16)))
        ln.copy_(cuda(np.array([3000 - 700 * k, 500 - 99 * k], np.int32)))
        first.fill_(30 * k)
        want = [[t.clone() for t in call()] for call in calls]
        torch.cuda.synchronize()
        for g, out in graphs * 2:
            g.replay()
        torch.cuda.synchronize()
        for (g, out), w in zip(graphs, want):
            assert all(torch.equal(a, b) for a, b in zip(out, w))
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        got = [call() for call in calls]
    torch.cuda.current_stream().wait_stream(other)
    assert all(torch.equal(a, b) for x, w in zip(got, want) for a, b in zip(x, w))
    from paper_2511_10645_amd import binding as B_
    native = B_._native()
    assert native is not B_._CtypesCalls
    try:
        B_._host = B_._CtypesCalls
        step = lambda: P.paro_paged_attention(cache, q[:2], tb, ln, P.Workspace(P.paro_workspace_bytes_attention(cache, hq, 2)), with_lse=True, cap=9.0, slopes=slopes)  # noqa: E731
        assert all(torch.equal(a, b) for call, w in zip(calls, want) for a, b in zip(call(), w))
        one = step()
    finally:
        B_._host = native
    assert all(torch.equal(a, b) for a, b in zip(step(), one))


@pytest.mark.parametrize("fmt", ["fp16", "mxfp4"])
@pytest.mark.parametrize("D,hq,hkv", [(64, 4, 2), (128, 4, 2), (256, 3, 1)])
@pytest.mark.parametrize("new,lengths", [([90, 70, 3, 150], [40, 1, 0, 100]), ([9, 3, 5, 1], [4, 1, 0, 1])])
def test_more_rows_than_tokens(P, fmt, D, hq, hkv, new, lengths):
    """Rows at positions below 0 see the prefix alone, their distances counted from there; without one, nothing."""
    say(f"more rows than tokens: {fmt} D {D} new {new} lengths {lengths}")
    case = filled(P, lengths, hkv, D, 16, fmt, 5)
    for prefix in (None, [3, 1, 2, 50], [2 ** 31 - 1, -4, 7, 0]):
        check(P, *case, new, lengths, hq, 7, prefix=prefix)
        check(P, *case, new, lengths, hq, 8, prefix=prefix, cap=20.0, slopes=slopes_of(hq), window=6)
