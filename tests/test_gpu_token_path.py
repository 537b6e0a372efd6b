"""The operators between the linears (norm, rotary positions, cache, attention) against 64-bit forms; bounds: token_path_ref.py."""
import sys

import numpy as np
import pytest

import token_path_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2511_10645_amd as paro
    return paro


def say(msg):
    print(msg, flush=True)
    sys.stdout.flush()


def cuda(x):
    import torch
    return torch.as_tensor(x).cuda()


def within(got, want, bound, what):
    err = np.abs(got.astype(np.float64) - want)
    worst = float(np.max(err / bound)) if err.size else 0.0
    say(f"  {what}: worst err/bound {worst:.3f}")
    assert worst <= 1.0


def strided(x, more=24):
    """The same rows inside wider ones (16-byte steps), the rest NaN."""
    import torch
    buf = torch.full((x.shape[0], x.shape[1] + more), float("nan"), dtype=torch.float16, device="cuda")
    buf[:, 8:8 + x.shape[1]] = cuda(x)
    return buf, buf[:, 8:8 + x.shape[1]]


# ---- norm ---------------------------------------------------------------------------------------------------------------

NORM_SHAPES = [(1, 8), (3, 128), (17, 136), (5, 512), (2, 520), (1, 2048), (33, 2056), (7, 4096), (1, 5120), (3, 776), (5, 1024), (3, 8192), (2, 14336), (1, 32768)]


def _norm_inputs(T, C, seed):
    rs = np.random.default_rng(seed)
    x, r = (rs.standard_normal((T, C)).astype(np.float16) for _ in range(2))
    r[:, rs.integers(0, C, 2)] *= 40
    return x, r, (1 + 0.3 * rs.standard_normal(C)).astype(np.float16)


@pytest.mark.parametrize("T,C", NORM_SHAPES)
@pytest.mark.parametrize("residual", [False, True])
def test_norm(P, T, C, residual):
    say(f"norm {T} x {C} residual {residual}")
    x, r, w = _norm_inputs(T, C, T * C)
    h_ref, y_ref = ref.rms_norm(x, r if residual else None, w, 1e-5)
    xb, xs = strided(x)
    _, rs_ = strided(r, 32)
    yb, ys = strided(np.zeros_like(x), 40)
    got = P.paro_rms_norm(xs, cuda(w), 1e-5, residual=rs_ if residual else None, Y=ys)
    if residual:
        got, h = got
        within(h.cpu().numpy(), h_ref, ref.F16 * np.abs(h_ref) + ref.TINY, "h")
    assert got is ys and bool(yb[:, :8].isnan().all()) and bool(yb[:, 8 + C:].isnan().all())
    within(got.cpu().numpy(), y_ref, ref.F16 * np.abs(y_ref) + ref.TINY, "y")


@pytest.mark.parametrize("T,C,group", [(1, 128, 128), (5, 128, 0), (3, 640, 128), (4, 1000, 0), (2, 2048, 128), (9, 4096, 128), (6, 5120, 0), (1, 8320, 128),
                                       (2, 32768, 128), (2, 32768, 0), (5, 1024, 128), (5, 776, 0), (515, 4096, 128), (514, 2176, 0), (2, 7000, 0)])
def test_norm_e4m3(P, T, C, group):
    say(f"norm e4m3 {T} x {C} group {group}")
    x, r, w = _norm_inputs(T, C, 7 * T + C)
    x[-1], r[-1] = 0, 0                                                # a row of zeros: codes 0
    if group:
        w[:group] = 0                                                  # and a group of zeros in every row
    h_ref, y_ref = ref.rms_norm(x, r, w, 1e-5)
    codes, scales, h = P.paro_rms_norm_quantize_e4m3(cuda(x), cuda(w), 1e-5, group=group, residual=cuda(r))
    within(h.cpu().numpy(), h_ref, ref.F16 * np.abs(h_ref) + ref.TINY, "h")
    blocks = y_ref.reshape(T, -1, group or C)
    want = np.maximum(np.abs(blocks).max(-1), 1e-30) / 448
    s = scales.cpu().numpy().astype(np.float64)
    assert s.shape == want.shape
    within(s, want, 2.0 ** -18 * want, "scales")                       # a sum of squares, a root, three products in fp32
    q = ref.e4m3_values()[codes.cpu().numpy()].reshape(blocks.shape)
    assert np.isfinite(q).all()
    exact = blocks / want[..., None]
    within(q, exact, ref.half_step(exact) + 2.0 ** -17 * np.abs(exact), "codes")
    assert not q[-1].any()


def test_norm_in_place_and_special_values(P):
    import torch
    say("norm in place, NaN and infinities stay in their rows")
    x, r, w = _norm_inputs(6, 1024, 5)
    h_ref, y_ref = ref.rms_norm(x, r, w, 1e-5)
    X, R = cuda(x), cuda(r)
    y, h = P.paro_rms_norm(X, cuda(w), 1e-5, residual=R, Y=X, H=R)
    assert y is X and h is R
    within(X.cpu().numpy(), y_ref, ref.F16 * np.abs(y_ref) + ref.TINY, "y in x")
    within(R.cpu().numpy(), h_ref, ref.F16 * np.abs(h_ref) + ref.TINY, "h in r")
    x[1, 3], x[4, 9] = np.nan, np.inf
    got = P.paro_rms_norm(cuda(x), cuda(w), 1e-5)
    codes, scales = P.paro_rms_norm_quantize_e4m3(cuda(x), cuda(w), 1e-5, group=128)
    _, y_ref = ref.rms_norm(x[[0, 2, 3, 5]], None, w, 1e-5)
    within(got[[0, 2, 3, 5]].cpu().numpy(), y_ref, ref.F16 * np.abs(y_ref) + ref.TINY, "the other rows")
    assert bool(got[1].isnan().all()) and bool(got[4, 9].isnan()) and not bool(got[4, :9].any())
    codes = codes.cpu().numpy()
    assert (codes[1] & 127 == 127).all() and codes[4, 9] & 127 == 127 and not (codes[[0, 2, 3, 5]] & 127 == 127).any()
    assert torch.isfinite(scales[[0, 2, 3, 5]]).all()
    big = torch.full((1, 4096), 60000.0, dtype=torch.float16, device="cuda")       # squares sum to 1.5e13, h to beyond fp16
    y, h = P.paro_rms_norm(big, torch.ones(4096, dtype=torch.float16, device="cuda"), 1e-5, residual=big.clone())
    assert bool(h.isinf().all()) and bool((y == 1).all())


# ---- rotary positions --------------------------------------------------------------------------------------------------

def _freqs(rot, base=10000.0):
    return (base ** (-np.arange(0, rot, 2) / rot)).astype(np.float32)


@pytest.mark.parametrize("T,heads,D,rot,layout,magnitude", [
    (1, 1, 16, 16, "halves", 1.0), (1, 32, 128, 128, "halves", 1.0), (5, 7, 64, 32, "interleaved", 1.0), (3, 5, 80, 32, "halves", 1.25),
    (33, 40, 128, 96, "interleaved", 1.1386), (255, 3, 96, 96, "halves", 1.0), (256, 3, 256, 64, "halves", 1.0), (1030, 9, 128, 128, "interleaved", 0.5),
    (517, 1, 512, 512, "halves", 1.0), (2, 71, 64, 64, "halves", 1.0)])
def test_rope(P, T, heads, D, rot, layout, magnitude):
    say(f"rope {T} x {heads} x {D}, {rot} {layout}")
    rs = np.random.default_rng(T + heads + D)
    x = rs.standard_normal((T, heads * D)).astype(np.float16)
    pos = rs.integers(-5, 1 << 20, T).astype(np.int32)
    pos[0], pos[-1] = 0, 2 ** 31 - 1
    f = _freqs(rot)
    rope = P.Rope(f, D, layout, magnitude)
    x3 = x.reshape(T, heads, D)
    want = ref.rotate(x3, pos, f, layout, magnitude)
    bound = ref.rotate_bound(x3, want, f, layout, magnitude)
    _, xs = strided(x)
    y = P.paro_rope(rope, xs, cuda(pos))
    within(y.cpu().numpy().reshape(x3.shape), want, bound, "y")
    if rot < D:                                                        # what is not rotated is copied
        assert np.array_equal(y.cpu().numpy().reshape(x3.shape)[..., rot:], x3[..., rot:])
    assert P.paro_rope(rope, xs, cuda(pos), xs) is xs
    assert (xs == y).all()


# ---- append ------------------------------------------------------------------------------------------------------------

def _append_case(P, T, hq, hkv, D, page, fmt, seed, rot=None, layout="halves", scale=1.0, strides=True):
    import torch
    rs = np.random.default_rng(seed)
    n_pages = -(-T // page) + 3
    cache = P.KVCache(n_pages, hkv, D, page, fmt)
    for t in (cache.k, cache.v):
        t.fill_(7)
    slots = rs.permutation(n_pages * page)[:T].astype(np.int64)
    qkv = (rs.standard_normal((T, (hq + 2 * hkv) * D)) * scale).astype(np.float16)
    pos = rs.integers(0, 100000, T).astype(np.int32)
    f = _freqs(rot or D)
    return cache, P.Rope(f, D, layout), f, slots, qkv, pos


@pytest.mark.parametrize("T,hq,hkv,D,page,fmt,rot,layout", [
    (1, 8, 2, 128, 16, "fp16", 128, "halves"), (1, 8, 2, 128, 16, "e4m3", 128, "halves"), (37, 4, 4, 64, 32, "fp16", 16, "interleaved"),
    (37, 4, 4, 64, 32, "e4m3", 48, "halves"), (300, 5, 1, 128, 64, "fp16", 64, "halves"), (300, 5, 1, 128, 64, "e4m3", 128, "interleaved"),
    (19, 16, 2, 256, 16, "fp16", 256, "halves"), (261, 3, 3, 256, 1024, "e4m3", 64, "interleaved"), (70, 8, 8, 128, 16, "e4m3", 32, "halves"),
    (1030, 4, 2, 128, 16, "fp16", 128, "halves"), (1031, 3, 1, 64, 32, "e4m3", 64, "interleaved"), (1025, 10, 2, 128, 16, "e4m3", 96, "halves"),
    (1024, 2, 2, 256, 64, "fp16", 128, "interleaved")])
def test_append(P, T, hq, hkv, D, page, fmt, rot, layout):
    say(f"append {T} tokens, {hq}/{hkv} x {D}, page {page} {fmt}, {rot} {layout}")
    cache, rope, f, slots, qkv, pos = _append_case(P, T, hq, hkv, D, page, fmt, T + D, rot, layout)
    q, k, v = np.split(qkv, [hq * D, (hq + hkv) * D], axis=1)
    x = cuda(qkv)
    before = [t.clone() for t in (cache.k, cache.v)]
    got = P.paro_kv_append(cache, x[:, hq * D:(hq + hkv) * D], x[:, (hq + hkv) * D:], cuda(slots), rope, cuda(pos), x[:, :hq * D])
    q3, k3, v3 = q.reshape(T, hq, D), k.reshape(T, hkv, D), v.reshape(T, hkv, D).astype(np.float64)
    want = ref.rotate(q3, pos, f, layout, 1.0)
    within(got.cpu().numpy().reshape(q3.shape), want, ref.rotate_bound(q3, want, f, layout, 1.0), "q")
    k_ref = ref.rotate(k3, pos, f, layout, 1.0)
    k_got, v_got = ref.cache_rows(cache, slots)
    if fmt == "fp16":
        within(k_got, k_ref, ref.rotate_bound(k3, k_ref, f, layout, 1.0), "k")
        assert np.array_equal(v_got, v3)
    else:
        lost = ref.rotate_bound(k3, k_ref, f, layout, 1.0) - ref.F16 * np.abs(k_ref) - ref.TINY       # the fp32 part alone
        for name, rows, have, s, err in (("k", k_ref, k_got, cache.k_scale, lost), ("v", v3, v_got, cache.v_scale, 0)):
            e = s.cpu().numpy()[slots // page, :, slots % page].astype(int) - 127
            least = np.clip(np.ceil(np.log2(np.abs(rows).max(-1) / 448)), -15, 8)
            sure = np.abs(np.log2(np.abs(rows).max(-1) / 448) - np.round(np.log2(np.abs(rows).max(-1) / 448))) > 1e-5
            assert np.array_equal(e[sure], least[sure]) and sure.mean() > 0.9
            unit = 2.0 ** e[..., None].astype(float)
            within(have, rows, ref.half_step(rows / unit) * unit * (1 + 2.0 ** -16) + err, name)
    # everything else in the cache is as it was
    other = np.setdiff1d(np.arange(cache.n_pages * page), slots)
    k_now, v_now = (t.clone() for t in (cache.k, cache.v))
    p, o = cuda(slots // page), cuda(slots % page)
    for now, was, at in ((k_now.movedim(3, 1), before[0].movedim(3, 1), None), (v_now.movedim(2, 1), before[1].movedim(2, 1), None)):
        now[p, o] = was[p, o]
        assert (now == was).all()
    assert len(other) > 0


@pytest.mark.parametrize("fmt", ["fp16", "e4m3"])
def test_append_leaves_out_and_in_place(P, fmt):
    import torch
    say(f"append {fmt}: slots that are not there, no rotation, queries in place, no queries")
    T, hq, hkv, D = 12, 4, 2, 64
    cache, rope, f, slots, qkv, pos = _append_case(P, T, hq, hkv, D, 16, fmt, 3)
    n = cache.n_pages * cache.page
    slots[[0, 5, 6, 11]] = -1, n, 2 ** 40, -(2 ** 62)
    kept = np.array([1, 2, 3, 4, 7, 8, 9, 10])
    x = cuda(qkv)
    q, k, v = x[:, :hq * D], x[:, hq * D:(hq + hkv) * D], x[:, (hq + hkv) * D:]
    before = cache.v.clone()
    assert P.paro_kv_append(cache, k, v, cuda(slots)) is None
    k_got, v_got = ref.cache_rows(cache, slots[kept])
    k3, v3 = (t.cpu().numpy().reshape(T, hkv, D)[kept].astype(np.float64) for t in (k, v))
    if fmt == "fp16":
        assert np.array_equal(k_got, k3) and np.array_equal(v_got, v3)
    else:
        assert np.abs(k_got - k3).max() < 0.07 * np.abs(k3).max() and np.abs(v_got - v3).max() < 0.07 * np.abs(v3).max()
    touched = (cache.v != before).any(-1).any(1).flatten().cpu().numpy()
    assert set(np.nonzero(touched)[0]) <= set(slots[kept].tolist())
    assert (P.paro_kv_append(cache, k, v, cuda(slots), Q=q) == q).all()        # no rotation: queries as they are
    want = P.paro_kv_append(cache, k, v, cuda(slots), rope, cuda(pos), q)
    assert P.paro_kv_append(cache, k, v, cuda(slots), rope, cuda(pos), q, q) is not None
    assert (x[:, :hq * D] == want).all()


def test_append_e4m3_extremes(P):
    say("append e4m3: the largest and the smallest rows, zeros, values that are not finite")
    import torch
    D = 64
    cache = P.KVCache(2, 1, D, 16, "e4m3")
    rows = np.zeros((8, D), dtype=np.float16)
    rows[0, :3] = 65504, -65504, 1                                     # 65504 / 2^8 rounds to 256, which would stand for 2^16
    rows[1, :2] = 448, 3
    rows[2, :2] = 449, 3
    rows[3, :4] = np.array([1, 2, -3, 5]) * 2.0 ** -24                 # subnormal: kept as they are
    rows[4, :3] = np.nan, np.inf, 2
    rows[5, :2] = -np.inf, 0
    rows[7, :2] = 2.0 ** -14, 6e-8
    slots = np.arange(8, dtype=np.int64) + 3
    P.paro_kv_append(cache, cuda(rows), cuda(rows), cuda(slots))
    for have, s in zip(ref.cache_rows(cache, slots), (cache.k_scale, cache.v_scale)):
        have = have[:, 0]
        e = s.cpu().numpy()[0, 0, 3:11].astype(int) - 127
        assert list(e) == [8, 0, 1, -15, -7, -15, -15, -15]
        assert list(have[0, :3]) == [61440, -61440, 1.0]
        assert list(have[1, :2]) == [448, 3] and have[2, 0] == 448
        assert np.array_equal(have[3], rows[3].astype(np.float64))
        assert np.isnan(have[4, :2]).all() and have[4, 2] == 2 and not have[4, 3:].any()
        assert np.isnan(have[5, 0]) and not have[5, 1:].any() and not have[6].any()
        assert have[7, 0] == 2.0 ** -14
    with np.errstate(over="ignore"):
        k, v = ref.cache_rows(cache, slots[[0, 1, 2, 3, 6, 7]])
        assert np.array_equal(k.astype(np.float16).astype(np.float64), k)          # every value is an fp16 value


# ---- attention ---------------------------------------------------------------------------------------------------------

def _attn(P, lengths, hq, hkv, D, page, fmt, seed, spread=1.0, spare=2, width=None):
    """A cache filled at random places, everything else in it NaN; per sequence the (k, v) rows in 64 bits."""
    import torch
    rs = np.random.default_rng(seed)
    held = [-(-n // page) for n in lengths]
    n_pages = sum(held) + spare
    cache = P.KVCache(n_pages, hkv, D, page, fmt)
    for t in (cache.k, cache.v):
        t.fill_(float("nan") if fmt == "fp16" else 127)
    if fmt == "e4m3":
        cache.k_scale.fill_(255)
        cache.v_scale.fill_(255)
    width = width or max(1, max(held))
    table = np.full((len(lengths), width), -7, dtype=np.int32)         # entries past a sequence's pages are not looked at
    order, at = rs.permutation(n_pages), 0
    for i, h in enumerate(held):
        table[i, :h] = order[at:at + h]
        at += h
    rows = []
    total = sum(lengths)
    slots = np.concatenate([table[i, np.arange(n) // page].astype(np.int64) * page + np.arange(n) % page for i, n in enumerate(lengths)]) if total else np.zeros(0, np.int64)
    q = (rs.standard_normal((len(lengths), hq * D)) * spread).astype(np.float16)
    if total:
        k, v = (rs.standard_normal((total, hkv * D)).astype(np.float16) for _ in range(2))
        v += np.float16(0.25)
        P.paro_kv_append(cache, cuda(k), cuda(v), cuda(slots))
        k, v = ref.cache_rows(cache, slots)
        assert np.isfinite(k).all() and np.isfinite(v).all()
    else:
        k = v = np.zeros((0, hkv, D))
    ends = np.cumsum([0] + list(lengths))
    rows = [(k[a:b], v[a:b]) for a, b in zip(ends[:-1], ends[1:])]
    return cache, table, q, rows


def _check(P, cache, table, q, rows, lengths, hq, scale, window=0, ws=None, **kw):
    import torch
    B = len(lengths)
    ws = ws or P.Workspace(P.paro_workspace_bytes_attention(cache, hq, B))
    o, lse = P.paro_paged_attention(cache, q if isinstance(q, torch.Tensor) else cuda(q), cuda(table), cuda(np.asarray(lengths, dtype=np.int32)), ws, scale,
                                    window, with_lse=True, **kw)
    o3, l2 = o.cpu().numpy().reshape(B, hq, -1), lse.cpu().numpy()
    qn = (q.cpu().numpy() if isinstance(q, torch.Tensor) else q).reshape(B, hq, -1)
    want = [ref.attention(qn[i], *(x[max(0, n - window) if window else 0:n] for x in rows[i]), scale) for i, n in enumerate(lengths)]
    within(o3, np.stack([w[0] for w in want]), np.stack([w[2] for w in want]), "o")
    l_ref, l_bound = np.stack([w[1] for w in want]), np.stack([w[3] for w in want])
    some = np.isfinite(l_ref)
    assert np.array_equal(l2[~some], l_ref[~some])
    within(l2[some], l_ref[some], l_bound[some], "lse")
    ex = P.paro_workspace_exchange_bytes_attention(cache, hq, B)
    assert ws.partials_clean(ex) and ws.error_word() == 0
    return o, lse


EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257]


@pytest.mark.parametrize("hq,hkv,D,page,fmt", [
    (4, 1, 64, 16, "fp16"), (4, 1, 64, 16, "e4m3"), (8, 2, 128, 16, "fp16"), (8, 2, 128, 32, "e4m3"), (3, 3, 128, 64, "fp16"), (5, 1, 128, 128, "e4m3"),
    (16, 1, 128, 16, "fp16"), (17, 1, 64, 16, "fp16"), (40, 1, 128, 16, "e4m3"), (6, 2, 256, 16, "fp16"), (16, 1, 256, 1024, "e4m3"), (71, 1, 64, 32, "e4m3")])
def test_attention_lengths(P, hq, hkv, D, page, fmt):
    say(f"attention {hq}/{hkv} x {D}, page {page} {fmt}")
    case = _attn(P, EDGES, hq, hkv, D, page, fmt, hq * D + page)
    _check(P, *case, EDGES, hq, D ** -0.5)


@pytest.mark.parametrize("n,hq,hkv,D,page,fmt", [(5000, 8, 2, 128, 16, "fp16"), (5003, 8, 2, 128, 32, "e4m3"), (20011, 4, 1, 64, 16, "fp16"),
                                                 (3001, 16, 1, 256, 64, "e4m3"), (40000, 1, 1, 128, 16, "fp16"), (9001, 32, 8, 128, 16, "fp16")])
def test_attention_split_and_joined(P, n, hq, hkv, D, page, fmt):
    say(f"attention of {n} tokens, {hq}/{hkv} x {D} {fmt}")
    lengths = [n]
    case = _attn(P, lengths, hq, hkv, D, page, fmt, n, spread=2.0)
    o, lse = _check(P, *case, lengths, hq, D ** -0.5)
    again, lse2 = _check(P, *case, lengths, hq, D ** -0.5)
    assert (o == again).all() and (lse == lse2).all()                  # not a matter of timing


@pytest.mark.parametrize("hq,hkv,D,fmt", [(4, 1, 64, "fp16"), (6, 2, 128, "e4m3"), (16, 16, 64, "fp16"), (33, 33, 64, "fp16"), (20, 1, 128, "fp16"), (4, 2, 256, "fp16"),
                                         (300, 300, 64, "e4m3")])
def test_attention_one_sequence(P, hq, hkv, D, fmt):
    """One sequence of lengths around the numbers of units at which a head takes another number of blocks, in a table that is wider."""
    say(f"attention of one sequence, {hq}/{hkv} x {D} {fmt}")
    lengths = [1, 32, 33, 128, 129, 160, 256, 257, 289, 383, 511, 1025] if hkv > 30 else [1, 33, 129, 160, 256, 257, 289, 383, 511, 700, 1200, 2047, 2049, 4100, 6001]
    cache, table, q, rows = _attn(P, [lengths[-1]], hq, hkv, D, 16, fmt, hq)
    for n in lengths:
        _check(P, cache, table, q, rows if n == lengths[-1] else [(rows[0][0][:n], rows[0][1][:n])], [n], hq, D ** -0.5)
    _check(P, cache, table, q, [(rows[0][0][:1000], rows[0][1][:1000])], [1000], hq, D ** -0.5, window=300)


@pytest.mark.parametrize("B", [64, 65, 150, 700, 4500])
def test_attention_many_ragged(P, B):
    say(f"attention of {B} sequences")
    rs = np.random.default_rng(B)
    lengths = [int(x) for x in np.exp(rs.uniform(0, np.log(600 if B < 200 else 100 if B < 4000 else 8), B))]
    lengths[B // 2], lengths[-1] = 3000, 0
    case = _attn(P, lengths, 4, 2, 64, 16, "fp16", B)
    _check(P, *case, lengths, 4, 0.125)


@pytest.mark.parametrize("window", [1, 16, 31, 32, 33, 100, 1000])
@pytest.mark.parametrize("fmt", ["fp16", "e4m3"])
def test_attention_window(P, window, fmt):
    say(f"attention within {window} {fmt}")
    lengths = [0, 1, 31, 32, 33, 99, 100, 101, 128, 700, 1000, 1001, 2500]
    case = _attn(P, lengths, 6, 2, 64, 16, fmt, window)
    _check(P, *case, lengths, 6, 0.125, window)


def test_attention_strides_streams_shared_rows(P):
    import torch
    say("attention: strided queries and outputs, a shared table row, another stream, a shared workspace")
    hq, hkv, D, page = 8, 2, 128, 16
    cache, table, q, rows = _attn(P, [200], hq, hkv, D, page, "fp16", 77)
    lengths = [200, 1, 0, 37, 150]
    rs = np.random.default_rng(1)
    q = rs.standard_normal((5, hq * D)).astype(np.float16)
    _, qs = strided(q)
    ob, os_ = strided(np.zeros_like(q), 16)
    ws = P.Workspace.shared([], attention=[(cache, hq, 5), (cache, hq, 64)])
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        t = cuda(table).expand(5, -1)
        o, lse = P.paro_paged_attention(cache, qs, t, cuda(np.asarray(lengths, np.int32)), ws, D ** -0.5, O=os_, with_lse=True)
    s.synchronize()
    assert o is os_
    for i, n in enumerate(lengths):
        w = ref.attention(q[i].reshape(hq, D), rows[0][0][:n], rows[0][1][:n], D ** -0.5)
        within(o[i].cpu().numpy().reshape(hq, D), w[0], w[2], f"row {i}")
    assert bool(ob[:, :8].isnan().all()) and bool(ob[:, 8 + hq * D:].isnan().all())


def test_attention_bounds_of_lengths_and_pages(P):
    import torch
    say("attention: lengths beyond the table or negative, pages that are not there")
    hq, hkv, D, page = 4, 2, 64, 16
    cache, table, q, rows = _attn(P, [96, 96, 96], hq, hkv, D, page, "fp16", 9)
    q = cuda(q)
    _check(P, cache, table, q, rows, [96, 96, 96], hq, 0.125)
    ws = P.Workspace(P.paro_workspace_bytes_attention(cache, hq, 3))
    o = P.paro_paged_attention(cache, q, cuda(table), cuda(np.array([2 ** 31 - 1, -5, 96], np.int32)), ws, 0.125)
    whole = P.paro_paged_attention(cache, q, cuda(table), cuda(np.array([96, 0, 96], np.int32)), ws, 0.125)
    assert (o == whole).all() and not bool(o[1].any())
    bad = table.copy()
    bad[0, 2], bad[1, :], bad[2, 5] = -1, cache.n_pages, 2 ** 31 - 1
    o, lse = P.paro_paged_attention(cache, q, cuda(bad), cuda(np.array([96, 96, 96], np.int32)), ws, 0.125, with_lse=True)
    for i, keep in ((0, [0, 1, 3, 4, 5]), (2, [0, 1, 2, 3, 4])):
        at = np.concatenate([np.arange(16) + 16 * p for p in keep])
        w = ref.attention(q[i].cpu().numpy().reshape(hq, D), rows[i][0][at], rows[i][1][at], 0.125)
        within(o[i].cpu().numpy().reshape(hq, D), w[0], w[2], f"row {i} without a page")
    assert not bool(o[1].any()) and bool((lse[1] == -np.inf).all())


@pytest.mark.parametrize("fmt", ["fp16", "e4m3"])
def test_attention_special_scores(P, fmt):
    import torch
    say(f"attention {fmt}: equal, huge, vanishing and infinite scores")
    hq, hkv, D, page, n = 2, 1, 64, 16, 300
    cache, table, q, rows = _attn(P, [n], hq, hkv, D, page, fmt, 4)
    _check(P, cache, table, np.zeros_like(q), rows, [n], hq, 0.125)     # all weights equal
    _check(P, cache, table, q, rows, [n], hq, 0.0)
    _check(P, cache, table, q, rows, [n], hq, -3.0)
    _check(P, cache, table, q, rows, [n], hq, 40.0)                    # one token has nearly all the weight
    if fmt == "fp16":
        first = (table[0, 0], table[0, 1])
        cache.k[first[0], 0, 0, 0, 0] = float("-inf")                  # token 0, channel 0
        q1 = np.abs(q)
        rows[0][0][0, 0, 0] = -np.inf
        o, lse = P.paro_paged_attention(cache, cuda(q1), cuda(table), cuda(np.array([n], np.int32)), ws_of(P, cache, hq, 1), 0.125, with_lse=True)
        w = ref.attention(q1[0].reshape(hq, D), rows[0][0][1:n], rows[0][1][1:n], 0.125)          # as if it were not there
        within(o.cpu().numpy().reshape(hq, D), w[0], w[2], "without token 0")
        o, lse = P.paro_paged_attention(cache, cuda(q1), cuda(table), cuda(np.array([1], np.int32)), ws_of(P, cache, hq, 1), 0.125, with_lse=True)
        assert not bool(o.any()) and bool((lse == -np.inf).all())      # nothing but -inf
        cache.k[first[1], 0, 0, 3, 0] = float("nan")                   # token 19
        o, lse = P.paro_paged_attention(cache, cuda(q1), cuda(table), cuda(np.array([n], np.int32)), ws_of(P, cache, hq, 1), 0.125, with_lse=True)
        assert bool(o.isnan().all()) and bool(lse.isnan().all())
        o = P.paro_paged_attention(cache, cuda(q1), cuda(table), cuda(np.array([19], np.int32)), ws_of(P, cache, hq, 1), 0.125)
        assert bool(torch.isfinite(o).all())                           # the NaN is past the end


def test_refusals_of_the_calls(P):
    import torch
    from paper_2511_10645_amd import binding as B_
    say("numbers beyond 32 bits, outputs without their inputs, other shapes, in both bindings")
    cache, table, q, _ = _attn(P, [20], 2, 1, 64, 16, "fp16", 1)
    x, w = torch.zeros((2, 128), dtype=torch.float16, device="cuda"), torch.ones(128, dtype=torch.float16, device="cuda")
    native = B_._native()
    try:
        for B_._host in (native, B_._CtypesCalls):
            for call in (lambda: P.paro_paged_attention(cache, cuda(q), cuda(table), cuda(np.array([20], np.int32)), ws_of(P, cache, 2, 1), window=2 ** 32 + 1),
                         lambda: P.paro_rms_norm_quantize_e4m3(x, w, 1e-5, group=2 ** 32 + 128), lambda: P.paro_rms_norm(x, w, 1e-5, H=x),
                         lambda: P.paro_rms_norm_quantize_e4m3(x, w, 1e-5, H=x), lambda: P.paro_rms_norm(x, w, 1e-5, residual=x[:1]),
                         lambda: P.paro_kv_append(cache, x[:, :64], x[:, :64], torch.zeros(2, dtype=torch.int64, device="cuda"), Qr=x)):
                with pytest.raises(AssertionError):
                    call()
            with pytest.raises(P.ParoError):
                P.paro_paged_attention(cache, cuda(q), cuda(table), cuda(np.array([20], np.int32)), ws_of(P, cache, 2, 1), window=-1)
            with pytest.raises(P.ParoError):
                P.paro_rms_norm_quantize_e4m3(x, w, 1e-5, group=64)
    finally:
        B_._host = native


def ws_of(P, cache, hq, B):
    return P.Workspace(P.paro_workspace_bytes_attention(cache, hq, B))


def test_attention_far_apart_weights(P):
    """A first token 20 nats above thousands of equal others: together these have a weight that single ones lose if they are rounded away."""
    import torch
    say("attention: one heavy token among many light ones")
    D, n = 64, 30000
    cache = P.KVCache(-(-n // 16), 1, D, 16, "fp16")
    k, v = np.zeros((n, D), np.float16), np.ones((n, D), np.float16)
    k[0, 0], v[0] = 20, 0
    q = np.zeros((1, D), np.float16)
    q[0, 0] = 1
    P.paro_kv_append(cache, cuda(k), cuda(v), cuda(np.arange(n, dtype=np.int64)))
    table = np.arange(-(-n // 16), dtype=np.int32)[None]
    k64, v64 = ref.cache_rows(cache, np.arange(n))
    _check(P, cache, table, q, [(k64, v64)], [n], 1, 1.0)


def test_offsets_past_32_bits(P):
    import torch
    say("append and attention at the end of a cache of 5 GiB of keys")
    hq, hkv, D, page = 8, 8, 128, 16
    n_pages = 5 * 2 ** 30 // (hkv * D * page * 2)
    k = torch.empty((n_pages, hkv, D // 8, page, 8), dtype=torch.float16, device="cuda")
    v = torch.empty((n_pages, hkv, page, D), dtype=torch.float16, device="cuda")
    cache = P.KVCache.from_device(k, v)
    rs = np.random.default_rng(2)
    n = 77
    table = (n_pages - 1 - np.arange(5, dtype=np.int32))[None]
    slots = table[0, np.arange(n) // page].astype(np.int64) * page + np.arange(n) % page
    kk, vv = (rs.standard_normal((n, hkv * D)).astype(np.float16) for _ in range(2))
    P.paro_kv_append(cache, cuda(kk), cuda(vv), cuda(slots))
    q = rs.standard_normal((1, hq * D)).astype(np.float16)
    rows = [(kk.reshape(n, hkv, D).astype(np.float64), vv.reshape(n, hkv, D).astype(np.float64))]
    _check(P, cache, table, q, rows, [n], hq, D ** -0.5)
    assert np.array_equal(v[n_pages - 1].cpu().numpy().transpose(1, 0, 2).reshape(page, -1), vv[:page])


def test_graph_replays_and_both_bindings(P):
    import torch
    say("a captured step, replayed with other inputs in place; the same calls through ctypes")
    hq, hkv, D, page, B = 8, 2, 128, 16, 3
    lengths = [700, 33, 1]
    cache, table, q, rows = _attn(P, lengths, hq, hkv, D, page, "fp16", 12)
    rope = P.Rope(_freqs(D), D)
    w = cuda((1 + 0.1 * np.random.default_rng(0).standard_normal(hq * D)).astype(np.float16))
    x, r = cuda(q).clone(), torch.zeros((B, hq * D), dtype=torch.float16, device="cuda")
    kv = torch.zeros((B, hkv * D), dtype=torch.float16, device="cuda")
    slots = cuda(np.array([table[i, (n - 1) // page] * page + (n - 1) % page for i, n in enumerate(lengths)], np.int64))
    pos, ln, tb = cuda(np.array(lengths, np.int32) - 1), cuda(np.array(lengths, np.int32)), cuda(table)
    ws = ws_of(P, cache, hq, B)

    def step():
        y, h = P.paro_rms_norm(x, w, 1e-5, residual=r)
        qr = P.paro_kv_append(cache, kv, kv, slots, rope, pos, y)
        return y, h, qr, *P.paro_paged_attention(cache, qr, tb, ln, ws, with_lse=True), *P.paro_rms_norm_quantize_e4m3(x, w, 1e-5, 128), P.paro_rope(rope, x, pos)

    step()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    for k in range(4):
        x.copy_(cuda((np.random.default_rng(k).standard_normal(x.shape)).astype(np.float16)))
        kv.copy_(x[:, :hkv * D])
        r.add_(0.5)
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert (a == b).all()
    from paper_2511_10645_amd import binding as B_
    native = B_._native()
    assert native is not B_._CtypesCalls
    try:
        B_._host = B_._CtypesCalls
        for a, b in zip(step(), want):
            assert (a == b).all()
    finally:
        B_._host = native
