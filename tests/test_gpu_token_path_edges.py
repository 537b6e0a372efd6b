"""The operators between the linears where their arithmetic, their split or their arguments come to an end; bounds: token_path_ref.py."""
import numpy as np
import pytest

import test_gpu_token_path as base
import token_path_ref as ref

pytestmark = pytest.mark.gpu
cuda, say, within, ws_of = base.cuda, base.say, base.within, base.ws_of


@pytest.fixture(scope="module")
def P():
    import paper_2511_10645_amd as paro
    return paro


@pytest.mark.parametrize("n", [96, 5000])
@pytest.mark.parametrize("scale", [1e6, 1.2e7, 2e7, 5e7, 1e8, 1.5e8, 3e8, 1e9, 1e30, -2e7, -1e8])
def test_attention_huge_finite_scores(P, n, scale):
    """Scores are +scale and -scale by turns: equal weights for one half, none for the other.  Bound: the n/2 equal terms are exact and
    summed in fp32, (n/2) 2^-24 of their mean size at most; lse passes five fp32 roundings."""
    say(f"attention of {n} tokens, scores +-{scale:g}")
    D = 64
    rs = np.random.default_rng(n)
    cache = P.KVCache(-(-n // 16), 1, D, 16)
    k, v, q = np.zeros((n, D), np.float16), rs.standard_normal((n, D)).astype(np.float16), np.zeros((1, D), np.float16)
    k[::2, 0], k[1::2, 0], q[0, 0] = 1, -1, 1
    P.paro_kv_append(cache, cuda(k), cuda(v), cuda(np.arange(n, dtype=np.int64)))
    table = cuda(np.arange(-(-n // 16), dtype=np.int32)[None])
    o, lse = P.paro_paged_attention(cache, cuda(q), table, cuda(np.array([n], np.int32)), ws_of(P, cache, 1, 1), scale, with_lse=True)
    half = v[0 if scale > 0 else 1::2].astype(np.float64)
    want = half.mean(0)
    within(o.cpu().numpy()[0], want, ref.F16 * np.abs(want) + ref.TINY + n / 2 * 2.0 ** -24 * np.abs(half).mean(0), "o")
    l_want = abs(scale) + np.log(n / 2)
    within(lse.cpu().numpy()[0], np.array([l_want]), np.array([2.0 ** -21 * l_want + 2.0 ** -20]), "lse")


@pytest.mark.parametrize("C", [128, 1024, 4096, 32768])
def test_norm_of_zeros_without_eps(P, C):
    """0 / 0 in both forms; with eps the row is zeros, and other rows are what they are."""
    import torch
    say(f"norm of a row of zeros, {C} channels")
    x, w = torch.ones((3, C), dtype=torch.float16, device="cuda"), torch.full((C,), 0.5, dtype=torch.float16, device="cuda")
    x[1] = 0
    r = -x
    r[0] = r[2] = 0
    for residual in (None, r):
        got = P.paro_rms_norm(x, w, 0.0, residual=residual)
        y = got if residual is None else got[0]
        assert bool(y[1].isnan().all()) and bool((y[[0, 2]] == 0.5).all())
        for group in (0, 128):
            codes, scales = P.paro_rms_norm_quantize_e4m3(x, w, 0.0, group, residual=residual)[:2]
            codes = codes.cpu().numpy()
            assert (codes[1] & 127 == 127).all() and (codes[[0, 2]] == 126).all()           # NaN; 448
            within(scales[[0, 2]].cpu().numpy(), np.full((2, scales.shape[1]), 0.5 / 448), np.full((1, 1), 2.0 ** -18 * 0.5 / 448), "scales")
            codes = P.paro_rms_norm_quantize_e4m3(x, w, 1e-5, group, residual=residual)[0]
            assert not bool(codes[1].any())


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 64, 4097])
def test_attention_window_beyond_every_token(P, window):
    say(f"attention within {window}")
    lengths = [0, 1, 700, 4096] + [33] * 20
    cache, table, q, rows = base._attn(P, lengths, 8, 4, 64, 16, "fp16", 8)
    o, lse = base._check(P, cache, table, q, rows, lengths, 8, 0.125, window)
    whole, lse_whole = base._check(P, cache, table, q, rows, lengths, 8, 0.125)
    assert (o == whole).all() and (lse == lse_whole).all()


def test_frequencies_and_caches_in_host_memory(P):
    import torch
    from paper_2511_10645_amd import binding as B_
    say("frequencies in a tensor of host memory are moved; a cache or frequencies that stay there are refused")
    f = base._freqs(64)
    x, pos = torch.randn((3, 128), device="cuda").half(), torch.arange(3, dtype=torch.int32, device="cuda")
    rope = P.Rope(torch.as_tensor(f), 64)
    assert rope.inv_freq.is_cuda and (P.paro_rope(rope, x, pos) == P.paro_rope(P.Rope(f, 64), x, pos)).all()
    there, cache, slots = P.Rope(f, 64, device="cpu"), P.KVCache(2, 2, 64, 16, device="cpu"), torch.arange(3, device="cuda")
    native = B_._native()
    try:
        for B_._host in (native, B_._CtypesCalls):
            for call in (lambda: P.paro_rope(there, x, pos), lambda: P.paro_kv_append(cache, x, x, slots),
                         lambda: P.paro_kv_append(P.KVCache(2, 2, 64, 16), x, x, slots, there, pos),
                         lambda: P.paro_paged_attention(cache, x, torch.zeros((3, 2), dtype=torch.int32, device="cuda"), pos, ws_of(P, cache, 2, 3))):
                with pytest.raises(AssertionError, match="one GPU"):
                    call()
    finally:
        B_._host = native


def counted(P, cache, hq, B):
    """A workspace, and a count of the partial results that calls have left in it: the scratch part is 512 of them, the maximum of a
    part's first query in front, and NaN here until it is written."""
    import torch
    total, exchange = P.paro_workspace_bytes_attention(cache, hq, B), P.paro_workspace_exchange_bytes_attention(cache, hq, B)
    ws = P.Workspace(total)
    parts = ws.buf[exchange:].view(torch.float32)[:512 * 16 * (cache.head_dim + 4)].view(512, -1)
    parts.fill_(float("nan"))
    return ws, lambda: int((~parts[:, 0].isnan()).sum())


@pytest.mark.parametrize("n,hkv,D,fmt", [(12000, 1, 128, "fp16"), (32768, 1, 128, "e4m3"), (32768, 2, 64, "fp16"), (16384, 4, 128, "fp16"), (16384, 1, 256, "fp16")])
def test_attention_of_few_heads_is_spread(P, n, hkv, D, fmt):
    """One long sequence: a block has two units of 32 tokens for each of its waves (4 with 256 channels, else 8) at most, whatever the
    number of heads, as long as there are 256 blocks for all."""
    say(f"attention of {n} tokens of {hkv} heads of {D} {fmt}")
    case = base._attn(P, [n], 2 * hkv, hkv, D, 16, fmt, n + hkv)
    ws, count = counted(P, case[0], 2 * hkv, 1)
    base._check(P, *case, [n], 2 * hkv, D ** -0.5, ws=ws)
    say(f"  {count()} parts")
    assert count() >= hkv * n / (32 * 2 * (4 if D == 256 else 8))


@pytest.mark.parametrize("lengths,hq,hkv,D,page,fmt,window", [
    ([40000, 700], 2, 1, 128, 16, "fp16", 0), ([60000], 4, 2, 64, 16, "fp16", 0), ([32768], 8, 4, 128, 32, "fp16", 0), ([32768], 8, 4, 128, 16, "e4m3", 0),
    ([33000], 20, 1, 128, 16, "e4m3", 0), ([20000], 16, 1, 256, 64, "fp16", 0), ([0, 50001, 1], 3, 1, 64, 16, "e4m3", 40000), ([17000, 17000, 16999], 5, 1, 256, 128, "e4m3", 0)])
def test_attention_joined_in_two_rounds(P, lengths, hq, hkv, D, page, fmt, window):
    """More than 32 blocks share a segment: groups of their parts are joined first.  Twice the same, with counters at zero between."""
    say(f"attention of {lengths}, {hq}/{hkv} x {D}, page {page} {fmt}, window {window}")
    case = base._attn(P, lengths, hq, hkv, D, page, fmt, sum(lengths), spread=1.5)
    ws, count = counted(P, case[0], hq, len(lengths))
    o, lse = base._check(P, *case, lengths, hq, D ** -0.5, window, ws=ws)
    segments = hkv * -(-hq // hkv // 16) * sum(n > 10000 for n in lengths)
    say(f"  {count()} parts of {segments} long segments")
    assert count() > 33 * segments + 2 * len(lengths)
    again, lse2 = base._check(P, *case, lengths, hq, D ** -0.5, window, ws=ws)
    assert (o == again).all() and (lse == lse2).all()


def test_attention_joined_in_two_rounds_replayed(P):
    import torch
    say("a captured call of 33 and more parts a head, replayed with other queries and lengths")
    case = base._attn(P, [33000], 8, 2, 64, 16, "fp16", 6)
    cache, table, q, rows = case
    ws, count = counted(P, cache, 8, 1)
    x, ln, tb = cuda(q).clone(), cuda(np.array([33000], np.int32)), cuda(table)
    P.paro_paged_attention(cache, x, tb, ln, ws)
    assert count() > 2 * 33
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out, lse = P.paro_paged_attention(cache, x, tb, ln, ws, with_lse=True)
    for n in (33000, 20000, 500, 33000):
        x.copy_(torch.randn(x.shape, device="cuda"))
        ln.fill_(n)
        want, l_want = P.paro_paged_attention(cache, x, tb, ln, ws_of(P, cache, 8, 1), with_lse=True)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert (out == want).all() and (lse == l_want).all()


@pytest.mark.parametrize("D,hq,hkv", [(64, 3, 1), (128, 4, 2), (256, 2, 1)])
def test_attention_over_all_of_e4m3(P, D, hq, hkv):
    """Every code at every scale that the append writes, from fp16's subnormals to 240 * 2^8: in sequences of one token, whose result is
    its value, and of 48 tokens of one scale."""
    import torch
    say(f"attention over every E4M3 value, {hq}/{hkv} x {D}")
    rs = np.random.default_rng(D)
    scales, page = np.arange(112, 136, dtype=np.uint8), 16
    n_pages = 5 * len(scales)
    codes = rs.integers(0, 256, (2, n_pages, hkv, page, D)).astype(np.uint8)
    s = np.broadcast_to(np.repeat(scales, 5)[:, None, None], (n_pages, hkv, page))
    most = np.where(s == 135, 0x77, 0x7e)[..., None]                    # 240 and 448
    codes = (codes & 128 | np.minimum(codes & 127, most)).astype(np.uint8)
    assert all(len(np.unique(codes[1, i:i + 5])) == (254 if i < n_pages - 5 else 240) for i in range(0, n_pages, 5))
    k = np.ascontiguousarray(codes[0].reshape(n_pages, hkv, page, D // 16, 16).transpose(0, 1, 3, 2, 4))
    cache = P.KVCache.from_device(cuda(k), cuda(codes[1]), cuda(s.copy()), cuda(s.copy()))
    q = (rs.standard_normal((2 * len(scales), hq * D)) * 0.01).astype(np.float16)
    table = np.zeros((2 * len(scales), 3), np.int32)
    table[::2, 0] = np.arange(0, n_pages, 5)
    table[1::2] = np.arange(0, n_pages, 5)[:, None] + [1, 2, 3]
    lengths = [1, 48] * len(scales)
    rows = [ref.cache_rows(cache, table[i, np.arange(n) // page].astype(np.int64) * page + np.arange(n) % page) for i, n in enumerate(lengths)]
    o, lse = base._check(P, cache, table, q, rows, lengths, hq, 2.0 ** -8)
    one = np.stack([rows[i][1][0] for i in range(0, len(lengths), 2)]).repeat(hq // hkv, axis=1)
    assert np.array_equal(o[::2].cpu().numpy().reshape(one.shape).astype(np.float64), one)
    # and rows that the append itself puts at these scales
    x = np.zeros((48, hkv, D))
    x[:] = rs.uniform(-1, 1, x.shape) * 2.0 ** np.linspace(-20, 15.9, 48)[:, None, None]
    x[0], x[1, :, ::2], x[2, :, 0] = 65504, -65504, 2.0 ** -24
    x = cuda(x.reshape(48, -1).astype(np.float16))
    cache = P.KVCache(3, hkv, D, page, "e4m3")
    P.paro_kv_append(cache, x, x, cuda(np.arange(48, dtype=np.int64)))
    held = ref.cache_rows(cache, np.arange(48))
    assert np.abs(held[1]).max() == 61440 and {int(b) for b in cache.v_scale.unique()} >= set(range(114, 136))
    for n in (1, 2, 3, 20, 48):
        base._check(P, cache, np.arange(3, dtype=np.int32)[None], q[:1], [(held[0][:n], held[1][:n])], [n], hq, 2.0 ** -10)


def test_attention_values_at_scores_of_minus_infinity(P):
    """A key that is not there for a query (score -inf) may hold anything else; its value has to be finite, for 0 * NaN is NaN.  Values past
    the end or on pages that are not there do not matter."""
    import torch
    say("attention: values that are not finite, at scores of -inf and in places that are left out")
    cache, table, q, rows = base._attn(P, [40], 2, 1, 64, 16, "fp16", 4)
    q = np.abs(q)
    cache.k[table[0, 0], 0, 0, 5, 0] = float("-inf")
    at = np.r_[0:5, 6:40]
    for value in (3.0, float("nan"), float("inf")):
        cache.v[table[0, 0], 0, 5] = value
        o, lse = P.paro_paged_attention(cache, cuda(q), cuda(table), cuda(np.array([40], np.int32)), ws_of(P, cache, 2, 1), 0.125, with_lse=True)
        w = ref.attention(q[0].reshape(2, 64), rows[0][0][at], rows[0][1][at], 0.125)
        within(lse.cpu().numpy()[0], w[1], w[3], "lse")
        if value == 3.0:
            within(o.cpu().numpy().reshape(2, 64), w[0], w[2], "o")
        else:
            assert bool(o.isnan().all())
    o = P.paro_paged_attention(cache, cuda(q), cuda(table), cuda(np.array([5], np.int32)), ws_of(P, cache, 2, 1), 0.125)
    assert bool(torch.isfinite(o).all())
    gone = table.copy()
    gone[0, 0] = -1
    o = P.paro_paged_attention(cache, cuda(q), cuda(gone), cuda(np.array([40], np.int32)), ws_of(P, cache, 2, 1), 0.125)
    w = ref.attention(q[0].reshape(2, 64), rows[0][0][16:], rows[0][1][16:], 0.125)
    within(o.cpu().numpy().reshape(2, 64), w[0], w[2], "without the page")
