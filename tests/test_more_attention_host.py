"""Refusals of the prompts' attention, of scores and of the MXFP4 cache, and the workspace's size: no GPU is needed."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2511_10645_amd as paro
from paper_2511_10645_amd import binding as B
from test_token_path_devices import gpu, ints, longs, rows, table, workspace

E_NULL, E_SHAPE, E_ALIGN, E_UNSUP, E_WS = 1, 2, 3, 5, 6
FAKE = 0x10000
r = ctypes.byref


def _cache(n_pages=4, page=16, kv_heads=2, head_dim=128, format=0, k=FAKE, v=FAKE, ks=None, vs=None):
    return B._CKVCache(n_pages, page, kv_heads, head_dim, format, k, v, ks, vs)


def _scores(cap=0.0, slopes=None):
    return B._CScores(cap, slopes)


def test_mxfp4_cache_refusals():
    L = paro.lib()
    a = lambda c: L.paro_kv_append(r(c), None, FAKE, 256, FAKE, 256, FAKE, None, 1, None, 0, 0, None, 0, None)
    assert a(_cache(format=4)) == E_NULL and a(_cache(format=4, ks=FAKE)) == E_NULL
    assert a(_cache(format=4, ks=FAKE + 2, vs=FAKE)) == E_ALIGN and a(_cache(format=4, ks=FAKE, vs=FAKE, v=FAKE + 8)) == E_ALIGN
    assert a(_cache(format=4, ks=FAKE, vs=FAKE, head_dim=96)) == E_UNSUP and a(_cache(format=3)) == E_UNSUP and a(_cache(format=5)) == E_UNSUP


def test_scores_refusals():
    L = paro.lib()
    need = L.paro_workspace_bytes_attention(r(_cache()), 8, 3)
    f = lambda s=None, scale=0.1, window=0, O=FAKE * 4, ws=FAKE, n=need: L.paro_paged_attention_scored(
        r(_cache()), FAKE, 1024, 8, FAKE, 4, 4, FAKE, 3, scale, window, r(s) if s else None, O, 1024, None, ws, n, None)
    for cap in (-1.0, math.nan, math.inf, 3e38):
        assert f(_scores(cap)) == E_SHAPE
    assert f(_scores(1e-30), scale=1e30) == E_SHAPE                     # scale / cap is not finite
    assert f(_scores(1.0, FAKE + 2)) == E_ALIGN and f(_scores(), scale=math.nan) == E_SHAPE and f(_scores(2.0), O=FAKE) == E_SHAPE
    assert f(_scores(2.0, FAKE), n=need - 1) == E_WS and f(None, ws=None) == E_WS and f(_scores(2.0), window=-1) == E_SHAPE


def test_prompt_refusals():
    L = paro.lib()
    need = L.paro_workspace_bytes_prompt(r(_cache()), 8, 5, 3)
    f = lambda c=_cache(), Q=FAKE, ldq=1024, hq=8, T=5, starts=FAKE, table=FAKE, ldt=4, width=4, lengths=FAKE, batch=3, scale=0.1, window=0, s=None, prefix=None, \
        first=None, O=FAKE * 4, ldo=1024, lse=None, ws=FAKE, n=need: L.paro_prompt_attention(
            r(c) if c else None, Q, ldq, hq, T, starts, table, ldt, width, lengths, batch, scale, window, r(s) if s else None, prefix, first, O, ldo, lse, ws, n, None)
    for name in ("c", "Q", "O", "starts", "table", "lengths"):
        assert f(**{name: None}) == E_NULL, name
    for bad in (dict(T=0), dict(batch=0), dict(hq=7), dict(hq=0), dict(width=0), dict(window=-1), dict(ldt=3), dict(O=FAKE), dict(scale=math.inf), dict(scale=3e38),
                dict(ldq=512), dict(ldo=512), dict(s=_scores(-1.0))):
        assert f(**bad) == E_SHAPE, bad
    for bad in (dict(Q=FAKE + 2), dict(ldo=1028), dict(starts=FAKE + 1), dict(lengths=FAKE + 2), dict(prefix=FAKE + 2), dict(first=FAKE + 1), dict(lse=FAKE + 2),
                dict(ws=FAKE + 128), dict(table=FAKE + 2), dict(s=_scores(0.0, FAKE + 1))):
        assert f(**bad) == E_ALIGN, bad
    assert f(ws=None) == E_WS and f(n=need - 1) == E_WS
    assert f(width=1 << 27, ldt=1 << 27) == E_UNSUP and f(T=(1 << 24) + 1, n=1 << 50) == E_UNSUP
    assert f(T=1 << 24, hq=128, ldq=16384, ldo=16384, n=1 << 50) == E_UNSUP             # 2^31 pairs of a row and a head
    assert f(T=1 << 22, batch=1 << 22, hq=256, ldq=32768, ldo=32768, c=_cache(kv_heads=256), n=1 << 50) == E_UNSUP
    assert f(c=_cache(format=4)) == E_NULL and f(c=_cache(page=8)) == E_UNSUP



@pytest.mark.parametrize("T,batch,hq,hkv,taken", [(2 ** 23 - 64, 1, 32, 8, True), (2 ** 22, 2 ** 17, 32, 8, True), (2 ** 23, 64, 32, 8, False), (2 ** 24, 1, 32, 8, False),
                                                   (2 ** 24, 1, 15, 5, True), (2 ** 24, 1, 17, 1, False), (64, 2 ** 19, 8, 8, True), (2 ** 22, 2 ** 22, 4, 4, False)])
def test_prompt_sizes(T, batch, hq, hkv, taken):
    """T q_heads + 32 kv_heads min(batch, T) up to 2^28 passes every check but the workspace's."""
    assert taken == (T * hq + 32 * min(batch, T) * hkv <= 2 ** 28)
    st = paro.lib().paro_prompt_attention(r(_cache(kv_heads=hkv)), FAKE, 65536, hq, T, FAKE, FAKE, 4, 4, FAKE, batch, 0.1, 0, None, None, None, FAKE * 4, 65536, None, None, 0, None)
    assert st == (E_WS if taken else E_UNSUP)


def test_prompt_workspace_serves_smaller_calls():
    L = paro.lib()
    size = lambda T, b, hq=32, **kw: (L.paro_workspace_exchange_bytes_prompt(r(_cache(kv_heads=8, **kw)), hq, T, b), L.paro_workspace_bytes_prompt(r(_cache(kv_heads=8, **kw)), hq, T, b))
    for kw in (dict(), dict(head_dim=64), dict(head_dim=256)):
        for T, b in ((1, 1), (7, 3), (64, 64), (500, 5), (4096, 1), (100000, 300)):
            e, n = size(T, b, **kw)
            assert e % 256 == 0 and n % 256 == 0 and 0 < e < n
            for t in {1, T // 3 + 1, T - 1, T}:
                for c in {1, b // 2 + 1, b}:
                    if t:
                        e1, n1 = size(t, c, **kw)
                        assert e1 <= e and n1 - e1 <= n - e
    assert size(5, 3, 7) == (0, 0) and size(0, 1) == (0, 0) and size(1, 0) == (0, 0) and L.paro_workspace_bytes_prompt(None, 8, 1, 1) == 0
    # one counter for every 32 pairs of a row and one of a head's 4 queries, and for a part of each of the 3 sequences
    assert size(500, 3)[0] == 256 + -(-4 * 8 * (500 * 4 // 32 + 3) // 256) * 256


def test_mxfp4_cache_tensors():
    cache = paro.KVCache(3, 2, 128, 32, "mxfp4", device="cpu")
    assert cache.c.format == 4 and cache.head_dim == 128 and cache.k.shape == (3, 2, 4, 32, 16) and cache.v.shape == (3, 2, 32, 64) and cache.k_scale.shape == (3, 2, 4, 32)
    again = paro.KVCache.from_device(cache.k, cache.v, cache.k_scale, cache.v_scale)
    assert again.format == "mxfp4" and again.c.head_dim == 128 and again.c.page == 32
    for k, v, ks, vs in ((cache.k, cache.v, cache.k_scale[:, :, :2].contiguous(), cache.v_scale), (cache.k, cache.v, cache.k_scale, cache.v_scale.transpose(2, 3)),
                         (cache.k, cache.v.half(), cache.k_scale, cache.v_scale), (cache.k[:, :, :3].contiguous(), cache.v, cache.k_scale, cache.v_scale),
                         (cache.k, cache.v, cache.k_scale, None)):
        with pytest.raises(AssertionError):
            paro.KVCache.from_device(k, v, ks, vs)


@pytest.fixture(params=["native", "ctypes"])
def host(request):
    native = B._native()
    B._host = native if request.param == "native" else B._CtypesCalls
    yield
    B._host = native


def test_tensors_on_the_host(host):
    h = lambda *s: torch.zeros(s, dtype=torch.float16)
    cache, ws, i32 = paro.KVCache(2, 2, 64, 16, "mxfp4", device="cpu"), paro.Workspace(1 << 12, device="cpu"), torch.zeros(3, dtype=torch.int32)
    t = torch.zeros((3, 2), dtype=torch.int32)
    for call in (lambda: paro.paro_paged_attention(cache, h(3, 128), t, i32, ws, cap=5.0), lambda: paro.paro_kv_append(cache, h(3, 128), h(3, 128), i32.long()),
                 lambda: paro.paro_prompt_attention(cache, h(3, 128), torch.zeros(4, dtype=torch.int32), t, i32, ws)):
        with pytest.raises(AssertionError):
            call()


def test_tensors_of_two_gpus_or_other_kinds(host):
    cache = paro.KVCache(2, 2, 64, 16, "mxfp4", device="cpu")
    cache.c.device = 0
    ws = workspace(gpu(1 << 12, dtype=torch.uint8))
    i, f = torch.int32, torch.float32
    starts, slopes = gpu(4, dtype=i), gpu(2, dtype=f)
    prompt = lambda q=rows(), st=starts, tb=table(), ln=ints(), w=ws, **kw: paro.paro_prompt_attention(cache, q, st, tb, ln, w, **kw)
    step = lambda **kw: paro.paro_paged_attention(cache, rows(), table(), ints(), ws, **kw)
    for call in (lambda: prompt(st=gpu(4, dtype=i, at=1)), lambda: prompt(tb=table(1)), lambda: prompt(ln=ints(1)), lambda: prompt(w=workspace(gpu(1 << 12, dtype=torch.uint8, at=1))),
                 lambda: prompt(slopes=gpu(2, dtype=f, at=1)), lambda: prompt(prefix=ints(1)), lambda: prompt(first=ints(1)), lambda: step(slopes=gpu(2, dtype=f, at=1)),
                 lambda: prompt(q=rows(1), st=gpu(4, dtype=i, at=1), tb=table(1), ln=ints(1), w=workspace(gpu(1 << 12, dtype=torch.uint8, at=1)))):
        with pytest.raises(AssertionError, match="one GPU|not the current one"):
            call()
    for call in (lambda: prompt(st=gpu(3, dtype=i)), lambda: prompt(st=longs()), lambda: prompt(slopes=gpu(3, dtype=f)), lambda: prompt(slopes=gpu(2)), lambda: prompt(prefix=gpu(4, dtype=i)),
                 lambda: prompt(first=gpu(4, dtype=i)), lambda: prompt(q=gpu(3, 100)), lambda: prompt(q=gpu(3, 128, dtype=f)), lambda: prompt(window=2 ** 31),
                 lambda: step(slopes=gpu(3, dtype=f)), lambda: step(slopes=gpu(2)), lambda: step(cap=1.0, window=2 ** 31)):
        with pytest.raises(AssertionError):
            call()
