"""Refusals of the operators between the linears, their workspace's size and the frequencies of rotary positions: no GPU is needed."""
import ctypes
import math

import numpy as np
import pytest

import paper_2511_10645_amd as paro
from paper_2511_10645_amd import binding as B

E_NULL, E_SHAPE, E_ALIGN, E_UNSUP, E_WS = 1, 2, 3, 5, 6
FAKE = 0x10000
r = ctypes.byref


def _cache(n_pages=4, page=16, kv_heads=2, head_dim=128, format=0, k=FAKE, v=FAKE, ks=None, vs=None):
    return B._CKVCache(n_pages, page, kv_heads, head_dim, format, k, v, ks, vs)


def _rope(head_dim=128, rot_dim=128, layout=0, magnitude=1.0, f=FAKE):
    return B._CRope(head_dim, rot_dim, layout, magnitude, f)


def test_norm_refusals():
    L = paro.lib()
    f = lambda X=FAKE, ldx=256, R=None, ldr=0, w=FAKE, eps=1e-5, T=2, C=256, H=None, ldh=0, Y=FAKE * 2, ldy=256: L.paro_rms_norm(
        X, ldx, R, ldr, w, eps, T, C, H, ldh, Y, ldy, None)
    q = lambda codes=FAKE, scales=FAKE, group=128, C=256, ldx=256, X=FAKE: L.paro_rms_norm_quantize_e4m3(
        X, ldx, None, 0, FAKE, 1e-5, group, 2, C, None, 0, codes, scales, None)
    assert f(X=None) == E_NULL and f(w=None) == E_NULL and f(Y=None) == E_NULL
    assert f(T=0) == E_SHAPE and f(C=0) == E_SHAPE and f(ldx=128) == E_SHAPE and f(ldy=248) == E_SHAPE
    assert f(eps=-1.0) == E_SHAPE and f(eps=math.nan) == E_SHAPE and f(eps=math.inf) == E_SHAPE
    assert f(C=252) == E_ALIGN and f(X=FAKE + 2) == E_ALIGN and f(ldx=260) == E_ALIGN and f(w=FAKE + 8) == E_ALIGN
    assert f(R=FAKE, ldr=8) == E_SHAPE and f(R=FAKE + 8, ldr=256) == E_ALIGN and f(H=FAKE, ldh=128) == E_SHAPE
    assert f(C=32776, ldx=32776, ldy=32776) == E_UNSUP and f(T=2 ** 21 + 1) == E_UNSUP and f(T=2 ** 31 - 1) == E_UNSUP
    assert f(H=FAKE * 2, ldh=256) == E_SHAPE                            # H and Y in one place
    assert f(Y=FAKE, ldy=512) == E_SHAPE and f(H=FAKE, ldh=512) == E_SHAPE        # in place with other strides
    assert q(codes=None) == E_NULL and q(scales=None) == E_NULL and q(group=64) == E_UNSUP and q(C=264, ldx=264) == E_SHAPE
    assert q(codes=FAKE + 4) == E_ALIGN and q(scales=FAKE + 2) == E_ALIGN and q(X=None) == E_NULL


def test_rope_and_append_refusals():
    L = paro.lib()
    f = lambda rp=_rope(), X=FAKE, ldx=256, pos=FAKE, heads=2, T=1, Y=FAKE * 2, ldy=256: L.paro_rope(r(rp) if rp else None, X, ldx, pos, heads, T, Y, ldy, None)
    assert f(rp=None) == E_NULL and f(rp=_rope(f=None)) == E_NULL and f(X=None) == E_NULL and f(pos=None) == E_NULL and f(Y=None) == E_NULL
    assert f(T=0) == E_SHAPE and f(heads=0) == E_SHAPE and f(heads=3) == E_SHAPE and f(rp=_rope(rot_dim=144)) == E_SHAPE
    assert f(rp=_rope(magnitude=math.inf)) == E_SHAPE and f(Y=FAKE, ldy=264) == E_SHAPE
    assert f(rp=_rope(rot_dim=24)) == E_UNSUP and f(rp=_rope(layout=2)) == E_UNSUP and f(rp=_rope(head_dim=100, rot_dim=16)) == E_UNSUP
    assert f(rp=_rope(head_dim=528, rot_dim=16)) == E_UNSUP and f(T=2 ** 31 - 1) == E_UNSUP
    assert f(X=FAKE + 2) == E_ALIGN and f(pos=FAKE + 2) == E_ALIGN and f(ldx=260) == E_ALIGN
    a = lambda c=_cache(), rp=_rope(), K=FAKE, ldk=256, V=FAKE, ldv=256, slots=FAKE, pos=FAKE, T=1, Q=FAKE, ldq=512, hq=4, Qr=FAKE * 2, ldqr=512: L.paro_kv_append(
        r(c) if c else None, r(rp) if rp else None, K, ldk, V, ldv, slots, pos, T, Q, ldq, hq, Qr, ldqr, None)
    assert a(c=None) == E_NULL and a(c=_cache(k=None)) == E_NULL and a(c=_cache(v=None)) == E_NULL and a(c=_cache(format=1)) == E_NULL
    assert a(K=None) == E_NULL and a(V=None) == E_NULL and a(slots=None) == E_NULL and a(pos=None) == E_NULL and a(Qr=None) == E_NULL
    assert a(c=_cache(n_pages=0)) == E_SHAPE and a(c=_cache(kv_heads=0)) == E_SHAPE and a(T=0) == E_SHAPE and a(hq=0) == E_SHAPE
    assert a(c=_cache(page=8)) == E_UNSUP and a(c=_cache(page=24)) == E_UNSUP and a(c=_cache(page=2048)) == E_UNSUP and a(c=_cache(head_dim=96)) == E_UNSUP
    assert a(c=_cache(format=2)) == E_UNSUP and a(T=2 ** 31 - 1) == E_UNSUP
    assert a(rp=_rope(head_dim=64, rot_dim=64)) == E_SHAPE and a(ldk=128) == E_SHAPE and a(ldv=128) == E_SHAPE and a(ldq=256) == E_SHAPE and a(ldqr=256) == E_SHAPE
    assert a(Q=FAKE, Qr=FAKE, ldqr=520) == E_SHAPE
    assert a(c=_cache(k=FAKE + 8)) == E_ALIGN and a(c=_cache(format=1, ks=FAKE + 1, vs=FAKE)) == E_ALIGN and a(slots=FAKE + 4) == E_ALIGN and a(pos=FAKE + 2) == E_ALIGN
    assert a(K=FAKE + 2) == E_ALIGN and a(ldv=260) == E_ALIGN


def test_attention_refusals_and_workspace():
    L = paro.lib()
    need = L.paro_workspace_bytes_attention(r(_cache()), 8, 3)
    f = lambda c=_cache(), Q=FAKE, ldq=1024, hq=8, table=FAKE, ldt=4, width=4, lengths=FAKE, batch=3, scale=0.1, window=0, O=FAKE * 4, ldo=1024, lse=None, ws=FAKE, n=need: \
        L.paro_paged_attention(r(c) if c else None, Q, ldq, hq, table, ldt, width, lengths, batch, scale, window, O, ldo, lse, ws, n, None)
    assert f(c=None) == E_NULL and f(Q=None) == E_NULL and f(O=None) == E_NULL and f(table=None) == E_NULL and f(lengths=None) == E_NULL
    assert f(batch=0) == E_SHAPE and f(hq=7) == E_SHAPE and f(hq=0) == E_SHAPE and f(width=0) == E_SHAPE and f(window=-1) == E_SHAPE and f(ldt=3) == E_SHAPE
    assert f(O=FAKE) == E_SHAPE                                         # the queries themselves
    assert f(scale=3e38) == E_SHAPE                                     # finite, but not in units of log2
    assert f(scale=math.nan) == E_SHAPE and f(scale=math.inf) == E_SHAPE and f(ldq=512) == E_SHAPE and f(ldo=512) == E_SHAPE
    assert f(Q=FAKE + 2) == E_ALIGN and f(ldo=1028) == E_ALIGN and f(lse=FAKE + 2) == E_ALIGN and f(ws=FAKE + 128) == E_ALIGN and f(lengths=FAKE + 1) == E_ALIGN
    assert f(ws=None) == E_WS and f(n=need - 1) == E_WS
    assert f(width=1 << 27, ldt=1 << 27) == E_UNSUP and f(batch=1 << 20, width=1 << 14, ldt=0, n=1 << 40) == E_UNSUP
    ex = L.paro_workspace_exchange_bytes_attention(r(_cache()), 8, 3)
    assert ex == 256 + 2304 and need > ex                             # 512 counters of groups of blocks, 6 of heads
    assert L.paro_workspace_exchange_bytes_attention(r(_cache()), 8, 1000) == 256 + 10240     # 2000 heads
    assert L.paro_workspace_exchange_bytes_attention(r(_cache(kv_heads=1)), 40, 100) == 256 + 3328        # 3 x 16 query heads
    assert L.paro_workspace_bytes_attention(r(_cache()), 7, 3) == 0 and L.paro_workspace_bytes_attention(None, 8, 3) == 0
    assert L.paro_workspace_bytes_attention(r(_cache()), 8, 0) == 0


def test_tensors_are_checked_in_both_bindings():
    """On the CPU every call is refused before the library sees a pointer."""
    import torch
    h = lambda *s: torch.zeros(s, dtype=torch.float16)
    cache, rope = paro.KVCache(2, 2, 64, 16, device="cpu"), paro.Rope(np.ones(32, np.float32), 64, device="cpu")
    ws = paro.Workspace(1 << 12, device="cpu")
    i32, i64 = torch.zeros(3, dtype=torch.int32), torch.zeros(3, dtype=torch.int64)
    native = B._native()
    try:
        for host in (native, B._CtypesCalls):
            B._host = host
            for call in (lambda: paro.paro_rms_norm(h(3, 64), h(64), 1e-5), lambda: paro.paro_rms_norm(torch.zeros(3, 64), h(64), 1e-5),
                         lambda: paro.paro_rms_norm(h(3, 128)[:, ::2], h(64), 1e-5), lambda: paro.paro_rms_norm_quantize_e4m3(h(3, 64), h(64), 1e-5),
                         lambda: paro.paro_rope(rope, h(3, 128), i32), lambda: paro.paro_kv_append(cache, h(3, 128), h(3, 128), i64),
                         lambda: paro.paro_paged_attention(cache, h(3, 128), torch.zeros((3, 2), dtype=torch.int32), i32, ws)):
                with pytest.raises(AssertionError):
                    call()
    finally:
        B._host = native
    with pytest.raises(TypeError):
        paro.paro_rope(cache, h(3, 128), i32)                           # a cache, not a rope
    with pytest.raises(TypeError):
        paro.paro_rms_norm(np.zeros((3, 64), np.float16), h(64), 1e-5)
    with pytest.raises(AssertionError):
        paro.KVCache.from_device(h(2, 2, 8, 16, 8), h(2, 2, 16, 128))
    with pytest.raises(KeyError):
        paro.Rope(np.ones(32, np.float32), 64, layout="pairs", device="cpu")


def test_rope_frequencies():
    n, base = 128, 500000.0
    f = base ** (-np.arange(0, n, 2) / n)
    got, m = paro.paro_rope_frequencies_host(n, base)
    assert m == 1 and np.array_equal(got, f.astype(np.float32))
    got, m = paro.paro_rope_frequencies_host(n, base, "linear", 4)
    assert m == 1 and np.allclose(got, f / 4, rtol=1e-7)
    got, _ = paro.paro_rope_frequencies_host(n, base, "base", 4)
    assert np.allclose(got, (base * 4 ** (n / (n - 2))) ** (-np.arange(0, n, 2) / n), rtol=1e-6)
    assert math.isclose(got[-1], f[-1] / 4, rel_tol=1e-6)              # the slowest pair turns as with "linear"
    got, m = paro.paro_rope_frequencies_host(n, base, "parts", 8, 8192, 1, 4)
    turns = 8192 * f / (2 * math.pi)
    assert m == 1 and np.array_equal(got[turns >= 4], f[turns >= 4].astype(np.float32)) and np.allclose(got[turns <= 1], f[turns <= 1] / 8, rtol=1e-7)
    between = (turns > 1) & (turns < 4)
    assert between.any() and (got[between] < f[between]).all() and (got[between] > f[between] / 8).all()
    got, m = paro.paro_rope_frequencies_host(n, 10000.0, "channels", 16, 4096, 1, 32)
    f = 10000.0 ** (-np.arange(0, n, 2) / n)
    assert math.isclose(m, 0.1 * math.log(16) + 1, rel_tol=1e-6)
    lo, hi = (n * math.log(4096 / (2 * math.pi * t)) / (2 * math.log(10000.0)) for t in (32, 1))
    i = np.arange(n // 2)
    s = 1 - np.clip((i - math.floor(lo)) / (math.ceil(hi) - math.floor(lo)), 0, 1)
    assert np.allclose(got, s * f + (1 - s) * f / 16, rtol=1e-6)
    L = paro.lib()
    buf = np.zeros(64, np.float32)
    g = lambda rot=128, base=1e4, kind=3, factor=2.0, trained=4096.0, low=1.0, high=4.0, p=buf.ctypes.data: L.paro_rope_frequencies_host(
        rot, base, kind, factor, trained, low, high, p, buf.ctypes.data)
    assert g(p=None) == E_NULL and g(kind=5) == E_UNSUP and g(kind=-1) == E_UNSUP
    for bad in (dict(rot=0), dict(rot=7), dict(base=1.0), dict(base=math.nan), dict(factor=0.5), dict(factor=math.inf), dict(trained=0.0), dict(low=0.0),
                dict(low=4.0), dict(high=math.inf), dict(kind=2, rot=2)):
        assert g(**bad) == E_SHAPE, bad
    assert g() == 0 and g(kind=0, factor=0.0, trained=0.0, low=0.0, high=0.0) == 0
