"""Calls whose weights of the softmax enter the product with the values as two fp16 numbers: bounds without the rounding of a weight to one."""
import numpy as np
import pytest

import more_attention_ref as more
from test_gpu_mxfp4_cache import cuda, filled, say, slopes_of, within
from test_gpu_prompt_attention import P, starts_of, workspace  # noqa: F401

pytestmark = pytest.mark.gpu


def check(P, cache, table, rows, new, lengths, hq, **kw):
    D, T = cache.head_dim, sum(new)
    # of 256 channels a quarter, so that what scores may be off by stays below a weight's 2^-11
    q = (np.random.default_rng(T + hq).standard_normal((T, hq * D)) * (0.25 if D == 256 else 1)).astype(np.float16)
    arrays = {k: cuda(v) if isinstance(v, np.ndarray) else v for k, v in kw.items()}
    o = P.paro_prompt_attention(cache, cuda(q), cuda(starts_of(new)), cuda(table), cuda(np.asarray(lengths, np.int32)), workspace(P, cache, hq, T, len(new)), **arrays)
    want, bound, r = np.zeros((T, hq, D)), np.zeros((T, hq, D)), 0
    for b, (m, n) in enumerate(zip(new, lengths)):
        for p in range(n - m, n):
            want[r], _, bound[r], _ = more.attention(q[r].reshape(hq, D), *rows[b], D ** -0.5, 0, p + 1, p, kw.get("cap", 0.0), kw.get("slopes"), rounded=False)
            # a weight held 2^10 times as two fp16 numbers: off by 2^-22 of itself (which more.attention's 2^-20 has room for) or by 2^-25, 2^-35 of the largest,
            # against a sum of 1 at least
            bound[r] += 2.0 ** -35 * np.repeat(np.abs(rows[b][1][:p + 1]).sum(0), hq // cache.kv_heads, 0)
            r += 1
    within(o.cpu().numpy().reshape(T, hq, D), want, bound, "o")


@pytest.mark.parametrize("fmt", ["fp16", "e4m3", "mxfp4"])
@pytest.mark.parametrize("hq,hkv,D", [(4, 2, 64), (8, 2, 128), (6, 2, 256)])
def test_few_rows(P, fmt, hq, hkv, D):
    say(f"few rows, {fmt} {hq}/{hkv} x {D}")
    new, lengths = [1, 3, 7, 5, 2], [1, 3, 70, 300, 1500]
    check(P, *filled(P, lengths, hkv, D, 16, fmt, D), new, lengths, hq)


@pytest.mark.parametrize("fmt", ["fp16", "e4m3", "mxfp4"])
@pytest.mark.parametrize("hq,hkv,D,scores", [(4, 1, 256, {}), (8, 2, 128, dict(cap=30.0)), (4, 1, 64, dict(slopes=slopes_of(4)))])
def test_many_rows(P, fmt, hq, hkv, D, scores):
    say(f"many rows, {fmt} {hq}/{hkv} x {D} {list(scores)}")
    new, lengths = [40, 70], [40, 600]
    check(P, *filled(P, lengths, hkv, D, 16, fmt, D), new, lengths, hq, **scores)
