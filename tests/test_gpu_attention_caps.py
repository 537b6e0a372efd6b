"""Caps that scores of 0 and scores far beyond them meet at the ends of what a call takes; bounds: more_attention_ref.py."""
import numpy as np
import pytest

import more_attention_ref as more
from test_gpu_mxfp4_cache import cuda, filled, say, within
from test_gpu_prompt_attention import P, starts_of, workspace  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["fp16", "e4m3", "mxfp4"])
@pytest.mark.parametrize("scale,cap", [(1000.0, 1e-35), (1000.0, 1000 / 3e38), (-1000.0, 1000 / 3e38), (1e36, 1e-2), (3e37, 0.1), (0.0, 1e-30), (1e-30, 1e-6), (2e38, 64.0)])
def test_scores_of_zero_and_far_beyond(P, fmt, scale, cap):
    import torch
    assert np.isfinite(np.float32(scale) / np.float32(cap)) and np.isfinite(np.float32(scale) * np.float32(1.4426950408889634))
    say(f"scale {scale:g} cap {cap:g} {fmt}: rows of zeros, ordinary ones, keys of zeros")
    hq, hkv, D, new, lengths = 4, 2, 128, [3, 70], [5, 90]
    cache, table, rows = filled(P, lengths, hkv, D, 16, fmt, 3)
    for t in range(0, 90, 7):                        # keys of zeros in sequence 1
        page, off = int(table[1, t // 16]), t % 16
        cache.k[page, :, :, off] = 0
        rows[1][0][t] = 0
    q = np.random.default_rng(4).standard_normal((73, hq * D)).astype(np.float16)
    q[::5] = 0
    scale, cap = float(np.float32(scale)), float(np.float32(cap))
    ln, tb = cuda(np.asarray(lengths, np.int32)), cuda(table)
    at = [(0, i, 2 + i) for i in range(3)] + [(1, 3 + i, 20 + i) for i in range(70)]

    def check(o, lse, wanted):
        for i, name in ((0, "o"), (1, "lse")):
            within((o.float().cpu().numpy().reshape(-1, hq, D), lse.cpu().numpy())[i], np.stack([w[i] for w in wanted]), np.stack([w[i + 2] for w in wanted]), name)

    o, lse = P.paro_prompt_attention(cache, cuda(q), cuda(starts_of(new)), tb, ln, workspace(P, cache, hq, 73, 2), scale, 0, cap, with_lse=True)
    assert torch.isfinite(o).all() and torch.isfinite(lse).all()
    check(o, lse, [more.attention(q[r].reshape(hq, D), *rows[b], scale, 0, p + 1, p, cap) for b, r, p in at])
    for pick in ((0, 3), (2, 5), (1, 72)):           # rows 0 and 5 are zeros
        o, lse = P.paro_paged_attention(cache, cuda(q[list(pick)]), tb, ln, P.Workspace(P.paro_workspace_bytes_attention(cache, hq, 2)), scale, 0, with_lse=True, cap=cap)
        assert torch.isfinite(o).all() and torch.isfinite(lse).all()
        check(o, lse, [more.attention(q[r].reshape(hq, D), *rows[b], scale, 0, n, n - 1, cap, rounded=False) for b, (r, n) in enumerate(zip(pick, lengths))])
