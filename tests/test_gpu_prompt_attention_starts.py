"""Starts that fall or lie outside the rows are taken as the largest before them, within 0..T: every such call equals the one with those."""
import numpy as np
import pytest

from test_gpu_mxfp4_cache import cuda, filled, say
from test_gpu_prompt_attention import P, workspace  # noqa: F401

pytestmark = pytest.mark.gpu

FALLING = [(500, [0, 300, 0, 500]), (500, [0, 500, 0, 500, 0, 500]), (500, [400, 100, 450, 20, 500]), (500, [-7, 300, 2 ** 31 - 1, -2 ** 31, 400]),
           (20, [0, 15, 3, 20]), (20, [5, 20, 0, 20, 0, 20])]


@pytest.mark.parametrize("T,starts", FALLING)
@pytest.mark.parametrize("fmt,hq,hkv,D", [("fp16", 8, 2, 128), ("mxfp4", 4, 1, 64), ("e4m3", 4, 2, 256)])
def test_falling(P, fmt, hq, hkv, D, T, starts):
    say(f"{T} rows, starts {starts}, {fmt} {hq}/{hkv} x {D}")
    run(P, fmt, hq, hkv, D, T, np.array(starts), [520] * (len(starts) - 1))


@pytest.mark.parametrize("seed", range(3))
def test_falling_beyond_64_sequences(P, seed):
    rs = np.random.default_rng(seed)
    starts = np.sort(rs.integers(0, 600, 201))
    starts[rs.integers(0, 201, 40)] = rs.integers(-50, 700, 40)
    say(f"200 sequences, seed {seed}")
    run(P, "fp16", 4, 2, 64, 600, starts, [int(n) for n in rs.integers(0, 30, 200)])


def run(P, fmt, hq, hkv, D, T, starts, lengths):
    import torch
    cache, table, _ = filled(P, lengths, hkv, D, 16, fmt, T)
    q, tb, ln = cuda(np.random.default_rng(1).standard_normal((T, hq * D)).astype(np.float16)), cuda(table), cuda(np.array(lengths, np.int32))
    ws = workspace(P, cache, hq, T, len(lengths))
    rising = np.maximum.accumulate(np.clip(starts, 0, T))
    got = []
    for st in (starts, rising):
        out = torch.full((T, hq * D), 7.0, dtype=torch.float16, device="cuda")
        P.paro_prompt_attention(cache, q, cuda(st.astype(np.int32)), tb, ln, ws, O=out)
        got.append(out)
    same = torch.equal(*got)
    assert same
    written = np.zeros(T, bool)
    written[rising[0]:rising[-1]] = True
    assert (got[0][cuda(~written)] == 7).all() and (got[0][cuda(written)] != 7).any(1).all()
    assert ws.partials_clean(P.paro_workspace_exchange_bytes_prompt(cache, hq, T, len(lengths)))
