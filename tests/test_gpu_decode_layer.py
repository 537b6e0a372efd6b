"""The operators together, as examples/decode_layer.py serves with them: a small layer against its formula in 64 bits, and decoding
token by token against the whole prompt at once.

Bound (2-norm of a row): a row passes about 8 fp16 roundings (norm, qkv, rotated q and k, attention, o, norm, gate/up, product, down), each 2^-11
of its size at most, and the linears multiply a rounding of their input by no more than their input; twice that for the two sums of the residual:
2 * 8 * 2^-11 = 8e-3.  An E4M3 cache adds half a unit of its 4 bits, 2^-4, to keys and values, independent from channel to channel."""
import os
import sys

import numpy as np
import pytest

import oracle
import token_path_ref as ref

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
BOUND = 2 * 8 * 2.0 ** -11


def far(got, want):
    return float(np.max(np.linalg.norm(got - want, axis=-1) / np.linalg.norm(want, axis=-1)))


def linear(lin, x):
    """W^ . transform(x) in 64 bits from the library's quantised weight."""
    import paper_2511_10645_amd as P
    r, w = lin.rot, P.paro_w4_dequant(lin.w).cpu().numpy().astype(np.float64)
    u = oracle.rotate_scale(np.ascontiguousarray(x.astype(np.float16)), r.pairs.cpu().numpy(), r.theta.cpu().numpy(), r.ch_scale.cpu().numpy())
    return u @ w.T


def layer_64(layer, x, positions):
    """One sequence's rows [T][hidden]."""
    D, T = layer.head_dim, len(x)
    w = [n.cpu().numpy() for n in layer.norms]
    _, n = ref.rms_norm(x, None, w[0], 1e-5)
    qkv = linear(layer.qkv, n)
    f = layer.rope.inv_freq.cpu().numpy()
    q, k, v = (t.reshape(T, -1, D) for t in np.split(qkv, [layer.q, layer.q + layer.kv], axis=1))
    q, k = (ref.rotate(t, positions, f, "halves", layer.rope.c.magnitude) for t in (q, k))
    a = np.stack([ref.attention(q[t], k[:t + 1], v[:t + 1], D ** -0.5)[0].reshape(-1) for t in range(T)])
    h, n = ref.rms_norm(linear(layer.o, a).astype(np.float64), x, w[1], 1e-5)
    gate, up = np.split(linear(layer.gate_up, n), 2, axis=1)
    return linear(layer.down, gate / (1 + np.exp(-gate)) * up) + h


@pytest.mark.parametrize("cache", ["fp16", "e4m3"])
def test_layer(cache):
    import torch
    import decode_layer as E
    batch, prompt, steps = 3, 37, 5
    seqs = E.Sequences(batch, prompt + steps, 16)
    layer = E.DecoderLayer(**E.SHAPES["tiny"], pages=seqs.pages, cache=cache)
    ws = layer.workspace((batch, batch * prompt, batch * (prompt + steps)))
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn((batch, prompt + steps, 512), generator=g, device="cuda").half()
    whole = E.prefill(layer, seqs, x, ws).float().cpu().numpy()
    seqs.lengths.zero_()
    first = E.prefill(layer, seqs, x[:, :prompt], ws).float().cpu().numpy()
    decode = E.Decoder(layer, seqs, 512, ws)
    later = [decode(x[:, prompt + i]).float().cpu().numpy() for i in range(steps)]
    torch.cuda.synchronize()
    assert seqs.lengths.tolist() == [prompt + steps] * batch and ws.error_word() == 0
    stepped = np.concatenate([first, np.stack(later, 1)], 1)
    want = np.stack([layer_64(layer, x[b].cpu().numpy(), np.arange(prompt + steps)) for b in range(batch)])
    bound = BOUND + (2.0 ** -4 if cache == "e4m3" else 0)
    print(f"{cache}: whole {far(whole, want):.2e}, stepped {far(stepped, want):.2e}, each other {far(stepped, whole):.2e}")
    assert far(whole, want) <= bound and far(stepped, want) <= bound and far(stepped, whole) <= bound
