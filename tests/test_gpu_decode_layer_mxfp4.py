"""The operators together over an MXFP4 cache, as examples/decode_layer.py serves with them: prompts in one or two pieces, then token by token.

Bound: that of test_gpu_decode_layer.py, and half a step of E2M1, 2^-2 of a value, for keys and values, independent from channel to channel."""
import numpy as np
import pytest

from test_gpu_decode_layer import BOUND, far, layer_64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", ["fp16", "mxfp4"])
def test_pieces_and_tokens(cache):
    import torch
    import decode_layer as E
    batch, prompt, steps = 3, 37, 4
    seqs = E.Sequences(batch, prompt + steps, 16)
    layer = E.DecoderLayer(**E.SHAPES["tiny"], pages=seqs.pages, cache=cache)
    ws = layer.workspace((batch, batch * prompt, batch * (prompt + steps)))
    x = torch.randn((batch, prompt + steps, 512), generator=torch.Generator(device="cuda").manual_seed(5), device="cuda").half()
    whole = E.prefill(layer, seqs, x, ws).float().cpu().numpy()
    seqs.lengths.zero_()
    first = [E.prefill(layer, seqs, x[:, a:b], ws).float().cpu().numpy() for a, b in ((0, 20), (20, prompt))]
    decode = E.Decoder(layer, seqs, 512, ws)
    later = [decode(x[:, prompt + i]).float().cpu().numpy() for i in range(steps)]
    torch.cuda.synchronize()
    assert seqs.lengths.tolist() == [prompt + steps] * batch and ws.error_word() == 0
    stepped = np.concatenate([*first, np.stack(later, 1)], 1)
    want = np.stack([layer_64(layer, x[b].cpu().numpy(), np.arange(prompt + steps)) for b in range(batch)])
    bound = BOUND + (2.0 ** -2 if cache == "mxfp4" else 0)
    print(f"{cache}: whole {far(whole, want):.2e}, stepped {far(stepped, want):.2e}, each other {far(stepped, whole):.2e}")
    assert far(whole, want) <= bound and far(stepped, want) <= bound and far(stepped, whole) <= bound
