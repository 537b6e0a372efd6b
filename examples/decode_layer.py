"""One quantised decoder layer that serves tokens: prompts into a paged cache, then one token of every sequence after the other.

    python examples/decode_layer.py [--batch 16] [--prompt 512] [--steps 64] [--cache fp16|e4m3] [--tiny]

The linears are the library's rotated W4A16 ones (random weights, transformed and quantised here), and everything between
them is the library's too, but for the gate's activation, which is torch's: norm with the residual, rotary positions on the way into the cache,
attention over the cache.  The decode step is captured once as a HIP graph and replayed.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2511_10645_amd as paro  # noqa: E402
import paro_inputs as pin  # noqa: E402

EPS = 1e-5


class Linear:
    """A rotated W4A16 linear with random weights: transform planned, weight quantised and repacked."""

    def __init__(self, seed: int, c_in: int, c_out: int):
        rs = np.random.default_rng(seed)
        groups = c_in // pin.GROUP
        pairs = pin.draw_matchings(rs, groups, pin.N_LAYERS)
        theta = rs.uniform(-np.pi, np.pi, size=pairs.shape[:3]).astype(np.float32)
        self.rot = paro.Rotation(pairs, theta, np.exp(rs.normal(0, 0.2, c_in)).astype(np.float16))
        paro.paro_rotation_plan_build(self.rot)
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.w = paro.paro_w4_quantize(self.rot, (torch.randn((c_out, c_in), generator=g, device="cuda") * c_in ** -0.5).half())
        paro.paro_w4_repack(self.w)

    def __call__(self, x, ws):
        return paro.paro_rotated_linear(self.rot, self.w, x, ws)


class DecoderLayer:
    def __init__(self, hidden: int, q_heads: int, kv_heads: int, head_dim: int, mlp: int, pages: int, page: int = 16, cache: str = "fp16", seed: int = 0):
        self.q, self.kv, self.mlp, self.head_dim, self.q_heads = q_heads * head_dim, kv_heads * head_dim, mlp, head_dim, q_heads
        self.qkv = Linear(seed, hidden, self.q + 2 * self.kv)
        self.o = Linear(seed + 1, self.q, hidden)
        self.gate_up = Linear(seed + 2, hidden, 2 * mlp)
        self.down = Linear(seed + 3, mlp, hidden)
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.norms = [(1 + 0.1 * torch.randn(hidden, generator=g, device="cuda")).half() for _ in range(2)]
        self.cache = paro.KVCache(pages, kv_heads, head_dim, page, cache)
        freqs, magnitude = paro.paro_rope_frequencies_host(head_dim, 500000.0, "parts", factor=8, trained=8192)
        self.rope = paro.Rope(freqs, head_dim, magnitude=magnitude)

    def workspace(self, tokens):
        """One for all calls of any of these token counts."""
        linears = (self.qkv, self.o, self.gate_up, self.down)
        return paro.Workspace.shared([(x.rot, x.w, t) for x in linears for t in tokens], attention=[(self.cache, self.q_heads, t) for t in tokens])

    def __call__(self, x, residual, positions, slots, table, lengths, ws):
        """x [T][hidden], one row per token; table and lengths: the tokens that each row attends to, its own among them."""
        if residual is None:
            n, h = paro.paro_rms_norm(x, self.norms[0], EPS), x
        else:
            n, h = paro.paro_rms_norm(x, self.norms[0], EPS, residual=residual)
        q, k, v = self.qkv(n, ws).split((self.q, self.kv, self.kv), 1)
        q = paro.paro_kv_append(self.cache, k, v, slots, self.rope, positions, q, q)
        a = paro.paro_paged_attention(self.cache, q, table, lengths, ws)
        n, h = paro.paro_rms_norm(self.o(a, ws), self.norms[1], EPS, residual=h)
        gate, up = self.gate_up(n, ws).split((self.mlp, self.mlp), 1)
        return self.down(torch.nn.functional.silu(gate) * up, ws), h


class Sequences:
    """Pages of a batch of sequences (all of one capacity, scattered over the cache) and how far each has come."""

    def __init__(self, batch: int, capacity: int, page: int, seed: int = 0):
        per = -(-capacity // page)
        self.pages, self.page, self.batch = batch * per, page, batch
        g = torch.Generator().manual_seed(seed)
        self.table = torch.randperm(self.pages, generator=g).int().view(batch, per).cuda()
        self.lengths = torch.zeros(batch, dtype=torch.int32, device="cuda")

    def slots(self, sequence, positions):
        p = positions.long()
        return self.table[sequence, p // self.page].long() * self.page + p % self.page


def prefill(layer: DecoderLayer, seqs: Sequences, x, ws):
    """x [batch][tokens][hidden]: the same number of prompt tokens for every sequence.  Every token is a row of its own that
    attends to the tokens before it; keys and values of all are in the cache before the attention reads it."""
    b, t, hidden = x.shape
    sequence = torch.arange(b, device="cuda").repeat_interleave(t)
    positions = (seqs.lengths[:, None] + torch.arange(t, device="cuda", dtype=torch.int32)).flatten()
    y, h = layer(x.reshape(b * t, hidden), None, positions, seqs.slots(sequence, positions), seqs.table[sequence], positions + 1, ws)
    seqs.lengths += t
    return (y + h).view(b, t, hidden)


class Decoder:
    """The captured step of one token per sequence.  A replay reads the memory that the capture saw, so everything that the step
    uses from outside is kept here."""

    def __init__(self, layer: DecoderLayer, seqs: Sequences, hidden: int, ws):
        self.x = torch.zeros((seqs.batch, hidden), dtype=torch.float16, device="cuda")
        self.rows = rows = torch.arange(seqs.batch, device="cuda")
        self.uses = layer, seqs, ws

        def step():
            positions = seqs.lengths.clone()
            y, h = layer(self.x, None, positions, seqs.slots(rows, positions), seqs.table, positions + 1, ws)
            seqs.lengths += 1
            return y + h

        before = seqs.lengths.clone()
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            step()                              # whatever a first call sets up is set up outside the capture
        torch.cuda.current_stream().wait_stream(s)
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self.out = step()
        seqs.lengths.copy_(before)

    def __call__(self, x):
        self.x.copy_(x)
        self.graph.replay()
        return self.out


SHAPES = {"8b": dict(hidden=4096, q_heads=32, kv_heads=8, head_dim=128, mlp=14336), "tiny": dict(hidden=512, q_heads=8, kv_heads=2, head_dim=64, mlp=1024)}


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--batch", type=int, default=16)
    ap.add_argument("--prompt", type=int, default=512)
    ap.add_argument("--steps", type=int, default=64)
    ap.add_argument("--cache", choices=("fp16", "e4m3"), default="fp16")
    ap.add_argument("--tiny", action="store_true")
    a = ap.parse_args()
    shape = SHAPES["tiny" if a.tiny else "8b"]
    seqs = Sequences(a.batch, a.prompt + a.steps + 2, 16)
    layer = DecoderLayer(**shape, pages=seqs.pages, cache=a.cache)
    ws = layer.workspace((a.batch, a.batch * a.prompt))
    g = torch.Generator(device="cuda").manual_seed(1)
    prompt = torch.randn((a.batch, a.prompt, shape["hidden"]), generator=g, device="cuda").half()
    prefill(layer, seqs, prompt, ws)
    torch.cuda.synchronize()
    seqs.lengths.zero_()
    t = time.perf_counter()
    y = prefill(layer, seqs, prompt, ws)
    torch.cuda.synchronize()
    print(f"prompt: {a.batch} x {a.prompt} tokens in {(time.perf_counter() - t) * 1e3:.2f} ms")
    decode = Decoder(layer, seqs, shape["hidden"], ws)

    def next_token(x):                          # stands in for the other layers: the row again, of the size of an embedding
        x = decode(x)
        return x / x.float().square().mean(1, keepdim=True).sqrt().half()

    x = next_token(y[:, -1])                    # the first time also loads torch's kernels and uploads the graph
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(a.steps):
        x = next_token(x)
    torch.cuda.synchronize()
    us = (time.perf_counter() - t) / a.steps * 1e6
    print(f"decode: {a.batch} sequences, cache {a.cache}, {us:.1f} us a step ({a.batch / us * 1e6:.0f} tokens/s through this layer), lengths now {int(seqs.lengths[0])}")
    print("finite:", bool(torch.isfinite(x).all()), " exchange error word:", ws.error_word())


if __name__ == "__main__":
    main()
