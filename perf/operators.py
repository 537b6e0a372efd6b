"""What stands between the quantised linears of a decoder layer when tokens are served, as cases that can be timed and compared.

Four operators, for fp16 activations as the linears take and give them:

  norm       ``paro_rms_norm`` / ``paro_rms_norm_quantize_e4m3``: h = x + r, y = h / sqrt(mean(h^2) + eps) * w; y in fp16, or in
             E4M3 with fp32 scales per row or per 128 channels
  rope       ``paro_rope``: rotary positions of the first channels of every head
  append     ``paro_kv_append``: the same rotation of queries and keys, keys and values written to their slots of a paged cache,
             in fp16 or in E4M3 with a power-of-two scale per token and head
  attention  ``paro_paged_attention``: one new token of every sequence against the paged cache

Head counts and widths are those of the layers of ``paro_inputs.CONFIGS``: 4096 -> 6144 is 32 query and 8 key-value heads of 128
channels, 5120 -> 7168 is 40 and 8; others are generic.  ``own`` false computes the formulas in elementary fp32 operations.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5


def listed():
    return [
        # the norm in front of a linear at batch-1 decode: a call's latency
        {"name": "norm_t1", "op": "norm", "tokens": 1, "width": 4096, "residual": True, "bits": 16, "group": 0},
        # the same over a prompt of odd length on the wider layer
        {"name": "norm_t2047", "op": "norm", "tokens": 2047, "width": 5120, "residual": True, "bits": 16, "group": 0},
        # 8-bit activations for a whole prefill batch, one scale per 128 channels (the linears' group)
        {"name": "norm_e4m3_t4096", "op": "norm", "tokens": 4096, "width": 4096, "residual": True, "bits": 8, "group": 128},
        # rotary positions alone: queries of 16 decoding sequences, adjacent channels paired, half of each head rotated
        {"name": "rope_t16", "op": "rope", "tokens": 16, "heads": 32, "dim": 128, "rot": 64, "layout": "interleaved", "scaling": "none", "longest": 4096},
        # the same over a long prompt of odd length, whole heads, frequencies stretched to a long context
        {"name": "rope_t4095", "op": "rope", "tokens": 4095, "heads": 40, "dim": 128, "rot": 128, "layout": "halves", "scaling": "parts", "longest": 32768},
        # one decode step of 16 sequences: every token goes to a page of its own
        {"name": "append_t16", "op": "append", "tokens": 16, "q_heads": 32, "kv_heads": 8, "dim": 128, "rot": 128, "layout": "halves", "bits": 16, "page": 16,
         "prompt": False},
        # a prompt into an 8-bit cache
        {"name": "append_e4m3_t2048", "op": "append", "tokens": 2048, "q_heads": 40, "kv_heads": 8, "dim": 128, "rot": 128, "layout": "halves", "bits": 8,
         "page": 16, "prompt": True},
        # one short conversation: a call's latency
        {"name": "attn_b1_700", "op": "attention", "batch": 1, "longest": 700, "shortest": 700, "q_heads": 32, "kv_heads": 8, "dim": 128, "bits": 16,
         "page": 16, "window": 0},
        # batched decode, 16 conversations of very different lengths
        {"name": "attn_b16_4096", "op": "attention", "batch": 16, "longest": 4096, "shortest": 1, "q_heads": 32, "kv_heads": 8, "dim": 128, "bits": 16,
         "page": 16, "window": 0},
        # a loaded server with an 8-bit cache
        {"name": "attn_e4m3_b64_8192", "op": "attention", "batch": 64, "longest": 8192, "shortest": 1000, "q_heads": 40, "kv_heads": 8, "dim": 128, "bits": 8,
         "page": 32, "window": 0},
        # one very long document: the cache's length is all there is to split
        {"name": "attn_b1_131071", "op": "attention", "batch": 1, "longest": 131071, "shortest": 131071, "q_heads": 32, "kv_heads": 8, "dim": 128, "bits": 16,
         "page": 16, "window": 0},
        # every query head with keys of its own, small heads, a sliding window
        {"name": "attn_window_b8", "op": "attention", "batch": 8, "longest": 6000, "shortest": 100, "q_heads": 16, "kv_heads": 16, "dim": 64, "bits": 16,
         "page": 64, "window": 1024},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choices(("norm", "rope", "append", "attention"), (20, 15, 20, 45))[0]
    if op == "norm":
        bits = rng.choice((16, 16, 8))
        return {"op": op, "tokens": _log(rng, 1, 4096), "width": 128 * _log(rng, 1, 40), "residual": rng.random() < 0.7, "bits": bits,
                "group": rng.choice((0, 128)) if bits == 8 else 0}
    dim = rng.choice((64, 128, 128, 128, 256))
    rot = rng.choice((dim, dim, dim // 2, dim // 4))
    layout = rng.choice(("halves", "halves", "interleaved"))
    if op == "rope":
        return {"op": op, "tokens": _log(rng, 1, 4095), "heads": _log(rng, 1, 40 * 128 // dim), "dim": dim, "rot": rot, "layout": layout,
                "scaling": rng.choice(("none", "linear", "parts")), "longest": _log(rng, 4096, 32768)}
    kv_heads, group = rng.choice((1, 2, 4, 8, 8, 16)), rng.choice((1, 2, 4, 4, 5, 7, 8))
    bits, page = rng.choice((16, 16, 8)), rng.choice((16, 16, 32, 64, 128))
    if op == "append":
        kv_heads, group, dim, rot, prompt = min(kv_heads, 8), min(group, 5), min(dim, 128), min(rot, 128), rng.random() < 0.5
        return {"op": op, "tokens": _log(rng, 1, 2048 if prompt else 256), "q_heads": kv_heads * group, "kv_heads": kv_heads, "dim": dim, "rot": rot,
                "layout": layout, "bits": bits, "page": page, "prompt": prompt}
    longest = _log(rng, 1, 65536)
    batch = _log(rng, 1, max(1, min(256, 64 * 4096 * 8 * 128 // (longest * kv_heads * dim * (bits // 8)))))
    return {"op": op, "batch": batch, "longest": longest, "shortest": rng.randint(0, longest), "q_heads": kv_heads * group, "kv_heads": kv_heads, "dim": dim,
            "bits": bits, "page": page, "window": rng.choice((0, 0, 0, _log(rng, 1, 4096)))}


def _lengths(c):
    """The sequences' lengths, few of them long: the shortest, the longest, and what lies between."""
    n, lo, hi = c["batch"], c["shortest"], c["longest"]
    return [hi if n == 1 else int(round(lo + (hi - lo) * (i / (n - 1)) ** 1.5)) for i in range(n)]


def _pages(c):
    return -(-c["longest"] // c["page"])


def work(c):
    if c["op"] == "norm":
        n = c["tokens"] * c["width"]
        out = 2 * n if c["bits"] == 16 else n + 4 * (n // c["group"] if c["group"] else c["tokens"])
        return {"bytes": n * (6 if c["residual"] else 2) + out + 2 * c["width"], "flops": 6 * n}
    if c["op"] == "rope":
        n = c["tokens"] * c["heads"] * c["dim"]
        return {"bytes": 4 * n + 4 * c["tokens"] + 2 * c["rot"], "flops": 3 * c["tokens"] * c["heads"] * c["rot"]}
    if c["op"] == "append":
        q, kv = (c["tokens"] * c[h] * c["dim"] for h in ("q_heads", "kv_heads"))
        held = 2 * kv if c["bits"] == 16 else kv + kv // c["dim"]
        return {"bytes": 4 * q + 4 * kv + 2 * held + 12 * c["tokens"] + 2 * c["rot"],
                "flops": 3 * c["tokens"] * (c["q_heads"] + c["kv_heads"]) * c["rot"]}
    seen = sum(min(n, c["window"]) if c["window"] else n for n in _lengths(c))
    row = 2 * c["dim"] if c["bits"] == 16 else c["dim"] + 1
    q = c["batch"] * c["q_heads"] * c["dim"]
    return {"bytes": 2 * seen * c["kv_heads"] * row + 4 * q + 4 * c["batch"] * c["q_heads"] + 4 * c["batch"] + 4 * (seen // c["page"] + c["batch"]),
            "flops": max(1, 4 * seen * c["q_heads"] * c["dim"])}


def _frequencies(rot, scaling):
    """Radians per position of each pair, for a model made for 8192 positions and used for four times as many."""
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    if scaling == "linear":
        f = f / 4
    elif scaling == "parts":                         # short waves as they are, long ones stretched, between them in proportion
        part = ((8192 * f / (2 * math.pi) - 1) / (4 - 1)).clamp(0, 1)
        f = part * f + (1 - part) * f / 4
    return f.float()


def _normal(g, *shape, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).half()


def _e4m3_exponent(most):
    """The least e in -15..8 with most <= 448 * 2^e (448: the largest E4M3 value)."""
    m, x = torch.frexp(most)
    return torch.where(most > 0, x - 9 + (m > 0.875).int(), torch.full_like(x, -15)).clamp(-15, 8)


def _e4m3_rows(v):
    """Rows of v as (E4M3 codes, exponents): one power of two per row."""
    e = _e4m3_exponent(v.abs().amax(-1))
    most = torch.where(e == 8, 240.0, 448.0).to(v.dtype).unsqueeze(-1)       # 448 * 2^8 would lie beyond fp16
    return torch.clamp(torch.ldexp(v, -e.unsqueeze(-1)), -most, most), e


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}
    if c["op"] == "norm":
        t, w = c["tokens"], c["width"]
        s["x"] = _normal(g, t, w, scale=0.5)
        s["r"] = None
        if c["residual"]:
            s["r"] = _normal(g, t, w)                # the residual stream has channels that are far larger than the others
            s["r"][:, torch.randint(0, w, (max(1, w // 512),), generator=g, device="cuda")] *= 30
        s["w"] = (1 + 0.2 * torch.randn(w, generator=g, device="cuda")).half()
        return s
    if c["op"] == "rope":
        s["x"] = _normal(g, c["tokens"], c["heads"] * c["dim"])
        first = int(torch.randint(0, c["longest"], (1,), generator=g, device="cuda"))
        s["positions"] = ((first + torch.arange(c["tokens"], device="cuda")) % c["longest"]).int()
        s["inv_freq"] = _frequencies(c["rot"], c["scaling"]).cuda()
        s["magnitude"] = 1.0 if c["scaling"] == "none" else 0.1 * math.log(4) + 1
        if own:
            import paper_2511_10645_amd as paro
            s["rope"] = paro.Rope(s["inv_freq"], c["dim"], c["layout"], s["magnitude"])
        return s
    dim, page, kv = c["dim"], c["page"], c["kv_heads"]
    if c["op"] == "append":
        t, q = c["tokens"], c["q_heads"]
        per = -(-t // page)
        n_pages = 2 * per + 3 if c["prompt"] else t + 3
        s["qkv"] = _normal(g, t, (q + 2 * kv) * dim)  # one linear's output: queries, keys, values side by side
        order = torch.randperm(n_pages, generator=g, device="cuda")
        if c["prompt"]:                              # consecutive positions of one sequence, page after page
            i = torch.arange(t, device="cuda")
            s["slots"], s["positions"] = order[i // page] * page + i % page, i.int()
        else:                                        # the next position of each of t sequences
            s["positions"] = torch.randint(0, 8192, (t,), generator=g, device="cuda").int()
            s["slots"] = order[:t] * page + s["positions"] % page
        s["inv_freq"] = _frequencies(c["rot"], "none").cuda()
    else:
        b, q = c["batch"], c["q_heads"]
        per = max(1, _pages(c))
        n_pages = sum(-(-n // page) for n in _lengths(c)) + 2
        lengths = torch.tensor(_lengths(c))[torch.randperm(b, generator=torch.Generator().manual_seed(seed))]
        held = (lengths + page - 1) // page
        first = torch.cumsum(held, 0) - held
        order = torch.randperm(n_pages, generator=g, device="cuda").int()
        at = first.cuda()[:, None] + torch.arange(per, device="cuda")
        s["table"] = torch.where(torch.arange(per, device="cuda") < held.cuda()[:, None], order[at.clamp(max=n_pages - 1)], 0).int().contiguous()
        s["lengths"] = lengths.int().cuda()
        s["q"] = _normal(g, b, q * dim, scale=1.5)
    k, v = (torch.randn((n_pages, kv, page, dim), generator=g, device="cuda") for _ in range(2))
    if c["op"] == "attention":                       # the first token of a sequence draws much of the weight, as in trained models
        live = lengths.nonzero().flatten().cuda()
        k[s["table"][live, 0].long(), :, 0] += 0.25 * s["q"].float().view(b, kv, -1, dim).mean(2)[live]
    unit = 8 if c["bits"] == 16 else 16
    if c["bits"] == 16:
        s["k"], s["v"], s["ks"], s["vs"] = k.half(), v.half(), None, None
    else:
        (k, ke), (v, ve) = _e4m3_rows(k), _e4m3_rows(v)
        s["k"], s["v"] = (x.to(torch.float8_e4m3fn).view(torch.uint8) for x in (k, v))
        s["ks"], s["vs"] = ((e + 127).to(torch.uint8) for e in (ke, ve))
    s["k"] = s["k"].view(n_pages, kv, page, dim // unit, unit).transpose(2, 3).contiguous()
    del k, v
    if own:
        import paper_2511_10645_amd as paro
        s["cache"] = paro.KVCache.from_device(s["k"], s["v"], s["ks"], s["vs"])
        if c["op"] == "append":
            s["rope"] = paro.Rope(s["inv_freq"], dim, c["layout"])
        else:
            s["ws"] = paro.Workspace(paro.paro_workspace_bytes_attention(s["cache"], c["q_heads"], c["batch"]))
    return s


def _rotated(x, positions, inv_freq, layout, magnitude):
    """x [tokens][heads][dim] in fp32 with the first 2 * len(inv_freq) channels of every head rotated."""
    n = inv_freq.numel()
    a = positions.to(x.dtype)[:, None] * inv_freq.to(x.dtype)
    cos, sin = (f(a)[:, None] * magnitude for f in (torch.cos, torch.sin))
    if layout == "halves":
        p, q = x[..., :n], x[..., n:2 * n]
        return torch.cat((p * cos - q * sin, p * sin + q * cos, x[..., 2 * n:]), -1)
    p, q = x[..., 0:2 * n:2], x[..., 1:2 * n:2]
    return torch.cat((torch.stack((p * cos - q * sin, p * sin + q * cos), -1).flatten(-2), x[..., 2 * n:]), -1)


def _normed(s, kind):
    h = s["x"].to(kind) if s["r"] is None else s["x"].to(kind) + s["r"].to(kind)
    return h, h * torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS) * s["w"].to(kind)


def _norm_outputs(s, y, h, h_type, y_type):
    """Outputs of the norm from unrounded values; the E4M3 ones as (codes, scales)."""
    c = s["case"]
    if c["bits"] == 16:
        out = {"y": y.to(y_type)}
    else:
        blocks = y.view(y.shape[0], -1, c["group"] or y.shape[1])
        most = blocks.abs().amax(-1).clamp(min=1e-30)
        codes = (blocks * (448.0 / most)[..., None]).clamp(-448, 448)
        out = {"codes": codes.view(y.shape).to(torch.float8_e4m3fn if y_type == torch.float16 else y_type), "scales": most / 448.0}
    if c["residual"]:
        out["h"] = h.to(h_type)
    return out


def _cache_outputs(s):
    if s["ks"] is None:
        return {"k": s["k"], "v": s["v"]}
    out = {n: s[n].view(torch.float8_e4m3fn) for n in ("k", "v")}
    return out | {n: s[n].view(torch.float8_e8m0fnu) for n in ("ks", "vs")}


def _heads(s):
    c = s["case"]
    t, q, kv, d = c["tokens"], c["q_heads"], c["kv_heads"], c["dim"]
    return (x.reshape(t, -1, d) for x in s["qkv"].split((q * d, kv * d, kv * d), 1))


def _written(s, k, v):
    """Plain form of the append: rows k, v [tokens][heads][dim] (fp32) into the cache."""
    c = s["case"]
    at, off = s["slots"] // c["page"], s["slots"] % c["page"]
    if c["bits"] == 16:
        k, v, unit = k.half(), v.half(), 8
    else:
        (k, ke), (v, ve) = _e4m3_rows(k), _e4m3_rows(v)
        s["ks"][at, :, off], s["vs"][at, :, off] = (ke + 127).to(torch.uint8), (ve + 127).to(torch.uint8)
        k, v, unit = k.to(torch.float8_e4m3fn).view(torch.uint8), v.to(torch.float8_e4m3fn).view(torch.uint8), 16
    s["k"][at, :, :, off], s["v"][at, :, off] = k.unflatten(-1, (-1, unit)), v


def _gathered(s, kind):
    """Keys and values [batch][heads][tokens][dim] of all pages of the table, as values of type `kind`."""
    c = s["case"]
    at = s["table"].long()
    k, v = s["k"][at].movedim(4, 3).flatten(4, 5), s["v"][at]      # [batch][page of the table][head][token][channel]
    if c["bits"] == 8:
        k, v = k.contiguous().view(torch.float8_e4m3fn).to(kind), v.contiguous().view(torch.float8_e4m3fn).to(kind)
        k = k * torch.exp2(s["ks"][at].to(kind) - 127)[..., None]
        v = v * torch.exp2(s["vs"][at].to(kind) - 127)[..., None]
    return (x.to(kind).transpose(1, 2).flatten(2, 3).contiguous() for x in (k, v))


def run(s):
    c = s["case"]
    if own:
        import paper_2511_10645_amd as paro
        if c["op"] == "norm":
            if c["bits"] == 16:
                got = paro.paro_rms_norm(s["x"], s["w"], EPS, residual=s["r"])
                return {"y": got[0], "h": got[1]} if c["residual"] else {"y": got}
            got = paro.paro_rms_norm_quantize_e4m3(s["x"], s["w"], EPS, group=c["group"], residual=s["r"])
            out = {"codes": got[0].view(torch.float8_e4m3fn), "scales": got[1]}
            return out | {"h": got[2]} if c["residual"] else out
        if c["op"] == "rope":
            return paro.paro_rope(s["rope"], s["x"], s["positions"])
        if c["op"] == "append":
            q, k, v = s["qkv"].split((c["q_heads"] * c["dim"], c["kv_heads"] * c["dim"], c["kv_heads"] * c["dim"]), 1)
            return {"q": paro.paro_kv_append(s["cache"], k, v, s["slots"], s["rope"], s["positions"], q)} | _cache_outputs(s)
        o, lse = paro.paro_paged_attention(s["cache"], s["q"], s["table"], s["lengths"], s["ws"], _scale(c), c["window"], with_lse=True)
        return {"o": o, "lse": lse}
    if c["op"] == "norm":
        h, y = _normed(s, torch.float32)
        return _norm_outputs(s, y, h, torch.float16, torch.float16)
    if c["op"] == "rope":
        x = s["x"].float().view(c["tokens"], c["heads"], c["dim"])
        return _rotated(x, s["positions"], s["inv_freq"], c["layout"], s["magnitude"]).half().view(c["tokens"], -1)
    if c["op"] == "append":
        q, k, v = (x.float() for x in _heads(s))
        q, k = (_rotated(x, s["positions"], s["inv_freq"], c["layout"], 1.0) for x in (q, k))
        _written(s, k, v)
        return {"q": q.half().flatten(1)} | _cache_outputs(s)
    b, kv, d = c["batch"], c["kv_heads"], c["dim"]
    k, v = _gathered(s, torch.float32)
    q = s["q"].float().view(b, kv, -1, d)
    scores = torch.matmul(q, k.transpose(2, 3).contiguous()) * _scale(c)
    at, n = torch.arange(k.shape[2], device="cuda"), s["lengths"][:, None]
    seen = (at < n) & (at >= n - c["window"]) if c["window"] else at < n
    scores = torch.where(seen[:, None, None], scores, -math.inf)
    most = scores.amax(-1, keepdim=True).clamp(min=-1e30)
    p = torch.exp(scores - most)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total > 0, total, 1.0)
    return {"o": o.half().view(b, -1), "lse": torch.where(total > 0, most + torch.log(total), -math.inf).view(b, -1)}


def _scale(c):
    return 1 / math.sqrt(c["dim"])


def exact(c, seed):
    """What run() returns, from the definitions in 64 bits: rows, heads and sequences one after the other."""
    s = prepare(c, seed)
    f64 = torch.float64
    if c["op"] == "norm":
        h = s["x"].double()
        if c["residual"]:
            h = h + s["r"].double()
        y = h / torch.sqrt((h * h).sum(1, keepdim=True) / c["width"] + EPS) * s["w"].double()
        return _norm_outputs(s, y, h, f64, f64)

    def rotated(x, magnitude):                       # [tokens][heads][dim] as complex numbers times e^(i * angle)
        n = c["rot"] // 2
        turn = torch.polar(torch.full((1,), magnitude, dtype=f64, device="cuda"), s["positions"].double()[:, None] * s["inv_freq"].double())[:, None]
        y = x.double().clone()
        first, second = (slice(0, n), slice(n, 2 * n)) if c["layout"] == "halves" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
        z = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * turn
        y[..., first], y[..., second] = z.real, z.imag
        return y

    if c["op"] == "rope":
        return rotated(s["x"].view(c["tokens"], c["heads"], c["dim"]), s["magnitude"]).view(c["tokens"], -1)
    if c["op"] == "append":
        q, k, v = _heads(s)
        q, k, v = rotated(q, 1.0), rotated(k, 1.0), v.double()
        held = _cache_outputs(s)
        out = {n: x.double() for n, x in held.items()}
        unit = 8 if c["bits"] == 16 else 16
        page, off = s["slots"] // c["page"], s["slots"] % c["page"]
        if c["bits"] == 8:
            unit2 = {n: torch.exp2(torch.ceil(torch.log2(x.abs().amax(-1) / 448)).clamp(-15, 8)) for n, x in (("k", k), ("v", v))}
            out["ks"][page, :, off], out["vs"][page, :, off] = unit2["k"], unit2["v"]
            k, v = k / unit2["k"][..., None], v / unit2["v"][..., None]
        for j in range(c["dim"] // unit):
            out["k"][page, :, j, off] = k[..., j * unit:(j + 1) * unit]
        out["v"][page, :, off] = v
        return {"q": q.flatten(1)} | out
    b, heads, kv, d = c["batch"], c["q_heads"], c["kv_heads"], c["dim"]
    o, lse = torch.zeros((b, heads, d), dtype=f64, device="cuda"), torch.full((b, heads), -math.inf, dtype=f64, device="cuda")
    for i, n in enumerate(s["lengths"].tolist()):
        if not n:
            continue
        lo = max(0, n - c["window"]) if c["window"] else 0
        pages = s["table"][i, :-(-n // c["page"])].long()
        k = s["k"][pages].permute(1, 0, 3, 2, 4).reshape(kv, -1, d)[:, lo:n].contiguous()
        v = s["v"][pages].permute(1, 0, 2, 3).reshape(kv, -1, d)[:, lo:n].contiguous()
        if c["bits"] == 8:
            ks, vs = (torch.exp2(s[x][pages].permute(1, 0, 2).reshape(kv, -1)[:, lo:n].double() - 127)[..., None] for x in ("ks", "vs"))
            k, v = k.view(torch.float8_e4m3fn).double() * ks, v.view(torch.float8_e4m3fn).double() * vs
        k, v = k.double(), v.double()
        for h in range(kv):
            q = s["q"][i].view(kv, -1, d)[h].double()
            x = q @ k[h].t().contiguous() / math.sqrt(d)
            rows = slice(h * heads // kv, (h + 1) * heads // kv)
            o[i, rows] = torch.softmax(x, -1) @ v[h]
            lse[i, rows] = torch.logsumexp(x, -1)
    return {"o": o.view(b, -1), "lse": lse}
