"""Serving more than one new token of a sequence at a time, from a smaller cache, with other scores: cases that can be timed and compared.

Two operators over the paged key-value cache that the linears of a decoder layer fill, each in the cache's three formats (fp16, E4M3
with a power-of-two scale per token and head, MXFP4: E2M1 with a power-of-two scale per token, head and 32 channels):

  step    one new token of every sequence: ``paro_paged_attention`` with capped scores, a distance bias, or from an MXFP4 cache, which
          ``paro_kv_append`` has just written the token into (rotated)
  prompt  the new tokens of every sequence, one to thousands: ``paro_prompt_attention``, after ``paro_kv_append`` where the case says so

  x = cap tanh(scale q . k / cap) - slope |p - t|,   o = sum_t softmax(x)_t v_t,   lse = ln sum_t exp(x_t)

over the tokens t that a row at position p attends to: first <= t, p - window < t, and t <= p or t < prefix.  Outputs are o and lse
(and the rotated queries where tokens are appended); what the append writes is what the attention then reads.

Head counts and widths are those of the layers of ``paro_inputs.CONFIGS``: 4096 -> 6144 is 32 query and 8 key-value heads of 128
channels, 5120 -> 7168 is 40 and 8; others are generic.  ``own`` false computes the formulas in elementary fp32 operations.
"""
from __future__ import annotations

import math

import torch

own = False

FORMATS = {16: "fp16", 8: "e4m3", 4: "mxfp4"}


def _step(name, batch, shortest, longest, q_heads, kv_heads, dim, bits, page, append, window=0, cap=0.0, bias=False):
    return {"name": name, "op": "step", "batch": batch, "shortest": shortest, "longest": longest, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim,
            "bits": bits, "page": page, "append": append, "window": window, "cap": cap, "bias": bias}


def _prompt(name, batch, new_short, new_long, held_short, held_long, q_heads, kv_heads, dim, bits, page, append, window=0, cap=0.0, bias=False, prefix=0,
            documents=0):
    return {"name": name, "op": "prompt", "batch": batch, "new_short": new_short, "new_long": new_long, "held_short": held_short, "held_long": held_long,
            "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim, "bits": bits, "page": page, "append": append, "window": window, "cap": cap, "bias": bias,
            "prefix": prefix, "documents": documents}


def listed():
    return [
        # one short conversation on a 4-bit cache: the latency of two calls
        _step("step_mxfp4_b1_700", 1, 700, 700, 32, 8, 128, 4, 16, True),
        # a loaded server on a 4-bit cache, wider layer, conversations of very different lengths
        _step("step_mxfp4_b64_8192", 64, 1000, 8192, 40, 8, 128, 4, 32, True),
        # one very long document in 4 bits: the cache's length is all there is to split
        _step("step_mxfp4_b1_131071", 1, 131071, 131071, 32, 8, 128, 4, 16, True),
        # scores capped by a tanh, wide heads, a sliding window over an fp16 cache
        _step("step_cap_b16_4096", 16, 1, 4096, 16, 4, 256, 16, 16, False, 2048, 50.0),
        # a bias by distance in place of rotary positions, over an 8-bit cache
        _step("step_bias_b32_4000", 32, 0, 4000, 32, 8, 128, 8, 64, False, 0, 0.0, True),
        # drafts of a few tokens checked at once: as many rows as a batched step has, several to a sequence
        _prompt("draft_b4_t5", 4, 5, 5, 900, 3001, 32, 8, 128, 16, 16, False),
        # a whole prompt of one sequence
        _prompt("prompt_t2048", 1, 2048, 2048, 0, 0, 32, 8, 128, 16, 16, False),
        # prompts of odd and very different lengths behind what is cached already, 8-bit cache, wider layer
        _prompt("prompt_e4m3_b7", 7, 1, 1501, 0, 1777, 40, 8, 128, 8, 32, True),
        # a piece of a long document: few rows, much of the cache
        _prompt("piece_t512_32768", 1, 512, 512, 32256, 32256, 32, 8, 128, 16, 16, False),
        # a long prompt into a 4-bit cache
        _prompt("prompt_mxfp4_t4095", 1, 4095, 4095, 0, 0, 32, 8, 128, 4, 16, True),
        # a prefix that is seen from both sides, capped scores, window, wide heads
        _prompt("prompt_prefix_cap", 3, 300, 1024, 0, 500, 16, 4, 256, 16, 64, False, 900, 50.0, False, 200),
        # documents packed into one sequence, bias by distance, every query head with keys of its own, small heads
        _prompt("prompt_documents", 2, 1999, 2500, 0, 0, 16, 16, 64, 16, 128, False, 0, 0.0, True, 0, 5),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    dim = rng.choice((64, 128, 128, 128, 256))
    kv_heads, group = rng.choice((1, 2, 4, 8, 8, 16)), rng.choice((1, 2, 4, 4, 5, 7, 8, 16))
    q_heads = kv_heads * group
    page, bits = rng.choice((16, 16, 32, 64, 128)), rng.choice((16, 8, 4, 4))
    window = rng.choice((0, 0, 0, _log(rng, 1, 4096)))
    cap, bias = rng.choice(((0.0, False), (0.0, False), (30.0, False), (50.0, False), (0.0, True), (40.0, True)))
    if rng.random() < 0.45:
        append = bits == 4 or rng.random() < 0.3
        if bits != 4 and not cap and not bias:       # that call is not one of these operators: it gets a cap
            cap = 50.0
        longest = _log(rng, 1, 65536)
        batch = _log(rng, 1, max(1, min(256, 64 * 4096 * 8 * 128 // (longest * kv_heads * dim))))
        return _without_name(_step("", batch, rng.randint(0, longest), longest, q_heads, kv_heads, dim, bits, page, append, window, cap, bias))
    new = _log(rng, 1, 4095)
    held = rng.choice((0, _log(rng, 1, 32768)))
    heads_most = max(1, 2 ** 29 // (new * (new + held)))                # of one sequence, so that a pass costs no more than a listed one's
    while q_heads * dim > 128 * heads_most and q_heads > 1:
        group, kv_heads = (group, kv_heads // 2) if kv_heads > 1 else (max(1, group // 2), 1)
        q_heads = kv_heads * group
    batch = _log(rng, 1, max(1, min(64, 128 * heads_most // (q_heads * dim))))
    return _without_name(_prompt("", batch, rng.randint(1, new), new, rng.randint(0, held), held, q_heads, kv_heads, dim, bits, page, rng.random() < 0.5, window,
                                 cap, bias, rng.choice((0, 0, _log(rng, 1, 1000))), rng.choice((0, 0, rng.randint(2, 9)))))


def _without_name(c):
    return {k: v for k, v in c.items() if k != "name"}


def _between(lo, hi, n, back=False):
    """n whole numbers from lo to hi, few of them large."""
    x = [hi if n == 1 else int(round(lo + (hi - lo) * (i / (n - 1)) ** 1.5)) for i in range(n)]
    return x[::-1] if back else x


def _sizes(c):
    """(new tokens, all tokens) of every sequence."""
    n = c["batch"]
    if c["op"] == "step":
        whole = _between(c["shortest"], c["longest"], n)
        return [min(1, x) for x in whole], whole
    new, held = _between(c["new_short"], c["new_long"], n), _between(c["held_short"], c["held_long"], n, True)
    return new, [a + b for a, b in zip(new, held)]


def _document(c, length):
    """Tokens of a document of a sequence of that length."""
    return -(-length // c["documents"])


def _range(c, p, length):
    """What a row at position p attends to: lo <= t < hi."""
    lo = max(0, p - c["window"] + 1) if c["window"] else 0
    hi = p + 1
    if c["op"] == "prompt":
        if c["documents"]:
            lo = max(lo, p // _document(c, length) * _document(c, length))
        hi = max(hi, min(c["prefix"], length))
    return lo, hi


def work(c):
    pairs = seen = 0
    new, whole = _sizes(c)
    for m, n in zip(new, whole):
        ranges = [_range(c, p, n) for p in range(n - m, n)]
        pairs += sum(max(0, hi - lo) for lo, hi in ranges)
        seen += max((hi for _, hi in ranges), default=0) - min((lo for lo, _ in ranges), default=0)
    rows, d, kv, q = sum(new) if c["op"] == "prompt" else c["batch"], c["dim"], c["kv_heads"], c["q_heads"]
    held = {16: 2 * d, 8: d + 1, 4: d // 2 + d // 32}[c["bits"]]           # of a token's keys in one head
    moved = 2 * seen * kv * held + rows * q * (4 * d + 4) + sum(-(-n // c["page"]) for n in whole) * 4 + 8 * c["batch"]
    if c["append"]:                                  # new keys and values in and out, queries in and out once more
        moved += 2 * sum(new) * kv * (2 * d + held) + 4 * rows * q * d + 12 * rows
    if c["op"] == "prompt" and c["documents"]:
        moved += 4 * rows
    return {"bytes": moved, "flops": max(1, 4 * pairs * q * d)}


# ---- Formats of the cache ---------------------------------------------------------------------------------------------------

E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _e4m3_rows(v):
    """Rows of v as (E4M3 bytes, scale bytes): the least power of two, 2^-15 to 2^8, with which all lie within 448 (240 with 2^8)."""
    most = v.abs().amax(-1)
    m, x = torch.frexp(most)
    e = torch.where(most > 0, x - 9 + (m > 0.875).int(), torch.full_like(x, -15)).clamp(-15, 8)
    within = torch.where(e == 8, 240.0, 448.0).to(v.dtype).unsqueeze(-1)
    codes = torch.clamp(torch.ldexp(v, -e.unsqueeze(-1)), -within, within).float().to(torch.float8_e4m3fn).view(torch.uint8)
    return codes, (e + 127).to(torch.uint8)


def _mxfp4_rows(v):
    """Rows of v as (pairs of E2M1 codes, scale bytes): 2^(floor(log2 max) - 2), 2^-23 to 2^13, for every 32 channels."""
    v = v.unflatten(-1, (-1, 32))
    most = v.abs().amax(-1)
    _, x = torch.frexp(most)
    e = torch.where(most > 0, x - 3, torch.full_like(x, -23)).clamp(-23, 13)
    a = torch.ldexp(v.abs(), -e.unsqueeze(-1)).clamp(max=6.0)
    code = torch.where(a < 2, torch.round(2 * a), torch.where(a < 4, 2 + torch.round(a), 4 + torch.round(a / 2)))      # halves to even
    code = (code.to(torch.uint8) + 8 * (v < 0).to(torch.uint8)).flatten(-2)
    return code[..., ::2] + 16 * code[..., 1::2], (e + 127).to(torch.uint8)


def _e2m1_pairs(kind):
    """The two values of every byte."""
    v = torch.tensor(E2M1 + tuple(-x for x in E2M1), dtype=kind, device="cuda")
    b = torch.arange(256, device="cuda")
    return torch.stack((v[b & 15], v[b >> 4]), -1)


def _stored(v, bits):
    """Rows [...][dim] as they are held: (bytes or fp16, scale bytes or None)."""
    return (v.half(), None) if bits == 16 else _e4m3_rows(v) if bits == 8 else _mxfp4_rows(v)


def _values(x, scale, bits, kind):
    """Rows [...][dim] as values, from what is held."""
    if bits == 16:
        return x.to(kind)
    if bits == 8:
        return x.contiguous().view(torch.float8_e4m3fn).to(kind) * torch.exp2(scale.to(kind) - 127).unsqueeze(-1)
    return _e2m1_pairs(kind)[x.int()].flatten(-2).unflatten(-1, (-1, 32)).mul_(torch.exp2(scale.to(kind) - 127).unsqueeze(-1)).flatten(-2)


def _unit(c):
    """Elements of k in 16 bytes."""
    return 8 if c["bits"] == 16 else 16


# ---- Inputs -----------------------------------------------------------------------------------------------------------------

def _slopes(heads):
    return torch.exp2(-8.0 * torch.arange(1, heads + 1, dtype=torch.float64) / heads).float()


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dim, page, kv, heads, bits, batch = (c[x] for x in ("dim", "page", "kv_heads", "q_heads", "bits", "batch"))
    new, whole = _sizes(c)
    order = torch.randperm(batch, generator=torch.Generator().manual_seed(seed))
    new, whole = torch.tensor(new)[order], torch.tensor(whole)[order]
    held = (whole + page - 1) // page
    per, n_pages = max(1, int(held.max())), int(held.sum()) + 2
    first_page = torch.cumsum(held, 0) - held
    pages = torch.randperm(n_pages, generator=g, device="cuda").int()
    at = first_page.cuda()[:, None] + torch.arange(per, device="cuda")
    s = {"case": c, "table": torch.where(torch.arange(per, device="cuda") < held.cuda()[:, None], pages[at.clamp(max=n_pages - 1)], 0).int().contiguous(),
         "lengths": whole.int().cuda(), "new": new}
    # the rows: every sequence's new tokens one after the other; a step has a row for every sequence, also for one without tokens
    count = torch.ones_like(new) if c["op"] == "step" else new
    starts = torch.cat((torch.zeros(1, dtype=torch.long), torch.cumsum(count, 0)))
    rows = int(starts[-1])
    sequence = torch.repeat_interleave(torch.arange(batch), count).cuda()
    p = (whole - count)[sequence.cpu()].cuda() + torch.arange(rows, device="cuda") - starts[sequence.cpu()].cuda()
    s |= {"starts": starts.int().cuda(), "sequence": sequence, "positions": p.clamp(min=0).int()}
    slots = s["table"].long()[sequence, p.clamp(min=0) // page] * page + p % page
    s["slots"] = torch.where(p >= 0, slots, -1)
    s["qkv"] = torch.randn((rows, (heads + 2 * kv) * dim), generator=g, device="cuda")
    s["qkv"][:, :heads * dim] *= 6.0 if c["cap"] else 1.5       # a cap is for scores that come near it
    s["qkv"] = s["qkv"].half()
    s["slopes"] = _slopes(heads).cuda() if c["bias"] else None
    s["prefix"] = s["first"] = None
    if c["op"] == "prompt":
        if c["prefix"]:
            s["prefix"] = torch.clamp(whole, max=c["prefix"]).int().cuda()
        if c["documents"]:
            size = torch.clamp(-(-whole // c["documents"]), min=1).cuda()[sequence]
            s["first"] = (p // size * size).int()
    s["inv_freq"] = (10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim)).float().cuda()
    k, v = (torch.randn((n_pages, kv, page, dim), generator=g, device="cuda") for _ in range(2))
    live = whole.nonzero().flatten().cuda()          # the first token of a sequence draws much of the weight, as in trained models
    towards = torch.zeros((batch, kv, dim), device="cuda").index_add_(0, sequence, s["qkv"][:, :heads * dim].float().view(rows, kv, -1, dim).mean(2))
    k[s["table"][live, 0].long(), :, 0] += 0.25 * (towards / count.clamp(min=1).cuda()[:, None, None])[live]
    (s["k"], s["ks"]), (s["v"], s["vs"]) = _stored(k, bits), _stored(v, bits)
    del k, v
    s["k"] = s["k"].unflatten(-1, (-1, _unit(c))).transpose(2, 3).contiguous()
    if bits == 4:
        s["ks"], s["vs"] = (x.transpose(2, 3).contiguous() for x in (s["ks"], s["vs"]))
    if own:
        import paper_2511_10645_amd as paro
        s["cache"] = paro.KVCache.from_device(s["k"], s["v"], s["ks"], s["vs"])
        s["rope"] = paro.Rope(s["inv_freq"], dim)
        if c["op"] == "step":
            s["ws"] = paro.Workspace(paro.paro_workspace_bytes_attention(s["cache"], heads, batch))
        else:
            s["ws"] = paro.Workspace(paro.paro_workspace_bytes_prompt(s["cache"], heads, rows, batch))
    return s


# ---- One pass ---------------------------------------------------------------------------------------------------------------

def _scale(c):
    return 1 / math.sqrt(c["dim"])


def _rotated(x, positions, inv_freq):
    """x [rows][heads][dim]: channels i and i + dim/2 rotated by position * inv_freq[i], the angle in 64 bits."""
    n = inv_freq.numel()
    a = positions.double()[:, None] * inv_freq.double()
    cos, sin = (f(a).to(x.dtype)[:, None] for f in (torch.cos, torch.sin))
    p, q = x[..., :n], x[..., n:]
    return torch.cat((p * cos - q * sin, p * sin + q * cos), -1)


def _written(s, k, v):
    """Rows k, v [rows][heads][dim] into their slots."""
    c = s["case"]
    live = s["slots"] >= 0
    slots, bits = s["slots"][live], c["bits"]
    at, off = slots // c["page"], slots % c["page"]
    (k, ks), (v, vs) = _stored(k[live], bits), _stored(v[live], bits)
    s["k"][at, :, :, off], s["v"][at, :, off] = k.unflatten(-1, (-1, _unit(c))), v
    if bits == 8:
        s["ks"][at, :, off], s["vs"][at, :, off] = ks, vs
    elif bits == 4:
        s["ks"][at, :, :, off], s["vs"][at, :, :, off] = ks, vs


def _gathered(s, kind):
    """Keys and values [batch][heads][tokens][dim] of all pages of the table."""
    bits, at = s["case"]["bits"], s["table"].long()
    k, v, ks, vs = s["k"][at].movedim(4, 3).flatten(4, 5), s["v"][at], None, None  # [batch][page of the table][head][token][channel]
    if bits < 16:
        ks, vs = (x[at] if bits == 8 else x[at].transpose(3, 4) for x in (s["ks"], s["vs"]))
    return (_values(x, e, bits, kind).transpose(1, 2).flatten(2, 3).contiguous() for x, e in ((k, ks), (v, vs)))


def _seen(s):
    """[rows][tokens]: what every row attends to."""
    c, p = s["case"], s["positions"].long()
    length = s["lengths"].long()[s["sequence"]]
    lo = (p - c["window"] + 1).clamp(min=0) if c["window"] else torch.zeros_like(p)
    hi = torch.minimum(p + 1, length)
    if s["first"] is not None:
        lo = torch.maximum(lo, s["first"].long())
    if s["prefix"] is not None:
        hi = torch.maximum(hi, s["prefix"].long()[s["sequence"]])
    t = torch.arange(s["table"].shape[1] * c["page"], device="cuda")
    return (t >= lo[:, None]) & (t < hi[:, None])


def _places(s):
    """Rows side by side: the place of every row in [batch][most rows of a sequence]."""
    most = max(1, int(s["new"].max())) if s["case"]["op"] == "prompt" else 1
    i = torch.arange(s["sequence"].numel(), device="cuda") - s["starts"].long()[s["sequence"]]
    return s["sequence"] * most + i, most


def run(s):
    c = s["case"]
    heads, kv, dim = c["q_heads"], c["kv_heads"], c["dim"]
    q, k, v = s["qkv"].split((heads * dim, kv * dim, kv * dim), 1)
    out = {}
    if own:
        import paper_2511_10645_amd as paro
        if c["append"]:
            q = out["q"] = paro.paro_kv_append(s["cache"], k, v, s["slots"], s["rope"], s["positions"], q)
        if c["op"] == "step":
            out["o"], out["lse"] = paro.paro_paged_attention(s["cache"], q, s["table"], s["lengths"], s["ws"], _scale(c), c["window"], with_lse=True, cap=c["cap"],
                                                             slopes=s["slopes"])
        else:
            out["o"], out["lse"] = paro.paro_prompt_attention(s["cache"], q, s["starts"], s["table"], s["lengths"], s["ws"], _scale(c), c["window"], with_lse=True,
                                                              cap=c["cap"], slopes=s["slopes"], prefix=s["prefix"], first=s["first"])
        return out
    rows = q.shape[0]
    if c["append"]:
        q, k = (_rotated(x.float().view(rows, -1, dim), s["positions"], s["inv_freq"]) for x in (q, k))
        _written(s, k, v.float().reshape(rows, kv, dim))
        q = out["q"] = q.half().flatten(1)
    k, v = _gathered(s, torch.float32)
    at, most = _places(s)
    b, tokens = c["batch"], k.shape[2]
    padded = torch.zeros((b * most, heads * dim), device="cuda")
    padded[at] = q.float()
    # [batch][key-value head][row, query head][token]
    padded = padded.view(b, most, kv, -1, dim).transpose(1, 2).flatten(2, 3).contiguous()
    x = torch.matmul(padded, k.transpose(2, 3).contiguous()).mul_(_scale(c)).view(b, kv, most, -1, tokens)
    if c["cap"]:
        x = torch.tanh(x.div_(c["cap"])).mul_(c["cap"])
    if c["bias"]:
        p = torch.zeros(b * most, dtype=torch.int32, device="cuda")
        p[at] = s["positions"]
        away = (p.view(b, 1, most, 1, 1) - torch.arange(tokens, device="cuda")).abs().float()
        x = x - s["slopes"].view(1, kv, 1, -1, 1) * away
    seen = torch.zeros((b * most, tokens), dtype=torch.bool, device="cuda")
    seen[at] = _seen(s)
    x = x.masked_fill(~seen.view(b, 1, most, 1, tokens), -math.inf)
    top = x.amax(-1, keepdim=True).clamp(min=-1e30)
    x = torch.exp(x - top)
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x.flatten(2, 3), v).view(b, kv, most, -1, dim) / torch.where(total > 0, total, 1.0)
    lse = torch.where(total > 0, top + torch.log(total), -math.inf)
    o, lse = (y.permute(0, 2, 1, 3, 4).reshape(b * most, -1)[at] for y in (o, lse))
    return out | {"o": o.half(), "lse": lse}


def exact(c, seed):
    """What run() returns, from the definitions in 64 bits: one sequence and key-value head after the other."""
    s = prepare(c, seed)
    f64 = torch.float64
    heads, kv, dim, page, bits = (c[x] for x in ("q_heads", "kv_heads", "dim", "page", "bits"))
    q, k_new, v_new = (x.double().unflatten(1, (-1, dim)) for x in s["qkv"].split((heads * dim, kv * dim, kv * dim), 1))
    out = {}
    if c["append"]:
        turn = torch.polar(torch.ones(1, dtype=f64, device="cuda"), s["positions"].double()[:, None] * s["inv_freq"].double())[:, None]

        def rotated(x):
            z = torch.complex(x[..., :dim // 2].contiguous(), x[..., dim // 2:].contiguous()) * turn
            return torch.cat((z.real, z.imag), -1)

        q, k_new = rotated(q), rotated(k_new)
        out["q"] = q.flatten(1)
        q = q.half().double()                        # what the attention is given

        def held(x):                                 # the values that the cache holds of rows x [..., dim]
            if bits == 16:
                return x.half().double()
            if bits == 8:
                e = torch.exp2(torch.ceil(torch.log2(x.abs().amax(-1, keepdim=True) / 448)).clamp(-15, 8))
                return (x / e).float().to(torch.float8_e4m3fn).double() * e
            y = x.unflatten(-1, (-1, 32))
            e = torch.exp2((torch.floor(torch.log2(y.abs().amax(-1, keepdim=True))) - 2).clamp(-23, 13))
            grid = torch.tensor(E2M1, dtype=f64, device="cuda")
            middle = (grid[1:] + grid[:-1]) / 2
            a = y.abs() / e                          # a middle goes to the even code
            below = torch.bucketize(a, middle)       # the number of middles below a
            tie = (below < 7) & (a == middle[below.clamp(max=6)]) & (below % 2 == 1)
            return (grid[below + tie.long()] * e * torch.sign(y)).flatten(-2)

        k_new, v_new = held(k_new), held(v_new)
    o, lse = torch.zeros((len(s["sequence"]), heads, dim), dtype=f64, device="cuda"), torch.full((len(s["sequence"]), heads), -math.inf, dtype=f64, device="cuda")
    starts, group = s["starts"].tolist(), heads // kv
    for i, n in enumerate(s["lengths"].tolist()):
        r0, r1 = starts[i], starts[i + 1]
        if not n or r0 == r1:
            continue
        pages = s["table"][i, :-(-n // page)].long()
        ends = [_range(c, p, n) for p in range(n - (r1 - r0), n)]
        lo, hi = (torch.tensor(x, device="cuda")[:, None] for x in zip(*ends))
        t = torch.arange(n, device="cuda")
        seen = (t >= lo) & (t < hi)                  # [rows][tokens]
        away = (torch.arange(n - (r1 - r0), n, device="cuda")[:, None] - t).abs().double()
        for h in range(kv):
            kv_rows = []
            for name, scale, fresh in (("k", "ks", k_new), ("v", "vs", v_new)):
                y = s[name][pages, h]
                y = y.transpose(1, 2).flatten(2, 3) if name == "k" else y      # [page][token][channels]
                e = None if bits == 16 else s[scale][pages, h] if bits == 8 else s[scale][pages, h].transpose(1, 2)
                y = _values(y, e, bits, f64).flatten(0, 1)[:n].contiguous()
                if c["append"]:
                    y[n - (r1 - r0):] = fresh[r0:r1, h]
                kv_rows.append(y)
            for j in range(group):
                head = h * group + j
                x = q[r0:r1, head].contiguous() @ kv_rows[0].t().contiguous() / math.sqrt(dim)
                if c["cap"]:
                    x = c["cap"] * torch.tanh(x / c["cap"])
                if c["bias"]:
                    x = x - float(s["slopes"][head]) * away
                x = torch.where(seen, x, -math.inf)
                some = seen.any(1)
                lse[r0:r1, head] = torch.logsumexp(x, 1)
                o[r0:r1, head] = torch.where(some[:, None], torch.softmax(x, 1), 0.0) @ kv_rows[1]
    return out | {"o": o.flatten(1), "lse": lse}
