"""The attention side of a decoder layer over the 4-bit KV cache, as cases that can be timed and compared.

Between the W4A4 linears of a layer a serving program norms and rotates the heads of queries and keys, writes keys and
values into pages of a 4-bit cache, reads tokens of it back, and attends: a whole prompt on its 16-bit keys and values,
or new tokens (one, a few drafted ones, a chunk) over the pages.

Kinds:
  rope     RMS norm per head, rotary positions (half or interleaved pairs, all or part of the head) and the Hadamard
           rotation of the heads, in one pass.
  cache    ``write``: queries, keys and values of new tokens as above, keys and values into the cache, and the same
           tokens read back; without it: cached tokens read back (a shared prefix, a cache that moves).
  paged    attention of each sequence's new tokens over its pages.
  prompt   attention of packed sequences of different lengths.

Sizes are the heads, head dimensions and token counts of the repository's workloads (Llama-2-7B: 32 heads, Llama-3-8B:
32 over 8, Llama-2-70B: 64 over 8; 128 channels) and generic ones around them.

``own`` chooses between the library's calls and their plain form, elementary torch operations in 32 bits. The order of
the sums that decide a code (squares, means: neighbours first; butterflies: distance 1 first) is the library's, so that
both find the same codes.
"""

from __future__ import annotations

import math
import random

import torch

own = False

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
EPS = 1e-6


def rope_case(name, T, heads, D, x, norm, rot, interleaved, rotate, max_pos):
    return {"name": name, "kind": "rope", "T": T, "heads": heads, "D": D, "x": x, "norm": norm, "rot": rot,
            "interleaved": interleaved, "rotate": rotate, "max_pos": max_pos}


def cache_case(name, write, T, q_heads, kv_heads, D, page, x, norm, rot, interleaved, max_pos):
    return {"name": name, "kind": "cache", "write": write, "T": T, "q_heads": q_heads, "kv_heads": kv_heads, "D": D,
            "page": page, "x": x, "norm": norm, "rot": rot, "interleaved": interleaved, "max_pos": max_pos}


def paged_case(name, B, q_heads, kv_heads, D, page, x, new, past, lengths):
    """``new`` and ``past``: (least, most) tokens of a sequence; ``lengths``: the seed of the batch's lengths."""
    return {"name": name, "kind": "paged", "B": B, "q_heads": q_heads, "kv_heads": kv_heads, "D": D, "page": page,
            "x": x, "new_lo": new[0], "new_hi": new[1], "past_lo": past[0], "past_hi": past[1], "lengths": lengths}


def prompt_case(name, B, q_heads, kv_heads, D, x, length, causal, lengths):
    return {"name": name, "kind": "prompt", "B": B, "q_heads": q_heads, "kv_heads": kv_heads, "D": D, "x": x,
            "len_lo": length[0], "len_hi": length[1], "causal": causal, "lengths": lengths}


def listed():
    return [
        # The queries and keys of one decoded token (Llama-3-8B heads), normed and rotated: latency alone.
        rope_case("rope_decode", 1, 40, 128, "bf16", True, 128, False, True, 8192),
        # A long prompt's queries and keys, half precision, part of the head rotated in interleaved pairs.
        rope_case("rope_prompt", 8191, 72, 128, "f16", False, 64, True, False, 16384),
        # One decode step of 32 streams: queries, keys and values of their new tokens, the cache written and read back.
        cache_case("cache_decode", True, 32, 32, 8, 128, 64, "bf16", True, 128, False, 8192),
        # A prompt of odd length entering the cache of a Llama-2-7B layer.
        cache_case("cache_prompt", True, 4097, 32, 32, 128, 32, "f16", False, 128, False, 8192),
        # A shared prefix read back from the cache, its keys rotated back.
        cache_case("cache_prefix", False, 16384, 0, 8, 128, 16, "bf16", False, 0, False, 0),
        # A single stream's next token over a short context.
        paged_case("decode_1", 1, 32, 8, 128, 64, "bf16", (1, 1), (776, 776), 0),
        # A serving batch: 64 streams of very different lengths, Llama-2-70B heads, small pages.
        paged_case("decode_ragged", 64, 64, 8, 128, 16, "f16", (1, 1), (1, 8191), 1),
        # Long contexts with a key head for each query head (Llama-2-7B).
        paged_case("decode_long", 4, 32, 32, 128, 128, "bf16", (1, 1), (65536, 65536), 2),
        # Four drafted tokens verified in each of 16 streams.
        paged_case("verify_4", 16, 32, 8, 128, 64, "bf16", (4, 4), (500, 6000), 3),
        # Chunks of two prompts that are being taken in piece by piece.
        paged_case("chunk_1000", 2, 32, 8, 128, 64, "bf16", (900, 1024), (15000, 16000), 4),
        # A batch of short prompts of different lengths, smaller heads, half precision.
        prompt_case("prompt_ragged", 24, 16, 4, 64, "f16", (5, 2000), True, 5),
        # One long prompt.
        prompt_case("prompt_8192", 1, 32, 8, 128, "bf16", (8192, 8192), True, 6),
    ]


def log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(["rope", "write", "read", "decode", "few", "chunk", "prompt"], [3, 3, 2, 5, 2, 3, 4])[0]
    D = rng.choice([64, 128, 128])
    page = rng.choice([16, 32, 64, 128])
    x16 = rng.choice(["bf16", "bf16", "f16"])
    x = rng.choice(["bf16", "f16", "f32"])
    rot = rng.choice([D, D, D // 2, D // 4])
    seed = rng.randrange(1 << 20)
    if kind == "rope":
        c = rope_case("", log_int(rng, 1, 8192), rng.choice([1, 8, 12, 32, 40, 64]), D, x, rng.random() < 0.5, rot,
                      rng.random() < 0.5, rng.random() < 0.5, 16384)
    elif kind in ("write", "read"):
        write = kind == "write"
        kv = rng.choice([1, 2, 8, 32])
        c = cache_case("", write, log_int(rng, 1, 8192), kv * rng.choice([1, 4]) if write else 0, kv, D, page, x,
                       write and rng.random() < 0.5, rot if write else 0, write and rng.random() < 0.5,
                       16384 if write else 0)
    elif kind == "prompt":
        kv = rng.choice([1, 2, 4, 8])
        heads = kv * rng.choice([1, 2, 4, 8])
        top = min(log_int(rng, 1, 6000), int(math.sqrt(1e9 / heads)))
        B = max(1, min(log_int(rng, 1, 64), 24000 // top, int(1e9 / heads / top ** 2)))
        c = prompt_case("", B, heads, kv, D, x16, (max(1, top // rng.choice([1, 4, 50])), top), rng.random() < 0.8, seed)
    else:
        kv = rng.choice([1, 2, 4, 8, 32])
        group = rng.choice([1, 4, 5, 8]) if kv < 32 else 1
        new = {"decode": (1, 1), "few": (1, rng.randint(2, 9)), "chunk": (log_int(rng, 4, 100), log_int(rng, 100, 1500))}[kind]
        top = log_int(rng, 1, 60000 if kind == "decode" else 16000)
        top = min(top, int(1e9 / (kv * group * new[1])))
        most = {"decode": 128, "few": 32, "chunk": 4}[kind]
        B = max(1, min(log_int(rng, 1, most), 240000 // top, 1900000 // (top * kv),
                       int(1e9 / (kv * group * new[1] * (top + new[1])))))
        c = paged_case("", B, kv * group, kv, D, page, x16, new, (max(0, top // rng.choice([1, 4, 50]) - 1), top), seed)
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# What a case is made of
# ---------------------------------------------------------------------------

def new_and_past(case):
    """Per sequence of a paged case: (new tokens, tokens cached before them)."""
    r = random.Random(case["lengths"])
    return [(r.randint(case["new_lo"], case["new_hi"]), r.randint(case["past_lo"], case["past_hi"]))
            for _ in range(case["B"])]


def prompt_lengths(case):
    r = random.Random(case["lengths"])
    return [r.randint(case["len_lo"], case["len_hi"]) for _ in range(case["B"])]


def generator(seed, salt):
    return torch.Generator(device="cuda").manual_seed((int(seed) * 1000003 + salt * 7919) % (1 << 62))


def table_of(max_pos, rot):
    """cos and sin of position x frequency, [max_pos][rot]: the cosines of rot / 2 frequencies, then the sines."""
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    a = torch.arange(max_pos, dtype=torch.float64, device="cuda")[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).float()


def heads_of(T, H, D, dtype, gen, outlier=0.0):
    x = torch.randn(T, H, D, generator=gen, device="cuda")
    if outlier:
        x[:, :, 0] += outlier * (1 + 0.1 * torch.randn(T, H, generator=gen, device="cuda"))
    return x.to(DT[dtype])


def norm_weights(H, D, gen):
    return 1 + 0.1 * torch.randn(H, D, generator=gen, device="cuda")


def cache_of(pages, H, page, D, used, gen, offset):
    """Pages as a quantizer leaves them: codes on a 4-bit grid, (scale, offset) pairs; slots that no token has
    reached hold what memory held before (here NaN pairs). ``used``: bool [pages, page]."""
    shape = (pages, H, page)
    codes = torch.empty(*shape, D // 2, dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 26) // (H * page * D))
    for a in range(0, pages, step):  # in pieces: the draws are wider than what they become
        u = (torch.randn(min(step, pages - a), H, page, D, generator=gen, device="cuda") * 2.4).round_().clamp_(-7, 7)
        u = (u + 8).to(torch.uint8)
        codes[a:a + step] = u[..., 0::2] | (u[..., 1::2] << 4)
    scale = 0.42 * torch.exp(0.15 * torch.randn(*shape, generator=gen, device="cuda"))
    off = offset * (1 + 0.1 * torch.randn(*shape, generator=gen, device="cuda"))
    par = torch.stack([scale, off], -1)
    par = torch.where(used[:, None, :, None], par, float("nan")).contiguous()
    return codes, par


def prepare(case, seed):
    gen = generator(seed, 1)
    kind, D = case["kind"], case["D"]
    s = {"case": dict(case)}
    if kind == "rope":
        T, H = case["T"], case["heads"]
        s["x"] = heads_of(T, H, D, case["x"], gen, 4.0)
        s["norm"] = norm_weights(H, D, gen) if case["norm"] else None
        s["pos"] = torch.randint(0, case["max_pos"], (T,), generator=gen, device="cuda", dtype=torch.int32)
        s["table"] = table_of(case["max_pos"], case["rot"])
    elif kind == "cache":
        T, Hq, H, P = case["T"], case["q_heads"], case["kv_heads"], case["page"]
        pages = -(-T // P) + 3
        s["slots"] = torch.randperm(pages * P, generator=gen, device="cuda")[:T].contiguous()
        used = torch.ones(pages, P, dtype=torch.bool, device="cuda")
        kc, kp = cache_of(pages, H, P, D, used, gen, 1.0)
        vc, vp = cache_of(pages, H, P, D, used, gen, 0.1)
        s["cache"] = (kc, kp, vc, vp)
        if case["write"]:
            qkv = torch.cat([heads_of(T, Hq, D, case["x"], gen, 2.0), heads_of(T, H, D, case["x"], gen, 20.0),
                             heads_of(T, H, D, case["x"], gen)], 1)  # one projection's output
            s["q"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
            s["q_norm"] = norm_weights(Hq, D, gen) if case["norm"] else None
            s["k_norm"] = norm_weights(H, D, gen) if case["norm"] else None
            s["pos"] = torch.randint(0, case["max_pos"], (T,), generator=gen, device="cuda", dtype=torch.int32)
            s["table"] = table_of(case["max_pos"], case["rot"])
    elif kind == "paged":
        B, Hq, H, P = case["B"], case["q_heads"], case["kv_heads"], case["page"]
        lengths = new_and_past(case)
        n = torch.tensor([a for a, _ in lengths], device="cuda")
        lens = torch.tensor([a + b for a, b in lengths], device="cuda")
        most = max(a + b for a, b in lengths)
        width = -(-most // P) + 1
        need = (lens + P - 1) // P
        total = int(need.sum()) + 2
        at = torch.arange(width, device="cuda")[None]
        first = torch.cumsum(need, 0) - need
        order = torch.randperm(total, generator=gen, device="cuda")
        table = torch.where(at < need[:, None], order[(first[:, None] + at).clamp(max=total - 1)], -1)
        used = torch.zeros(total, P, dtype=torch.bool, device="cuda")
        token = at[:, :, None] * P + torch.arange(P, device="cuda")
        used[table.clamp(min=0)[(table >= 0)]] = (token < lens[:, None, None])[table >= 0]
        kc, kp = cache_of(total, H, P, D, used, gen, 1.0)
        vc, vp = cache_of(total, H, P, D, used, gen, 0.1)
        s["cache"] = (kc, kp, vc, vp)
        s["table"] = table.to(torch.int32).contiguous()
        s["lens"] = lens.to(torch.int32)
        s["cu"] = torch.cat([torch.zeros(1, device="cuda", dtype=torch.int64), torch.cumsum(n, 0)]).to(torch.int32)
        s["max_new"] = max(a for a, _ in lengths)
        s["max_len"] = most
        s["q"] = heads_of(sum(a for a, _ in lengths), Hq, D, case["x"], gen)
        s["scale"] = 1 / math.sqrt(D)
    else:
        lengths = prompt_lengths(case)
        T, Hq, H = sum(lengths), case["q_heads"], case["kv_heads"]
        qkv = heads_of(T, Hq + 2 * H, D, case["x"], gen)
        s["q"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
        n = torch.tensor(lengths, device="cuda")
        s["cu"] = torch.cat([torch.zeros(1, device="cuda", dtype=torch.int64), torch.cumsum(n, 0)]).to(torch.int32)
        s["max_new"] = max(lengths)
        s["scale"] = 1 / math.sqrt(D)
    return s


def visible_pairs(case):
    if case["kind"] == "paged":
        return sum(n * past + n * (n + 1) // 2 for n, past in new_and_past(case))
    if case["causal"]:
        return sum(n * (n + 1) // 2 for n in prompt_lengths(case))
    return sum(n * n for n in prompt_lengths(case))


def work(case):
    kind, D, xb = case["kind"], case["D"], BYTES[case["x"]]
    if kind == "rope":
        T, H = case["T"], case["heads"]
        values = T * H * D
        norm = 4 * H * D if case["norm"] else 0
        flops = values * (3 + (5 if case["norm"] else 0) + (math.log2(D) if case["rotate"] else 0))
        return {"bytes": 2 * values * xb + norm + T * 4 + min(T, case["max_pos"]) * case["rot"] * 4, "flops": flops}
    if kind == "cache":
        T, Hq, H = case["T"], case["q_heads"], case["kv_heads"]
        held = T * H * (D + 16)
        b = held + T * 8 + 2 * T * H * D * xb
        f = T * H * D * (2 + math.log2(D) + 2)
        if case["write"]:
            b += held + 2 * T * H * D * xb + 2 * T * Hq * D * xb + T * 4 + min(T, case["max_pos"]) * case["rot"] * 4
            f += T * (Hq + 2 * H) * D * (3 + math.log2(D) + 4)
        return {"bytes": b, "flops": f}
    Hq, H = case["q_heads"], case["kv_heads"]
    flops = 4.0 * D * Hq * visible_pairs(case)
    if kind == "paged":
        lengths = new_and_past(case)
        new, held = sum(n for n, _ in lengths), sum(n + p for n, p in lengths)
        pages = sum(-(-(n + p) // case["page"]) for n, p in lengths)
        return {"bytes": held * H * (D + 16) + new * Hq * (2 * D * xb + 4) + 4 * pages + 8 * case["B"], "flops": flops}
    T = sum(prompt_lengths(case))
    return {"bytes": T * D * xb * (2 * Hq + 2 * H) + 4 * T * Hq + 4 * case["B"], "flops": flops}


# ---------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------

def total(x):
    """Sums of the last dimension, neighbours first."""
    while x.shape[-1] > 1:
        x = x[..., 0::2] + x[..., 1::2]
    return x


def hadamard(x):
    """x H over the last dimension, not normalised, distance 1 first."""
    shape, h = x.shape, 1
    while h < shape[-1]:
        x = x.reshape(*shape[:-1], shape[-1] // (2 * h), 2, h)
        a, b = x[..., 0, :], x[..., 1, :]
        x = torch.stack([a + b, a - b], -2)
        h *= 2
    return x.reshape(shape)


def root(D):
    return torch.tensor(1 / math.sqrt(D), dtype=torch.float32, device="cuda")


def normed(x, w):
    if w is None:
        return x
    mean = total(x * x) * (1.0 / x.shape[-1])
    return x * torch.div(torch.ones_like(mean), torch.sqrt(mean + EPS)) * w


def roped(x, pos, table, rot, interleaved):
    if not rot:
        return x
    t = table[pos.long()][:, None]
    c, s = t[..., :rot // 2], t[..., rot // 2:]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    a, b = a * c - b * s, b * c + a * s
    y = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([y, x[..., rot:]], -1)


def quantized(y, rotate):
    """Codes u, scales and offsets of heads y: the offset is the mean of what is stored."""
    D = y.shape[-1]
    if rotate:
        off = y[..., :1] * root(D)
        r = hadamard(torch.cat([torch.zeros_like(off), y[..., 1:]], -1))
    else:
        off = total(y) * (1.0 / D)
        r = y - off
    top = r.abs().amax(-1, keepdim=True)
    u = torch.round(r * torch.div(torch.full_like(top, 7.0), top)).clamp(-7, 7)
    u = torch.where(top > 0, u, torch.zeros_like(u)) + 8
    scale = top * root(D) * (1 / 7) if rotate else top * (1 / 7)
    return u.to(torch.uint8), torch.cat([scale, off], -1)


def unpacked(codes):
    return torch.stack([codes & 15, codes >> 4], -1).flatten(-2).float() - 8


def values(codes, par):
    return unpacked(codes) * par[..., :1] + par[..., 1:]


def plain_rope(s):
    c = s["case"]
    y = roped(normed(s["x"].float(), s["norm"]), s["pos"], s["table"], c["rot"], c["interleaved"])
    if c["rotate"]:
        y = hadamard(y) * root(c["D"])
    return y.to(s["x"].dtype)


def plain_cache(s):
    c = s["case"]
    kc, kp, vc, vp = s["cache"]
    page, at, dt = s["slots"] // c["page"], s["slots"] % c["page"], DT[c["x"]]
    out = []
    if c["write"]:
        q = roped(normed(s["q"].float(), s["q_norm"]), s["pos"], s["table"], c["rot"], c["interleaved"])
        out.append((hadamard(q) * root(c["D"])).to(dt))
        k = roped(normed(s["k"].float(), s["k_norm"]), s["pos"], s["table"], c["rot"], c["interleaved"])
        u, kp[page, :, at] = quantized(k, True)
        kc[page, :, at] = u[..., 0::2] | (u[..., 1::2] << 4)
        u, vp[page, :, at] = quantized(s["v"].float(), False)
        vc[page, :, at] = u[..., 0::2] | (u[..., 1::2] << 4)
    k = values(kc[page, :, at], kp[page, :, at])
    out.append((hadamard(k) * root(c["D"])).to(dt))
    out.append(values(vc[page, :, at], vp[page, :, at]).to(dt))
    return out


def attended(q, k, v, seen, scale):
    """q [B, H, G, n, D], k and v [B, H, L, D], seen [B, n, L] -> out [B, H, G, n, D], lse [B, H, G, n]."""
    B, H, G, n, D = q.shape
    z = torch.matmul(q.reshape(B, H, G * n, D), k.transpose(-1, -2)).reshape(B, H, G, n, -1)
    z.mul_(scale).masked_fill_(~seen[:, None, None], float("-inf"))
    top = z.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    z.sub_(top).exp_()
    sums = z.sum(-1, keepdim=True)
    out = torch.matmul(z.reshape(B, H, G * n, -1), v).reshape(B, H, G, n, D) / torch.where(sums > 0, sums, 1.0)
    return out, (top + torch.log(sums))[..., 0]


def padded(x, first, counts, most):
    """Rows first[b] .. + counts[b] of x as [B, most, ...] (what lies past a sequence repeats some row), and the rows'
    places."""
    i = torch.arange(most, device="cuda")
    at = torch.minimum(first[:, None] + i, first[:, None] + (counts[:, None] - 1).clamp(min=0)).clamp(max=x.shape[0] - 1)
    return x[at], i[None] < counts[:, None]


def unpadded(out, lse, live, dtype):
    """[B, H, G, n, D] -> [T, H * G, D] and [T, H * G] of the live rows, in order."""
    B, H, G, n, D = out.shape
    return (out.permute(0, 3, 1, 2, 4).reshape(B, n, H * G, D)[live].to(dtype),
            lse.permute(0, 3, 1, 2).reshape(B, n, H * G)[live])


def plain_paged(s):
    c = s["case"]
    H, G, D, P = c["kv_heads"], c["q_heads"] // c["kv_heads"], c["D"], c["page"]
    kc, kp, vc, vp = s["cache"]
    lens, cu = s["lens"].long(), s["cu"].long()
    n = cu[1:] - cu[:-1]
    q, live = padded(s["q"].float(), cu[:-1], n, s["max_new"])
    q = q.reshape(c["B"], -1, H, G, D).permute(0, 2, 3, 1, 4)
    j = torch.arange(s["max_len"], device="cuda")
    page, at = s["table"].long()[:, j // P].clamp(min=0), (j % P)[None]
    there = j[None] < lens[:, None]
    k = torch.where(there[:, :, None, None], values(kc[page, :, at], kp[page, :, at]), 0.0).transpose(1, 2)
    v = torch.where(there[:, :, None, None], values(vc[page, :, at], vp[page, :, at]), 0.0).transpose(1, 2)
    i = torch.arange(s["max_new"], device="cuda")
    seen = (j[None, None] <= (lens - n)[:, None, None] + i[None, :, None]) & there[:, None]
    out, lse = attended(q, k, v, seen, s["scale"])
    return unpadded(out, lse, live, s["q"].dtype)


def plain_prompt(s):
    c = s["case"]
    H, G, D = c["kv_heads"], c["q_heads"] // c["kv_heads"], c["D"]
    cu = s["cu"].long()
    n = cu[1:] - cu[:-1]
    q, live = padded(s["q"].float(), cu[:-1], n, s["max_new"])
    q = q.reshape(c["B"], -1, H, G, D).permute(0, 2, 3, 1, 4)
    k = padded(s["k"].float(), cu[:-1], n, s["max_new"])[0].transpose(1, 2)
    v = padded(s["v"].float(), cu[:-1], n, s["max_new"])[0].transpose(1, 2)
    i = torch.arange(s["max_new"], device="cuda")
    seen = live[:, None, :] & ((i[None, :] <= i[:, None]) if c["causal"] else (i[None, :] >= 0))[None]
    out, lse = attended(q, k, v, seen, s["scale"])
    return unpadded(out, lse, live, s["q"].dtype)


# ---------------------------------------------------------------------------
# The library's calls
# ---------------------------------------------------------------------------

def own_run(s):
    from paper_2606_07116_gb300 import offq as Q
    c = s["case"]
    kind = c["kind"]
    if kind == "rope":
        return Q.rope_heads(s["x"], s["pos"], s["table"], norm=s["norm"], eps=EPS, interleaved=c["interleaved"],
                            rotate=c["rotate"])
    if kind == "prompt":
        return Q.prompt_attention(s["q"], s["k"], s["v"], s["cu"], scale=s["scale"], causal=c["causal"], lse=True)
    cache = Q.KV4Cache(*s["cache"])
    if kind == "paged":
        return Q.paged_attention(s["q"], cache, s["table"], s["lens"], s["cu"], s["max_new"], scale=s["scale"], lse=True)
    out = []
    if c["write"]:
        out.append(Q.kv4_paged_write(cache, s["k"], s["v"], s["slots"], s["pos"], s["table"], q=s["q"],
                                     q_norm=s["q_norm"], k_norm=s["k_norm"], eps=EPS, interleaved=c["interleaved"]))
    k, v = Q.kv4_paged_read(cache, s["slots"], out_dtype=DT[c["x"]])
    return out + [k, v]


def run(s):
    if own:
        return own_run(s)
    return {"rope": plain_rope, "cache": plain_cache, "paged": plain_paged, "prompt": plain_prompt}[s["case"]["kind"]](s)


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------

def exact_matrix(D):
    """The Sylvester Hadamard matrix / sqrt(D): entry (i, j) is the parity of i & j."""
    i = torch.arange(D, device="cuda")
    bits = i[:, None] & i[None, :]
    parity = sum((bits >> b) & 1 for b in range(8)) % 2
    return (1.0 - 2.0 * parity.double()) / math.sqrt(D)


def exact_heads(x, w, pos, table, rot, interleaved):
    y = x.double()
    if w is not None:
        y = y / torch.sqrt((y ** 2).mean(-1, keepdim=True) + EPS) * w.double()
    z = y.clone()
    for m in range(rot // 2):
        a, b = (2 * m, 2 * m + 1) if interleaved else (m, m + rot // 2)
        c, s = table[pos.long(), m].double()[:, None], table[pos.long(), m + rot // 2].double()[:, None]
        z[..., a] = y[..., a] * c - y[..., b] * s
        z[..., b] = y[..., b] * c + y[..., a] * s
    return z


def exact_quantized(y):
    """The values that the 4-bit grid has for y."""
    o = y.mean(-1, keepdim=True)
    r = y - o
    s = r.abs().amax(-1, keepdim=True) / 7
    return s * torch.round(r / torch.where(s > 0, s, 1.0)).clamp(-7, 7) + o


def exact_token(codes, par, page, at):
    """Values [L, H, D] of the tokens in (page, at)."""
    b = codes[page, :, at].long()
    u = torch.empty(*b.shape[:-1], 2 * b.shape[-1], dtype=torch.float64, device="cuda")
    u[..., 0::2] = (b % 16 - 8).double()
    u[..., 1::2] = (b // 16 - 8).double()
    p = par[page, :, at].double()
    return u * p[..., 0:1] + p[..., 1:2]


def exact_attention(q, k, v, causal_from, scale):
    """One sequence: q [n, Hq, D] over k, v [L, H, D]; query i sees keys 0 .. causal_from + i (all for None)."""
    n, Hq, D = q.shape
    L, H = k.shape[0], k.shape[1]
    out = torch.zeros(n, Hq, D, dtype=torch.float64, device="cuda")
    lse = torch.full((n, Hq), float("-inf"), dtype=torch.float64, device="cuda")
    hidden = None
    if causal_from is not None:
        hidden = torch.arange(L, device="cuda")[None, :] > causal_from + torch.arange(n, device="cuda")[:, None]
    for h in range(Hq):
        z = q[:, h].double() @ k[:, h * H // Hq].double().T * scale
        if hidden is not None:
            z = z.masked_fill(hidden, float("-inf"))
        lse[:, h] = torch.logsumexp(z, 1)
        out[:, h] = torch.softmax(z, 1) @ v[:, h * H // Hq].double()
    return out, lse


def exact(case, seed):
    s = prepare(case, seed)
    kind, D = case["kind"], case["D"]
    if kind == "rope":
        y = exact_heads(s["x"], s["norm"], s["pos"], s["table"], case["rot"], case["interleaved"])
        return y @ exact_matrix(D) if case["rotate"] else y
    if kind == "cache":
        page, at = s["slots"] // case["page"], s["slots"] % case["page"]
        M = exact_matrix(D)
        if not case["write"]:
            kc, kp, vc, vp = s["cache"]
            return [exact_token(kc, kp, page, at) @ M, exact_token(vc, vp, page, at)]
        q = exact_heads(s["q"], s["q_norm"], s["pos"], s["table"], case["rot"], case["interleaved"]) @ M
        k = exact_heads(s["k"], s["k_norm"], s["pos"], s["table"], case["rot"], case["interleaved"]) @ M
        return [q, exact_quantized(k) @ M, exact_quantized(s["v"].double())]
    if 4.0 * D * case["q_heads"] * visible_pairs(case) > 3e12:
        return None
    outs, lses, row = [], [], 0
    if kind == "paged":
        kc, kp, vc, vp = s["cache"]
        for b, (n, past) in enumerate(new_and_past(case)):
            j = torch.arange(n + past, device="cuda")
            page, at = s["table"][b].long()[j // case["page"]], j % case["page"]
            o, l = exact_attention(s["q"][row:row + n], exact_token(kc, kp, page, at), exact_token(vc, vp, page, at),
                                   past, s["scale"])
            outs.append(o)
            lses.append(l)
            row += n
    else:
        for n in prompt_lengths(case):
            o, l = exact_attention(s["q"][row:row + n], s["k"][row:row + n], s["v"][row:row + n],
                                   0 if case["causal"] else None, s["scale"])
            outs.append(o)
            lses.append(l)
            row += n
    return torch.cat(outs), torch.cat(lses)
