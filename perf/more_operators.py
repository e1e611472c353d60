"""Attention with a sliding window and attention over shared prefixes, as cases that can be timed and compared.

Layers with a sliding window, and streams that run past the length a model was trained on, see their newest tokens and a
few first ones; a batch that answers on one document, or starts with one system prompt, sees the same long prefix. Both
read the paged 4-bit cache of the other operators; a prompt is attended on its 16-bit keys and values.

Kinds:
  window   new tokens (one, a few drafted ones, a chunk) over the pages of their sequences: each query sees the window of
           newest tokens up to itself and the sinks. Pages that no query sees any more were given back: their table
           entries are -1.
  prompt   the same inside packed prompts of different lengths.
  prefix   new tokens of sequences that share prefixes: each query sees its sequence's prefix and its own tokens.

Sizes are the heads, head dimensions and token counts of the repository's workloads (Llama-2-7B: 32 heads, Llama-3-8B:
32 over 8, Llama-2-70B: 64 over 8; 128 channels) and generic ones around them.

``own`` chooses between the library's calls and their plain form, elementary torch operations in 32 bits.
"""

from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DT = {"bf16": torch.bfloat16, "f16": torch.float16}
XB = 2  # bytes of a query's or output's channel


def window_case(name, B, q_heads, kv_heads, D, page, x, new, past, window, sinks, lengths):
    """``new`` and ``past``: (least, most) tokens of a sequence; ``lengths``: the seed of the batch's lengths."""
    return {"name": name, "kind": "window", "B": B, "q_heads": q_heads, "kv_heads": kv_heads, "D": D, "page": page,
            "x": x, "new_lo": new[0], "new_hi": new[1], "past_lo": past[0], "past_hi": past[1], "window": window,
            "sinks": sinks, "lengths": lengths}


def prompt_case(name, B, q_heads, kv_heads, D, x, length, window, sinks, lengths):
    return {"name": name, "kind": "prompt", "B": B, "q_heads": q_heads, "kv_heads": kv_heads, "D": D, "x": x,
            "len_lo": length[0], "len_hi": length[1], "window": window, "sinks": sinks, "lengths": lengths}


def prefix_case(name, prefixes, prefix, B, q_heads, kv_heads, D, page, x, new, past, lengths):
    """``prefixes`` prefixes of (least, most) = ``prefix`` tokens, shared by runs of the B sequences."""
    return {"name": name, "kind": "prefix", "prefixes": prefixes, "prefix_lo": prefix[0], "prefix_hi": prefix[1], "B": B,
            "q_heads": q_heads, "kv_heads": kv_heads, "D": D, "page": page, "x": x, "new_lo": new[0], "new_hi": new[1],
            "past_lo": past[0], "past_hi": past[1], "lengths": lengths}


def listed():
    return [
        # A single stream's next token far into a conversation (Llama-3-8B heads): latency.
        window_case("window_decode_1", 1, 32, 8, 128, 64, "bf16", (1, 1), (6000, 6000), 1024, 4, 0),
        # A serving batch: 64 streams of very different lengths, Llama-2-70B heads, small pages.
        window_case("window_decode_ragged", 64, 64, 8, 128, 16, "f16", (1, 1), (1, 40000), 4096, 4, 1),
        # Four drafted tokens verified in each of 16 streams, smaller heads, an odd window without sinks.
        window_case("window_verify_4", 16, 16, 4, 64, 32, "bf16", (4, 4), (500, 20000), 1001, 0, 2),
        # Chunks of two long prompts that are being taken in piece by piece.
        window_case("window_chunk_1000", 2, 32, 8, 128, 64, "bf16", (900, 1024), (15000, 16000), 4096, 16, 3),
        # A batch of prompts of different lengths, smaller heads, half precision, a short window.
        prompt_case("prompt_ragged", 24, 16, 4, 64, "f16", (5, 2000), 300, 1, 4),
        # One prompt of odd length with an odd number of heads per key head and many sinks.
        prompt_case("prompt_5001", 1, 20, 4, 128, "bf16", (5001, 5001), 512, 64, 5),
        # One long prompt, Llama-3-8B heads.
        prompt_case("prompt_16384", 1, 32, 8, 128, "bf16", (16384, 16384), 4096, 4, 6),
        # Two streams behind a short system prompt: latency.
        prefix_case("prefix_decode_2", 1, (500, 500), 2, 32, 8, 128, 64, "bf16", (1, 1), (0, 60), 7),
        # 64 streams that answer on one document, Llama-2-70B heads, small pages.
        prefix_case("prefix_decode_64", 1, (8000, 8000), 64, 64, 8, 128, 16, "f16", (1, 1), (0, 2000), 8),
        # A large batch behind a long context.
        prefix_case("prefix_decode_256", 1, (32768, 32768), 256, 32, 8, 128, 64, "bf16", (1, 1), (100, 1000), 9),
        # Several system prompts, a few drafted tokens, a key head for each query head (Llama-2-7B).
        prefix_case("prefix_groups", 5, (300, 6000), 30, 32, 32, 128, 128, "f16", (1, 3), (0, 1500), 10),
        # Questions of different lengths taken in behind a common document.
        prefix_case("prefix_chunks", 1, (6000, 6000), 6, 32, 8, 128, 64, "bf16", (100, 700), (0, 0), 11),
    ]


def log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(["decode", "few", "chunk", "prompt", "prefix", "prefix_chunk"], [4, 2, 3, 4, 5, 2])[0]
    D = rng.choice([64, 128, 128])
    page = rng.choice([16, 32, 64, 128, 256])
    x = rng.choice(["bf16", "bf16", "f16"])
    seed = rng.randrange(1 << 20)
    kv = rng.choice([1, 2, 4, 8, 32])
    group = rng.choice([1, 2, 4, 5, 8]) if kv < 32 else 1
    heads = kv * group
    window = log_int(rng, 1, 8192)
    sinks = rng.choice([0, 1, 4, 4, 16, rng.randint(5, 300)])
    if kind == "prompt":
        top = log_int(rng, 1, 20000)
        seen = min(window + sinks, top)
        B = max(1, min(log_int(rng, 1, 64), 24000 // top, int(1.8e9 / heads / top / seen)))
        top = min(top, int(1.8e9 / heads / seen))
        c = prompt_case("", B, heads, kv, D, x, (max(1, top // rng.choice([1, 4, 50])), top), window, sinks, seed)
    elif kind in ("prefix", "prefix_chunk"):
        chunk = kind == "prefix_chunk"
        new = (1, rng.choice([1, 1, 1, 2, 4])) if not chunk else (log_int(rng, 1, 30), log_int(rng, 30, 700))
        prefix = log_int(rng, 1, 40000)
        B = log_int(rng, 1, 8 if chunk else 256)
        B = max(1, min(B, int(2e8 / (heads * new[1] * prefix))))
        past = 0 if chunk and rng.random() < 0.5 else log_int(rng, 1, 3000)
        past = min(past, int(1.2e6 / (B * kv)))
        groups = min(B, log_int(rng, 1, 8))
        prefix = max(1, min(prefix, int(1.2e6 / (groups * kv))))
        c = prefix_case("", groups, (max(1, prefix // rng.choice([1, 1, 4, 50])), prefix), B, heads, kv, D, page, x, new,
                        (past // rng.choice([1, 4, 50]), past), seed)
    else:
        new = {"decode": (1, 1), "few": (1, rng.randint(2, 9)), "chunk": (log_int(rng, 4, 100), log_int(rng, 100, 1500))}[kind]
        top = log_int(rng, 1, 60000)
        seen = min(window + sinks, top) + new[1]
        most = {"decode": 128, "few": 32, "chunk": 4}[kind]
        B = max(1, min(log_int(rng, 1, most), 1500000 // (seen * kv), int(2e8 / (heads * new[1] * seen))))
        c = window_case("", B, heads, kv, D, page, x, new, (max(0, top // rng.choice([1, 4, 50]) - 1), top), window, sinks,
                        seed)
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# What a case is made of
# ---------------------------------------------------------------------------

def new_and_past(case):
    """Per sequence of a paged case: (new tokens, tokens of its own cached before them)."""
    r = random.Random(case["lengths"])
    return [(r.randint(case["new_lo"], case["new_hi"]), r.randint(case["past_lo"], case["past_hi"]))
            for _ in range(case["B"])]


def prompt_lengths(case):
    r = random.Random(case["lengths"])
    return [r.randint(case["len_lo"], case["len_hi"]) for _ in range(case["B"])]


def prefix_runs(case):
    """Per prefix: (tokens, first sequence, sequences)."""
    r = random.Random(case["lengths"] + 1)
    cuts = sorted(r.sample(range(1, case["B"]), case["prefixes"] - 1))
    return [(r.randint(case["prefix_lo"], case["prefix_hi"]), a, b - a)
            for a, b in zip([0] + cuts, cuts + [case["B"]])]


def generator(seed, salt):
    return torch.Generator(device="cuda").manual_seed((int(seed) * 1000003 + salt * 7919) % (1 << 62))


def heads_of(T, H, D, dtype, gen):
    return torch.randn(T, H, D, generator=gen, device="cuda").to(DT[dtype])


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
    return codes, torch.where(used[:, None, :, None], par, float("nan")).contiguous()


def tables_of(runs, page, gen):
    """For runs of (tokens, first token that is still held, tokens at the start that are) a row each: block tables over
    shuffled pages, -1 where a page was given back or never taken, and which slots of the pages hold tokens."""
    held = [[i for i in range(-(-n // page)) if i * page < first or (i + 1) * page > lo] for n, lo, first in runs]
    total = sum(len(h) for h in held) + 2
    order = np.array(torch.randperm(total, generator=gen, device="cuda").cpu())
    table = np.full((len(runs), max(-(-n // page) for n, _, _ in runs) + 1), -1, np.int32)
    used = np.zeros((total, page), bool)
    at = 0
    for b, ((n, _, _), h) in enumerate(zip(runs, held)):
        table[b, h] = order[at:at + len(h)]
        for i in h:
            used[table[b, i], :n - i * page] = True
        at += len(h)
    return torch.from_numpy(table).cuda(), torch.from_numpy(used).cuda()


def cumulative(n):
    return torch.tensor([0] + list(np.cumsum(n)), dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = generator(seed, 1)
    kind, D, Hq, H = case["kind"], case["D"], case["q_heads"], case["kv_heads"]
    s = {"case": dict(case), "scale": 1 / math.sqrt(D)}
    if kind == "prompt":
        lengths = prompt_lengths(case)
        qkv = heads_of(sum(lengths), Hq + 2 * H, D, case["x"], gen)  # one projection's output
        s["q"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
        s["cu"] = cumulative(lengths)
        s["max_new"] = max(lengths)
        return s
    lengths = new_and_past(case)
    runs = [(n + past, 0, 0) for n, past in lengths]
    if kind == "window":
        runs = [(n + past, max(0, past + 1 - case["window"]), case["sinks"]) for n, past in lengths]
    shared = prefix_runs(case) if kind == "prefix" else []
    table, used = tables_of([(n, 0, 0) for n, _, _ in shared] + runs, case["page"], gen)
    kc, kp = cache_of(used.shape[0], H, case["page"], D, used, gen, 1.0)
    vc, vp = cache_of(used.shape[0], H, case["page"], D, used, gen, 0.1)
    s["cache"] = (kc, kp, vc, vp)
    s["table"] = table[len(shared):].contiguous()
    s["lens"] = torch.tensor([n for n, _, _ in runs], dtype=torch.int32, device="cuda")
    s["cu"] = cumulative([n for n, _ in lengths])
    s["max_new"] = max(n for n, _ in lengths)
    s["max_len"] = max(n for n, _, _ in runs)
    s["q"] = heads_of(sum(n for n, _ in lengths), Hq, D, case["x"], gen)
    if shared:
        s["prefix_table"] = table[:len(shared)].contiguous()
        s["prefix_lens"] = torch.tensor([n for n, _, _ in shared], dtype=torch.int32, device="cuda")
        s["prefix_cu"] = cumulative([n for _, _, n in shared])
        s["max_prefix"] = max(n for n, _, _ in shared)
        s["max_shared"] = max(sum(n for n, _ in lengths[a:a + k]) for _, a, k in shared)
    return s


def in_window(past, n, window, sinks):
    """Pairs of n queries after `past` tokens and the keys they see."""
    p = np.arange(past, past + n, dtype=np.int64)
    return int((np.minimum(p + 1, window) + np.minimum(sinks, np.maximum(p + 1 - window, 0))).sum())


def work(case):
    kind, D, Hq, H = case["kind"], case["D"], case["q_heads"], case["kv_heads"]
    if kind == "prompt":
        lengths = prompt_lengths(case)
        T = sum(lengths)
        pairs = sum(in_window(0, n, case["window"], case["sinks"]) for n in lengths)
        return {"bytes": T * D * XB * (2 * Hq + 2 * H) + 4 * T * Hq + 4 * case["B"], "flops": 4.0 * D * Hq * pairs}
    lengths = new_and_past(case)
    new = sum(n for n, _ in lengths)
    held = [n + past for n, past in lengths]
    pairs = sum(n * past + n * (n + 1) // 2 for n, past in lengths)
    if kind == "window":
        W, S = case["window"], case["sinks"]
        lo = [max(0, past + 1 - W) for _, past in lengths]
        held = [n + past - a + min(S, a) for (n, past), a in zip(lengths, lo)]
        pairs = sum(in_window(past, n, W, S) for n, past in lengths)
    if kind == "prefix":
        for tokens, a, k in prefix_runs(case):
            held.append(tokens)
            pairs += tokens * sum(n for n, _ in lengths[a:a + k])
    pages = sum(-(-n // case["page"]) for n in held)
    return {"bytes": sum(held) * H * (D + 16) + new * Hq * (2 * D * XB + 4) + 4 * pages + 8 * case["B"],
            "flops": 4.0 * D * Hq * pairs}


# ---------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------

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


def unpacked(codes):
    return torch.stack([codes & 15, codes >> 4], -1).flatten(-2).float() - 8


def gathered(cache, table, page, tokens, there):
    """Keys and values [B, H, L, D] of the tokens [B, L] of each row of the table, zeros where not `there`."""
    kc, kp, vc, vp = cache
    at = torch.gather(table.long(), 1, (tokens // page).clamp(max=table.shape[1] - 1)).clamp(min=0)
    slot = tokens % page
    return [torch.where(there[:, :, None, None], unpacked(c[at, :, slot]) * p[at, :, slot][..., :1] + p[at, :, slot][..., 1:],
                        0.0).transpose(1, 2) for c, p in ((kc, kp), (vc, vp))]


def padded(x, first, counts, most):
    """Rows first[b] .. + counts[b] of x as [B, most, ...] (what lies past a sequence repeats some row), and the rows'
    places."""
    i = torch.arange(most, device="cuda")
    at = torch.minimum(first[:, None] + i, first[:, None] + (counts[:, None] - 1).clamp(min=0)).clamp(max=x.shape[0] - 1)
    return x[at], i[None] < counts[:, None]


def grouped(q, H):
    """[B, n, Hq, D] -> [B, H, G, n, D]."""
    B, n, Hq, D = q.shape
    return q.reshape(B, n, H, Hq // H, D).permute(0, 2, 3, 1, 4)


def unpadded(out, lse, live):
    """[B, H, G, n, D] -> [T, H * G, D] and [T, H * G] of the live rows, in order."""
    B, H, G, n, D = out.shape
    return out.permute(0, 3, 1, 2, 4).reshape(B, n, H * G, D)[live], lse.permute(0, 3, 1, 2).reshape(B, n, H * G)[live]


def plain_window(s):
    c = s["case"]
    W, S = c["window"], c["sinks"]
    lens, cu = s["lens"].long(), s["cu"].long()
    n = cu[1:] - cu[:-1]
    q, live = padded(s["q"].float(), cu[:-1], n, s["max_new"])
    # The tokens that some query of a sequence sees: the sinks, then those from its first query's window on.
    lo = torch.minimum((lens - n + 1 - W).clamp(min=0), lens)
    S = min(S, s["max_len"])
    most = min(W + s["max_new"], s["max_len"])
    i = torch.arange(S + most, device="cuda")[None]
    tokens = torch.where(i < S, i, i - S + lo[:, None])
    there = torch.where(i < S, i < torch.minimum(lo, lens)[:, None], tokens < lens[:, None])
    k, v = gathered(s["cache"], s["table"], c["page"], tokens.clamp(max=s["max_len"] - 1), there)
    at = (lens - n)[:, None] + torch.arange(s["max_new"], device="cuda")
    seen = there[:, None] & (tokens[:, None] <= at[..., None]) & ((tokens[:, None] > at[..., None] - W) | (tokens[:, None] < S))
    out, lse = attended(grouped(q, c["kv_heads"]), k, v, seen, s["scale"])
    out, lse = unpadded(out, lse, live)
    return out.to(s["q"].dtype), lse


def plain_prompt(s):
    c = s["case"]
    W, S, H, T = c["window"], c["sinks"], c["kv_heads"], s["q"].shape[0]
    cu = s["cu"].long()
    n = cu[1:] - cu[:-1]
    q, live = padded(s["q"].float(), cu[:-1], n, s["max_new"])
    k = padded(s["k"].float(), cu[:-1], n, s["max_new"])[0].transpose(1, 2)
    v = padded(s["v"].float(), cu[:-1], n, s["max_new"])[0].transpose(1, 2)
    outs, lses = [], []
    for a in range(0, s["max_new"], 1024):  # queries of a piece over the keys that they can see
        b = min(a + 1024, s["max_new"])
        lo = max(0, a + 1 - W)
        j = torch.cat([torch.arange(min(S, lo), device="cuda"), torch.arange(lo, b, device="cuda")])
        at = torch.arange(a, b, device="cuda")[:, None]
        seen = (j[None] <= at) & ((j[None] > at - W) | (j[None] < S))
        out, lse = attended(grouped(q[:, a:b], H), k[:, :, j], v[:, :, j], seen[None] & (j < n[:, None])[:, None], s["scale"])
        outs.append(out)
        lses.append(lse)
    out, lse = unpadded(torch.cat(outs, 3), torch.cat(lses, 3), live)
    return out.to(s["q"].dtype), lse


def plain_prefix(s):
    c = s["case"]
    H = c["kv_heads"]
    lens, cu, runs = s["lens"].long(), s["cu"].long(), s["prefix_cu"].long()
    # All queries of a prefix's sequences over the prefix.
    first, n = cu[runs[:-1]], cu[runs[1:]] - cu[runs[:-1]]
    q, live = padded(s["q"].float(), first, n, s["max_shared"])
    j = torch.arange(s["max_prefix"], device="cuda")[None].expand(n.shape[0], -1)
    there = j < s["prefix_lens"].long()[:, None]
    k, v = gathered(s["cache"], s["prefix_table"], c["page"], j, there)
    out1, lse1 = unpadded(*attended(grouped(q, H), k, v, there[:, None].expand(-1, s["max_shared"], -1), s["scale"]), live)
    # Each sequence's over its own tokens.
    n = cu[1:] - cu[:-1]
    q, live = padded(s["q"].float(), cu[:-1], n, s["max_new"])
    j = torch.arange(s["max_len"], device="cuda")[None].expand(n.shape[0], -1)
    there = j < lens[:, None]
    k, v = gathered(s["cache"], s["table"], c["page"], j, there)
    at = (lens - n)[:, None] + torch.arange(s["max_new"], device="cuda")
    out2, lse2 = unpadded(*attended(grouped(q, H), k, v, there[:, None] & (j[:, None] <= at[..., None]), s["scale"]), live)
    top = torch.maximum(lse1, lse2)
    a, b = torch.exp(lse1 - top), torch.exp(lse2 - top)
    return ((out1 * a[..., None] + out2 * b[..., None]) / (a + b)[..., None]).to(s["q"].dtype), top + torch.log(a + b)


# ---------------------------------------------------------------------------
# The library's calls
# ---------------------------------------------------------------------------

def own_run(s):
    from paper_2606_07116_gb300 import offq as Q
    c = s["case"]
    if c["kind"] == "prompt":
        return Q.prompt_attention(s["q"], s["k"], s["v"], s["cu"], scale=s["scale"], lse=True, window=c["window"],
                                  sinks=c["sinks"])
    cache = Q.KV4Cache(*s["cache"])
    if c["kind"] == "window":
        return Q.paged_attention(s["q"], cache, s["table"], s["lens"], s["cu"], s["max_new"], scale=s["scale"], lse=True,
                                 window=c["window"], sinks=c["sinks"])
    return Q.paged_attention(s["q"], cache, s["table"], s["lens"], s["cu"], s["max_new"], scale=s["scale"], lse=True,
                             prefix=Q.SharedPrefix(s["prefix_table"], s["prefix_lens"], s["prefix_cu"]))


def run(s):
    if own:
        return own_run(s)
    return {"window": plain_window, "prompt": plain_prompt, "prefix": plain_prefix}[s["case"]["kind"]](s)


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------

def exact_tokens(s, row, count):
    """Keys and values [count, H, D] of the first tokens of a row of page numbers; a token without a page is NaN."""
    kc, kp, vc, vp = s["cache"]
    j = torch.arange(count, device="cuda")
    page, at = row.long()[j // s["case"]["page"]], j % s["case"]["page"]
    gone = (page < 0)[:, None, None]
    both = []
    for codes, par in ((kc, kp), (vc, vp)):
        b = codes[page.clamp(min=0), :, at].long()
        u = torch.empty(*b.shape[:-1], 2 * b.shape[-1], dtype=torch.float64, device="cuda")
        u[..., 0::2] = (b % 16 - 8).double()
        u[..., 1::2] = (b // 16 - 8).double()
        p = par[page.clamp(min=0), :, at].double()
        both.append((u * p[..., 0:1] + p[..., 1:2]).masked_fill(gone, float("nan")))
    return both


def exact_sequence(q, k, v, hidden, scale):
    """q [n, Hq, D] over k, v [L, H, D]; hidden [n, L] (None: nothing is). In pieces of queries; each takes the columns
    that some query of it sees."""
    n, Hq, D = q.shape
    out = torch.empty(n, Hq, D, dtype=torch.float64, device="cuda")
    lse = torch.empty(n, Hq, dtype=torch.float64, device="cuda")
    for a in range(0, n, 2048):
        part = slice(a, a + 2048)
        cols = slice(None) if hidden is None else torch.nonzero(~hidden[part].all(0))[:, 0]
        for h in range(Hq):
            kh, vh = k[cols, h * k.shape[1] // Hq].double(), v[cols, h * k.shape[1] // Hq].double()
            z = q[part, h].double() @ kh.T * scale
            if hidden is not None:
                z = z.masked_fill(hidden[part][:, cols], float("-inf"))
            lse[part, h] = torch.logsumexp(z, 1)
            out[part, h] = torch.softmax(z, 1) @ vh
    return out, lse


def exact(case, seed):
    s = prepare(case, seed)
    if work(case)["flops"] > 3e12:
        return None
    outs, lses, row = [], [], 0
    if case["kind"] == "prefix":
        lengths = new_and_past(case)
        for g, (tokens, first, count) in enumerate(prefix_runs(case)):
            pk, pv = exact_tokens(s, s["prefix_table"][g], tokens)
            own_kv = [exact_tokens(s, s["table"][b], sum(lengths[b])) for b in range(first, first + count)]
            # One row of scores: the prefix, then the tokens of all of its sequences, the others' hidden.
            total = sum(n for n, _ in lengths[first:first + count])
            hidden = torch.ones(total, tokens + sum(k.shape[0] for k, _ in own_kv), dtype=torch.bool, device="cuda")
            hidden[:, :tokens] = False
            i, col = 0, tokens
            for n, past in lengths[first:first + count]:
                for r in range(n):
                    hidden[i + r, col:col + past + r + 1] = False
                i, col = i + n, col + past + n
            k = torch.cat([pk] + [x for x, _ in own_kv])
            v = torch.cat([pv] + [x for _, x in own_kv])
            o, l = exact_sequence(s["q"][row:row + total], k, v, hidden, s["scale"])
            outs.append(o)
            lses.append(l)
            row += total
        return torch.cat(outs), torch.cat(lses)
    W, S = case["window"], case["sinks"]
    lengths = [(n, 0) for n in prompt_lengths(case)] if case["kind"] == "prompt" else new_and_past(case)
    for b, (n, past) in enumerate(lengths):
        if case["kind"] == "prompt":
            k, v = s["k"][row:row + n], s["v"][row:row + n]
        else:
            k, v = exact_tokens(s, s["table"][b], n + past)
        ago = torch.arange(past, past + n, device="cuda")[:, None] - torch.arange(n + past, device="cuda")[None]
        hidden = (ago < 0) | ((ago >= W) & (torch.arange(n + past, device="cuda") >= S)[None])
        o, l = exact_sequence(s["q"][row:row + n], k, v, hidden, s["scale"])
        outs.append(o)
        lses.append(l)
        row += n
    return torch.cat(outs), torch.cat(lses)
