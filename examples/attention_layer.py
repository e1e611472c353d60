"""An attention layer on W4A4 linears and the paged 4-bit cache: prompts, chunks of new tokens and single tokens.

    python examples/attention_layer.py            # 4 prompts, a chunk each, then single tokens; prints the times

The layer's two linears (queries, keys and values in one; output) are offq's W4A4 linears. Between them:
* a prompt's queries and keys take norm, rotary positions (rope_heads) and attend in 16 bits (prompt_attention), while
  its keys and values go into the cache (kv4_paged_write);
* new tokens after that, a chunk or one per sequence, write the cache and get their queries ready in one launch
  (kv4_paged_write), then attend over the pages (paged_attention);
* kv4_paged_read gives cached tokens back, here to check a step against softmax(q K^T) V in float64.
"""

from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2606_07116_gb300 import offq as Q  # noqa: E402


class Linear:
    """y = x W^T with 4-bit weights and activations; blocks of g channels share a rotation and an offset."""

    def __init__(self, w: torch.Tensor, g: int):
        self.g, self.weight = g, Q.prepare_weight(w, g)

    def __call__(self, x: torch.Tensor) -> torch.Tensor:
        return Q.w4a4_linear(*Q.quantize_act(x, self.g), *self.weight, self.g)


class Pages:
    """The pages of up to B sequences: a free list here, the table and the lengths on the device."""

    def __init__(self, pages: int, B: int, width: int, page_size: int):
        self.free, self.used, self.page_size = list(range(pages))[::-1], [0] * B, page_size
        self.table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
        self.lens = torch.zeros(B, dtype=torch.int32, device="cuda")

    def reserve(self, tokens) -> None:
        """Pages so that sequence b can hold tokens[b]."""
        for b, n in enumerate(tokens):
            need = -(-n // self.page_size)
            if need > self.table.shape[1] or need - self.used[b] > len(self.free):
                raise RuntimeError("the cache is full")
            if need > self.used[b]:
                new = [self.free.pop() for _ in range(need - self.used[b])]
                self.table[b, self.used[b]:need] = torch.tensor(new, dtype=torch.int32, device="cuda")
                self.used[b] = need

    def slots(self, seq: torch.Tensor, positions: torch.Tensor) -> torch.Tensor:
        """Slots of the tokens at `positions` of the sequences `seq`."""
        pos = positions.long()
        return self.table[seq, pos // self.page_size].long() * self.page_size + pos % self.page_size


class AttentionLayer:
    def __init__(self, hidden: int, Hq: int, H: int, D: int, max_len: int, g: int = 1024, pages: int = 256, B: int = 4,
                 page_size: int = 64, dtype: torch.dtype = torch.bfloat16, seed: int = 0):
        gen = torch.Generator("cuda").manual_seed(seed)
        def weight(n, k):
            return (torch.randn(n, k, generator=gen, device="cuda") * k ** -0.5).to(dtype)
        self.Hq, self.H, self.D = Hq, H, D
        self.qkv = Linear(weight((Hq + 2 * H) * D, hidden), g)
        self.out = Linear(weight(hidden, Hq * D), g)
        self.q_norm = torch.ones(Hq, D, device="cuda")
        self.k_norm = torch.ones(H, D, device="cuda")
        self.rope = Q.rope_table(max_len, D)
        self.cache = Q.kv4_cache(pages, H, D, page_size)
        self.pages = Pages(pages, B, -(-max_len // page_size), page_size)

    def heads(self, x: torch.Tensor):
        """Queries, keys and values [T, heads, D]: parts of one linear's rows, used where they lie."""
        y = self.qkv(x).view(x.shape[0], self.Hq + 2 * self.H, self.D)
        return y[:, :self.Hq], y[:, self.Hq:self.Hq + self.H], y[:, self.Hq + self.H:]

    def prompt(self, x: torch.Tensor, lengths) -> torch.Tensor:
        """Whole prompts, packed: x [sum(lengths), hidden]. Fills empty sequences 0 .. len(lengths) - 1."""
        q, k, v = self.heads(x)
        self.pages.reserve(lengths)
        n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        pos = torch.cat([torch.arange(i, dtype=torch.int32, device="cuda") for i in lengths])
        seq = torch.repeat_interleave(torch.arange(len(lengths), device="cuda"), n.long())
        Q.kv4_paged_write(self.cache, k, v, self.pages.slots(seq, pos), pos, self.rope, k_norm=self.k_norm)
        q = Q.rope_heads(q, pos, self.rope, self.q_norm)
        k = Q.rope_heads(k, pos, self.rope, self.k_norm)
        cu = torch.nn.functional.pad(n.cumsum(0), (1, 0)).int()
        self.pages.lens[:len(lengths)] = n
        return self.out(Q.prompt_attention(q, k, v, cu).flatten(1))

    def extend(self, x: torch.Tensor, n: int, attention=Q.paged_attention) -> torch.Tensor:
        """n more tokens for every sequence, x [B n, hidden]; their pages are reserved. Nothing here waits for the
        device or depends on a length, so a graph that captured it stays right as the sequences grow."""
        B, dev = self.pages.lens.shape[0], x.device
        q, k, v = self.heads(x)
        seq = torch.arange(B * n, device=dev) // n
        pos = (self.pages.lens[:, None] + torch.arange(n, dtype=torch.int32, device=dev)).flatten()
        q = Q.kv4_paged_write(self.cache, k, v, self.pages.slots(seq, pos), pos, self.rope, q, self.q_norm, self.k_norm)
        self.pages.lens += n
        cu = torch.arange(0, B * n + 1, n, dtype=torch.int32, device=dev)
        return self.out(attention(q, self.cache, self.pages.table, self.pages.lens, cu, n).flatten(1))

    def attention64(self, q, cache, table, lens, cu, n):
        """What paged_attention computes, from the tokens that kv4_paged_read gives back. The queries hold H3, so the
        keys keep theirs."""
        out = torch.empty(q.shape, dtype=torch.float64, device=q.device)
        for b, L in enumerate(lens.tolist()):
            at = torch.arange(L, device=q.device)
            k, v = Q.kv4_paged_read(cache, self.pages.slots(torch.full_like(at, b), at), rotate=False,
                                    out_dtype=torch.float32)
            k, v = (t.double().repeat_interleave(self.Hq // self.H, 1) for t in (k, v))
            s = torch.einsum("ihd,jhd->hij", q[cu[b]:cu[b + 1]].double(), k) * self.D ** -0.5
            seen = at[None] <= L - n + torch.arange(n, device=q.device)[:, None]
            out[cu[b]:cu[b + 1]] = torch.einsum("hij,jhd->ihd", s.masked_fill(~seen, float("-inf")).softmax(-1), v)
        return out


def main() -> None:
    hidden, lengths, chunk, tokens = 4096, [1500, 700, 2048, 33], 40, 64
    layer = AttentionLayer(hidden, 32, 8, 128, max_len=4096, B=len(lengths))
    gen = torch.Generator("cuda").manual_seed(1)

    def rows(n):
        return torch.randn(n, hidden, generator=gen, device="cuda").to(torch.bfloat16)

    def timed(name, f, n):
        f()
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        for _ in range(n):
            f()
        b.record()
        b.synchronize()
        print(f"{name}: {a.elapsed_time(b) * 1e3 / n:.1f} us")

    def compared(q, *args):
        out, ref = Q.paged_attention(q, *args), layer.attention64(q, *args)
        print(f"largest difference from float64 attention over the same cache: {(out - ref).abs().max():.1e} "
              f"(largest value {ref.abs().max():.2f})")
        return out

    x = rows(sum(lengths))
    timed(f"prompts of {lengths} tokens", lambda: layer.prompt(x, lengths), 10)

    layer.pages.reserve([n + chunk + tokens + 2 for n in lengths])
    x = rows(len(lengths) * chunk)

    def more():
        layer.pages.lens.copy_(past)
        layer.extend(x, chunk)
    past = layer.pages.lens.clone()
    timed(f"{chunk} more tokens each", more, 10)

    x = rows(len(lengths))
    layer.extend(x, 1, compared)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = layer.extend(x, 1)

    def decode():
        graph.replay()
        x.copy_(y)
    timed("one token each, from a graph", decode, tokens)
    if Q.offq_get_device_status() != Q.OFFQ_OK:
        raise SystemExit("a kernel reported an error")
    print("lengths now", layer.pages.lens.tolist())


if __name__ == "__main__":
    main()
