"""Attention with any mask against the float64 oracle, and pages to run it on.

Tolerances, from the arithmetic (u = 2^-24; e = 2^-8 for bf16, 2^-11 for f16, the unit roundoff):
* A score sums D exact products in fp32. Allowing each addition a whole ulp (tensor cores may truncate) it is
  within 2 D u of its sum of magnitudes; scale, offset and softmax scale add at most 8 u. dz is the largest such
  bound over the keys that a row sees.
* A weight then carries dz, 2^-20 of the exponential (twice where two parts of a row are joined), and e where it is
  rounded to the 16-bit type that the product with the values takes; sums over L keys in fp32 add 2 L u. Numerator
  and denominator: twice that. out moves by that relative bound times sum_j w_j |v_j|, and is rounded once (e |out|;
  half the smallest step of f16, 2^-25, where it is subnormal).
* lse moves by dz + 2^-20 (twice where joined) + 2 L u and its own rounding, 2 u |lse|."""

import numpy as np
import torch

import oracle.attention_oracle as A
from paper_2606_07116_gb300 import offq as Q
from parity import U32

DT = {"bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def check(out, lse, q, k_mag, k, v, v_mag, scale, seen, dt, joined=False):
    """One sequence's rows against the oracle; k_mag and v_mag bound the magnitudes that a cached value is summed from."""
    D, L, e = q.shape[-1], k.shape[0], UNIT[dt]
    ref, ref_lse, w = A.attention_masked(q, k, v, scale, seen)
    G = q.shape[1] // k.shape[1]
    ex = 2.0 ** (-19 if joined else -20)
    if L:
        mags = np.stack([np.abs(q[:, h]) @ k_mag[:, h // G].T for h in range(q.shape[1])], 1) * scale
        dz = (2 * D + 8) * U32 * np.where(seen[:, None], mags, 0).max(-1)
        spread = np.stack([w[:, h] @ v_mag[:, h // G] for h in range(q.shape[1])], 1)
    else:
        dz, spread = np.zeros(ref_lse.shape), np.zeros(ref.shape)
    rel = 2 * (dz + ex + e + 2 * L * U32)
    tol = rel[..., None] * spread + e * np.abs(ref) + (2.0 ** -25 if dt == "f16" else 0)
    assert np.all(np.isfinite(out))
    worst = np.max(np.abs(out - ref) / (tol + 1e-300)) if out.size else 0
    assert worst <= 1, worst
    empty = np.isinf(ref_lse)
    assert np.array_equal(empty, np.isinf(lse)) and np.all(lse[empty] < 0) and np.all(out[empty] == 0)
    tol = dz + ex + 2 * L * U32 + 2 * U32 * np.abs(np.where(empty, 0, ref_lse))
    assert np.all(np.abs(np.where(empty, 0, lse) - np.where(empty, 0, ref_lse)) <= tol)


class Pages:
    """Rows of pages: `runs` is a list of bool arrays, which tokens of a row some query sees. Pages without such a token
    have entry -1, slots without one hold NaN pairs; the others a random code and pair."""

    def __init__(self, runs, H, D, page, seed, k_off=6.0, table_pad=1):
        rng = np.random.default_rng(seed)
        held = [[i for i in range(-(-len(r) // page)) if r[i * page:(i + 1) * page].any()] for r in runs]
        total = sum(map(len, held)) + 2
        self.table = np.full((len(runs), max([-(-len(r) // page) for r in runs] + [0]) + table_pad), -1, np.int32)
        order = rng.permutation(total)
        used = np.zeros((total, page), bool)
        at = 0
        for b, (r, h) in enumerate(zip(runs, held)):
            for i in h:
                self.table[b, i] = order[at]
                at += 1
                part = r[i * page:(i + 1) * page]
                used[self.table[b, i], :len(part)] = part
        self.codes = [rng.integers(0, 256, (total, H, page, D // 2), dtype=np.uint8) for _ in range(2)]
        for c in self.codes:  # nibbles 1..15, as the quantizer leaves them
            c[(c & 15) == 0] |= 1
            c[(c >> 4) == 0] |= 16
        self.pairs = [np.stack([0.3 * np.exp(0.3 * rng.standard_normal((total, H, page))),
                                o * (1 + 0.2 * rng.standard_normal((total, H, page)))], -1).astype(np.float32)
                      for o in (k_off, 0.2)]
        self.pairs = [np.where(used[:, None, :, None], p, np.float32("nan")) for p in self.pairs]
        self.page = page

    def cache(self):
        return Q.KV4Cache(*(torch.from_numpy(x).cuda() for x in (self.codes[0], self.pairs[0], self.codes[1], self.pairs[1])))

    def tokens(self, b, count):
        """Keys, their magnitudes, values, theirs: [count, H, D] of row b; zeros where no token is."""
        j = np.arange(count)
        pages = self.table[b][j // self.page] if count else j
        out = []
        for c, p in zip(self.codes, self.pairs):
            x, qc, s, o = A.cached(c, p, np.maximum(pages, 0), j % self.page)
            gone = (pages < 0)[:, None] | np.isnan(s)
            out += [np.where(gone[..., None], 0, x), np.where(gone[..., None], 0, np.abs(qc) * s[..., None] + np.abs(o)[..., None])]
        return out


def queries(T, Hq, D, dt, seed, pad=0):
    """[T, Hq, D] on the host, with room for other heads between tokens; its values in 64 bits."""
    x = torch.from_numpy(np.random.default_rng(seed).standard_normal((T, Hq + pad, D))).to(DT[dt])
    return x, x[:, :Hq].double().numpy()


def cumulative(n):
    return np.concatenate([[0], np.cumsum(n)]).astype(np.int32)


def i32(x):
    return torch.as_tensor(np.asarray(x, np.int32)).cuda()
