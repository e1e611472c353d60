"""Paged attention where the values' scales differ by many powers of two: what a key adds to an output is its weight
times its value, so a large value that a row does not see, or hardly weighs, may cost the others nothing.

Tolerances, from the arithmetic (u = 2^-24):
* Scores as in test_gpu_attention, with the bias of the codes in their magnitudes (they enter as 16 + u, and 24 times the
  query's sum leaves again). They are taken relative to a reference that holds the base 2 logarithm of a scale, at most
  128 in magnitude: 4 u of that and of the score's magnitudes.
* Exponentials and the rescaling where a reference moves: 2^-18 for all of them. Sums over L keys: 2 L u. Numerator and
  denominator: twice that, of sum_j w_j |v_j|.
* A weight times its value's scale is rounded to a half: 2^-11 of itself, and 2^-25 where it is below the smallest normal
  half, in units in which the largest of the row's visible keys is at least 1. Once with few rows; with many a block's
  weights may be rounded again for each of its three later groups of 32 keys. Each meets a code of at most 7.
* out is rounded once to its type."""

import math

import numpy as np
import pytest
import torch

import oracle.attention_oracle as A
from paper_2606_07116_gb300 import build as B
from paper_2606_07116_gb300 import offq as Q
from parity import U32

pytestmark = pytest.mark.gpu

DT = {"bf16": (torch.bfloat16, 2.0 ** -8, 0.0), "f16": (torch.float16, 2.0 ** -11, 2.0 ** -24)}
L, H, PAGE = 300, 2, 32


@pytest.fixture(scope="module", autouse=True)
def _lib():
    B.build()
    Q.load_library()


def check_paged(out, lse, q, keys, values, scale, dt, rounds):
    """The rows of one sequence, its last tokens, against the oracle. keys, values: as A.cached gives them; rounds: how
    often a weight is rounded."""
    _, unit, least = DT[dt]
    (k, kq, ks, ko), (v, vq, vs, vo) = keys, values
    n, Hq, D = q.shape
    tokens, G = k.shape[0], Hq // k.shape[1]
    sees = np.array([tokens - n + i + 1 for i in range(n)])
    ref, ref_lse, w = A.attention(q, k, v, scale, sees)
    if n == 0:
        return
    empty = np.isinf(ref_lse)
    assert np.array_equal(empty, np.isinf(lse)) and np.all(lse[empty] < 0) and np.all(out[empty] == 0)
    if tokens == 0:
        return
    k_mag = (np.abs(kq) + 24) * ks[..., None] + np.abs(ko)[..., None]
    for h in range(Hq):
        g = h // G
        mags = np.where(np.arange(tokens) < sees[:, None], np.abs(q[:, h]) @ k_mag[:, g].T * scale, 0).max(-1)
        dz = (2 * D + 8) * U32 * mags + 4 * U32 * (mags + 128)
        coded = w[:, h] @ (np.abs(vq[:, g]) * vs[:, g, None])
        spread = coded + w[:, h] @ np.broadcast_to(np.abs(vo[:, g, None]), vq[:, g].shape)
        top = (w[:, h] * vs[:, g]).max(-1)
        tol = (2 * (dz + 2.0 ** -18 + 2 * tokens * U32)[:, None] * spread + rounds * 2.0 ** -11 * coded
               + (rounds * 7 * tokens * 2.0 ** -25 * top)[:, None] + unit * np.abs(ref[:, h]) + least)
        assert np.all(np.isfinite(out[:, h]))
        worst = np.max(np.abs(out[:, h] - ref[:, h]) / (tol + 1e-300))
        assert worst <= 1, (h, worst)
        seen = ~empty[:, h]
        assert np.all(np.abs(lse[seen, h] - ref_lse[seen, h]) <=
                      (dz + 2.0 ** -18 + 2 * tokens * U32)[seen] + 2 * U32 * np.abs(ref_lse[seen, h]))


def _run(scales, n, Hq, D, dt, unlikely=(), seed=0):
    """n new tokens at the end of L cached ones whose values have these scales (and offsets of a fifth of them, or 0.2
    where the scale is 0); the keys at `unlikely` have scores far below the others'."""
    rng = np.random.default_rng(seed)
    kind = DT[dt][0]
    pages = -(-L // PAGE)
    codes = [rng.integers(0, 256, (pages, H, PAGE, D // 2), dtype=np.uint8) for _ in range(2)]
    for c in codes:  # nibbles 1..15, as the quantizer leaves them
        c[(c & 15) == 0] |= 1
        c[(c >> 4) == 0] |= 16
    at = np.arange(L)
    pairs = np.full((2, pages, H, PAGE, 2), np.nan, np.float32)
    ks, ko = 0.05 * np.exp(0.3 * rng.standard_normal((L, H))), 0.1 * rng.standard_normal((L, H))
    ko[list(unlikely)] = -6.0
    vs = scales[:, None] * np.exp(0.2 * rng.standard_normal((L, H)))
    vo = np.where(vs > 0, 0.2 * vs, 0.2) * rng.choice([-1.0, 1.0], (L, H))
    pairs[0, at // PAGE, :, at % PAGE] = np.stack([ks, ko], -1)
    pairs[1, at // PAGE, :, at % PAGE] = np.stack([vs, vo], -1)
    q = torch.from_numpy(1 + 0.3 * rng.standard_normal((n, Hq, D))).to(kind)
    cache = Q.KV4Cache(*(torch.from_numpy(x).cuda() for x in (codes[0], pairs[0], codes[1], pairs[1])))
    i32 = dict(dtype=torch.int32, device="cuda")
    out, lse = Q.paged_attention(q.cuda(), cache, torch.arange(pages, **i32)[None], torch.tensor([L], **i32),
                                 torch.tensor([0, n], **i32), n, lse=True)
    assert Q.offq_get_device_status() == Q.OFFQ_OK
    out, lse, q = out.cpu().double().numpy(), lse.cpu().double().numpy(), q.double().numpy()
    held = [A.cached(c, p, at // PAGE, at % PAGE) for c, p in zip(codes, pairs)]
    check_paged(out, lse, q, *held, D ** -0.5, dt, 1 if n * Hq // H <= 16 else 4)


FORMS = [(1, 2, 128, "bf16"), (1, 16, 64, "bf16"), (4, 8, 128, "bf16"), (7, 4, 64, "f16"),       # few rows
         (17, 2, 128, "bf16"), (40, 8, 128, "bf16"), (40, 4, 64, "f16"), (220, 4, 128, "bf16")]  # many


def _powers(lo, hi, dt):
    """Exponents between lo and hi, in halves less above so that the outputs stay in range."""
    return (lo, min(hi, 8)) if dt == "f16" else (lo, hi)


@pytest.mark.parametrize("n,Hq,D,dt", FORMS)
def test_a_large_value_that_most_rows_do_not_see(n, Hq, D, dt):
    lo, hi = _powers(-15, 15, dt)
    scales = np.full(L, 2.0 ** lo)
    scales[-1] = 2.0 ** hi
    _run(scales, n, Hq, D, dt, seed=1)


@pytest.mark.parametrize("n,Hq,D,dt", FORMS)
def test_large_values_of_hardly_any_weight(n, Hq, D, dt):
    lo, hi = _powers(-15, 15, dt)
    scales = np.full(L, 2.0 ** lo)
    big = [5, 70, 131, 200]
    scales[big] = 2.0 ** hi
    _run(scales, n, Hq, D, dt, unlikely=big, seed=2)


@pytest.mark.parametrize("n,Hq,D,dt", FORMS)
def test_mixed_rising_and_falling_scales(n, Hq, D, dt):
    lo, hi = _powers(-15, 15, dt)
    for i, e in enumerate((np.random.default_rng(3).uniform(lo, hi, L), np.linspace(lo, hi, L), np.linspace(hi, lo, L))):
        _run(2.0 ** e, n, Hq, D, dt, seed=3 + i)


@pytest.mark.parametrize("n,Hq,D,dt", FORMS)
def test_scales_of_zero(n, Hq, D, dt):
    """Values that are their offset alone: all of them, a first block of them, every other one."""
    for i, some in enumerate((np.ones(L, bool), np.arange(L) < 140, np.arange(L) % 2 == 0)):
        _run(np.where(some, 0.0, 0.5), n, Hq, D, dt, seed=6 + i)


@pytest.mark.parametrize("n,Hq,D", [(n, Hq, D) for n, Hq, D, dt in FORMS if dt == "bf16"])
@pytest.mark.parametrize("lo,hi", [(-45, -45), (-60, -60), (-55, -30), (70, 70), (60, 100), (-60, 100)])
def test_tiny_and_huge_scales(n, Hq, D, lo, hi):
    _run(2.0 ** np.random.default_rng(9).uniform(lo, hi, L), n, Hq, D, "bf16", seed=9)
