"""Paged attention under a window and behind prefixes in batches that a CTA does not list at once (256 or 512 sequences and
prefixes): each CTA reads the list a second time to find its share. And what stands out of a window's sight. Tolerances in
attention_parity."""

import numpy as np
import pytest
import torch

import oracle.attention_oracle as A
from attention_parity import Pages, check, cumulative, i32, queries
from paper_2606_07116_gb300 import build as B
from paper_2606_07116_gb300 import offq as Q
from test_gpu_attention_prefix import _shared
from test_gpu_attention_window import _paged

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    B.build()
    Q.load_library()


def _ragged(count, most_new, most_past, seed, none=7):
    """New tokens and lengths of `count` sequences, every `none`-th without queries."""
    r = np.random.default_rng(seed)
    news = [0 if b % none == none - 1 else int(r.integers(1, most_new + 1)) for b in range(count)]
    return news, [n + int(r.integers(0, most_past + 1)) for n in news]


@pytest.mark.parametrize("count", [300, 700])
@pytest.mark.parametrize("Hq,H,D,page,dt", [(2, 1, 64, 16, "bf16"), (6, 2, 128, 32, "f16"), (12, 1, 64, 16, "f16")])
def test_single_tokens_under_a_window(count, Hq, H, D, page, dt):
    news, lens = _ragged(count, 1, 150, count + Hq)
    _paged(lens, news, Hq, H, D, page, dt, 40, 4, seed=count)
    _paged(lens, news, Hq, H, D, page, dt, 1000, 0, seed=count)


@pytest.mark.parametrize("count", [300, 700])
@pytest.mark.parametrize("most_new", [12, 44])
def test_several_tokens_under_a_window(count, most_new):
    """In both forms, and (the last) with a single long chunk at the list's end."""
    news, lens = _ragged(count, most_new, 90, count + most_new)
    _paged(lens, news, 4, 2, 64, 16, "bf16", 33, 5, seed=count)
    _paged(lens[:-1] + [500], news[:-1] + [400], 2, 1, 64, 16, "f16", 70, 0, seed=count + 1)


def test_chunks_alone_under_a_window():
    """Batches that take the many-row form alone: all chunks alike in length, or nearly."""
    for count in (300, 600):
        _paged([40 + b % 50 for b in range(count)], [40] * count, 2, 1, 64, 16, "bf16", 50, 3, seed=count)
        _paged([40 + b % 50 for b in range(count)], [40] * (count - 1) + [38], 2, 1, 64, 16, "f16", 30, 0, seed=count + 1)


@pytest.mark.parametrize("count", [300, 600])
def test_rows_of_both_forms_behind_prefixes(count):
    """Prefixes with a row and with hundreds of them, and sequences with few and many of their own."""
    r = np.random.default_rng(count)
    cuts = sorted({0, 2, 3, 40, 41, 200, *(int(x) for x in r.integers(201, count, 60)), count})
    prefix = [int(x) for x in r.integers(0, 90, len(cuts) - 1)]
    for most_new, seed in ((1, 1), (3, 2), (24, 3)):
        news, lens = _ragged(count, most_new, 60, seed, none=11)
        _shared(prefix, cuts, lens, news, 4, 2, 64, 16, "bf16", seed=seed)


def test_long_lists_of_prefixes_ahead_of_chunks():
    """550 prefixes, most without sequences, ahead of 60 sequences of 40 tokens."""
    r = np.random.default_rng(9)
    cu = sorted(int(x) for x in r.integers(0, 61, 549))
    cu = [0] + cu + [60]
    _shared([int(x) for x in r.integers(1, 50, 550)], cu, [40 + b % 30 for b in range(60)], [40] * 60, 2, 1, 64, 16, "bf16", seed=4)


@pytest.mark.parametrize("new", [1, 7, 60])
def test_what_is_out_of_sight_is_not_looked_at(new):
    """Entries that are no pages, and pages of NaN pairs, outside the window and the sinks."""
    L, window, sinks, page = 400, 60, 4, 16
    pages = Pages([np.ones(L, bool)], 2, 128, page, 5)
    qb, q64 = queries(new, 8, 128, "bf16", 6)
    seen = A.in_window(L - new, new, L, window, sinks)
    some = seen.any(0)
    hidden = [i for i in range(L // page) if not some[i * page:(i + 1) * page].any()]
    assert len(hidden) >= 10
    k, k_mag, v, v_mag = pages.tokens(0, L)
    for entry in (-1, 1 << 20, -2 ** 31, 2 ** 31 - 1, int(pages.table[0, hidden[0]])):
        table = pages.table.copy()
        table[0, hidden] = entry
        for p in pages.pairs:
            p[pages.table[0, hidden]] = np.nan
        out, lse = Q.paged_attention(qb.cuda(), pages.cache(), i32(table), i32([L]), i32([0, new]), new, lse=True,
                                     window=window, sinks=sinks)
        assert Q.offq_get_device_status() == Q.OFFQ_OK
        check(out.cpu().double().numpy(), lse.cpu().double().numpy(), q64, k_mag, k, v, v_mag, 128 ** -0.5, seen, "bf16")
