"""Infinities and NaN of keys do not reach queries that do not see them, in the same tile or block or not. Tolerances in
attention_parity."""

import numpy as np
import pytest
import torch

import oracle.attention_oracle as A
from attention_parity import Pages, check, cumulative, i32, queries
from paper_2606_07116_gb300 import build as B
from paper_2606_07116_gb300 import offq as Q

pytestmark = pytest.mark.gpu

BAD = (float("inf"), float("-inf"), float("nan"))


@pytest.fixture(scope="module", autouse=True)
def _lib():
    B.build()
    Q.load_library()


def _seen(n, L, window, sinks):
    """What the last n of L tokens see."""
    return A.in_window(L - n, n, L, L + 1 if window is None else window, sinks)


@pytest.mark.parametrize("window,sinks", [(None, 0), (20, 4), (150, 0)])
@pytest.mark.parametrize("Hq,H,D,dt", [(4, 2, 128, "bf16"), (3, 1, 64, "f16")])
def test_prompts(window, sinks, Hq, H, D, dt):
    lengths, at = [300, 77, 500], [[40, 130, 131, 290], [76], [200, 320]]
    x, x64 = queries(sum(lengths), Hq + 2 * H, D, dt, 3)
    cu, kw = cumulative(lengths), {} if window is None else dict(window=window, sinks=sinks)
    for b, places in enumerate(at):
        for i, j in enumerate(places):
            x[cu[b] + j, Hq:Hq + H] = BAD[i % 3]
    x = x.cuda()
    out, lse = Q.prompt_attention(x[:, :Hq], x[:, Hq:Hq + H], x[:, Hq + H:], i32(cu), lse=True, **kw)
    out, lse = out.cpu().double().numpy(), lse.cpu().double().numpy()
    for b, (n, places) in enumerate(zip(lengths, at)):
        seen = _seen(n, n, window, sinks)
        clean = ~seen[:, places].any(1)
        assert clean.sum() >= 40 or window is None
        rows = np.arange(cu[b], cu[b + 1])
        q, k, v = x64[rows, :Hq], x64[rows, Hq:Hq + H], x64[rows, Hq + H:]
        check(out[rows][clean], lse[rows][clean], q[clean], np.abs(k), k, v, np.abs(v), D ** -0.5, seen[clean], dt)
    assert Q.offq_get_device_status() == Q.OFFQ_OK


@pytest.mark.parametrize("window,sinks", [(None, 0), (20, 4), (150, 0)])
@pytest.mark.parametrize("new", [4, 7, 150])
def test_pages(new, window, sinks):
    """New tokens in the few-row and the many-row form; the bad pairs are of tokens among the new ones and right before."""
    L, D = 400, 128
    pages = Pages([np.ones(L, bool)], 2, D, 16, 7)
    qb, q64 = queries(new, 8, D, "bf16", 8)
    k, k_mag, v, v_mag = pages.tokens(0, L)
    places = [L - 2] if new < 100 else [L - 100, L - 130, L - 3]
    if window == 20 and new == 150:
        places.append(L - 165)
    for i, j in enumerate(places):
        pages.pairs[0][pages.table[0, j // 16], :, j % 16] = BAD[i % 3]
    kw = {} if window is None else dict(window=window, sinks=sinks)
    out, lse = Q.paged_attention(qb.cuda(), pages.cache(), i32(pages.table), i32([L]), i32([0, new]), new, lse=True, **kw)
    out, lse = out.cpu().double().numpy(), lse.cpu().double().numpy()
    seen = _seen(new, L, window, sinks)
    clean = ~seen[:, places].any(1)
    assert clean.sum() >= 2
    check(out[clean], lse[clean], q64[clean], k_mag, k, v, v_mag, D ** -0.5, seen[clean], "bf16")
    assert Q.offq_get_device_status() == Q.OFFQ_OK
