"""Attention of sequences behind shared prefixes (paged_attention with prefix=) against the float64 oracle; tolerances
in attention_parity."""

import numpy as np
import pytest
import torch

from attention_parity import Pages, check, cumulative, i32, queries
from paper_2606_07116_gb300 import build as B
from paper_2606_07116_gb300 import offq as Q

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    B.build()
    Q.load_library()


def _call(pages, P, q, lens, cu, max_q, prefix_lens, cu_prefix, **kw):
    prefix = Q.SharedPrefix(i32(pages.table[:P]), i32(prefix_lens), i32(cu_prefix))
    return Q.paged_attention(q, pages.cache(), i32(pages.table[P:]), i32(lens), i32(cu), max_q, prefix=prefix, **kw)


def _check_all(out, lse, pages, P, q64, lens, cu, prefix_lens, cu_prefix, scale, dt):
    out, lse = out.cpu().double().numpy(), lse.cpu().double().numpy()
    for b, L in enumerate(lens):
        g = [g for g in range(P) if cu_prefix[g] <= b < cu_prefix[g + 1]]
        before = prefix_lens[g[0]] if g else 0
        parts = [pages.tokens(g[0] if g else 0, before), pages.tokens(P + b, L)]
        k, k_mag, v, v_mag = (np.concatenate(x) for x in zip(*parts))
        n = cu[b + 1] - cu[b]
        seen = np.arange(before + L)[None] <= before + L - n + np.arange(n)[:, None]
        seen[:, :before] = True
        rows = slice(cu[b], cu[b + 1])
        check(out[rows], lse[rows], q64[rows], k_mag, k, v, v_mag, scale, seen, dt, joined=True)


def _shared(prefix_lens, cu_prefix, lens, news, Hq, H, D, page, dt, seed=0, q_pad=0, table_pad=1, k_off=6.0, scale=None,
            max_q=None):
    P, cu, scale = len(prefix_lens), cumulative(news), scale or D ** -0.5
    pages = Pages([np.ones(L, bool) for L in list(prefix_lens) + list(lens)], H, D, page, seed, k_off, table_pad)
    qb, q64 = queries(sum(news), Hq, D, dt, seed + 1, q_pad)
    out, lse = _call(pages, P, qb.cuda()[:, :Hq], lens, cu, max_q or max(news), prefix_lens, cu_prefix, scale=scale, lse=True)
    assert Q.offq_get_device_status() == Q.OFFQ_OK
    _check_all(out, lse, pages, P, q64, lens, cu, prefix_lens, cu_prefix, scale, dt)


HEADS = [(8, 2, 128, 64, "bf16"), (5, 1, 64, 16, "f16"), (4, 4, 128, 32, "f16"), (16, 1, 64, 256, "bf16"), (24, 2, 128, 16, "bf16")]


@pytest.mark.parametrize("Hq,H,D,page,dt", HEADS)
@pytest.mark.parametrize("prefix", [1, 31, 32, 33, 127, 128, 129, 500])
def test_one_prefix_single_tokens(prefix, Hq, H, D, page, dt):
    _shared([prefix], [0, 2], [1, 40], [1, 1], Hq, H, D, page, dt, seed=prefix)
    _shared([prefix], [0, 9], [1, 2, 15, 16, 17, 33, 100, 257, 600], [1] * 9, Hq, H, D, page, dt, seed=prefix + 1)


@pytest.mark.parametrize("Hq,H,D,page,dt", HEADS)
@pytest.mark.parametrize("news", [[2, 1, 3, 1, 4], [4] * 5, [7, 8, 5, 1, 6], [1, 17, 9, 2, 1], [33, 5, 1, 64, 1], [150, 40, 1, 1, 129]])
def test_several_prefixes_and_new_tokens(news, Hq, H, D, page, dt):
    lens = [n + past for n, past in zip(news, (77, 0, 300, 5, 130))]
    _shared([130, 1, 700], [0, 2, 3, 5], lens, news, Hq, H, D, page, dt, seed=sum(news))
    _shared([300], [0, 5], lens, news, Hq, H, D, page, dt, seed=sum(news) + 1)


def test_groups_of_every_row_count_around_the_forms():
    """Rows of a prefix per key head from 1 to past two tiles, with single tokens."""
    for B in (1, 2, 3, 4, 5, 8, 15, 16, 17, 31, 32, 33, 63, 64, 65, 96):
        _shared([200], [0, B], [3 + 7 * (b % 5) for b in range(B)], [1] * B, 8, 2, 64, 16, "bf16", seed=B)


def test_a_long_prefix():
    _shared([5000], [0, 3], [70, 1, 500], [1, 1, 1], 8, 2, 128, 64, "bf16", seed=1)
    _shared([4097], [0, 40], [10 + b for b in range(40)], [1] * 40, 8, 2, 128, 16, "f16", seed=2)
    _shared([3001, 2000], [0, 2, 3], [300, 41, 7], [280, 41, 7], 4, 1, 128, 64, "bf16", seed=3)


def test_empty_prefixes_and_sequences():
    """Prefixes of no tokens, of no sequences; sequences before, between and behind the prefixes', without tokens of their own,
    with more queries than tokens, without queries."""
    for new in (1, 2, 40):
        news = [new, new, 0, new, 1, new, new]
        lens = [30, 0, 50, new // 2, 0, 7, 90]
        _shared([0, 100, 64], [1, 2, 2, 5], lens, news, 8, 2, 128, 16, "bf16", seed=new)
        _shared([33, 0, 64, 1], [0, 1, 4, 4, 7], lens, news, 6, 2, 64, 32, "f16", seed=new + 1)
        _shared([40], [7, 7], lens, news, 6, 2, 64, 32, "f16", seed=new + 2)


def test_strided_queries_wide_tables_large_scores():
    _shared([400], [0, 2], [50, 700], [1, 1], 8, 2, 128, 16, "bf16", seed=7, q_pad=3, table_pad=40)
    _shared([400], [0, 2], [50, 700], [20, 300], 8, 2, 64, 16, "f16", seed=8, q_pad=5, table_pad=9)
    _shared([600], [0, 2], [330, 20], [100, 3], 8, 2, 128, 64, "bf16", seed=10, k_off=60.0)
    _shared([600], [0, 2], [400, 20], [200, 4], 8, 2, 128, 64, "f16", seed=12, scale=3.0)


def test_many_sequences_and_prefixes():
    """More of both than a warp, and than a block, looks at in one go."""
    B = 700
    r = np.random.default_rng(5)
    cuts = np.sort(r.integers(0, B + 1, 299))
    cu = [int(x) for x in [0, *cuts, B]]
    _shared([int(x) for x in r.integers(0, 60, 300)], cu, [int(x) for x in r.integers(1, 50, B)], [1] * B, 2, 1, 64, 16, "bf16", seed=6)


@pytest.mark.parametrize("new", [1, 50])
def test_a_shared_prefix_is_a_prefix_of_each(new):
    """The same tokens as whole pages of every sequence's own table."""
    page, before, lens = 32, 320, [60, 200, 51]
    pages = Pages([np.ones(L, bool) for L in [before] + lens], 2, 128, page, 3)
    qb, _ = queries(3 * new, 8, 128, "bf16", 4)
    cu = cumulative([new] * 3)
    out, lse = _call(pages, 1, qb.cuda(), lens, cu, new, [before], [0, 3], lse=True)
    whole = np.concatenate([np.repeat(pages.table[:1, :before // page], 3, 0), pages.table[1:]], 1)
    ref, ref_lse = Q.paged_attention(qb.cuda(), pages.cache(), i32(whole), i32([before + L for L in lens]), i32(cu), new, lse=True)
    # both: outputs as bf16 (half a step), weights as halves
    torch.testing.assert_close(out.float(), ref.float(), rtol=2.0 ** -7, atol=2.0 ** -8)
    torch.testing.assert_close(lse, ref_lse, rtol=2.0 ** -18, atol=2.0 ** -16)


def test_no_prefixes_is_plain_attention():
    pages = Pages([np.ones(L, bool) for L in (50, 70)], 2, 128, 16, 3)
    qb, _ = queries(2, 8, 128, "bf16", 4)
    none = Q.SharedPrefix(torch.empty((0, 3), dtype=torch.int32, device="cuda"), i32([]), i32([0]))
    args = (qb.cuda(), pages.cache(), i32(pages.table), i32([50, 70]), i32([0, 1, 2]), 1)
    assert torch.equal(Q.paged_attention(*args), Q.paged_attention(*args, prefix=none))


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("cu_prefix,prefix_lens", [([0, 2, 9], [100, 80]), ([0, 2, 1], [100, 80]), ([-1, 2, 2], [100, 80]),
                                                   ([0, 2, 4], [100, -5]), ([0, 2, 4], [100, 1 << 30])])
def test_prefixes_out_of_range_are_reported(cu_prefix, prefix_lens, new):
    """They are left out of their sequences' attention (a length past the table is cut there); the others' rows are right."""
    lens = [50 + new, 20 + new, new, new]
    pages = Pages([np.ones(L, bool) for L in [100, 80] + lens], 2, 128, 16, 3, table_pad=0)
    qb, q64 = queries(4 * new, 8, 128, "bf16", 4)
    cu = cumulative([new] * 4)
    table = pages.table.copy()
    table[1, 5:] = 0  # a length past the table meets pages of something
    pages.table[:] = table
    out, lse = _call(pages, 2, qb.cuda(), lens, cu, new, prefix_lens, cu_prefix, lse=True)
    assert Q.offq_get_device_status() == Q.OFFQ_ERR_INVALID_ARG
    good = [b for b in range(4) if any(0 <= cu_prefix[g] <= b < cu_prefix[g + 1] <= 4 and prefix_lens[g] == (100, 80)[g]
                                       for g in range(2))]
    for b in good:
        rows = slice(cu[b], cu[b + 1])
        _check_all(out[rows], lse[rows], _Row(pages, b), 1, q64[rows], lens[b:b + 1], [0, new], [100], [0, 1], 128 ** -0.5, "bf16")


class _Row:
    """The first prefix and one sequence of pages of two prefixes."""
    def __init__(self, pages, b):
        self.tokens = lambda i, count: pages.tokens(0 if i == 0 else 2 + b, count)


def test_a_sequence_with_too_many_queries_takes_its_prefix_along():
    """More queries than max_q: that sequence's rows stay, and where the prefix's count passes B * max_q so do the others'
    sums over it."""
    pages = Pages([np.ones(L, bool) for L in (64, 40, 40)], 2, 128, 16, 3)
    qb, _ = queries(30, 8, 128, "bf16", 4)
    out = torch.full((30, 8, 128), 5.0, dtype=torch.bfloat16, device="cuda")
    _call(pages, 1, qb.cuda(), [40, 40], [0, 1, 29], 1, [64], [0, 2], out=out)
    assert Q.offq_get_device_status() == Q.OFFQ_ERR_INVALID_ARG
    assert torch.all(out[1:] == 5.0) and not torch.any(out[:1] == 5.0)
    own = Q.paged_attention(qb.cuda()[:1], pages.cache(), i32(pages.table[1:2]), i32([40]), i32([0, 1]), 1)
    torch.testing.assert_close(out[:1], own, rtol=2.0 ** -7, atol=2.0 ** -8)


def test_rows_outside_the_sequences_are_left_alone():
    pages = Pages([np.ones(L, bool) for L in (70, 90, 60)], 2, 128, 16, 7)
    qb, _ = queries(60, 8, 128, "bf16", 8)
    for cu, m in (([3, 4, 6], 2), ([3, 43, 50], 40)):
        out = torch.full((60, 8, 128), 5.0, dtype=torch.bfloat16, device="cuda")
        _call(pages, 1, qb.cuda(), [90, 60], cu, m, [70], [0, 2], out=out)
        assert torch.all(out[:3] == 5.0) and torch.all(out[cu[2]:] == 5.0) and not torch.any(out[3:cu[2]] == 5.0)
    assert Q.offq_get_device_status() == Q.OFFQ_OK


def test_another_stream_and_a_graph():
    """Captured on a stream of its own, replayed over other queries, lengths and prefixes, while the same call runs eagerly
    with its own workspace."""
    Hq, H, D, page = 8, 2, 128, 16
    pages = Pages([np.ones(L, bool) for L in (300, 150, 90, 200, 33)], H, D, page, 15)
    cache, cu = pages.cache(), i32([0, 1, 2, 3])
    table, prefix = i32(pages.table[2:]), Q.SharedPrefix(i32(pages.table[:2]), i32([300, 150]), i32([0, 2, 3]))
    x, n = torch.zeros((3, Hq, D), dtype=torch.bfloat16, device="cuda"), i32([90, 200, 33])

    def call():
        return Q.paged_attention(x, cache, table, n, cu, 1, prefix=prefix)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call()
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            out = call()
    torch.cuda.current_stream().wait_stream(s)
    for step, (lens, own, runs) in enumerate((([300, 150], [90, 200, 33], [0, 2, 3]), ([10, 150], [1, 100, 30], [0, 1, 3]))):
        x.normal_(generator=torch.Generator(device="cuda").manual_seed(step))
        n.copy_(i32(own))
        prefix.lens.copy_(i32(lens))
        prefix.cu.copy_(i32(runs))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, call())
    assert Q.offq_get_device_status() == Q.OFFQ_OK


def test_calls_on_two_streams_at_once():
    """Behind prefixes and under a window, single tokens and chunks, side by side on two streams: each call has a workspace of
    its own, and gives what it gives alone."""
    pages = Pages([np.ones(L, bool) for L in (900, 400, 700, 333)], 2, 128, 16, 31)
    cache, prefix = pages.cache(), Q.SharedPrefix(i32(pages.table[:1]), i32([900]), i32([0, 3]))
    table, lens = i32(pages.table[1:]), i32([400, 700, 333])
    streams = [torch.cuda.Stream() for _ in range(2)]
    calls = []
    for new in (1, 50):
        q = queries(3 * new, 8, 128, "bf16", 32 + new)[0].cuda()
        args = (q, cache, table, lens, i32(cumulative([new] * 3)), new)
        calls += [(args, dict(prefix=prefix)), (args, dict(window=200, sinks=4))]
    alone = [Q.paged_attention(*args, **kw) for args, kw in calls]
    torch.cuda.synchronize()
    got = []
    for _ in range(20):
        for i in range(len(calls)):
            for s, k in zip(streams, (i, (i + 1) % len(calls))):
                args, kw = calls[k]
                got.append((k, Q.paged_attention(*args, stream=s, **kw)))
    torch.cuda.synchronize()
    assert all(torch.equal(alone[k], out) for k, out in got)
    assert Q.offq_get_device_status() == Q.OFFQ_OK


@pytest.mark.parametrize("Hq,H,D,page,dt", [(8, 2, 128, 64, "bf16"), (5, 1, 64, 16, "f16"), (16, 16, 128, 32, "bf16")])
def test_few_rows_among_many(Hq, H, D, page, dt):
    """Sequences, and prefixes, with one query, few and none beside long ones: few enough to take the many-row form with them,
    or too many. And a bound on the queries that no sequence reaches."""
    for news in ([1], [3, 0, 1, 70], [90, 1, 2, 1], [1] * 15 + [70, 0, 2, 66, 40], [65] * 3 + [1] * 30):
        lens, B = [n + 11 * b % 300 for b, n in enumerate(news)], len(news)
        for max_q in (max(news), max(news) + 100):
            _shared([140, 0, 33], [0, B // 2, B // 2, max(B // 2, B - 1)], lens, news, Hq, H, D, page, dt, seed=B, max_q=max_q)
