"""Attention over a sliding window with sinks (paged_attention and prompt_attention with window=) against the float64
oracle; tolerances in attention_parity. Pages that no query sees have no page number, slots that none sees hold NaN."""

import numpy as np
import pytest
import torch

import oracle.attention_oracle as A
from attention_parity import DT, Pages, check, cumulative, i32, queries
from paper_2606_07116_gb300 import build as B
from paper_2606_07116_gb300 import offq as Q

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    B.build()
    Q.load_library()


def _paged(lens, news, Hq, H, D, page, dt, window, sinks, seed=0, q_pad=0, table_pad=1, k_off=6.0, scale=None, max_q=None):
    seen = [A.in_window(L - n, n, L, window, sinks) for L, n in zip(lens, news)]
    pages = Pages([s.any(0) for s in seen], H, D, page, seed, k_off, table_pad)
    qb, q64 = queries(sum(news), Hq, D, dt, seed + 1, q_pad)
    cu, scale = cumulative(news), scale or D ** -0.5
    out, lse = Q.paged_attention(qb.cuda()[:, :Hq], pages.cache(), i32(pages.table), i32(lens), i32(cu),
                                 max_q or max(news + [0]), scale=scale, lse=True, window=window, sinks=sinks)
    assert Q.offq_get_device_status() == Q.OFFQ_OK
    out, lse = out.cpu().double().numpy(), lse.cpu().double().numpy()
    for b, L in enumerate(lens):
        k, k_mag, v, v_mag = pages.tokens(b, L)
        rows = slice(cu[b], cu[b + 1])
        check(out[rows], lse[rows], q64[rows], k_mag, k, v, v_mag, scale, seen[b], dt)


WINDOWS = [(1, 0), (1, 1), (2, 4), (15, 4), (16, 0), (31, 1), (32, 16), (33, 4), (64, 33), (100, 4), (257, 300), (5000, 4)]


@pytest.mark.parametrize("window,sinks", WINDOWS)
@pytest.mark.parametrize("Hq,H,D,page,dt", [(8, 2, 128, 64, "bf16"), (5, 1, 64, 16, "f16"), (24, 2, 128, 256, "f16"),
                                            (16, 1, 64, 32, "bf16")])
def test_single_tokens(window, sinks, Hq, H, D, page, dt):
    _paged([1, 2, 15, 16, 17, 33, 100, 257, 1000, 1025], [1] * 10, Hq, H, D, page, dt, window, sinks, seed=window)


@pytest.mark.parametrize("window,sinks", WINDOWS)
@pytest.mark.parametrize("news", [[2, 1, 3], [4, 4, 4], [17, 1, 9], [33, 5, 0], [64, 128, 129], [200, 1, 70]])
def test_several_new_tokens(news, window, sinks):
    lens = [n + past for n, past in zip(news, (77, 300, 511))]
    for Hq, H, D, page, dt in ((8, 2, 128, 64, "bf16"), (5, 1, 64, 16, "f16"), (14, 2, 128, 16, "f16")):
        _paged(lens, news, Hq, H, D, page, dt, window, sinks, seed=sum(news) + Hq)


def test_long_pasts():
    for window, sinks in ((1000, 4), (129, 0), (640, 130)):
        _paged([5000], [1], 8, 2, 128, 64, "bf16", window, sinks, seed=1)
        _paged([5000, 3333], [300, 41], 4, 1, 128, 16, "bf16", window, sinks, seed=2)
        _paged([4000, 129, 4097], [40, 128, 2], 4, 2, 64, 128, "f16", window, sinks, seed=3)


def test_rows_that_see_nothing_and_empty_sequences():
    for dt in ("bf16", "f16"):
        _paged([0, 3, 5, 0, 40], [2, 8, 0, 1, 50], 8, 2, 128, 16, dt, 3, 2, seed=4)
        _paged([0], [1], 4, 4, 64, 64, dt, 1, 0, seed=5)
        _paged([10, 0, 200], [140, 150, 201], 4, 1, 128, 64, dt, 7, 4, seed=6)


def test_strided_queries_wide_tables_large_scores():
    _paged([50, 700], [1, 1], 8, 2, 128, 16, "bf16", 60, 4, seed=7, q_pad=3, table_pad=40)
    _paged([50, 700], [20, 300], 8, 2, 64, 16, "f16", 60, 4, seed=8, q_pad=5, table_pad=9)
    _paged([600, 330], [100, 3], 8, 2, 128, 64, "bf16", 90, 4, seed=10, k_off=60.0)
    _paged([600, 400], [200, 4], 8, 2, 128, 64, "f16", 90, 4, seed=12, scale=3.0)


@pytest.mark.parametrize("news", [[1, 1, 1], [5, 1, 90]])
def test_a_window_longer_than_the_sequences_is_full_attention(news):
    """The largest window that the library takes, and larger ones, which the helper cuts to it."""
    lens = [40 + news[0], 700 + news[1], 333 + news[2]]
    pages = Pages([np.ones(L, bool) for L in lens], 2, 128, 64, 3)
    qb, _ = queries(sum(news), 8, 128, "bf16", 4)
    args = (qb.cuda(), pages.cache(), i32(pages.table), i32(lens), i32(cumulative(news)), max(news))
    full = Q.paged_attention(*args, lse=True)
    for window, sinks in ((2 ** 31 - 1, 0), (2 ** 40, 4), (max(lens), 0), (1, 2 ** 40), (2 ** 31 - 1, 2 ** 31 - 1)):
        part = Q.paged_attention(*args, lse=True, window=window, sinks=sinks)
        for a, b in zip(full, part):
            torch.testing.assert_close(a, b, rtol=2.0 ** -7, atol=2.0 ** -8)
    assert Q.offq_get_device_status() == Q.OFFQ_OK


@pytest.mark.parametrize("new", [1, 70])
def test_a_missing_page_inside_the_window_is_reported(new):
    pages = Pages([np.ones(400, bool)], 2, 128, 16, 5)
    qb, q64 = queries(new, 8, 128, "bf16", 6)
    table = pages.table.copy()
    table[0, 20] = 1 << 20  # tokens 320 .. 335
    args = (qb.cuda(), pages.cache(), i32(table), i32([400]), i32([0, new]), new)
    out, lse = Q.paged_attention(*args, lse=True, window=200, sinks=4)
    assert Q.offq_get_device_status() == Q.OFFQ_ERR_INVALID_ARG
    seen = A.in_window(400 - new, new, 400, 200, 4)
    seen[:, 320:336] = False
    k, k_mag, v, v_mag = pages.tokens(0, 400)
    check(out.cpu().double().numpy(), lse.cpu().double().numpy(), q64, k_mag, k, v, v_mag, 128 ** -0.5, seen, "bf16")
    out2 = Q.paged_attention(*args, window=60, sinks=4)  # out of sight now: entries there are not looked at
    if new == 1:
        assert Q.offq_get_device_status() == Q.OFFQ_OK
        seen = A.in_window(399, 1, 400, 60, 4)
        ref = A.attention_masked(q64, k, v, 128 ** -0.5, seen)[0]
        np.testing.assert_allclose(out2.cpu().double().numpy(), ref, atol=2.0 ** -5 * np.abs(v_mag).max())
    else:
        assert Q.offq_get_device_status() == Q.OFFQ_ERR_INVALID_ARG


def test_rows_outside_the_sequences_are_left_alone():
    pages = Pages([np.ones(90, bool), np.ones(60, bool)], 2, 128, 16, 7)
    qb, _ = queries(60, 8, 128, "bf16", 8)
    for cu, m in (([3, 4, 6], 2), ([3, 43, 50], 40)):
        out = torch.full((60, 8, 128), 5.0, dtype=torch.bfloat16, device="cuda")
        Q.paged_attention(qb.cuda(), pages.cache(), i32(pages.table), i32([90, 60]), i32(cu), m, out=out, window=20, sinks=3)
        assert torch.all(out[:3] == 5.0) and torch.all(out[cu[2]:] == 5.0) and not torch.any(out[3:cu[2]] == 5.0)
    assert Q.offq_get_device_status() == Q.OFFQ_OK


def _prompt(lengths, Hq, H, D, dt, window, sinks, seed=0, poison=()):
    x, x64 = queries(sum(lengths), Hq + 2 * H, D, dt, seed)
    cu, scale = cumulative(lengths), D ** -0.5
    for b in poison:
        x[cu[b]:cu[b + 1]] = float("nan")
        x[cu[b]:cu[b + 1]:3] = float("inf")
    x = x.cuda()
    out, lse = Q.prompt_attention(x[:, :Hq], x[:, Hq:Hq + H], x[:, Hq + H:], i32(cu), lse=True, window=window, sinks=sinks)
    assert Q.offq_get_device_status() == Q.OFFQ_OK
    out, lse = out.cpu().double().numpy(), lse.cpu().double().numpy()
    for b, n in enumerate(lengths):
        if b in poison:
            continue
        rows = slice(cu[b], cu[b + 1])
        q, k, v = x64[rows, :Hq], x64[rows, Hq:Hq + H], x64[rows, Hq + H:]
        check(out[rows], lse[rows], q, np.abs(k), k, v, np.abs(v), scale, A.in_window(0, n, n, window, sinks), dt)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 4), (64, 8), (127, 9), (128, 0), (129, 64), (200, 128),
                                          (300, 130), (100, 257), (4000, 4)])
@pytest.mark.parametrize("Hq,H,D,dt", [(4, 2, 128, "bf16"), (3, 1, 64, "f16"), (5, 1, 128, "f16"), (2, 1, 64, "bf16")])
def test_prompts(window, sinks, Hq, H, D, dt):
    _prompt([1, 2, 127, 128, 129, 300, 777, 5], Hq, H, D, dt, window, sinks, seed=window)


def test_a_long_prompt():
    for Hq in (2, 3):
        _prompt([2500], Hq, 1, 128, "bf16", 700, 4, seed=1)
        _prompt([1301, 1100], Hq, 1, 64, "f16", 257, 20, seed=2)


def test_a_prompt_of_infinities_and_nan_stays_alone():
    for D in (64, 128):
        for window, sinks in ((20, 4), (129, 0), (140, 9)):
            _prompt([300, 60, 330, 40, 200], 2, 1, D, "bf16", window, sinks, seed=3, poison=(1, 3))


def test_prompt_rows_outside_the_sequences_are_left_alone():
    x, _ = queries(400, 4, 128, "bf16", 9)
    x = x.cuda()
    out = torch.full((400, 2, 128), 5.0, dtype=torch.bfloat16, device="cuda")
    Q.prompt_attention(x[:, :2], x[:, 2:3], x[:, 3:4], i32([4, 9, 380]), out=out, window=30, sinks=2)
    assert torch.all(out[:4] == 5.0) and torch.all(out[380:] == 5.0) and not torch.any(out[4:380] == 5.0)


def test_prompt_and_pages_agree():
    """The last tokens of a prompt through both: exact codes as keys and values, offsets zero."""
    n, Hq, H, D, window, sinks = 500, 8, 2, 128, 130, 5
    gen = torch.Generator().manual_seed(11)
    codes = torch.randint(1, 16, (2, n, H, D), generator=gen)
    q = torch.randn((n, Hq, D), generator=gen).to(torch.bfloat16).cuda()
    k, v = ((c - 8).to(torch.bfloat16).cuda() for c in codes)
    cache = Q.kv4_cache(-(-n // 64), H, D, 64)
    for c, par, u in ((cache.k_codes, cache.k_params, codes[0]), (cache.v_codes, cache.v_params, codes[1])):
        u = torch.nn.functional.pad(u, (0, 0, 0, 0, 0, -n % 64)).to(torch.uint8).cuda()
        u = u.view(-1, 64, H, D).transpose(1, 2)
        c.copy_(u[..., 0::2] | (u[..., 1::2] << 4))
        par[..., 0], par[..., 1] = 1.0, 0.0
    table = torch.arange(cache[0].shape[0], dtype=torch.int32, device="cuda")[None].contiguous()
    whole = Q.prompt_attention(q, k, v, i32([0, n]), scale=0.01, window=window, sinks=sinks)
    for new in (1, 4, 100, n):
        part = Q.paged_attention(q[n - new:], cache, table, i32([n]), i32([0, new]), new, scale=0.01, window=window, sinks=sinks)
        # weights as bf16 on one side, outputs as bf16 on both, values up to 7
        torch.testing.assert_close(whole[n - new:], part, rtol=0, atol=7 * 4 * 2.0 ** -8)


def test_a_graph_follows_the_window():
    """One captured step, replayed as the sequences grow: the window moves with the lengths on the device."""
    Hq, H, D, page = 8, 2, 128, 16
    lens = [90, 350]
    pages = Pages([np.ones(L + 40, bool) for L in lens], H, D, page, 15)
    cache, table, cu = pages.cache(), i32(pages.table), i32([0, 1, 2])
    x = torch.zeros((2, Hq, D), dtype=torch.bfloat16, device="cuda")
    n = i32(lens)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        Q.paged_attention(x, cache, table, n, cu, 1, window=40, sinks=4)
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            out = Q.paged_attention(x, cache, table, n, cu, 1, window=40, sinks=4)
    torch.cuda.current_stream().wait_stream(s)
    for step in range(0, 40, 7):
        x.normal_(generator=torch.Generator(device="cuda").manual_seed(step))
        n.copy_(i32([L + step for L in lens]))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, Q.paged_attention(x, cache, table, n, cu, 1, window=40, sinks=4))
    assert Q.offq_get_device_status() == Q.OFFQ_OK


@pytest.mark.parametrize("new", [1, 40])
def test_the_longest_context(new):
    """Token numbers up to the last that the library takes, of which the window and the sinks alone have pages."""
    most, page, window, sinks, D = 0x7FFFFF00, 256, 300, 4, 64
    rows = np.zeros(3 * page, bool)  # the first page, and the last two
    rows[:sinks] = True
    rows[page + 2 * page - window - new + 1:] = True
    pages = Pages([rows], 1, D, page, 17, table_pad=0)
    table = torch.full((1, most // page), -1, dtype=torch.int32, device="cuda")
    table[0, 0] = int(pages.table[0, 0])
    table[0, -2:] = torch.from_numpy(pages.table[0, 1:]).cuda()
    qb, q64 = queries(new, 4, D, "bf16", 18)
    out, lse = Q.paged_attention(qb.cuda(), pages.cache(), table, i32([most]), i32([0, new]), new, lse=True, window=window,
                                 sinks=sinks)
    assert Q.offq_get_device_status() == Q.OFFQ_OK
    at = 3 * page - new  # as positions of a sequence of three pages, whose window is the same
    seen = A.in_window(at, new, 3 * page, window, sinks)
    k, k_mag, v, v_mag = pages.tokens(0, 3 * page)
    check(out.cpu().double().numpy(), lse.cpu().double().numpy(), q64, k_mag, k, v, v_mag, D ** -0.5, seen, "bf16")


def test_calls_that_need_no_workspace():
    """Few and short sequences, and tables that are too wide or batches too large for that: the same results with the
    workspace that the call asks for, a larger one, and none where it asks for none."""
    for L, B_, width, news in ((300, 2, 20, 1), (300, 2, 20, 4), (300, 2, 200, 1), (40, 70, 4, 1), (1000, 16, 70, 3)):
        pages = Pages([np.ones(L, bool)] * B_, 2, 128, 16, 21, table_pad=max(1, width - -(-L // 16)))
        qb, q64 = queries(B_ * news, 8, 128, "bf16", 22)
        args = (qb.cuda(), pages.cache(), i32(pages.table), i32([L] * B_), i32(cumulative([news] * B_)), news)
        for window, sinks in ((30, 4), (900, 0), (4000, 40)):
            need = Q.load_library().offq_paged_attention_window_workspace(B_ * news, 8, 2, 128, B_, news, 16,
                                                                          pages.table.shape[1], window, sinks)
            most = Q.paged_attention_workspace(B_ * news, 8, 2, 128, B_, news)
            tokens = min(pages.table.shape[1] * 16, window + sinks + news + 64)
            assert need == (0 if B_ * 2 <= torch.cuda.get_device_properties(0).multi_processor_count and tokens <= 1280
                            else most)
            kw = dict(window=window, sinks=sinks, lse=True)
            a = Q.paged_attention(*args, **kw)
            b = Q.paged_attention(*args, workspace=torch.empty(most, dtype=torch.uint8, device="cuda"), **kw)
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
            if need > 0:
                with pytest.raises(Q.OffqError):
                    Q.paged_attention(*args, workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"), **kw)
            seen = A.in_window(L - news, news, L, window, sinks)
            for s in (0, B_ - 1):
                k, k_mag, v, v_mag = pages.tokens(s, L)
                rows = slice(s * news, (s + 1) * news)
                check(a[0][rows].cpu().double().numpy(), a[1][rows].cpu().double().numpy(), q64[rows], k_mag, k, v, v_mag,
                      128 ** -0.5, seen, "bf16")
    assert Q.offq_get_device_status() == Q.OFFQ_OK


@pytest.mark.parametrize("new", [1, 3, 60])
def test_outputs_inside_wider_rows(new):
    """out= as the middle heads of wider rows: what stands around them stays."""
    pages = Pages([np.ones(200, bool), np.ones(150, bool)], 2, 128, 16, 41)
    T = 2 * new
    qb, _ = queries(T, 8, 128, "bf16", 42)
    args = (qb.cuda(), pages.cache(), i32(pages.table), i32([200, 150]), i32([0, new, T]), new)
    prefix = Q.SharedPrefix(i32(pages.table[:1]), i32([77]), i32([0, 2]))
    x, _ = queries(300, 12, 128, "bf16", 43)
    x = x.cuda()
    prompt = (x[:, :8], x[:, 8:10], x[:, 10:], i32([0, 130, 300]))
    for call, n in ((lambda **kw: Q.paged_attention(*args, window=40, sinks=4, **kw), T),
                    (lambda **kw: Q.paged_attention(*args, prefix=prefix, **kw), T),
                    (lambda **kw: Q.prompt_attention(*prompt, window=40, sinks=4, **kw), 300)):
        wide = torch.full((n, 11, 128), 5.0, dtype=torch.bfloat16, device="cuda")
        out = call(out=wide[:, 2:10])
        assert out.data_ptr() == wide[:, 2:].data_ptr()
        assert torch.equal(out, call()) and torch.all(wide[:, :2] == 5.0) and torch.all(wide[:, 10:] == 5.0)


@pytest.mark.parametrize("new", [1, 9])
def test_a_graph_of_a_large_batch(new):
    """More units than SMs, so parts that cross CTAs; captured, and replayed as lengths grow, as calls compute it."""
    B_, H = 40, 8
    lens = [60 + 37 * b for b in range(B_)]
    pages = Pages([np.ones(L + 20, bool) for L in lens], H, 64, 32, 51)
    cache, table, n = pages.cache(), i32(pages.table), i32(lens)
    cu = i32(cumulative([new] * B_))
    prefix = Q.SharedPrefix(table[3:5].contiguous(), i32([90, 100]), i32([0, 25, B_]))
    x = torch.zeros((B_ * new, 2 * H, 64), dtype=torch.float16, device="cuda")

    def calls():
        return (Q.paged_attention(x, cache, table, n, cu, new, window=700, sinks=3),
                Q.paged_attention(x, cache, table, n, cu, new, prefix=prefix))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        calls()
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            a, b = calls()
    torch.cuda.current_stream().wait_stream(s)
    for step in (0, 11, 20):
        x.normal_(generator=torch.Generator(device="cuda").manual_seed(step))
        n.copy_(i32([L + step for L in lens]))
        graph.replay()
        torch.cuda.synchronize()
        c, d = calls()
        assert torch.equal(a, c) and torch.equal(b, d)
    assert Q.offq_get_device_status() == Q.OFFQ_OK


@pytest.mark.parametrize("Hq,H,D,page,dt", [(8, 2, 128, 64, "bf16"), (5, 1, 64, 16, "f16"), (16, 16, 128, 32, "bf16")])
def test_few_rows_among_many(Hq, H, D, page, dt):
    """Sequences with one query, few and none beside long ones: few enough to take the many-row form with them, or too many.
    And a bound on the queries that no sequence reaches."""
    for news in ([1], [3, 0, 1, 70], [90, 1, 2, 1], [1] * 15 + [70, 0, 2, 66, 40], [65] * 3 + [1] * 30):
        lens = [n + 11 * b % 300 for b, n in enumerate(news)]
        for max_q in (max(news), max(news) + 100):
            _paged(lens, news, Hq, H, D, page, dt, 50, 4, seed=len(news), max_q=max_q)
