"""Paged attention calls that are given no workspace, in a row, on several streams, from threads and in a graph."""

import threading

import pytest
import torch

from paper_2606_07116_gb300 import build as B
from paper_2606_07116_gb300 import offq as Q

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    B.build()
    Q.load_library()


def _inputs(seed, n, L=1500, Hq=8, H=2, D=128, page=16):
    """One sequence: n new tokens over L cached ones, so that its heads cross thread blocks and are joined."""
    gen = torch.Generator("cuda").manual_seed(seed)
    pages = -(-L // page)
    cache = Q.kv4_cache(pages, H, D, page)
    for codes, params in ((cache.k_codes, cache.k_params), (cache.v_codes, cache.v_params)):
        codes.copy_(torch.randint(0, 256, codes.shape, generator=gen, device="cuda", dtype=torch.uint8) | 17)
        params.copy_(torch.rand(params.shape, generator=gen, device="cuda") * 0.2 + 0.05)
    q = torch.randn(n, Hq, D, generator=gen, device="cuda").to(torch.bfloat16)
    table = torch.randperm(pages, generator=gen, device="cuda").int()[None]
    return (q, cache, table, torch.tensor([L], dtype=torch.int32, device="cuda"),
            torch.tensor([0, n], dtype=torch.int32, device="cuda"), n)


def _given(args):
    q, cache, _, lens, _, n = args
    size = Q.paged_attention_workspace(q.shape[0], q.shape[1], cache.k_codes.shape[1], q.shape[2], lens.shape[0], n)
    out = Q.paged_attention(*args, workspace=torch.empty(size, dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("n", [1, 40])
def test_calls_in_a_row(n):
    sets = [_inputs(seed, n) for seed in range(4)]
    want = [_given(x) for x in sets]
    got = [Q.paged_attention(*x) for x in sets for _ in range(3)]
    assert all(torch.equal(g, want[i // 3]) for i, g in enumerate(got))
    more = _inputs(9, 400)
    assert torch.equal(Q.paged_attention(*more), _given(more))
    assert torch.equal(Q.paged_attention(*sets[0]), want[0])


@pytest.mark.parametrize("n", [1, 40])
def test_streams(n):
    sets = [_inputs(seed, n) for seed in range(4)]
    want = [_given(x) for x in sets]
    streams = [torch.cuda.Stream() for _ in range(4)]
    got = []
    for _ in range(5):
        for i, s in enumerate(streams):   # as the current stream, as an argument, as a handle
            out = torch.empty_like(want[i])
            s.wait_stream(torch.cuda.current_stream())
            if i % 2 == 0:
                with torch.cuda.stream(s):
                    Q.paged_attention(*sets[i], out=out)
            else:
                Q.paged_attention(*sets[i], out=out, stream=s if i == 1 else s.cuda_stream)
            got.append((i, out))
            torch.full((1 << 21,), 255, dtype=torch.uint8, device="cuda")  # takes what a call may have let go too soon
    torch.cuda.synchronize()
    assert all(torch.equal(out, want[i]) for i, out in got)


@pytest.mark.parametrize("n", [1, 40])
def test_a_graph_beside_other_calls(n):
    a, b = _inputs(1, n), _inputs(2, n)
    want = _given(a), _given(b)
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = Q.paged_attention(*a)
    with torch.cuda.stream(s):
        others = [Q.paged_attention(*b) for _ in range(3)]
        graph.replay()
        others += [Q.paged_attention(*b) for _ in range(3)]
    torch.cuda.synchronize()
    assert torch.equal(out, want[0]) and all(torch.equal(x, want[1]) for x in others)


def test_threads_on_one_stream():
    sets = [_inputs(seed, 1) for seed in range(4)]
    want = [_given(x) for x in sets]
    wrong = []

    def work(i):
        got = [Q.paged_attention(*sets[i]) for _ in range(50)]
        torch.cuda.synchronize()
        wrong.extend(i for g in got if not torch.equal(g, want[i]))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert wrong == []


def test_tables_that_are_views():
    """Columns from the middle of a wider table, whose last row ends with its memory, and one row for all sequences."""
    q, cache, table, _, _, _ = _inputs(5, 3, L=400)
    q = q.contiguous()
    cu = torch.arange(4, dtype=torch.int32, device="cuda")
    lens = torch.tensor([400, 77, 399], dtype=torch.int32, device="cuda")
    want = Q.paged_attention(q, cache, table.repeat(3, 1), lens, cu, 1)
    wide = torch.full((3, table.shape[1] + 9), -1, dtype=torch.int32, device="cuda")
    wide[:, 9:] = table
    for view in (wide[:, 9:], table.expand(3, -1)):
        assert torch.equal(Q.paged_attention(q, cache, view, lens, cu, 1), want)
        assert torch.equal(Q.paged_attention(q, cache, view, lens, cu, 1, stream=torch.cuda.current_stream()), want)
        assert Q.offq_get_device_status() == Q.OFFQ_OK
        # A length that the view's pages do not hold is an error, not a read of what lies behind them.
        Q.paged_attention(q, cache, view, lens + 16, cu, 1)
        assert Q.offq_get_device_status() == Q.OFFQ_ERR_INVALID_ARG
