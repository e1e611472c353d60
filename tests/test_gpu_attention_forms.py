"""Which kernels a paged call under a window or behind prefixes launches: the few-row form and its joining, the many-row form
and its, and the joining of both parts of a row behind prefixes. Calls are captured and their launches counted, none runs. And
the workspaces that go with the forms."""

import ctypes

import pytest
import torch

from paper_2606_07116_gb300 import build as B
from paper_2606_07116_gb300 import offq as Q

pytestmark = pytest.mark.gpu

FEW, MANY, BOTH_PARTS = 2, 2, 1


@pytest.fixture(scope="module", autouse=True)
def _lib():
    B.build()
    Q.load_library()


def launches(news, tokens, H, G, prefix=None, D=128, page=64, max_q=None, **kw):
    """Kernels of a call for these new tokens, with tables of `tokens` tokens a sequence (prefix: (tokens, counts))."""
    cuda = ctypes.CDLL("libcuda.so.1")
    T, n = sum(news), len(news)
    i32 = dict(dtype=torch.int32, device="cuda")
    cache = Q.kv4_cache(2, H, D, page)
    table = torch.zeros((n, -(-tokens // page)), **i32)
    lens, cu = torch.tensor([tokens] * n, **i32), torch.tensor([0] + list(torch.tensor(news).cumsum(0)), **i32)
    q = torch.zeros((T, H * G, D), dtype=torch.bfloat16, device="cuda")
    max_q, P = max_q or max(news), 0
    if prefix is not None:
        P = len(prefix[1])
        kw["prefix"] = Q.SharedPrefix(torch.zeros((P, -(-prefix[0] // page)), **i32), torch.tensor([prefix[0]] * P, **i32),
                                      torch.tensor([0] + list(torch.tensor(prefix[1]).cumsum(0)), **i32))
    out, workspace = torch.empty_like(q), torch.empty(Q.paged_attention_workspace(T, H * G, H, D, n, max_q, P),
                                                      dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph, count = ctypes.c_void_p(), ctypes.c_size_t()
    handle = ctypes.c_void_p(s.cuda_stream)
    assert cuda.cuStreamBeginCapture_v2(handle, 2) == 0
    try:
        Q.paged_attention(q, cache, table, lens, cu, max_q, out=out, workspace=workspace, stream=s, **kw)
    finally:
        assert cuda.cuStreamEndCapture(handle, ctypes.byref(graph)) == 0
    assert cuda.cuGraphGetNodes(graph, None, ctypes.byref(count)) == 0
    assert cuda.cuGraphDestroy(graph) == 0
    return count.value


@pytest.mark.parametrize("kw,more", [(dict(window=1 << 20, sinks=4), 0), (dict(prefix=(4000, [2])), BOTH_PARTS)])
def test_long_chunks_take_the_many_row_form_alone(kw, more):
    for news in ([1000, 900], [1000, 1000]):
        for H, G in ((8, 4), (32, 1)):
            assert launches(news, 5000, H, G, **kw) == MANY + more


@pytest.mark.parametrize("kw,more", [(dict(window=1 << 20, sinks=4), 0), (dict(prefix=(4000, [2])), BOTH_PARTS)])
def test_a_single_token_beside_a_chunk_counts_with_what_it_may_see(kw, more):
    """One token and 1000: 32 tiles in the many-row form, of as many blocks as the table or the window has."""
    assert launches([1000, 1], 60000, 32, 1, **kw) == FEW + MANY + more
    assert launches([1000, 1], 500000, 8, 4, **kw) == FEW + MANY + more
    assert launches([1000, 1], 1024, 8, 4, **kw) == MANY + more
    assert launches([1000, 1, 1], 500000, 8, 4, **({**kw, "prefix": (4000, [3])} if "prefix" in kw else kw)) == FEW + MANY + more


def test_a_short_window_bounds_what_a_single_token_sees():
    assert launches([1000, 1], 500000, 8, 4, window=1000, sinks=4) == MANY
    assert launches([1000, 1], 500000, 8, 4, window=100000) == FEW + MANY
    assert launches([1000, 1], 500000, 8, 4, window=1000, sinks=100000) == FEW + MANY


@pytest.mark.parametrize("kw,more", [(dict(window=1 << 20), 0), (dict(prefix=(4000, [64])), BOTH_PARTS)])
def test_short_sequences_next_to_the_longest_are_counted(kw, more):
    """63 sequences of eight queries, 32 rows each, and one of nine: the few-row form has work for all but one."""
    assert launches([8] * 63 + [9], 2000, 2, 4, **kw) == FEW + MANY + more


def test_prefixes_that_may_have_few_rows_are_counted():
    """A single token behind 200000 tokens of its own prefix, beside a chunk behind another."""
    assert launches([1000, 1], 1024, 8, 4, prefix=(200000, [1, 1])) == FEW + MANY + BOTH_PARTS
    assert launches([1000, 1], 1024, 8, 4, prefix=(1000, [1, 1])) == MANY + BOTH_PARTS


def test_workspaces_behind_prefixes_go_by_the_rows_that_a_prefix_may_have():
    """Two fp32 sums and statistics for each query and head, and the parts of the form that a prefix's rows take, whatever the
    sequences' own rows are."""
    sums = lambda T, Hq, D: T * Hq * (8 * D + 16)  # noqa: E731
    for D in (64, 128):
        few, many = Q.paged_attention_workspace(1, 8, 8, D, 1, 1), Q.paged_attention_workspace(100, 8, 8, D, 1, 100)
        assert 0 < few < many
        for Hq, H, n, new, parts in ((8, 8, 32, 1, few), (8, 8, 33, 1, many), (32, 8, 8, 1, few), (32, 8, 9, 1, many),
                                     (32, 8, 64, 1, many), (8, 8, 1, 20, few), (8, 8, 1, 32, few), (8, 8, 1, 33, many)):
            got = Q.paged_attention_workspace(n * new, Hq, H, D, n, new, prefixes=1)
            assert got == sums(n * new, Hq, D) + parts, (Hq, H, n, new)
    assert Q.paged_attention_workspace(64, 32, 8, 128, 64, 1) < Q.paged_attention_workspace(64, 32, 8, 128, 64, 1, 1) - sums(64, 32, 128)
    assert Q.paged_attention_workspace(20, 8, 8, 128, 1, 20) > Q.paged_attention_workspace(20, 8, 8, 128, 1, 20, 1) - sums(20, 8, 128)


@pytest.mark.parametrize("n", [8, 9])
def test_a_workspace_of_just_the_bytes_asked_for_is_enough(n):
    """Single tokens of 32 rows behind a prefix, and of 36."""
    Hq, H, D, page = 32, 8, 128, 16
    gen = torch.Generator("cuda").manual_seed(n)
    i32 = dict(dtype=torch.int32, device="cuda")
    cache = Q.kv4_cache(16, H, D, page)
    for c in (cache.k_codes, cache.v_codes):
        c.random_(0, 256, generator=gen)
    for p in (cache.k_params, cache.v_params):
        p.uniform_(0.1, 0.3, generator=gen)
    q = torch.randn((n, Hq, D), generator=gen, device="cuda").to(torch.bfloat16)
    prefix = Q.SharedPrefix(torch.arange(8, **i32)[None], torch.tensor([120], **i32), torch.tensor([0, n], **i32))
    table = (8 + torch.arange(n, **i32) % 8)[:, None].contiguous()
    args = (q, cache, table, torch.full((n,), 9, **i32), torch.arange(n + 1, **i32), 1)
    need = Q.paged_attention_workspace(n, Hq, H, D, n, 1, 1)
    room = torch.full((need + 256,), 77, dtype=torch.uint8, device="cuda")
    out = Q.paged_attention(*args, prefix=prefix, workspace=room[:need])
    assert torch.equal(out, Q.paged_attention(*args, prefix=prefix)) and torch.all(room[need:] == 77)
    assert Q.offq_get_device_status() == Q.OFFQ_OK
    with pytest.raises(Q.OffqError):
        Q.paged_attention(*args, prefix=prefix, workspace=room[:need - 1])
