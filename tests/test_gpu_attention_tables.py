"""Block tables that are parts of wider ones: a sequence holds the pages of the columns that are given, no others."""

import pytest
import torch

from paper_2606_07116_gb300 import build as B
from paper_2606_07116_gb300 import offq as Q

pytestmark = pytest.mark.gpu
PAGE = 16


@pytest.fixture(scope="module", autouse=True)
def _lib():
    B.build()
    Q.load_library()


def _inputs(n, pages=34, H=2, D=128):
    gen = torch.Generator("cuda").manual_seed(n)
    cache = Q.kv4_cache(pages, H, D, PAGE)
    for codes, params in ((cache.k_codes, cache.k_params), (cache.v_codes, cache.v_params)):
        codes.copy_(torch.randint(0, 256, codes.shape, generator=gen, device="cuda", dtype=torch.uint8) | 17)
        params.copy_(torch.rand(params.shape, generator=gen, device="cuda") * 0.2 + 0.05)
    q = torch.randn(3 * n, 8, D, generator=gen, device="cuda").to(torch.bfloat16)
    wide = torch.stack([torch.randperm(pages, generator=gen, device="cuda") for _ in range(5)]).int()
    return q, cache, wide, torch.arange(0, 3 * n + 1, n, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("rows,columns", [(slice(0, 3), slice(0, 25)), (slice(1, 4), slice(4, 29)),
                                          (slice(0, 5, 2), slice(9, 34)), (slice(2, 5), slice(0, 34))])
def test_columns_of_a_wider_table(n, rows, columns):
    q, cache, wide, cu = _inputs(n)
    view = wide[rows, columns]
    lens = torch.tensor([PAGE * view.shape[1], 77, 300], dtype=torch.int32, device="cuda")
    want = Q.paged_attention(q, cache, view.clone(memory_format=torch.contiguous_format), lens, cu, n)
    assert torch.equal(Q.paged_attention(q, cache, view, lens, cu, n), want)
    assert Q.offq_get_device_status() == Q.OFFQ_OK
    lens[0] += 1  # a page more than the view's
    got = Q.paged_attention(q, cache, view, lens, cu, n)
    assert Q.offq_get_device_status() == Q.OFFQ_ERR_INVALID_ARG
    assert torch.equal(got[n:], want[n:])  # the other sequences are unharmed


@pytest.mark.parametrize("n", [1, 40])
def test_a_table_without_columns(n):
    """Sequences that hold nothing yet: zeros and -inf; a length that has no page is reported."""
    q, cache, wide, cu = _inputs(n)
    for table in (wide[:3, :0], torch.empty((3, 0), dtype=torch.int32, device="cuda")):
        lens = torch.zeros(3, dtype=torch.int32, device="cuda")
        out, lse = Q.paged_attention(q, cache, table, lens, cu, n, lse=True)
        assert torch.all(out == 0) and torch.all(lse == float("-inf"))
        assert Q.offq_get_device_status() == Q.OFFQ_OK
        lens[1] = 1
        Q.paged_attention(q, cache, table, lens, cu, n)
        assert Q.offq_get_device_status() == Q.OFFQ_ERR_INVALID_ARG
