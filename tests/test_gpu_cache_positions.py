"""A token whose position is outside the rotary table reaches the cache with neither its key nor its value."""

import pytest
import torch

from paper_2606_07116_gb300 import build as B
from paper_2606_07116_gb300 import offq as Q

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    B.build()
    Q.load_library()


@pytest.mark.parametrize("T,H,D,rot,queries", [(4, 2, 128, 128, True), (5, 1, 64, 32, False), (700, 8, 128, 64, True)])
def test_a_position_outside_the_table_leaves_the_slot(T, H, D, rot, queries):
    gen = torch.Generator("cuda").manual_seed(T)
    x = torch.randn((T, 3 * H, D), generator=gen, device="cuda").to(torch.bfloat16)
    q, k, v = x[:, :H], x[:, H:2 * H], x[:, 2 * H:]
    table = Q.rope_table(50, rot)
    pos = torch.arange(T, dtype=torch.int32, device="cuda") % 50
    bad = torch.tensor([1, T - 1], device="cuda")
    pos[bad] = torch.tensor([50, -1], dtype=torch.int32, device="cuda")
    page = 16
    slots = torch.randperm(-(-T // page) * page, generator=gen, device="cuda")[:T]

    def written(pos):
        cache = Q.kv4_cache(-(-T // page), H, D, page)
        for t in cache:
            t.view(torch.uint8).fill_(0xA5)
        Q.kv4_paged_write(cache, k, v, slots, pos, table, q=q if queries else None)
        return [t.view(torch.uint8).transpose(1, 2).flatten(0, 1)[slots] for t in cache]
    want = written(pos.clamp(0, 49))
    assert Q.offq_get_device_status() == Q.OFFQ_OK
    got = written(pos)
    assert Q.offq_get_device_status() == Q.OFFQ_ERR_INVALID_ARG
    good = torch.ones(T, dtype=torch.bool, device="cuda")
    good[bad] = False
    for g, w in zip(got, want):
        assert torch.equal(g[good], w[good])
        assert torch.all(g[bad] == 0xA5)
