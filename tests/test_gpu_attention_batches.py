"""Attention of batches larger than one pass of a kernel over its sequences: the few-row form's CTAs take 512 or 256 at a
time, the many-row form's and the prompts' search 32. Tolerances of the paged calls as derived in
test_gpu_attention_scales (a weight is rounded to a half whatever the queries' type), of prompts in test_gpu_attention."""

import numpy as np
import pytest
import torch

import oracle.attention_oracle as A
from paper_2606_07116_gb300 import build as B
from paper_2606_07116_gb300 import offq as Q
from test_gpu_attention import _prompt
from test_gpu_attention_scales import DT, check_paged

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    B.build()
    Q.load_library()


def _paged(lens, news, Hq, H, D, page, dt, seed):
    rng = np.random.default_rng(seed)
    need = [-(-n // page) for n in lens]
    pages = sum(need) + 1
    codes = [rng.integers(0, 256, (pages, H, page, D // 2), dtype=np.uint8) | 17 for _ in range(2)]
    pairs = [np.stack([0.3 * np.exp(0.3 * rng.standard_normal((pages, H, page))),
                       o * rng.standard_normal((pages, H, page))], -1).astype(np.float32) for o in (0.3, 0.2)]
    order, width = rng.permutation(pages), max(need) + 1
    table = np.full((len(lens), width), -1, np.int32)
    first = np.cumsum([0] + need)
    for b, n in enumerate(need):
        table[b, :n] = order[first[b]:first[b] + n]
    cu = np.cumsum([0] + list(news)).astype(np.int32)
    q = torch.from_numpy(rng.standard_normal((cu[-1], Hq, D))).to(DT[dt][0])
    cache = Q.KV4Cache(*(torch.from_numpy(x).cuda() for x in (codes[0], pairs[0], codes[1], pairs[1])))
    out, lse = Q.paged_attention(q.cuda(), cache, torch.from_numpy(table).cuda(),
                                 torch.tensor(lens, dtype=torch.int32).cuda(), torch.from_numpy(cu).cuda(), max(news),
                                 lse=True)
    assert Q.offq_get_device_status() == Q.OFFQ_OK
    out, lse, q = out.cpu().double().numpy(), lse.cpu().double().numpy(), q.double().numpy()
    for b, n in enumerate(lens):
        j, r = np.arange(n), slice(cu[b], cu[b + 1])
        held = [A.cached(c, p, table[b][j // page], j % page) for c, p in zip(codes, pairs)]
        check_paged(out[r], lse[r], q[r], *held, D ** -0.5, dt, 1 if news[b] * Hq // H <= 16 else 4)


@pytest.mark.parametrize("D,dt", [(128, "bf16"), (64, "f16")])
@pytest.mark.parametrize("many,new,Hq,H", [(1100, 1, 4, 2), (600, 1, 12, 1), (560, 5, 4, 2)])
def test_hundreds_of_short_sequences(many, new, Hq, H, D, dt):
    rng = np.random.default_rng(many)
    lens = rng.integers(0, 70, many)
    lens[rng.random(many) < 0.1] = 0
    lens[[3, many // 2, many - 1]] = 900, 400, 333
    news = np.where(rng.random(many) < 0.1, 0, rng.integers(1, new + 1, many))
    news[-1] = new
    _paged(lens.tolist(), news.tolist(), Hq, H, D, 16, dt, many)


@pytest.mark.parametrize("D,dt", [(128, "bf16"), (64, "f16")])
def test_dozens_of_chunks(D, dt):
    rng = np.random.default_rng(7)
    news = rng.integers(0, 60, 75)
    news[[0, 33, 74]] = 130, 70, 61
    lens = np.maximum(news + rng.integers(-5, 150, 75), 0)
    _paged(lens.tolist(), news.tolist(), 4, 2, D, 32, dt, 8)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("Hq,H,D,dt", [(4, 2, 128, "bf16"), (3, 1, 64, "f16")])
def test_dozens_of_prompts(Hq, H, D, dt, causal):
    rng = np.random.default_rng(9)
    lengths = rng.integers(0, 140, 75)
    lengths[[1, 40, 74]] = 600, 300, 257
    _prompt(lengths.tolist(), Hq, H, D, dt, causal, seed=10)
