"""The example layer: prompts, chunks and single tokens through one cache, against the float64 oracle.

Tolerances are those of the attention tests. The example's own float64 attention reads the cache back in fp32: its
keys and values are within 2 u of |code| scale + |offset|, which is far inside them."""

import importlib.util
import os

import numpy as np
import pytest
import torch

import oracle.attention_oracle as A
from conftest import ROOT
from paper_2606_07116_gb300 import build as B
from paper_2606_07116_gb300 import offq as Q
from test_gpu_attention import _check

pytestmark = pytest.mark.gpu

spec = importlib.util.spec_from_file_location("attention_layer", os.path.join(ROOT, "examples", "attention_layer.py"))
E = importlib.util.module_from_spec(spec)
spec.loader.exec_module(E)

HIDDEN, LENGTHS = 512, [70, 1, 33]


@pytest.fixture(scope="module", autouse=True)
def _lib():
    B.build()
    Q.load_library()


def _layer(D):
    return E.AttentionLayer(HIDDEN, 512 // D, 2, D, max_len=256, g=512, pages=40, B=len(LENGTHS), page_size=16)


def _rows(n, seed):
    return torch.randn(n, HIDDEN, generator=torch.Generator("cuda").manual_seed(seed), device="cuda").to(torch.bfloat16)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [1, 3, 21])
def test_new_tokens_after_prompts(n, D):
    layer = _layer(D)
    layer.prompt(_rows(sum(LENGTHS), 1), LENGTHS)
    layer.pages.reserve([m + n for m in LENGTHS])
    scale = D ** -0.5
    seen = []

    def checked(q, cache, table, lens, cu, n):
        out, lse = Q.paged_attention(q, cache, table, lens, cu, n, lse=True)
        codes = [c.cpu().numpy() for c in cache]
        got, got_lse, q64 = (t.double().cpu().numpy() for t in (out, lse, q))
        own = layer.attention64(q, cache, table, lens, cu, n).cpu().numpy()
        for b, L in enumerate(lens.tolist()):
            j, rows = np.arange(L), slice(b * n, b * n + n)
            page = table[b].cpu().numpy()[j // 16]
            (k, kq, ks, ko), (v, vq, vs, vo) = (A.cached(c, p, page, j % 16) for c, p in (codes[:2], codes[2:]))
            mags = [np.abs(x) * s[..., None] + np.abs(o)[..., None] for x, s, o in ((kq, ks, ko), (vq, vs, vo))]
            sees = [L - n + i + 1 for i in range(n)]
            _check(got[rows], got_lse[rows], q64[rows], mags[0], k, v, mags[1], scale, sees, "bf16")
            _check(own[rows], got_lse[rows], q64[rows], mags[0], k, v, mags[1], scale, sees, "bf16")
        seen.append(lens.tolist())
        return out

    y = layer.extend(_rows(len(LENGTHS) * n, 2), n, checked)
    assert y.shape == (len(LENGTHS) * n, HIDDEN) and torch.isfinite(y).all()
    assert seen == [[m + n for m in LENGTHS]]
    assert Q.offq_get_device_status() == Q.OFFQ_OK


def test_a_graph_decodes_what_calls_decode():
    got = []
    for captured in (False, True):
        layer = _layer(64)
        layer.prompt(_rows(sum(LENGTHS), 1), LENGTHS)
        layer.pages.reserve([m + 6 for m in LENGTHS])
        x, ys = _rows(len(LENGTHS), 2), []
        if captured:
            graph = torch.cuda.CUDAGraph()
            torch.cuda.synchronize()
            with torch.cuda.graph(graph):
                y = layer.extend(x, 1)
        for _ in range(6):
            if captured:
                graph.replay()
            else:
                y = layer.extend(x, 1)
            ys.append(y.clone())
            x.copy_(y)
        got.append((torch.stack(ys), layer.pages.lens.tolist()))
    assert torch.equal(got[0][0], got[1][0]) and got[0][1] == got[1][1] == [m + 6 for m in LENGTHS]


def test_a_full_cache_is_refused():
    layer = _layer(64)
    with pytest.raises(RuntimeError):
        layer.pages.reserve([257, 1, 1])
    with pytest.raises(RuntimeError):
        layer.pages.reserve([256, 256, 256])
