"""The example layer under a sliding window, with pages given back as it moves, and behind tokens that its sequences share:
prompts, chunks and single tokens through one cache.

Both sides of a comparison work on the same cached values: the call's output is rounded to bf16 (half a step, 2^-8 of
itself), its weights to halves (2^-11), scores and sums are fp32. The example's own float64 attention reads values back in
fp32 (2^-24)."""

import importlib.util
import os

import pytest
import torch

from conftest import ROOT
from paper_2606_07116_gb300 import build as B
from paper_2606_07116_gb300 import offq as Q

pytestmark = pytest.mark.gpu

spec = importlib.util.spec_from_file_location("attention_layer", os.path.join(ROOT, "examples", "attention_layer.py"))
E = importlib.util.module_from_spec(spec)
spec.loader.exec_module(E)

HIDDEN = 512


@pytest.fixture(scope="module", autouse=True)
def _lib():
    B.build()
    Q.load_library()


def _rows(n, seed):
    return torch.randn(n, HIDDEN, generator=torch.Generator("cuda").manual_seed(seed), device="cuda").to(torch.bfloat16)


def _checked(layer, calls):
    def attention(q, *args, **kw):
        out, ref = Q.paged_attention(q, *args, **kw), layer.attention64(q, *args, **kw)
        calls.append(kw)
        # 2^-8 |out| for the output, 2 * 2^-11 of the largest value for numerator and denominator; scores of this size
        # (|z| < 40) are off by less than 2^-12 of a weight.
        torch.testing.assert_close(out.double(), ref, rtol=2.0 ** -8, atol=2.0 ** -9 * ref.abs().max().item())
        return out
    return attention


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window,sinks", [(24, 4), (50, 0), (17, 20)])
def test_a_window_that_moves(window, sinks, D):
    lengths, page = [70, 1, 133], 16
    layer = E.AttentionLayer(HIDDEN, 512 // D, 2, D, max_len=256, g=512, pages=40, B=3, page_size=page, window=window,
                             sinks=sinks)
    y = layer.prompt(_rows(sum(lengths), 1), lengths)
    assert torch.isfinite(y).all()
    calls = []
    for step, n in enumerate((1, 1, 5, 20, 1, 3)):
        layer.pages.release(lengths, window, sinks)
        lengths = [m + n for m in lengths]
        layer.pages.reserve(lengths)
        y = layer.extend(_rows(3 * n, 2 + step), n, _checked(layer, calls))
        assert torch.isfinite(y).all() and layer.pages.lens.tolist() == lengths
    assert calls == [{"window": window, "sinks": sinks}] * 6
    for b, m in enumerate(lengths):  # what was given back: whole pages between sinks and window, as of the last step
        kept = [i for i in range(-(-m // page)) if i * page < sinks or (i + 1) * page > m - 3 + 1 - window]
        held = (layer.pages.table[b] >= 0).nonzero()[:, 0].tolist()
        assert held == kept
    assert Q.offq_get_device_status() == Q.OFFQ_OK


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("shared", [1, 48, 101])
def test_sequences_behind_shared_tokens(shared, D):
    layer = E.AttentionLayer(HIDDEN, 512 // D, 2, D, max_len=256, g=512, pages=60, B=5, page_size=16)
    y = layer.share(_rows(shared, 1))
    assert y.shape == (shared, HIDDEN) and torch.isfinite(y).all() and layer.before == shared
    calls, total = [], 0
    for step, n in enumerate((30, 1, 1, 4, 1)):
        total += n
        layer.pages.reserve([total] * 5)
        y = layer.extend(_rows(5 * n, 2 + step), n, _checked(layer, calls))
        assert torch.isfinite(y).all()
    assert len(calls) == 5 and all(set(kw) == {"prefix"} for kw in calls)
    assert Q.offq_get_device_status() == Q.OFFQ_OK


def test_a_graph_decodes_behind_shared_tokens_what_calls_decode():
    got = []
    for captured in (False, True):
        layer = E.AttentionLayer(HIDDEN, 8, 2, 64, max_len=256, g=512, pages=60, B=4, page_size=16)
        layer.share(_rows(90, 1))
        layer.pages.reserve([20] * 4)
        layer.extend(_rows(4 * 9, 2), 9)
        x, ys = _rows(4, 3), []
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
        got.append(torch.stack(ys))
    assert torch.equal(*got)


def test_a_full_cache_refuses_to_share():
    layer = E.AttentionLayer(HIDDEN, 8, 2, 64, max_len=256, g=512, pages=4, B=2, page_size=16)
    with pytest.raises(RuntimeError):
        layer.share(_rows(65, 1))


def test_what_cannot_share_tokens_refuses_to():
    """A layer with a window, one that shares some already, and one whose sequences hold tokens: each goes on as it was."""
    def layer(**kw):
        return E.AttentionLayer(HIDDEN, 8, 2, 64, max_len=256, g=512, pages=30, B=2, page_size=16, **kw)

    def refuses(one):
        seen, before, free = one.seen, one.before, list(one.pages.free)
        with pytest.raises(ValueError):
            one.share(_rows(20, 5))
        assert one.seen is seen and one.before == before and one.pages.free == free
    windowed, behind, held = layer(window=24, sinks=4), layer(), layer()
    refuses(windowed)
    behind.share(_rows(20, 1))
    refuses(behind)
    held.prompt(_rows(9, 2), [4, 5])
    refuses(held)
    for one, n, lengths in ((windowed, 3, [3, 3]), (behind, 3, [3, 3]), (held, 2, [6, 7])):
        one.pages.reserve(lengths)
        assert torch.isfinite(one.extend(_rows(2 * n, 6), n, _checked(one, []))).all()
    with pytest.raises(ValueError):
        behind.prompt(_rows(9, 2), [4, 5])
    assert Q.offq_get_device_status() == Q.OFFQ_OK
