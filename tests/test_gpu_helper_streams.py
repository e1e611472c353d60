"""Helpers given a stream that is not the current one, beside work of the current stream on memory it has let go."""

import pytest
import torch

from paper_2606_07116_gb300 import build as B
from paper_2606_07116_gb300 import offq as Q

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    B.build()
    Q.load_library()


def _calls():
    gen = torch.Generator("cuda").manual_seed(3)
    x = torch.randn((600, 6, 128), generator=gen, device="cuda").to(torch.bfloat16)
    q, k, v = x[:, :4], x[:, 4:5], x[:, 5:]
    cache = Q.kv4_cache(10, 1, 128, 64)
    slots = torch.arange(600, device="cuda")
    Q.kv4_paged_write(cache, k, v, slots)
    i32 = dict(dtype=torch.int32, device="cuda")
    paged = (q[-40:], cache, torch.arange(10, **i32)[None], torch.tensor([600], **i32), torch.tensor([0, 40], **i32), 40)
    cu = torch.tensor([0, 600], **i32)
    return {
        "rope_heads": lambda **s: (Q.rope_heads(q, rotate=True, **s),),
        "kv4_paged_write": lambda **s: (Q.kv4_paged_write(cache, k, v, slots, q=q, **s),),
        "kv4_paged_read": lambda **s: Q.kv4_paged_read(cache, slots, **s),
        "paged_attention": lambda **s: Q.paged_attention(*paged, lse=True, **s),
        "prompt_attention": lambda **s: Q.prompt_attention(q, k, v, cu, lse=True, **s),
    }


@pytest.mark.parametrize("name", ["rope_heads", "kv4_paged_write", "kv4_paged_read", "paged_attention",
                                  "prompt_attention"])
@pytest.mark.parametrize("handle", [False, True])
def test_outputs_are_not_memory_that_the_current_stream_still_uses(name, handle):
    call = _calls()[name]
    want = call()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    let_go = [torch.empty_like(w) for w in want]
    at = {t.data_ptr() for t in let_go}
    torch.cuda._sleep(20_000_000)
    for t in let_go:
        t.fill_(7.0)   # queued behind the sleep; its memory is the current stream's to give again
    del t, let_go
    got = call(stream=s.cuda_stream if handle else s)
    s.synchronize()
    assert not at & {g.data_ptr() for g in got}
    torch.cuda.synchronize()
    assert all(torch.equal(g, w) for g, w in zip(got, want))


@pytest.mark.parametrize("handle", [0, 1, 2])
def test_the_runtimes_own_handles(handle):
    """The default stream as 0 and as the runtime's legacy handle, and the per-thread default stream, which is ordered
    with it."""
    x = torch.randn((96, 4096), generator=torch.Generator("cuda").manual_seed(1), device="cuda").to(torch.bfloat16)
    for call in list(_calls().values()) + [lambda **s: Q.quantize_act(x, 1024, **s)]:
        want = call()
        with torch.cuda.stream(torch.cuda.Stream()):   # not the current stream
            got = call(stream=handle)
        torch.cuda.synchronize()
        assert all(torch.equal(g.view(torch.uint8), w.view(torch.uint8)) for g, w in zip(got, want))
