"""Argument checks of attention over a window and behind shared prefixes (no GPU: no call here reaches a CUDA runtime
function)."""

import ctypes
import math

import pytest
import torch

from paper_2606_07116_gb300 import build as B
from paper_2606_07116_gb300 import offq as Q

P = ctypes.c_void_p
A16 = P(0x10000)
A8 = P(0x10008)
BAD, UNSUP, ALIGN, OK = Q.OFFQ_ERR_INVALID_ARG, Q.OFFQ_ERR_UNSUPPORTED, Q.OFFQ_ERR_MISALIGNED, Q.OFFQ_OK


@pytest.fixture(scope="module")
def lib():
    B.build()
    return Q.load_library()


PAGED_BAD = (dict(dt=9), dict(Tq=-1), dict(Hq=0), dict(H=0), dict(Hq=7), dict(ldq=1000), dict(ldo=1000), dict(B=-1),
             dict(max_q=-1), dict(scale=0.0), dict(scale=math.nan), dict(scale=math.inf), dict(q=None), dict(kc=None),
             dict(kp=None), dict(vc=None), dict(vp=None), dict(table=None), dict(lens=None), dict(cu=None),
             dict(out=None), dict(pages=0), dict(page=0), dict(ldt=-1), dict(wb=-1))
PAGED_UNSUP = (dict(dt=Q.OFFQ_F32), dict(D=96), dict(page=8), dict(page=96), dict(Hq=130, H=2, ldq=1 << 15, ldo=1 << 15),
               dict(B=70000), dict(Tq=(1 << 24) + 1))
PAGED_ALIGN = (dict(q=A8), dict(out=A8), dict(ldq=1028), dict(ldo=1028), dict(kc=A8), dict(vp=A8), dict(ws=A8),
               dict(lse=P(0x10002)), dict(table=P(0x10002)), dict(cu=P(0x10002)), dict(lens=P(0x10002)))
PAGED_OK = (dict(Tq=0, q=None), dict(B=0), dict(max_q=0))


def test_paged_window_argument_checks(lib):
    def call(q=A16, dt=Q.OFFQ_BF16, Tq=4, Hq=8, H=2, D=128, ldq=1024, kc=A16, kp=A16, vc=A16, vp=A16, pages=4, page=16,
             table=A16, ldt=4, lens=A16, cu=A16, B=2, max_q=2, scale=0.1, window=5, sinks=1, out=A16, ldo=1024, lse=None,
             ws=A16, wb=1 << 40):
        return lib.offq_paged_attention_window(q, dt, Tq, Hq, H, D, ldq, kc, kp, vc, vp, pages, page, table, ldt, lens,
                                               cu, B, max_q, scale, window, sinks, out, ldo, lse, ws, wb, None)
    for kw in PAGED_BAD + (dict(window=0), dict(window=-4), dict(sinks=-1)):
        assert call(**kw) == BAD, kw
    for kw in PAGED_UNSUP:
        assert call(**kw) == UNSUP, kw
    for kw in PAGED_ALIGN:
        assert call(**kw) == ALIGN, kw
    for kw in PAGED_OK:
        assert call(**kw) == OK, kw
        assert call(**kw, window=0) == BAD


def test_paged_prefix_argument_checks(lib):
    def call(q=A16, dt=Q.OFFQ_BF16, Tq=4, Hq=8, H=2, D=128, ldq=1024, kc=A16, kp=A16, vc=A16, vp=A16, pages=4, page=16,
             table=A16, ldt=4, lens=A16, cu=A16, B=2, max_q=2, pt=A16, ldp=3, pl=A16, cp=A16, prefixes=1, scale=0.1,
             out=A16, ldo=1024, lse=None, ws=A16, wb=1 << 40):
        return lib.offq_paged_attention_prefix(q, dt, Tq, Hq, H, D, ldq, kc, kp, vc, vp, pages, page, table, ldt, lens,
                                               cu, B, max_q, pt, ldp, pl, cp, prefixes, scale, out, ldo, lse, ws, wb, None)
    for kw in PAGED_BAD + (dict(prefixes=-1), dict(ldp=-1), dict(pt=None), dict(pl=None), dict(cp=None)):
        assert call(**kw) == BAD, kw
    for kw in PAGED_UNSUP + (dict(prefixes=65536),):
        assert call(**kw) == UNSUP, kw
    for kw in PAGED_ALIGN + (dict(pt=P(0x10002)), dict(pl=P(0x10002)), dict(cp=P(0x10002))):
        assert call(**kw) == ALIGN, kw
    for kw in PAGED_OK:
        assert call(**kw) == OK, kw


def test_prefix_workspace_refusals(lib):
    f = lib.offq_paged_attention_prefix_workspace
    assert f(4, 8, 2, 128, 2, 2, -1) == -1 and f(4, 8, 2, 128, 2, 2, 65536) == -1 and f(4, 7, 2, 128, 2, 2, 1) == -1
    assert f(0, 8, 2, 128, 2, 2, 1) == 0 and f(4, 8, 2, 128, 0, 2, 1) == 0 and f(4, 8, 2, 128, 2, 0, 1) == 0


def test_prompt_window_argument_checks(lib):
    def call(q=A16, k=A16, v=A16, dt=Q.OFFQ_BF16, T=4, Hq=8, H=2, D=128, ldq=1024, ldk=256, ldv=256, cu=A16, B=1,
             scale=0.1, window=5, sinks=1, out=A16, ldo=1024, lse=None):
        return lib.offq_prompt_attention_window(q, k, v, dt, T, Hq, H, D, ldq, ldk, ldv, cu, B, scale, window, sinks, out,
                                                ldo, lse, None)
    for kw in (dict(dt=4), dict(T=-1), dict(Hq=9), dict(H=0), dict(ldq=8), dict(ldk=8), dict(ldv=8), dict(ldo=8),
               dict(q=None), dict(k=None), dict(v=None), dict(cu=None), dict(out=None), dict(scale=0.0), dict(B=-1),
               dict(window=0), dict(window=-1), dict(sinks=-1)):
        assert call(**kw) == BAD, kw
    for kw in (dict(dt=Q.OFFQ_F32), dict(D=96), dict(B=70000)):
        assert call(**kw) == UNSUP, kw
    for kw in (dict(q=A8), dict(k=A8), dict(v=A8), dict(out=A8), dict(ldq=1028), dict(ldk=260), dict(ldv=260),
               dict(lse=P(0x10002))):
        assert call(**kw) == ALIGN, kw
    assert call(T=0) == OK and call(B=0) == OK


def test_helpers_refuse_what_does_not_go_together():
    cache = Q.kv4_cache(2, 2, 128, 16, device="cpu")
    q = torch.zeros((2, 4, 128), dtype=torch.bfloat16)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    args = (q, cache, i32(2, 3), i32(2), i32(3), 1)
    good = Q.SharedPrefix(i32(1, 2), i32(1), i32(2))
    for kw in (dict(sinks=4), dict(window=0), dict(window=-1), dict(window=4, sinks=-1), dict(window=4, prefix=good),
               dict(prefix=good._replace(lens=i32(1).long())), dict(prefix=good._replace(cu=i32(3))),
               dict(prefix=good._replace(table=i32(2, 2))), dict(prefix=good._replace(table=i32(2))),
               dict(prefix=good._replace(table=i32(1, 2).long())), dict(prefix=good._replace(table=i32(1, 8)[:, ::2]))):
        with pytest.raises(ValueError):
            Q.paged_attention(*args, **kw)
    kv = torch.zeros((2, 2, 128), dtype=torch.bfloat16)
    for kw in (dict(sinks=4), dict(window=0), dict(window=4, sinks=-1), dict(window=4, causal=False)):
        with pytest.raises(ValueError):
            Q.prompt_attention(q, kv, kv, i32(2), **kw)


class _Recorded:
    """A library that keeps the arguments of each call."""
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 64 if name.endswith("_workspace") else Q.OFFQ_OK
        return call


def test_helpers_reach_the_calls(monkeypatch):
    """Which call a helper makes; windows and sinks past 32 bits are cut; a part of a wider prefix table is copied."""
    lib = _Recorded()
    monkeypatch.setattr(Q, "load_library", lambda: lib)
    monkeypatch.setattr(Q, "_ptr", lambda t: t)
    monkeypatch.setattr(Q, "_stream", lambda s: s)
    Q._workspace_bytes.cache_clear()
    cache = Q.kv4_cache(2, 2, 128, 16, device="cpu")
    q, kv = torch.zeros((2, 4, 128), dtype=torch.bfloat16), torch.zeros((2, 2, 128), dtype=torch.bfloat16)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    args = (q, cache, i32(2, 3), i32(2), i32(3), 1)
    Q.paged_attention(*args, window=1 << 40, sinks=1 << 33)
    assert lib.calls[-1][0] == "offq_paged_attention_window" and lib.calls[-1][1][20:22] == (2 ** 31 - 1, 2 ** 31 - 1)
    wide = i32(2, 9)
    Q.paged_attention(*args, prefix=Q.SharedPrefix(wide[:, 4:], i32(2), i32(3)))
    name, given = lib.calls[-1]
    assert name == "offq_paged_attention_prefix" and given[20] == 5 and given[23] == 2
    assert given[19].is_contiguous() and given[19].data_ptr() != wide[:, 4:].data_ptr()
    assert ("offq_paged_attention_prefix_workspace", (2, 4, 2, 128, 2, 1, 2)) in lib.calls
    Q.paged_attention(*args, prefix=Q.SharedPrefix(i32(0, 5), i32(0), i32(1)))
    assert lib.calls[-1][0] == "offq_paged_attention"
    Q.prompt_attention(q, kv, kv, i32(2), window=7, sinks=2)
    assert lib.calls[-1][0] == "offq_prompt_attention_window" and lib.calls[-1][1][14:16] == (7, 2)
    Q._workspace_bytes.cache_clear()


def test_window_workspace_refusals(lib):
    f = lib.offq_paged_attention_window_workspace
    good = (4, 8, 2, 128, 2, 2, 16, 9, 30, 4)
    for at, x in ((0, -1), (1, 7), (3, 96), (4, -1), (5, -1), (6, 8), (6, 48), (6, 512), (7, -1), (8, 0), (9, -1)):
        assert f(*good[:at], x, *good[at + 1:]) == -1, (at, x)
    for at in (0, 4, 5):
        assert f(*good[:at], 0, *good[at + 1:]) == 0
