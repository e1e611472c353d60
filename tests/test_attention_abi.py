"""Argument checks of the calls between the projections and attention, the rotary table, and the helpers'
own refusals (no GPU: no call here reaches a CUDA runtime function)."""

import ctypes
import math

import numpy as np
import pytest
import torch

import oracle.attention_oracle as A
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


def test_rope_heads_argument_checks(lib):
    def call(x=A16, dt=Q.OFFQ_BF16, T=4, H=8, D=128, ld=1024, pos=A16, table=A16, max_pos=10, rot=128, norm=None,
             eps=1e-6, flags=0, out=A16, odt=Q.OFFQ_BF16, ldo=1024):
        return lib.offq_rope_heads(x, dt, T, H, D, ld, pos, table, max_pos, rot, norm, eps, flags, out, odt, ldo, None)
    for kw in (dict(dt=7), dict(odt=-1), dict(T=-1), dict(H=0), dict(D=0), dict(ld=1000), dict(ldo=1000), dict(x=None),
               dict(out=None), dict(pos=None), dict(table=None), dict(max_pos=0), dict(rot=-2), dict(rot=130),
               dict(rot=33), dict(flags=2), dict(flags=16), dict(eps=-1.0), dict(eps=math.nan)):
        assert call(**kw) == BAD, kw
    for kw in (dict(D=96), dict(D=256, ld=2048, ldo=2048), dict(rot=24), dict(H=70000, ld=1 << 24, ldo=1 << 24)):
        assert call(**kw) == UNSUP, kw
    for kw in (dict(x=A8), dict(out=A8), dict(ld=1028), dict(ldo=1028), dict(table=A8), dict(norm=A8),
               dict(pos=P(0x10002))):
        assert call(**kw) == ALIGN, kw
    assert call(T=0, x=None) == OK


def test_paged_write_argument_checks(lib):
    def call(q=A16, k=A16, v=A16, dt=Q.OFFQ_BF16, T=4, Hq=8, H=2, D=128, ldq=1024, ldk=256, ldv=256, pos=A16,
             table=A16, max_pos=10, rot=128, qn=None, kn=None, eps=1e-6, flags=3, slots=A16, kc=A16, kp=A16, vc=A16,
             vp=A16, pages=4, page=16, qo=A16, odt=Q.OFFQ_BF16, ldqo=1024):
        return lib.offq_kv4_paged_write(q, k, v, dt, T, Hq, H, D, ldq, ldk, ldv, pos, table, max_pos, rot, qn, kn, eps,
                                        flags, slots, kc, kp, vc, vp, pages, page, qo, odt, ldqo, None)
    for kw in (dict(dt=3), dict(T=-1), dict(Hq=-1), dict(H=0), dict(ldq=1000), dict(ldk=128), dict(ldv=128),
               dict(q=None), dict(k=None), dict(v=None), dict(slots=None), dict(kc=None), dict(kp=None), dict(vc=None),
               dict(vp=None), dict(qo=None), dict(odt=9), dict(ldqo=100), dict(pages=0), dict(page=0), dict(flags=16),
               dict(eps=-1.0), dict(pos=None), dict(rot=200)):
        assert call(**kw) == BAD, kw
    for kw in (dict(D=32), dict(page=8), dict(page=48), dict(page=512), dict(rot=8)):
        assert call(**kw) == UNSUP, kw
    for kw in (dict(q=A8), dict(k=A8), dict(v=A8), dict(ldk=260), dict(kc=A8), dict(kp=A8), dict(vc=A8), dict(vp=A8),
               dict(qo=A8), dict(slots=P(0x10004)), dict(qn=A8), dict(kn=A8)):
        assert call(**kw) == ALIGN, kw
    assert call(T=0, k=None) == OK
    assert call(T=0, Hq=0, q=None, qo=None) == OK


def test_paged_read_argument_checks(lib):
    def call(kc=A16, kp=A16, vc=A16, vp=A16, pages=4, page=16, H=2, D=128, slots=A16, T=4, flags=1, ko=A16, vo=A16,
             odt=Q.OFFQ_BF16, ldk=256, ldv=256):
        return lib.offq_kv4_paged_read(kc, kp, vc, vp, pages, page, H, D, slots, T, flags, ko, vo, odt, ldk, ldv, None)
    for kw in (dict(odt=5), dict(T=-1), dict(H=0), dict(pages=0), dict(page=-16), dict(slots=None), dict(kc=None),
               dict(vp=None), dict(ldk=128), dict(ldv=128), dict(flags=2)):
        assert call(**kw) == BAD, kw
    for kw in (dict(D=96), dict(page=24)):
        assert call(**kw) == UNSUP, kw
    for kw in (dict(ko=A8), dict(vo=A8), dict(kc=A8), dict(slots=P(0x10004)), dict(ldk=260)):
        assert call(**kw) == ALIGN, kw
    assert call(T=0) == OK and call(ko=None, vo=None) == OK


def test_paged_attention_argument_checks(lib):
    def call(q=A16, dt=Q.OFFQ_BF16, Tq=4, Hq=8, H=2, D=128, ldq=1024, kc=A16, kp=A16, vc=A16, vp=A16, pages=4, page=16,
             table=A16, ldt=4, lens=A16, cu=A16, B=2, max_q=2, scale=0.1, out=A16, ldo=1024, lse=None, ws=A16,
             wb=1 << 40):
        return lib.offq_paged_attention(q, dt, Tq, Hq, H, D, ldq, kc, kp, vc, vp, pages, page, table, ldt, lens, cu, B,
                                        max_q, scale, out, ldo, lse, ws, wb, None)
    for kw in (dict(dt=9), dict(Tq=-1), dict(Hq=0), dict(H=0), dict(Hq=7), dict(ldq=1000), dict(ldo=1000), dict(B=-1),
               dict(max_q=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf),
               dict(q=None), dict(kc=None), dict(kp=None), dict(vc=None), dict(vp=None), dict(table=None),
               dict(lens=None), dict(cu=None), dict(out=None), dict(pages=0), dict(page=0), dict(ldt=-1), dict(wb=-1)):
        assert call(**kw) == BAD, kw
    for kw in (dict(dt=Q.OFFQ_F32), dict(D=96), dict(page=8), dict(page=96), dict(Hq=130, H=2, ldq=1 << 15, ldo=1 << 15),
               dict(B=70000), dict(Tq=(1 << 24) + 1)):
        assert call(**kw) == UNSUP, kw
    for kw in (dict(q=A8), dict(out=A8), dict(ldq=1028), dict(ldo=1028), dict(kc=A8), dict(vp=A8), dict(ws=A8),
               dict(lse=P(0x10002)), dict(table=P(0x10002))):
        assert call(**kw) == ALIGN, kw
    for kw in (dict(Tq=0, q=None), dict(B=0), dict(max_q=0)):
        assert call(**kw) == OK, kw


def test_prompt_attention_argument_checks(lib):
    def call(q=A16, k=A16, v=A16, dt=Q.OFFQ_BF16, T=4, Hq=8, H=2, D=128, ldq=1024, ldk=256, ldv=256, cu=A16, B=1,
             scale=0.1, causal=1, out=A16, ldo=1024, lse=None):
        return lib.offq_prompt_attention(q, k, v, dt, T, Hq, H, D, ldq, ldk, ldv, cu, B, scale, causal, out, ldo, lse,
                                         None)
    for kw in (dict(dt=4), dict(T=-1), dict(Hq=9), dict(H=0), dict(ldq=8), dict(ldk=8), dict(ldv=8), dict(ldo=8),
               dict(q=None), dict(k=None), dict(v=None), dict(cu=None), dict(out=None), dict(scale=0.0), dict(B=-1)):
        assert call(**kw) == BAD, kw
    for kw in (dict(dt=Q.OFFQ_F32), dict(D=96), dict(B=70000)):
        assert call(**kw) == UNSUP, kw
    for kw in (dict(q=A8), dict(k=A8), dict(v=A8), dict(out=A8), dict(ldq=1028), dict(ldk=260), dict(ldv=260),
               dict(lse=P(0x10002))):
        assert call(**kw) == ALIGN, kw
    assert call(T=0) == OK and call(B=0) == OK


def test_helpers_refuse_other_types_and_shapes():
    cache = Q.kv4_cache(2, 2, 128, 16, device="cpu")
    k = torch.zeros((3, 2, 128), dtype=torch.bfloat16)
    slots = torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError):
        Q.kv4_paged_write(cache, k, k, slots.to(torch.int32))
    with pytest.raises(ValueError):
        Q.kv4_paged_write(cache, k[:, :1], k[:, :1], slots)                  # the cache has two heads
    with pytest.raises(ValueError):
        Q.kv4_paged_write(cache, k, k.to(torch.float16), slots)
    with pytest.raises(ValueError):
        Q.kv4_paged_write(cache, k, k, slots, table=Q.rope_table(8, 64, device="cpu"))   # no positions
    with pytest.raises(ValueError):
        Q.rope_heads(k.transpose(0, 1))                                      # heads not contiguous
    with pytest.raises(ValueError):
        Q.rope_heads(k, norm=torch.ones(2, 64))
    with pytest.raises(ValueError):
        Q.prompt_attention(k, k, k[:2], torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        Q.prompt_attention(k, k, k, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError):
        Q.paged_attention(k, cache, torch.zeros(1, 2), torch.zeros(1, dtype=torch.int32),
                          torch.zeros(2, dtype=torch.int32), 3)
    with pytest.raises(ValueError):
        Q.rope_table(8, 7)
    with pytest.raises(ValueError):
        Q.rope_table(8, 64, scaling="other")


def test_rope_table():
    """Position p turns pair m by p base^(-2m / rot); the scalings by their formulas."""
    rot, n = 64, 300
    m = np.arange(rot // 2)
    f = 10000.0 ** (-2.0 * m / rot)
    p = np.arange(n)[:, None]
    t = Q.rope_table(n, rot, device="cpu").double().numpy()
    assert np.abs(t[:, :32] - np.cos(p * f)).max() <= 2.0 ** -24 and np.abs(t[:, 32:] - np.sin(p * f)).max() <= 2.0 ** -24
    lin = Q.rope_table(n, rot, scaling="linear", factor=4.0, device="cpu").double().numpy()
    assert np.abs(lin[:, :32] - np.cos(p / 4.0 * f)).max() <= 1e-6
    ntk = Q.rope_table(n, rot, scaling="ntk", factor=4.0, device="cpu").double().numpy()
    g = (10000.0 * 4.0 ** (rot / (rot - 2))) ** (-2.0 * m / rot)
    assert np.abs(ntk[:, 32:] - np.sin(p * g)).max() <= 1e-6
    assert abs(g[-1] / f[-1] - 0.25) < 1e-9 and g[0] == f[0]
    yarn = Q.rope_table(n, rot, scaling="yarn", factor=4.0, original_len=4096, device="cpu").double().numpy()
    amp = 0.1 * math.log(4.0) + 1
    assert np.abs(yarn[:, 0] - amp * np.cos(p[:, 0] * f[0])).max() <= 1e-6          # many turns: kept
    assert np.abs(yarn[:, 31] - amp * np.cos(p[:, 0] * f[31] / 4)).max() <= 1e-6    # under one turn: divided


def test_oracle_rotary_keeps_relative_positions():
    """q . k after rotary positions depends on the positions' difference alone (both pair layouts), and H3 keeps it."""
    rng = np.random.default_rng(0)
    q, k = rng.standard_normal((1, 1, 64)), rng.standard_normal((1, 1, 64))
    table = Q.rope_table(64, 32, device="cpu").double().numpy()
    for inter in (False, True):
        dots = []
        for a, b in ((5, 2), (40, 37), (63, 60)):
            x = A.heads(q, np.array([a]), table, interleaved=inter, rotate=True)
            y = A.heads(k, np.array([b]), table, interleaved=inter, rotate=True)
            dots.append(float((x * y).sum()))
        assert np.ptp(dots) < 1e-5


def test_oracle_attention_against_its_definition():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((3, 4, 8)), rng.standard_normal((5, 2, 8)), rng.standard_normal((5, 2, 8))
    out, lse, w = A.attention(q, k, v, 0.3, [0, 2, 9])
    assert np.all(out[0] == 0) and np.all(np.isinf(lse[0]))
    z = 0.3 * k[:2, 1] @ q[1, 3]
    assert np.allclose(out[1, 3], np.exp(z) @ v[:2, 1] / np.exp(z).sum()) and np.isclose(lse[1, 3], np.log(np.exp(z).sum()))
    assert np.allclose(w[2].sum(-1), 1)
