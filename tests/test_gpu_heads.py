"""GPU parity of norm + rotary + H3 of heads (offq_rope_heads) and of the paged 4-bit cache's write and
read (offq_kv4_paged_write, offq_kv4_paged_read) against the float64 oracle.

Tolerances, from the arithmetic (fp32, u = 2^-24):
* Norm: a balanced sum of D <= 128 squares (7 additions and the square: 8 u relative, halved by the root),
  mean, + eps, root, reciprocal and two products: at most 10 u relative. Rotary: two products and an
  addition, 2 u (|a c| + |b s|). Hadamard: log2 D additions and a product, (log2 D + 1) u of the sum of
  magnitudes over sqrt(D). Together at most HEAD_U = 22 u times A, A the sum of the magnitudes that enter
  the value (the pair's, or with the Hadamard the head's over sqrt(D)); then half an ulp of the output.
* Codes: r / s moves by at most 2 HEAD_U A / s code units (the residual, and the scale over at most 7
  steps) and 8 u of itself, so a code may differ only that near a tie, and then by one step.
* Values read back: s (u - 8) + o takes two roundings, the Hadamard as above."""

import math

import numpy as np
import pytest
import torch

import oracle.attention_oracle as A
from paper_2606_07116_gb300 import build as B
from paper_2606_07116_gb300 import offq as Q
from parity import U32

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
HEAD_U = 22 * U32


@pytest.fixture(scope="module", autouse=True)
def _lib():
    B.build()
    Q.load_library()


def _x(T, H, D, dt, seed, outlier=15.0):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((T, H, D))
    x[:, :, 0] += outlier * (1 + 0.1 * rng.standard_normal((T, H)))
    t = torch.from_numpy(x).to(DT[dt])
    return t.cuda(), t.double().numpy()


def _rotary(T, rot, seed, max_pos=700):
    rng = np.random.default_rng(seed)
    table = Q.rope_table(max_pos, rot)
    pos = rng.integers(0, max_pos, T)
    return (torch.from_numpy(pos.astype(np.int32)).cuda(), table), (pos, table.cpu().double().numpy())


def _magnitude(x, norm, eps, rotate):
    """A of the module's text: bounds the magnitudes that enter each value."""
    y = np.abs(A.norm_heads(x, norm, eps))
    if rotate:
        return np.broadcast_to(1.5 * y.sum(-1, keepdims=True) / math.sqrt(y.shape[-1]), y.shape)
    return y.max(-1, keepdims=True) * 2 * np.ones_like(y)


def _norm(H, D, seed):
    w = (1 + 0.3 * np.random.default_rng(seed).standard_normal((H, D))).astype(np.float32)
    return torch.from_numpy(w).cuda(), w.astype(np.float64)


@pytest.mark.parametrize("T,H,D,rot,interleaved,norm,rotate,dt,odt", [
    (1, 1, 128, 128, False, False, False, "bf16", "bf16"),
    (1, 40, 128, 128, False, True, True, "bf16", "f32"),
    (3, 5, 64, 64, False, True, False, "f16", "f16"),
    (7, 3, 64, 32, True, False, True, "f32", "f32"),
    (33, 12, 128, 64, True, True, True, "f16", "bf16"),
    (65, 7, 128, 96, False, False, False, "f32", "f32"),
    (130, 9, 64, 48, False, True, True, "bf16", "f32"),
    (2, 33, 128, 16, True, False, False, "bf16", "bf16"),
    (5, 2, 128, 0, False, True, True, "f32", "f16"),
    (1501, 24, 128, 128, False, True, True, "bf16", "f32"),
])
def test_rope_heads(T, H, D, rot, interleaved, norm, rotate, dt, odt):
    x, x64 = _x(T, H, D, dt, 3 * T + H)
    (pos, table), (pos64, table64) = _rotary(T, rot, T) if rot else ((None, None), (None, None))
    w, w64 = _norm(H, D, H) if norm else (None, None)
    y = Q.rope_heads(x, pos, table, norm=w, eps=1e-5, interleaved=interleaved, rotate=rotate, out_dtype=DT[odt])
    ref = A.heads(x64, pos64, table64, w64, 1e-5, interleaved, rotate)
    tol = HEAD_U * _magnitude(x64, w64, 1e-5, rotate) + HALF_ULP[odt] * np.abs(ref) + 1e-30
    tol = tol + (2.0 ** -24 if odt == "f16" else 0)
    assert np.all(np.abs(y.cpu().double().numpy() - ref) <= tol)
    assert Q.offq_get_device_status() == Q.OFFQ_OK


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,rot", [(D, rot) for D in (64, 128) for rot in range(16, D + 1, 16)])
def test_every_rotary_size(D, rot, interleaved):
    test_rope_heads(9, 6, D, rot, interleaved, True, True, "bf16", "f32")
    test_rope_heads(2, 5, D, rot, interleaved, False, False, "f16", "f32")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_products_are_rounded_one_by_one(interleaved, D):
    """x c - y s and y c + x s: the bits of three fp32 operations each, for whole and partly rotated heads."""
    for rot in (D, D // 2, D - 16):
        x, _ = _x(50, 6, D, "f32", rot)
        (pos, table), _ = _rotary(50, rot, 7)
        y = Q.rope_heads(x, pos, table, interleaved=interleaved)
        c, s = (t[:, None].cpu() for t in table[pos.long()].split(rot // 2, 1))
        a, b = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
        x, ref = x.cpu(), x.cpu().clone()
        ref[..., a] = x[..., a] * c - x[..., b] * s
        ref[..., b] = x[..., b] * c + x[..., a] * s
        assert torch.equal(y.cpu(), ref)


@pytest.mark.parametrize("D", [64, 128])
def test_codes_are_those_of_single_operations(D):
    """u = rne(fl(x * fl(7 / max|x|))) + 8 to the bit, with as many near ties as 100000 heads have."""
    T, H, page = 12500, 8, 256
    x, _ = _x(T, H, D, "f32", D)
    cache = Q.kv4_cache(-(-T // page), H, D, page)
    slots = torch.arange(T, device="cuda")
    Q.kv4_paged_write(cache, x, x, slots, rotate=False, offset=False)
    p = x * (7.0 / x.abs().amax(-1, keepdim=True))
    u = (torch.round(p) + 8).to(torch.uint8)
    want = u[..., 0::2] | u[..., 1::2] << 4
    for codes in (cache.k_codes, cache.v_codes):
        got = codes.permute(0, 2, 1, 3).reshape(-1, H, D // 2)[:T]
        assert torch.equal(got, want)


def test_rope_heads_in_place_and_strided():
    T, H, D = 37, 6, 128
    x, x64 = _x(T, H + 3, D, "bf16", 5)
    (pos, table), (pos64, table64) = _rotary(T, D, 6)
    part = x[:, 2:2 + H]
    before = x.clone()
    Q.rope_heads(part, pos, table, out=part)
    ref = A.heads(x64[:, 2:2 + H], pos64, table64)
    tol = HEAD_U * _magnitude(x64[:, 2:2 + H], None, 0, False) + HALF_ULP["bf16"] * np.abs(ref)
    assert np.all(np.abs(part.cpu().double().numpy() - ref) <= tol)
    assert torch.equal(x[:, :2], before[:, :2]) and torch.equal(x[:, 2 + H:], before[:, 2 + H:])


def test_a_position_outside_the_table_is_reported_and_leaves_its_rows():
    x, _ = _x(4, 3, 128, "bf16", 1)
    table = Q.rope_table(50, 128)
    pos = torch.tensor([0, 50, -1, 49], dtype=torch.int32, device="cuda")
    out = torch.full((4, 3, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    Q.rope_heads(x, pos, table, out=out)
    assert Q.offq_get_device_status() == Q.OFFQ_ERR_INVALID_ARG
    assert Q.offq_get_device_status() == Q.OFFQ_OK
    assert torch.all(out[1:3] == 7.0)
    good = Q.rope_heads(x[[0, 3]], pos[[0, 3]], table)
    assert torch.equal(out[[0, 3]], good)


def _check_codes(q, s, o, y, mag, offset, rotated_x0=None):
    """q, s, o of the library [T, H, ...] against the oracle's codes of y."""
    qr, sr, orf, r = A.quantize_heads(y, offset)
    err = HEAD_U * mag.max(-1)
    assert np.all(np.abs(s - sr) <= 2 * err / 7 + 8 * U32 * sr)
    assert np.all(np.abs(o - orf) <= err + 8 * U32 * np.abs(orf))
    z = np.abs(np.divide(r, sr[..., None], out=np.zeros_like(r), where=sr[..., None] > 0))
    window = np.divide(4 * err, sr, out=np.zeros_like(sr), where=sr > 0)[..., None] + 8 * 8 * U32
    diff = q != qr
    assert np.all(np.abs(q - qr) <= 1)
    assert np.all(np.abs(z - np.floor(z) - 0.5)[diff] <= np.broadcast_to(window, z.shape)[diff])


@pytest.mark.parametrize("T,Hq,H,D,page,rot,interleaved,norm,rotate,rotate_v,offset,dt", [
    (1, 32, 8, 128, 64, 128, False, True, True, False, True, "bf16"),
    (1, 0, 1, 64, 16, 64, False, False, True, False, True, "f16"),
    (17, 5, 5, 128, 16, 64, True, True, True, True, True, "f32"),
    (33, 3, 3, 64, 32, 32, False, True, False, False, True, "f32"),
    (70, 7, 1, 128, 128, 0, False, False, True, False, False, "bf16"),
    (301, 12, 6, 64, 256, 64, True, False, True, True, True, "f16"),
    (1025, 8, 8, 128, 64, 128, False, True, True, False, True, "f32"),
])
def test_paged_write_and_read(T, Hq, H, D, page, rot, interleaved, norm, rotate, rotate_v, offset, dt):
    pages = -(-T // page) + 2
    cache = Q.kv4_cache(pages, H, D, page)
    for t in cache:
        t.view(torch.uint8).fill_(0xA5)
    qkv, qkv64 = _x(T, Hq + 2 * H, D, dt, T + D)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
    slots = np.random.default_rng(T).permutation(pages * page)[:T]
    (pos, table), (pos64, table64) = _rotary(T, rot, T) if rot else ((None, None), (None, None))
    qw, qw64 = _norm(Hq, D, 1) if norm and Hq else (None, None)
    kw, kw64 = _norm(H, D, 2) if norm else (None, None)
    sl = torch.from_numpy(slots).cuda()
    qo = Q.kv4_paged_write(cache, k, v, sl, pos, table, q=q if Hq else None, q_norm=qw, k_norm=kw, eps=1e-5,
                           interleaved=interleaved, rotate=rotate, rotate_v=rotate_v, offset=offset,
                           out_dtype=torch.float32)
    assert Q.offq_get_device_status() == Q.OFFQ_OK
    x64 = qkv64
    if Hq:
        ref = A.heads(x64[:, :Hq], pos64, table64, qw64, 1e-5, interleaved, rotate)
        tol = HEAD_U * _magnitude(x64[:, :Hq], qw64, 1e-5, rotate) + U32 * np.abs(ref)
        assert np.all(np.abs(qo.cpu().double().numpy() - ref) <= tol)
    kc, kp, vc, vp = (t.cpu().numpy() for t in cache)
    at = (slots // page, slots % page)
    ky = A.heads(x64[:, Hq:Hq + H], pos64, table64, kw64, 1e-5, interleaved, rotate)
    vy = A.heads(x64[:, Hq + H:], rotate=rotate_v)
    for codes, params, y, mag in ((kc, kp, ky, _magnitude(x64[:, Hq:Hq + H], kw64, 1e-5, rotate)),
                                  (vc, vp, vy, _magnitude(x64[:, Hq + H:], None, 0, rotate_v))):
        _, qc, s, o = A.cached(codes, params, *at)
        _check_codes(qc, s, o, y, mag, offset)
    used = np.zeros((pages, page), bool)
    used[at] = True
    for t in (kc, kp.view(np.uint8), vc, vp.view(np.uint8)):
        assert np.all(t.transpose(0, 2, 1, 3)[~used] == 0xA5)  # other slots are left alone

    for odt in ("f32", "bf16", "f16"):
        kr, vr = Q.kv4_paged_read(cache, sl, rotate=rotate, rotate_v=rotate_v, out_dtype=DT[odt])
        for got, codes, params, rot_back in ((kr, kc, kp, rotate), (vr, vc, vp, rotate_v)):
            val = A.cached(codes, params, *at)[0]
            mag = np.abs(val)
            ref = A.hadamard_heads(val) if rot_back else val
            big = 7 * params[at[0], :, at[1], 0].astype(np.float64)[..., None] + np.abs(params[at[0], :, at[1], 1])[..., None]
            tol = (2 * U32 * big * math.sqrt(D) + HEAD_U * mag.sum(-1, keepdims=True) / math.sqrt(D) if rot_back
                   else 2 * U32 * big) + HALF_ULP[odt] * np.abs(ref) + (2.0 ** -24 if odt == "f16" else 0)
            assert np.all(np.abs(got.cpu().double().numpy() - ref) <= tol)


def test_codes_agree_with_the_contiguous_cache_quantizer():
    """The paged write's keys without norm and rotary are offq_kv4_quantize's, up to rounding ties."""
    T, H, D = 200, 4, 128
    x, x64 = _x(T, H, D, "bf16", 9)
    cache = Q.kv4_cache(2, H, D, 128)
    Q.kv4_paged_write(cache, x, x, torch.arange(T, device="cuda"))
    codes, scale, off = Q.kv4_quantize(x)
    got = cache.k_codes.transpose(1, 2).reshape(256, H, D // 2)[:T]
    diff = A.unpack_codes(got.cpu().numpy()) - A.unpack_codes(codes.cpu().numpy())
    assert np.abs(diff).max() <= 1 and np.count_nonzero(diff) <= 1e-4 * diff.size
    par = cache.k_params.transpose(1, 2).reshape(256, H, 2)[:T]
    assert torch.allclose(par[..., 0], scale, rtol=1e-5, atol=0) and torch.allclose(par[..., 1], off, rtol=1e-5, atol=1e-6)


def test_slots_outside_the_cache():
    H, D, page = 2, 128, 16
    x, _ = _x(4, H, D, "bf16", 2)
    cache = Q.kv4_cache(2, H, D, page)
    for t in cache:
        t.view(torch.uint8).zero_()
    slots = torch.tensor([-1, 3, -7, 20], device="cuda")
    Q.kv4_paged_write(cache, x, x, slots)
    assert Q.offq_get_device_status() == Q.OFFQ_OK  # negative slots are padding
    written = (cache.k_params[..., 0] != 0).sum().item()
    assert written == 2 * H
    Q.kv4_paged_write(cache, x, x, torch.tensor([1, 32, 2, 1 << 40], device="cuda"))
    assert Q.offq_get_device_status() == Q.OFFQ_ERR_INVALID_ARG
    k, v = Q.kv4_paged_read(cache, torch.tensor([-1, 3, 32], device="cuda"))
    assert Q.offq_get_device_status() == Q.OFFQ_ERR_INVALID_ARG
    assert torch.all(k[0] == 0) and torch.all(v[2] == 0) and torch.any(k[1] != 0)


def test_zero_and_constant_heads():
    """All-zero heads quantize to scale 0 and code 8; a constant value head to its mean alone."""
    x = torch.zeros((2, 1, 64), dtype=torch.float16, device="cuda")
    v = torch.full_like(x, 1.5)
    cache = Q.kv4_cache(1, 1, 64, 16)
    Q.kv4_paged_write(cache, x, v, torch.arange(2, device="cuda"))
    assert torch.all(cache.k_codes[0, 0, :2] == 0x88) and torch.all(cache.v_codes[0, 0, :2] == 0x88)
    assert torch.all(cache.k_params[0, 0, :2] == 0)
    assert torch.equal(cache.v_params[0, 0, :2].cpu(), torch.tensor([[0.0, 1.5]] * 2))


def test_no_tokens():
    cache = Q.kv4_cache(1, 2, 128, 16)
    x = torch.empty((0, 2, 128), dtype=torch.bfloat16, device="cuda")
    assert Q.rope_heads(x).shape == (0, 2, 128)
    slots = torch.empty((0,), dtype=torch.int64, device="cuda")
    assert Q.kv4_paged_write(cache, x, x, slots) is None
    assert Q.kv4_paged_read(cache, slots)[0].shape == (0, 2, 128)


def test_another_stream():
    """Written and read on a stream that is not the current one."""
    s = torch.cuda.Stream()
    x, x64 = _x(64, 4, 128, "bf16", 8)
    cache = Q.kv4_cache(4, 4, 128, 16)
    slots = torch.arange(64, device="cuda")
    s.wait_stream(torch.cuda.current_stream())
    Q.kv4_paged_write(cache, x, x, slots, stream=s)
    s.synchronize()
    ref = A.quantize_heads(x64)
    val = A.cached(cache.v_codes.cpu().numpy(), cache.v_params.cpu().numpy(), np.arange(64) // 16, np.arange(64) % 16)[0]
    step = ref[1][..., None]
    assert np.all(np.abs(val - x64) <= 0.5001 * step + 1e-5)
