"""GPU parity of attention over the paged 4-bit cache (offq_paged_attention) and inside packed prompts
(offq_prompt_attention) against the float64 oracle.

Tolerances, from the arithmetic (u = 2^-24; e = 2^-8 for bf16, 2^-11 for f16, the unit roundoff):
* A score sums D exact products in fp32. Allowing each addition a whole ulp (tensor cores may truncate) it is
  within 2 D u of its sum of magnitudes; scale, offset and softmax scale add at most 8 u. dz is the largest such
  bound over a row's keys.
* A weight then carries dz, 2^-20 of the exponential, and e where it is rounded to the 16-bit type that the
  product with the values takes; sums over L keys in fp32 add 2 L u. Numerator and denominator: twice that. out
  moves by that relative bound times sum_j w_j |v_j|, and is rounded once (e |out|).
* lse moves by dz + 2^-20 + 2 L u and its own rounding, 2 u |lse|."""

import numpy as np
import pytest
import torch

import oracle.attention_oracle as A
from paper_2606_07116_gb300 import build as B
from paper_2606_07116_gb300 import offq as Q
from parity import U32

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    B.build()
    Q.load_library()


def _check(out, lse, q, k_mag, k, v, v_mag, scale, sees, dt):
    """One sequence's rows against the oracle."""
    D, L, e = q.shape[-1], k.shape[0], UNIT[dt]
    ref, ref_lse, w = A.attention(q, k, v, scale, sees)
    G = q.shape[1] // k.shape[1]
    if L:
        mags = np.stack([np.abs(q[:, h]) @ k_mag[:, h // G].T for h in range(q.shape[1])], 1) * scale
        seen = np.arange(L)[None, None] < np.asarray(sees)[:, None, None]
        dz = (2 * D + 8) * U32 * np.where(seen, mags, 0).max(-1)
        spread = np.stack([w[:, h] @ v_mag[:, h // G] for h in range(q.shape[1])], 1)
    else:
        dz, spread = np.zeros(ref_lse.shape), np.zeros(ref.shape)
    rel = 2 * (dz + 2.0 ** -20 + e + 2 * L * U32)
    tol = rel[..., None] * spread + e * np.abs(ref) + (2.0 ** -24 if dt == "f16" else 0)
    assert np.all(np.isfinite(out))
    worst = np.max(np.abs(out - ref) / (tol + 1e-300)) if out.size else 0
    assert worst <= 1, worst
    empty = np.isinf(ref_lse)
    assert np.array_equal(empty, np.isinf(lse)) and np.all(lse[empty] < 0) and np.all(out[empty] == 0)
    tol = dz + 2.0 ** -20 + 2 * L * U32 + 2 * U32 * np.abs(np.where(empty, 0, ref_lse))
    assert np.all(np.abs(np.where(empty, 0, lse) - np.where(empty, 0, ref_lse)) <= tol)


def _cache(total, H, D, page, seed, k_off=6.0):
    """Pages of random codes with NaN in every (scale, offset) pair; the pairs to put where tokens are."""
    rng = np.random.default_rng(seed)
    codes = [rng.integers(0, 256, (total, H, page, D // 2), dtype=np.uint8) for _ in range(2)]
    for c in codes:  # nibbles 1..15, as the quantizer leaves them
        c[(c & 15) == 0] |= 1
        c[(c >> 4) == 0] |= 16
    pairs = [np.stack([0.3 * np.exp(0.3 * rng.standard_normal((total, H, page))),
                       o * (1 + 0.2 * rng.standard_normal((total, H, page)))], -1).astype(np.float32) for o in (k_off, 0.2)]
    return codes, pairs


def _paged(lens, news, Hq, H, D, page, dt, seed=0, q_pad=0, table_pad=1, k_off=6.0, scale=None):
    rng = np.random.default_rng(seed + 1)
    B_ = len(lens)
    need = [-(-l // page) for l in lens]
    total = sum(need) + 2
    codes, pairs = _cache(total, H, D, page, seed, k_off)
    order = rng.permutation(total)
    width = max(need + [0]) + table_pad
    table = np.full((B_, width), -1, np.int32)
    used = np.zeros((total, page), bool)
    at = 0
    for b in range(B_):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
        for j in range(lens[b]):
            used[table[b, j // page], j % page] = True
    pairs = [np.where(used[:, None, :, None], p, np.float32("nan")) for p in pairs]
    Tq = sum(news)
    qb = torch.from_numpy(rng.standard_normal((Tq, Hq + q_pad, D))).to(DT[dt])
    q = qb.cuda()[:, :Hq]
    cu = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
    cache = Q.KV4Cache(*(torch.from_numpy(x).cuda() for x in (codes[0], pairs[0], codes[1], pairs[1])))
    scale = scale or D ** -0.5
    out, lse = Q.paged_attention(q, cache, torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32).cuda(),
                                 torch.from_numpy(cu).cuda(), max(news + [0]), scale=scale, lse=True)
    assert Q.offq_get_device_status() == Q.OFFQ_OK
    out, lse, q64 = out.cpu().double().numpy(), lse.cpu().double().numpy(), qb[:, :Hq].double().numpy()
    for b in range(B_):
        j = np.arange(lens[b])
        val = []
        for c, p in zip(codes, pairs):
            x, qc, s, o = A.cached(c, p, table[b][j // page], j % page)
            val.append((x, np.abs(qc) * s[..., None] + np.abs(o)[..., None]))
        rows = slice(cu[b], cu[b + 1])
        sees = [lens[b] - news[b] + i + 1 for i in range(news[b])]
        _check(out[rows], lse[rows], q64[rows], val[0][1], val[0][0], val[1][0], val[1][1], scale, sees, dt)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("Hq,H,page", [(8, 8, 16), (8, 2, 64), (5, 1, 32), (16, 1, 128), (24, 2, 256), (6, 2, 16)])
def test_single_tokens(Hq, H, page, dt, D):
    _paged([1, 2, 15, 16, 17, 33, 100, 257, 1000], [1] * 9, Hq, H, D, page, dt, seed=Hq + page)


@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_single_stream_lengths(dt):
    for L in (1, 31, 32, 33, 64, 127, 128, 129, 500, 4097):
        _paged([L], [1], 8, 2, 128, 64, dt, seed=L)


@pytest.mark.parametrize("news", [[2, 1, 3], [4, 4, 4], [9, 1, 17], [33, 5, 0], [64, 128, 129], [200, 1, 70]])
@pytest.mark.parametrize("Hq,H,D,page,dt", [(8, 2, 128, 64, "bf16"), (5, 1, 64, 16, "f16"), (4, 4, 128, 32, "bf16"),
                                            (16, 2, 64, 128, "bf16"), (14, 2, 128, 16, "f16")])
def test_several_new_tokens(news, Hq, H, D, page, dt):
    lens = [n + past for n, past in zip(news, (77, 300, 511))]
    _paged(lens, news, Hq, H, D, page, dt, seed=sum(news) + Hq)


def test_chunk_alone_and_long_past():
    _paged([300], [300], 4, 1, 128, 64, "bf16", seed=1)      # the whole prompt as one chunk
    _paged([2300], [150], 4, 1, 128, 16, "bf16", seed=2)
    _paged([3000, 129], [40, 128], 4, 2, 64, 32, "f16", seed=3)


def test_rows_that_see_nothing_and_empty_sequences():
    """More queries than cached tokens, sequences without tokens or queries: zeros and -inf, no NaN."""
    for dt in ("bf16", "f16"):
        _paged([0, 3, 5, 0, 40], [2, 8, 0, 1, 50], 8, 2, 128, 16, dt, seed=4)
        _paged([0], [1], 4, 4, 64, 64, dt, seed=5)
        _paged([10, 0, 200], [140, 150, 201], 4, 1, 128, 64, dt, seed=6)


def test_strided_queries_and_wide_tables():
    _paged([50, 700], [1, 1], 8, 2, 128, 16, "bf16", seed=7, q_pad=3, table_pad=40)
    _paged([50, 700], [20, 300], 8, 2, 64, 16, "f16", seed=8, q_pad=5, table_pad=9)


def test_large_offsets_and_scores():
    """Offsets far above the residual (what H3 makes of an outlier channel), and scores that saturate the softmax."""
    _paged([600, 33], [1, 1], 8, 2, 128, 64, "bf16", seed=9, k_off=60.0)
    _paged([600, 330], [100, 3], 8, 2, 128, 64, "bf16", seed=10, k_off=60.0)
    _paged([600, 33], [1, 4], 8, 2, 128, 64, "f16", seed=11, scale=3.0)
    _paged([600, 400], [200, 4], 8, 2, 128, 64, "f16", seed=12, scale=3.0)


@pytest.mark.parametrize("new", [1, 100])
def test_offsets_past_32_bits(new):
    """Pages at the far end of a cache whose codes take more than 4 GiB."""
    H, D, page, dt = 8, 128, 256, "bf16"
    total = (1 << 32) // (H * page * (D // 2)) + 8
    L = 700
    codes, pairs = _cache(3, H, D, page, 13)
    cache = Q.kv4_cache(total, H, D, page)
    where = torch.tensor([total - 1, 0, total - 5], device="cuda")
    for t, x in zip(cache, (codes[0], pairs[0], codes[1], pairs[1])):
        t[where] = torch.from_numpy(x).cuda()
    q = torch.randn((new, 8, D), generator=torch.Generator().manual_seed(1)).to(DT[dt])
    out, lse = Q.paged_attention(q.cuda(), cache, where.to(torch.int32)[None].contiguous(),
                                 torch.tensor([L], dtype=torch.int32).cuda(),
                                 torch.tensor([0, new], dtype=torch.int32).cuda(), new, lse=True)
    j = np.arange(L)
    k, kq, ks, ko = A.cached(codes[0], pairs[0], j // page, j % page)
    v, vq, vs, vo = A.cached(codes[1], pairs[1], j // page, j % page)
    _check(out.cpu().double().numpy(), lse.cpu().double().numpy(), q.double().numpy(),
           np.abs(kq) * ks[..., None] + np.abs(ko)[..., None], k, v, np.abs(vq) * vs[..., None] + np.abs(vo)[..., None],
           D ** -0.5, [L - new + i + 1 for i in range(new)], dt)


def _small(news=(1, 1), lens=(40, 70), pages=8, page=16, table=None, Hq=4, H=2, D=128, max_q=None):
    codes, pairs = _cache(pages, H, D, page, 14)
    cache = Q.KV4Cache(*(torch.from_numpy(x).cuda() for x in (codes[0], pairs[0], codes[1], pairs[1])))
    table = torch.tensor([[0, 1, 2, 3, 4], [5, 6, 7, 1, 2]] if table is None else table, dtype=torch.int32).cuda()
    cu = torch.tensor([0, news[0], sum(news)], dtype=torch.int32).cuda()
    q = torch.randn((sum(news), Hq, D), generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).cuda()
    out = torch.full_like(q, 9.0)
    lens = torch.tensor(lens, dtype=torch.int32).cuda()
    Q.paged_attention(q, cache, table, lens, cu, max(news) if max_q is None else max_q, out=out)
    return out


@pytest.mark.parametrize("news", [(1, 1), (90, 3)])
def test_bad_pages_lengths_and_counts_are_reported(news):
    good = _small(news)
    assert Q.offq_get_device_status() == Q.OFFQ_OK
    bad = _small(news, table=[[0, 1, 8, 3, 4], [5, 6, 7, 1, 2]])     # a page past the cache
    assert Q.offq_get_device_status() == Q.OFFQ_ERR_INVALID_ARG
    assert torch.equal(bad[news[0]:], good[news[0]:])                # the other sequence is unharmed
    bad = _small(news, table=[[0, 1, 2, 3, 4], [-2, 6, 7, 1, 2]])
    assert Q.offq_get_device_status() == Q.OFFQ_ERR_INVALID_ARG
    assert torch.equal(bad[:news[0]], good[:news[0]])
    bad = _small(news, lens=(40, 81))                                # past the table
    assert Q.offq_get_device_status() == Q.OFFQ_ERR_INVALID_ARG
    assert torch.equal(bad[:news[0]], good[:news[0]])


def test_more_queries_than_max_q_are_reported():
    good = _small((1, 20))
    assert Q.offq_get_device_status() == Q.OFFQ_OK
    bad = _small((1, 20), max_q=1)
    assert Q.offq_get_device_status() == Q.OFFQ_ERR_INVALID_ARG
    assert torch.equal(bad[:1], good[:1]) and torch.all(bad[1:] == 9.0)


def test_repeated_calls_give_the_same_bits():
    a, b = _small((90, 3)), _small((90, 3))
    assert torch.equal(a, b)
    a, b = _small(), _small()
    assert torch.equal(a, b)


def _prompt(lengths, Hq, H, D, dt, causal=True, seed=0, pad=0, poison=(), outlier=0.0, scale=None):
    rng = np.random.default_rng(seed)
    T = sum(lengths)
    x = rng.standard_normal((T, Hq + 2 * H + pad, D))
    x[:, :Hq + H, 0] += outlier
    cu = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    for b in poison:  # a sequence full of infinities and NaN
        x[cu[b]:cu[b + 1]] = np.where(rng.random(x[cu[b]:cu[b + 1]].shape) < 0.5, np.inf, np.nan)
    t = torch.from_numpy(x).to(DT[dt])
    g, x64 = t.cuda(), t.double().numpy()
    out, lse = Q.prompt_attention(g[:, :Hq], g[:, Hq:Hq + H], g[:, Hq + H:Hq + 2 * H], torch.from_numpy(cu).cuda(),
                                  scale=scale, causal=causal, lse=True)
    assert Q.offq_get_device_status() == Q.OFFQ_OK
    out, lse = out.cpu().double().numpy(), lse.cpu().double().numpy()
    for b, n in enumerate(lengths):
        if b in poison:
            continue
        r = slice(cu[b], cu[b + 1])
        q, k, v = x64[r, :Hq], x64[r, Hq:Hq + H], x64[r, Hq + H:Hq + 2 * H]
        _check(out[r], lse[r], q, np.abs(k), k, v, np.abs(v), scale or D ** -0.5,
               [i + 1 if causal else n for i in range(n)], dt)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("D,dt", [(128, "bf16"), (64, "bf16"), (128, "f16"), (64, "f16")])
@pytest.mark.parametrize("Hq,H", [(2, 2), (4, 1), (6, 2)])
def test_packed_prompts(Hq, H, D, dt, causal):
    _prompt([1, 2, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300], Hq, H, D, dt, causal, seed=Hq)


@pytest.mark.parametrize("n", [1, 100, 513, 1100])
def test_one_prompt(n):
    _prompt([n], 2, 1, 128, "bf16", seed=n)


def test_empty_sequences_and_strides():
    _prompt([0, 5, 0, 0, 200, 0], 4, 2, 128, "bf16", seed=1, pad=3)
    _prompt([3, 0, 140], 4, 2, 64, "f16", causal=False, seed=2, pad=1)


@pytest.mark.parametrize("causal", [True, False])
def test_a_sequence_of_infinities_and_nan_stays_alone(causal):
    for D in (64, 128):
        _prompt([70, 60, 130, 40, 200], 2, 1, D, "bf16", causal, seed=3, poison=(1, 3))


def test_large_scores():
    _prompt([300, 40], 2, 1, 128, "bf16", seed=4, outlier=30.0)
    _prompt([300, 40], 2, 1, 128, "f16", seed=5, scale=4.0)


def test_rows_outside_the_sequences_are_left_alone():
    x = torch.randn((20, 4, 128), generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).cuda()
    out = torch.full((20, 2, 128), 5.0, dtype=torch.bfloat16, device="cuda")
    cu = torch.tensor([4, 9, 15], dtype=torch.int32).cuda()
    Q.prompt_attention(x[:, :2], x[:, 2:3], x[:, 3:4], cu, out=out)
    assert torch.all(out[:4] == 5.0) and torch.all(out[15:] == 5.0) and not torch.any(out[4:15] == 5.0)


def test_a_sequence_past_the_rows_is_reported():
    x = torch.randn((20, 4, 128), generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).cuda()
    good = Q.prompt_attention(x[:, :2], x[:, 2:3], x[:, 3:4], torch.tensor([0, 8, 20], dtype=torch.int32).cuda())
    bad = Q.prompt_attention(x[:, :2], x[:, 2:3], x[:, 3:4], torch.tensor([0, 8, 400], dtype=torch.int32).cuda())
    assert Q.offq_get_device_status() == Q.OFFQ_ERR_INVALID_ARG
    assert torch.equal(bad[:8], good[:8])


def test_another_stream_and_a_graph():
    """Both calls captured into a CUDA graph on their own stream, then replayed over new inputs."""
    Hq, H, D, page, L = 4, 2, 128, 16, 90
    codes, pairs = _cache(6, H, D, page, 15)
    cache = Q.KV4Cache(*(torch.from_numpy(x).cuda() for x in (codes[0], pairs[0], codes[1], pairs[1])))
    table = torch.arange(6, dtype=torch.int32).cuda()[None].contiguous()
    lens, cu = torch.tensor([L], dtype=torch.int32).cuda(), torch.tensor([0, 1], dtype=torch.int32).cuda()
    q = torch.zeros((1, Hq, D), dtype=torch.bfloat16, device="cuda")
    x = torch.zeros((150, Hq + 2 * H, D), dtype=torch.bfloat16, device="cuda")
    cx = torch.tensor([0, 150], dtype=torch.int32).cuda()

    def calls():
        return (Q.paged_attention(q, cache, table, lens, cu, 1),
                Q.prompt_attention(x[:, :Hq], x[:, Hq:Hq + H], x[:, Hq + H:], cx))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        calls()
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            a, b = calls()
    torch.cuda.current_stream().wait_stream(s)
    gen = torch.Generator(device="cuda").manual_seed(1)
    q.normal_(generator=gen)
    x.normal_(generator=gen)
    lens.fill_(77)
    graph.replay()
    torch.cuda.synchronize()
    a2, b2 = calls()
    assert torch.equal(a, a2) and torch.equal(b, b2)
