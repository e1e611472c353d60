// Attention of few query rows over the paged 4-bit cache (offq_paged_attention with up to 16 rows
// n * Hq / H per sequence and key head: single tokens, drafted tokens).
//
// Every cached byte is read once for all rows of its key head, so the cache bounds it: D + 16 bytes per
// token and head (144 at D = 128) against 4 D multiply-adds per row.
//
// Work is a list of 32-token stages, sequence by sequence, head by head. The CTAs (one per SM) take equal
// contiguous shares of it, the warps of a CTA equal shares of those: any mix of lengths loads the chip
// evenly and in one wave. A warp that holds a whole (sequence, head) writes its output; parts are joined
// in shared memory at the CTA's end, and what crosses CTAs in a second small kernel (at most a first and a
// last part per CTA: the workspace does not grow with the batch).
//
// A warp stages its tokens itself, by asynchronous copies of 16 bytes a lane (a head's tokens of a page are contiguous)
// into a ring of its own, and all lanes read fragments for warp-level MMAs of 16 tokens:
//   S^T [tokens x rows]  = codes K [16 x 16 channels] * Q^T [16 channels x 8 rows]
//   O^T [channels x rows] += codes V^T [16 channels x 16 tokens] * P^T [16 tokens x 8 rows]
// with the rows on the MMA's 8-wide side, as there are few. Channels may be contracted in any order and tokens
// too, so fragments are what a lane finds in its 16-byte reads. A key's nibble u = q + 8 becomes the 16-bit float
// 16 + u (its bits placed below the exponent of 16.0), exact: half a shift and half a logical operation a code; the 24
// on top of q leaves as -24 times the query's sum. A value's becomes 1024 + u or 1024 + 16 u as a half (one shift
// for 8 codes) and one packed multiply-add takes it to q: left in, the bias would be summed over the whole context, and
// what is left of values that average out would be its rounding errors.
//   z_j = s_j (acc_j - 24 Q) + o_j Q,  Q = sum of the query;   out = (O + sum p o_v) / sum p,
// O summed with P' = p s_v as halves, p = 2^(z - m). The reference m follows the largest z_j + log2(s_v), so that P'
// fits a half whatever the values' size; it moves only when some P' passes 2^8 (or p 2^32). Scores are taken relative
// to it as they are made; a stage that must move it, or has tokens that some row does not see, does its softmax again.
//
// Copies of 16 bytes a lane rather than one lane's bulk copies: those cost more instructions than they save (4 streams of 65536
// tokens 233 against 212 us; pages of 16 tokens, 64 streams of 1 to 8191, 96 against 84). 16 warps of 8 rows (128 registers, two
// stages each) or 8 of 16 rows (250, four stages): more warps spill (12 of 16 rows: 50 us where 8 take 36).
// Measured: 4 x 65536 tokens, 32 heads of 128: 212 us, 5.7 TB/s, integer pipe and issue slots at 60 %. 64 streams of 1 to 8191,
// 64 heads on 8: 84 us, 4.0 TB/s, 17 us of them whatever the lengths. 16 x 4 tokens over 500 to 6000: 36 us.
#include <algorithm>
#include <type_traits>

#include "attn.cuh"

namespace {

using namespace offq;

constexpr int kTile = 32;   // tokens per stage
constexpr float kBias = 24.0f;
constexpr int kLeastStages = 8;   // of a CTA

template <int D, int NT>
struct FewLayout {
  static constexpr int kWarps = NT == 1 ? 16 : 8;   // as many as registers allow
  static constexpr int kStages = NT == 1 ? 2 : 4;
  static constexpr int kCodeBytes = kTile * D / 2;
  static constexpr int kStageBytes = 2 * kCodeBytes + 2 * kTile * 8;
  static constexpr int kRows = 8 * NT;
  static constexpr int kRing = kStages * kStageBytes;            // a warp's ring; its last part goes there too
  static constexpr int kPartFloats = kRows * (D + 2);            // O, then m and l
  static constexpr int kPartBytes = kPartFloats * 4;
  static constexpr int kPartOff = kWarps * kRing;                // the warps' first parts
  static constexpr int kCtrlOff = kPartOff + kWarps * kPartBytes;
  static constexpr int kBytes = kCtrlOff + 2048;
  static_assert(kPartBytes <= kRing, "a part fits into its warp's ring");
  static_assert(kBytes <= 232448, "shared memory");
};

// Control block behind the parts.
template <int D, int NT>
struct FewCtrl {
  long long scan[FewLayout<D, NT>::kWarps];
  long long start[FewLayout<D, NT>::kWarps];  // unit offset inside sequence seq
  int seq[FewLayout<D, NT>::kWarps];
  int4 part[2 * FewLayout<D, NT>::kWarps];    // (sequence or -1, head, first stage, last stage) of each part
};

__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, bool half) {
  if (half)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// 16 bytes to shared memory, past the L1; a warp's copies up to commit() are one group.
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void wait_but() {  // for all groups but the last N
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

template <int W>
struct Words {
  uint32_t w[W];
};
template <int W>
__device__ __forceinline__ Words<W> lds(uint32_t addr) {
  Words<W> r;
  if constexpr (W == 4)
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]) : "r"(addr) : "memory");
  else if constexpr (W == 2)
    asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=r"(r.w[0]), "=r"(r.w[1]) : "r"(addr) : "memory");
  else
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(r.w[0]) : "r"(addr) : "memory");
  return r;
}

// Stages of a sequence: none without queries (or with more rows than this form takes), one at least with.
__device__ __forceinline__ int stages_of(const AttnArgs& a, const PagedSeq& s) {
  if (s.n == 0 || s.n * a.G > a.few_rows) return 0;
  return max(1, (s.len + kTile - 1) / kTile);
}

// Header of a part that crosses CTAs: its head's (sequence, head) as one number, negative for none, whether it reaches
// its sequence's last stage, and the sequence's first query row and rows per key head.
struct PartHead {
  int id, ends, first, rows;
};

// The workspace: per CTA two headers (a part begun by an earlier CTA, a part left to later ones), then their
// sums, rows x D floats, maxima and weight sums.
template <int D, int NT>
__device__ __forceinline__ PartHead* part_head(void* ws, int cta, int which) {
  return static_cast<PartHead*>(ws) + 2 * cta + which;
}
template <int D, int NT>
__device__ __forceinline__ float* part_sums(void* ws, int ctas, int cta, int which) {
  return reinterpret_cast<float*>(static_cast<PartHead*>(ws) + 2 * ctas) +
         static_cast<int64_t>(2 * cta + which) * FewLayout<D, NT>::kPartFloats;
}

// Channels d .. d + 7 of row r of (sequence starting at query row `first`, head h).
template <int D, typename T>
__device__ __forceinline__ void write_out8(const AttnArgs& a, int first, int h, int r, int d, const float (&v)[8]) {
  const int64_t t = static_cast<int64_t>(first) + r / a.G;
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (std::is_same<T, __nv_bfloat16>::value) {
      w[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
    } else {
      w[i] = pack_f16(v[2 * i], v[2 * i + 1]);
    }
  }
  *reinterpret_cast<uint4*>(static_cast<T*>(a.out) + t * a.ld_out + static_cast<int64_t>(h * a.G + r % a.G) * D + d) =
      make_uint4(w[0], w[1], w[2], w[3]);
}

template <int D, int NT, typename T>
__global__ void __launch_bounds__(FewLayout<D, NT>::kWarps * 32, 1) paged_few_kernel(const AttnArgs a) {
  using L = FewLayout<D, NT>;
  constexpr bool kHalf = std::is_same<T, __half>::value;
  constexpr int kThreads = L::kWarps * 32;
  constexpr int kMt = D / 16;    // 16-channel tiles of O^T
  constexpr int kKw = D / 32;    // words of 8 codes a lane holds of a key
  constexpr int kVw = D / 64;    // and of a value
  extern __shared__ __align__(16) uint8_t smem[];
  auto* ctrl = reinterpret_cast<FewCtrl<D, NT>*>(smem + L::kCtrlOff);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
  const uint32_t ring = smem_u32(smem) + warp * L::kRing;
  if (tid < 2 * L::kWarps) ctrl->part[tid] = make_int4(-1, 0, 0, 0);
  griddep_wait();
  griddep_launch_dependents();

  // The whole work, this CTA's share and its warps' places in it.
  long long mine = 0;
  for (int b = tid; b < a.B; b += kThreads) {
    const PagedSeq s = paged_seq(a, b);
    if (s.bad && blockIdx.x == 0) *a.status = OFFQ_ERR_INVALID_ARG;
    mine += static_cast<long long>(stages_of(a, s)) * a.H;
  }
  auto warp_sum = [&](long long v) {
#pragma unroll
    for (int m = 16; m > 0; m >>= 1) v += __shfl_xor_sync(kAllLanes, v, m);
    return v;
  };
  const long long wsum = warp_sum(mine);
  if (lane == 0) ctrl->scan[warp] = wsum;
  __syncthreads();
  long long total = 0;
#pragma unroll
  for (int i = 0; i < L::kWarps; ++i) total += ctrl->scan[i];
  // Little work goes to fewer CTAs, some stages each: their warps take them at once, and joining inside a CTA is cheaper.
  const long long ctas = min((total + kLeastStages - 1) / kLeastStages, static_cast<long long>(gridDim.x));
  const long long lo = blockIdx.x < ctas ? total * blockIdx.x / ctas : 0;
  const long long hi = blockIdx.x < ctas ? total * (blockIdx.x + 1) / ctas : 0;
  PartHead* heads = part_head<D, NT>(a.workspace, blockIdx.x, 0);
  if (lo == hi) {
    if (tid < 2) heads[tid] = PartHead{-1, 0, 0, 0};
    return;
  }
  long long before = 0;
  for (int base = 0; base < a.B && before < hi; base += kThreads) {
    long long val = 0;
    if (base + tid < a.B) val = static_cast<long long>(stages_of(a, paged_seq(a, base + tid))) * a.H;
    long long incl = val;
#pragma unroll
    for (int m = 1; m < 32; m <<= 1) {
      const long long o = __shfl_up_sync(kAllLanes, incl, m);
      if (lane >= m) incl += o;
    }
    __syncthreads();
    if (lane == 31) ctrl->scan[warp] = incl;
    __syncthreads();
    long long chunk = 0;
#pragma unroll
    for (int i = 0; i < L::kWarps; ++i) {
      if (i < warp) incl += ctrl->scan[i];
      chunk += ctrl->scan[i];
    }
    const long long first = before + incl - val;
#pragma unroll 1
    for (int k = 0; k < L::kWarps; ++k) {
      const long long at = lo + (hi - lo) * k / L::kWarps;
      if (at >= first && at < first + val) {
        ctrl->seq[k] = base + tid;
        ctrl->start[k] = at - first;
      }
    }
    before += chunk;
  }
  __syncthreads();

  const long long w0 = lo + (hi - lo) * warp / L::kWarps, w1 = lo + (hi - lo) * (warp + 1) / L::kWarps;
  int todo = static_cast<int>(w1 - w0), ahead = todo;  // stages to compute, to issue
  if (todo > 0) {
    int b = ctrl->seq[warp];
    PagedSeq s = paged_seq(a, b);
    int stages = stages_of(a, s);
    int h = static_cast<int>(ctrl->start[warp] / stages), t = static_cast<int>(ctrl->start[warp] % stages);

    // Where the copies are: they run ahead across heads and sequences.
    int pb = b, ph = h, pt = t, pstages = stages, plen = s.len, window = -64, entry = 0;
    int64_t page_row = -1;   // first row of the page the copies are in
    bool turn = true;        // that page is not known yet
    uint32_t missing = 0;    // bit 2 slot + half: that half of the slot's stage has no page
    auto find_page = [&](int tok) {  // first row of the page of token tok, or -1
      const int index = tok >> a.page_shift;
      if (index < window || index >= window + 32) {
        window = index;
        entry = static_cast<int64_t>(index + lane) << a.page_shift < plen
                    ? __ldg(a.table + static_cast<int64_t>(pb) * a.ld_table + index + lane) : 0;
      }
      const int page = __shfl_sync(kAllLanes, entry, index - window);
      if (page >= 0 && page < a.pages) return (static_cast<int64_t>(page) * a.H + ph) << a.page_shift;
      if (lane == 0) *a.status = OFFQ_ERR_INVALID_ARG;
      return static_cast<int64_t>(-1);
    };
    auto copy = [&](uint32_t stage, int half, int64_t row) {  // the codes of 16 tokens
#pragma unroll
      for (int i = 0; i < D / 64; ++i) {
        const uint32_t at = (i * 32 + lane) * 16;
        copy16(stage + half * 8 * D + at, a.k_codes + row * (D / 2) + at);
        copy16(stage + L::kCodeBytes + half * 8 * D + at, a.v_codes + row * (D / 2) + at);
      }
    };
    auto issue = [&](int slot) {
      const uint32_t stage = ring + slot * L::kStageBytes;
      const int tok = pt * kTile, in_page = tok & ((1 << a.page_shift) - 1);
      int64_t r0, r1;  // first rows of the stage's halves, or -1
      if (a.page_shift >= 5) {
        if (turn || in_page == 0) page_row = tok < plen ? find_page(tok) : -1;
        turn = false;
        r0 = page_row < 0 ? -1 : page_row + in_page;
        r1 = page_row < 0 ? -1 : r0 + 16;
      } else {  // two pages of 16 tokens
        r0 = tok < plen ? find_page(tok) : -1;
        r1 = tok + 16 < plen ? find_page(tok + 16) : -1;
      }
      missing &= ~(3u << (2 * slot));
      missing |= ((r0 < 0 ? 1u : 0u) | (r1 < 0 ? 2u : 0u)) << (2 * slot);
      if (r0 >= 0) copy(stage, 0, r0);
      if (r1 >= 0) copy(stage, 1, r1);
      // Scale and offset pairs: 8 lanes for the keys of each half, 8 for the values.
      const int64_t r = lane & 8 ? r1 : r0;
      if (r >= 0) copy16(stage + 2 * L::kCodeBytes + lane * 16, (lane & 16 ? a.v_params : a.k_params) + r * 2 + (lane & 7) * 4);
      if (--ahead > 0 && ++pt == pstages) {
        pt = 0;
        turn = true;
        if (++ph == a.H) {
          ph = 0;
          window = -64;
          PagedSeq n;
          do {
            n = paged_seq(a, ++pb);
            pstages = stages_of(a, n);
          } while (pstages == 0);
          plen = n.len;
        }
      }
    };
#pragma unroll
    for (int i = 0; i < L::kStages; ++i) {
      if (ahead > 0) issue(i);
      commit();
    }

    const int tok_k = (g & ~1) + ((g & 1) ^ ((g >> 1) & 1));              // token of score row g (of 8)
    const int tok_v0 = 2 * c + (c & 1), tok_v1 = 2 * c + 1 - (c & 1);     // tokens of weight rows 2c, 2c + 1
    const float sc = a.scale * kLog2e;
    uint32_t qf[NT][2 * (D / 16)];
    float qs[NT][2], m[NT][2], l[NT][2], w[NT][2], o[NT][kMt][4];
    int sees[NT][2], sees_least = 0, t_first = t, rows = 0;
    bool begin = true, first_part = true;
#pragma unroll 1
    for (int it = 0; it < todo; ++it) {
      const int slot = it % L::kStages;
      if (begin) {
        begin = false;
        t_first = t;
        rows = s.n * a.G;
        sees_least = max(0, s.len - s.n + 1);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const int r = 8 * nt + g;
          const T* src = static_cast<const T*>(a.q) + (static_cast<int64_t>(s.first) + r / a.G) * a.ld_q +
                         static_cast<int64_t>(h * a.G + r % a.G) * D + c * (D / 4);
          float sum = 0.f;
#pragma unroll
          for (int i = 0; i < kKw; ++i) {
            const uint4 u = r < rows ? __ldg(reinterpret_cast<const uint4*>(src) + i) : make_uint4(0u, 0u, 0u, 0u);
            qf[nt][4 * i] = __byte_perm(u.x, u.z, 0x5410);
            qf[nt][4 * i + 1] = __byte_perm(u.x, u.z, 0x7632);
            qf[nt][4 * i + 2] = __byte_perm(u.y, u.w, 0x5410);
            qf[nt][4 * i + 3] = __byte_perm(u.y, u.w, 0x7632);
            const uint32_t x[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              if constexpr (kHalf) {
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&x[k]));
                sum += f.x + f.y;
              } else {
                sum += __uint_as_float(x[k] << 16) + __uint_as_float(x[k] & 0xFFFF0000u);
              }
            }
          }
          sum += __shfl_xor_sync(kAllLanes, sum, 1);
          sum += __shfl_xor_sync(kAllLanes, sum, 2);
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            qs[nt][j] = __shfl_sync(kAllLanes, sum, 4 * (2 * c + j));
            l[nt][j] = w[nt][j] = 0.f;
            const int rr = 8 * nt + 2 * c + j;
            sees[nt][j] = rr < rows ? max(0, min(s.len, s.len - s.n + rr / a.G + 1)) : 0;
            m[nt][j] = sees[nt][j] > 0 ? -INFINITY : 0.f;  // a row without keys has no maximum to wait for
          }
#pragma unroll
          for (int mt = 0; mt < kMt; ++mt)
#pragma unroll
            for (int k = 0; k < 4; ++k) o[nt][mt][k] = 0.f;
        }
      }
      wait_but<L::kStages - 1>();
      __syncwarp();
      const uint32_t stage = ring + slot * L::kStageBytes;
      const uint32_t gone = missing >> (2 * slot) & 3u;

      // Scores of 32 tokens: rows g and g + 8 of each 16, columns 2c and 2c + 1 of each 8 query rows.
      float acc[2][NT][4] = {}, p[2][NT][4], pv[2][NT][4];
      float sk[2][2], bk[2][2], sv[2][2], ov[2][2];   // [half][row]: z = sk acc + bk Q; value scale and offset
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const uint32_t at = stage + (half * 16 + tok_k) * (D / 2) + c * (D / 8);
        const Words<kKw> k0 = lds<kKw>(at), k1 = lds<kKw>(at + 8 * (D / 2));
#pragma unroll
        for (int i = 0; i < kKw; ++i) {
#pragma unroll
          for (int n = 0; n < 4; n += 2) {
            const uint32_t f[4] = {widen<T>(k0.w[i], n), widen<T>(k1.w[i], n), widen<T>(k0.w[i], n + 1),
                                   widen<T>(k1.w[i], n + 1)};
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma16816(acc[half][nt], f, qf[nt][4 * i + n], qf[nt][4 * i + n + 1], kHalf);
          }
        }
        const uint32_t par = stage + 2 * L::kCodeBytes + (half * 16 + tok_k) * 8;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const Words<2> k = lds<2>(par + 64 * i), v = lds<2>(par + kTile * 8 + 64 * i);
          sk[half][i] = __uint_as_float(k.w[0]) * sc;
          bk[half][i] = fmaf(-kBias, sk[half][i], __uint_as_float(k.w[1]) * sc);
          sv[half][i] = __uint_as_float(v.w[0]);
          ov[half][i] = __uint_as_float(v.w[1]);
        }
      }
      bool redo = (t + 1) * kTile > sees_least || gone != 0;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float top = -INFINITY, most = 0.f;
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float x = fmaf(sk[half][k >> 1], acc[half][nt][k], fmaf(bk[half][k >> 1], qs[nt][k & 1], -m[nt][k & 1]));
            top = fmaxf(top, x);
            p[half][nt][k] = ex2(x);
            pv[half][nt][k] = p[half][nt][k] * sv[half][k >> 1];
            most = fmaxf(most, pv[half][nt][k]);
          }
        redo |= !(top <= 32.f) || !(most <= 256.f);
      }
      if (__any_sync(kAllLanes, redo)) {
        float lift[2][2];
        bool none[2][2];
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int i = 0; i < 2; ++i) {  // what nobody sees may hold anything
            none[half][i] = t * kTile + half * 16 + tok_k + 8 * i >= s.len || (gone >> half & 1u);
            if (none[half][i]) sv[half][i] = ov[half][i] = 0.f;
            lift[half][i] = fmaxf(__log2f(sv[half][i]), kLeastLog2);
          }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float keep[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            float top = -INFINITY;
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const int k = 2 * i + j;
                float z = fmaf(sk[half][i], acc[half][nt][k], bk[half][i] * qs[nt][j]);
                if (none[half][i] || t * kTile + half * 16 + tok_k + 8 * i >= sees[nt][j]) z = -INFINITY;
                acc[half][nt][k] = z;
                top = fmaxf(top, z + lift[half][i]);
              }
#pragma unroll
            for (int k = 4; k < 32; k <<= 1) top = fmaxf(top, __shfl_xor_sync(kAllLanes, top, k));
            top = fmaxf(top, m[nt][j]);
            keep[j] = m[nt][j] == -INFINITY ? 0.f : ex2(m[nt][j] - top);
            m[nt][j] = top;
            l[nt][j] *= keep[j];
            w[nt][j] *= keep[j];
            const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const int k = 2 * i + j;
                p[half][nt][k] = ex2(acc[half][nt][k] - ref);
                pv[half][nt][k] = p[half][nt][k] * sv[half][i];
              }
          }
#pragma unroll
          for (int mt = 0; mt < kMt; ++mt) {
            o[nt][mt][0] *= keep[0];
            o[nt][mt][1] *= keep[1];
            o[nt][mt][2] *= keep[0];
            o[nt][mt][3] *= keep[1];
          }
        }
      }

      // Sums, and O^T += V^T P^T.
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        uint32_t pt0[NT], pt1[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            l[nt][k & 1] += p[half][nt][k];
            w[nt][k & 1] = fmaf(p[half][nt][k], ov[half][k >> 1], w[nt][k & 1]);
          }
          pt0[nt] = transpose8x8(pack_f16(pv[half][nt][0], pv[half][nt][1]));
          pt1[nt] = transpose8x8(pack_f16(pv[half][nt][2], pv[half][nt][3]));
        }
        const uint32_t at = stage + L::kCodeBytes + half * 16 * (D / 2) + g * (D / 16);
        const Words<kVw> va = lds<kVw>(at + tok_v0 * (D / 2)), vb = lds<kVw>(at + tok_v1 * (D / 2));
        const Words<kVw> vc = lds<kVw>(at + (tok_v0 + 8) * (D / 2)), vd = lds<kVw>(at + (tok_v1 + 8) * (D / 2));
#pragma unroll
        for (int i = 0; i < kVw; ++i) {
#pragma unroll
          for (int part = 0; part < 2; ++part) {
            const uint32_t x = __byte_perm(va.w[i], vb.w[i], part ? 0x7632 : 0x5410);
            const uint32_t y = __byte_perm(vc.w[i], vd.w[i], part ? 0x7632 : 0x5410);
#pragma unroll
            for (int n = 0; n < 2; ++n) {
              uint32_t f[4];
              widen_signed(n ? x >> 8 : x, f[0], f[1]);
              widen_signed(n ? y >> 8 : y, f[2], f[3]);
              const int mt = 4 * i + 2 * part + n;
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) mma16816(o[nt][mt], f, pt0[nt], pt1[nt], true);
            }
          }
        }
      }
      __syncwarp();
      if (ahead > 0) issue(slot);
      commit();  // with nothing in it too: a stage is as many groups back as the ring is long

      ++t;
      if (t < stages && it + 1 < todo) continue;
      // The end of this head's stages, or of the warp's.
      const bool complete = t_first == 0 && t == stages;
      float* part = reinterpret_cast<float*>(first_part ? smem + L::kPartOff + warp * L::kPartBytes
                                                        : smem + warp * L::kRing);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
          for (int k = 4; k < 32; k <<= 1) {
            l[nt][j] += __shfl_xor_sync(kAllLanes, l[nt][j], k);
            w[nt][j] += __shfl_xor_sync(kAllLanes, w[nt][j], k);
          }
          const int r = 8 * nt + 2 * c + j;
          if (complete) {
            if (r < rows) {
              const float inv = l[nt][j] > 0.f ? __fdividef(1.f, l[nt][j]) : 0.f;
#pragma unroll
              for (int q8 = 0; q8 < kMt / 4; ++q8) {
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = (o[nt][4 * q8 + e / 2][j + 2 * (e & 1)] + w[nt][j]) * inv;
                write_out8<D, T>(a, s.first, h, r, g * (D / 8) + 8 * q8, v);
              }
              if (g == 0) write_lse(a, s.first, h, r, m[nt][j], l[nt][j]);
            }
          } else {
#pragma unroll
            for (int e = 0; e < D / 8; ++e) part[r * D + g * (D / 8) + e] = o[nt][e / 2][j + 2 * (e & 1)] + w[nt][j];
            if (g == 0) {
              part[L::kRows * D + r] = m[nt][j];
              part[L::kRows * D + L::kRows + r] = l[nt][j];
            }
          }
        }
      }
      if (!complete && lane == 0) ctrl->part[2 * warp + (first_part ? 0 : 1)] = make_int4(b, h, t_first, t == stages ? -1 : t);
      first_part = false;
      begin = true;
      if (it + 1 < todo) {
        t = 0;
        if (++h == a.H) {
          h = 0;
          do {
            s = paged_seq(a, ++b);
            stages = stages_of(a, s);
          } while (stages == 0);
        }
      }
    }
  }

  // Parts of the same head, in order of their stages, into one: an output where they are all of it, else a part
  // for the joining kernel. Each warp looks at all of them at once, a lane a part.
  __syncthreads();
  constexpr int kParts = 2 * L::kWarps;
  static_assert(kParts <= 32, "a lane for each part");
  const int4 mypart = lane < kParts ? ctrl->part[lane] : make_int4(-1, 0, 0, 0);
  const int my_id = mypart.x < 0 ? -1 : mypart.x * a.H + mypart.y;
  uint32_t left = __ballot_sync(kAllLanes, my_id >= 0);
  bool have0 = false, have1 = false;
  while (left != 0) {
    const int i = __ffs(left) - 1;
    const int id = __shfl_sync(kAllLanes, my_id, i), b = __shfl_sync(kAllLanes, mypart.x, i);
    const uint32_t same = __ballot_sync(kAllLanes, my_id == id);
    const int begins = __shfl_sync(kAllLanes, mypart.z, i), last = __shfl_sync(kAllLanes, mypart.w, 31 - __clz(same));
    left &= ~same;
    const bool complete = begins == 0 && last < 0;
    const int which = begins == 0 ? 1 : 0, h = id - b * a.H;
    float* dst = part_sums<D, NT>(a.workspace, gridDim.x, blockIdx.x, which);
    const PagedSeq s = paged_seq(a, b);
    if (!complete) (which ? have1 : have0) = true;
    if (!complete && tid == 0) heads[which] = PartHead{id, last < 0, s.first, s.n * a.G};
    for (int u = tid; u < L::kRows * (D / 8); u += kThreads) {
      const int r = u / (D / 8), d = u % (D / 8) * 8;
      float top = -INFINITY, sum = 0.f, v[8] = {};
      for (uint32_t rest = same; rest != 0; rest &= rest - 1) {
        const int k = __ffs(rest) - 1;
        const float* src = reinterpret_cast<const float*>(k & 1 ? smem + (k >> 1) * L::kRing
                                                                : smem + L::kPartOff + (k >> 1) * L::kPartBytes);
        const float mk = src[L::kRows * D + r], next = fmaxf(top, mk);
        const float x = top == -INFINITY ? 0.f : ex2(top - next), y = mk == -INFINITY ? 0.f : ex2(mk - next);
        sum = sum * x + src[L::kRows * D + L::kRows + r] * y;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = v[e] * x + src[r * D + d + e] * y;
        top = next;
      }
      if (complete) {
        if (r < s.n * a.G) {
          const float inv = sum > 0.f ? __fdividef(1.f, sum) : 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] *= inv;
          write_out8<D, T>(a, s.first, h, r, d, v);
          if (d == 0) write_lse(a, s.first, h, r, top, sum);
        }
      } else {
        reinterpret_cast<float4*>(dst + r * D + d)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4*>(dst + r * D + d)[1] = make_float4(v[4], v[5], v[6], v[7]);
        if (d == 0) {
          dst[L::kRows * D + r] = top;
          dst[L::kRows * D + L::kRows + r] = sum;
        }
      }
    }
    __syncwarp();
  }
  if (tid == 0) {
    if (!have0) heads[0] = PartHead{-1, 0, 0, 0};
    if (!have1) heads[1] = PartHead{-1, 0, 0, 0};
  }
}

// A head that crosses CTAs: begun at the end of CTA c, then the first parts of the CTAs after it up to its last.
template <int D, int NT, typename T>
__global__ void __launch_bounds__(256) join_parts_kernel(const AttnArgs a, int ctas) {
  using L = FewLayout<D, NT>;
  __shared__ int s_last;
  const int cta = blockIdx.x, tid = threadIdx.x;
  if (tid == 0) s_last = 0x7FFFFFFF;
  griddep_wait();
  griddep_launch_dependents();
  // This CTA's last part and the first parts of all CTAs after it, in one go.
  const PartHead p = *part_head<D, NT>(a.workspace, cta, 1);
  PartHead n = {-1, 0, 0, 0};
  const int k = cta + 1 + tid;
  if (k < ctas) n = *part_head<D, NT>(a.workspace, k, 0);
  __syncthreads();
  if (p.id < 0) return;
  if (n.id == p.id && n.ends) atomicMin(&s_last, k);
  for (int far = k + blockDim.x; far < ctas; far += blockDim.x) {
    n = *part_head<D, NT>(a.workspace, far, 0);
    if (n.id == p.id && n.ends) atomicMin(&s_last, far);
  }
  __syncthreads();
  const int last = s_last;
  if (last >= ctas) return;  // not this call's parts (a workspace that another call writes): none is read past them
  const int rows = p.rows, h = p.id % a.H;
  for (int u = tid; u < rows * (D / 8); u += blockDim.x) {
    const int r = u / (D / 8), d = u % (D / 8) * 8;
    float top = -INFINITY, sum = 0.f, v[8] = {};
    constexpr int kAtOnce = 8;  // parts whose loads are in flight together
    for (int k0 = cta; k0 <= last; k0 += kAtOnce) {
      float mk[kAtOnce], lk[kAtOnce];
      float4 x0[kAtOnce], x1[kAtOnce];
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        mk[j] = -INFINITY;
        lk[j] = 0.f;
        x0[j] = x1[j] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (k0 + j <= last) {
          const float* src = part_sums<D, NT>(a.workspace, ctas, k0 + j, k0 + j == cta ? 1 : 0);
          mk[j] = src[L::kRows * D + r];
          lk[j] = src[L::kRows * D + L::kRows + r];
          x0[j] = reinterpret_cast<const float4*>(src + r * D + d)[0];
          x1[j] = reinterpret_cast<const float4*>(src + r * D + d)[1];
        }
      }
      float next = top;
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) next = fmaxf(next, mk[j]);
      const float x = top == -INFINITY ? 0.f : ex2(top - next);
      sum *= x;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] *= x;
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        const float y = mk[j] == -INFINITY ? 0.f : ex2(mk[j] - next);
        sum = fmaf(lk[j], y, sum);
        v[0] = fmaf(x0[j].x, y, v[0]);
        v[1] = fmaf(x0[j].y, y, v[1]);
        v[2] = fmaf(x0[j].z, y, v[2]);
        v[3] = fmaf(x0[j].w, y, v[3]);
        v[4] = fmaf(x1[j].x, y, v[4]);
        v[5] = fmaf(x1[j].y, y, v[5]);
        v[6] = fmaf(x1[j].z, y, v[6]);
        v[7] = fmaf(x1[j].w, y, v[7]);
      }
      top = next;
    }
    const float inv = sum > 0.f ? __fdividef(1.f, sum) : 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= inv;
    write_out8<D, T>(a, p.first, h, r, d, v);
    if (d == 0) write_lse(a, p.first, h, r, top, sum);
  }
}

template <int D, int NT, typename T>
int launch_few(const AttnArgs& a, cudaStream_t s) {
  using L = FewLayout<D, NT>;
  static_assert(sizeof(FewCtrl<D, NT>) <= 2048, "control block");
  const int sms = device_sms();
  if (sms == 0 || !smem_optin<paged_few_kernel<D, NT, T>>(L::kBytes)) return OFFQ_ERR_CUDA;
  if (const int rc = launch_pdl(paged_few_kernel<D, NT, T>, dim3(sms), dim3(L::kWarps * 32), L::kBytes, s, a);
      rc != OFFQ_OK)
    return rc;
  return launch_pdl(join_parts_kernel<D, NT, T>, dim3(sms), dim3(256), 0, s, a, sms);
}

template <int D>
int launch_few_d(const AttnArgs& a, int dtype, cudaStream_t s) {
  const bool two = std::min<int64_t>(static_cast<int64_t>(a.max_q) * a.G, a.few_rows) > 8;
  if (dtype == OFFQ_BF16) return two ? launch_few<D, 2, __nv_bfloat16>(a, s) : launch_few<D, 1, __nv_bfloat16>(a, s);
  return two ? launch_few<D, 2, __half>(a, s) : launch_few<D, 1, __half>(a, s);
}

}  // namespace

namespace offq {

int64_t paged_few_workspace(int head_dim) {
  const int sms = device_sms();
  const int64_t floats = kFewRows * (head_dim + 2);
  return sms == 0 ? -1 : 2 * static_cast<int64_t>(sms) * (static_cast<int64_t>(sizeof(PartHead)) + 4 * floats);
}

int paged_few(const AttnArgs& a, int dtype, int head_dim, cudaStream_t s) {
  return head_dim == 128 ? launch_few_d<128>(a, dtype, s) : launch_few_d<64>(a, dtype, s);
}

}  // namespace offq
