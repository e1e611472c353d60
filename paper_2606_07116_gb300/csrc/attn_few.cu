// Attention of few query rows over the paged 4-bit cache (offq_paged_attention with up to 16 rows
// n * Hq / H per sequence and key head: single tokens, drafted tokens; under a window and behind shared prefixes up to 32).
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
// Window and sinks: a sequence's stages leave out the gap between the sinks and the window of its first query, whole stages of it,
// and number the rest 0, 1, ...; only the copies know the difference. Halves of a stage that no query sees are not copied (their
// page may be gone), and a row's hidden keys are taken out in the stages at the gap alone, as the last stage's are.
// Shared prefixes: the list begins with the prefixes, each a sequence with all queries that stand behind it, in groups of 8 or 16
// rows, and goes on with the sequences' own tokens. Sums and statistics of both go to memory (csrc/attn_prefix.cu). A group more
// reads its pages from the L2 and costs less than the many-row form up to 32 rows, which is as far as it was built: 8 single tokens
// of 32 heads on 8 behind 32768 tokens 44 us (four groups of 8) against 74, behind 131072 124 against 190; 32 sequences of 32 rows
// under a window of 4096 98 (two groups of 16) against 204.
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
// 64 heads on 8: 82 us, 4.1 TB/s. 16 x 4 tokens over 500 to 6000: 36 us. 64 streams of 1 to 40000 under a window of 4096 and 4
// sinks: 70 us, 4.1 TB/s over all and 5.1 while it streams (issue slots 61 %, integer pipe 55 %); 11 us pass before the first
// stage is there, most of it code that no cache holds yet, and 3 after the last. 30 sequences behind five prefixes: 59 us of 76.
#include <algorithm>
#include <type_traits>

#include "attn.cuh"

namespace {

using namespace offq;

constexpr int kTile = 32;   // tokens per stage
constexpr float kBias = 24.0f;
constexpr int kLeastStages = 8;   // of a CTA
// What a unit costs a warp besides its stages (queries, the output), in stages.
template <AttnMode M>
constexpr int kUnitCost = M == kCausal ? 0 : 2;

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

// What sequences cost, in stages: with what their units cost besides, and without.
struct Cost {
  long long all, stages;
};

// Control block behind the parts.
template <int D, int NT>
struct FewCtrl {
  Cost scan[FewLayout<D, NT>::kWarps];
  int4 part[2 * FewLayout<D, NT>::kWarps];    // (sequence or -1, unit in it, first stage, last stage) of each part
  int2 rows[2 * FewLayout<D, NT>::kWarps];    // first query row of its sequence, rows of the unit
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

// Behind shared prefixes, and under a window in the kernel of 16 rows, a sequence's rows may be several groups of what it holds. A unit of its work is a group and a
// head, number group * H + head, and the groups read the same pages one after the other, from the L2 but for the first.
constexpr int kMostGroups = 4;
template <AttnMode M, int ROWS>
constexpr bool kGrouped = M == kShared || (M == kWindowed && ROWS == 16);
template <AttnMode M, int ROWS>
__device__ __forceinline__ int groups_of(const AttnArgs& a, const PagedSeq& s) {
  return kGrouped<M, ROWS> ? (s.n * a.G + ROWS - 1) / ROWS : 1;
}
// The units of all sequences as one list: unit u of sequence b (fits an int: two lists of 65535 sequences, 4096 heads).
template <AttnMode M, int ROWS>
__device__ __forceinline__ int unit_id(const AttnArgs& a, int b, int u) {
  return b * (kGrouped<M, ROWS> ? kMostGroups : 1) * a.H + u;
}
struct Unit {
  int b, h, row0;
};
template <AttnMode M, int ROWS>
__device__ __forceinline__ Unit unit_at(const AttnArgs& a, int id) {
  const int b = id / a.H;
  if constexpr (kGrouped<M, ROWS>) return {b / kMostGroups, id - b * a.H, b % kMostGroups * ROWS};
  return {b, id - b * a.H, 0};
}

// A sequence in this form's numbers: under a window without the gap that none of its queries sees, whole stages of it.
template <AttnMode M>
__device__ __forceinline__ PagedSeq few_seq(const AttnArgs& a, int b) {
  PagedSeq s = paged_seq<M>(a, b);
  if constexpr (M == kWindowed) {
    s.len -= window_gap(a, position<M>(s), kTile).shift;
  }
  return s;
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

// Channels d .. d + 7 of row r of (sequence b of the list, which starts at query row `first`, head h): outputs, with kShared sums.
template <int D, typename T, AttnMode M>
__device__ __forceinline__ void write_row8(const AttnArgs& a, int b, int first, int h, int r, int d, const float (&v)[8]) {
  if constexpr (M == kShared) {
    float* dst = shared_sums<D>(a, b, first, h, r);
#pragma unroll
    for (int e = 0; e < 4; ++e) *reinterpret_cast<float2*>(dst + shared_at(d + e)) = make_float2(v[e], v[e + 4]);
    return;
  }
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
template <AttnMode M>
__device__ __forceinline__ void write_row_stats(const AttnArgs& a, int b, int first, int h, int r, float m, float l) {
  if constexpr (M == kShared)
    write_stats(a, b, first, h, r, m, l);
  else
    write_lse(a, first, h, r, m, l);
}

template <int D, int NT, typename T, AttnMode M>
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
  const int B = listed<M>(a);
  auto cost = [&](const PagedSeq& s) {
    const int stages = stages_of(a, s);
    const long long units = stages > 0 ? static_cast<long long>(a.H) * groups_of<M, L::kRows>(a, s) : 0;
    if (M != kCausal && a.whole) return Cost{units, units * stages};
    return Cost{units * (stages + kUnitCost<M>), units * stages};
  };
  Listed* list = reinterpret_cast<Listed*>(smem);  // where the rings will be
  static_assert(kThreads * sizeof(Listed) <= L::kPartOff, "the list fits");
  // The sequences base .. base + kThreads - 1 into the list, behind what cost `before`; their cost.
  auto enlist = [&](int base, const Cost& before) {
    PagedSeq s = {};
    Cost n = {0, 0};
    if (base + tid < B) {
      s = few_seq<M>(a, base + tid);
      n = cost(s);
    }
    Cost incl = n;
#pragma unroll 1
    for (int m = 1; m < 32; m <<= 1) {
      const long long x = __shfl_up_sync(kAllLanes, incl.all, m), y = __shfl_up_sync(kAllLanes, incl.stages, m);
      if (lane >= m) {
        incl.all += x;
        incl.stages += y;
      }
    }
    if (lane == 31) ctrl->scan[warp] = incl;
    __syncthreads();
    Cost chunk = {0, 0};
#pragma unroll 4
    for (int i = 0; i < L::kWarps; ++i) {
      if (i == warp) {
        incl.all += chunk.all;
        incl.stages += chunk.stages;
      }
      chunk.all += ctrl->scan[i].all;
      chunk.stages += ctrl->scan[i].stages;
    }
    list[tid] = Listed{before.all + incl.all - n.all, before.stages + incl.stages - n.stages, s};
    __syncthreads();
    if (s.bad && blockIdx.x == 0) *a.status = OFFQ_ERR_INVALID_ARG;
    return chunk;
  };
  // Most lists are no longer than the CTA and are read once; others a second time, to find this CTA's share in them.
  Cost first = enlist(0, Cost{0, 0}), total = first;
  for (int base = kThreads; base < B; base += kThreads) {
    const Cost more = enlist(base, Cost{0, 0});
    total.all += more.all;
    total.stages += more.stages;
  }
  // Little work goes to fewer CTAs, some stages each: their warps take them at once, and joining inside a CTA is cheaper.
  const int least = M != kCausal && a.whole ? 1 : kLeastStages;
  const int ctas = static_cast<int>(min((total.all + least - 1) / least, static_cast<long long>(gridDim.x)));
  const int cta = blockIdx.x;
  PartHead* heads = M != kCausal && a.whole ? nullptr : part_head<D, NT>(a.workspace, blockIdx.x, 0);
  if (cta >= ctas) {
    if (tid < 2 && heads != nullptr) heads[tid] = PartHead{-1, 0, 0, 0};
    return;
  }
  const long long lo = divide(total.all * cta, ctas).q, hi = divide(total.all * (cta + 1), ctas).q;
  const long long w0 = lo + (hi - lo) * warp / L::kWarps, w1 = lo + (hi - lo) * (warp + 1) / L::kWarps;
  int b0 = 0, unit0 = 0, t0 = 0;  // of this warp's first stage: sequence, unit in it, stage
  PagedSeq s0 = {};
  long long from = 0, to = total.stages;  // stages before it, and up to the warp's end
  Cost before = {0, 0};
  for (int base = 0; base < B && before.all <= hi; base += kThreads) {
    const Cost chunk = B <= kThreads ? first : enlist(base, before);
    if (M != kCausal && a.whole) {  // unit number lo, a share of its stages for each warp
      if (lo >= before.all && lo < before.all + chunk.all) {
        const int at = find_listed(list, kThreads, lo);
        const Listed found = list[at];
        const int stages = stages_of(a, found.s);
        unit0 = static_cast<int>(lo - found.start);
        t0 = static_cast<int>(static_cast<long long>(stages) * warp / L::kWarps);
        from = t0;
        to = static_cast<long long>(stages) * (warp + 1) / L::kWarps;
        b0 = base + at;
        s0 = found.s;
      }
      before.all += chunk.all;
      __syncthreads();
      continue;
    }
#pragma unroll 1
    for (int end = 0; end < 2; ++end) {
      const long long x = end ? w1 : w0;
      if (x < before.all || x >= before.all + chunk.all) continue;
      const int at = find_listed(list, kThreads, x);
      const Listed found = list[at];
      const int stages = stages_of(a, found.s);
      const Divided in = divide(x - found.start, stages + kUnitCost<M>);
      const int t = max(0, static_cast<int>(in.r) - kUnitCost<M>);
      const long long passed = found.steps + in.q * stages + t;
      if (end) {
        to = passed;
      } else {
        from = passed;
        b0 = base + at;
        s0 = found.s;
        unit0 = static_cast<int>(in.q);
        t0 = t;
      }
    }
    before.all += chunk.all;
    before.stages += chunk.stages;
    __syncthreads();
  }

  int todo = static_cast<int>(to - from), ahead = todo;  // stages to compute, to issue
  if (todo > 0) {
    int b = b0, h = unit0, t = t0;
    PagedSeq s = s0;
    int stages = stages_of(a, s);
    int row0 = 0, pgroup = 0, pgroups = 1;  // this unit's first row; where the copies are
    if constexpr (kGrouped<M, L::kRows>) {
      pgroup = h / a.H;
      pgroups = groups_of<M, L::kRows>(a, s);
      h %= a.H;
      row0 = pgroup * L::kRows;
    }

    // Where the copies are: they run ahead across heads and sequences.
    int pb = b, ph = h, pt = t, pstages = stages, plen = s.len, listed_from = -64, entry = 0;
    const int cut = M == kWindowed ? window_gap(a, 0, kTile).cut : 0;
    // Under a window: tokens left out at `cut`, and the first that a window leaves in.
    int pshift = M == kWindowed ? window_gap(a, position<M>(paged_seq<M>(a, b)), kTile).shift : 0;
    int pfrom = M == kWindowed ? window_from(a, position<M>(s) + 1) : 0;
    int64_t page_row = -1;   // first row of the page the copies are in
    bool turn = true;        // that page is not known yet
    uint32_t missing = 0;    // bit 2 slot + half: that half of the slot's stage has no page
    auto find_page = [&](int tok) {  // first row of the page of token tok, or -1
      const int index = tok >> a.page_shift;
      if (index < listed_from || index >= listed_from + 32) {
        listed_from = index;
        entry = static_cast<int64_t>(index + lane) << a.page_shift < plen + pshift ? __ldg(pages_of<M>(a, pb) + index + lane) : 0;
      }
      const int page = __shfl_sync(kAllLanes, entry, index - listed_from);
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
      const int at = pt * kTile, tok = M == kWindowed && at >= cut ? at + pshift : at;
      const int in_page = tok & ((1 << a.page_shift) - 1);
      // Halves of which some token may be seen: the others have no page under a window.
      bool need0 = at < plen, need1 = at + 16 < plen;
      if constexpr (M == kWindowed) {
        need0 = need0 && (at < a.sinks || at + 16 > pfrom);
        need1 = need1 && (at + 16 < a.sinks || at + 32 > pfrom);
      }
      int64_t r0, r1;  // first rows of the stage's halves, or -1
      if (a.page_shift >= 5) {
        if (turn || in_page == 0 || (M == kWindowed && at == cut)) page_row = at < plen ? find_page(tok) : -1;
        turn = false;
        r0 = page_row < 0 ? -1 : page_row + in_page;
        r1 = page_row < 0 ? -1 : r0 + 16;
        if (M == kWindowed && !need0) r0 = -1;
        if (M == kWindowed && !need1) r1 = -1;
      } else {  // two pages of 16 tokens
        r0 = need0 ? find_page(tok) : -1;
        r1 = need1 ? find_page(tok + 16) : -1;
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
        bool next = false;  // the next sequence
        if (++ph == a.H) {
          ph = 0;
          next = true;
          if constexpr (kGrouped<M, L::kRows>) {
            next = ++pgroup == pgroups;
            if (next) pgroup = 0;
          }
        }
        if (next) {
          listed_from = -64;
          PagedSeq n;
          do {
            n = few_seq<M>(a, ++pb);
            pstages = stages_of(a, n);
          } while (pstages == 0);
          plen = n.len;
          if constexpr (kGrouped<M, L::kRows>) pgroups = groups_of<M, L::kRows>(a, n);
          if constexpr (M == kWindowed) {
            pfrom = window_from(a, position<M>(n) + 1);
            pshift = window_gap(a, position<M>(paged_seq<M>(a, pb)), kTile).shift;
          }
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
        if constexpr (kGrouped<M, L::kRows>) rows = min(rows - row0, L::kRows);
        sees_least = M == kShared ? min(s.len, max(0, s.at + 1)) : max(0, s.len - s.n + 1);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const int r = 8 * nt + g, rr = row0 + r;
          const T* src = static_cast<const T*>(a.q) + (static_cast<int64_t>(s.first) + rr / a.G) * a.ld_q +
                         static_cast<int64_t>(h * a.G + rr % a.G) * D + c * (D / 4);
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
            sees[nt][j] = rr < rows ? max(0, min(s.len, position<M>(s) + (row0 + rr) / a.G + 1)) : 0;
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
      if constexpr (M == kWindowed) redo |= t * kTile < window_from(a, s.len) && (t + 1) * kTile > a.sinks;
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
            const int tok = t * kTile + half * 16 + tok_k + 8 * i;
            none[half][i] = tok >= s.len || (gone >> half & 1u);
            if constexpr (M == kWindowed) none[half][i] |= tok >= a.sinks && tok < window_from(a, position<M>(s) + 1);
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
                const int tok = t * kTile + half * 16 + tok_k + 8 * i;
                if (none[half][i] || tok >= sees[nt][j]) z = -INFINITY;
                if (M == kWindowed && tok >= a.sinks && tok < window_from(a, sees[nt][j])) z = -INFINITY;
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
              const float inv = M == kShared ? 1.f : l[nt][j] > 0.f ? __fdividef(1.f, l[nt][j]) : 0.f;
#pragma unroll
              for (int q8 = 0; q8 < kMt / 4; ++q8) {
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = (o[nt][4 * q8 + e / 2][j + 2 * (e & 1)] + w[nt][j]) * inv;
                write_row8<D, T, M>(a, b, s.first, h, row0 + r, g * (D / 8) + 8 * q8, v);
              }
              if (g == 0) write_row_stats<M>(a, b, s.first, h, row0 + r, m[nt][j], l[nt][j]);
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
      if (!complete && lane == 0) {
        ctrl->rows[2 * warp + (first_part ? 0 : 1)] = make_int2(s.first, rows);
        ctrl->part[2 * warp + (first_part ? 0 : 1)] = make_int4(b, kGrouped<M, L::kRows> ? row0 / L::kRows * a.H + h : h, t_first, t == stages ? -1 : t);
      }
      first_part = false;
      begin = true;
      if (it + 1 < todo) {
        t = 0;
        bool next = false;  // the next sequence
        if (++h == a.H) {
          h = 0;
          next = true;
          if constexpr (kGrouped<M, L::kRows>) {
            row0 += L::kRows;
            next = row0 >= s.n * a.G;
            if (next) row0 = 0;
          }
        }
        if (next) {
          do {
            s = few_seq<M>(a, ++b);
            stages = stages_of(a, s);
          } while (stages == 0);
        }
      }
    }
  }

  // Parts of the same unit, in order of their stages, into one: an output where they are all of it, else a part
  // for the joining kernel. Each warp looks at all of them at once, a lane a part, and joins its share of the units (some
  // warps a unit where units are few): by all warps one after the other they took up to 10 us.
  __syncthreads();
  constexpr int kParts = 2 * L::kWarps;
  static_assert(kParts <= 32, "a lane for each part");
  const int4 mypart = lane < kParts ? ctrl->part[lane] : make_int4(-1, 0, 0, 0);
  const int my_id = mypart.x < 0 ? -1 : unit_id<M, L::kRows>(a, mypart.x, mypart.y);
  const uint32_t same_id = __match_any_sync(kAllLanes, my_id);
  uint32_t left = __ballot_sync(kAllLanes, my_id >= 0 && __ffs(same_id) - 1 == lane);  // the first part of each unit
  const int slices = max(1, min(L::kRows * (D / 8) / 32, L::kWarps / max(1, __popc(left))));
  bool have0 = false, have1 = false;
  for (int turn = warp / slices; left != 0; left &= left - 1, turn = turn == 0 ? L::kWarps / slices - 1 : turn - 1) {
    const int i = __ffs(left) - 1;
    const int id = __shfl_sync(kAllLanes, my_id, i);
    const uint32_t same = __shfl_sync(kAllLanes, same_id, i);
    const int begins = __shfl_sync(kAllLanes, mypart.z, i), last = __shfl_sync(kAllLanes, mypart.w, 31 - __clz(same));
    const bool complete = begins == 0 && last < 0;
    const int which = begins == 0 ? 1 : 0;
    if (!complete) (which ? have1 : have0) = true;
    if (turn != 0 || warp / slices >= L::kWarps / slices) continue;
    const Unit unit = unit_at<M, L::kRows>(a, id);
    float* dst = part_sums<D, NT>(a.workspace, gridDim.x, blockIdx.x, which);
    const int first = ctrl->rows[i].x, rows = ctrl->rows[i].y;
    const int slice = warp % slices;
    if (!complete && slice == 0 && lane == 0) heads[which] = PartHead{id, last < 0, first, rows};
    for (int u = slice * 32 + lane; u < L::kRows * (D / 8); u += slices * 32) {
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
        if (r < rows) {
          const float inv = M == kShared ? 1.f : sum > 0.f ? __fdividef(1.f, sum) : 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] *= inv;
          write_row8<D, T, M>(a, unit.b, first, unit.h, unit.row0 + r, d, v);
          if (d == 0) write_row_stats<M>(a, unit.b, first, unit.h, unit.row0 + r, top, sum);
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
  if (tid == 0 && heads != nullptr) {
    if (!have0) heads[0] = PartHead{-1, 0, 0, 0};
    if (!have1) heads[1] = PartHead{-1, 0, 0, 0};
  }
}

// A head that crosses CTAs: begun at the end of CTA c, then the first parts of the CTAs after it up to its last.
template <int D, int NT, typename T, AttnMode M>
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
  const int rows = p.rows;
  const Unit unit = unit_at<M, L::kRows>(a, p.id);
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
    const float inv = M == kShared ? 1.f : sum > 0.f ? __fdividef(1.f, sum) : 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= inv;
    write_row8<D, T, M>(a, unit.b, p.first, unit.h, unit.row0 + r, d, v);
    if (d == 0) write_row_stats<M>(a, unit.b, p.first, unit.h, unit.row0 + r, top, sum);
  }
}

template <int D, int NT, typename T, AttnMode M>
int launch_few(const AttnArgs& a, cudaStream_t s) {
  using L = FewLayout<D, NT>;
  static_assert(sizeof(FewCtrl<D, NT>) <= 2048, "control block");
  const int sms = device_sms();
  if (sms == 0 || !smem_optin<paged_few_kernel<D, NT, T, M>>(L::kBytes)) return OFFQ_ERR_CUDA;
  if (const int rc = launch_pdl(paged_few_kernel<D, NT, T, M>, dim3(sms), dim3(L::kWarps * 32), L::kBytes, s, a);
      rc != OFFQ_OK)
    return rc;
  if (a.whole) return OFFQ_OK;
  return launch_pdl(join_parts_kernel<D, NT, T, M>, dim3(sms), dim3(256), 0, s, a, sms);
}

template <AttnMode M, int D>
int launch_few_d(const AttnArgs& a, int dtype, cudaStream_t s) {
  const bool two = std::min<int64_t>(static_cast<int64_t>(a.max_q) * a.G, kFewRows) > 8;
  if (dtype == OFFQ_BF16) return two ? launch_few<D, 2, __nv_bfloat16, M>(a, s) : launch_few<D, 1, __nv_bfloat16, M>(a, s);
  return two ? launch_few<D, 2, __half, M>(a, s) : launch_few<D, 1, __half, M>(a, s);
}

template <AttnMode M>
int launch_few_m(const AttnArgs& a, int dtype, int head_dim, cudaStream_t s) {
  return head_dim == 128 ? launch_few_d<M, 128>(a, dtype, s) : launch_few_d<M, 64>(a, dtype, s);
}

}  // namespace

namespace offq {

bool paged_few_whole(const AttnArgs& a, AttnMode mode) {
  if (mode == kCausal) return false;
  const int64_t own = static_cast<int64_t>(a.max_q) * a.G, held = std::min<int64_t>(own, kFewRows) > 8 ? 16 : 8;
  auto groups = [&](int64_t rows) { return (std::min<int64_t>(rows, a.few_rows) + held - 1) / held; };
  int64_t units = groups(own) * a.B, tokens = a.ld_table << a.page_shift;
  if (mode == kWindowed) tokens = std::min(tokens, static_cast<int64_t>(a.window) + a.sinks + a.max_q + 2 * kTile);
  if (mode == kShared) {
    units += groups(std::min(a.Tq, static_cast<int64_t>(a.B) * a.max_q) * a.G) * a.P;
    tokens = std::max(tokens, a.ld_prefix << a.page_shift);
  }
  return units * a.H <= device_sms() && tokens <= kMostWhole * kTile;
}

int64_t paged_few_workspace(int head_dim) {
  const int sms = device_sms();
  const int64_t floats = kFewRows * (head_dim + 2);
  return sms == 0 ? -1 : 2 * static_cast<int64_t>(sms) * (static_cast<int64_t>(sizeof(PartHead)) + 4 * floats);
}

int paged_few(const AttnArgs& a, AttnMode mode, int dtype, int head_dim, cudaStream_t s) {
  switch (mode) {
    case kWindowed: return launch_few_m<kWindowed>(a, dtype, head_dim, s);
    case kShared: return launch_few_m<kShared>(a, dtype, head_dim, s);
    default: return launch_few_m<kCausal>(a, dtype, head_dim, s);
  }
}

}  // namespace offq
