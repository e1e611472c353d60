// What the attention kernels share: their arguments, the checks of what stands in device buffers, and
// the pieces of a softmax.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "offq.h"
#include "offq_device.cuh"
#include "offq_host.h"

namespace offq {

constexpr uint32_t kAllLanes = 0xFFFFFFFFu;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// Paged: what a value's scale adds to the reference of a row's exponentials is its log2, this at least (zero has none). An
// exponential is then 2^(64 + kMostLog2) at most, and its sums over any context stay far from an overflow.
constexpr float kLeastLog2 = -64.f;

struct AttnArgs {
  const void* q;
  int64_t ld_q;
  int64_t Tq;
  int Hq, H, G;   // query heads, key heads, query heads per key head
  const void* k;  // prompts
  const void* v;
  int64_t ld_k, ld_v;
  const uint8_t* k_codes;  // paged
  const uint8_t* v_codes;
  const float* k_params;
  const float* v_params;
  int64_t pages;
  int page_shift;
  const int32_t* table;
  int64_t ld_table;
  const int32_t* lens;
  const int32_t* cu;
  int B;
  int max_q;
  int few_rows;   // sequences with at most this many rows n * G take the few-row form
  int causal;     // prompts
  int window, sinks;  // kWindowed: at most kMostTokens each
  int whole;          // the few-row form gives every CTA a whole unit: no part crosses CTAs
  const int32_t* prefix_table;  // kShared
  int64_t ld_prefix;
  const int32_t* prefix_lens;
  const int32_t* cu_prefix;
  int P;
  float* sums;    // kShared: of the prefixes, then of the sequences' own tokens: [2][Tq][Hq][head_dim]
  float2* stats;  // and [2][Tq][Hq] (reference, sum of weights)
  float scale;
  void* out;
  int64_t ld_out;
  float* lse;
  void* workspace;
  int* status;
};

// Most tokens of a sequence: the number of a token past its end by up to two blocks of 128 is an int.
constexpr int kMostTokens = 0x7FFFFF00;
// Most tokens of a shared prefix: the positions of all queries behind it are ints.
constexpr int kMostPrefix = 0x7E000000;

// What a query at position p of its sequence sees (of the tokens that the sequence has):
enum AttnMode {
  kCausal,    // 0 .. p
  kWindowed,  // those of 0 .. p among the first `sinks` or the last `window`
  // The list of sequences is that of the prefixes, each with all queries of its sequences (who see all of it), then the
  // sequences with their own tokens, as in kCausal. Sums and statistics of both go to the workspace.
  kShared
};

// A sequence of the paged call: its first query row, queries, cached tokens and its first query's position (a prefix's
// queries stand behind it). One whose entries are out of range (negative or too long counts) has no queries; `bad`
// says so.
struct PagedSeq {
  int first, n, len, at;
  bool bad;
};

// Sequences in the list of a call.
template <AttnMode M>
__device__ __forceinline__ int listed(const AttnArgs& a) {
  return M == kShared ? a.P + a.B : a.B;
}

// The page numbers of a sequence.
template <AttnMode M>
__device__ __forceinline__ const int32_t* pages_of(const AttnArgs& a, int b) {
  if constexpr (M == kShared) {
    if (b < a.P) return a.prefix_table + static_cast<int64_t>(b) * a.ld_prefix;
    b -= a.P;
  }
  return a.table + static_cast<int64_t>(b) * a.ld_table;
}

template <AttnMode M>
__device__ __forceinline__ PagedSeq paged_seq(const AttnArgs& a, int b) {
  PagedSeq s;
  int c0 = 0, c1 = 0, l = 0;
  int64_t ld = a.ld_table, most_q = a.max_q;
  bool bad = false, prefix = false;
  if constexpr (M == kShared) {
    prefix = b < a.P;
    if (prefix) {
      const int s0 = __ldg(a.cu_prefix + b), s1 = __ldg(a.cu_prefix + b + 1);
      bad = s0 < 0 || s1 < s0 || s1 > a.B;
      c0 = bad ? 0 : __ldg(a.cu + s0);
      c1 = bad ? 0 : __ldg(a.cu + s1);
      l = __ldg(a.prefix_lens + b);
      ld = a.ld_prefix;
      most_q = min(a.Tq, static_cast<int64_t>(a.B) * a.max_q);
    } else {
      b -= a.P;
    }
  }
  if (!prefix) {
    c0 = __ldg(a.cu + b);
    c1 = __ldg(a.cu + b + 1);
    l = __ldg(a.lens + b);
  }
  const int64_t most = min(ld << a.page_shift, static_cast<int64_t>(prefix ? kMostPrefix : kMostTokens));
  s.first = c0;
  s.n = c1 - c0;
  s.len = static_cast<int>(min(static_cast<int64_t>(max(l, 0)), most));
  s.bad = bad || l < 0 || l > most;
  if (c0 < 0 || c1 < c0 || c1 > a.Tq || s.n > most_q) {
    s.bad = true;
    s.n = 0;
  }
  s.at = prefix ? s.len : s.len - s.n;
  return s;
}

// Position of a sequence's first query.
template <AttnMode M>
__device__ __forceinline__ int position(const PagedSeq& s) {
  return M == kShared ? s.at : s.len - s.n;
}

// What no query of a run sees between the sinks and the window of its first query, which stands at position `at`: the tokens
// `cut` .. `cut + shift - 1`, both multiples of `step` (a power of two). A kernel leaves them out: it numbers
// the others 0, 1, ... in order, positions and lengths less `shift`, and only where it loads has to know.
struct Gap {
  int cut, shift;
};
__device__ __forceinline__ Gap window_gap(const AttnArgs& a, int at, int step) {
  Gap g;
  g.cut = (a.sinks + step - 1) & -step;
  g.shift = at >= a.window ? max(0, ((at + 1 - a.window) & -step) - g.cut) : 0;
  return g;
}
// The first token that the window of a query leaves in, given the tokens up to itself (both in a run's numbers).
__device__ __forceinline__ int window_from(const AttnArgs& a, int upto) { return upto > a.window ? upto - a.window : 0; }

// x / y and the rest, x >= 0 and y > 0. A division of 64 bits is a call of some hundred instructions, a quarter of a microsecond
// where they are not in a cache yet; few numbers here need one.
struct Divided {
  long long q, r;
};
__device__ __forceinline__ Divided divide(long long x, long long y) {
  if (((x | y) >> 32) != 0) return {x / y, x % y};
  const uint32_t a = static_cast<uint32_t>(x), b = static_cast<uint32_t>(y), q = a / b;
  return {q, a - q * b};
}

// Sequences of a list that a CTA looks at together, in shared memory: where each begins in units of cost, and in steps.
struct Listed {
  long long start, steps;
  PagedSeq s;
};
// Of `count` (up to 512, a multiple of 32) the last that begins at x or before it. The lanes of a warp look together.
__device__ __forceinline__ int find_listed(const Listed* list, int count, long long x) {
  const int lane = threadIdx.x & 31, per = count / 32;
  const int block = __popc(__ballot_sync(kAllLanes, list[lane * per].start <= x)) - 1;
  return block * per + __popc(__ballot_sync(kAllLanes, lane < per && list[block * per + min(lane, per - 1)].start <= x)) - 1;
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Nibbles n (0..3) of both 16-bit halves of w as two 16-bit floats 16 + u of type T: the bits land below the exponent
// of 16.0 (mantissa weight 1 is bit 3 in bf16, bit 6 in f16).
template <typename T>
__device__ __forceinline__ uint32_t widen(uint32_t w, int n) {
  constexpr bool kHalf = std::is_same<T, __half>::value;
  constexpr int kAt = kHalf ? 6 : 3;
  constexpr uint32_t kMask = (0xFu << kAt) * 0x10001u, kMagic = kHalf ? 0x4C004C00u : 0x41804180u;
  const int sh = kAt - 4 * n;
  const uint32_t x = sh >= 0 ? w << sh : w >> -sh;
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(x), "n"(kMask), "n"(kMagic));  // (x & mask) | magic
  return r;
}

// Nibbles 0 and 1 of both halves of w as signed codes q in f16 (2 and 3 of w shifted right by 8).
__device__ __forceinline__ void widen_signed(uint32_t w, uint32_t& even, uint32_t& odd) {
  uint32_t x, y;
  asm("lop3.b32 %0, %1, 0x000F000F, 0x64006400, 0xEA;" : "=r"(x) : "r"(w));  // 1024 + u
  asm("lop3.b32 %0, %1, 0x00F000F0, 0x64006400, 0xEA;" : "=r"(y) : "r"(w));  // 1024 + 16 u
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(even) : "r"(x), "r"(0x64086408u));                        // - 1032
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(odd) : "r"(y), "r"(0x2C002C00u), "r"(0xD480D480u));  // / 16 - 72
}

// Word k of the four lanes c of a quad becomes word c of lane k.
__device__ __forceinline__ void transpose_words(uint32_t (&w)[4], int c) {
#pragma unroll
  for (int step = 2; step > 0; step >>= 1) {
    const bool high = (c & step) != 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int k = step == 2 ? i : 2 * i;  // words k and k + step change places between the lanes
      const uint32_t got = __shfl_xor_sync(kAllLanes, high ? w[k] : w[k + step], step);
      if (high)
        w[k] = got;
      else
        w[k + step] = got;
    }
  }
}

// The log of a row's sum l of exponentials 2^(z - m), row r of (sequence starting at query row `first`, key head h).
__device__ __forceinline__ void write_lse(const AttnArgs& a, int first, int h, int r, float m, float l) {
  if (a.lse == nullptr) return;
  a.lse[(static_cast<int64_t>(first) + r / a.G) * a.Hq + h * a.G + r % a.G] =
      l > 0.f ? (m + __log2f(l)) * kLn2 : -INFINITY;
}

// kShared: sums over a prefix (b < P) or over a sequence's own tokens, the channels of row r of (first query row, key head h),
// and the row's statistics.
template <int D>
__device__ __forceinline__ float* shared_sums(const AttnArgs& a, int b, int first, int h, int r) {
  const int64_t t = (b < a.P ? 0 : a.Tq) + first + r / a.G;
  return a.sums + (t * a.Hq + h * a.G + r % a.G) * D;
}
// Where channel d stands in a row of sums: of 16 channels, d and d + 4, then d + 8 and d + 12 side by side, as a lane of the
// many-row form holds them.
__host__ __device__ constexpr int shared_at(int d) { return (d & ~15) + (d & 3) * 4 + (d >> 3 & 1) * 2 + (d >> 2 & 1); }
__device__ __forceinline__ void write_stats(const AttnArgs& a, int b, int first, int h, int r, float m, float l) {
  const int64_t t = (b < a.P ? 0 : a.Tq) + first + r / a.G;
  a.stats[t * a.Hq + h * a.G + r % a.G] = make_float2(m, l);
}

// The few-row form of offq_paged_attention (csrc/attn_few.cu): rows n * G of a sequence that it takes, its
// workspace, and its launch with arguments already checked.
constexpr int kFewRows = 16;
// Under a window and behind shared prefixes it takes groups of 8 or 16 rows, up to this many in all.
constexpr int kFewGroupedRows = 32;
// Under a window or behind shared prefixes: whether every CTA gets a whole unit, so that no parts are joined behind it and a call
// under a window needs no workspace. So where there are no more units than CTAs and none is longer than this many stages of 32
// tokens. A launch less is what it saves: 19 us a call from the host against 25, at any of these lengths (1 to 4 streams of 1 or 4
// tokens, 2 to 32 key heads). In a graph it crosses at 700 tokens under a window: 10 us against 12 at 400, 12.0 against 12.2 at
// 700, 13.5 against 12.2 at 1200 and with 16 rows a key head 15.5 against 13; behind 500 shared tokens 14.2 against 15.4, behind
// 1000 16.2 against 15.6. The limit is the one of calls from the host.
constexpr int64_t kMostWhole = 40;
bool paged_few_whole(const AttnArgs& a, AttnMode mode);
int64_t paged_few_workspace(int head_dim);
int paged_few(const AttnArgs& a, AttnMode mode, int dtype, int head_dim, cudaStream_t s);

// The many-row form (csrc/attn_chunk.cu): sequences with more rows.
int64_t paged_chunk_workspace(int head_dim);
int paged_chunk(const AttnArgs& a, AttnMode mode, int dtype, int head_dim, cudaStream_t s);
// The outputs of a shared-prefix call from its two sums a row (csrc/attn_prefix.cu).
int join_shared(const AttnArgs& a, int dtype, int head_dim, cudaStream_t s);
// Prompts on the tensor cores (csrc/attn_prompt.cu), arguments already checked.
int prompt_tc(const AttnArgs& a, AttnMode mode, int dtype, int head_dim, cudaStream_t s);

}  // namespace offq
