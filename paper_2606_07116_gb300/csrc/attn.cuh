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
  float scale;
  void* out;
  int64_t ld_out;
  float* lse;
  void* workspace;
  int* status;
};

// Most tokens of a sequence: the number of a token past its end by up to two blocks of 128 is an int.
constexpr int kMostTokens = 0x7FFFFF00;

// A sequence of the paged call: its first query row, queries and cached tokens. One whose entries are out of
// range (negative or too long counts) has no queries; `bad` says so.
struct PagedSeq {
  int first, n, len;
  bool bad;
};

__device__ __forceinline__ PagedSeq paged_seq(const AttnArgs& a, int b) {
  const int c0 = __ldg(a.cu + b), c1 = __ldg(a.cu + b + 1), l = __ldg(a.lens + b);
  const int64_t most = min(a.ld_table << a.page_shift, static_cast<int64_t>(kMostTokens));
  PagedSeq s;
  s.first = c0;
  s.n = c1 - c0;
  s.len = static_cast<int>(min(static_cast<int64_t>(max(l, 0)), most));
  s.bad = l < 0 || l > most;
  if (c0 < 0 || c1 < c0 || c1 > a.Tq || s.n > a.max_q) {
    s.bad = true;
    s.n = 0;
  }
  return s;
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

// The log of a row's sum l of exponentials 2^(z - m), row r of (sequence starting at query row `first`, key head h).
__device__ __forceinline__ void write_lse(const AttnArgs& a, int first, int h, int r, float m, float l) {
  if (a.lse == nullptr) return;
  a.lse[(static_cast<int64_t>(first) + r / a.G) * a.Hq + h * a.G + r % a.G] =
      l > 0.f ? (m + __log2f(l)) * kLn2 : -INFINITY;
}

// The few-row form of offq_paged_attention (csrc/attn_few.cu): rows n * G of a sequence that it takes, its
// workspace, and its launch with arguments already checked.
constexpr int kFewRows = 16;
int64_t paged_few_workspace(int head_dim);
int paged_few(const AttnArgs& a, int dtype, int head_dim, cudaStream_t s);

// The many-row form (csrc/attn_chunk.cu): sequences with more rows.
int64_t paged_chunk_workspace(int head_dim);
int paged_chunk(const AttnArgs& a, int dtype, int head_dim, cudaStream_t s);
// Prompts on the tensor cores (csrc/attn_prompt.cu), arguments already checked.
int prompt_tc(const AttnArgs& a, int dtype, int head_dim, cudaStream_t s);

}  // namespace offq
