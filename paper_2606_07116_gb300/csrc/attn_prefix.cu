// The last step of attention behind shared prefixes (offq_paged_attention_prefix): a row's sums over its prefix and over its
// sequence's own tokens, which the few-row and the many-row form left in the workspace, become its output.
//
// With (O, m, l) of either part, O = sum_j p_j v_j, l = sum_j p_j, p_j = 2^(z_j - m):
//   M = max(m0, m1), e_i = 2^(m_i - M), out = (e0 O0 + e1 O1) / (e0 l0 + e1 l1), lse = ln 2 (M + log2(e0 l0 + e1 l1)).
// A row that sees nothing in a part has l = 0 there, whatever its m.
#include <algorithm>

#include "attn.cuh"

namespace {

using namespace offq;

constexpr int kThreads = 256;
constexpr int kFlight = 4;  // rows of a thread whose reads are in flight together

// The prefix whose sequences b is one of, or -1. The warp looks at 32 of them at once.
__device__ __forceinline__ int prefix_of(const AttnArgs& a, int b) {
  const int lane = threadIdx.x & 31;
  int lo = 0, hi = a.P;
  while (hi - lo > 1) {  // the last that begins at b or before it is in lo .. hi - 1
    const int step = (hi - lo + 31) / 32, at = lo + lane * step;
    const int begun = __popc(__ballot_sync(kAllLanes, at < hi && __ldg(a.cu_prefix + at) <= b));
    lo += max(0, begun - 1) * step;
    hi = min(hi, lo + step);
  }
  return __ldg(a.cu_prefix + lo) <= b && b < __ldg(a.cu_prefix + lo + 1) ? lo : -1;
}

template <int D, typename T>
__global__ void __launch_bounds__(kThreads) join_shared_kernel(const AttnArgs a) {
  constexpr int kLanes = D / 4;             // of a (query, head): four channels each
  constexpr int kRows = kThreads / kLanes;  // that a block covers at once
  griddep_wait();
  griddep_launch_dependents();
  const int b = blockIdx.x;
  const PagedSeq s = paged_seq<kShared>(a, a.P + b);
  const int64_t rows = static_cast<int64_t>(s.n) * a.Hq;
  if (static_cast<int64_t>(blockIdx.y) * kRows * kFlight >= rows) return;
  // Sums of a prefix are there for the rows of its own range alone.
  const int g = prefix_of(a, b);
  const PagedSeq p = paged_seq<kShared>(a, max(g, 0));
  const bool shared = g >= 0 && p.first <= s.first && s.first + s.n <= p.first + p.n;
  const int at = threadIdx.x % kLanes, c = threadIdx.x & 3;
  const int64_t row0 = static_cast<int64_t>(s.first) * a.Hq, own = a.Tq * a.Hq;
  for (int64_t base = static_cast<int64_t>(blockIdx.y) * kRows * kFlight; base < rows;
       base += static_cast<int64_t>(gridDim.y) * kRows * kFlight) {
    float2 s0[kFlight], s1[kFlight];
    float4 x[kFlight], y[kFlight];
#pragma unroll
    for (int i = 0; i < kFlight; ++i) {  // reads in flight together
      const int64_t r = base + i * kRows + threadIdx.x / kLanes, row = row0 + r;
      s0[i] = s1[i] = make_float2(-INFINITY, 0.f);
      x[i] = y[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (r >= rows) continue;
      if (shared) {
        s0[i] = a.stats[row];
        x[i] = reinterpret_cast<const float4*>(a.sums + row * D)[at];
      }
      s1[i] = a.stats[own + row];
      y[i] = reinterpret_cast<const float4*>(a.sums + (own + row) * D)[at];
    }
#pragma unroll
    for (int i = 0; i < kFlight; ++i) {
      const int64_t r = base + i * kRows + threadIdx.x / kLanes, row = row0 + r;
      const float m0 = s0[i].y > 0.f ? s0[i].x : -INFINITY, m1 = s1[i].y > 0.f ? s1[i].x : -INFINITY, m = fmaxf(m0, m1);
      const float e0 = m0 == -INFINITY ? 0.f : ex2(m0 - m), e1 = m1 == -INFINITY ? 0.f : ex2(m1 - m);
      const float l = e0 * s0[i].y + e1 * s1[i].y, inv = l > 0.f ? __fdividef(1.f, l) : 0.f;
      const float f0 = e0 * inv, f1 = e1 * inv;
      // Channels c, c + 4, c + 8, c + 12 of 16 become 4 c .. 4 c + 3.
      uint32_t w[4] = {__float_as_uint(fmaf(x[i].x, f0, y[i].x * f1)), __float_as_uint(fmaf(x[i].y, f0, y[i].y * f1)),
                       __float_as_uint(fmaf(x[i].z, f0, y[i].z * f1)), __float_as_uint(fmaf(x[i].w, f0, y[i].w * f1))};
      transpose_words(w, c);
      if (r >= rows) continue;
      uint2 u;
      if constexpr (std::is_same<T, __nv_bfloat16>::value) {
        const __nv_bfloat162 h0 = __floats2bfloat162_rn(__uint_as_float(w[0]), __uint_as_float(w[1]));
        const __nv_bfloat162 h1 = __floats2bfloat162_rn(__uint_as_float(w[2]), __uint_as_float(w[3]));
        u = make_uint2(*reinterpret_cast<const uint32_t*>(&h0), *reinterpret_cast<const uint32_t*>(&h1));
      } else {
        const __half2 h0 = __floats2half2_rn(__uint_as_float(w[0]), __uint_as_float(w[1]));
        const __half2 h1 = __floats2half2_rn(__uint_as_float(w[2]), __uint_as_float(w[3]));
        u = make_uint2(*reinterpret_cast<const uint32_t*>(&h0), *reinterpret_cast<const uint32_t*>(&h1));
      }
      const int64_t t = row / a.Hq;
      reinterpret_cast<uint2*>(static_cast<T*>(a.out) + t * a.ld_out + (row - t * a.Hq) * D)[at] = u;
      if (at == 0 && a.lse != nullptr) a.lse[row] = l > 0.f ? (m + __log2f(l)) * kLn2 : -INFINITY;
    }
  }
}

template <int D, typename T>
int launch_join(const AttnArgs& a, cudaStream_t s) {
  constexpr int kAtOnce = kThreads / (D / 4) * kFlight;
  // The longest sequence's rows, but no more blocks in all than some waves: each looks for its prefix first (48 us for 2400
  // tokens of 32 heads with a block for every 16 rows).
  const int sms = device_sms();
  if (sms == 0) return OFFQ_ERR_CUDA;
  const int64_t rows = static_cast<int64_t>(std::min<int64_t>(a.max_q, a.Tq)) * a.Hq;
  const int64_t blocks = std::min((rows + kAtOnce - 1) / kAtOnce, std::max(int64_t{1}, int64_t{16} * sms / a.B));
  return launch_pdl(join_shared_kernel<D, T>, dim3(a.B, static_cast<unsigned>(blocks)), dim3(kThreads), 0, s, a);
}

}  // namespace

namespace offq {

int join_shared(const AttnArgs& a, int dtype, int head_dim, cudaStream_t s) {
  if (head_dim == 128) return dtype == OFFQ_BF16 ? launch_join<128, __nv_bfloat16>(a, s) : launch_join<128, __half>(a, s);
  return dtype == OFFQ_BF16 ? launch_join<64, __nv_bfloat16>(a, s) : launch_join<64, __half>(a, s);
}

}  // namespace offq
