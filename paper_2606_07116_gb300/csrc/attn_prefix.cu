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
  griddep_wait();
  griddep_launch_dependents();
  const int b = blockIdx.x;
  const PagedSeq s = paged_seq<kShared>(a, a.P + b);
  const int64_t items = static_cast<int64_t>(s.n) * a.Hq * (D / 16);
  int64_t u = static_cast<int64_t>(blockIdx.y) * kThreads + threadIdx.x;
  if (u - (threadIdx.x & 31) >= items) return;  // whole warps: their lanes look for the prefix together
  // Sums of a prefix are there for the rows of its own range alone.
  const int g = prefix_of(a, b);
  const PagedSeq p = paged_seq<kShared>(a, max(g, 0));
  const bool shared = g >= 0 && p.first <= s.first && s.first + s.n <= p.first + p.n;
  for (; u < items; u += static_cast<int64_t>(gridDim.y) * kThreads) {
    const int d = static_cast<int>(u % (D / 16)) * 16;
    const int64_t row = static_cast<int64_t>(s.first) * a.Hq + u / (D / 16), own = a.Tq * a.Hq + row;
    const float2 none = make_float2(-INFINITY, 0.f);
    const float2 s0 = shared ? a.stats[row] : none, s1 = a.stats[own];
    float4 x[4] = {}, y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (shared) x[i] = reinterpret_cast<const float4*>(a.sums + row * D + d)[i];
      y[i] = reinterpret_cast<const float4*>(a.sums + own * D + d)[i];
    }
    const float m0 = s0.y > 0.f ? s0.x : -INFINITY, m1 = s1.y > 0.f ? s1.x : -INFINITY, m = fmaxf(m0, m1);
    const float e0 = m0 == -INFINITY ? 0.f : ex2(m0 - m), e1 = m1 == -INFINITY ? 0.f : ex2(m1 - m);
    const float l = e0 * s0.y + e1 * s1.y, inv = l > 0.f ? __fdividef(1.f, l) : 0.f;
    const float f0 = e0 * inv, f1 = e1 * inv;
    float v[16];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float p0[4] = {x[i].x, x[i].y, x[i].z, x[i].w}, p1[4] = {y[i].x, y[i].y, y[i].z, y[i].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) v[i + 8 * (e >> 1) + 4 * (e & 1)] = fmaf(p0[e], f0, p1[e] * f1);  // shared_at's order undone
    }
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (std::is_same<T, __nv_bfloat16>::value) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
      } else {
        const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
      }
    }
    const int64_t t = row / a.Hq;
    uint4* to = reinterpret_cast<uint4*>(static_cast<T*>(a.out) + t * a.ld_out + (row - t * a.Hq) * D + d);
    to[0] = make_uint4(w[0], w[1], w[2], w[3]);
    to[1] = make_uint4(w[4], w[5], w[6], w[7]);
    if (d == 0 && a.lse != nullptr) a.lse[row] = l > 0.f ? (m + __log2f(l)) * kLn2 : -INFINITY;
  }
}

template <int D, typename T>
int launch_join(const AttnArgs& a, cudaStream_t s) {
  const int64_t items = static_cast<int64_t>(std::min<int64_t>(a.max_q, a.Tq)) * a.Hq * (D / 16);
  // The longest sequence's items, but no more blocks in all than a few waves.
  const int64_t blocks = std::min((items + kThreads - 1) / kThreads, std::max(int64_t{1}, int64_t{32768} / a.B));
  return launch_pdl(join_shared_kernel<D, T>, dim3(a.B, static_cast<unsigned>(blocks)), dim3(kThreads), 0, s, a);
}

}  // namespace

namespace offq {

int join_shared(const AttnArgs& a, int dtype, int head_dim, cudaStream_t s) {
  if (head_dim == 128) return dtype == OFFQ_BF16 ? launch_join<128, __nv_bfloat16>(a, s) : launch_join<128, __half>(a, s);
  return dtype == OFFQ_BF16 ? launch_join<64, __nv_bfloat16>(a, s) : launch_join<64, __half>(a, s);
}

}  // namespace offq
