// Heads on their way into attention: RMS norm, rotary positions and the per-head Hadamard H3 in one
// pass (offq_rope_heads); the same for queries and keys with keys and values quantized into a paged
// 4-bit cache (offq_kv4_paged_write); cached tokens read back (offq_kv4_paged_read).
//
// For a head x of D channels (all fp32):
//   norm    x <- (x * (1 / sqrt(mean(x^2) + eps))) * w[h]
//   rotary  (x_a, x_b) <- (x_a c - x_b s, x_b c + x_a s) on the first rot_dim channels, pairs
//           (m, m + rot_dim / 2) or (2m, 2m + 1), c and s from the table row of the position
//   H3      y = x H_D / sqrt(D), a radix-2 tree of additions, distance 1 first
//   codes   o = mean(y) (with H3: x_0 / sqrt(D)), r = y - o, s = max|r| / 7,
//           u = clamp(rne(r * (7 / max|r|)), -7, 7) + 8
// Every operation above is rounded on its own (no contraction), so the codes are a function of the
// formula and not of the compiler.
//
// A lane owns 16 channels, 8 neighbours (one 16-byte load of a 16-bit type) in each half of a head, so a head of 128 takes
// a fourth of a warp. The last butterfly and, where the whole head rotates, both channels of a rotary pair are in the
// lane, and all arithmetic goes two channels at a time; sums, maxima and three butterflies are xor shuffles. With 8 channels
// a lane 4097 tokens of 96 heads took 58 us to write (217 instructions a pair of heads) and take 41 now (120).
// A warp stays with one token and takes several groups of heads, with the token's cosines and sines
// in registers: they would otherwise be read again for each head, four times the data's own bytes. Without a cache the
// reads of two groups are issued before the first is worked on (8191 tokens of 72 heads: 51 us, with one 56); with one the
// registers serve more warps instead (59 us with the reading back, with two 65). CTAs of one warp leave no registers idle and
// end one by one: with eight warps a CTA the same took 57 and 69 us.
//
// Measured: 8191 tokens x 72 heads of 128 (f16, rotary on 64 channels) 51 us, 5.9 TB/s, 88 % of the copy bandwidth. 4097
// tokens x 32 query, 32 key and 32 value heads of 128 written in 41 us, 3.8 TB/s: reads' latency and issue slots (55 %). 16384
// tokens x 8 heads of 128 read back in 22 us, 3.9 TB/s, 77 % of the issue slots: widening, butterflies in packed halves.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <type_traits>

#include "offq.h"
#include "offq_device.cuh"
#include "offq_host.h"

namespace {

using namespace offq;

constexpr int kE = 8;            // a lane's channels in each half of a head
constexpr int kReadWarps = 4;    // warps per CTA of the reading kernel (one, two or eight are 2 to 30 % slower)
constexpr int kMostGroups = 8;   // groups of heads of a warp
constexpr int kReadGroups = 4;   // of a warp that reads the cache: all are read at once
constexpr uint32_t kAll = 0xFFFFFFFFu;

struct HeadArgs {
  // Heads of a token: H[0] queries, H[1] keys, H[2] values.
  const void* x[3];
  int64_t ld[3];
  int H[3];
  const float* norm[2];
  int64_t T;
  const int32_t* pos;
  const float* table;
  int64_t max_pos;
  int rot;           // channels that take the rotary positions (0: none)
  int interleaved;
  float eps;
  int rotate[3];     // H3
  int offset;
  void* out;         // queries
  int64_t ld_out;
  const int64_t* slots;
  uint8_t* codes[2];
  float* params[2];
  int64_t slots_in_cache;
  int page_shift;
  int iters;         // groups of heads per warp
  float zero;        // -0 (mul2)
  int* status;
};

// 8 channels as they lie in memory, and as floats.
template <typename T>
struct Raw8 {
  uint4 u[sizeof(T) / 2];
};
template <typename T>
__device__ __forceinline__ void read8(const T* p, Raw8<T>& r) {
#pragma unroll
  for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) r.u[i] = __ldg(reinterpret_cast<const uint4*>(p) + i);
}
template <typename T>
__device__ __forceinline__ void widen8(const Raw8<T>& r, float (&v)[kE]) {
  if constexpr (sizeof(T) == 4) {
    v[0] = __uint_as_float(r.u[0].x); v[1] = __uint_as_float(r.u[0].y);
    v[2] = __uint_as_float(r.u[0].z); v[3] = __uint_as_float(r.u[0].w);
    v[4] = __uint_as_float(r.u[1].x); v[5] = __uint_as_float(r.u[1].y);
    v[6] = __uint_as_float(r.u[1].z); v[7] = __uint_as_float(r.u[1].w);
  } else {
    const uint32_t w[4] = {r.u[0].x, r.u[0].y, r.u[0].z, r.u[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (std::is_same<T, __nv_bfloat16>::value) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
      } else {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
      }
    }
  }
}

template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&v)[kE]) {
  Raw8<T> r;
  read8(p, r);
  widen8(r, v);
}

template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&v)[kE]) {
  if constexpr (sizeof(T) == 4) {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (std::is_same<T, __nv_bfloat16>::value) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&b);
      } else {
        const __half2 b = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&b);
      }
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// A lane's channels of a head on its way in: 8 l + e in the low half of v[e], D / 2 + 8 l + e in the high half. Two
// operations at once, each rounded as a single one is.
using Pairs = uint64_t[kE];

__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t sub2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("sub.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
// a b, as a multiply-add of a -0 that the compiler does not know: a packed product that meets a packed sum would become one
// multiply-add with one rounding, in spite of the .rn of both.
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b, float zero) { return fma2v(a, b, pack2(zero, zero)); }

__device__ __forceinline__ uint64_t shfl_xor2(uint64_t v, int m) {
  float x, y;
  unpack2(v, x, y);
  return pack2(__shfl_xor_sync(kAll, x, m), __shfl_xor_sync(kAll, y, m));
}
__device__ __forceinline__ void pairs_of(const float (&lo)[kE], const float (&hi)[kE], Pairs& v) {
#pragma unroll
  for (int e = 0; e < kE; ++e) v[e] = pack2(lo[e], hi[e]);
}

// Sum of a head's channels, neighbours first, in every lane of the head.
template <int D>
__device__ __forceinline__ float head_sum(const Pairs& v) {
  uint64_t s = add2(add2(add2(v[0], v[1]), add2(v[2], v[3])), add2(add2(v[4], v[5]), add2(v[6], v[7])));
#pragma unroll
  for (int m = 1; m < D / (2 * kE); m <<= 1) s = add2(s, shfl_xor2(s, m));
  float x, y;
  unpack2(s, x, y);
  return __fadd_rn(x, y);
}

template <int D>
__device__ __forceinline__ float head_absmax(const Pairs& v) {
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < kE; ++e) {
    float x, y;
    unpack2(v[e], x, y);
    asm("max.f32 %0, %0, %1, %2;" : "+f"(s) : "f"(fabsf(x)), "f"(fabsf(y)));
  }
#pragma unroll
  for (int m = 1; m < D / (2 * kE); m <<= 1) s = fmaxf(s, __shfl_xor_sync(kAll, s, m));
  return s;
}

// x H_D, not normalised.
template <int D>
__device__ __forceinline__ void head_hadamard(Pairs& v, int lane) {
#pragma unroll
  for (int d = 1; d < kE; d <<= 1)
#pragma unroll
    for (int e = 0; e < kE; ++e)
      if ((e & d) == 0) {
        const uint64_t x = v[e], y = v[e + d];
        v[e] = add2(x, y);
        v[e + d] = sub2(x, y);
      }
#pragma unroll
  for (int m = 1; m < D / (2 * kE); m <<= 1) {
    const float sign = (lane & m) ? -1.f : 1.f;
#pragma unroll
    for (int e = 0; e < kE; ++e) v[e] = fma2v(pack2(sign, sign), v[e], shfl_xor2(v[e], m));  // the product with +-1 is exact
  }
#pragma unroll
  for (int e = 0; e < kE; ++e) {
    float x, y;
    unpack2(v[e], x, y);
    v[e] = pack2(__fadd_rn(x, y), __fsub_rn(x, y));
  }
}

// Cosines and sines of this lane's channels. Neighbouring pairs: four of the low channels, four of the high ones.
// Pairs half the rotated channels apart: those of the low channels, x c + y s with the sine's sign taken in; the high channels'
// are the same with the other sign where all channels rotate, and else are read when they are needed. 1 and 0
// past the rotated channels.
struct Angles {
  float c[kE], s[kE];
};

// Of the 8 channels from d0 on, in pairs rot / 2 apart.
__device__ __forceinline__ void half_angles(const float* row, int rot, int d0, Angles& t) {
  const int half = rot / 2;
  if (d0 >= rot) {
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      t.c[e] = 1.f;
      t.s[e] = 0.f;
    }
    return;
  }
  const int f = d0 < half ? d0 : d0 - half;
  load8(row + f, t.c);
  load8(row + half + f, t.s);
  if (d0 < half) {
#pragma unroll
    for (int e = 0; e < kE; ++e) t.s[e] = -t.s[e];
  }
}

template <int D>
__device__ __forceinline__ void load_angles(const HeadArgs& a, const float* row, int l, Angles& t) {
  if (!a.interleaved) return half_angles(row, a.rot, l * kE, t);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int d0 = i * (D / 2) + l * kE;
    float4 c = make_float4(1.f, 1.f, 1.f, 1.f), s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (d0 < a.rot) {
      c = __ldg(reinterpret_cast<const float4*>(row + d0 / 2));
      s = __ldg(reinterpret_cast<const float4*>(row + a.rot / 2 + d0 / 2));
    }
    t.c[4 * i] = c.x; t.c[4 * i + 1] = c.y; t.c[4 * i + 2] = c.z; t.c[4 * i + 3] = c.w;
    t.s[4 * i] = s.x; t.s[4 * i + 1] = s.y; t.s[4 * i + 2] = s.z; t.s[4 * i + 3] = s.w;
  }
}

template <int D>
__device__ __forceinline__ void rotary(const HeadArgs& a, const float* row, const Angles& t, int lane, Pairs& v) {
  constexpr int kLanes = D / (2 * kE);
  if (a.interleaved) {
#pragma unroll
    for (int m = 0; m < kE / 2; ++m) {
      const uint64_t x = v[2 * m], y = v[2 * m + 1], c = pack2(t.c[m], t.c[4 + m]), s = pack2(t.s[m], t.s[4 + m]);
      v[2 * m] = sub2(mul2(x, c, a.zero), mul2(y, s, a.zero));
      v[2 * m + 1] = add2(mul2(y, c, a.zero), mul2(x, s, a.zero));
    }
  } else if (a.rot == D) {  // both channels of a pair are this lane's
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      float x, y;
      unpack2(v[e], x, y);
      v[e] = add2(mul2(v[e], pack2(t.c[e], t.c[e]), a.zero), mul2(pack2(y, x), pack2(t.s[e], -t.s[e]), a.zero));
    }
  } else {  // rot is a multiple of 16: a pair's other channel is the same element of another eight
    const int l = lane % kLanes, n = a.rot / (2 * kE), base = lane - l;
    auto other = [&](int o) { return o < n ? o + n : o < 2 * n ? o - n : o; };
    const int p0 = other(l), p1 = other(l + kLanes);
    Angles u;
    half_angles(row, a.rot, D / 2 + l * kE, u);
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      float x, y;
      unpack2(v[e], x, y);
      const float a0 = __shfl_sync(kAll, x, base + p0 % kLanes), b0 = __shfl_sync(kAll, y, base + p0 % kLanes);
      const float a1 = __shfl_sync(kAll, x, base + p1 % kLanes), b1 = __shfl_sync(kAll, y, base + p1 % kLanes);
      const uint64_t o = pack2(p0 < kLanes ? a0 : b0, p1 < kLanes ? a1 : b1);
      v[e] = add2(mul2(v[e], pack2(t.c[e], u.c[e]), a.zero), mul2(o, pack2(t.s[e], u.s[e]), a.zero));
    }
  }
}

// Codes of a head y (before H3 where `rotate`) into its slot.
template <int D>
__device__ __forceinline__ void quantize_head(Pairs& v, bool rotate, bool offset, bool live, int lane, float zero,
                                              uint8_t* codes, float* params) {
  constexpr float kRoot = D == 128 ? 0.08838834764831844055f : 0.125f;  // 1 / sqrt(D) in fp32
  constexpr int kLanes = D / (2 * kE);
  const int l = lane % kLanes;
  float o = 0.f;
  if (rotate) {
    if (offset) {
      float x, y;
      unpack2(v[0], x, y);
      o = __fmul_rn(__shfl_sync(kAll, x, lane - l), kRoot);
      if (l == 0) v[0] = pack2(0.f, y);  // the first row of H_D is all ones: without x_0 the mean is 0
    }
    head_hadamard<D>(v, lane);
  } else if (offset) {
    o = __fmul_rn(head_sum<D>(v), 1.0f / D);
#pragma unroll
    for (int e = 0; e < kE; ++e) v[e] = sub2(v[e], pack2(o, o));
  }
  const float top = head_absmax<D>(v);
  const float inv = top > 0.f ? __fdiv_rn(7.0f, top) : 0.f;
  // |r inv| <= 7 (1 + 2^-22), so rounding alone keeps the codes in -7 .. 7. Adding 1.5 * 2^23 + 8 rounds to the nearest
  // even integer (the spacing there is 1) and leaves u = q + 8 in the low bits; eight are packed by shifted sums, and
  // what the upper bits add up to is taken off at the end.
  uint32_t w0 = 0, w1 = 0;
#pragma unroll
  for (int e = kE - 1; e >= 0; --e) {
    float x, y;
    unpack2(add2(mul2(v[e], pack2(inv, inv), zero), pack2(12582920.0f, 12582920.0f)), x, y);
    w0 = (w0 << 4) + __float_as_uint(x);
    w1 = (w1 << 4) + __float_as_uint(y);
  }
  if (!live) return;
  reinterpret_cast<uint32_t*>(codes)[l] = w0 - 0x4B400000u * 0x11111111u;
  reinterpret_cast<uint32_t*>(codes)[l + kLanes] = w1 - 0x4B400000u * 0x11111111u;
  if (l == 0) {
    const float s = rotate ? __fmul_rn(__fmul_rn(top, kRoot), 1.0f / 7.0f) : __fmul_rn(top, 1.0f / 7.0f);
    *reinterpret_cast<float2*>(params) = make_float2(s, o);
  }
}

// `groups` groups of heads of token t, from head h0 on (this lane's first head). KIND 0: queries, 1: keys, 2: values.
template <int D, typename Tin, typename Tout, int KIND, int kAhead>
__device__ __forceinline__ void run_heads(const HeadArgs& a, int64_t t, int h0, int groups, int lane) {
  constexpr int kLanes = D / (2 * kE), kUnits = 32 / kLanes;
  constexpr float kRoot = D == 128 ? 0.08838834764831844055f : 0.125f;
  const int l = lane % kLanes, heads = a.H[KIND];
  const Tin* x = static_cast<const Tin*>(a.x[KIND]) + t * a.ld[KIND] + l * kE;
  bool ok = true;
  Angles ang;
  const float* row = nullptr;
  if (a.rot != 0) {  // of a value too: a slot does not get a new value beside an old key
    const int64_t p = __ldg(a.pos + t);
    ok = p >= 0 && p < a.max_pos;
    if (!ok && lane == 0) *a.status = OFFQ_ERR_INVALID_ARG;
    if constexpr (KIND < 2) {
      row = a.table + (ok ? p : 0) * a.rot;
      load_angles<D>(a, row, l, ang);
    }
  }
  uint8_t* codes = nullptr;
  float* params = nullptr;
  if (KIND > 0) {
    const int64_t slot = __ldg(a.slots + t);
    if (slot >= a.slots_in_cache && lane == 0) *a.status = OFFQ_ERR_INVALID_ARG;
    ok = ok && slot >= 0 && slot < a.slots_in_cache;
    const int64_t page = slot >> a.page_shift, at = slot & ((1 << a.page_shift) - 1);
    const int64_t first = ok ? ((page * heads) << a.page_shift) + at : 0;
    codes = a.codes[KIND - 1] + first * (D / 2);
    params = a.params[KIND - 1] + first * 2;
  }
  const float* norm = KIND < 2 ? a.norm[KIND == 1] : nullptr;
  for (int base = 0; base < groups; base += kAhead) {
    Raw8<Tin> raw[kAhead][2];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (base + u < groups) {
        const Tin* from = x + min(h0 + (base + u) * kUnits, heads - 1) * D;
        read8(from, raw[u][0]);
        read8(from + D / 2, raw[u][1]);
      }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (base + u >= groups) break;
      const int h = h0 + (base + u) * kUnits;
      const bool live = ok && h < heads;
      float lo[kE], hi[kE];
      Pairs v;
      widen8(raw[u][0], lo);
      widen8(raw[u][1], hi);
      pairs_of(lo, hi, v);
      if (KIND < 2) {
        if (norm != nullptr) {
          Pairs wt;
#pragma unroll
          for (int e = 0; e < kE; ++e) wt[e] = mul2(v[e], v[e], a.zero);
          const float mean = __fmul_rn(head_sum<D>(wt), 1.0f / D);
          const float inv = __fdiv_rn(1.0f, __fsqrt_rn(__fadd_rn(mean, a.eps)));
          const float* weights = norm + min(h, heads - 1) * D + l * kE;
          load8(weights, lo);
          load8(weights + D / 2, hi);
          pairs_of(lo, hi, wt);
#pragma unroll
          for (int e = 0; e < kE; ++e) v[e] = mul2(mul2(v[e], pack2(inv, inv), a.zero), wt[e], a.zero);
        }
        if (a.rot != 0) rotary<D>(a, row, ang, lane, v);
      }
      if constexpr (KIND == 0) {
        if (a.rotate[0]) {
          head_hadamard<D>(v, lane);
#pragma unroll
          for (int e = 0; e < kE; ++e) v[e] = mul2(v[e], pack2(kRoot, kRoot), a.zero);
        }
        if (live) {
          Tout* to = static_cast<Tout*>(a.out) + t * a.ld_out + h * D + l * kE;
#pragma unroll
          for (int e = 0; e < kE; ++e) unpack2(v[e], lo[e], hi[e]);
          store8(to, lo);
          store8(to + D / 2, hi);
        }
      } else {
        const int64_t at = static_cast<int64_t>(live ? h : 0) << a.page_shift;
        quantize_head<D>(v, a.rotate[KIND] != 0, a.offset != 0, live, lane, a.zero, codes + at * (D / 2), params + at * 2);
      }
    }
  }
}

// A warp takes up to `iters` groups of one kind of heads of one token. kCache: keys and values too.
template <int D, typename Tin, typename Tout, bool kCache>
__global__ void __launch_bounds__(32, kCache ? 28 : 24) heads_kernel(const HeadArgs a) {
  constexpr int kUnits = 64 * kE / D;  // heads per warp
  constexpr int kAhead = kCache ? 1 : 2;  // groups of heads read ahead
  const int lane = threadIdx.x, unit = lane / (D / (2 * kE));
  griddep_wait();
  griddep_launch_dependents();
  const int gq = (a.H[0] + kUnits - 1) / kUnits, gk = (a.H[1] + kUnits - 1) / kUnits;
  const int pq = (gq + a.iters - 1) / a.iters, pk = (gk + a.iters - 1) / a.iters, parts = pq + 2 * pk;
  const int64_t w = blockIdx.x;
  const int64_t t = w / parts;
  if (t >= a.T) return;
  const int part = static_cast<int>(w % parts);
  const int first = (part < pq ? part : (part - pq) % max(pk, 1)) * a.iters;
  const int h0 = first * kUnits + unit;
  if (part < pq) {
    run_heads<D, Tin, Tout, 0, kAhead>(a, t, h0, min(a.iters, gq - first), lane);
  } else if constexpr (kCache) {
    if (part < pq + pk)
      run_heads<D, Tin, Tout, 1, kAhead>(a, t, h0, min(a.iters, gk - first), lane);
    else
      run_heads<D, Tin, Tout, 2, kAhead>(a, t, h0, min(a.iters, gk - first), lane);
  }
}

struct ReadArgs {
  const uint8_t* codes[2];
  const float* params[2];
  void* out[2];
  int64_t ld[2];
  int rotate[2];
  int64_t T, slots_in_cache;
  int H, page_shift;
  const int64_t* slots;
  int iters;
  int* status;
};

// Values s (u - 8) + o of cached heads, keys taken back by H3 (symmetric and orthonormal: its own inverse).
template <int D, typename Tout>
__global__ void __launch_bounds__(kReadWarps * 32) read_kernel(const ReadArgs a) {
  constexpr int kLanes = D / (2 * kE), kUnits = 32 / kLanes;
  constexpr float kRoot = D == 128 ? 0.08838834764831844055f : 0.125f;
  const int lane = threadIdx.x & 31, l = lane % kLanes, unit = lane / kLanes;
  griddep_wait();
  griddep_launch_dependents();
  const int groups = (a.H + kUnits - 1) / kUnits, per = (groups + a.iters - 1) / a.iters;
  const int64_t w = static_cast<int64_t>(blockIdx.x) * kReadWarps + (threadIdx.x >> 5);
  const int64_t t = w / (2 * per);
  if (t >= a.T) return;
  const int part = static_cast<int>(w % (2 * per)), kind = part >= per;
  Tout* out = static_cast<Tout*>(kind ? a.out[1] : a.out[0]);
  if (out == nullptr) return;
  const int first = (part - kind * per) * a.iters, count = min(a.iters, groups - first), h0 = first * kUnits + unit;
  const int64_t slot = __ldg(a.slots + t);
  if (slot >= a.slots_in_cache && lane == 0) *a.status = OFFQ_ERR_INVALID_ARG;
  const bool there = slot >= 0 && slot < a.slots_in_cache, rotate = (kind ? a.rotate[1] : a.rotate[0]) != 0;
  const int64_t row = there ? (((slot >> a.page_shift) * a.H) << a.page_shift) + (slot & ((1 << a.page_shift) - 1)) : 0;
  const uint32_t* from = reinterpret_cast<const uint32_t*>((kind ? a.codes[1] : a.codes[0]) + row * (D / 2)) + l;
  const float2* params = reinterpret_cast<const float2*>(kind ? a.params[1] : a.params[0]) + row;
  out += t * (kind ? a.ld[1] : a.ld[0]) + l * kE;
  uint32_t codes[kReadGroups][2];  // channels 8 l .. 8 l + 7 and those D / 2 further on
  float2 par[kReadGroups];
#pragma unroll
  for (int u = 0; u < kReadGroups; ++u) {
    const int h = h0 + u * kUnits;
    codes[u][0] = codes[u][1] = 0x88888888u;  // zeros
    par[u] = make_float2(0.f, 0.f);
    if (u < count && h < a.H && there) {
      const int64_t at = static_cast<int64_t>(h) << a.page_shift;
      codes[u][0] = __ldg(from + at * (D / 8));
      codes[u][1] = __ldg(from + at * (D / 8) + kLanes);
      par[u] = __ldg(params + at);
    }
  }
#pragma unroll
  for (int u = 0; u < kReadGroups; ++u) {
    if (u >= count) break;
    const int h = h0 + u * kUnits;
    // Codes q of channels e and e + 4 as halves: the nibble below the exponent of 1024, less its bias.
    __half2 q[2][4];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t w = codes[u][i], x = ((e < 2 ? w : w >> 8) & (e & 1 ? 0x00F000F0u : 0x000F000Fu)) | 0x64006400u;
        const __half2 y = *reinterpret_cast<const __half2*>(&x);
        q[i][e] = e & 1 ? __hfma2(y, __float2half2_rn(0.0625f), __float2half2_rn(-72.f)) : __hsub2(y, __float2half2_rn(1032.f));
      }
    float scale = par[u].x, v[2][kE];
    if (rotate) {
      // H of the integers q (sums of at most 128 x 8: exact in halves); the offset meets channel 0 alone.
      auto both = [](__half2& x, __half2& y) {
        const __half2 d = __hsub2(x, y);
        x = __hadd2(x, y);
        y = d;
      };
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        both(q[i][0], q[i][1]);
        both(q[i][2], q[i][3]);
        both(q[i][0], q[i][2]);
        both(q[i][1], q[i][3]);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          q[i][e] = __hfma2(q[i][e], __halves2half2(__float2half(1.f), __float2half(-1.f)), __lowhigh2highlow(q[i][e]));
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) both(q[0][e], q[1][e]);
#pragma unroll
      for (int m = 1; m < kLanes; m <<= 1) {
        const __half2 sign = __float2half2_rn((lane & m) ? -1.f : 1.f);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) q[i][e] = __hfma2(sign, q[i][e], __shfl_xor_sync(kAll, q[i][e], m));
      }
      scale *= kRoot;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 f = __half22float2(q[i][e]);
        v[i][e] = rotate ? f.x * scale : fmaf(f.x, scale, par[u].y);
        v[i][e + 4] = rotate ? f.y * scale : fmaf(f.y, scale, par[u].y);
      }
    }
    if (rotate && l == 0) v[0][0] = fmaf(par[u].y, D * kRoot, v[0][0]);
    if (h < a.H) {
      store8(out + h * D, v[0]);
      store8(out + h * D + D / 2, v[1]);
    }
  }
}

// Groups of heads per warp: several where there are enough warps to fill the chip without it.
int groups_per_warp(int64_t T, int groups, int sms, int most) {
  const int64_t per = T * groups / (static_cast<int64_t>(sms) * 64);
  return static_cast<int>(std::clamp<int64_t>(per, 1, most));
}

template <int D, typename Tin, typename Tout>
int launch_heads(HeadArgs a, int sms, cudaStream_t s) {
  constexpr int kUnits = 64 * kE / D;
  const int gq = (a.H[0] + kUnits - 1) / kUnits, gk = (a.H[1] + kUnits - 1) / kUnits;
  a.iters = groups_per_warp(a.T, gq + 2 * gk, sms, kMostGroups);
  a.zero = -0.0f;
  const int64_t parts = (gq + a.iters - 1) / a.iters + 2 * ((gk + a.iters - 1) / a.iters);
  const int64_t blocks = a.T * parts;
  if (blocks > 0x7FFFFFFF) return OFFQ_ERR_UNSUPPORTED;
  const dim3 grid(static_cast<unsigned>(blocks)), block(32);
  return a.H[1] > 0 ? launch_pdl(heads_kernel<D, Tin, Tout, true>, grid, block, 0, s, a)
                    : launch_pdl(heads_kernel<D, Tin, Tout, false>, grid, block, 0, s, a);
}

template <int D, typename Tin>
int launch_heads_out(const HeadArgs& a, int out_dtype, int sms, cudaStream_t s) {
  switch (out_dtype) {
    case OFFQ_F32: return launch_heads<D, Tin, float>(a, sms, s);
    case OFFQ_BF16: return launch_heads<D, Tin, __nv_bfloat16>(a, sms, s);
    default: return launch_heads<D, Tin, __half>(a, sms, s);
  }
}

template <int D>
int launch_heads_in(const HeadArgs& a, int dtype, int out_dtype, int sms, cudaStream_t s) {
  switch (dtype) {
    case OFFQ_F32: return launch_heads_out<D, float>(a, out_dtype, sms, s);
    case OFFQ_BF16: return launch_heads_out<D, __nv_bfloat16>(a, out_dtype, sms, s);
    default: return launch_heads_out<D, __half>(a, out_dtype, sms, s);
  }
}

int run_heads(HeadArgs& a, int dtype, int out_dtype, int head_dim, void* stream) {
  a.status = device_status_ptr();
  const int sms = device_sms();
  if (a.status == nullptr || sms == 0) return OFFQ_ERR_CUDA;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return head_dim == 128 ? launch_heads_in<128>(a, dtype, out_dtype, sms, s)
                         : launch_heads_in<64>(a, dtype, out_dtype, sms, s);
}

template <int D, typename Tout>
int launch_read(ReadArgs a, int sms, cudaStream_t s) {
  constexpr int kUnits = 64 * kE / D;
  const int groups = (a.H + kUnits - 1) / kUnits;
  a.iters = groups_per_warp(a.T, 2 * groups, sms, kReadGroups);
  const int64_t warps = a.T * 2 * ((groups + a.iters - 1) / a.iters), blocks = (warps + kReadWarps - 1) / kReadWarps;
  if (blocks > 0x7FFFFFFF) return OFFQ_ERR_UNSUPPORTED;
  return launch_pdl(read_kernel<D, Tout>, dim3(static_cast<unsigned>(blocks)), dim3(kReadWarps * 32), 0, s, a);
}

bool dtype_ok(int d) { return elem_bytes(d) != 0; }

// Shape rules that the calls of this file share.
int check_heads(int64_t T, int64_t H, int32_t head_dim) {
  if (T < 0 || H < 1 || head_dim < 1) return OFFQ_ERR_INVALID_ARG;
  if ((head_dim != 64 && head_dim != 128) || H > 65535 || T > (int64_t{1} << 31)) return OFFQ_ERR_UNSUPPORTED;
  return OFFQ_OK;
}

int check_rotary(const int32_t* positions, const float* table, int64_t max_pos, int32_t rot_dim, int32_t head_dim) {
  if (rot_dim < 0 || rot_dim > head_dim || rot_dim % 2 != 0) return OFFQ_ERR_INVALID_ARG;
  if (rot_dim % 16 != 0) return OFFQ_ERR_UNSUPPORTED;
  if (rot_dim > 0 && (positions == nullptr || table == nullptr || max_pos < 1)) return OFFQ_ERR_INVALID_ARG;
  return OFFQ_OK;
}

bool row_ok(const void* p, int64_t ld, int bytes) { return aligned(p, 16) && (ld * bytes) % 16 == 0; }

}  // namespace

extern "C" int offq_rope_heads(const void* x, int dtype, int64_t T, int32_t H, int32_t head_dim, int64_t ld_token,
                               const int32_t* positions, const float* table, int64_t max_pos, int32_t rot_dim,
                               const float* norm, float eps, int32_t flags, void* out, int out_dtype, int64_t ld_out,
                               void* stream) {
  if (!dtype_ok(dtype) || !dtype_ok(out_dtype) || (flags & ~(OFFQ_ROTATE | OFFQ_INTERLEAVED)) != 0 || !(eps >= 0.f))
    return OFFQ_ERR_INVALID_ARG;
  if (const int rc = check_heads(T, H, head_dim); rc != OFFQ_OK) return rc;
  const int64_t width = static_cast<int64_t>(H) * head_dim;
  if (ld_token < width || ld_out < width) return OFFQ_ERR_INVALID_ARG;
  if (T == 0) return OFFQ_OK;
  if (x == nullptr || out == nullptr) return OFFQ_ERR_INVALID_ARG;
  if (const int rc = check_rotary(positions, table, max_pos, rot_dim, head_dim); rc != OFFQ_OK) return rc;
  if (!row_ok(x, ld_token, elem_bytes(dtype)) || !row_ok(out, ld_out, elem_bytes(out_dtype)) || !aligned(table, 16) ||
      !aligned(norm, 16) || !aligned(positions, 4))
    return OFFQ_ERR_MISALIGNED;
  HeadArgs a = {};
  a.x[0] = x;
  a.ld[0] = ld_token;
  a.H[0] = H;
  a.norm[0] = norm;
  a.T = T;
  a.pos = positions;
  a.table = table;
  a.max_pos = max_pos;
  a.rot = rot_dim;
  a.interleaved = (flags & OFFQ_INTERLEAVED) != 0;
  a.eps = eps;
  a.rotate[0] = (flags & OFFQ_ROTATE) != 0;
  a.out = out;
  a.ld_out = ld_out;
  return run_heads(a, dtype, out_dtype, head_dim, stream);
}

extern "C" int offq_kv4_paged_write(const void* q, const void* k, const void* v, int dtype, int64_t T, int32_t Hq,
                                    int32_t H, int32_t head_dim, int64_t ld_q, int64_t ld_k, int64_t ld_v,
                                    const int32_t* positions, const float* table, int64_t max_pos, int32_t rot_dim,
                                    const float* q_norm, const float* k_norm, float eps, int32_t flags,
                                    const int64_t* slots, uint8_t* k_codes, float* k_params, uint8_t* v_codes,
                                    float* v_params, int64_t pages, int32_t page_size, void* q_out, int out_dtype,
                                    int64_t ld_q_out, void* stream) {
  if (!dtype_ok(dtype) || !(eps >= 0.f) ||
      (flags & ~(OFFQ_ROTATE | OFFQ_OFFSET | OFFQ_INTERLEAVED | OFFQ_ROTATE_V)) != 0 || Hq < 0)
    return OFFQ_ERR_INVALID_ARG;
  if (const int rc = check_heads(T, H, head_dim); rc != OFFQ_OK) return rc;
  if (Hq > 65535) return OFFQ_ERR_UNSUPPORTED;
  const int64_t width = static_cast<int64_t>(H) * head_dim, q_width = static_cast<int64_t>(Hq) * head_dim;
  if (ld_k < width || ld_v < width || pages < 1 || page_size < 1) return OFFQ_ERR_INVALID_ARG;
  if (!is_pow2(page_size) || page_size < 16 || page_size > 256 || pages > (int64_t{1} << 31)) return OFFQ_ERR_UNSUPPORTED;
  if (Hq > 0 && (ld_q < q_width || ld_q_out < q_width || !dtype_ok(out_dtype))) return OFFQ_ERR_INVALID_ARG;
  if (T == 0) return OFFQ_OK;
  if (k == nullptr || v == nullptr || slots == nullptr || k_codes == nullptr || k_params == nullptr ||
      v_codes == nullptr || v_params == nullptr || (Hq > 0 && (q == nullptr || q_out == nullptr)))
    return OFFQ_ERR_INVALID_ARG;
  if (const int rc = check_rotary(positions, table, max_pos, rot_dim, head_dim); rc != OFFQ_OK) return rc;
  const int b = elem_bytes(dtype);
  if (!row_ok(k, ld_k, b) || !row_ok(v, ld_v, b) || !aligned(table, 16) || !aligned(q_norm, 16) ||
      !aligned(k_norm, 16) || !aligned(positions, 4) || !aligned(slots, 8) || !aligned(k_codes, 16) ||
      !aligned(v_codes, 16) || !aligned(k_params, 16) || !aligned(v_params, 16) ||
      (Hq > 0 && (!row_ok(q, ld_q, b) || !row_ok(q_out, ld_q_out, elem_bytes(out_dtype)))))
    return OFFQ_ERR_MISALIGNED;
  HeadArgs a = {};
  a.x[0] = q;
  a.x[1] = k;
  a.x[2] = v;
  a.ld[0] = ld_q;
  a.ld[1] = ld_k;
  a.ld[2] = ld_v;
  a.H[0] = Hq;
  a.H[1] = a.H[2] = H;
  a.norm[0] = q_norm;
  a.norm[1] = k_norm;
  a.T = T;
  a.pos = positions;
  a.table = table;
  a.max_pos = max_pos;
  a.rot = rot_dim;
  a.interleaved = (flags & OFFQ_INTERLEAVED) != 0;
  a.eps = eps;
  a.rotate[0] = a.rotate[1] = (flags & OFFQ_ROTATE) != 0;
  a.rotate[2] = (flags & OFFQ_ROTATE_V) != 0;
  a.offset = (flags & OFFQ_OFFSET) != 0;
  a.out = q_out;
  a.ld_out = ld_q_out;
  a.slots = slots;
  a.codes[0] = k_codes;
  a.codes[1] = v_codes;
  a.params[0] = k_params;
  a.params[1] = v_params;
  a.slots_in_cache = pages * page_size;
  a.page_shift = __builtin_ctz(static_cast<unsigned>(page_size));
  return run_heads(a, dtype, Hq > 0 ? out_dtype : OFFQ_F32, head_dim, stream);
}

extern "C" int offq_kv4_paged_read(const uint8_t* k_codes, const float* k_params, const uint8_t* v_codes,
                                   const float* v_params, int64_t pages, int32_t page_size, int32_t H,
                                   int32_t head_dim, const int64_t* slots, int64_t T, int32_t flags, void* k_out,
                                   void* v_out, int out_dtype, int64_t ld_k, int64_t ld_v, void* stream) {
  if (!dtype_ok(out_dtype) || (flags & ~(OFFQ_ROTATE | OFFQ_ROTATE_V)) != 0) return OFFQ_ERR_INVALID_ARG;
  if (const int rc = check_heads(T, H, head_dim); rc != OFFQ_OK) return rc;
  const int64_t width = static_cast<int64_t>(H) * head_dim;
  if (pages < 1 || page_size < 1 || (k_out != nullptr && ld_k < width) || (v_out != nullptr && ld_v < width))
    return OFFQ_ERR_INVALID_ARG;
  if (!is_pow2(page_size) || page_size < 16 || page_size > 256 || pages > (int64_t{1} << 31)) return OFFQ_ERR_UNSUPPORTED;
  if (T == 0 || (k_out == nullptr && v_out == nullptr)) return OFFQ_OK;
  if (slots == nullptr || (k_out != nullptr && (k_codes == nullptr || k_params == nullptr)) ||
      (v_out != nullptr && (v_codes == nullptr || v_params == nullptr)))
    return OFFQ_ERR_INVALID_ARG;
  const int b = elem_bytes(out_dtype);
  if (!aligned(slots, 8) || !aligned(k_codes, 16) || !aligned(v_codes, 16) || !aligned(k_params, 16) ||
      !aligned(v_params, 16) || (k_out != nullptr && !row_ok(k_out, ld_k, b)) ||
      (v_out != nullptr && !row_ok(v_out, ld_v, b)))
    return OFFQ_ERR_MISALIGNED;
  ReadArgs a = {};
  a.codes[0] = k_codes;
  a.codes[1] = v_codes;
  a.params[0] = k_params;
  a.params[1] = v_params;
  a.out[0] = k_out;
  a.out[1] = v_out;
  a.ld[0] = ld_k;
  a.ld[1] = ld_v;
  a.rotate[0] = (flags & OFFQ_ROTATE) != 0;
  a.rotate[1] = (flags & OFFQ_ROTATE_V) != 0;
  a.T = T;
  a.slots_in_cache = pages * page_size;
  a.H = H;
  a.page_shift = __builtin_ctz(static_cast<unsigned>(page_size));
  a.slots = slots;
  a.status = device_status_ptr();
  const int sms = device_sms();
  if (a.status == nullptr || sms == 0) return OFFQ_ERR_CUDA;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (head_dim == 128) {
    switch (out_dtype) {
      case OFFQ_F32: return launch_read<128, float>(a, sms, s);
      case OFFQ_BF16: return launch_read<128, __nv_bfloat16>(a, sms, s);
      default: return launch_read<128, __half>(a, sms, s);
    }
  }
  switch (out_dtype) {
    case OFFQ_F32: return launch_read<64, float>(a, sms, s);
    case OFFQ_BF16: return launch_read<64, __nv_bfloat16>(a, sms, s);
    default: return launch_read<64, __half>(a, sms, s);
  }
}
