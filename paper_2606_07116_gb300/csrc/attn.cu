// Attention: packed prompts on 16-bit keys and values (offq_prompt_attention) and new tokens over
// the paged 4-bit cache (offq_paged_attention).
//
// out_i = sum_j p_ij v_j / sum_j p_ij,  p_ij = exp(scale q_i . k_j - m_i),  lse_i = m_i + log sum_j p_ij
// over the keys j that query i sees. A warp takes one query of one head; a lane scores one key of
// each 32, and the running maximum, sum and output are rescaled once per 32 keys, in fp32.
#include <algorithm>

#include "attn.cuh"

namespace {

using namespace offq;

constexpr int kRowWarps = 4;

__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f(__half x) { return __half2float(x); }

// Value d of key (or value) j of head h of the sequence.
template <int D, typename T, bool kPaged>
__device__ __forceinline__ float element(const AttnArgs& a, int which, int b, int64_t start, int j, int h, int d) {
  if constexpr (kPaged) {
    const int64_t page = a.table[b * a.ld_table + (j >> a.page_shift)];
    if (page < 0 || page >= a.pages) {
      *a.status = OFFQ_ERR_INVALID_ARG;
      return which ? 0.f : -INFINITY;
    }
    const int64_t row = ((page * a.H + h) << a.page_shift) + (j & ((1 << a.page_shift) - 1));
    const uint32_t c = (which ? a.v_codes : a.k_codes)[row * (D / 2) + d / 2];
    const float* par = (which ? a.v_params : a.k_params) + 2 * row;
    const int u = static_cast<int>((d & 1) ? c >> 4 : c & 15u) - 8;
    return static_cast<float>(u) * par[0] + par[1];
  } else {
    const T* x = static_cast<const T*>(which ? a.v : a.k);
    return to_f(x[(start + j) * (which ? a.ld_v : a.ld_k) + static_cast<int64_t>(h) * D + d]);
  }
}

template <int D, typename T, bool kPaged>
__global__ void __launch_bounds__(kRowWarps * 32) attention_rows_kernel(const AttnArgs a) {
  __shared__ float qs[kRowWarps][D];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  griddep_wait();
  griddep_launch_dependents();
  const int64_t r = static_cast<int64_t>(blockIdx.x) * kRowWarps + warp;
  const int64_t t = r / a.Hq;
  const int hq = static_cast<int>(r % a.Hq), h = hq / a.G;
  if (t >= a.Tq) return;
  int b = 0;
  while (b < a.B && t >= a.cu[b + 1]) ++b;
  if (b == a.B || t < a.cu[b]) return;
  const int64_t start = a.cu[b], end = min(static_cast<int64_t>(a.cu[b + 1]), a.Tq);
  int i = static_cast<int>(t - start), n = static_cast<int>(end - start), len = n;
  if constexpr (kPaged) {
    const PagedSeq s = paged_seq(a, b);
    if (s.bad) *a.status = OFFQ_ERR_INVALID_ARG;
    if (s.n * a.G <= a.few_rows) return;
    len = s.len;
  } else if (a.cu[b + 1] > a.Tq) {
    *a.status = OFFQ_ERR_INVALID_ARG;
  }
  const int seen = kPaged ? min(len, len - n + i + 1) : a.causal ? i + 1 : n;
  for (int d = lane; d < D; d += 32)
    qs[warp][d] = to_f(static_cast<const T*>(a.q)[t * a.ld_q + static_cast<int64_t>(hq) * D + d]);
  __syncwarp();
  float m = -INFINITY, sum = 0.f, acc[D / 32] = {};
  for (int j0 = 0; j0 < seen; j0 += 32) {
    float s = -INFINITY;
    if (j0 + lane < seen) {
      s = 0.f;
      for (int d = 0; d < D; ++d) {
        const float k = element<D, T, kPaged>(a, 0, b, start, j0 + lane, h, d);
        if (kPaged && k == -INFINITY) {
          s = k;
          break;
        }
        s = fmaf(qs[warp][d], k, s);
      }
      s *= a.scale;
    }
    float top = s;
#pragma unroll
    for (int k = 16; k > 0; k >>= 1) top = fmaxf(top, __shfl_xor_sync(kAllLanes, top, k));
    const float next = fmaxf(m, top), keep = next == -INFINITY ? 1.f : __expf(m - next);
    const float p = s != -INFINITY && next != -INFINITY ? __expf(s - next) : 0.f;
    m = next;
    sum = sum * keep + p;
#pragma unroll
    for (int e = 0; e < D / 32; ++e) acc[e] *= keep;
    const int most = min(32, seen - j0);
    for (int k = 0; k < most; ++k) {
      const float pk = __shfl_sync(kAllLanes, p, k);
#pragma unroll
      for (int e = 0; e < D / 32; ++e)
        acc[e] = fmaf(pk, element<D, T, kPaged>(a, 1, b, start, j0 + k, h, lane + 32 * e), acc[e]);
    }
  }
#pragma unroll
  for (int k = 16; k > 0; k >>= 1) sum += __shfl_xor_sync(kAllLanes, sum, k);
  const float inv = sum > 0.f ? 1.f / sum : 0.f;
#pragma unroll
  for (int e = 0; e < D / 32; ++e)
    static_cast<T*>(a.out)[t * a.ld_out + static_cast<int64_t>(hq) * D + lane + 32 * e] = static_cast<T>(acc[e] * inv);
  if (a.lse != nullptr && lane == 0) a.lse[t * a.Hq + hq] = m + logf(sum);
}

template <bool kPaged>
int launch_rows(const AttnArgs& a, int dtype, int head_dim, cudaStream_t s) {
  const dim3 grid(static_cast<unsigned>((a.Tq * a.Hq + kRowWarps - 1) / kRowWarps)), block(kRowWarps * 32);
  if (head_dim == 128)
    return dtype == OFFQ_BF16 ? launch_pdl(attention_rows_kernel<128, __nv_bfloat16, kPaged>, grid, block, 0, s, a)
                              : launch_pdl(attention_rows_kernel<128, __half, kPaged>, grid, block, 0, s, a);
  return dtype == OFFQ_BF16 ? launch_pdl(attention_rows_kernel<64, __nv_bfloat16, kPaged>, grid, block, 0, s, a)
                            : launch_pdl(attention_rows_kernel<64, __half, kPaged>, grid, block, 0, s, a);
}

// What both calls ask of their queries, heads and outputs.
int check_attention(const void* q, int dtype, int64_t Tq, int32_t Hq, int32_t H, int32_t head_dim, int64_t ld_q,
                    int32_t B, float scale, int64_t ld_out) {
  if (elem_bytes(dtype) == 0 || Tq < 0 || Hq < 1 || H < 1 || Hq % H != 0 || head_dim < 1 || B < 0)
    return OFFQ_ERR_INVALID_ARG;
  if (!(scale > 0.f) || scale > 1e30f) return OFFQ_ERR_INVALID_ARG;
  if (dtype == OFFQ_F32 || (head_dim != 64 && head_dim != 128) || Hq > 4096 || Hq / H > 64 || B > 65535 ||
      Tq > (int64_t{1} << 24))
    return OFFQ_ERR_UNSUPPORTED;
  const int64_t width = static_cast<int64_t>(Hq) * head_dim;
  if (ld_q < width || ld_out < width) return OFFQ_ERR_INVALID_ARG;
  return OFFQ_OK;
}

bool row_ok(const void* p, int64_t ld) { return aligned(p, 16) && ld % 8 == 0; }

}  // namespace

extern "C" int64_t offq_paged_attention_workspace(int64_t Tq, int32_t Hq, int32_t H, int32_t head_dim, int32_t B,
                                                  int32_t max_q) {
  if (check_attention(nullptr, OFFQ_BF16, Tq, Hq, H, head_dim, int64_t{1} << 40, B, 1.f, int64_t{1} << 40) != OFFQ_OK ||
      max_q < 0)
    return -1;
  return Tq == 0 || B == 0 || max_q == 0 ? 0 : paged_few_workspace(head_dim);
}

extern "C" int offq_paged_attention(const void* q, int dtype, int64_t Tq, int32_t Hq, int32_t H, int32_t head_dim,
                                    int64_t ld_q, const uint8_t* k_codes, const float* k_params,
                                    const uint8_t* v_codes, const float* v_params, int64_t pages, int32_t page_size,
                                    const int32_t* block_table, int64_t ld_table, const int32_t* lens,
                                    const int32_t* cu_q, int32_t B, int32_t max_q, float scale, void* out,
                                    int64_t ld_out, float* lse, void* workspace, int64_t workspace_bytes,
                                    void* stream) {
  if (const int rc = check_attention(q, dtype, Tq, Hq, H, head_dim, ld_q, B, scale, ld_out); rc != OFFQ_OK) return rc;
  if (pages < 1 || page_size < 1 || ld_table < 0 || max_q < 0 || workspace_bytes < 0) return OFFQ_ERR_INVALID_ARG;
  if (!is_pow2(page_size) || page_size < 16 || page_size > 256 || pages > (int64_t{1} << 31)) return OFFQ_ERR_UNSUPPORTED;
  if (Tq == 0 || B == 0 || max_q == 0) return OFFQ_OK;
  if (q == nullptr || k_codes == nullptr || k_params == nullptr || v_codes == nullptr || v_params == nullptr ||
      block_table == nullptr || lens == nullptr || cu_q == nullptr || out == nullptr)
    return OFFQ_ERR_INVALID_ARG;
  if (!row_ok(q, ld_q) || !row_ok(out, ld_out) || !aligned(k_codes, 16) || !aligned(k_params, 16) ||
      !aligned(v_codes, 16) || !aligned(v_params, 16) || !aligned(block_table, 4) || !aligned(lens, 4) ||
      !aligned(cu_q, 4) || !aligned(lse, 4) || !aligned(workspace, 16))
    return OFFQ_ERR_MISALIGNED;
  AttnArgs a = {};
  a.q = q;
  a.ld_q = ld_q;
  a.Tq = Tq;
  a.Hq = Hq;
  a.H = H;
  a.G = Hq / H;
  a.k_codes = k_codes;
  a.v_codes = v_codes;
  a.k_params = k_params;
  a.v_params = v_params;
  a.pages = pages;
  a.page_shift = __builtin_ctz(static_cast<unsigned>(page_size));
  a.table = block_table;
  a.ld_table = ld_table;
  a.lens = lens;
  a.cu = cu_q;
  a.B = B;
  a.max_q = max_q;
  a.causal = 1;
  a.scale = scale;
  a.out = out;
  a.ld_out = ld_out;
  a.lse = lse;
  a.status = device_status_ptr();
  const int64_t need = paged_few_workspace(head_dim);
  if (a.status == nullptr || need < 0) return OFFQ_ERR_CUDA;
  if (workspace == nullptr || workspace_bytes < need) return OFFQ_ERR_INVALID_ARG;
  a.workspace = workspace;
  a.few_rows = kFewRows;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (const int rc = paged_few(a, dtype, head_dim, s); rc != OFFQ_OK) return rc;
  return static_cast<int64_t>(max_q) * a.G > kFewRows ? launch_rows<true>(a, dtype, head_dim, s) : OFFQ_OK;
}

extern "C" int offq_prompt_attention(const void* q, const void* k, const void* v, int dtype, int64_t T, int32_t Hq,
                                     int32_t H, int32_t head_dim, int64_t ld_q, int64_t ld_k, int64_t ld_v,
                                     const int32_t* cu, int32_t B, float scale, int32_t causal, void* out,
                                     int64_t ld_out, float* lse, void* stream) {
  if (const int rc = check_attention(q, dtype, T, Hq, H, head_dim, ld_q, B, scale, ld_out); rc != OFFQ_OK) return rc;
  const int64_t width = static_cast<int64_t>(H) * head_dim;
  if (ld_k < width || ld_v < width) return OFFQ_ERR_INVALID_ARG;
  if (T == 0 || B == 0) return OFFQ_OK;
  if (q == nullptr || k == nullptr || v == nullptr || cu == nullptr || out == nullptr) return OFFQ_ERR_INVALID_ARG;
  if (!row_ok(q, ld_q) || !row_ok(k, ld_k) || !row_ok(v, ld_v) || !row_ok(out, ld_out) || !aligned(cu, 4) ||
      !aligned(lse, 4))
    return OFFQ_ERR_MISALIGNED;
  AttnArgs a = {};
  a.q = q;
  a.ld_q = ld_q;
  a.Tq = T;
  a.Hq = Hq;
  a.H = H;
  a.G = Hq / H;
  a.k = k;
  a.v = v;
  a.ld_k = ld_k;
  a.ld_v = ld_v;
  a.cu = cu;
  a.B = B;
  a.causal = causal != 0;
  a.scale = scale;
  a.out = out;
  a.ld_out = ld_out;
  a.lse = lse;
  a.status = device_status_ptr();
  if (a.status == nullptr) return OFFQ_ERR_CUDA;
  return prompt_tc(a, dtype, head_dim, static_cast<cudaStream_t>(stream));
}
