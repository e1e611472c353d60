// Attention's entry points: packed prompts on 16-bit keys and values (offq_prompt_attention,
// csrc/attn_prompt.cu) and new tokens over the paged 4-bit cache (offq_paged_attention: csrc/attn_few.cu
// for few rows per sequence and key head, csrc/attn_chunk.cu for many).
//
// out_i = sum_j p_ij v_j / sum_j p_ij,  p_ij = exp(scale q_i . k_j - m_i),  lse_i = m_i + log sum_j p_ij
// over the keys j that query i sees, m_i any number near their largest score.
#include <algorithm>

#include "attn.cuh"

namespace {

using namespace offq;

// What both calls ask of their queries, heads and outputs.
int check_attention(int dtype, int64_t Tq, int32_t Hq, int32_t H, int32_t head_dim, int64_t ld_q,
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

// Calls whose sequences may all have few rows need the small form's parts alone; others may take both forms, one
// after the other on the same bytes.
int64_t workspace_bytes_for(int head_dim, int64_t most_rows) {
  const int64_t few = paged_few_workspace(head_dim), chunk = paged_chunk_workspace(head_dim);
  if (few < 0 || chunk < 0) return -1;
  return most_rows > kFewRows ? std::max(few, chunk) : few;
}

bool row_ok(const void* p, int64_t ld) { return aligned(p, 16) && ld % 8 == 0; }

}  // namespace

extern "C" int64_t offq_paged_attention_workspace(int64_t Tq, int32_t Hq, int32_t H, int32_t head_dim, int32_t B,
                                                  int32_t max_q) {
  if (check_attention(OFFQ_BF16, Tq, Hq, H, head_dim, int64_t{1} << 40, B, 1.f, int64_t{1} << 40) != OFFQ_OK ||
      max_q < 0)
    return -1;
  if (Tq == 0 || B == 0 || max_q == 0) return 0;
  return workspace_bytes_for(head_dim, static_cast<int64_t>(max_q) * (Hq / H));
}

extern "C" int offq_paged_attention(const void* q, int dtype, int64_t Tq, int32_t Hq, int32_t H, int32_t head_dim,
                                    int64_t ld_q, const uint8_t* k_codes, const float* k_params,
                                    const uint8_t* v_codes, const float* v_params, int64_t pages, int32_t page_size,
                                    const int32_t* block_table, int64_t ld_table, const int32_t* lens,
                                    const int32_t* cu_q, int32_t B, int32_t max_q, float scale, void* out,
                                    int64_t ld_out, float* lse, void* workspace, int64_t workspace_bytes,
                                    void* stream) {
  if (const int rc = check_attention(dtype, Tq, Hq, H, head_dim, ld_q, B, scale, ld_out); rc != OFFQ_OK) return rc;
  if (pages < 1 || page_size < 1 || ld_table < 0 || max_q < 0 || workspace_bytes < 0) return OFFQ_ERR_INVALID_ARG;
  if (!is_pow2(page_size) || page_size < 16 || page_size > 256 || pages > (int64_t{1} << 31)) return OFFQ_ERR_UNSUPPORTED;
  if (Tq == 0 || B == 0 || max_q == 0) return OFFQ_OK;
  if (q == nullptr || k_codes == nullptr || k_params == nullptr || v_codes == nullptr || v_params == nullptr ||
      (block_table == nullptr && ld_table > 0) || lens == nullptr || cu_q == nullptr || out == nullptr)
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
  a.scale = scale;
  a.out = out;
  a.ld_out = ld_out;
  a.lse = lse;
  a.status = device_status_ptr();
  const int64_t most_rows = static_cast<int64_t>(max_q) * a.G;
  const int64_t need = workspace_bytes_for(head_dim, most_rows);
  if (a.status == nullptr || need < 0) return OFFQ_ERR_CUDA;
  if (workspace == nullptr || workspace_bytes < need) return OFFQ_ERR_INVALID_ARG;
  a.workspace = workspace;
  a.few_rows = kFewRows;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (const int rc = paged_few(a, dtype, head_dim, s); rc != OFFQ_OK) return rc;
  return most_rows > kFewRows ? paged_chunk(a, dtype, head_dim, s) : OFFQ_OK;
}

extern "C" int offq_prompt_attention(const void* q, const void* k, const void* v, int dtype, int64_t T, int32_t Hq,
                                     int32_t H, int32_t head_dim, int64_t ld_q, int64_t ld_k, int64_t ld_v,
                                     const int32_t* cu, int32_t B, float scale, int32_t causal, void* out,
                                     int64_t ld_out, float* lse, void* stream) {
  if (const int rc = check_attention(dtype, T, Hq, H, head_dim, ld_q, B, scale, ld_out); rc != OFFQ_OK) return rc;
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
