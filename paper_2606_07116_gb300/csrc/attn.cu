// Attention's entry points: packed prompts on 16-bit keys and values (offq_prompt_attention,
// csrc/attn_prompt.cu) and new tokens over the paged 4-bit cache (offq_paged_attention: csrc/attn_few.cu
// for few rows per sequence and key head, csrc/attn_chunk.cu for many); either over a window and sinks, and the latter
// behind prefixes that sequences share (csrc/attn_prefix.cu joins what the forms found).
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

// Most rows of a sequence that the few-row form takes.
int few_rows_of(AttnMode mode) { return mode == kCausal ? kFewRows : kFewGroupedRows; }

// Calls whose sequences may all have few rows need the small form's parts alone; others may take both forms, one
// after the other on the same bytes.
int64_t workspace_bytes_for(int head_dim, int64_t most_rows, AttnMode mode) {
  const int64_t few = paged_few_workspace(head_dim), chunk = paged_chunk_workspace(head_dim);
  if (few < 0 || chunk < 0) return -1;
  return most_rows > few_rows_of(mode) ? std::max(few, chunk) : few;
}

// Whether all sequences of a call that may have many rows take that form, and the other's two kernels (6 us on the device, as much
// to launch) stay away. A sequence with few rows costs a tile a head there, and a tile its blocks of 128 tokens and kTileBlocks
// more, 2.8 us each on one SM. How many there can be: of B sequences of up to `most` queries that share Tq, at most
// (B most - Tq) / (most - few) have no more than `few`; prefixes with few rows have one of them behind each. Their tokens are what
// tables and windows have room for, as lengths stand on the device. (Rows of q outside the sequences are counted as theirs: with
// many of them a batch of short sequences may be taken for long ones.)
// Measured, one chunk of 1000 tokens beside 1, 4 and 8 short sequences, 2 to 32 key heads, under a window and behind 4000 tokens: up
// to 600 blocks this form alone is 3 to 15 us faster (137 us against 147 for 600), at 1000 between 9 faster and 4 slower, at 1600 up
// to 12 slower, at 3200 6 to 31. Tables with more room than their sequences have tokens count for the two forms.
bool many_rows_alone(const AttnArgs& a, AttnMode mode) {
  constexpr int64_t kMostShortBlocks = 1000, kTileBlocks = 4;
  const int64_t most = std::min<int64_t>(a.max_q, a.Tq), few = kFewGroupedRows / a.G;
  if (most <= few) return false;
  const int64_t spare = static_cast<int64_t>(a.B) * most - a.Tq;
  const int64_t short_ones = std::min<int64_t>(a.B, std::max<int64_t>(0, spare) / (most - few));
  auto blocks = [&](int64_t tokens) { return (tokens + 127) / 128 + kTileBlocks; };
  int64_t tokens = a.ld_table << a.page_shift;
  if (mode == kWindowed) tokens = std::min(tokens, static_cast<int64_t>(a.window) + a.sinks + few + 16);
  int64_t cost = short_ones * blocks(tokens);
  if (mode == kShared) cost += std::min<int64_t>(a.P, short_ones) * blocks(a.ld_prefix << a.page_shift);
  return cost * a.H <= kMostShortBlocks;
}

// Behind shared prefixes: the most rows that a prefix may have, and the bytes of all rows' two sums and statistics.
int64_t shared_rows(int64_t Tq, int32_t B, int32_t max_q, int32_t G) {
  return std::min(Tq, static_cast<int64_t>(B) * max_q) * G;
}
int64_t sums_bytes(int64_t Tq, int32_t Hq, int32_t head_dim) {
  return 2 * Tq * Hq * (static_cast<int64_t>(sizeof(float)) * head_dim + static_cast<int64_t>(sizeof(float2)));
}

bool row_ok(const void* p, int64_t ld) { return aligned(p, 16) && ld % 8 == 0; }

}  // namespace

extern "C" int64_t offq_paged_attention_workspace(int64_t Tq, int32_t Hq, int32_t H, int32_t head_dim, int32_t B,
                                                  int32_t max_q) {
  if (check_attention(OFFQ_BF16, Tq, Hq, H, head_dim, int64_t{1} << 40, B, 1.f, int64_t{1} << 40) != OFFQ_OK ||
      max_q < 0)
    return -1;
  if (Tq == 0 || B == 0 || max_q == 0) return 0;
  return workspace_bytes_for(head_dim, static_cast<int64_t>(max_q) * (Hq / H), kCausal);
}

extern "C" int64_t offq_paged_attention_prefix_workspace(int64_t Tq, int32_t Hq, int32_t H, int32_t head_dim, int32_t B,
                                                         int32_t max_q, int32_t P) {
  if (P < 0 || P > 65535) return -1;
  const int64_t parts = offq_paged_attention_workspace(Tq, Hq, H, head_dim, B, max_q);
  if (parts <= 0 || P == 0) return parts;
  const int64_t most = workspace_bytes_for(head_dim, shared_rows(Tq, B, max_q, Hq / H), kShared);
  return most < 0 ? -1 : most + sums_bytes(Tq, Hq, head_dim);
}

extern "C" int64_t offq_paged_attention_window_workspace(int64_t Tq, int32_t Hq, int32_t H, int32_t head_dim, int32_t B,
                                                         int32_t max_q, int32_t page_size, int64_t ld_table,
                                                         int32_t window, int32_t sinks) {
  if (!is_pow2(page_size) || page_size < 16 || page_size > 256 || ld_table < 0 || window < 1 || sinks < 0) return -1;
  if (const int64_t none = offq_paged_attention_workspace(Tq, Hq, H, head_dim, B, max_q); none <= 0) return none;
  AttnArgs a = {};
  a.Tq = Tq;
  a.H = H;
  a.G = Hq / H;
  a.B = B;
  a.max_q = max_q;
  a.page_shift = __builtin_ctz(static_cast<unsigned>(page_size));
  a.ld_table = ld_table;
  a.window = std::min(window, kMostTokens);
  a.sinks = std::min(sinks, kMostTokens);
  a.few_rows = few_rows_of(kWindowed);
  const int64_t rows = static_cast<int64_t>(max_q) * a.G;
  return rows <= a.few_rows && paged_few_whole(a, kWindowed) ? 0 : workspace_bytes_for(head_dim, rows, kWindowed);
}

namespace {

// The paged calls' own arguments: checks and launches. `mode` says which of them was made.
int paged_call(AttnArgs& a, AttnMode mode, int dtype, int32_t head_dim, int32_t page_size, int64_t workspace_bytes,
               void* stream) {
  if (const int rc = check_attention(dtype, a.Tq, a.Hq, a.H, head_dim, a.ld_q, a.B, a.scale, a.ld_out); rc != OFFQ_OK)
    return rc;
  if (a.pages < 1 || page_size < 1 || a.ld_table < 0 || a.max_q < 0 || workspace_bytes < 0) return OFFQ_ERR_INVALID_ARG;
  if (mode == kWindowed && (a.window < 1 || a.sinks < 0)) return OFFQ_ERR_INVALID_ARG;
  if (mode == kShared && (a.P < 0 || a.ld_prefix < 0)) return OFFQ_ERR_INVALID_ARG;
  if (!is_pow2(page_size) || page_size < 16 || page_size > 256 || a.pages > (int64_t{1} << 31)) return OFFQ_ERR_UNSUPPORTED;
  if (mode == kShared && a.P > 65535) return OFFQ_ERR_UNSUPPORTED;
  if (a.Tq == 0 || a.B == 0 || a.max_q == 0) return OFFQ_OK;
  if (a.q == nullptr || a.k_codes == nullptr || a.k_params == nullptr || a.v_codes == nullptr || a.v_params == nullptr ||
      (a.table == nullptr && a.ld_table > 0) || a.lens == nullptr || a.cu == nullptr || a.out == nullptr)
    return OFFQ_ERR_INVALID_ARG;
  if (mode == kShared && a.P == 0) mode = kCausal;
  if (mode == kShared && ((a.prefix_table == nullptr && a.ld_prefix > 0) || a.prefix_lens == nullptr || a.cu_prefix == nullptr))
    return OFFQ_ERR_INVALID_ARG;
  if (!row_ok(a.q, a.ld_q) || !row_ok(a.out, a.ld_out) || !aligned(a.k_codes, 16) || !aligned(a.k_params, 16) ||
      !aligned(a.v_codes, 16) || !aligned(a.v_params, 16) || !aligned(a.table, 4) || !aligned(a.lens, 4) ||
      !aligned(a.cu, 4) || !aligned(a.lse, 4) || !aligned(a.workspace, 16))
    return OFFQ_ERR_MISALIGNED;
  if (mode == kShared && (!aligned(a.prefix_table, 4) || !aligned(a.prefix_lens, 4) || !aligned(a.cu_prefix, 4)))
    return OFFQ_ERR_MISALIGNED;
  a.G = a.Hq / a.H;
  a.page_shift = __builtin_ctz(static_cast<unsigned>(page_size));
  a.window = std::min(a.window, kMostTokens);
  a.sinks = std::min(a.sinks, kMostTokens);
  a.status = device_status_ptr();
  const int64_t own_rows = static_cast<int64_t>(a.max_q) * a.G;
  const int64_t most_rows = mode == kShared ? shared_rows(a.Tq, a.B, a.max_q, a.G) : own_rows;
  const bool many = most_rows > few_rows_of(mode), one_form = many && mode != kCausal && many_rows_alone(a, mode);
  const int64_t parts = workspace_bytes_for(head_dim, most_rows, mode);
  if (a.status == nullptr || parts < 0) return OFFQ_ERR_CUDA;
  a.few_rows = one_form ? 0 : few_rows_of(mode);
  a.whole = paged_few_whole(a, mode);
  int64_t need = mode == kShared ? parts + sums_bytes(a.Tq, a.Hq, head_dim) : parts;
  if (mode == kWindowed && a.whole && !many) need = 0;
  if (need > 0 && (a.workspace == nullptr || workspace_bytes < need)) return OFFQ_ERR_INVALID_ARG;
  if (mode == kShared) {
    a.sums = reinterpret_cast<float*>(static_cast<uint8_t*>(a.workspace) + parts);
    a.stats = reinterpret_cast<float2*>(a.sums + 2 * a.Tq * a.Hq * head_dim);
  }
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (!one_form)
    if (const int rc = paged_few(a, mode, dtype, head_dim, s); rc != OFFQ_OK) return rc;
  if (many)
    if (const int rc = paged_chunk(a, mode, dtype, head_dim, s); rc != OFFQ_OK) return rc;
  return mode == kShared ? join_shared(a, dtype, head_dim, s) : OFFQ_OK;
}

AttnArgs paged_args(const void* q, int64_t Tq, int32_t Hq, int32_t H, int64_t ld_q, const uint8_t* k_codes,
                    const float* k_params, const uint8_t* v_codes, const float* v_params, int64_t pages,
                    const int32_t* block_table, int64_t ld_table, const int32_t* lens, const int32_t* cu_q, int32_t B,
                    int32_t max_q, float scale, void* out, int64_t ld_out, float* lse, void* workspace) {
  AttnArgs a = {};
  a.q = q;
  a.ld_q = ld_q;
  a.Tq = Tq;
  a.Hq = Hq;
  a.H = H;
  a.k_codes = k_codes;
  a.v_codes = v_codes;
  a.k_params = k_params;
  a.v_params = v_params;
  a.pages = pages;
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
  a.workspace = workspace;
  return a;
}

int prompt_call(AttnArgs& a, AttnMode mode, int dtype, int32_t head_dim, void* stream) {
  if (const int rc = check_attention(dtype, a.Tq, a.Hq, a.H, head_dim, a.ld_q, a.B, a.scale, a.ld_out); rc != OFFQ_OK)
    return rc;
  const int64_t width = static_cast<int64_t>(a.H) * head_dim;
  if (a.ld_k < width || a.ld_v < width) return OFFQ_ERR_INVALID_ARG;
  if (mode == kWindowed && (a.window < 1 || a.sinks < 0)) return OFFQ_ERR_INVALID_ARG;
  if (a.Tq == 0 || a.B == 0) return OFFQ_OK;
  if (a.q == nullptr || a.k == nullptr || a.v == nullptr || a.cu == nullptr || a.out == nullptr) return OFFQ_ERR_INVALID_ARG;
  if (!row_ok(a.q, a.ld_q) || !row_ok(a.k, a.ld_k) || !row_ok(a.v, a.ld_v) || !row_ok(a.out, a.ld_out) ||
      !aligned(a.cu, 4) || !aligned(a.lse, 4))
    return OFFQ_ERR_MISALIGNED;
  a.G = a.Hq / a.H;
  a.window = std::min(a.window, kMostTokens);
  a.sinks = std::min(a.sinks, kMostTokens);
  a.status = device_status_ptr();
  if (a.status == nullptr) return OFFQ_ERR_CUDA;
  return prompt_tc(a, mode, dtype, head_dim, static_cast<cudaStream_t>(stream));
}

AttnArgs prompt_args(const void* q, const void* k, const void* v, int64_t T, int32_t Hq, int32_t H, int64_t ld_q,
                     int64_t ld_k, int64_t ld_v, const int32_t* cu, int32_t B, float scale, void* out, int64_t ld_out,
                     float* lse) {
  AttnArgs a = {};
  a.q = q;
  a.ld_q = ld_q;
  a.Tq = T;
  a.Hq = Hq;
  a.H = H;
  a.k = k;
  a.v = v;
  a.ld_k = ld_k;
  a.ld_v = ld_v;
  a.cu = cu;
  a.B = B;
  a.scale = scale;
  a.out = out;
  a.ld_out = ld_out;
  a.lse = lse;
  return a;
}

}  // namespace

extern "C" int offq_paged_attention(const void* q, int dtype, int64_t Tq, int32_t Hq, int32_t H, int32_t head_dim,
                                    int64_t ld_q, const uint8_t* k_codes, const float* k_params,
                                    const uint8_t* v_codes, const float* v_params, int64_t pages, int32_t page_size,
                                    const int32_t* block_table, int64_t ld_table, const int32_t* lens,
                                    const int32_t* cu_q, int32_t B, int32_t max_q, float scale, void* out,
                                    int64_t ld_out, float* lse, void* workspace, int64_t workspace_bytes,
                                    void* stream) {
  AttnArgs a = paged_args(q, Tq, Hq, H, ld_q, k_codes, k_params, v_codes, v_params, pages, block_table, ld_table, lens, cu_q,
                          B, max_q, scale, out, ld_out, lse, workspace);
  return paged_call(a, kCausal, dtype, head_dim, page_size, workspace_bytes, stream);
}

extern "C" int offq_paged_attention_window(const void* q, int dtype, int64_t Tq, int32_t Hq, int32_t H, int32_t head_dim,
                                           int64_t ld_q, const uint8_t* k_codes, const float* k_params,
                                           const uint8_t* v_codes, const float* v_params, int64_t pages,
                                           int32_t page_size, const int32_t* block_table, int64_t ld_table,
                                           const int32_t* lens, const int32_t* cu_q, int32_t B, int32_t max_q,
                                           float scale, int32_t window, int32_t sinks, void* out, int64_t ld_out,
                                           float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
  AttnArgs a = paged_args(q, Tq, Hq, H, ld_q, k_codes, k_params, v_codes, v_params, pages, block_table, ld_table, lens, cu_q,
                          B, max_q, scale, out, ld_out, lse, workspace);
  a.window = window;
  a.sinks = sinks;
  return paged_call(a, kWindowed, dtype, head_dim, page_size, workspace_bytes, stream);
}

extern "C" int offq_paged_attention_prefix(const void* q, int dtype, int64_t Tq, int32_t Hq, int32_t H, int32_t head_dim,
                                           int64_t ld_q, const uint8_t* k_codes, const float* k_params,
                                           const uint8_t* v_codes, const float* v_params, int64_t pages,
                                           int32_t page_size, const int32_t* block_table, int64_t ld_table,
                                           const int32_t* lens, const int32_t* cu_q, int32_t B, int32_t max_q,
                                           const int32_t* prefix_table, int64_t ld_prefix, const int32_t* prefix_lens,
                                           const int32_t* cu_prefix, int32_t P, float scale, void* out, int64_t ld_out,
                                           float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
  AttnArgs a = paged_args(q, Tq, Hq, H, ld_q, k_codes, k_params, v_codes, v_params, pages, block_table, ld_table, lens, cu_q,
                          B, max_q, scale, out, ld_out, lse, workspace);
  a.prefix_table = prefix_table;
  a.ld_prefix = ld_prefix;
  a.prefix_lens = prefix_lens;
  a.cu_prefix = cu_prefix;
  a.P = P;
  return paged_call(a, kShared, dtype, head_dim, page_size, workspace_bytes, stream);
}

extern "C" int offq_prompt_attention(const void* q, const void* k, const void* v, int dtype, int64_t T, int32_t Hq,
                                     int32_t H, int32_t head_dim, int64_t ld_q, int64_t ld_k, int64_t ld_v,
                                     const int32_t* cu, int32_t B, float scale, int32_t causal, void* out,
                                     int64_t ld_out, float* lse, void* stream) {
  AttnArgs a = prompt_args(q, k, v, T, Hq, H, ld_q, ld_k, ld_v, cu, B, scale, out, ld_out, lse);
  a.causal = causal != 0;
  return prompt_call(a, kCausal, dtype, head_dim, stream);
}

extern "C" int offq_prompt_attention_window(const void* q, const void* k, const void* v, int dtype, int64_t T, int32_t Hq,
                                            int32_t H, int32_t head_dim, int64_t ld_q, int64_t ld_k, int64_t ld_v,
                                            const int32_t* cu, int32_t B, float scale, int32_t window, int32_t sinks,
                                            void* out, int64_t ld_out, float* lse, void* stream) {
  AttnArgs a = prompt_args(q, k, v, T, Hq, H, ld_q, ld_k, ld_v, cu, B, scale, out, ld_out, lse);
  a.causal = 1;
  a.window = window;
  a.sinks = sinks;
  return prompt_call(a, kWindowed, dtype, head_dim, stream);
}
