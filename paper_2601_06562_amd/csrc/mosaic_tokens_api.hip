// C ABI entry points of the token operators: argument validation, then enqueue.  See include/mosaic_tokens.h.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <initializer_list>

#include "mosaic_arguments.h"
#include "mosaic_tokens_internal.h"

namespace {

using namespace mosaic::arguments;

constexpr int32_t kMostVocab = INT32_MAX - 256;
// Listed rows: the kernels number them in 32 bits, in tiles of up to 256, the last of which ends below 2^31 as well.
constexpr int64_t kMostListed = ((int64_t)1 << 31) - 256;

int check_vocab(int32_t V) {
  if (V <= 0) return MOSAIC_ERR_INVALID_ARG;
  return V > kMostVocab ? MOSAIC_ERR_UNSUPPORTED_SHAPE : MOSAIC_OK;
}

// The row numbers that tokens, lists and counts are.
bool bad_list(const int32_t* tokens, const int32_t* count) { return tokens == nullptr || misaligned(tokens, 4) || misaligned(count, 4); }

struct EmbeddingSpace {
  int64_t partials, total;   // offsets, bytes; the sort's space comes first
};
EmbeddingSpace embedding_space(int64_t T, int32_t d) {
  EmbeddingSpace s;
  s.partials = mosaic::sort_tokens_bytes(T);
  s.total = s.partials + 4 * mosaic::token_sum_partials(T, d) * d;
  return s;
}

mosaic::FillArgs clear_matrix(void* base, int32_t type, int64_t ld, int64_t rows, int32_t d) {
  const int64_t bytes = type == MOSAIC_F32 ? 4 : 2;
  return mosaic::FillArgs{base, ld * bytes, rows, d * bytes, 0u};
}

int check_dropout(int32_t type, int64_t T, int32_t d, float p, int32_t site, int64_t first_row) {
  if (!known_type(type) || !(p >= 0.f && p <= 1.f - 0x1p-16f) || site < 0 || site == INT32_MAX || first_row < 0)
    return MOSAIC_ERR_INVALID_ARG;
  MOSAIC_RETURN_IF(check_sizes(T, d, MOSAIC_MAX_ROW));
  return first_row > INT64_MAX - T ? MOSAIC_ERR_UNSUPPORTED_SHAPE : MOSAIC_OK;
}
mosaic::DropoutArgs dropout_args(int64_t T, int32_t d, float p, uint64_t seed, int32_t site, int64_t first_row) {
  mosaic::DropoutArgs a = {};
  a.T = T;
  a.d = d;
  a.first_row = first_row;
  a.border = (uint32_t)lrint((double)p * 65536.0);
  a.grow = (float)(65536.0 / (65536.0 - a.border));
  a.key_low = (uint32_t)seed;
  a.key_high = (uint32_t)(seed >> 32);
  a.site = (uint32_t)site + 1;
  return a;
}

// The sizes of a list of rows; rows are asked for only where there are some.
int check_list_sizes(int64_t T, int64_t ld_h, int64_t max_rows, int32_t d, int32_t V) {
  MOSAIC_RETURN_IF(check_sizes(T, d, MOSAIC_MAX_ROW));
  MOSAIC_RETURN_IF(check_vocab(V));
  if (max_rows < 0) return MOSAIC_ERR_INVALID_ARG;
  if (max_rows > kMostListed || ld_h < d || ld_h % 8 != 0 || ld_h > kMaxStride) return MOSAIC_ERR_UNSUPPORTED_SHAPE;
  return MOSAIC_OK;
}

}  // namespace

extern "C" {

int mosaic_embedding_forward(const int32_t* tokens, int64_t T, const int32_t* count, const void* table, int32_t table_type,
                             int64_t ld_table, int32_t V, int32_t d, float scale, void* out, int32_t out_type,
                             int64_t ld_out, void* stream) {
  if (!known_type(table_type) || !known_type(out_type) || !isfinite(scale)) return MOSAIC_ERR_INVALID_ARG;
  MOSAIC_RETURN_IF(check_sizes(T, d, MOSAIC_MAX_ROW));
  MOSAIC_RETURN_IF(check_vocab(V));
  if (T == 0) return MOSAIC_OK;
  if (bad_list(tokens, count)) return MOSAIC_ERR_INVALID_ARG;
  MOSAIC_RETURN_IF(check_matrix(table, ld_table, d));
  MOSAIC_RETURN_IF(check_matrix(out, ld_out, d));
  mosaic::EmbedArgs a = {};
  a.tokens = tokens;
  a.count = count;
  a.table = table;
  a.out = out;
  a.T = T;
  a.ld_table = ld_table;
  a.ld_out = ld_out;
  a.V = V;
  a.d = d;
  a.scale = scale;
  return launched(mosaic::launch_embedding_forward(a, table_type == MOSAIC_F32, out_type == MOSAIC_F32, static_cast<hipStream_t>(stream)));
}

int64_t mosaic_embedding_backward_workspace_bytes(int64_t T, int32_t d, int32_t V) {
  if (check_sizes(T, d, MOSAIC_MAX_ROW) != MOSAIC_OK || check_vocab(V) != MOSAIC_OK) return 0;
  return embedding_space(T, d).total;
}

int mosaic_embedding_backward(const void* dout, int32_t dout_type, int64_t ld_dout, const int32_t* tokens, int64_t T,
                              const int32_t* count, int32_t V, int32_t d, float scale, void* dtable, int32_t dtable_type,
                              int64_t ld_dtable, int32_t accumulate, void* workspace, int64_t workspace_bytes,
                              void* stream) {
  if (!known_type(dout_type) || !known_type(dtable_type) || !isfinite(scale) || (accumulate != 0 && dtable_type != MOSAIC_F32))
    return MOSAIC_ERR_INVALID_ARG;
  MOSAIC_RETURN_IF(check_sizes(T, d, MOSAIC_MAX_ROW));
  MOSAIC_RETURN_IF(check_vocab(V));
  MOSAIC_RETURN_IF(check_matrix(dtable, ld_dtable, d));
  if (T > 0) {
    if (bad_list(tokens, count)) return MOSAIC_ERR_INVALID_ARG;
    MOSAIC_RETURN_IF(check_matrix(dout, ld_dout, d));
    if (workspace == nullptr || misaligned(workspace)) return MOSAIC_ERR_INVALID_ARG;
    if (workspace_bytes < mosaic_embedding_backward_workspace_bytes(T, d, V)) return MOSAIC_ERR_WORKSPACE_TOO_SMALL;
  } else if (accumulate != 0) {
    return MOSAIC_OK;
  }
  hipStream_t on = static_cast<hipStream_t>(stream);
  const mosaic::FillArgs fill = clear_matrix(dtable, dtable_type, ld_dtable, accumulate != 0 ? 0 : V, d);
  if (T == 0) return launched(mosaic::launch_fill(fill, on));
  mosaic::TokenSumArgs a = {};
  if (mosaic::launch_sort_tokens(tokens, T, count, V, workspace, fill, &a.sorted, on) != 0) return MOSAIC_ERR_HIP;
  a.rows = dout;
  a.partials = reinterpret_cast<float*>(static_cast<char*>(workspace) + embedding_space(T, d).partials);
  a.sums = dtable;
  a.n = T;
  a.ld_rows = ld_dout;
  a.ld_sums = ld_dtable;
  a.V = V;
  a.d = d;
  a.accumulate = accumulate != 0;
  a.scale = scale;
  return launched(mosaic::launch_token_sums(a, dout_type == MOSAIC_F32, dtable_type == MOSAIC_F32, on));
}

int mosaic_dropout_forward(const void* x, int64_t ld_x, const void* residual, int32_t stream_type, int64_t ld_residual,
                           int64_t T, int32_t d, float p, uint64_t seed, int32_t site, int64_t first_row, void* out,
                           int64_t ld_out, void* stream) {
  MOSAIC_RETURN_IF(check_dropout(stream_type, T, d, p, site, first_row));
  if (T == 0) return MOSAIC_OK;
  MOSAIC_RETURN_IF(check_matrix(x, ld_x, d));
  MOSAIC_RETURN_IF(check_optional(residual, ld_residual, d));
  MOSAIC_RETURN_IF(check_matrix(out, ld_out, d));
  mosaic::DropoutArgs a = dropout_args(T, d, p, seed, site, first_row);
  a.x = x;
  a.residual = residual;
  a.out = out;
  a.ld_x = ld_x;
  a.ld_residual = ld_residual;
  a.ld_out = ld_out;
  return launched(mosaic::launch_dropout(a, false, stream_type == MOSAIC_F32, static_cast<hipStream_t>(stream)));
}

int mosaic_dropout_backward(const void* dout, int32_t stream_type, int64_t ld_dout, int64_t T, int32_t d, float p,
                            uint64_t seed, int32_t site, int64_t first_row, void* dx, int64_t ld_dx, void* stream) {
  MOSAIC_RETURN_IF(check_dropout(stream_type, T, d, p, site, first_row));
  if (T == 0) return MOSAIC_OK;
  MOSAIC_RETURN_IF(check_matrix(dout, ld_dout, d));
  MOSAIC_RETURN_IF(check_matrix(dx, ld_dx, d));
  mosaic::DropoutArgs a = dropout_args(T, d, p, seed, site, first_row);
  a.x = dout;
  a.out = dx;
  a.ld_x = ld_dout;
  a.ld_out = ld_dx;
  return launched(mosaic::launch_dropout(a, stream_type == MOSAIC_F32, false, static_cast<hipStream_t>(stream)));
}

int64_t mosaic_masked_logprobs_workspace_bytes(int64_t T, int64_t ld_h, int64_t max_rows, int32_t d, int32_t V, int32_t n_top) {
  if (check_list_sizes(T, ld_h, max_rows, d, V) != MOSAIC_OK || n_top < 0 || n_top > MOSAIC_MAX_TOP) return 0;
  return mosaic::logprob_workspace_bytes(T, ld_h, max_rows, d, V, n_top);
}

int mosaic_masked_logprobs(const void* hidden, int64_t ld_h, int64_t T, int32_t d, const void* w, int64_t ld_w, int32_t V,
                           const int32_t* idx, const int32_t* count, int64_t max_rows, const int32_t* targets,
                           float* out_logprob, float* out_entropy, float* out_lse, int32_t n_top, int32_t* top_id,
                           float* top_logprob, void* workspace, int64_t workspace_bytes, void* stream) {
  if (n_top < 0 || n_top > MOSAIC_MAX_TOP || (idx == nullptr) != (count == nullptr)) return MOSAIC_ERR_INVALID_ARG;
  MOSAIC_RETURN_IF(check_list_sizes(T, ld_h, max_rows, d, V));
  if (idx == nullptr && max_rows != T) return MOSAIC_ERR_INVALID_ARG;
  if (T == 0 || max_rows == 0) return MOSAIC_OK;
  if ((out_logprob == nullptr && out_entropy == nullptr && out_lse == nullptr && n_top == 0) ||
      (out_logprob != nullptr && targets == nullptr) || (n_top > 0 && (top_id == nullptr || top_logprob == nullptr)))
    return MOSAIC_ERR_INVALID_ARG;
  for (const void* p : {(const void*)idx, (const void*)count, (const void*)targets, (const void*)out_logprob, (const void*)out_entropy,
                        (const void*)out_lse, (const void*)top_id, (const void*)top_logprob})
    if (misaligned(p, 4)) return MOSAIC_ERR_INVALID_ARG;
  MOSAIC_RETURN_IF(check_matrix(hidden, ld_h, d));
  MOSAIC_RETURN_IF(check_matrix(w, ld_w, d));
  if (workspace == nullptr || misaligned(workspace)) return MOSAIC_ERR_INVALID_ARG;
  if (workspace_bytes < mosaic_masked_logprobs_workspace_bytes(T, ld_h, max_rows, d, V, n_top)) return MOSAIC_ERR_WORKSPACE_TOO_SMALL;
  mosaic::LogprobArgs a = {};
  a.hidden = hidden;
  a.w = w;
  a.idx = idx;
  a.count = count;
  a.targets = out_logprob != nullptr ? targets : nullptr;
  a.out_logprob = out_logprob;
  a.out_entropy = out_entropy;
  a.out_lse = out_lse;
  a.top_id = top_id;
  a.top_logprob = top_logprob;
  a.workspace = workspace;
  a.ld_h = ld_h;
  a.ld_w = ld_w;
  a.T = T;
  a.max_rows = max_rows;
  a.d = d;
  a.V = V;
  a.n_top = n_top;
  return launched(mosaic::launch_logprobs(a, static_cast<hipStream_t>(stream)));
}

int64_t mosaic_masked_logprobs_backward_workspace_bytes(int64_t max_rows, int32_t d, int32_t V, int64_t budget_bytes) {
  if (check_list_sizes(0, d, max_rows, d, V) != MOSAIC_OK || max_rows == 0) return 0;
  return mosaic::logprob_backward_workspace_bytes(max_rows, d, V, budget_bytes);
}

int mosaic_masked_logprobs_backward(const void* hidden, int64_t ld_h, int64_t T, int32_t d, const void* w, int64_t ld_w, int32_t V,
                                    const int32_t* idx, const int32_t* count, int64_t max_rows, const int32_t* targets,
                                    const float* logprob, const float* entropy, const float* lse, const float* dlogprob,
                                    const float* dentropy, void* dx, int64_t ld_dx, void* dw, int32_t dw_type, int64_t ld_dw,
                                    int32_t accumulate, void* workspace, int64_t workspace_bytes, void* stream) {
  if (!known_type(dw_type) || (accumulate != 0 && dw != nullptr && dw_type != MOSAIC_F32) || (idx == nullptr) != (count == nullptr))
    return MOSAIC_ERR_INVALID_ARG;
  MOSAIC_RETURN_IF(check_list_sizes(T, ld_h, max_rows, d, V));
  if (idx == nullptr && max_rows != T) return MOSAIC_ERR_INVALID_ARG;
  MOSAIC_RETURN_IF(check_optional(dw, ld_dw, d));
  const bool some = T > 0 && max_rows > 0;
  if (some) {
    if ((dx == nullptr && dw == nullptr) || (dlogprob == nullptr && dentropy == nullptr) || lse == nullptr ||
        (dlogprob != nullptr && (targets == nullptr || logprob == nullptr)) || (dentropy != nullptr && entropy == nullptr))
      return MOSAIC_ERR_INVALID_ARG;
    for (const void* p : {(const void*)idx, (const void*)count, (const void*)targets, (const void*)logprob, (const void*)entropy,
                          (const void*)lse, (const void*)dlogprob, (const void*)dentropy})
      if (misaligned(p, 4)) return MOSAIC_ERR_INVALID_ARG;
    MOSAIC_RETURN_IF(check_matrix(hidden, ld_h, d));
    MOSAIC_RETURN_IF(check_matrix(w, ld_w, d));
    MOSAIC_RETURN_IF(check_optional(dx, ld_dx, d));
    if (workspace == nullptr || misaligned(workspace)) return MOSAIC_ERR_INVALID_ARG;
    if (workspace_bytes < mosaic::logprob_backward_least_bytes(max_rows, d, V)) return MOSAIC_ERR_WORKSPACE_TOO_SMALL;
  }
  hipStream_t on = static_cast<hipStream_t>(stream);
  if (!some) {   // no rows: dw is cleared
    if (dw == nullptr || accumulate != 0) return MOSAIC_OK;
    return launched(mosaic::launch_fill(clear_matrix(dw, dw_type, ld_dw, V, d), on));
  }
  mosaic::LogprobBackwardArgs a = {};
  a.hidden = hidden;
  a.w = w;
  a.idx = idx;
  a.count = count;
  a.targets = dlogprob != nullptr ? targets : nullptr;
  a.logprob = logprob;
  a.entropy = entropy;
  a.lse = lse;
  a.dlogprob = dlogprob;
  a.dentropy = dentropy;
  a.dx = dx;
  a.dw = dw;
  a.workspace = workspace;
  a.ld_h = ld_h;
  a.ld_w = ld_w;
  a.ld_dx = ld_dx;
  a.ld_dw = ld_dw;
  a.T = T;
  a.max_rows = max_rows;
  a.workspace_bytes = workspace_bytes;
  a.d = d;
  a.V = V;
  a.dw_f32 = dw_type == MOSAIC_F32;
  a.accumulate = accumulate != 0;
  return launched(mosaic::launch_logprobs_backward(a, on));
}

}  // extern "C"
