// Internal declarations of the token operators (mosaic_tokens.h): argument blocks, launchers, layouts of workspaces.
#ifndef MOSAIC_TOKENS_INTERNAL_H_
#define MOSAIC_TOKENS_INTERNAL_H_

#include "mosaic_layer_internal.h"
#include "mosaic_tokens.h"

namespace mosaic {

// ---- embedding lookup (mosaic_embed.hip)
struct EmbedArgs {
  const int32_t* tokens;
  const int32_t* count;   // or nullptr
  const void* table;
  void* out;
  int64_t T, ld_table, ld_out;   // strides in elements
  int32_t V, d;
  float scale;
};
int launch_embedding_forward(const EmbedArgs& a, bool table_f32, bool out_f32, hipStream_t stream);

// Memory to be filled with a word: `rows` rows, `ld` bytes apart, of `row_bytes` bytes, a multiple of 16 as the base is.
struct FillArgs {
  void* base;
  int64_t ld, rows, row_bytes;
  uint32_t word;
};
int launch_fill(const FillArgs& f, hipStream_t stream);

// Positions sorted by their tokens: keys ascending, positions of a key ascending; what is left out has the key V and comes last.
struct SortedTokens {
  int32_t* keys;       // [n]
  int32_t* at;         // [n]
};
// Bytes that sorting n tokens takes.  `fill` (of no rows: nothing) is filled beside the sort.
int64_t sort_tokens_bytes(int64_t n);
int launch_sort_tokens(const int32_t* tokens, int64_t n, const int32_t* count, int32_t V, void* space, const FillArgs& fill, SortedTokens* out,
                       hipStream_t stream);

// Sums of rows by token, over sorted positions.
struct TokenSumArgs {
  SortedTokens sorted;
  const void* rows;      // [n, ld_rows]
  const float* weights;  // a factor for each row, or nullptr
  float* partials;       // [token_sum_partials(n), d]
  void* sums;            // of token v: row v; compact: row first[v], the place of its first position.  Rows without tokens are not written
  int32_t* first;        // compact: [V], written for tokens that there are; else nullptr
  int64_t n, ld_rows, ld_sums;
  int32_t V, d, accumulate;
  float scale;
};
int64_t token_sum_partials(int64_t n, int32_t d);
int launch_token_sums(const TokenSumArgs& a, bool rows_f32, bool sums_f32, hipStream_t stream);

// ---- dropout (mosaic_embed.hip)
struct DropoutArgs {
  const void* x;
  const void* residual;   // of out's type, or nullptr
  void* out;
  int64_t T, ld_x, ld_residual, ld_out, first_row;
  int32_t d;
  uint32_t border, key_low, key_high, site;
  float grow;
};
int launch_dropout(const DropoutArgs& a, bool x_f32, bool out_f32, hipStream_t stream);

// ---- log probabilities of given tokens (mosaic_logprob.hip)
struct LogprobArgs {
  const void* hidden;
  const void* w;
  const int32_t* idx;       // or nullptr: row j is row j
  const int32_t* count;     // or nullptr: max_rows of them
  const int32_t* targets;   // or nullptr
  float* out_logprob;       // or nullptr, as the next ones
  float* out_entropy;
  float* out_lse;
  int32_t* top_id;
  float* top_logprob;
  void* workspace;
  int64_t ld_h, ld_w, T, max_rows;   // strides in elements
  int32_t d, V, n_top;
};
int64_t logprob_workspace_bytes(int64_t T, int64_t ld_h, int64_t max_rows, int32_t d, int32_t V, int32_t n_top);
int launch_logprobs(const LogprobArgs& a, hipStream_t stream);

struct LogprobBackwardArgs {
  const void* hidden;
  const void* w;
  const int32_t* idx;        // or nullptr
  const int32_t* count;      // or nullptr
  const int32_t* targets;    // with dlogprob and logprob, or nullptr
  const float *logprob, *entropy, *lse, *dlogprob, *dentropy;   // entropy and dentropy: or nullptr
  void* dx;                  // bf16, or nullptr
  void* dw;                  // or nullptr
  void* workspace;
  int64_t ld_h, ld_w, ld_dx, ld_dw, T, max_rows, workspace_bytes;
  int32_t d, V, dw_f32, accumulate;
};
int64_t logprob_backward_workspace_bytes(int64_t max_rows, int32_t d, int32_t V, int64_t budget_bytes);
int64_t logprob_backward_least_bytes(int64_t max_rows, int32_t d, int32_t V);
int launch_logprobs_backward(const LogprobBackwardArgs& a, hipStream_t stream);

}  // namespace mosaic
#endif
