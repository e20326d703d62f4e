// C ABI entry points of the layer operators: argument validation, then enqueue.  See include/mosaic_layer.h.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "mosaic_layer_internal.h"

namespace {

constexpr int64_t kMaxRows = (int64_t)1 << 31;
constexpr int64_t kMaxStride = (int64_t)1 << 21;   // elements: 256 rows of a tile stay within 2^31 bytes

bool misaligned(const void* p, uintptr_t bytes = 16) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }

// A [rows, cols] matrix argument.  INVALID_ARG: absent or misaligned; UNSUPPORTED_SHAPE: a stride the kernels do not take.
int check_matrix(const void* p, int64_t ld, int64_t cols) {
  if (p == nullptr || misaligned(p)) return MOSAIC_ERR_INVALID_ARG;
  if (ld < cols || ld % 8 != 0 || ld > kMaxStride) return MOSAIC_ERR_UNSUPPORTED_SHAPE;
  return MOSAIC_OK;
}
int check_optional(const void* p, int64_t ld, int64_t cols) { return p == nullptr ? MOSAIC_OK : check_matrix(p, ld, cols); }

int check_sizes(int64_t T, int64_t cols, int64_t most) {
  if (T < 0 || cols <= 0) return MOSAIC_ERR_INVALID_ARG;
  if (T >= kMaxRows || cols % 8 != 0 || cols > most) return MOSAIC_ERR_UNSUPPORTED_SHAPE;
  return MOSAIC_OK;
}

bool known_type(int32_t t) { return t == MOSAIC_BF16 || t == MOSAIC_F32; }

int check_q8(const mosaic_q8_rows* q, int32_t d) {
  if (q == nullptr || q->values == nullptr || q->scales == nullptr || misaligned(q->values, 8) || misaligned(q->scales, 4) ||
      (q->format != MOSAIC_INT8 && q->format != MOSAIC_E4M3) || (q->group != 32 && q->group != 64 && q->group != 128))
    return MOSAIC_ERR_INVALID_ARG;
  if (q->ld_values < d || q->ld_values % 8 != 0 || q->ld_scales < (d + q->group - 1) / q->group)
    return MOSAIC_ERR_UNSUPPORTED_SHAPE;
  return MOSAIC_OK;
}

int64_t round_up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// Workspace of a feed-forward backward pass: dg | du, the restored input, the partial sums of dx, which only up to
// kPartialT rows are summed in parts.  A workspace for T rows serves fewer rows, too.
struct FfnSpace {
  int64_t restored, partials, total;   // offsets, bytes
};
constexpr int64_t kPartialT = 4096;
FfnSpace ffn_space(int64_t T, int32_t d, int32_t F, bool q8) {
  FfnSpace s;
  s.restored = round_up(4 * mosaic::ffn_gradient_rows(T) * F, 256);
  s.partials = s.restored + (q8 ? round_up(2 * T * d, 256) : 0);
  const int64_t few = T < kPartialT ? T : kPartialT;   // the most that up to T rows need with their sums
  const int64_t with_sums = round_up(4 * mosaic::ffn_gradient_rows(few) * F, 256) + (q8 ? round_up(2 * few * d, 256) : 0) +
                            4 * mosaic::ffn_partial_rows(few) * d;
  s.total = with_sums > s.partials ? with_sums : s.partials;
  return s;
}

int launched(int rc) { return rc == 0 ? MOSAIC_OK : MOSAIC_ERR_HIP; }

#define MOSAIC_RETURN_IF(expr)                  \
  do {                                          \
    const int status_ = (expr);                 \
    if (status_ != MOSAIC_OK) return status_;   \
  } while (0)

}  // namespace

extern "C" {

int mosaic_checkpoint_store(const void* x, int32_t type, int64_t ld_x, int64_t T, int32_t d, const mosaic_q8_rows* q8,
                            void* stream) {
  if (!known_type(type)) return MOSAIC_ERR_INVALID_ARG;
  MOSAIC_RETURN_IF(check_sizes(T, d, MOSAIC_MAX_NORM_ROW));
  if (T == 0) return MOSAIC_OK;
  MOSAIC_RETURN_IF(check_matrix(x, ld_x, d));
  MOSAIC_RETURN_IF(check_q8(q8, d));
  return launched(mosaic::launch_checkpoint_store(x, type == MOSAIC_F32, ld_x, T, d, *q8, static_cast<hipStream_t>(stream)));
}

int mosaic_checkpoint_load(const mosaic_q8_rows* q8, int64_t T, int32_t d, void* out, int32_t type, int64_t ld_out,
                           void* stream) {
  if (!known_type(type)) return MOSAIC_ERR_INVALID_ARG;
  MOSAIC_RETURN_IF(check_sizes(T, d, MOSAIC_MAX_NORM_ROW));
  if (T == 0) return MOSAIC_OK;
  MOSAIC_RETURN_IF(check_matrix(out, ld_out, d));
  MOSAIC_RETURN_IF(check_q8(q8, d));
  return launched(mosaic::launch_checkpoint_load(*q8, T, d, out, type == MOSAIC_F32, ld_out, static_cast<hipStream_t>(stream)));
}

int mosaic_rmsnorm_forward(const void* x, int64_t ld_x, const void* residual, int32_t stream_type, int64_t ld_residual,
                           const void* gamma, int32_t gamma_type, float eps, int64_t T, int32_t d, const int32_t* idx,
                           const int32_t* count, int64_t max_rows, void* sum, int64_t ld_sum, void* y, int64_t ld_y,
                           const mosaic_q8_rows* q8, void* stream) {
  if (!known_type(stream_type) || !known_type(gamma_type) || !(eps > 0.f) || isinf(eps) ||
      (idx == nullptr) != (count == nullptr) || (idx != nullptr && (max_rows < 0 || max_rows > T)))
    return MOSAIC_ERR_INVALID_ARG;
  MOSAIC_RETURN_IF(check_sizes(T, d, MOSAIC_MAX_NORM_ROW));
  if (T == 0 || (idx != nullptr && max_rows == 0)) return MOSAIC_OK;
  if ((x == nullptr && residual == nullptr) || (sum == nullptr && y == nullptr && q8 == nullptr) || gamma == nullptr ||
      misaligned(gamma) || misaligned(idx, 4) || misaligned(count, 4))
    return MOSAIC_ERR_INVALID_ARG;
  MOSAIC_RETURN_IF(check_optional(x, ld_x, d));
  MOSAIC_RETURN_IF(check_optional(residual, ld_residual, d));
  MOSAIC_RETURN_IF(check_optional(sum, ld_sum, d));
  MOSAIC_RETURN_IF(check_optional(y, ld_y, d));
  if (q8 != nullptr) MOSAIC_RETURN_IF(check_q8(q8, d));
  mosaic::NormForwardArgs a = {};
  a.x = x;
  a.residual = residual;
  a.gamma = gamma;
  a.idx = idx;
  a.count = count;
  a.sum = sum;
  a.y = y;
  if (q8 != nullptr) a.q8 = *q8;
  a.ld_x = ld_x;
  a.ld_residual = ld_residual;
  a.ld_sum = ld_sum;
  a.ld_y = ld_y;
  a.T = T;
  a.max_rows = max_rows;
  a.eps = eps;
  a.d = d;
  a.gamma_f32 = gamma_type == MOSAIC_F32;
  return launched(mosaic::launch_rmsnorm_forward(a, stream_type == MOSAIC_F32, static_cast<hipStream_t>(stream)));
}

int64_t mosaic_rmsnorm_backward_workspace_bytes(int64_t T, int32_t d) {
  if (check_sizes(T, d, MOSAIC_MAX_NORM_ROW) != MOSAIC_OK) return 0;
  return 4 * mosaic::norm_backward_partials(T, d) * d;
}

int mosaic_rmsnorm_backward(const void* dy, int64_t ld_dy, const void* h, int64_t ld_h, const mosaic_q8_rows* q8,
                            int32_t stream_type, const void* gamma, int32_t gamma_type, float eps, int64_t T, int32_t d,
                            const void* dsum_in, int64_t ld_dsum_in, void* dsum, int64_t ld_dsum, float* dgamma,
                            int32_t accumulate, void* workspace, int64_t workspace_bytes, void* stream) {
  if (!known_type(stream_type) || !known_type(gamma_type) || !(eps > 0.f) || isinf(eps) ||
      (dsum == nullptr && dgamma == nullptr) || misaligned(dgamma))
    return MOSAIC_ERR_INVALID_ARG;
  MOSAIC_RETURN_IF(check_sizes(T, d, MOSAIC_MAX_NORM_ROW));
  if (T > 0) {
    if ((h == nullptr) == (q8 == nullptr) || gamma == nullptr || misaligned(gamma)) return MOSAIC_ERR_INVALID_ARG;
    MOSAIC_RETURN_IF(check_matrix(dy, ld_dy, d));
    MOSAIC_RETURN_IF(check_optional(h, ld_h, d));
    if (q8 != nullptr) MOSAIC_RETURN_IF(check_q8(q8, d));
    MOSAIC_RETURN_IF(check_optional(dsum_in, ld_dsum_in, d));
    MOSAIC_RETURN_IF(check_optional(dsum, ld_dsum, d));
    if (dgamma != nullptr) {
      if (workspace == nullptr || misaligned(workspace)) return MOSAIC_ERR_INVALID_ARG;
      if (workspace_bytes < mosaic_rmsnorm_backward_workspace_bytes(T, d)) return MOSAIC_ERR_WORKSPACE_TOO_SMALL;
    }
  }
  if (T == 0 && (dgamma == nullptr || accumulate)) return MOSAIC_OK;
  mosaic::NormBackwardArgs a = {};
  a.dy = dy;
  a.h = h;
  if (q8 != nullptr) a.q8 = *q8;
  a.gamma = gamma;
  a.dsum_in = dsum_in;
  a.dsum = dsum;
  a.dgamma = dgamma;
  a.partials = static_cast<float*>(workspace);
  a.ld_dy = ld_dy;
  a.ld_h = ld_h;
  a.ld_dsum_in = ld_dsum_in;
  a.ld_dsum = ld_dsum;
  a.T = T;
  a.eps = eps;
  a.d = d;
  a.gamma_f32 = gamma_type == MOSAIC_F32;
  a.accumulate = accumulate != 0;
  return launched(mosaic::launch_rmsnorm_backward(a, stream_type == MOSAIC_F32, static_cast<hipStream_t>(stream)));
}

int mosaic_gated_ffn_forward(const void* x, int64_t ld_x, const void* w_gate, const void* w_up, int64_t ld_w, int64_t T,
                             int32_t d, int32_t F, int32_t activation, void* out, int64_t ld_out, void* stream) {
  if (activation != MOSAIC_SILU && activation != MOSAIC_GELU_TANH) return MOSAIC_ERR_INVALID_ARG;
  MOSAIC_RETURN_IF(check_sizes(T, d, MOSAIC_MAX_ROW));
  MOSAIC_RETURN_IF(check_sizes(T, F, MOSAIC_MAX_ROW));
  if (T == 0) return MOSAIC_OK;
  MOSAIC_RETURN_IF(check_matrix(x, ld_x, d));
  MOSAIC_RETURN_IF(check_matrix(w_gate, ld_w, d));
  MOSAIC_RETURN_IF(check_matrix(w_up, ld_w, d));
  MOSAIC_RETURN_IF(check_matrix(out, ld_out, F));
  mosaic::FfnForwardArgs a = {};
  a.x = x;
  a.w_gate = w_gate;
  a.w_up = w_up;
  a.out = out;
  a.ld_x = ld_x;
  a.ld_w = ld_w;
  a.ld_out = ld_out;
  a.T = T;
  a.d = d;
  a.F = F;
  a.activation = activation;
  return launched(mosaic::launch_gated_ffn_forward(a, static_cast<hipStream_t>(stream)));
}

int64_t mosaic_gated_ffn_backward_workspace_bytes(int64_t T, int32_t d, int32_t F, int32_t q8_input) {
  if (check_sizes(T, d, q8_input != 0 ? MOSAIC_MAX_NORM_ROW : MOSAIC_MAX_ROW) != MOSAIC_OK ||
      check_sizes(T, F, MOSAIC_MAX_ROW) != MOSAIC_OK)
    return 0;
  return ffn_space(T, d, F, q8_input != 0).total;
}

int mosaic_gated_ffn_backward(const void* dout, int64_t ld_dout, const void* x, int64_t ld_x, const mosaic_q8_rows* q8,
                              const void* w_gate, const void* w_up, int64_t ld_w, int64_t T, int32_t d, int32_t F,
                              int32_t activation, void* out, int64_t ld_out, void* dx, int64_t ld_dx, void* dw_gate,
                              void* dw_up, int32_t dw_type, int64_t ld_dw, int32_t accumulate, void* workspace,
                              int64_t workspace_bytes, void* stream) {
  if ((activation != MOSAIC_SILU && activation != MOSAIC_GELU_TANH) || !known_type(dw_type) ||
      (dw_gate == nullptr) != (dw_up == nullptr) || (accumulate != 0 && dw_gate != nullptr && dw_type != MOSAIC_F32) ||
      (dx == nullptr && dw_gate == nullptr && out == nullptr))
    return MOSAIC_ERR_INVALID_ARG;
  MOSAIC_RETURN_IF(check_sizes(T, d, q8 != nullptr ? MOSAIC_MAX_NORM_ROW : MOSAIC_MAX_ROW));
  MOSAIC_RETURN_IF(check_sizes(T, F, MOSAIC_MAX_ROW));
  MOSAIC_RETURN_IF(check_optional(dw_gate, ld_dw, d));
  MOSAIC_RETURN_IF(check_optional(dw_up, ld_dw, d));
  if (T > 0) {
    if ((x == nullptr) == (q8 == nullptr)) return MOSAIC_ERR_INVALID_ARG;
    MOSAIC_RETURN_IF(check_matrix(dout, ld_dout, F));
    MOSAIC_RETURN_IF(check_optional(x, ld_x, d));
    if (q8 != nullptr) MOSAIC_RETURN_IF(check_q8(q8, d));
    MOSAIC_RETURN_IF(check_matrix(w_gate, ld_w, d));
    MOSAIC_RETURN_IF(check_matrix(w_up, ld_w, d));
    MOSAIC_RETURN_IF(check_optional(out, ld_out, F));
    MOSAIC_RETURN_IF(check_optional(dx, ld_dx, d));
    if (workspace == nullptr || misaligned(workspace)) return MOSAIC_ERR_INVALID_ARG;
    if (workspace_bytes < mosaic_gated_ffn_backward_workspace_bytes(T, d, F, q8 != nullptr))
      return MOSAIC_ERR_WORKSPACE_TOO_SMALL;
  }
  if (T == 0 && (dw_gate == nullptr || accumulate != 0)) return MOSAIC_OK;
  const FfnSpace at = ffn_space(T, d, F, q8 != nullptr);
  char* ws = static_cast<char*>(workspace);
  mosaic::FfnBackwardArgs a = {};
  a.dout = dout;
  a.x = x;
  a.ld_x = ld_x;
  if (T > 0 && q8 != nullptr) {
    a.x = ws + at.restored;
    a.ld_x = d;
    const int rc = mosaic::launch_checkpoint_load(*q8, T, d, ws + at.restored, false, d, static_cast<hipStream_t>(stream));
    if (rc != 0) return MOSAIC_ERR_HIP;
  }
  a.w_gate = w_gate;
  a.w_up = w_up;
  a.out = out;
  a.dx = dx;
  a.dw_gate = dw_gate;
  a.dw_up = dw_up;
  a.grads = ws;
  a.partials = reinterpret_cast<float*>(ws + at.partials);
  a.ld_dout = ld_dout;
  a.ld_w = ld_w;
  a.ld_out = ld_out;
  a.ld_dx = ld_dx;
  a.ld_dw = ld_dw;
  a.T = T;
  a.d = d;
  a.F = F;
  a.activation = activation;
  a.dw_f32 = dw_type == MOSAIC_F32;
  a.accumulate = accumulate != 0;
  return launched(mosaic::launch_gated_ffn_backward(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
