// Internal declarations of the layer operators (mosaic_layer.h): argument blocks, launchers, small device helpers.
#ifndef MOSAIC_LAYER_INTERNAL_H_
#define MOSAIC_LAYER_INTERNAL_H_

#include "mosaic_internal.h"
#include "mosaic_layer.h"

namespace mosaic {

// ---- norms and 8-bit rows (mosaic_norm.hip)
struct NormForwardArgs {
  const void* x;          // bf16 or nullptr
  const void* residual;   // stream type or nullptr
  const void* gamma;
  const int32_t* idx;     // nullptr: all rows
  const int32_t* count;
  void* sum;              // stream type or nullptr
  void* y;                // bf16 or nullptr
  mosaic_q8_rows q8;      // values == nullptr: none
  int64_t ld_x, ld_residual, ld_sum, ld_y;
  int64_t T, max_rows;
  float eps;
  int32_t d, gamma_f32;
};
int launch_rmsnorm_forward(const NormForwardArgs& a, bool stream_f32, hipStream_t stream);

struct NormBackwardArgs {
  const void* dy;         // bf16
  const void* h;          // stream type, or nullptr and q8
  mosaic_q8_rows q8;
  const void* gamma;
  const void* dsum_in;    // stream type or nullptr
  void* dsum;             // stream type or nullptr
  float* dgamma;          // or nullptr
  float* partials;        // [norm_backward_partials(T, d), d]
  int64_t ld_dy, ld_h, ld_dsum_in, ld_dsum;
  int64_t T;
  float eps;
  int32_t d, gamma_f32, accumulate;
};
int64_t norm_backward_partials(int64_t T, int32_t d);
int launch_rmsnorm_backward(const NormBackwardArgs& a, bool stream_f32, hipStream_t stream);

int launch_checkpoint_store(const void* x, bool f32, int64_t ld_x, int64_t T, int32_t d, const mosaic_q8_rows& q8,
                            hipStream_t stream);
int launch_checkpoint_load(const mosaic_q8_rows& q8, int64_t T, int32_t d, void* out, bool f32, int64_t ld_out,
                           hipStream_t stream);

// ---- gated feed-forward block (mosaic_ffn.hip)
struct FfnForwardArgs {
  const void* x;
  const void* w_gate;
  const void* w_up;
  void* out;
  int64_t ld_x, ld_w, ld_out, T;
  int32_t d, F, activation;
};
int launch_gated_ffn_forward(const FfnForwardArgs& a, hipStream_t stream);

struct FfnBackwardArgs {
  const void* dout;
  const void* x;
  const void* w_gate;
  const void* w_up;
  void* out;      // or nullptr
  void* dx;       // or nullptr
  void* dw_gate;  // or nullptr
  void* dw_up;
  void* grads;      // bf16 [ffn_gradient_rows(T), 2 F]: dg | du, for few rows their low halves behind them
  float* partials;  // fp32 [ffn_partial_rows(T), d]: sums of dx over parts of K and halves
  int64_t ld_dout, ld_x, ld_w, ld_out, ld_dx, ld_dw, T;
  int32_t d, F, activation, dw_f32, accumulate;
};
int64_t ffn_gradient_rows(int64_t T);
int64_t ffn_partial_rows(int64_t T);
int launch_gated_ffn_backward(const FfnBackwardArgs& a, hipStream_t stream);

#ifdef __HIPCC__
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;

// Eight consecutive elements, as 32-bit numbers.
__device__ __forceinline__ void load8(const __bf16* p, float (&v)[8]) {
  const bf16x8_t t = *reinterpret_cast<const bf16x8_t*>(p);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (float)t[i];
}
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const f32x4_t a = *reinterpret_cast<const f32x4_t*>(p), b = *reinterpret_cast<const f32x4_t*>(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[i + 4] = b[i]; }
}
__device__ __forceinline__ void store8(__bf16* p, const float (&v)[8]) {
  bf16x8_t t;
#pragma unroll
  for (int i = 0; i < 8; ++i) t[i] = (__bf16)v[i];   // to nearest, ties to even
  *reinterpret_cast<bf16x8_t*>(p) = t;
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  *reinterpret_cast<f32x4_t*>(p) = f32x4_t{v[0], v[1], v[2], v[3]};
  *reinterpret_cast<f32x4_t*>(p + 4) = f32x4_t{v[4], v[5], v[6], v[7]};
}
#endif

}  // namespace mosaic
#endif
