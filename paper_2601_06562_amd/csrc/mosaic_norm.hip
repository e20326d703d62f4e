// Root-mean-square norm with the residual's addition and an 8-bit output, its backward pass, and activations stored
// in 8 bits.  All of it is bound by memory: every element is read once and written once, a row stays in registers between
// the sum of its squares and its use.  (Times below are of one MI355X, on which a copy of 2 GiB runs at 4.9 TB/s, read and
// written; a call of few rows is a launch, 4 us, and what the host does for it.)
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mosaic_layer_internal.h"

namespace mosaic {
namespace {

// ---- 8 bits: a lane holds 8 consecutive columns, so a group is 4, 8 or 16 neighbouring lanes.

constexpr float kTiny = 0x1p-112f;   // below it top / a could overflow, and scales would lie among the denormals

// Largest magnitude over the lanes of a group, as bits: the order of non-negative floats is that of their bits, and every
// NaN and infinity stays at or above 0x7f800000.
__device__ __forceinline__ uint32_t group_max_bits(const float (&v)[8], int lanes) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t b = __float_as_uint(v[i]) & 0x7fffffffu;
    m = b > m ? b : m;
  }
  for (int x = 1; x < lanes; x <<= 1) {
    const uint32_t o = (uint32_t)__shfl_xor((int)m, x, 64);
    m = o > m ? o : m;
  }
  return m;
}

// Eight values of a group whose largest magnitude has the bits `m`, as bytes; *scale is what restores them.
__device__ __forceinline__ uint2 to_q8(const float (&v)[8], uint32_t m, int format, float* scale) {
  const float top = format == MOSAIC_INT8 ? 127.0f : 448.0f;
  const float a = __uint_as_float(m);
  const bool finite = m < 0x7f800000u, stored = finite && a >= kTiny;
  *scale = finite ? (stored ? a / top : 0.0f) : __builtin_nanf("");
  if (!stored) return uint2{0u, 0u};
  const float up = top / a;
  uint2 w;
  if (format == MOSAIC_INT8) {
    uint32_t b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = (uint32_t)(int)__builtin_rintf(v[i] * up) & 0xffu;
    w.x = b[0] | b[1] << 8 | b[2] << 16 | b[3] << 24;
    w.y = b[4] | b[5] << 8 | b[6] << 16 | b[7] << 24;
  } else {
    int lo = 0, hi = 0;   // to nearest, ties to even; |v * up| <= 448 (1 + 2^-23), which rounds to 448
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * up, v[1] * up, lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[2] * up, v[3] * up, lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[4] * up, v[5] * up, hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[6] * up, v[7] * up, hi, true);
    w.x = (uint32_t)lo;
    w.y = (uint32_t)hi;
  }
  return w;
}

// What eight stored bytes stand for: value * scale, rounded to bf16 (so that a backward pass on the matrix cores and one
// in 32 bits see the same numbers).
__device__ __forceinline__ void from_q8(uint2 w, float scale, int format, float (&v)[8]) {
  if (format == MOSAIC_INT8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[i] = (float)(int8_t)(w.x >> (8 * i));
      v[i + 4] = (float)(int8_t)(w.y >> (8 * i));
    }
  } else {
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.x, true);
    const f32x2 c = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.y, false), e = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.y, true);
    v[0] = a[0]; v[1] = a[1]; v[2] = b[0]; v[3] = b[1];
    v[4] = c[0]; v[5] = c[1]; v[6] = e[0]; v[7] = e[1];
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (float)(__bf16)(v[i] * scale);
}

__device__ __forceinline__ void store_q8(const mosaic_q8_rows& q, int group_shift, int64_t row, int c, bool in,
                                         const float (&v)[8]) {
  const int lanes = 1 << (group_shift - 3);
  const uint32_t m = group_max_bits(v, lanes);
  float scale;
  const uint2 w = to_q8(v, m, q.format, &scale);
  if (!in) return;
  *reinterpret_cast<uint2*>(static_cast<uint8_t*>(q.values) + row * q.ld_values + c) = w;
  if ((c & ((1 << group_shift) - 1)) == 0) q.scales[row * q.ld_scales + (c >> group_shift)] = scale;
}

__device__ __forceinline__ int group_shift_of(int group) { return group == 32 ? 5 : group == 64 ? 6 : 7; }

__device__ __forceinline__ void load_q8(const mosaic_q8_rows& q, int group_shift, int64_t row, int c, float (&v)[8]) {
  const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(q.values) + row * q.ld_values + c);
  from_q8(w, q.scales[row * q.ld_scales + (c >> group_shift)], q.format, v);
}

__device__ __forceinline__ void load_gamma(const void* gamma, int f32, int c, float (&v)[8]) {
  if (f32) load8(static_cast<const float*>(gamma) + c, v);
  else load8(static_cast<const __bf16*>(gamma) + c, v);
}

// Sum over the R lanes of a row.  R > 64: over the block's waves through `lds`, whose half `turn` is this call's (the
// barrier of the next call stands between a half's use and its next).
template <int R, int N>
__device__ __forceinline__ void row_sum(float (&s)[N], float* lds, int turn) {
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) {
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] += __shfl_xor(s[i], x, 64);
  }
  if constexpr (R > 64) {
    constexpr int W = R / 64;
    float* at = lds + turn * (W * N);
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) at[i * W + (threadIdx.x >> 6)] = s[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float t = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) t += at[i * W + w];
      s[i] = t;
    }
  }
}

// y = s rstd gamma, s = x + residual in 32 bits, rstd = 1 / sqrt(mean s^2 + eps): R lanes hold a row (a wave, or a block of
// four), NV vectors of 8 columns each, so that the sum of squares is one exchange and the row is not read again.  Four waves a
// row beyond 1024 columns: 16384 x 4096 in bf16 in 97 us, where a wave a row, with four times the registers and fewer rows in
// flight, took 145.  32768 x 4096, 32-bit stream, with the 8-bit output: 332 us, 5.7 TB/s.  1 row: 4 us.
// Beyond 8192 columns a lane holds 64 of them and fewer rows are in flight: 4096 x 16384 in 143 us, 3.8 TB/s (32-bit stream
// 184, 4.4).
constexpr int kThreads = 256;

template <typename S, int R, int NV>
__global__ __launch_bounds__(kThreads) void rmsnorm_forward_kernel(const NormForwardArgs p) {
  constexpr int kRows = kThreads / R;
  constexpr bool kEarly = NV <= 2;   // room for the gains beside the row
  __shared__ float lds[2 * (R > 64 ? R / 64 : 1)];
  const int lane = threadIdx.x % R;
  int64_t n = p.T;
  if (p.idx != nullptr) {
    n = *p.count;
    if (n > p.max_rows) n = p.max_rows;
  }
  const int shift = group_shift_of(p.q8.group);
  int turn = 0;
  for (int64_t j = (int64_t)blockIdx.x * kRows + threadIdx.x / R; j < n; j += (int64_t)gridDim.x * kRows) {
    int64_t t = j;
    if (p.idx != nullptr) {
      t = p.idx[j];
      if (t < 0 || t >= p.T) continue;   // the same for all lanes of a row, and so, R > 64, for the block
    }
    float h[NV][8];
    float ss[1] = {0.f};
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * R + lane) * 8;
#pragma unroll
      for (int i = 0; i < 8; ++i) h[v][i] = 0.f;
      if (c < p.d && p.residual != nullptr) load8(static_cast<const S*>(p.residual) + t * p.ld_residual + c, h[v]);
    }
    if (p.x != nullptr) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = (v * R + lane) * 8;
        float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (c < p.d) load8(static_cast<const __bf16*>(p.x) + t * p.ld_x + c, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[v][i] += x[i];
      }
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * R + lane) * 8;
      if (c < p.d && p.sum != nullptr) store8(static_cast<S*>(p.sum) + t * p.ld_sum + c, h[v]);
#pragma unroll
      for (int i = 0; i < 8; ++i) ss[0] = __builtin_fmaf(h[v][i], h[v][i], ss[0]);
    }
    float gain[kEarly ? NV : 1][8];
    if constexpr (kEarly) {   // on their way while the sum is taken
#pragma unroll
      for (int v = 0; v < NV; ++v)
        if ((v * R + lane) * 8 < p.d) load_gamma(p.gamma, p.gamma_f32, (v * R + lane) * 8, gain[v]);
    }
    row_sum<R>(ss, lds, turn);
    turn ^= 1;
    const float rstd = 1.0f / __builtin_sqrtf(ss[0] / (float)p.d + p.eps);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * R + lane) * 8;
      const bool in = c < p.d;
      float (&g)[8] = gain[kEarly ? v : 0];
      if (!kEarly && in) load_gamma(p.gamma, p.gamma_f32, c, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) h[v][i] = in ? h[v][i] * rstd * g[i] : 0.f;
      if (in && p.y != nullptr) store8(static_cast<__bf16*>(p.y) + t * p.ld_y + c, h[v]);
      if (p.q8.values != nullptr) store_q8(p.q8, shift, t, c, in, h[v]);
    }
  }
}

enum { kFromBf16 = 0, kFromF32 = 1, kFromQ8 = 2 };
template <int FROM> struct Kept { using type = __bf16; };
template <> struct Kept<kFromF32> { using type = float; };
template <> struct Kept<kFromQ8> { using type = uint8_t; };

// Eight consecutive elements as they lie in memory.
template <typename T> struct Raw;
template <> struct Raw<__bf16> {
  bf16x8_t v;
  __device__ __forceinline__ void clear() { v = bf16x8_t{}; }
  __device__ __forceinline__ void load(const __bf16* p) { v = *reinterpret_cast<const bf16x8_t*>(p); }
  __device__ __forceinline__ void get(float (&f)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = (float)v[i];
  }
};
template <> struct Raw<float> {
  f32x4_t a, b;
  __device__ __forceinline__ void clear() { a = b = f32x4_t{}; }
  __device__ __forceinline__ void load(const float* p) {
    a = *reinterpret_cast<const f32x4_t*>(p);
    b = *reinterpret_cast<const f32x4_t*>(p + 4);
  }
  __device__ __forceinline__ void get(float (&f)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[i] = a[i]; f[i + 4] = b[i]; }
  }
};
template <> struct Raw<uint8_t> {
  uint2 bits;
  __device__ __forceinline__ void clear() { bits = uint2{0u, 0u}; }
  __device__ __forceinline__ void load(const uint8_t* p) { bits = *reinterpret_cast<const uint2*>(p); }
};

// The rows are dealt to gridDim.x * kRows groups of R lanes, each of which sums its rows' dy * n per column in registers
// and leaves one partial sum; norm_gamma_kernel adds those up.  Rows in turn, not in blocks: the same sums on every call.
// With n = h rstd and c = gamma dy the gradient is rstd (c - n mean(c n)): both sums of a row are one exchange.
// 16384 x 4096 in bf16: 110 us, 4.9 TB/s; without the next row on its way 114.  1003 x 3584 from 8 bits: 11 us, of which the
// traffic is 5: two rows a block leave little to overlap, and one or four a block take as long.  Beyond 4096 columns the next row
// is not asked for ahead, beyond 8192 a SIMD holds one wave: 8192 x 8192 in 112 us, 4.8 TB/s, 4096 x 16384 in 141, 3.8.
template <int FROM, typename S, int R, int NV>
__global__ __launch_bounds__(kThreads) void rmsnorm_backward_kernel(const NormBackwardArgs p) {
  constexpr int kRows = kThreads / R;
  __shared__ float lds[4 * (R > 64 ? R / 64 : 1)];
  const int lane = threadIdx.x % R;
  const int64_t first = (int64_t)blockIdx.x * kRows + threadIdx.x / R, stride = (int64_t)gridDim.x * kRows;
  const int shift = FROM == kFromQ8 ? group_shift_of(p.q8.group) : 0;
  // A row as it is loaded.  Where it fits the next row is asked for while one is worked on.
  struct Row {
    Raw<__bf16> dy[NV];
    Raw<typename Kept<FROM>::type> h[NV];
    float scale[FROM == kFromQ8 ? NV : 1];
    Raw<S> in[NV];
  };
  constexpr bool kAhead = NV <= 2;
  auto load = [&](Row& r, int64_t t) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * R + lane) * 8;
      r.dy[v].clear();
      r.h[v].clear();
      r.in[v].clear();
      if (FROM == kFromQ8) r.scale[v] = 0.f;
      if (c >= p.d) continue;
      r.dy[v].load(static_cast<const __bf16*>(p.dy) + t * p.ld_dy + c);
      if constexpr (FROM == kFromQ8) {
        r.h[v].load(static_cast<const uint8_t*>(p.q8.values) + t * p.q8.ld_values + c);
        r.scale[v] = p.q8.scales[t * p.q8.ld_scales + (c >> shift)];
      } else {
        r.h[v].load(static_cast<const typename Kept<FROM>::type*>(p.h) + t * p.ld_h + c);
      }
      if (p.dsum_in != nullptr) r.in[v].load(static_cast<const S*>(p.dsum_in) + t * p.ld_dsum_in + c);
    }
  };
  float dgamma[NV][8];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
#pragma unroll
    for (int i = 0; i < 8; ++i) dgamma[v][i] = 0.f;
  }
  Row row;
  if (kAhead && first < p.T) load(row, first);
  int turn = 0;
  for (int64_t t = first; t < p.T; t += stride) {
    if (!kAhead) load(row, t);
    float h[NV][8], dy[NV][8], out[NV][8];
    float s[2] = {0.f, 0.f};   // sums of h^2 and of gamma dy h
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * R + lane) * 8;
      row.dy[v].get(dy[v]);
      if constexpr (FROM == kFromQ8) from_q8(row.h[v].bits, row.scale[v], p.q8.format, h[v]);
      else row.h[v].get(h[v]);
      row.in[v].get(out[v]);
      float g[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (c < p.d) load_gamma(p.gamma, p.gamma_f32, c, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        s[0] = __builtin_fmaf(h[v][i], h[v][i], s[0]);
        s[1] = __builtin_fmaf(g[i] * dy[v][i], h[v][i], s[1]);
      }
    }
    if (kAhead && t + stride < p.T) load(row, t + stride);
    row_sum<R>(s, lds, turn);
    turn ^= 1;
    const float rstd = 1.0f / __builtin_sqrtf(s[0] / (float)p.d + p.eps);
    const float along = s[1] / (float)p.d * rstd;   // mean of c n
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * R + lane) * 8;
      if (c >= p.d) continue;
      float g[8];
      load_gamma(p.gamma, p.gamma_f32, c, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float n = h[v][i] * rstd;
        out[v][i] = __builtin_fmaf(rstd, __builtin_fmaf(-n, along, g[i] * dy[v][i]), out[v][i]);
        dgamma[v][i] = __builtin_fmaf(dy[v][i], n, dgamma[v][i]);
      }
      if (p.dsum != nullptr) store8(static_cast<S*>(p.dsum) + t * p.ld_dsum + c, out[v]);
    }
  }
  if (p.dgamma == nullptr) return;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * R + lane) * 8;
    if (c < p.d) store8(p.partials + first * p.d + c, dgamma[v]);
  }
}

// Adds `n` partial rows: 8 lanes of four columns, 64 strips of rows, joined in the waves, then in LDS (0.3 us less than by
// halves through LDS).  512 rows of 3584: 5 us, a launch and two rounds of loads; with 4 lanes, twice the blocks, 4.1 there but
// 1.5 us more at 8192 columns.
constexpr int kGammaThreads = 512, kGammaLanes = 8, kGammaStrips = kGammaThreads / kGammaLanes;
__global__ __launch_bounds__(kGammaThreads) void norm_gamma_kernel(const float* __restrict__ partials, int n, int d,
                                                                   int accumulate, float* __restrict__ dgamma) {
  __shared__ f32x4_t wave[kGammaThreads / 64][kGammaLanes];
  const int q = threadIdx.x % kGammaLanes, r0 = threadIdx.x / kGammaLanes;
  const int c = ((int)blockIdx.x * kGammaLanes + q) * 4;
  f32x4_t s = {0.f, 0.f, 0.f, 0.f};
  if (c < d) {
#pragma unroll 8
    for (int r = r0; r < n; r += kGammaStrips) s += *reinterpret_cast<const f32x4_t*>(partials + (int64_t)r * d + c);
  }
#pragma unroll
  for (int x = kGammaLanes; x < 64; x <<= 1) {
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] += __shfl_xor(s[i], x, 64);
  }
  if ((threadIdx.x & 63) < kGammaLanes) wave[threadIdx.x >> 6][q] = s;
  __syncthreads();
  if (r0 == 0 && c < d) {
#pragma unroll
    for (int w = 1; w < kGammaThreads / 64; ++w) s += wave[w][q];
    f32x4_t* out = reinterpret_cast<f32x4_t*>(dgamma + c);
    *out = accumulate ? *out + s : s;
  }
}

// A wave per row and turn; `padded` columns so that the lanes of a group all take part in its maximum.  The scale needs the
// group's columns alone, which neighbouring lanes hold: no exchange beyond 16 lanes, one pass.
// 65535 x 3584: bf16 stored in 134 to 148 us, restored in 116 to 130 (4.8 to 6.1 TB/s); 32-bit stored in 228, restored in 309
// (5.1 and 3.8 TB/s).
template <typename S>
__global__ __launch_bounds__(256) void checkpoint_store_kernel(const S* __restrict__ x, int64_t ld_x, int64_t T, int d,
                                                               const mosaic_q8_rows q8) {
  const int shift = group_shift_of(q8.group);
  const int padded = (d + q8.group - 1) >> shift << shift;
  for (int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); t < T; t += (int64_t)gridDim.x * 4) {
    for (int c = (threadIdx.x & 63) * 8; c < padded; c += 512) {
      float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (c < d) load8(x + t * ld_x + c, v);
      store_q8(q8, shift, t, c, c < d, v);
    }
  }
}

template <typename S>
__global__ __launch_bounds__(256) void checkpoint_load_kernel(const mosaic_q8_rows q8, int64_t T, int d, S* __restrict__ out,
                                                              int64_t ld_out) {
  const int shift = group_shift_of(q8.group);
  for (int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); t < T; t += (int64_t)gridDim.x * 4) {
#pragma unroll 4
    for (int c = (threadIdx.x & 63) * 8; c < d; c += 512) {
      float v[8];
      load_q8(q8, shift, t, c, v);
      store8(out + t * ld_out + c, v);
    }
  }
}

constexpr int64_t kMostBlocks = 1 << 20;   // beyond it the blocks take further rows (a launch has under 2^32 threads)
unsigned blocks_for(int64_t rows, int rows_per_block) {
  const int64_t b = (rows + rows_per_block - 1) / rows_per_block;
  return (unsigned)(b > kMostBlocks ? kMostBlocks : b);
}

// Lanes a row.
int lanes_for(int32_t d) { return d <= 1024 ? 64 : 256; }

template <typename S, int R, int NV>
int forward_as(const NormForwardArgs& a, int64_t rows, hipStream_t stream) {
  return launch_kernel(rmsnorm_forward_kernel<S, R, NV>, dim3(blocks_for(rows, kThreads / R)),
                       dim3(kThreads), stream, a);
}

template <typename S>
int forward_of(const NormForwardArgs& a, hipStream_t stream) {
  const int64_t rows = a.idx != nullptr ? a.max_rows : a.T;
  const int32_t d = a.d;
  if (d <= 512) return forward_as<S, 64, 1>(a, rows, stream);
  if (d <= 1024) return forward_as<S, 64, 2>(a, rows, stream);
  if (d <= 2048) return forward_as<S, 256, 1>(a, rows, stream);
  if (d <= 4096) return forward_as<S, 256, 2>(a, rows, stream);
  if (d <= 8192) return forward_as<S, 256, 4>(a, rows, stream);
  return forward_as<S, 256, 8>(a, rows, stream);
}

template <int FROM, typename S, int R, int NV>
int backward_as(const NormBackwardArgs& a, int64_t partials, hipStream_t stream) {
  constexpr int kRows = kThreads / R;
  return launch_kernel(rmsnorm_backward_kernel<FROM, S, R, NV>, dim3((unsigned)(partials / kRows)), dim3(kThreads),
                       stream, a);
}

template <int FROM, typename S>
int backward_of(const NormBackwardArgs& a, int64_t partials, hipStream_t stream) {
  const int32_t d = a.d;
  if (d <= 512) return backward_as<FROM, S, 64, 1>(a, partials, stream);
  if (d <= 1024) return backward_as<FROM, S, 64, 2>(a, partials, stream);
  if (d <= 2048) return backward_as<FROM, S, 256, 1>(a, partials, stream);
  if (d <= 4096) return backward_as<FROM, S, 256, 2>(a, partials, stream);
  if (d <= 8192) return backward_as<FROM, S, 256, 4>(a, partials, stream);
  return backward_as<FROM, S, 256, 8>(a, partials, stream);
}

}  // namespace

int launch_rmsnorm_forward(const NormForwardArgs& a, bool stream_f32, hipStream_t stream) {
  return stream_f32 ? forward_of<float>(a, stream) : forward_of<__bf16>(a, stream);
}

// Partial sums of dgamma, one for every group of lanes: two blocks a CU keep the memory busy, with at least two rows for a
// group, so that the next one can be on its way, and the sums cost a fraction of the rows.
constexpr int64_t kBackwardBlocks = 512;   // 16384 x 4096: 110 us, with 256 blocks 119; 8192 x 8192: 114, with 768 blocks 133
int64_t norm_backward_partials(int64_t T, int32_t d) {
  const int64_t groups = kThreads / lanes_for(d);
  int64_t blocks = (T + 2 * groups - 1) / (2 * groups);
  blocks = blocks > kBackwardBlocks ? kBackwardBlocks : blocks;
  return blocks * groups;
}

int launch_rmsnorm_backward(const NormBackwardArgs& a, bool stream_f32, hipStream_t stream) {
  const int64_t partials = norm_backward_partials(a.T, a.d);
  int rc = 0;
  if (a.T > 0) {
    if (a.h == nullptr) rc = stream_f32 ? backward_of<kFromQ8, float>(a, partials, stream) : backward_of<kFromQ8, __bf16>(a, partials, stream);
    else if (stream_f32) rc = backward_of<kFromF32, float>(a, partials, stream);
    else rc = backward_of<kFromBf16, __bf16>(a, partials, stream);
  }
  if (rc != 0 || a.dgamma == nullptr) return rc;
  return launch_kernel(norm_gamma_kernel, dim3((unsigned)((a.d + 4 * kGammaLanes - 1) / (4 * kGammaLanes))), dim3(kGammaThreads),
                       stream, a.partials, (int)partials, a.d, a.accumulate, a.dgamma);
}

int launch_checkpoint_store(const void* x, bool f32, int64_t ld_x, int64_t T, int32_t d, const mosaic_q8_rows& q8,
                            hipStream_t stream) {
  const dim3 grid(blocks_for(T, 4)), block(256);
  return f32 ? launch_kernel(checkpoint_store_kernel<float>, grid, block, stream, static_cast<const float*>(x), ld_x, T, d, q8)
             : launch_kernel(checkpoint_store_kernel<__bf16>, grid, block, stream, static_cast<const __bf16*>(x), ld_x, T, d, q8);
}

int launch_checkpoint_load(const mosaic_q8_rows& q8, int64_t T, int32_t d, void* out, bool f32, int64_t ld_out,
                           hipStream_t stream) {
  const dim3 grid(blocks_for(T, 4)), block(256);
  return f32 ? launch_kernel(checkpoint_load_kernel<float>, grid, block, stream, q8, T, d, static_cast<float*>(out), ld_out)
             : launch_kernel(checkpoint_load_kernel<__bf16>, grid, block, stream, q8, T, d, static_cast<__bf16*>(out), ld_out);
}

}  // namespace mosaic
