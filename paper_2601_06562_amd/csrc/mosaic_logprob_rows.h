// What the kernels that make logits tile by tile do with them (mosaic_logprob.hip, mosaic_logprob_w4.h): statistics of rows,
// candidates for their most probable ids, gradients at the logits.  Device code.
//
// In both kernels a wave holds 128 ids of a tile by 16 QB rows, in blocks of 16 x 16: lane l has ids 16 i + 4 (l / 16) + r, i < 8,
// r < 4, of rows 16 j + l % 16, j < QB ("columns").  A row of a wave lies in four lanes, 16 apart; what is kept of it between tiles
// one of them holds, its owner: of column j lane group j % 4.  `load(j, x)` gives a column's 32 elements, x[4 i + r].  ROLLED:
// columns are taken in a loop, so that the code is there once; where the compiler holds the accumulators, unrolled costs less.
#ifndef MOSAIC_LOGPROB_ROWS_H_
#define MOSAIC_LOGPROB_ROWS_H_

#include <hip/hip_runtime.h>
#include <limits.h>
#include <stdint.h>

#include "mosaic_schedule.h"
#include "mosaic_tile.h"
#include "mosaic_tokens_internal.h"

namespace mosaic {
namespace logprob {

using namespace tile;

constexpr int kCus = 256;
constexpr int kVocab = 256;            // ids of a tile
constexpr int kHalf = kVocab / 2;      // ids of a wave's half
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNeg = -0x1p100f;      // "minus infinity" that survives subtraction; a power of two, so that
constexpr float kNegExponent = kNeg * kLog2e;   // this is exact
constexpr int kMostTop = MOSAIC_MAX_TOP;
constexpr int kListRoom = 16;          // candidates a lane keeps of a row until they are sorted in

// A candidate for a row's most probable ids: a positive double that is the larger the earlier it comes, by logit, then by the lower id
// (32 bits of one in the order of unsigned numbers, 31 of the other counted down: no NaN but of a NaN), so that two instructions put
// two in order, where a comparison of 64-bit whole numbers and the selects behind it are seven.  0: none.
typedef double Candidate;
__device__ __forceinline__ Candidate candidate_of(float x, int32_t id) {
  const uint32_t b = __float_as_uint(x + 0.f), up = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);   // (-0 as 0)
  return __longlong_as_double((long long)((uint64_t)up << 31 | (0x7fffffffu - (uint32_t)id)));
}
__device__ __forceinline__ float logit_of(Candidate c) {
  const uint32_t up = (uint32_t)((uint64_t)__double_as_longlong(c) >> 31);
  return __uint_as_float(up ^ ((up & 0x80000000u) != 0 ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ int32_t id_of(Candidate c) { return (int32_t)(0x7fffffffu - ((uint32_t)__double_as_longlong(c) & 0x7fffffffu)); }
// The first and the second of two; as statements, since the compiler quiets what it takes for signalling NaNs beforehand.
__device__ __forceinline__ Candidate first_of_two(Candidate a, Candidate b) {
  Candidate c;
  asm("v_max_f64 %0, %1, %2" : "=v"(c) : "v"(a), "v"(b));
  return c;
}
__device__ __forceinline__ Candidate second_of_two(Candidate a, Candidate b) {
  Candidate c;
  asm("v_min_f64 %0, %1, %2" : "=v"(c) : "v"(a), "v"(b));
  return c;
}

struct Entry { float x; int32_t id; };   // of a lane's own list

struct LogitParams {
  const char* w;
  const char* x;
  int64_t ld_w, ld_x;        // bytes
  const int32_t* idx;        // or nullptr: x holds the listed rows side by side
  const int32_t* count;      // or nullptr
  const int32_t* targets;    // or nullptr
  int32_t T, max_rows, V, d, n_top;
  // statistics: of the halves of every part of the vocabulary (`found` says how many parts, and the rows of one)
  float *part_e, *part_s, *part_t;
  Candidate* part_top;       // n_top each
  float* target_logit;       // [max_rows]
  Entry* lists;              // of every block's waves: kListRoom x columns x 64 lanes
  int32_t* found;
  ScheduleInput sched;       // mosaic_logprob_w4.h
  // gradients: of V ids from `first_id` on, for max_rows rows (zeros from the last listed one on)
  const float *lse, *entropy, *dlogprob, *dentropy;   // the last three each with what needs them, else nullptr
  char* dl;                  // bf16 [max_rows, ld_dl]
  int64_t ld_dl, low;        // bytes; low: from a row to what its rounding left over, 0: not wanted
  int32_t first_id, all_ids;
  int32_t dl_ids;            // ids that dl holds, a multiple of 8
};
// Alternatives are a kernel's own: without them its code is a quarter, and most of a short call's time goes to fetching code.  So are
// gradients with low halves: asked for at each tile, they took 1% of a call without.
enum { kStatistics, kAlternatives, kGradients, kGradientsLow };
constexpr bool gradient_mode(int mode) { return mode == kGradients || mode == kGradientsLow; }

// A kernel's arguments, read where they are used: what is made of a tile uses many, and kept from one tile to the next they would
// take the scalar registers that the products need.
typedef const __attribute__((address_space(4))) LogitParams* Arguments;
__device__ __forceinline__ Arguments arguments_again() {
  auto at = __builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(at));
  return (Arguments)at;
}

__device__ __forceinline__ int rows_found(const LogitParams& p) {
  if (p.count == nullptr) return p.max_rows;
  const int n = *p.count;
  return n < 0 ? 0 : n < p.max_rows ? n : p.max_rows;
}

// A pointer among them points into device memory, which the compiler cannot tell of one that it did not see passed in.
template <typename T>
__device__ __forceinline__ __attribute__((address_space(1))) T* in_memory(T* x) { return (__attribute__((address_space(1))) T*)x; }
// The same number, of which the compiler does not know that it is the same from one turn of a loop to the next: left alone it makes a
// loop of its own for every such condition (a width's code 60 KB, which no instruction cache holds).
__device__ __forceinline__ int opaque(int x) {
  x = __builtin_amdgcn_readfirstlane(x);
  asm volatile("" : "+s"(x));
  return x;
}

// Over the four lanes that hold one row.
template <typename F>
__device__ __forceinline__ float over_row(float x, F f) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  const float y = f(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(y), __float_as_uint(y), false, false);
  return f(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float row_max(float x) { return over_row(x, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ float row_min(float x) { return over_row(x, [](float a, float b) { return fminf(a, b); }); }
__device__ __forceinline__ float row_sum(float x) { return over_row(x, [](float a, float b) { return a + b; }); }

// The largest number below x (of those that are no denormals).
__device__ __forceinline__ float below(float x) {
  const int b = __float_as_int(x);
  if (__builtin_fabsf(x) < 0x1p-125f) return -0x1p-125f;
  return __int_as_float(b > 0 ? b - 1 : b + 1);
}

// What a lane holds between tiles, of rows 16 (4 k + lane / 16) + lane % 16 of its wave, k < kOwn.  With u = x log2 e - e, e a whole
// number, so that a change of e only ever scales s by a power of two and u is rounded once:
//   s, t   sum 2^u, sum u 2^u        (log-sum-exp: (e + log2 s) / log2 e;  entropy: (log2 s - t / s) / log2 e)
//   tau    ids of later tiles with a logit of tau or less are none of the n_top best of this half
//   n      candidates that are sorted in
template <int QB>
struct Rows {
  static constexpr int kOwn = (QB + 3) / 4;
  float e[kOwn], s[kOwn], t[kOwn], tau[kOwn];
  int n[kOwn];
  uint32_t listed[kOwn];   // of columns 4 k .. 4 k + 3, a byte each: candidates in this lane's own lists

  // row0: the wave's first row.  Rows past the last have no candidates.
  __device__ __forceinline__ void clear(int row0, int rows) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
      e[k] = kNegExponent;
      s[k] = t[k] = 0.f;
      tau[k] = row0 + 64 * k + lane < rows ? kNeg : __builtin_inff();
      n[k] = 0;
      listed[k] = 0;
    }
  }
};

// Element k of an array of one or two, k the same in all lanes.
template <typename T, int N>
__device__ __forceinline__ T pick(const T (&a)[N], int k) {
  if constexpr (N == 1) return a[0];
  else return k == 0 ? a[0] : a[1];
}
template <typename T, int N>
__device__ __forceinline__ void put(T (&a)[N], int k, bool own, T v) {
  a[0] = own && k == 0 ? v : a[0];
  if constexpr (N > 1) a[1] = own && k == 1 ? v : a[1];
}

// Sorts the candidates of this lane's own row k into the n best of before, in part_top at `to`: by logit, then by id.
template <int N, int QB>
__device__ __forceinline__ void sort_in(Rows<QB>& st, int k, const Entry* lists, Candidate* to, bool owner, int n) {
  const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4;
  const uint32_t own_lists = pick(st.listed, k);
  int here[4], most = 0;   // of the row's four lanes
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    here[q] = __shfl((int)own_lists, l16 + 16 * q, 64) >> (8 * g) & 255;
    most = here[q] > most ? here[q] : most;
  }
  const int before = pick(st.n, k);
  int all = before;
  float last = kNeg;
  if (owner) {
    const Entry* from = lists + (int64_t)(4 * k + g) * kListRoom * 64 + l16;
    Candidate best[N];
#pragma unroll
    for (int m = 0; m < N; ++m) {
      const Candidate c = to[m < before ? m : 0];
      best[m] = m < before ? c : 0.0;
    }
    // four entries of each lane's list at a time, the next ones under way
    constexpr int kAtOnce = 4;
    Entry ahead[kAtOnce][4];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) ahead[i][q] = from[i * 64 + 16 * q];
#pragma unroll 1
    for (int e = 0; e < most; e += kAtOnce) {
      Candidate c[kAtOnce][4];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const bool in = e + i < here[q];
          all += in ? 1 : 0;
          c[i][q] = in ? candidate_of(ahead[i][q].x, ahead[i][q].id) : 0.0;
          ahead[i][q] = from[(e + kAtOnce + i < kListRoom ? e + kAtOnce + i : 0) * 64 + 16 * q];
        }
      }
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          Candidate x = c[i][q];
#pragma unroll
          for (int m = 0; m < N; ++m) {
            const Candidate other = best[m];
            best[m] = first_of_two(x, other);
            x = second_of_two(x, other);
          }
        }
      }
    }
#pragma unroll
    for (int m = 0; m < N; ++m) {
      if (m < n) {
        to[m] = best[m];
        last = best[m] != 0.0 ? logit_of(best[m]) : kNeg;
      }
    }
  }
  put(st.n, k, owner, all < n ? all : n);
  put(st.tau, k, owner && all >= n, fmaxf(last, kNeg));
}

// All own rows.  place(k, in): where the candidates of own row k go, and whether there is such a row.
template <int QB, class Place>
__device__ __forceinline__ void sort_all_in(Rows<QB>& st, const Entry* lists, int n, Place place) {
  const int g = (threadIdx.x & 63) >> 4;
  __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "workgroup");   // the lists' entries were stored by other lanes
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll 1
  for (int k = 0; k < Rows<QB>::kOwn; ++k) {
    bool in = 4 * k + g < QB;
    Candidate* to = place(k, in);
    if (n <= 8) sort_in<8, QB>(st, k, lists, to, in, n);
    else sort_in<16, QB>(st, k, lists, to, in, n);
    put(st.listed, k, true, 0u);
  }
  __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "workgroup");   // and are free for others
}

template <bool ROLLED, int N, class F>
__device__ __forceinline__ void each_column(F f) {
  if constexpr (ROLLED) {
#pragma unroll 1
    for (int j = 0; j < N; ++j) f(j);
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) f(j);
  }
}

// Sorts N = 2, 4, 8, ... numbers that first fall and then rise, or the reverse, largest first.
template <int N>
__device__ __forceinline__ void sort_bitonic(float* v) {
#pragma unroll
  for (int half = N / 2; half >= 1; half /= 2) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if ((i & half) != 0) continue;
      const float a = v[i], b = v[i + half];
      v[i] = fmaxf(a, b);
      v[i + half] = fminf(a, b);
    }
  }
}
// Sorts any eight, largest first.
__device__ __forceinline__ void sort_eight(float (&v)[8]) {
#pragma unroll
  for (int n = 2; n <= 8; n *= 2) {
#pragma unroll
    for (int i = 0; i < 8; i += n) {   // every other run the other way round
      if (n < 8 && (i & n) != 0) {
#pragma unroll
        for (int k = 0; k < n; ++k) v[i + k] = -v[i + k];
      }
#pragma unroll
      for (int half = n / 2; half >= 1; half /= 2) {
#pragma unroll
        for (int k = 0; k < n; ++k) {
          if ((k & half) != 0) continue;
          const float x = v[i + k], y = v[i + k + half];
          v[i + k] = fmaxf(x, y);
          v[i + k + half] = fminf(x, y);
        }
      }
      if (n < 8 && (i & n) != 0) {
#pragma unroll
        for (int k = 0; k < n; ++k) v[i + k] = -v[i + k];
      }
    }
  }
}
template <int N>
__device__ __forceinline__ void exchange16(const float (&v)[N], float (&lo)[N], float (&hi)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[i]), __float_as_uint(v[i]), false, false);
    lo[i] = __uint_as_float(r[0]);
    hi[i] = __uint_as_float(r[1]);
  }
}
template <int N>
__device__ __forceinline__ void exchange32(const float (&v)[N], float (&lo)[N], float (&hi)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[i]), __float_as_uint(v[i]), false, false);
    lo[i] = __uint_as_float(r[0]);
    hi[i] = __uint_as_float(r[1]);
  }
}
// A number that at least n of a row's ids of this tile reach: the n-th largest of the largest of 16 sets of eight ids, four of
// which lie in each of the row's lanes; for n > 8 the 16th of 32 sets of four.  Of two sorted lists, one reversed, the larger of
// each two are the largest of all.  q: the largest of each quad.  Of 128 ids 3.5, 5.8, 10.6 and 22 reach it for n = 3, 5, 8 and 16.
__device__ __forceinline__ float reached_by(const float (&q)[8], int n) {
  float bound;
  if (n <= 8) {
    float v[4], lo[4], hi[4], all[8], low[8], high[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = fmaxf(q[2 * i], q[2 * i + 1]);
    const float a = fmaxf(v[0], v[1]), b = fminf(v[0], v[1]), c = fminf(v[2], v[3]), d = fmaxf(v[2], v[3]);   // falls, then rises
    v[0] = a; v[1] = b; v[2] = c; v[3] = d;
    sort_bitonic<4>(v);
    exchange16(v, lo, hi);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      all[i] = lo[i];
      all[4 + i] = hi[3 - i];
    }
    sort_bitonic<8>(all);
    exchange32(all, low, high);
#pragma unroll
    for (int i = 0; i < 8; ++i) all[i] = fmaxf(low[i], high[7 - i]);
    sort_bitonic<8>(all);
    bound = all[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) bound = i < n ? all[i] : bound;
  } else {
    float v[8], lo[8], hi[8], all[16], low[16], high[16];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = q[i];
    sort_eight(v);
    exchange16(v, lo, hi);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      all[i] = lo[i];
      all[8 + i] = hi[7 - i];
    }
    sort_bitonic<16>(all);
    exchange32(all, low, high);
    bound = fmaxf(low[0], high[15]);
#pragma unroll
    for (int i = 1; i < 16; ++i) bound = fminf(bound, fmaxf(low[i], high[15 - i]));
  }
  return bound;
}

// A lane's list of a column, as a buffer that nothing goes beyond.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t list_buffer(Entry* list) {
  return __builtin_amdgcn_make_buffer_rsrc(list, 0, kListRoom * 64 * (int)sizeof(Entry), 0x00020000);
}
// Puts x and its id at `to` of a lane's list and moves on, where x is above `pass`; elsewhere it goes past the buffer, which drops it: a
// branch around each store, which some lane nearly always takes, is two jumps (900 rows of 32000 x 1024, five alternatives: 128 us, so
// 122; a column's stores are a microsecond of the 2.5 that it takes then).
__device__ __forceinline__ void append_above(float x, float pass, int32_t id, __amdgpu_buffer_rsrc_t list, uint32_t& to) {
  typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_t;
  static_assert(sizeof(Entry) == 8, "an entry is two words");
  const bool in = x > pass;
  __builtin_amdgcn_raw_buffer_store_b64(u32x2_t{__float_as_uint(x), (uint32_t)id}, list, (int)(in ? to : kOutside), 0, 0);
  to = in ? to + 64 * (uint32_t)sizeof(Entry) : to;
}

// Works a finished tile into the rows' states.  v0: the id of this lane's first element; ids below `from` and from `end` on are
// not counted; target: of the own rows, less than 0: none.  begins: the first tile of its unit.  now: whether the candidates so far
// are sorted in at the end.  place(k, in): where the candidates of own row k go.
template <int QB, bool ROLLED, bool TOP, bool EIGHT, class Load, class Place>
__device__ __forceinline__ void reduce_tile(Load load, Rows<QB>& st, int64_t v0, int64_t from, int64_t end,
                                            const int (&target)[Rows<QB>::kOwn], int row0, Entry* lists, bool begins, bool now,
                                            Place place) {
  constexpr int kOwn = Rows<QB>::kOwn;
  const Arguments p = arguments_again();
  const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4;
  const int n_top = TOP ? p->n_top : 0;
  const bool cut = v0 - 4 * g < from || v0 - 4 * g + kHalf > end;      // (the same in all lanes)
  const int lo = from > v0 ? (int)(from - v0) : 0, hi = end < v0 + kHalf ? (int)(end - v0) : kHalf;
  int wanted[kOwn];        // of the own rows: where the target lies in the half, from its first id on, or -1
  bool some = false;
#pragma unroll
  for (int k = 0; k < kOwn; ++k) {
    const int64_t at = (int64_t)target[k] - (v0 - 4 * g);
    wanted[k] = target[k] >= 0 && at >= 0 && at < kHalf ? (int)at : -1;
    some = some || wanted[k] >= 0;
  }
  enum { kCut = 1, kTarget = 2, kBegins = 4, kAgain = 8 };
  int all_flags = (cut ? kCut : 0) | (__any(some) ? kTarget : 0) | (begins ? kBegins : 0);
  float tile_e[kOwn], tile_s[kOwn], tile_t[kOwn];
  float tau[kOwn];         // of the own rows: what candidates of this tile have to pass
  uint32_t next[kOwn];     // of columns 4 k .., a byte each: the first quad of this lane that is still to be looked at
#pragma unroll
  for (int k = 0; k < kOwn; ++k) { tile_e[k] = kNegExponent; tile_s[k] = tile_t[k] = 0.f; tau[k] = st.tau[k]; next[k] = 0; }
#pragma unroll 1
  for (;;) {
    bool full = false;
    each_column<ROLLED, QB>([&](int j) __attribute__((always_inline)) {
      const int k = j >> 2, at = 8 * (j & 3), owner = 16 * (j & 3) + l16;
      const bool own = g == (j & 3);
      const int flags = opaque(all_flags);
      float pass = 0.f;
      if constexpr (TOP) pass = __shfl(pick(tau, k), owner, 64);
      float x[32];
      load(j, x);
      if (flags & kCut) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) x[4 * i + r] = 16 * i + r >= lo && 16 * i + r < hi ? x[4 * i + r] : kNeg;
      }
      float most[8];       // of quads
#pragma unroll
      for (int i = 0; i < 8; ++i) most[i] = fmaxf(fmaxf(fmaxf(x[4 * i], x[4 * i + 1]), x[4 * i + 2]), x[4 * i + 3]);
      if (!(flags & kAgain)) {
        const float lane_m = fmaxf(fmaxf(fmaxf(fmaxf(most[0], most[1]), most[2]), fmaxf(fmaxf(most[3], most[4]), most[5])), fmaxf(most[6], most[7]));
        const float e = __builtin_ceilf(fmaxf(row_max(lane_m), kNeg) * kLog2e);
        float s[4] = {0.f, 0.f, 0.f, 0.f}, t[4] = {0.f, 0.f, 0.f, 0.f};
        // an exponential at a time, with the next but one's argument and the last one's sums beside it: their unit takes four times as long
        float u[32], z[32];
        u[0] = __builtin_fmaf(x[0], kLog2e, -e);
        u[1] = __builtin_fmaf(x[1], kLog2e, -e);
#pragma unroll
        for (int i = 0; i <= 32; ++i) {
          __builtin_amdgcn_sched_barrier(0);
          if (i < 32) z[i] = __builtin_amdgcn_exp2f(u[i]);
          if (i + 2 < 32) u[i + 2] = __builtin_fmaf(x[i + 2], kLog2e, -e);
          if (i > 0) {
            s[(i - 1) & 3] += z[i - 1];
            t[(i - 1) & 3] = __builtin_fmaf(u[i - 1], z[i - 1], t[(i - 1) & 3]);
          }
        }
        put(tile_e, k, own, e);
        put(tile_s, k, own, row_sum((s[0] + s[1]) + (s[2] + s[3])));
        put(tile_t, k, own, row_sum((t[0] + t[1]) + (t[2] + t[3])));
        if (flags & kTarget) {        // the target's logit, in the one lane that holds it
          const int rel = __shfl(pick(wanted, k), owner, 64) - 4 * g;
          float logit = 0.f;
          bool here = false;
#pragma unroll
          for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const bool it = rel == 16 * i + r;
              logit = it ? x[4 * i + r] : logit;
              here = here || it;
            }
          if (here && rel >= lo && rel < hi) in_memory(p->target_logit)[row0 + 16 * j + l16] = logit;
        }
      }
      if constexpr (TOP) {
        if ((flags & (kBegins | kAgain)) == kBegins) {
          const float bound = below(fmaxf(reached_by(most, n_top), kNeg));
          pass = fmaxf(fmaxf(pass, bound), kNeg);
          put(tau, k, own, pass);
        }
        // Candidates go to this lane's own list of the column.  Where it is full the lane stops at the quad that does not fit, and goes
        // on there once all have been sorted in.
        int done = (int)(pick(next, k) >> at & 255), n = (int)(pick(st.listed, k) >> at & 255);
        bool stopped = false;
        const __amdgpu_buffer_rsrc_t list = list_buffer(lists + j * (kListRoom * 64));
        uint32_t to = (uint32_t)(n * 64 + lane) * (uint32_t)sizeof(Entry);
        constexpr uint32_t kFull = (kListRoom - 4) * 64 * (uint32_t)sizeof(Entry);
        const int id0 = (int)v0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const bool want = (most[i] > pass) & (i >= done) & !stopped;
          if (__any(want)) {
            const bool fits = to < kFull + 64 * (uint32_t)sizeof(Entry);
            stopped = stopped | (want & !fits);
            done = (want & !fits) ? i : done;
            // Most lanes put down one of a quad or none.  With EIGHT waves a compute unit, whose stores take turns, all four of a quad are
            // only gone through where some lane has a second one (900 rows of 32003 x 1032, five alternatives: 236 us, so 187); with
            // four waves telling that takes longer (32000 x 1024: 125 us, so 129).
            const float above = (want & fits) ? pass : __builtin_inff(), *const v = x + 4 * i;
            bool each = true;
            if constexpr (EIGHT) {
              const float second = fmaxf(fminf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), fmaxf(fminf(v[0], v[1]), fminf(v[2], v[3])));
              each = __any(second > above);
            }
            if (each) {
#pragma unroll
              for (int r = 0; r < 4; ++r) append_above(v[r], above, id0 + 16 * i + r, list, to);
            } else {
              const int r = v[0] == most[i] ? 0 : v[1] == most[i] ? 1 : v[2] == most[i] ? 2 : 3;
              append_above(most[i], above, id0 + 16 * i + r, list, to);
            }
          }
        }
        n = (int)(to / (64 * (uint32_t)sizeof(Entry)));
        full = full || stopped;
        put(next, k, true, (pick(next, k) & ~(255u << at)) | (uint32_t)(stopped ? done : 8) << at);
        put(st.listed, k, true, (pick(st.listed, k) & ~(255u << at)) | (uint32_t)n << at);
      }
    });
    bool more = false;
    if constexpr (TOP) {
      more = __any(full);
#pragma unroll
      for (int k = 0; k < kOwn; ++k) st.tau[k] = fmaxf(st.tau[k], tau[k]);   // (what no id of this tile needs to pass none of a later one does)
      if (more || now) sort_all_in(st, lists, n_top, place);
    }
    if (!(all_flags & kAgain)) {
#pragma unroll
      for (int k = 0; k < kOwn; ++k) {
        const float to = fmaxf(st.e[k], tile_e[k]), a = __builtin_amdgcn_exp2f(st.e[k] - to), b = __builtin_amdgcn_exp2f(tile_e[k] - to);
        st.t[k] = a * (st.t[k] + st.s[k] * (st.e[k] - to)) + b * (tile_t[k] + tile_s[k] * (tile_e[k] - to));
        st.s[k] = a * st.s[k] + b * tile_s[k];
        st.e[k] = to;
      }
    }
    if (!more) return;
    all_flags |= kAgain;
#pragma unroll
    for (int k = 0; k < kOwn; ++k) tau[k] = fmaxf(tau[k], below(st.tau[k]));   // an id of this tile may equal the n_top-th best and come before it
  }
}

// Whether the candidates of a unit's `tiles` tiles so far are sorted in now: after 1, 2, 4, 8, ... of them, of a long unit, and at its
// end.
__device__ __forceinline__ bool sort_now(int tiles, int of) { return tiles == of || (of > 2 && (tiles & (tiles - 1)) == 0); }

// The gradient at a finished tile's logits, in 16 bits, as the matrix products behind take it:
//   dl[v] = - p[v] (g + h (log p[v] + H))      g, h: the gradients of the row's log probability and entropy H
// with 0 at the target, whose one-hot term outweighs the others; the target's whole term goes past the 16 bits.  What the rounding
// leaves over is a second number of 16 bits where the sums show it (LOW): for results in 32 bits, and in the sums of few rows.
// v0: the first id of the wave.
template <int QB>
struct GradientRows {   // what a lane holds of its own rows (as Rows)
  static constexpr int kOwn = (QB + 3) / 4;
  float lse[kOwn], g[kOwn], h[kOwn], entropy[kOwn];
  int target[kOwn];

  __device__ __forceinline__ void read(const LogitParams& p, int row0, int found) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
      const int row = row0 + 64 * k + lane;
      const bool listed = 4 * k + (lane >> 4) < QB && row < found;
      lse[k] = listed ? in_memory(p.lse)[row] : 0.f;
      target[k] = listed && p.targets != nullptr ? in_memory(p.targets)[row] : -1;
      g[k] = (uint32_t)target[k] < (uint32_t)p.all_ids ? in_memory(p.dlogprob)[row] : 0.f;
      h[k] = listed && p.dentropy != nullptr ? in_memory(p.dentropy)[row] : 0.f;
      entropy[k] = listed && p.dentropy != nullptr ? in_memory(p.entropy)[row] : 0.f;
    }
  }
};
template <int QB, bool ROLLED, bool LOW, class Load>
__device__ __forceinline__ void gradient_tile(Load load, const GradientRows<QB>& of, int64_t v0, int row0, int found) {
  const Arguments p = arguments_again();
  const int lane = threadIdx.x & 63, l16 = lane & 15, g4 = lane >> 4, run = first_of<4>(lane);
  const int there = p->V - v0 < kHalf ? (int)(p->V - v0) - 4 * g4 : kHalf;   // ids there are from this lane's first on
  each_column<ROLLED, QB>([&](int j) __attribute__((always_inline)) {
    const int owner = 16 * (j & 3) + l16, row = row0 + 16 * j + l16;
    const bool in = row < p->max_rows, listed = row < found;
    const float lse = __shfl(pick(of.lse, j >> 2), owner, 64), g = __shfl(pick(of.g, j >> 2), owner, 64);
    float h = 0.f, entropy = 0.f;
    if (p->dentropy != nullptr) {
      h = __shfl(pick(of.h, j >> 2), owner, 64);
      entropy = __shfl(pick(of.entropy, j >> 2), owner, 64);
    }
    const int target = __shfl(pick(of.target, j >> 2), owner, 64);
    const int64_t from = (int64_t)target - p->first_id - v0;
    const int rel = target >= 0 && from >= 0 && from < kHalf ? (int)from - 4 * g4 : -kHalf;
    float x[32];
    load(j, x);
#pragma unroll
    for (int b = 0; b < 8; b += 4) {
      Quad o[4], low[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float v[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int at = 16 * (b + k) + r;
          const float logp = x[4 * (b + k) + r] - lse;
          const float prob = __builtin_amdgcn_exp2f(logp * kLog2e);
          const float d = -prob * (p->dentropy != nullptr ? g + h * (logp + entropy) : g);
          v[r] = listed && rel != at && at < there ? d : 0.f;
        }
        pack(o[k], v);
        if constexpr (LOW) pack_low(low[k], o[k], v);
      }
      gather(o);
      const int c = (int)(v0 + 16 * b) + run;
      if (in) store_quads(p->dl + row * p->ld_dl, c, p->dl_ids, o);
      if constexpr (LOW) {
        gather(low);
        if (in) store_quads(p->dl + p->low + row * p->ld_dl, c, p->dl_ids, low);
      }
    }
  });
}

// The 4-wave kernels (mosaic_logprob_w4.h): whether they take these sizes, and their launches.
bool w4_takes(int32_t d, int32_t V);
int launch_statistics_w4(const LogitParams& p, hipStream_t stream);
int launch_alternatives_w4(const LogitParams& p, hipStream_t stream);
int launch_gradients_w4(const LogitParams& p, hipStream_t stream);        // without low halves
int launch_gradients_low_w4(const LogitParams& p, hipStream_t stream);    // with them
int64_t w4_list_bytes();

}  // namespace logprob
}  // namespace mosaic
#endif
