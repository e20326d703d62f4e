// Tokens into rows: embedding lookup with scaling, its gradient by sorted tokens, and dropout from a counter-based generator.
// All of it is bound by memory.  Lookup of 32768 rows of 4096 into 32 bits 102 us, 6.6 TB/s of what it reads and writes; the gradient of
// as many rows at a table of 126464 x 4096 in 16 bits 280 us, 4.7 TB/s, of which clearing the table beside the sort is 190.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mosaic_tokens_internal.h"

namespace mosaic {
namespace {

constexpr int kThreads = 256;
constexpr int kStripe = kThreads * 8;   // columns of a block, 8 a lane

__device__ __forceinline__ int64_t rows_of(int64_t T, const int32_t* count) {
  if (count == nullptr) return T;
  const int64_t n = *count;
  return n < 0 ? 0 : n < T ? n : T;
}

// A block's lanes take eight columns of a stripe each: eight side by side or, so that a store of a wave fills whole lines where
// the output has 32 bits, four and four more half a stripe on.
template <typename O>
struct Columns {
  static constexpr bool kSplit = sizeof(O) == 4;
  static constexpr int kSecond = kSplit ? kStripe / 2 : 4;   // from the first four to the others
  static __device__ __forceinline__ int first(int stripe) { return stripe * kStripe + (int)threadIdx.x * (kSplit ? 4 : 8); }
};
__device__ __forceinline__ void load4(const __bf16* p, float* v) {
  const bf16x4_t t = *reinterpret_cast<const bf16x4_t*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = (float)t[i];
}
__device__ __forceinline__ void load4(const float* p, float* v) {
  const f32x4_t t = *reinterpret_cast<const f32x4_t*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = t[i];
}
// The lane's columns of a row; c: the first.  (d is a multiple of 8, so a group of four is there or not.)
template <typename O, typename S>
__device__ __forceinline__ void load_columns(const S* row, int c, int d, float (&v)[8]) {
  if constexpr (Columns<O>::kSplit) {
    if (c < d) load4(row + c, v);
    if (c + Columns<O>::kSecond < d) load4(row + c + Columns<O>::kSecond, v + 4);
  } else {
    if (c < d) load8(row + c, v);
  }
}
// PAST: past the caches; what is written once and is larger than they are only takes the room of what is read.
template <bool PAST>
__device__ __forceinline__ void store_columns(float* row, int c, int d, const float (&v)[8]) {
  const f32x4_t a = {v[0], v[1], v[2], v[3]}, b = {v[4], v[5], v[6], v[7]};
  f32x4_t *const at = reinterpret_cast<f32x4_t*>(row + c), *const then = reinterpret_cast<f32x4_t*>(row + c + Columns<float>::kSecond);
  if constexpr (PAST) {
    if (c < d) __builtin_nontemporal_store(a, at);
    if (c + Columns<float>::kSecond < d) __builtin_nontemporal_store(b, then);
  } else {
    if (c < d) *at = a;
    if (c + Columns<float>::kSecond < d) *then = b;
  }
}
template <bool PAST>
__device__ __forceinline__ void store_columns(__bf16* row, int c, int d, const float (&v)[8]) {
  bf16x8_t t;
#pragma unroll
  for (int i = 0; i < 8; ++i) t[i] = (__bf16)v[i];
  if (c >= d) return;
  if constexpr (PAST) __builtin_nontemporal_store(t, reinterpret_cast<bf16x8_t*>(row + c));
  else *reinterpret_cast<bf16x8_t*>(row + c) = t;
}

// ---- lookup: out[t] = scale * table[tokens[t]], a block ROWS rows of a stripe of columns, all loads under way at once.  37 rows of
// 3584 take 6 us, of which the kernel is 2.5.
template <typename S, typename O, int ROWS, bool PAST>
__global__ __launch_bounds__(kThreads) void embedding_kernel(const EmbedArgs p) {
  const int64_t n = rows_of(p.T, p.count);
  const int c = Columns<O>::first((int)blockIdx.y);
  if (c >= p.d) return;
  for (int64_t t0 = (int64_t)blockIdx.x * ROWS; t0 < n; t0 += (int64_t)gridDim.x * ROWS) {
    int token[ROWS];
    float v[ROWS][8];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) token[r] = t0 + r < n ? p.tokens[t0 + r] : -1;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[r][i] = 0.f;
      if ((uint32_t)token[r] < (uint32_t)p.V) load_columns<O>(static_cast<const S*>(p.table) + (int64_t)token[r] * p.ld_table, c, p.d, v[r]);
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      if (t0 + r >= n) break;
      if ((uint32_t)token[r] < (uint32_t)p.V) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[r][i] *= p.scale;
      }
      store_columns<PAST>(static_cast<O*>(p.out) + (t0 + r) * p.ld_out, c, p.d, v[r]);
    }
  }
}

// ---- positions by token: a stable sort by digits, lowest first.  A block counts the digits of its piece; then every block adds
// up what lies ahead of each of its digits and places its piece, a wave's keys in their order: the rank of a key among the 64
// of a round is the number of lower lanes with the same digit, found by a ballot for each bit (so that a token of half of all
// positions costs no more than others).
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kMostDigitBits = 10, kMostBins = 1 << kMostDigitBits;
constexpr int kMostSortBlocks = 64;
constexpr int kFillRows = 32;              // rows that a block fills
constexpr int64_t kSortPiece = 1024;       // keys of a block, at least (gradient of 12000 rows of 512: 51 us, with 4096 keys 61)
// Up to here one block sorts, in one launch (gradient of 3000 rows of 512: 31 us, in launches of several blocks 36; 6000: 42 and 40;
// 8000: 48 and 41).
constexpr int64_t kOneBlockKeys = 6144;

struct SortArgs {
  const int32_t* tokens;   // first pass: what keys and positions are made from
  const int32_t* count;
  const int32_t *from_keys, *from_at;
  int32_t *to_keys, *to_at;
  int32_t* counts;         // [blocks, kMostBins]
  int64_t n, piece;        // piece: keys of a block, a multiple of kSortThreads
  int32_t V, blocks, shift, bits;
  int32_t first;           // whether this pass is the first
};

__device__ __forceinline__ int32_t key_at(const SortArgs& p, int64_t i, int64_t valid) {
  if (!p.first) return p.from_keys[i];
  const int32_t t = i < valid ? p.tokens[i] : -1;
  return (uint32_t)t < (uint32_t)p.V ? t : p.V;
}

// Part `part` of the memory that is to be filled, by block `block` of `blocks`: what sums go to is cleared while their tokens are
// sorted, which takes a few blocks and little but waiting.
struct FillPart { FillArgs fill; int64_t first, rows; };   // rows from `first` on
__device__ __forceinline__ void fill_rows(const FillPart& p, int64_t block) {
  typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;
  const uint32_t w = p.fill.word;
  const u32x4_t v = {w, w, w, w};
  const int64_t r0 = p.first + block * kFillRows, r1 = r0 + kFillRows < p.first + p.rows ? r0 + kFillRows : p.first + p.rows;
  const int each = (int)(p.fill.row_bytes / 16);
  int64_t r = r0 + (int)threadIdx.x / each;
  int c = (int)threadIdx.x % each;
  const int by_rows = kSortThreads / each, by_cols = kSortThreads % each;
  while (r < r1) {
    __builtin_nontemporal_store(v, reinterpret_cast<u32x4_t*>(static_cast<char*>(p.fill.base) + r * p.fill.ld + (int64_t)c * 16));
    r += by_rows;
    c += by_cols;
    if (c >= each) {
      c -= each;
      ++r;
    }
  }
}

__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(const SortArgs p, const FillPart fill) {
  __shared__ int32_t bins[kMostBins];
  if ((int)blockIdx.x >= p.blocks) {
    fill_rows(fill, blockIdx.x - p.blocks);
    return;
  }
  const int n_bins = 1 << p.bits;
  for (int b = threadIdx.x; b < n_bins; b += kSortThreads) bins[b] = 0;
  __syncthreads();
  const int64_t valid = rows_of(p.n, p.count), from = blockIdx.x * p.piece, end = from + p.piece < p.n ? from + p.piece : p.n;
  for (int64_t i = from + threadIdx.x; i < end; i += kSortThreads)
    atomicAdd(&bins[key_at(p, i, valid) >> p.shift & (n_bins - 1)], 1);
  __syncthreads();
  for (int b = threadIdx.x; b < n_bins; b += kSortThreads) p.counts[(int64_t)blockIdx.x * kMostBins + b] = bins[b];
}

struct SortLds {
  int32_t place[kSortWaves][kMostBins];   // how many keys of a digit a wave has, then where its next one goes
  int32_t wave_sum[kSortWaves];
};

// One pass over block `block`'s piece.  `counts`: nullptr where it is the only block.  A wave takes consecutive keys, 64 a round, and
// holds those of up to kHeld rounds; beyond, it reads them again.
constexpr int kHeld = 8;
__device__ __forceinline__ void sort_piece(const SortArgs& p, SortLds& lds, int block, const int32_t* counts) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n_bins = 1 << p.bits;
  const int64_t valid = rows_of(p.n, p.count);
  const int64_t each = p.piece / kSortWaves, from = block * p.piece + wave * each;
  const int64_t end = from + each < p.n ? from + each : p.n;
  const bool held = each <= 64 * kHeld;
  int32_t key_of[kHeld], at_of[kHeld];
#pragma unroll
  for (int r = 0; r < kHeld; ++r) {
    const int64_t i = from + 64 * r + lane;
    key_of[r] = 0;
    at_of[r] = (int32_t)i;
    if (held && i < end) {
      key_of[r] = key_at(p, i, valid);
      if (!p.first) at_of[r] = p.from_at[i];
    }
  }
  // of a thread's digit (there are no more digits than threads): keys of other blocks that come ahead, and of all
  int ahead = 0, all = 0;
  if (counts != nullptr && tid < n_bins) {
    constexpr int kAtOnce = 16;
    for (int b0 = 0; b0 < p.blocks; b0 += kAtOnce) {
      int c[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) c[i] = b0 + i < p.blocks ? counts[(int64_t)(b0 + i) * kMostBins + tid] : 0;
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        ahead += b0 + i < block ? c[i] : 0;
        all += c[i];
      }
    }
  }
  for (int b = lane; b < n_bins; b += 64) lds.place[wave][b] = 0;
  __builtin_amdgcn_wave_barrier();
  if (held) {
#pragma unroll
    for (int r = 0; r < kHeld; ++r)
      if (from + 64 * r + lane < end) atomicAdd(&lds.place[wave][key_of[r] >> p.shift & (n_bins - 1)], 1);
  } else {
    for (int64_t i = from + lane; i < end; i += 64) atomicAdd(&lds.place[wave][key_at(p, i, valid) >> p.shift & (n_bins - 1)], 1);
  }
  __syncthreads();
  int here[kSortWaves];
  if (tid < n_bins) {
    int sum = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      here[w] = lds.place[w][tid];
      sum += here[w];
    }
    if (counts == nullptr) all = sum;
  }
  int sum = all;   // inclusive, over the wave, then over the block
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) {
    const int o = __shfl_up(sum, x, 64);
    if (lane >= x) sum += o;
  }
  if (lane == 63) lds.wave_sum[wave] = sum;
  __syncthreads();
  if (tid < n_bins) {
    int at = sum - all + ahead;
    for (int w = 0; w < wave; ++w) at += lds.wave_sum[w];
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      lds.place[w][tid] = at;
      at += here[w];
    }
  }
  __syncthreads();
  auto put = [&](bool in, int32_t key, int32_t at) __attribute__((always_inline)) {
    const int digit = key >> p.shift & (n_bins - 1);
    uint64_t same = __ballot(in);
    for (int b = 0; b < p.bits; ++b) {
      const uint64_t set = __ballot((digit >> b & 1) != 0);
      same &= (digit >> b & 1) != 0 ? set : ~set;
    }
    const int rank = __popcll(same & (((uint64_t)1 << lane) - 1));
    int to = 0;
    if (in) to = *(volatile int32_t*)&lds.place[wave][digit];
    __builtin_amdgcn_wave_barrier();   // all lanes have read before one of them moves the place on
    if (in && rank == 0) *(volatile int32_t*)&lds.place[wave][digit] = to + __popcll(same);
    __builtin_amdgcn_wave_barrier();
    if (in) {
      p.to_keys[to + rank] = key;
      p.to_at[to + rank] = at;
    }
  };
  if (held) {
#pragma unroll
    for (int r = 0; r < kHeld; ++r)
      if (from + 64 * r < end) put(from + 64 * r + lane < end, key_of[r], at_of[r]);
  } else {
    for (int64_t i0 = from; i0 < end; i0 += 64) {
      const bool in = i0 + lane < end;
      put(in, in ? key_at(p, i0 + lane, valid) : 0, !in ? 0 : p.first ? (int32_t)(i0 + lane) : p.from_at[i0 + lane]);
    }
  }
}

__global__ __launch_bounds__(kSortThreads) void sort_place_kernel(const SortArgs p, const FillPart fill) {
  __shared__ SortLds lds;
  if ((int)blockIdx.x >= p.blocks) {
    fill_rows(fill, blockIdx.x - p.blocks);
    return;
  }
  sort_piece(p, lds, (int)blockIdx.x, p.counts);
}

// All passes in one block: keys and positions go to and fro between two buffers.
__global__ __launch_bounds__(kSortThreads) void sort_one_block_kernel(SortArgs p, int32_t passes, int32_t* other_keys, int32_t* other_at,
                                                                      const FillPart fill) {
  __shared__ SortLds lds;
  if (blockIdx.x > 0) {
    fill_rows(fill, blockIdx.x - 1);
    return;
  }
  for (int pass = 0; pass < passes; ++pass) {
    p.first = pass == 0;
    sort_piece(p, lds, 0, nullptr);
    __threadfence_block();
    __syncthreads();
    p.shift += p.bits;
    int32_t *const k = p.to_keys, *const a = p.to_at;
    p.to_keys = other_keys;
    p.to_at = other_at;
    other_keys = k;
    other_at = a;
    p.from_keys = k;
    p.from_at = a;
  }
}

struct SortPlan { int32_t passes, bits, blocks; int64_t piece; };
SortPlan plan_sort(int64_t n, int32_t V) {
  const int key_bits = 32 - __builtin_clz((unsigned)V);   // keys 0 .. V
  SortPlan s;
  s.passes = (key_bits + kMostDigitBits - 1) / kMostDigitBits;
  s.bits = (key_bits + s.passes - 1) / s.passes;
  const int64_t least = n <= kOneBlockKeys ? n : kSortPiece, even = (n + kMostSortBlocks - 1) / kMostSortBlocks;
  s.piece = ((least > even ? least : even) + kSortThreads - 1) / kSortThreads * kSortThreads;
  s.blocks = (int32_t)((n + s.piece - 1) / s.piece);
  return s;
}
int64_t padded(int64_t bytes) { return (bytes + 255) / 256 * 256; }

// ---- sums of rows by token.  A block takes each_of(n, d) sorted positions and a stripe of columns: 8 rows under way at once, added in
// order; a token's sum goes out where the token ends.  A token whose positions reach over the end of a block's piece leaves a
// partial sum there (0: it began ahead of the piece, 1: it goes on behind it), joined in order by a second kernel.
//
// Few positions a block keep more blocks busy and a lone row's chain short, many leave fewer partial sums to join: the choice goes by
// what there is for all blocks.  Half of the tokens the same, us with 8, 16, 32 and 64: 3000 rows of 512 28, 31, 41 and 60; 12000 48,
// 45, 55 and 72; 32768 of 1024 84, 75, 72 and 96; 131072 of 512 244, 192, 165 and 158; 32768 of 4096 with 32 and 64 275 and 269.
int64_t stripes_of(int32_t d) { return (d + kStripe - 1) / kStripe; }
int each_of(int64_t n, int32_t d) {
  const int64_t m = n * stripes_of(d);
  return m >= 65536 ? 64 : m >= 32768 ? 32 : m >= 8192 ? 16 : 8;
}
constexpr int kMostEach = 64;

struct SumParams {
  TokenSumArgs a;
  int32_t each, stripes;
  int64_t pieces, blocks;
};
constexpr int64_t kMostBlocks = 1 << 22;   // of a launch; further work is taken in turn

template <typename O>
__device__ __forceinline__ void put_sum(const TokenSumArgs& a, int32_t key, int64_t place, int c, float (&s)[8]) {
  const int64_t row = a.first != nullptr ? place : key;
  O* to = static_cast<O*>(a.sums) + row * a.ld_sums + c;
#pragma unroll
  for (int i = 0; i < 8; ++i) s[i] *= a.scale;
  if constexpr (sizeof(O) == 4) {
    if (a.accumulate) {
      float old[8];
      load8(to, old);
#pragma unroll
      for (int i = 0; i < 8; ++i) s[i] += old[i];
    }
  }
  store8(to, s);
}

// Piece and stripe `block`.
template <typename S, typename O>
__device__ __forceinline__ void sum_piece(const SumParams& p, int64_t block, int32_t* keys, int32_t* ats, float* weights) {
  const TokenSumArgs& a = p.a;
  const int tid = threadIdx.x;
  const int64_t piece = block / p.stripes, e0 = piece * p.each;
  const int c = (int)(block % p.stripes) * kStripe + tid * 8;
  if (tid < p.each + 2) {
    const int64_t e = e0 + tid - 1;
    keys[tid] = e >= 0 && e < a.n ? a.sorted.keys[e] : a.V;
    if (tid >= 1 && tid <= p.each && e < a.n) {
      const int32_t at = a.sorted.at[e];
      ats[tid - 1] = at;
      weights[tid - 1] = a.weights != nullptr ? a.weights[at] : 1.f;
    }
  }
  __syncthreads();
  int end = 0;   // positions of tokens in the piece; V comes last
  while (end < p.each && keys[end + 1] < a.V) ++end;
  const bool in = c < a.d;
  float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  int run = 0;   // where the token's positions begin
  for (int g = 0; g < end; g += 8) {
    float v[8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[i][k] = 0.f;
      if (in && g + i < end) load8(static_cast<const S*>(a.rows) + (int64_t)ats[g + i] * a.ld_rows + c, v[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (g + i < end) {
#pragma unroll
        for (int k = 0; k < 8; ++k) s[k] = __builtin_fmaf(v[i][k], weights[g + i], s[k]);
        const int32_t key = keys[g + i + 1];
        const bool before = run == 0 && keys[0] == key;          // it began ahead of the piece
        const bool behind = g + i + 1 == p.each && keys[p.each + 1] == key;
        if (g + i + 1 == end || keys[g + i + 2] != key) {        // its last position here
          if (in) {
            if (before || behind) store8(a.partials + (2 * piece + (before ? 0 : 1)) * a.d + c, s);
            else put_sum<O>(a, key, e0 + run, c, s);
          }
          if (a.first != nullptr && !before && c == 0) a.first[key] = (int32_t)(e0 + run);
#pragma unroll
          for (int k = 0; k < 8; ++k) s[k] = 0.f;
          run = g + i + 1;
        }
      }
    }
  }
  __syncthreads();   // the arrays are free for the next piece
}

template <typename S, typename O>
__global__ __launch_bounds__(kThreads) void token_sum_kernel(const SumParams p) {
  __shared__ int32_t keys[kMostEach + 2], ats[kMostEach];   // keys: with the ones before and behind the piece
  __shared__ float weights[kMostEach];
  for (int64_t block = blockIdx.x; block < p.blocks; block += gridDim.x) sum_piece<S, O>(p, block, keys, ats, weights);
}

// Joins the partial sums of tokens that reach over pieces: a block looks through pieces (64 at once) for those at whose end a
// token goes on that began in them.  A wave joins a token of few partial sums by itself, the block's waves taking such tokens in
// turn; of one with more than kAlone the waves take a sixteenth each, in order, and the sixteenths are added in order.  A lane has
// four columns.  Bound by the time to memory, which other kernels wrote: the keys of 64 pieces are asked for at once, and a token's
// partial sums eight at a time (1003 rows of 1024: 8 us; with a branch around each load, and registers spilled for it, 35).
constexpr int kJoinWaves = 16, kAlone = 16;

template <typename O>
__device__ __forceinline__ void put_joined(const TokenSumArgs& a, int64_t row, int c, f32x4_t t) {
  t *= a.scale;
  if constexpr (sizeof(O) == 4) {
    f32x4_t* to = reinterpret_cast<f32x4_t*>(static_cast<float*>(a.sums) + row * a.ld_sums + c);
    *to = a.accumulate ? *to + t : t;
  } else {
    *reinterpret_cast<bf16x4_t*>(static_cast<__bf16*>(a.sums) + row * a.ld_sums + c) =
        bf16x4_t{(__bf16)t[0], (__bf16)t[1], (__bf16)t[2], (__bf16)t[3]};
  }
}
// Partial sums m0 .. m1 - 1 of the token that goes on behind piece `from`, added in order, eight under way at once: past the last
// one it is read again and counts nothing, since loads behind a branch each would be waited for one by one.
__device__ __forceinline__ f32x4_t add_partials(const TokenSumArgs& a, int64_t from, int64_t m0, int64_t m1, int c, bool in) {
  f32x4_t s = {0.f, 0.f, 0.f, 0.f};
  const float* base = a.partials + (in ? c : 0);
#pragma unroll 1
  for (int64_t m = m0; m < m1; m += 8) {
    f32x4_t v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t k = m + i < m1 ? m + i : m1 - 1;
      v[i] = *reinterpret_cast<const f32x4_t*>(base + (k == 0 ? 2 * from + 1 : 2 * (from + k)) * a.d);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (m + i < m1) s += v[i];
    }
  }
  return s;
}

template <typename O>
__global__ __launch_bounds__(64 * kJoinWaves) void token_join_kernel(const SumParams p) {
  const TokenSumArgs& a = p.a;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int c = ((int)blockIdx.x * 64 + lane) * 4;
  const bool in = c < a.d;
  __shared__ f32x4_t parts[kJoinWaves][64];
  // How many partial sums the token `key` has that goes on behind piece `from`, the one of lane `at`: its own and those of pieces that
  // begin inside of it, which are the first ones behind.  `key_behind` tells it for the pieces from `at` on; where they all are in
  // the token, the lanes probe 64 further ones at once.
  auto count_partials = [&](int64_t from, int at, int32_t key, int32_t key_behind) __attribute__((always_inline)) {
    const int64_t past = (from + 1) * p.each;
    const uint64_t others = ~(__ballot(key_behind == key) >> at);   // (what comes in from above counts as others)
    const int near = others == 0 ? 64 : __builtin_ctzll(others);     // no bit at all: lane 0 and 64 pieces in one token
    const bool ended = near < 64 - at;
    int64_t more = near, span = ended ? 0 : p.pieces - 1 - from - near;
    while (span > 0) {
      const int64_t step = (span + 63) / 64, probe = more + (lane + 1) * step - 1, e = past + probe * p.each;
      const uint64_t same = __ballot(probe < more + span && e < a.n && a.sorted.keys[e < a.n ? e : 0] == key);
      const int64_t whole = ~same == 0 ? 64 : __builtin_ctzll(~same), rest = span - whole * step;
      more += whole * step;
      span = step - 1 < rest ? step - 1 : rest;
    }
    return more + 1;
  };
  for (int64_t base = (int64_t)blockIdx.y * 64; base < p.pieces; base += (int64_t)gridDim.y * 64) {
    // keys behind the piece, at its end, ahead of it: all asked for at once, since what another kernel wrote is far away
    const int64_t piece = base + lane, next = (piece + 1) * p.each;
    int32_t key_behind = a.V, key_last = a.V, key_ahead = a.V;
    if (next < a.n) {
      key_behind = a.sorted.keys[next];
      key_last = a.sorted.keys[next - 1];
      if (piece > 0) key_ahead = a.sorted.keys[piece * p.each - 1];
    }
    // a token reaches over the end, and the piece does not begin inside of it
    const bool begins = key_behind < a.V && key_last == key_behind && key_ahead != key_behind;
    const uint64_t found = __ballot(begins);
    // A token of more partial sums than kAlone is that of the last piece found in 64, or the next one found lies as far behind.
    int turn = 0;
    for (uint64_t left = found; left != 0; left &= left - 1, ++turn) {
      if (turn % kJoinWaves != wave) continue;
      const int at = __builtin_ctzll(left);
      const int64_t from = base + at;
      const int32_t key = __shfl(key_behind, at, 64);
      const int64_t all = count_partials(from, at, key, key_behind);
      if (all > kAlone) continue;
      const int64_t row = a.first != nullptr ? a.first[key] : key;
      const f32x4_t s = add_partials(a, from, 0, all, c, in);
      if (in) put_joined<O>(a, row, c, s);
    }
    for (uint64_t left = found; left != 0; left &= left - 1) {
      const int at = __builtin_ctzll(left);
      const int64_t from = base + at, behind = (left & (left - 1)) != 0 ? base + __builtin_ctzll(left & (left - 1)) : p.pieces;
      if (behind - from < kAlone) continue;   // it has ended by then
      const int32_t key = __shfl(key_behind, at, 64);
      const int64_t all = count_partials(from, at, key, key_behind);
      if (all <= kAlone) continue;
      const int64_t row = a.first != nullptr ? a.first[key] : key;
      parts[wave][lane] = add_partials(a, from, all * wave / kJoinWaves, all * (wave + 1) / kJoinWaves, c, in);
      __syncthreads();
      if (wave == 0 && in) {
        f32x4_t t = parts[0][lane];
#pragma unroll
        for (int w = 1; w < kJoinWaves; ++w) t += parts[w][lane];
        put_joined<O>(a, row, c, t);
      }
      __syncthreads();
    }
  }
}

__global__ __launch_bounds__(kSortThreads) void fill_kernel(const FillPart p) { fill_rows(p, blockIdx.x); }

// ---- dropout

// Four words of Philox4x32-10: 16 bits for each of 8 columns.
__device__ __forceinline__ void philox(uint32_t (&c)[4], uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int round = 0; round < 10; ++round) {
    const uint64_t a = (uint64_t)0xD2511F53u * c[0], b = (uint64_t)0xCD9E8D57u * c[2];
    const uint32_t n0 = (uint32_t)(b >> 32) ^ c[1] ^ k0, n2 = (uint32_t)(a >> 32) ^ c[3] ^ k1;
    c[0] = n0;
    c[1] = (uint32_t)b;
    c[2] = n2;
    c[3] = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
}

// A block takes a row of a stripe of columns (32768 x 4096 with a 32-bit residual 250 us, 5.4 TB/s, as the largest copies reach;
// two and four rows, loaded at once, 251 and 258, in 16 bits 80 and 83 us where one takes 74).  Ten rounds of the generator for eight
// columns hide behind the memory.
template <typename S, typename O, bool ADD, bool PAST>
__global__ __launch_bounds__(kThreads) void dropout_kernel(const DropoutArgs p) {
  const int c = (int)blockIdx.y * kStripe + (int)threadIdx.x * 8;   // eight columns share the generator's words
  if (c >= p.d) return;
  for (int64_t t = blockIdx.x; t < p.T; t += gridDim.x) {
    float v[8], add[8];
    load8(static_cast<const S*>(p.x) + t * p.ld_x + c, v);
    if constexpr (ADD) load8(static_cast<const O*>(p.residual) + t * p.ld_residual + c, add);
    const uint64_t row = (uint64_t)(p.first_row + t);
    uint32_t w[4] = {(uint32_t)c >> 3, (uint32_t)row, (uint32_t)(row >> 32), p.site};
    philox(w, p.key_low, p.key_high);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t bits = i & 1 ? w[i >> 1] >> 16 : w[i >> 1] & 0xffffu;
      v[i] = bits >= p.border ? v[i] * p.grow : 0.f;
      if constexpr (ADD) v[i] += add[i];
    }
    O* const out = static_cast<O*>(p.out) + t * p.ld_out;
    if constexpr (PAST) store_columns<true>(out, c, p.d, v);   // (a lane's columns side by side: of 16 bits)
    else store8(out + c, v);
  }
}

// A grid of blocks of `rows` rows by stripes of columns.
dim3 row_grid(int64_t T, int rows, int d) {
  const int64_t blocks = (T + rows - 1) / rows;
  return dim3((unsigned)(blocks < kMostBlocks ? blocks : kMostBlocks), (unsigned)((d + kStripe - 1) / kStripe));
}
// A lookup's output from half of the memory-side cache on is written past the caches, which keeps the rows that are read in them (into 32
// bits 32768 x 4096: 146 -> 115 us, 16000 x 4096, 262 MB: 75 -> 57; 16000 x 1024, 66 MB: 16.4 either way, and what comes next
// finds it there); so is a dropout's of 16 bits, which reads as much as it writes, each once.
constexpr int64_t kPastBytes = (int64_t)128 << 20;
constexpr int kPastRows = 2;   // rows of a block then: one 155 us, two 114, four 115; below, one takes what two and four do

template <typename S, typename O>
int launch_embedding(const EmbedArgs& a, hipStream_t stream) {
  if (a.T * a.d * (int64_t)sizeof(O) >= kPastBytes)
    return launch_kernel(embedding_kernel<S, O, kPastRows, true>, row_grid(a.T, kPastRows, a.d), dim3(kThreads), stream, a);
  return launch_kernel(embedding_kernel<S, O, 1, false>, row_grid(a.T, 1, a.d), dim3(kThreads), stream, a);
}

template <typename S, typename O, bool ADD>
int launch_dropout_as(const DropoutArgs& a, hipStream_t stream) {
  if constexpr (sizeof(O) == 2) {
    if (a.T * a.d * (int64_t)sizeof(O) >= kPastBytes)
      return launch_kernel(dropout_kernel<S, O, ADD, true>, row_grid(a.T, 1, a.d), dim3(kThreads), stream, a);
  }
  return launch_kernel(dropout_kernel<S, O, ADD, false>, row_grid(a.T, 1, a.d), dim3(kThreads), stream, a);
}

template <typename S, typename O>
int launch_sums(const SumParams& p, hipStream_t stream) {
  const TokenSumArgs& a = p.a;
  if (p.blocks > 0 && launch_kernel(token_sum_kernel<S, O>, dim3((unsigned)(p.blocks < kMostBlocks ? p.blocks : kMostBlocks)),
                                    dim3(kThreads), stream, p) != 0)
    return -1;
  if (p.pieces <= 1) return 0;
  const int64_t groups = (p.pieces + 63) / 64;
  return launch_kernel(token_join_kernel<O>, dim3((unsigned)((a.d + 255) / 256), (unsigned)(groups < 64 ? groups : 64)),
                       dim3(64 * kJoinWaves), stream, p);
}

}  // namespace

int launch_embedding_forward(const EmbedArgs& a, bool table_f32, bool out_f32, hipStream_t stream) {
  if (table_f32) return out_f32 ? launch_embedding<float, float>(a, stream) : launch_embedding<float, __bf16>(a, stream);
  return out_f32 ? launch_embedding<__bf16, float>(a, stream) : launch_embedding<__bf16, __bf16>(a, stream);
}

// Two buffers of keys and positions, the digits' counts.
int64_t sort_tokens_bytes(int64_t n) { return 4 * padded(4 * n) + padded((int64_t)kMostBins * kMostSortBlocks * 4); }

namespace {
constexpr int64_t kMostFillBlocks = 1 << 20;   // of a launch (rows past them: a block fills more)
// Part l of `of` of what is to be filled, and the blocks it takes.
FillPart fill_part(const FillArgs& f, int l, int of, int64_t* blocks) {
  const int64_t tiles = (f.rows + kFillRows - 1) / kFillRows, from = tiles * l / of, to = tiles * (l + 1) / of;
  FillPart p = {f, from * kFillRows, 0};
  p.rows = (to * kFillRows < f.rows ? to * kFillRows : f.rows) - p.first;
  if (p.rows < 0) p.rows = 0;
  *blocks = (p.rows + kFillRows - 1) / kFillRows;
  return p;
}
}  // namespace

int launch_fill(const FillArgs& f, hipStream_t stream) {
  const int of = (int)((f.rows + kFillRows * kMostFillBlocks - 1) / (kFillRows * kMostFillBlocks));
  for (int l = 0; l < of; ++l) {
    int64_t blocks;
    const FillPart p = fill_part(f, l, of, &blocks);
    if (blocks > 0 && launch_kernel(fill_kernel, dim3((unsigned)blocks), dim3(kSortThreads), stream, p) != 0) return -1;
  }
  return 0;
}

int launch_sort_tokens(const int32_t* tokens, int64_t n, const int32_t* count, int32_t V, void* space, const FillArgs& fill, SortedTokens* out,
                       hipStream_t stream) {
  const SortPlan plan = plan_sort(n, V);
  char* at = static_cast<char*>(space);
  int32_t* keys[2];
  int32_t* ats[2];
  for (int i = 0; i < 2; ++i) {
    keys[i] = reinterpret_cast<int32_t*>(at);
    ats[i] = reinterpret_cast<int32_t*>(at + padded(4 * n));
    at += 2 * padded(4 * n);
  }
  SortArgs a = {};
  a.tokens = tokens;
  a.count = count;
  a.counts = reinterpret_cast<int32_t*>(at);
  a.n = n;
  a.piece = plan.piece;
  a.V = V;
  a.blocks = plan.blocks;
  a.bits = plan.bits;
  const int last = (plan.passes - 1) & 1;
  *out = SortedTokens{keys[last], ats[last]};
  a.to_keys = keys[0];
  a.to_at = ats[0];
  const int launches = plan.blocks == 1 ? 1 : 2 * plan.passes;
  FillArgs f = fill;
  if (f.rows > kFillRows * kMostFillBlocks) {   // more than these launches have blocks for
    if (launch_fill(f, stream) != 0) return -1;
    f.rows = 0;
  }
  int64_t blocks;
  if (plan.blocks == 1) {
    const FillPart part = fill_part(f, 0, 1, &blocks);
    return launch_kernel(sort_one_block_kernel, dim3((unsigned)(1 + blocks)), dim3(kSortThreads), stream, a, plan.passes, keys[1], ats[1], part);
  }
  for (int pass = 0; pass < plan.passes; ++pass) {
    a.first = pass == 0;
    a.shift = pass * plan.bits;
    a.from_keys = keys[(pass + 1) & 1];
    a.from_at = ats[(pass + 1) & 1];
    a.to_keys = keys[pass & 1];
    a.to_at = ats[pass & 1];
    FillPart part = fill_part(f, 2 * pass, launches, &blocks);
    if (launch_kernel(sort_count_kernel, dim3((unsigned)(plan.blocks + blocks)), dim3(kSortThreads), stream, a, part) != 0) return -1;
    part = fill_part(f, 2 * pass + 1, launches, &blocks);
    if (launch_kernel(sort_place_kernel, dim3((unsigned)(plan.blocks + blocks)), dim3(kSortThreads), stream, a, part) != 0) return -1;
  }
  return 0;
}

// Room for up to n positions: fewer of them can have more pieces where each_of() steps up.
int64_t token_sum_partials(int64_t n, int32_t d) {
  int64_t most = (n + each_of(n, d) - 1) / each_of(n, d);
  for (const int64_t step : {8192, 32768, 65536}) {
    const int64_t first = (step + stripes_of(d) - 1) / stripes_of(d), below = (first + each_of(first - 1, d) - 2) / each_of(first - 1, d);
    if (n >= first && most < below) most = below;
  }
  return 2 * most;
}

int launch_token_sums(const TokenSumArgs& a, bool rows_f32, bool sums_f32, hipStream_t stream) {
  SumParams p = {};
  p.a = a;
  p.each = each_of(a.n, a.d);
  p.stripes = (int32_t)stripes_of(a.d);
  p.pieces = (a.n + p.each - 1) / p.each;
  p.blocks = p.pieces * p.stripes;
  if (rows_f32) return sums_f32 ? launch_sums<float, float>(p, stream) : launch_sums<float, __bf16>(p, stream);
  return sums_f32 ? launch_sums<__bf16, float>(p, stream) : launch_sums<__bf16, __bf16>(p, stream);
}

int launch_dropout(const DropoutArgs& a, bool x_f32, bool out_f32, hipStream_t stream) {
  const bool add = a.residual != nullptr;
  if (x_f32) return launch_dropout_as<float, __bf16, false>(a, stream);   // the backward pass
  if (out_f32) return add ? launch_dropout_as<__bf16, float, true>(a, stream) : launch_dropout_as<__bf16, float, false>(a, stream);
  return add ? launch_dropout_as<__bf16, __bf16, true>(a, stream) : launch_dropout_as<__bf16, __bf16, false>(a, stream);
}

}  // namespace mosaic
