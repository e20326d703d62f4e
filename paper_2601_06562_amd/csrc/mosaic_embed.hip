// Tokens into rows: embedding lookup with scaling, its gradient by sorted tokens, and dropout from a counter-based generator.
// All of it is bound by memory.
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

// ---- lookup: out[t] = scale * table[tokens[t]], a block ROWS rows of a stripe of columns, all loads under way at once.
template <typename S, typename O, int ROWS>
__global__ __launch_bounds__(kThreads) void embedding_kernel(const EmbedArgs p) {
  const int64_t n = rows_of(p.T, p.count);
  const int c = (int)blockIdx.y * kStripe + (int)threadIdx.x * 8;
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
      if ((uint32_t)token[r] < (uint32_t)p.V) load8(static_cast<const S*>(p.table) + (int64_t)token[r] * p.ld_table + c, v[r]);
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      if (t0 + r >= n) break;
      if ((uint32_t)token[r] < (uint32_t)p.V) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[r][i] *= p.scale;
      }
      store8(static_cast<O*>(p.out) + (t0 + r) * p.ld_out + c, v[r]);
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
constexpr int64_t kSortPiece = 4096;       // keys of a block, at least
constexpr int64_t kOneBlockKeys = 8192;    // up to here one block sorts, in one launch

struct SortArgs {
  const int32_t* tokens;   // first pass: what keys and positions are made from
  const int32_t* count;
  const int32_t *from_keys, *from_at;
  int32_t *to_keys, *to_at;
  int32_t* counts;         // [bins, blocks]
  uint32_t* present;
  int64_t n, piece;        // piece: keys of a block, a multiple of kSortThreads
  int32_t V, blocks, shift, bits;
  int32_t first, last;     // whether this pass is the first, the last
};

__device__ __forceinline__ int32_t key_at(const SortArgs& p, int64_t i, int64_t valid) {
  if (!p.first) return p.from_keys[i];
  const int32_t t = i < valid ? p.tokens[i] : -1;
  return (uint32_t)t < (uint32_t)p.V ? t : p.V;
}

__device__ __forceinline__ void clear_present(const SortArgs& p, int64_t first, int64_t stride) {
  for (int64_t i = first; i < (p.V + 31) / 32; i += stride) p.present[i] = 0;
}

__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(const SortArgs p) {
  __shared__ int32_t bins[kMostBins];
  const int n_bins = 1 << p.bits;
  if (p.first) clear_present(p, (int64_t)blockIdx.x * kSortThreads + threadIdx.x, (int64_t)gridDim.x * kSortThreads);
  for (int b = threadIdx.x; b < n_bins; b += kSortThreads) bins[b] = 0;
  __syncthreads();
  const int64_t valid = rows_of(p.n, p.count), from = blockIdx.x * p.piece, end = from + p.piece < p.n ? from + p.piece : p.n;
  for (int64_t i = from + threadIdx.x; i < end; i += kSortThreads)
    atomicAdd(&bins[key_at(p, i, valid) >> p.shift & (n_bins - 1)], 1);
  __syncthreads();
  for (int b = threadIdx.x; b < n_bins; b += kSortThreads) p.counts[(int64_t)b * p.blocks + blockIdx.x] = bins[b];
}

struct SortLds {
  int32_t place[kSortWaves][kMostBins];   // how many keys of a digit a wave has, then where its next one goes
  int32_t wave_sum[kSortWaves];
};

// One pass over block `block`'s piece.  `counts`: nullptr where it is the only block.
__device__ __forceinline__ void sort_piece(const SortArgs& p, SortLds& lds, int block, const int32_t* counts) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n_bins = 1 << p.bits;
  const int64_t valid = rows_of(p.n, p.count);
  // a wave takes consecutive keys, 64 a round
  const int64_t each = p.piece / kSortWaves, from = block * p.piece + wave * each;
  const int64_t end = from + each < p.n ? from + each : p.n;
  for (int i = tid; i < kSortWaves * kMostBins; i += kSortThreads) (&lds.place[0][0])[i] = 0;
  __syncthreads();
  for (int64_t i = from + lane; i < end; i += 64) atomicAdd(&lds.place[wave][key_at(p, i, valid) >> p.shift & (n_bins - 1)], 1);
  __syncthreads();
  // a thread a digit (there are no more digits than threads)
  int here = 0, ahead = 0, all = 0;
  if (tid < n_bins) {
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) here += lds.place[w][tid];
    if (counts == nullptr) {
      all = here;
    } else {
      for (int b = 0; b < p.blocks; ++b) {
        const int c = counts[(int64_t)tid * p.blocks + b];
        ahead += b < block ? c : 0;
        all += c;
      }
    }
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
      const int c = lds.place[w][tid];
      lds.place[w][tid] = at;
      at += c;
    }
  }
  __syncthreads();
  for (int64_t i0 = from; i0 < end; i0 += 64) {
    const int64_t i = i0 + lane;
    const bool in = i < end;
    const int32_t key = in ? key_at(p, i, valid) : 0;
    const int32_t at = in ? (p.first ? (int32_t)i : p.from_at[i]) : 0;
    const int32_t left = __shfl_up(key, 1, 64);
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
      // (positions of one token mostly lie side by side by then, and one of them says so)
      if (p.last && key < p.V && (lane == 0 || key != left)) atomicOr(&p.present[key >> 5], 1u << (key & 31));
    }
  }
}

__global__ __launch_bounds__(kSortThreads) void sort_place_kernel(const SortArgs p) {
  __shared__ SortLds lds;
  sort_piece(p, lds, (int)blockIdx.x, p.counts);
}

// All passes in one block: keys and positions go to and fro between two buffers.
__global__ __launch_bounds__(kSortThreads) void sort_one_block_kernel(SortArgs p, int32_t passes, int32_t* other_keys, int32_t* other_at) {
  __shared__ SortLds lds;
  clear_present(p, threadIdx.x, kSortThreads);
  for (int pass = 0; pass < passes; ++pass) {
    p.first = pass == 0;
    p.last = pass == passes - 1;
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

// ---- sums of rows by token.  A block takes kEach(n) sorted positions and a stripe of columns: 8 rows under way at once, added in
// order; a token's sum goes out where the token ends.  A token whose positions reach over the end of a block's piece leaves a
// partial sum there (0: it began ahead of the piece, 1: it goes on behind it), joined in order by a second kernel.  Blocks past
// those of the sums clear the rows that no token names.
__host__ __device__ inline int each_of(int64_t n) { return n >= 32768 ? 64 : n >= 8192 ? 32 : n >= 2048 ? 16 : 8; }
constexpr int kMostEach = 64;
constexpr int kClearRows = 32;

struct SumParams {
  TokenSumArgs a;
  int32_t each, stripes;
  int64_t pieces, sum_blocks, blocks;   // blocks: those that sum, then those that clear
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

// What one block does: piece and stripe `block`, or, past those, rows to clear.
template <typename S, typename O>
__device__ __forceinline__ void sum_or_clear(const SumParams& p, int64_t block, int32_t* keys, int32_t* ats, float* weights) {
  const TokenSumArgs& a = p.a;
  const int tid = threadIdx.x;
  if (block >= p.sum_blocks) {
    const int64_t r0 = (block - p.sum_blocks) * kClearRows;
    const float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    static_assert(kClearRows == 32, "a word of bits");
    const uint32_t present = a.sorted.present == nullptr ? 0u : a.sorted.present[r0 / 32];
    for (int r = 0; r < kClearRows && r0 + r < a.V; ++r) {
      if (present >> r & 1) continue;
      for (int c = tid * 8; c < a.d; c += kStripe) store8(static_cast<O*>(a.sums) + (r0 + r) * a.ld_sums + c, zero);
    }
    return;
  }
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
  for (int64_t block = blockIdx.x; block < p.blocks; block += gridDim.x) sum_or_clear<S, O>(p, block, keys, ats, weights);
}

// Joins the partial sums of tokens that reach over pieces: a block looks through pieces (64 at once) for those at whose end a
// token goes on that began in them; its 16 waves take a sixteenth of the token's partial sums each, in order, and the
// sixteenths are added in order.  A lane has four columns.
constexpr int kJoinWaves = 16;
template <typename O>
__global__ __launch_bounds__(64 * kJoinWaves) void token_join_kernel(const SumParams p) {
  const TokenSumArgs& a = p.a;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c = ((int)blockIdx.x * 64 + lane) * 4;
  const bool in = c < a.d;
  __shared__ f32x4_t parts[kJoinWaves][64];
  for (int64_t base = (int64_t)blockIdx.y * 64; base < p.pieces; base += (int64_t)gridDim.y * 64) {
    const int64_t piece = base + lane, next = (piece + 1) * p.each;
    bool begins = false;
    if (next < a.n) {
      const int32_t key = a.sorted.keys[next];
      // it reaches over the end, and the piece does not begin inside of it
      begins = key < a.V && a.sorted.keys[next - 1] == key && (piece == 0 || a.sorted.keys[piece * p.each - 1] != key);
    }
    for (uint64_t left = __ballot(begins); left != 0; left &= left - 1) {
      const int64_t from = base + __builtin_ctzll(left), past = (from + 1) * p.each;   // past: the first position behind the piece
      const int32_t key = a.sorted.keys[past];
      int64_t more = 0;   // pieces behind it that begin inside of the token
      for (;;) {
        const int64_t at = past + (more + lane) * p.each;
        const uint64_t same = __ballot(at < a.n && a.sorted.keys[at < a.n ? at : 0] == key);
        more += ~same == 0 ? 64 : __builtin_ctzll(~same);
        if (~same != 0) break;
      }
      const int64_t all = more + 1, m0 = all * wave / kJoinWaves, m1 = all * (wave + 1) / kJoinWaves;
      f32x4_t s = {0.f, 0.f, 0.f, 0.f};
      for (int64_t m = m0; m < m1; m += 8) {
        f32x4_t v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          v[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
          const int64_t slot = m + i == 0 ? 2 * from + 1 : 2 * (from + m + i);
          if (in && m + i < m1) v[i] = *reinterpret_cast<const f32x4_t*>(a.partials + slot * a.d + c);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) s += v[i];
      }
      parts[wave][lane] = s;
      __syncthreads();
      if (wave == 0 && in) {
        f32x4_t t = parts[0][lane];
#pragma unroll
        for (int w = 1; w < kJoinWaves; ++w) t += parts[w][lane];
        t *= a.scale;
        int64_t row = key;
        if (a.first != nullptr) row = a.first[key];
        if constexpr (sizeof(O) == 4) {
          f32x4_t* to = reinterpret_cast<f32x4_t*>(static_cast<float*>(a.sums) + row * a.ld_sums + c);
          *to = a.accumulate ? *to + t : t;
        } else {
          *reinterpret_cast<bf16x4_t*>(static_cast<__bf16*>(a.sums) + row * a.ld_sums + c) =
              bf16x4_t{(__bf16)t[0], (__bf16)t[1], (__bf16)t[2], (__bf16)t[3]};
        }
      }
      __syncthreads();
    }
  }
}

__global__ __launch_bounds__(kThreads) void fill_none_kernel(int32_t* first, int32_t V) {
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < V; i += (int64_t)gridDim.x * kThreads) first[i] = -1;
}

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

template <typename S, typename O, bool ADD, int ROWS>
__global__ __launch_bounds__(kThreads) void dropout_kernel(const DropoutArgs p) {
  const int c = (int)blockIdx.y * kStripe + (int)threadIdx.x * 8;
  if (c >= p.d) return;
  for (int64_t t0 = (int64_t)blockIdx.x * ROWS; t0 < p.T; t0 += (int64_t)gridDim.x * ROWS) {
    float v[ROWS][8], add[ADD ? ROWS : 1][8];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      if (t0 + r < p.T) {
        load8(static_cast<const S*>(p.x) + (t0 + r) * p.ld_x + c, v[r]);
        if constexpr (ADD) load8(static_cast<const O*>(p.residual) + (t0 + r) * p.ld_residual + c, add[r]);
      }
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      if (t0 + r >= p.T) break;
      const uint64_t row = (uint64_t)(p.first_row + t0 + r);
      uint32_t w[4] = {(uint32_t)c >> 3, (uint32_t)row, (uint32_t)(row >> 32), p.site};
      philox(w, p.key_low, p.key_high);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t bits = i & 1 ? w[i >> 1] >> 16 : w[i >> 1] & 0xffffu;
        v[r][i] = bits >= p.border ? v[r][i] * p.grow : 0.f;
        if constexpr (ADD) v[r][i] += add[r][i];
      }
      store8(static_cast<O*>(p.out) + (t0 + r) * p.ld_out + c, v[r]);
    }
  }
}

// A grid of blocks of `rows` rows by stripes of columns.
dim3 row_grid(int64_t T, int rows, int d) {
  const int64_t blocks = (T + rows - 1) / rows;
  return dim3((unsigned)(blocks < kMostBlocks ? blocks : kMostBlocks), (unsigned)((d + kStripe - 1) / kStripe));
}
// Rows of a block: several once there are blocks enough.
bool many_rows(int64_t T, int32_t d) { return T * ((d + kStripe - 1) / kStripe) >= 8192; }
constexpr int kManyRows = 4;

template <typename S, typename O>
int launch_embedding(const EmbedArgs& a, hipStream_t stream) {
  if (many_rows(a.T, a.d)) return launch_kernel(embedding_kernel<S, O, kManyRows>, row_grid(a.T, kManyRows, a.d), dim3(kThreads), stream, a);
  return launch_kernel(embedding_kernel<S, O, 1>, row_grid(a.T, 1, a.d), dim3(kThreads), stream, a);
}

template <typename S, typename O, bool ADD>
int launch_dropout_as(const DropoutArgs& a, hipStream_t stream) {
  if (many_rows(a.T, a.d)) return launch_kernel(dropout_kernel<S, O, ADD, kManyRows>, row_grid(a.T, kManyRows, a.d), dim3(kThreads), stream, a);
  return launch_kernel(dropout_kernel<S, O, ADD, 1>, row_grid(a.T, 1, a.d), dim3(kThreads), stream, a);
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

// Two buffers of keys and positions, the digits' counts, the bits of what is present.
int64_t sort_tokens_bytes(int64_t n, int32_t V) {
  return 4 * padded(4 * n) + padded((int64_t)kMostBins * kMostSortBlocks * 4) + padded(((int64_t)V + 31) / 32 * 4);
}

int launch_sort_tokens(const int32_t* tokens, int64_t n, const int32_t* count, int32_t V, void* space, SortedTokens* out,
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
  a.present = reinterpret_cast<uint32_t*>(at + padded((int64_t)kMostBins * kMostSortBlocks * 4));
  a.n = n;
  a.piece = plan.piece;
  a.V = V;
  a.blocks = plan.blocks;
  a.bits = plan.bits;
  const int last = (plan.passes - 1) & 1;
  *out = SortedTokens{keys[last], ats[last], a.present};
  a.to_keys = keys[0];
  a.to_at = ats[0];
  if (plan.blocks == 1)
    return launch_kernel(sort_one_block_kernel, dim3(1), dim3(kSortThreads), stream, a, plan.passes, keys[1], ats[1]);
  for (int pass = 0; pass < plan.passes; ++pass) {
    a.first = pass == 0;
    a.last = pass == plan.passes - 1;
    a.shift = pass * plan.bits;
    a.from_keys = keys[(pass + 1) & 1];
    a.from_at = ats[(pass + 1) & 1];
    a.to_keys = keys[pass & 1];
    a.to_at = ats[pass & 1];
    if (launch_kernel(sort_count_kernel, dim3((unsigned)plan.blocks), dim3(kSortThreads), stream, a) != 0 ||
        launch_kernel(sort_place_kernel, dim3((unsigned)plan.blocks), dim3(kSortThreads), stream, a) != 0)
      return -1;
  }
  return 0;
}

int64_t token_sum_partials(int64_t n) { return 2 * ((n + each_of(n) - 1) / each_of(n)); }

int launch_token_sums(const TokenSumArgs& a, bool rows_f32, bool sums_f32, hipStream_t stream) {
  SumParams p = {};
  p.a = a;
  p.each = each_of(a.n);
  p.stripes = (a.d + kStripe - 1) / kStripe;
  p.pieces = (a.n + p.each - 1) / p.each;
  p.sum_blocks = p.pieces * p.stripes;
  if (a.first != nullptr &&
      launch_kernel(fill_none_kernel, dim3((unsigned)((a.V + kThreads - 1) / kThreads < 1024 ? (a.V + kThreads - 1) / kThreads : 1024)),
                    dim3(kThreads), stream, a.first, a.V) != 0)
    return -1;
  p.blocks = p.sum_blocks + (a.accumulate || a.first != nullptr ? 0 : ((int64_t)a.V + kClearRows - 1) / kClearRows);
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
