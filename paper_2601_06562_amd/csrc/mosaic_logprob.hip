// Log probabilities of given tokens at listed rows, with entropy and the most probable alternatives, and their gradients: the
// logits of a tile are made on the matrix cores, worked on in the accumulators, and never written.
//
// The kernels here take any sizes; where the hand-scheduled K-loop takes them too (mosaic_logprob_w4.h) that one runs.  A tile is 256
// vocabulary ids ("P", the weights' rows) by 64, 128 or 256 listed rows ("Q", gathered as they are copied), K in
// steps of 64 through rings of slots in LDS.  A unit is a tile of rows and a part of the vocabulary, whose tiles a block takes one
// after another; the state of a row is held between them.  32003 x 1032: 900 rows 83 us, 3000 rows 200 (0.99 PFLOP/s), where the
// hand-scheduled loop takes 64 and 164 for 32000 x 1024; five alternatives 187 and 551, there 117 and 276.
#include <hip/hip_runtime.h>
#include <limits.h>
#include <stdint.h>

#include "mosaic_logprob_rows.h"

namespace mosaic {
namespace {

using namespace logprob;

constexpr int kMostSplits = 256;       // parts of the vocabulary
constexpr int kMostUnits = 512;        // units, where there is more than one part

// Rows of a tile for so many rows, by what a step of 64 k takes: 256 rows 1.50 us, 128 rows 0.92.
__host__ __device__ inline int tile_rows(int64_t rows) {
  if (rows <= 64) return 64;
  if (rows <= 128) return 128;
  return 92 * ((rows + 127) / 128) < 150 * ((rows + 255) / 256) ? 128 : 256;
}

// With alternatives a tile has 128 rows at most: beside the accumulators of 256 their state does not fit into registers (32003 x 1032,
// five alternatives, a store for every id: 900 rows 382 us, of 128 rows 233; 3000 rows 1102 and 671).
constexpr int kListedTile = 128;

// Into how many parts the vocabulary's tiles go: the least time of the longest block, a unit costing about two tiles' steps of
// 64 k more than its tiles.  One lane tries every 64th count.
__device__ __forceinline__ int choose_parts(int row_tiles, int vocab_tiles, int steps) {
  const int lane = threadIdx.x & 63;
  uint32_t best = 0xffffffffu;
  for (int s = lane + 1; s <= kMostSplits; s += 64) {
    if (s > vocab_tiles || (s > 1 && row_tiles * s > kMostUnits)) break;
    const uint32_t rounds = (uint32_t)(row_tiles * s + kCus - 1) / kCus, longest = (uint32_t)(vocab_tiles + s - 1) / s;
    const uint64_t cost = (uint64_t)rounds * ((uint64_t)longest * steps + 2);
    const uint32_t c = (uint32_t)(cost < 0x7fffff ? cost : 0x7fffff) << 9 | s;   // equal costs: the fewest parts
    best = c < best ? c : best;
  }
#pragma unroll
  for (int x = 32; x >= 1; x >>= 1) {
    const uint32_t o = (uint32_t)__shfl_xor((int)best, x, 64);
    best = o < best ? o : best;
  }
  return __builtin_amdgcn_readfirstlane((int)(best & 511));
}

// Copies of rows along K: 8 rows of 128 bytes a copy and wave, pieces at piece ^ (row / 2 % 8).
template <int N>
struct RowCopier {
  uint32_t offset[N];
  uint32_t past;   // bit i: this lane's piece of copy i lies past the end of K in the last step, where K is no multiple of 64

  static __device__ __forceinline__ int row_of(int wave, int lane, int i) { return (wave * N + i) * 8 + (lane >> 3); }
  // Row `row` of the tile lies `bytes` from the base, or nowhere.
  __device__ __forceinline__ void place(int i, int lane, int row, bool there, uint32_t bytes, int tail) {
    const int k = ((lane & 7) ^ (row >> 1 & 7)) * 8;
    offset[i] = there ? bytes + k * 2 : kOutside;
    past = (past & ~(1u << i)) | (there && tail != 0 && k >= tail ? 1u : 0u) << i;
  }
  __device__ __forceinline__ void flip() {   // into the last step, or out of it
#pragma unroll
    for (int i = 0; i < N; ++i) offset[i] ^= (past >> i & 1) << 31;
  }
  __device__ __forceinline__ void one(int i, u32x4_t r, uint32_t to, int wave) const {
    const uint32_t m0 = __builtin_amdgcn_readfirstlane((int)(to + (wave * N + i) * 1024));
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(m0), "v"(offset[i]), "s"(r));
  }
};

// All units of this block, in tiles of TQ rows.
template <int MODE, int TQ, int SP, int SQ>
__device__ __forceinline__ void run_units(const LogitParams& p, char* smem, int rows, int found) {
  constexpr int QB = TQ / 64, kBytesP = kVocab * kTileK * 2, kBytesQ = TQ * kTileK * 2;
  constexpr int kCopiesP = 4, kCopiesQ = QB, kBlocksP = 8;
  constexpr bool kSplit = SP != SQ;
  static_assert(!kSplit || SP == SQ + 1, "the waits of the loop");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int wp = wave >> 2, wq = wave & 3;
  const int steps = (p.d + kTileK - 1) / kTileK, tail = p.d % kTileK;
  const int row_tiles = (rows + TQ - 1) / TQ, vocab_tiles = (int)(((int64_t)p.V + kVocab - 1) / kVocab);
  const int parts = choose_parts(row_tiles, vocab_tiles, steps);

  // Block b runs on XCD b % 8; every XCD gets a run of units, and within it panels of row tiles, so that what is in flight
  // behind one L2 shares weights and rows.
  const int n = row_tiles * parts, blocks = (int)gridDim.x, xcd = (int)blockIdx.x % kXcds;
  const int stride = blocks / kXcds + (xcd < blocks % kXcds ? 1 : 0);
  int unit = xcd * (n / kXcds) + (xcd < n % kXcds ? xcd : n % kXcds);
  const int end = unit + n / kXcds + (xcd < n % kXcds ? 1 : 0);
  unit += (int)blockIdx.x / kXcds;
  if (unit >= end) return;
  const int panel = row_tiles < 8 ? row_tiles : 8;

  Entry* const lists = p.lists == nullptr ? nullptr : p.lists + ((int64_t)blockIdx.x * 8 + wave) * (64 * QB) * kListRoom;

  // Of the tile whose copies are issued.
  int part = 0, row0 = 0, vt = 0, vt_begin = 0, vt_end = 0, turned = 0;
  RowCopier<kCopiesP> cp;
  RowCopier<kCopiesQ> cq;
  cp.past = cq.past = 0;
  const char* q_base = p.x;
  // Where an operand's copies come from: K goes round from step `turned` on; steps past the last bring zeros.
  struct Walk { u32x4_t from; int k, left; };
  Walk wp_, wq_;
  auto start_unit = [&]() __attribute__((always_inline)) {
    const int per_panel = panel * parts, pn = unit / per_panel, in = unit - pn * per_panel;
    const int deep = row_tiles - pn * panel < panel ? row_tiles - pn * panel : panel;
    part = in / deep;
    row0 = (pn * panel + in % deep) * TQ;
    vt = vt_begin = (int)((int64_t)vocab_tiles * part / parts);
    vt_end = (int)((int64_t)vocab_tiles * (part + 1) / parts);
    if (p.idx == nullptr) q_base = p.x + (int64_t)row0 * p.ld_x;
#pragma unroll
    for (int i = 0; i < kCopiesQ; ++i) {
      const int row = RowCopier<kCopiesQ>::row_of(wave, lane, i);
      const bool there = row0 + row < rows;
      uint32_t bytes = (uint32_t)row * (uint32_t)p.ld_x;
      if (p.idx != nullptr && there) {
        int t = p.idx[row0 + row];
        t = t < 0 ? 0 : (t > p.T - 1 ? p.T - 1 : t);   // a bad entry of a caller's list reads a valid row
        bytes = (uint32_t)t * (uint32_t)p.ld_x;
      }
      cq.place(i, lane, row, there, bytes, tail);
    }
  };
  const char* p_base = p.w;
  auto start_tile = [&]() __attribute__((always_inline)) {
    const int64_t v = (int64_t)vt * kVocab;
    p_base = p.w + v * p.ld_w;
#pragma unroll
    for (int i = 0; i < kCopiesP; ++i) {
      const int row = RowCopier<kCopiesP>::row_of(wave, lane, i);
      cp.place(i, lane, row, v + row < p.V, (uint32_t)row * (uint32_t)p.ld_w, tail);
    }
    turned = row_tiles == 1 ? vt % steps : 0;   // with one tile of rows blocks begin at different places of K
  };
  auto first = [&](Walk& w, const char* base, auto& c) __attribute__((always_inline)) {
    w.k = turned;
    w.left = steps;
    w.from = buffer_from(base + (int64_t)turned * (kTileK * 2), kOutside);
    if (tail != 0 && w.k == steps - 1) c.flip();
  };
  auto next = [&](Walk& w, auto& c) __attribute__((always_inline)) {
    if (--w.left <= 0) {
      if (w.left == 0 && tail != 0 && w.k == steps - 1) c.flip();
      w.from[2] = 0;
      return;
    }
    const bool wrap = w.k + 1 == steps;
    if (tail != 0 && (wrap || w.k + 2 == steps)) c.flip();   // out of the last step, or into it
    const int64_t by = wrap ? -(int64_t)(steps - 1) * (kTileK * 2) : kTileK * 2;
    const uint64_t b = ((uint64_t)w.from[1] << 32 | w.from[0]) + (uint64_t)by;
    w.from[0] = (uint32_t)b;
    w.from[1] = (uint32_t)(b >> 32);
    w.k = wrap ? 0 : w.k + 1;
  };

  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_ptr_t)smem;
  const uint32_t ring_p = lds0, ring_q = lds0 + SP * kBytesP;
  auto copy_p = [&](uint32_t to, int c) __attribute__((always_inline)) { cp.one(c, wp_.from, to, wave); };
  auto copy_q = [&](uint32_t to, int c) __attribute__((always_inline)) { cq.one(c, wq_.from, to, wave); };
  Reader<kVocab, false> rp;
  Reader<TQ, false> rq;
  rp.place(ring_p, wp * kHalf, lane);
  rq.place(ring_q, wq * 16 * QB, lane);

  f32x4_t acc[kBlocksP][QB];
  struct Half { bf16x8_t p[kBlocksP], q[QB]; };
  constexpr int kReads = kBlocksP + QB;
  auto read = [&](Half& h, int kk, int c) __attribute__((always_inline)) {
    if (c < QB) h.q[c] = rq.get(c, kk);
    else h.p[c - QB] = rp.get(c - QB, kk);
  };
  // The largest tile takes both halves of K of a block back to back, which draws less power.
  constexpr bool kPaired = TQ == 256;
  static_assert(!kPaired || (kSplit && SQ == 2), "the copies of a step");
  bf16x8_t fq[2 * QB], fp[2][2][2];
  auto read_pair = [&](int i, int c) __attribute__((always_inline)) { fp[i / 2 % 2][c / 2][c % 2] = rp.get((i + c / 2) % kBlocksP, c % 2); };
  struct Copies { int p, q; uint32_t to_p, to_q; };
  auto half_step = [&](const Half& use, Half& fill, int kk, const Copies& n) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kBlocksP; ++i) {
#pragma unroll
      for (int m = 0; m < QB; ++m) {
        const int j = i & 1 ? QB - 1 - m : m;
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(use.p[i], use.q[j], acc[i][j], 0, 0, 0);
      }
#pragma unroll
      for (int c = kReads * i / (kBlocksP - 1); c < kReads * (i + 1) / (kBlocksP - 1) && c < kReads; ++c) read(fill, kk, c);
#pragma unroll
      for (int c = (n.p + n.q) * i / kBlocksP; c < (n.p + n.q) * (i + 1) / kBlocksP; ++c) {
        if (c < n.p) copy_p(n.to_p, c);
        else copy_q(n.to_q, c - n.p);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  uint32_t slot_p = ring_p, slot_q = ring_q;   // of the step being multiplied
  auto next_p = [&](uint32_t s) __attribute__((always_inline)) { return s == ring_p + (SP - 1) * kBytesP ? ring_p : s + kBytesP; };
  auto next_q = [&](uint32_t s) __attribute__((always_inline)) { return s == ring_q + (SQ - 1) * kBytesQ ? ring_q : s + kBytesQ; };
  auto last_p = [&]() __attribute__((always_inline)) { return slot_p == ring_p ? ring_p + (SP - 1) * kBytesP : slot_p - kBytesP; };
  // The meeting of a step: its slots have been read by this wave, and its copies for the next have arrived; so, then, for all waves.
  auto meet = [&]() __attribute__((always_inline)) {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((SP - 2) * kCopiesP + (SQ - 2) * kCopiesQ) : "memory");
    const uint32_t to_p = next_p(slot_p), to_q = next_q(slot_q);
    rp.move((int)(to_p - slot_p));
    rq.move((int)(to_q - slot_q));
    slot_p = to_p;
    slot_q = to_q;
  };

  if (!gradient_mode(MODE) && blockIdx.x == 0 && threadIdx.x == 0) {
    p.found[0] = 2 * parts;
    p.found[1] = rows;
  }
  Rows<QB> st;
  int done_vt = -1, done_row0 = 0, done_part = 0, done_tiles = 0, unit_tiles = 0;   // the tile whose logits are in the accumulators
  bool done_last = false, fresh = true;                                             // the last of its unit; fresh: a unit is to be begun
  auto load = [&](int j, float (&x)[32]) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < QB; ++c) {
      if (c != j) continue;
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) x[4 * i + r] = acc[i][c][r];
    }
  };
  for (;;) {
    const bool more = unit < end;
    if (more) {
      if (fresh) start_unit();
      start_tile();
      uint32_t to_p = slot_p, to_q = slot_q;
#pragma unroll
      for (int s = 0; s < SQ; ++s) {
        if (s < SP - (kSplit ? 1 : 0)) {
          if (s == 0) first(wp_, p_base, cp);
          else next(wp_, cp);
#pragma unroll
          for (int c = 0; c < kCopiesP; ++c) copy_p(to_p, c);
          to_p = next_p(to_p);
        }
        if (s == 0) first(wq_, q_base, cq);
        else next(wq_, cq);
#pragma unroll
        for (int c = 0; c < kCopiesQ; ++c) copy_q(to_q, c);
        to_q = next_q(to_q);
      }
    }
    if (done_vt >= 0) {
      const int64_t v = (int64_t)done_vt * kVocab + wp * kHalf;
      const int q0 = done_row0 + wq * 16 * QB, g = lane >> 4;
      if constexpr (gradient_mode(MODE)) {
        GradientRows<QB> of;
        of.read(p, q0, found);
        gradient_tile<QB, false, MODE == kGradientsLow>(load, of, v, q0, found);
      } else {
        if (done_tiles == 0) st.clear(q0, rows);
        const int own_row = q0 + 16 * g + (lane & 15);
        const int target[1] = {g < QB && p.targets != nullptr && own_row < rows ? p.targets[own_row] : -1};
        const int64_t of_half = (int64_t)(2 * done_part + wp) * rows;
        auto place = [&](int k, bool& in) __attribute__((always_inline)) {
          const int row = q0 + 16 * (4 * k + g) + (lane & 15);
          in = in && row < rows;
          return p.part_top + (of_half + (in ? row : 0)) * p.n_top;
        };
        ++done_tiles;
        // (with alternatives column by column in a loop: unrolled, 2129 registers are spilled and 900 rows take 1902 us)
        reduce_tile<QB, MODE == kAlternatives, MODE == kAlternatives, true>(load, st, v + 4 * g, 0, p.V, target, q0, lists, done_tiles == 1, sort_now(done_tiles, unit_tiles), place);
        if (done_last) {
#pragma unroll
          for (int k = 0; k < Rows<QB>::kOwn; ++k) {
            const int row = q0 + 16 * (4 * k + g) + (lane & 15);
            if (4 * k + g < QB && row < rows) {
              p.part_e[of_half + row] = st.e[k];
              p.part_s[of_half + row] = st.s[k];
              p.part_t[of_half + row] = st.t[k];
            }
          }
          done_tiles = 0;
        }
      }
    }
    if (!more) break;
    // The first slots; with the last tile's stores behind them no count tells them from the others.
    constexpr int kLater = (SP - (kSplit ? 2 : 1)) * kCopiesP + (SQ - 1) * kCopiesQ;
    if (done_vt < 0) asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(kLater) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
    for (int i = 0; i < kBlocksP; ++i)
#pragma unroll
      for (int j = 0; j < QB; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    if constexpr (kPaired) {
#pragma unroll
      for (int c = 0; c < 2 * QB; ++c) fq[c] = rq.get(c % QB, c / QB);
#pragma unroll
      for (int c = 0; c < 4; ++c) read_pair(0, c);
      for (int step = 0; step < steps; ++step) {
        const uint32_t free_p = last_p(), free_q = slot_q;
        next(wp_, cp);
#pragma unroll
        for (int i = 0; i < kBlocksP; i += 2) {
#pragma unroll
          for (int j = 0; j < QB; ++j) {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
#pragma unroll
              for (int kk = 0; kk < 2; ++kk) {
                f32x4_t& sum = acc[i + b][j];
                sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fp[i / 2 % 2][b][kk], fq[kk * QB + j], sum, 0, 0, 0);
              }
            }
            if (j < 2) {
              read_pair(i + 2, 2 * j);
              read_pair(i + 2, 2 * j + 1);
            }
            if (i == kBlocksP - 4 && j == 2) {   // all of this step has been read
              meet();
              next(wq_, cq);
            }
            if (i == kBlocksP - 2) {   // the next step's, as this one's last products go
              fq[j] = rq.get(j, 0);
              fq[QB + j] = rq.get(j, 1);
            }
            const int at = i / 2 * QB + j, from_q = (kBlocksP / 2 - 1) * QB - 1;   // P's copies before the meeting, Q's behind it
            if (at < 2 * kCopiesP && at % 2 == 1) copy_p(free_p, at / 2);
            if (at >= from_q && at - from_q < kCopiesQ) copy_q(free_q, at - from_q);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      }
    } else {
      Half h0, h1;
#pragma unroll
      for (int c = 0; c < kReads; ++c) read(h0, 0, c);
      for (int step = 0; step < steps; ++step) {
        if constexpr (kSplit) next(wp_, cp);
        half_step(h0, h1, 1, Copies{kSplit ? kCopiesP : 0, 0, last_p(), 0});
        const Copies n = {kSplit ? 0 : kCopiesP, kCopiesQ, slot_p, slot_q};
        meet();
        if constexpr (!kSplit) next(wp_, cp);
        next(wq_, cq);
        half_step(h1, h0, 0, n);
      }
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    done_vt = vt;
    done_row0 = row0;
    done_part = part;
    unit_tiles = vt_end - vt_begin;
    done_last = fresh = ++vt == vt_end;
    if (fresh) unit += stride;
  }
}

constexpr int kLds = 160 * 1024;
static_assert(ring_bytes(kVocab, 256, 3, 2) <= kLds && ring_bytes(kVocab, 128, 3, 3) <= kLds && ring_bytes(kVocab, 64, 4, 4) <= kLds, "rings");

template <int MODE>
__global__ __launch_bounds__(kThreads) void logprob_kernel(const LogitParams p) {
  __shared__ __attribute__((aligned(1024))) char smem[kLds];
  const int rows = rows_found(p);
  if (rows <= 0) return;
  const int tile = tile_rows(rows);
  if constexpr (MODE != kAlternatives) {
    if (tile == 256) return run_units<MODE, 256, 3, 2>(p, smem, rows, rows);
  }
  if (tile >= kListedTile) run_units<MODE, kListedTile, 3, 3>(p, smem, rows, rows);
  else run_units<MODE, 64, 4, 4>(p, smem, rows, rows);
}
template <int MODE, int TQ, int SP, int SQ>
__global__ __launch_bounds__(kThreads) void logit_gradient_kernel(const LogitParams p) {
  __shared__ __attribute__((aligned(1024))) char smem[ring_bytes(kVocab, TQ, SP, SQ)];
  run_units<MODE, TQ, SP, SQ>(p, smem, p.max_rows, rows_found(p));
}

// Joins a row's parts, a wave a row: a lane takes every 64th half.  Bound by the time to memory, which another kernel wrote: the
// loads of a row go out together.
constexpr int kJoinWaves = 4;
struct JoinParams {
  LogitParams l;
  float *out_logprob, *out_entropy, *out_lse, *top_logprob;
  int32_t* top_id;
  int64_t entries;   // of the parts' arrays
};
template <typename T, typename F>
__device__ __forceinline__ T over_wave(T v, F f) {
#pragma unroll
  for (int x = 32; x >= 1; x >>= 1) v = f(v, __shfl_xor(v, x, 64));
  return v;
}
// HELD: halves of a lane, at most.  Every lane loads as much, what lies past the halves counting nothing: loads behind a branch each
// would be waited for one by one.
template <int HELD>
__device__ __forceinline__ void join_rows(const JoinParams& p, int rows, int halves, int stride) {
  const LogitParams& l = p.l;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  for (int64_t row = (int64_t)blockIdx.x * kJoinWaves + wave; row < rows; row += (int64_t)gridDim.x * kJoinWaves) {
    float pe[HELD], ps[HELD], pt[HELD];
    Candidate head[HELD], second[HELD];
    int taken[HELD];
    float e = kNegExponent;
    const int target = p.out_logprob != nullptr ? l.targets[row] : -1;
    const float target_logit = p.out_logprob != nullptr ? l.target_logit[row] : 0.f;   // (holds nothing where there is no target)
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
      const int64_t at = (int64_t)(lane + 64 * i < halves ? lane + 64 * i : 0) * stride + row;
      pe[i] = l.part_e[at];
      ps[i] = l.part_s[at];
      pt[i] = l.part_t[at];
    }
    if (l.n_top > 0) {
#pragma unroll
      for (int i = 0; i < HELD; ++i) {
        const Candidate* const best = l.part_top + ((int64_t)(lane + 64 * i < halves ? lane + 64 * i : 0) * stride + row) * l.n_top;
        head[i] = best[0];
        second[i] = best[l.n_top > 1 ? 1 : 0];
      }
    }
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
      const bool there = lane + 64 * i < halves;
      pe[i] = there ? pe[i] : kNegExponent;
      ps[i] = there ? ps[i] : 0.f;
      pt[i] = there ? pt[i] : 0.f;
      taken[i] = 0;
      e = fmaxf(e, pe[i]);
    }
    e = over_wave(e, [](float a, float b) { return fmaxf(a, b); });
    double s = 0.0, t = 0.0;
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
      const float by = pe[i] - e, scale = __builtin_amdgcn_exp2f(by);
      s += (double)(scale * ps[i]);
      t += (double)scale * ((double)pt[i] + (double)ps[i] * by);
    }
    s = over_wave(s, [](double a, double b) { return a + b; });
    t = over_wave(t, [](double a, double b) { return a + b; });
    // back from powers of two, by the factor that the exponents were made with
    const double log_s = log2(s), lse = ((double)e + log_s) / (double)kLog2e;
    if (lane == 0) {
      if (p.out_lse != nullptr) p.out_lse[row] = (float)lse;
      // an entropy is never below zero, a log probability never above it, whatever the last bits of a certain row's sums say
      const float entropy = (float)((log_s - t / s) / (double)kLog2e);
      if (p.out_entropy != nullptr) p.out_entropy[row] = entropy < 0.f ? 0.f : entropy;
      if (p.out_logprob != nullptr) {
        const float logp = (uint32_t)target < (uint32_t)l.V ? (float)((double)target_logit - lse) : 0.f;
        p.out_logprob[row] = logp > 0.f ? 0.f : logp;
      }
    }
    if (l.n_top == 0) continue;
    // The best n_top of the halves' best: a lane holds the first two candidates left of its halves and, each time the best of all is
    // its own, fetches another of that half.
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
      const bool there = lane + 64 * i < halves;
      head[i] = there ? head[i] : 0.0;
      second[i] = there && l.n_top > 1 ? second[i] : 0.0;
    }
    for (int k = 0; k < l.n_top; ++k) {
      Candidate best = 0.0;
#pragma unroll
      for (int i = 0; i < HELD; ++i) best = first_of_two(head[i], best);
      best = over_wave(best, [](double a, double b) { return first_of_two(a, b); });
#pragma unroll
      for (int i = 0; i < HELD; ++i) {
        if (best != 0.0 && head[i] == best) {   // (ids differ, so it is one lane's)
          ++taken[i];
          head[i] = second[i];
          second[i] = taken[i] + 1 < l.n_top ? l.part_top[((int64_t)(lane + 64 * i) * stride + row) * l.n_top + taken[i] + 1] : 0.0;
        }
      }
      if (lane == 0) {
        const float logp = best != 0.0 ? (float)((double)logit_of(best) - lse) : -__builtin_inff();
        p.top_id[row * l.n_top + k] = best != 0.0 ? id_of(best) : -1;
        p.top_logprob[row * l.n_top + k] = logp > 0.f ? 0.f : logp;
      }
    }
  }
}
__global__ __launch_bounds__(64 * kJoinWaves) void logprob_join_kernel(const JoinParams p) {
  const LogitParams& l = p.l;
  const int parts = l.found[0], stride = l.found[1], rows = rows_found(l);
  if (rows <= 0) return;
  // (whatever another call on the same workspace left there, nobody is to be led beyond the arrays)
  const int halves = stride >= rows && parts > 0 && parts <= 2 * kMostSplits && (int64_t)parts * stride <= p.entries ? parts : 0;
  if (halves <= 64) join_rows<1>(p, rows, halves, stride);
  else if (halves <= 128) join_rows<2>(p, rows, halves, stride);
  else join_rows<2 * kMostSplits / 64>(p, rows, halves, stride);
}

// Rows gathered side by side.  copies: 0, the listed ones alone; 1 or 2, with zeros from the last listed one on, and so often, one
// behind the other.
__global__ __launch_bounds__(256) void gather_rows_kernel(const __bf16* x, int64_t ld_x, const int32_t* idx, const int32_t* count, int T,
                                                          int max_rows, int d, __bf16* out, int copies) {
  const int n = count == nullptr ? max_rows : *count;
  const int per_row = d / 8;
  const int64_t all = (int64_t)(copies == 0 && n < max_rows ? n : max_rows) * per_row;
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < all; e += (int64_t)gridDim.x * 256) {
    const int64_t j = e / per_row;
    const int c = (int)(e - j * per_row) * 8;
    bf16x8_t v = {};
    if (j < n) {
      int64_t t = idx == nullptr ? j : idx[j];
      t = t < 0 ? 0 : (t > T - 1 ? T - 1 : t);
      v = *reinterpret_cast<const bf16x8_t*>(x + t * ld_x + c);
    }
    *reinterpret_cast<bf16x8_t*>(out + j * d + c) = v;
    if (copies == 2) *reinterpret_cast<bf16x8_t*>(out + (max_rows + j) * d + c) = v;
  }
}

// What a row's target adds beside the products of dl: coef[j] = g (1 - p) - h p (log p + H), p = exp(logprob[j]).
struct TermParams {
  const int32_t *targets, *count;
  const float *logprob, *entropy, *dlogprob, *dentropy;
  float* coef;
  int32_t max_rows, V;
};
__global__ __launch_bounds__(256) void target_terms_kernel(const TermParams p) {
  const int found = p.count == nullptr ? p.max_rows : *p.count;
  for (int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x; j < p.max_rows; j += (int64_t)gridDim.x * 256) {
    float c = 0.f;
    if (j < found) {
      const int target = p.targets[j];
      if ((uint32_t)target < (uint32_t)p.V) {
        const float logp = p.logprob[j], prob = expf(logp);
        c = p.dlogprob[j] * -expm1f(logp);
        if (p.dentropy != nullptr) c -= p.dentropy[j] * prob * (logp + p.entropy[j]);
      }
    }
    p.coef[j] = c;
  }
}

// dx[j] = the parts' sums (of both halves where dl had two) + coef[j] w[targets[j]], rounded once.
struct RowsOutParams {
  const float* parts;
  const __bf16* w;
  const int32_t *targets, *count;   // targets: or nullptr
  const float* coef;
  __bf16* dx;
  int64_t ld_w, ld_dx;
  int32_t n_parts, max_rows, d, V;
};
__global__ __launch_bounds__(256) void rows_out_kernel(const RowsOutParams p) {
  constexpr int kAtOnce = 4;
  const int n = p.count == nullptr ? p.max_rows : *p.count;
  const int64_t rows = n < p.max_rows ? n : p.max_rows, per_row = p.d / 8, all = rows * per_row;
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < all; e += (int64_t)gridDim.x * 256) {
    const int64_t j = e / per_row;
    const int c = (int)(e - j * per_row) * 8;
    float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const int target = p.targets != nullptr ? p.targets[j] : -1;
    if ((uint32_t)target < (uint32_t)p.V) {
      const float coef = p.coef[j];
      load8(p.w + target * p.ld_w + c, s);
#pragma unroll
      for (int i = 0; i < 8; ++i) s[i] *= coef;
    }
    for (int k = 0; k < p.n_parts; k += kAtOnce) {
      float v[kAtOnce][8];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
#pragma unroll
        for (int x = 0; x < 8; ++x) v[i][x] = 0.f;
        if (k + i < p.n_parts) load8(p.parts + ((int64_t)(k + i) * p.max_rows + j) * p.d + c, v[i]);
      }
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i)
#pragma unroll
        for (int x = 0; x < 8; ++x) s[x] += v[i][x];
    }
    store8(p.dx + j * p.ld_dx + c, s);
  }
}

int64_t padded(int64_t bytes) { return (bytes + 255) / 256 * 256; }

// Where 32-bit offsets reach all hidden rows they are gathered as they are copied, else beforehand.
bool far_rows(int64_t T, int64_t ld_h) { return T * ld_h * 2 > (int64_t)kOutside; }

struct Space { int64_t found, lists, e, s, t, top, target, rows, total, entries, slots; };
Space space_of(int64_t T, int64_t ld_h, int64_t max_rows, int32_t d, int32_t V, int32_t n_top) {
  Space s;
  const int64_t tile = max_rows <= 64 ? 64 : max_rows <= 128 ? 128 : 256;
  int64_t lists;
  if (w4_takes(d, V)) {   // room for two rounds of units, and for four parts and a round more of many rows: grows with the bound
    const int64_t row_tiles = (max_rows + 255) / 256, vocab_tiles = ((int64_t)V + kVocab - 1) / kVocab;
    const int64_t most = vocab_tiles < MOSAIC_MAX_VOCAB_SPLITS ? vocab_tiles : MOSAIC_MAX_VOCAB_SPLITS;
    const int64_t wide = 4 * row_tiles + kCus, units = wide > 2 * kCus ? wide : 2 * kCus;
    s.slots = 256 * (units < row_tiles * most ? units : row_tiles * most);
    s.entries = 2 * s.slots;
    lists = w4_list_bytes();
  } else {
    // up to kMostUnits units, at most kMostSplits parts, and one part whatever the rows
    const int64_t most = (int64_t)kMostSplits * max_rows < kMostUnits * tile ? (int64_t)kMostSplits * max_rows : kMostUnits * tile;
    s.slots = most > max_rows ? most : max_rows;
    s.entries = 2 * s.slots;
    lists = (int64_t)kCus * 8 * (tile < kListedTile ? tile : kListedTile) * kListRoom * (int64_t)sizeof(Entry);
  }
  s.found = 0;
  s.lists = 256;
  s.e = s.lists + (n_top > 0 ? lists : 0);
  s.s = s.e + padded(4 * s.entries);
  s.t = s.s + padded(4 * s.entries);
  s.top = s.t + padded(4 * s.entries);
  s.target = s.top + padded((int64_t)sizeof(Candidate) * s.entries * n_top);
  s.rows = s.target + padded(4 * max_rows);
  s.total = s.rows + (far_rows(T, ld_h) ? 2 * max_rows * d : 0);
  return s;
}

}  // namespace

int64_t logprob_workspace_bytes(int64_t T, int64_t ld_h, int64_t max_rows, int32_t d, int32_t V, int32_t n_top) {
  return space_of(T, ld_h, max_rows, d, V, n_top).total;
}

int launch_logprobs(const LogprobArgs& a, hipStream_t stream) {
  const Space at = space_of(a.T, a.ld_h, a.max_rows, a.d, a.V, a.n_top);
  char* ws = static_cast<char*>(a.workspace);
  LogitParams p = {};
  p.w = static_cast<const char*>(a.w);
  p.x = static_cast<const char*>(a.hidden);
  p.ld_w = a.ld_w * 2;
  p.ld_x = a.ld_h * 2;
  p.idx = a.idx;
  p.count = a.count;
  p.targets = a.targets;
  p.T = (int32_t)a.T;
  p.max_rows = (int32_t)a.max_rows;
  p.V = a.V;
  p.d = a.d;
  p.n_top = a.n_top;
  p.found = reinterpret_cast<int32_t*>(ws + at.found);
  p.part_e = reinterpret_cast<float*>(ws + at.e);
  p.part_s = reinterpret_cast<float*>(ws + at.s);
  p.part_t = reinterpret_cast<float*>(ws + at.t);
  p.part_top = reinterpret_cast<Candidate*>(ws + at.top);
  p.target_logit = reinterpret_cast<float*>(ws + at.target);
  p.lists = a.n_top > 0 ? reinterpret_cast<Entry*>(ws + at.lists) : nullptr;
  if (a.idx != nullptr && far_rows(a.T, a.ld_h)) {
    __bf16* rows = reinterpret_cast<__bf16*>(ws + at.rows);
    const int64_t pieces = a.max_rows * (a.d / 8);
    if (launch_kernel(gather_rows_kernel, dim3((unsigned)((pieces + 255) / 256 < 65536 ? (pieces + 255) / 256 : 65536)), dim3(256),
                      stream, static_cast<const __bf16*>(a.hidden), a.ld_h, a.idx, a.count, (int)a.T, (int)a.max_rows, a.d, rows, 0) != 0)
      return -1;
    p.x = reinterpret_cast<const char*>(rows);
    p.ld_x = (int64_t)a.d * 2;
    p.idx = nullptr;
  }
  if (w4_takes(a.d, a.V)) {
    p.sched.slots64 = (uint32_t)(at.slots / 64 < INT32_MAX ? at.slots / 64 : INT32_MAX);
    if ((a.n_top > 0 ? launch_alternatives_w4(p, stream) : launch_statistics_w4(p, stream)) != 0) return -1;
  } else if (launch_kernel(a.n_top > 0 ? logprob_kernel<kAlternatives> : logprob_kernel<kStatistics>, dim3(kCus), dim3(kThreads), stream, p) != 0) {
    return -1;
  }
  JoinParams j = {};
  j.entries = at.entries;
  j.l = p;
  j.out_logprob = a.out_logprob;
  j.out_entropy = a.out_entropy;
  j.out_lse = a.out_lse;
  j.top_logprob = a.top_logprob;
  j.top_id = a.top_id;
  const int64_t blocks = (a.max_rows + kJoinWaves - 1) / kJoinWaves;
  return launch_kernel(logprob_join_kernel, dim3((unsigned)(blocks < 8192 ? blocks : 8192)), dim3(64 * kJoinWaves), stream, j);
}

// ---- gradients.  Per part of the vocabulary: dl of its ids, then both products of it.
namespace {

// Of dl, where the caller sets no other bound: what is written for a part of the vocabulary and read twice fits the memory-side cache,
// and a part has enough ids to fill the chip (2048 rows of 126464 ids: two parts).
constexpr int64_t kDlBytes = (int64_t)256 << 20;
// Up to here dl carries what its rounding leaves over into both results, as the feed-forward block's; beyond, into dw of 32 bits alone:
// results of 16 bits are rounded by more than it adds (dw and dx of 2048 rows of 126464 x 4096 are 0.00170 and 0.00171 off in the 2-norm,
// rounded alone 0.00165 and 0.00166; 900 of 32000 x 1024 0.00175 and 0.00176 for 0.00166 and 0.00167).  dw of 32 bits is 6e-7 off, with
// terms of 16 bits 4e-4; its products are twice as many: 2048 rows of 126464 x 4096 6.6 ms, with terms of 16 bits 5.0, dw of 16 bits 4.8.
constexpr int64_t kLowRows = 32;

struct GradientSpace {
  int64_t rows, coef, sort, sums, extra, slot, parts, dl, least;   // offsets; least: bytes for one tile of ids
  int64_t dx_rows;   // of dl in dx's product
  int32_t splits;
};
constexpr int64_t kSlotBytes = 4096;   // the slots are filled in rows of so many bytes
int64_t slot_rows(int32_t V) { return (4 * (int64_t)V + kSlotBytes - 1) / kSlotBytes; }
GradientSpace gradient_space(int64_t max_rows, int32_t d, int32_t V) {
  GradientSpace s;
  s.dx_rows = max_rows <= kLowRows ? 2 * max_rows : max_rows;
  s.splits = plan_row_product(s.dx_rows, d, V < 65536 ? V : 65536).splits;
  s.rows = 0;
  s.coef = s.rows + padded(4 * max_rows * d);   // twice: K of dw where dl has two numbers an entry
  s.sort = s.coef + padded(4 * max_rows);
  s.sums = s.sort + padded(sort_tokens_bytes(max_rows));
  s.extra = s.sums + padded(4 * token_sum_partials(max_rows, d) * d);
  s.slot = s.extra + padded(4 * max_rows * d);
  s.parts = s.slot + slot_rows(V) * kSlotBytes;
  const int64_t most = max_rows <= kLowRows || max_rows > 2 * kLowRows ? s.dx_rows : 2 * kLowRows;   // so that fewer rows need no more
  s.dl = s.parts + padded(4 * most_part_rows(most) * d);
  s.least = s.dl + 4 * max_rows * kVocab;
  return s;
}
// Ids at a time with so many bytes for dl, evenly, in whole tiles.
constexpr int64_t kMostIds = (int64_t)1 << 18;
int64_t ids_at_once(int64_t dl_rows, int32_t V, int64_t bytes) {
  int64_t most = bytes / (2 * dl_rows) / kVocab * kVocab;
  if (most > kMostIds) most = kMostIds;
  if (most < kVocab) most = kVocab;
  const int64_t parts = ((int64_t)V + most - 1) / most;
  return (((int64_t)V + parts - 1) / parts + kVocab - 1) / kVocab * kVocab;
}

template <int MODE>
int launch_gradient_tiles(const LogitParams& p, hipStream_t stream) {
  const int tile = tile_rows(p.max_rows);
  if (tile == 256) return launch_kernel(logit_gradient_kernel<MODE, 256, 3, 2>, dim3(kCus), dim3(kThreads), stream, p);
  if (tile == 128) return launch_kernel(logit_gradient_kernel<MODE, 128, 3, 3>, dim3(kCus), dim3(kThreads), stream, p);
  return launch_kernel(logit_gradient_kernel<MODE, 64, 4, 4>, dim3(kCus), dim3(kThreads), stream, p);
}

// dl of `n` ids from v on: whole tiles of ids on the 4-wave kernel where it takes them.
int launch_dl(LogitParams p, int64_t v, int64_t n, hipStream_t stream) {
  const int64_t whole = w4_takes(p.d, kVocab) ? n / kVocab * kVocab : 0;
  const char* w = p.w + v * p.ld_w;
  char* dl = p.dl;
  const int64_t parts[2][2] = {{0, whole}, {whole, n - whole}};
  for (int k = 0; k < 2; ++k) {
    if (parts[k][1] == 0) continue;
    p.w = w + parts[k][0] * p.ld_w;
    p.dl = dl + parts[k][0] * 2;
    p.V = (int32_t)parts[k][1];
    p.dl_ids = (p.V + 7) / 8 * 8;
    p.first_id = (int32_t)(v + parts[k][0]);
    const auto launch = p.low != 0 ? (k == 0 ? launch_gradients_low_w4 : launch_gradient_tiles<kGradientsLow>)
                                   : (k == 0 ? launch_gradients_w4 : launch_gradient_tiles<kGradients>);
    if (launch(p, stream) != 0) return -1;
  }
  return 0;
}

}  // namespace

int64_t logprob_backward_workspace_bytes(int64_t max_rows, int32_t d, int32_t V, int64_t budget_bytes) {
  const GradientSpace at = gradient_space(max_rows, d, V);
  const int64_t room = budget_bytes > 0 ? budget_bytes - at.dl : kDlBytes;
  return at.dl + 4 * max_rows * ids_at_once(2 * max_rows, V, room);   // with two numbers an entry
}
int64_t logprob_backward_least_bytes(int64_t max_rows, int32_t d, int32_t V) { return gradient_space(max_rows, d, V).least; }

int launch_logprobs_backward(const LogprobBackwardArgs& a, hipStream_t stream) {
  const GradientSpace at = gradient_space(a.max_rows, a.d, a.V);
  const bool dw = a.dw != nullptr, low = a.max_rows <= kLowRows || (dw && a.dw_f32 != 0);   // whether dl has two numbers an entry
  const int64_t dl_rows = low ? 2 * a.max_rows : a.max_rows;
  char* ws = static_cast<char*>(a.workspace);
  __bf16* rows = reinterpret_cast<__bf16*>(ws + at.rows);
  float* coef = reinterpret_cast<float*>(ws + at.coef);
  float* extra = reinterpret_cast<float*>(ws + at.extra);
  int32_t* slot = reinterpret_cast<int32_t*>(ws + at.slot);
  float* parts = reinterpret_cast<float*>(ws + at.parts);
  const int64_t pieces = (a.max_rows * (a.d / 8) + 255) / 256;
  const dim3 grid((unsigned)(pieces < 65536 ? pieces : 65536));
  if (launch_kernel(gather_rows_kernel, grid, dim3(256), stream, static_cast<const __bf16*>(a.hidden), a.ld_h, a.idx, a.count, (int)a.T,
                    (int)a.max_rows, a.d, rows, low ? 2 : 1) != 0)
    return -1;
  // the targets' own terms: for dw summed by target
  if (a.targets != nullptr) {
    TermParams t = {a.targets, a.count, a.logprob, a.entropy, a.dlogprob, a.dentropy, coef, (int32_t)a.max_rows, a.V};
    const int64_t blocks = (a.max_rows + 255) / 256;
    if (launch_kernel(target_terms_kernel, dim3((unsigned)(blocks < 1024 ? blocks : 1024)), dim3(256), stream, t) != 0) return -1;
    if (dw) {
      TokenSumArgs sum = {};
      const FillArgs none = {slot, kSlotBytes, slot_rows(a.V), kSlotBytes, 0xffffffffu};   // no target names an id: -1
      if (launch_sort_tokens(a.targets, a.max_rows, a.count, a.V, ws + at.sort, none, &sum.sorted, stream) != 0) return -1;
      sum.rows = rows;
      sum.weights = coef;
      sum.partials = reinterpret_cast<float*>(ws + at.sums);
      sum.sums = extra;
      sum.first = slot;
      sum.n = a.max_rows;
      sum.ld_rows = sum.ld_sums = a.d;
      sum.V = a.V;
      sum.d = a.d;
      sum.scale = 1.f;
      if (launch_token_sums(sum, false, true, stream) != 0) return -1;
    }
  }
  const int64_t each = ids_at_once(dl_rows, a.V, a.workspace_bytes - at.dl);
  LogitParams p = {};
  p.w = static_cast<const char*>(a.w);
  p.x = reinterpret_cast<const char*>(rows);
  p.ld_w = a.ld_w * 2;
  p.ld_x = (int64_t)a.d * 2;
  p.count = a.count;
  p.targets = a.targets;
  p.T = (int32_t)a.T;
  p.max_rows = (int32_t)a.max_rows;
  p.d = a.d;
  p.lse = a.lse;
  p.entropy = a.entropy;
  p.dlogprob = a.dlogprob;
  p.dentropy = a.dentropy;
  p.dl = ws + at.dl;
  p.ld_dl = each * 2;
  p.low = low ? a.max_rows * p.ld_dl : 0;
  p.all_ids = a.V;
  for (int64_t v = 0; v < a.V; v += each) {
    const int64_t n = a.V - v < each ? a.V - v : each;
    if (launch_dl(p, v, n, stream) != 0) return -1;
    if (a.dx != nullptr) {
      ProductArgs x = {};
      x.p = p.w + v * p.ld_w;
      x.q = p.dl;
      x.out = parts;
      x.ld_p = a.ld_w;
      x.ld_q = each;
      x.ld_out = a.d;
      x.rows = at.dx_rows;
      x.depth = n;
      x.cols = a.d;
      x.splits = at.splits;
      x.f32 = 1;
      x.accumulate = v > 0;
      if (launch_row_product(x, stream) != 0) return -1;
    }
    if (dw) {
      ProductArgs w = {};
      w.p = rows;
      w.q = p.dl;
      w.out = static_cast<char*>(a.dw) + v * a.ld_dw * (a.dw_f32 ? 4 : 2);
      w.slot = a.targets != nullptr ? slot + v : nullptr;
      w.extra = extra;
      w.ld_p = w.ld_extra = a.d;
      w.ld_q = each;
      w.ld_out = a.ld_dw;
      w.rows = n;
      w.depth = dl_rows;
      w.cols = a.d;
      w.splits = 1;
      w.f32 = a.dw_f32;
      w.accumulate = a.accumulate;
      if (launch_column_product(w, stream) != 0) return -1;
    }
  }
  if (a.dx == nullptr) return 0;
  RowsOutParams o = {};
  o.parts = parts;
  o.w = static_cast<const __bf16*>(a.w);
  o.targets = a.targets;
  o.count = a.count;
  o.coef = coef;
  o.dx = static_cast<__bf16*>(a.dx);
  o.ld_w = a.ld_w;
  o.ld_dx = a.ld_dx;
  o.n_parts = at.splits * (int32_t)(at.dx_rows / a.max_rows);
  o.max_rows = (int32_t)a.max_rows;
  o.d = a.d;
  o.V = a.V;
  return launch_kernel(rows_out_kernel, grid, dim3(256), stream, o);
}

}  // namespace mosaic
