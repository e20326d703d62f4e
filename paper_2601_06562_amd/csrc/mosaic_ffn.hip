// Gated feed-forward block, act(x Wg^T) * (x Wu^T), and its gradients, on the matrix cores.
//
// All products run through one kernel: a tile of "P" rows by "Q" rows (256 x 256 where there is work enough), K in steps of 64.
// P is the operand whose rows are the output's contiguous columns (the accumulator layout gives a lane four consecutive P
// rows of one Q row), Q the one whose rows are the output's rows:
//   forward, and the projections again in the backward pass:  P = rows of Wg and as many of Wu, Q = x; the two projections
//     of an element meet in one lane, so the activation and the product need no exchange
//   dx:  P = columns of Wg, then of Wu (K = 2 F), Q = dg | du
//   dw:  P = columns of x (K = T), Q = columns of dg | du
// Operands that lie across K are read from LDS by transposing reads; nothing is transposed in memory.
//
// What bounds it, on MI355X (16384 rows of d 4096, F 12288, 256 x 256 tiles; cards differ by 4%): forward 2230 to 2320 us, 1.42
// to 1.48 PFLOP/s, the projections with the gradients' epilogue 2500, dx 2270, dw 2290.  The matrix cores are busy 78% of the
// cycles, LDS 30% and without conflicts, at a clock of 1.65 GHz that the card's power sets: without barriers and waits the same
// tile gains 3%.  A library's plain product of the same sizes takes 2100 us.  The projections of the backward pass, which have
// the most operands, keep some scalar registers in vector lanes; those are read back between tiles and where a step does
// more than move the descriptors on, not in the steps that only do that.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mosaic_ffn_choice.h"
#include "mosaic_layer_internal.h"
#include "mosaic_tile.h"

namespace mosaic {
namespace {

using namespace ffn;
using namespace tile;

struct GemmArgs {
  const char* p0;      // P: weights (gate / its columns), or x
  const char* p1;      // up
  const char* q;       // x, or dg | du
  int64_t ld_p, ld_q;  // bytes
  int64_t rows_q;      // Q rows of the output
  int32_t rows_p;      // P rows of the output: F, d
  int64_t depth;       // K: of a segment, where there are two (kDx: gate, up)
  int32_t tiles_p, tiles_q;
  int32_t splits;      // kDx: parts of K
  int32_t F, f32, accumulate;
  const char* dout;
  int64_t ld_dout;     // bytes, as the strides below
  char* out0;          // forward: out; kRecompute: out or nullptr; kDx: dx or the partial sums; kDw: dw_gate
  char* out1;          // kRecompute: dg | du; kDw: dw_up
  int64_t ld_out0, ld_out1;
  int64_t low;         // kRecompute: from a row of dg | du to that of its low halves, bytes; 0: none are wanted
  int32_t repeat;      // kDw: rows of x there are where K, one step then, takes them twice; else 0
  const int32_t* slot; // kOneDw: for each output row the row of `extra` that is added to it, or -1; nullptr: none
  const float* extra;
  int64_t ld_extra;    // elements
};

__device__ __forceinline__ float sigmoid(float z) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504088896340736f));
}

// The activation of g and its slope.  GELU in its tanh form is g sigmoid(2 z); beyond |g| = 16 the sigmoid is 0 or 1 to the
// last bit, and the clamp keeps z and its slope finite (a NaN passes it).
template <int ACT>
__device__ __forceinline__ void activate(float g, float& a, float& slope) {
  if constexpr (ACT == MOSAIC_SILU) {
    const float s = sigmoid(g);
    a = g * s;
    slope = s * (1.0f + g * (1.0f - s));
  } else {
    const float c = g > 16.0f ? 16.0f : g < -16.0f ? -16.0f : g;
    constexpr float k2 = 1.59576912160573081f;   // 2 sqrt(2 / pi)
    const float s = sigmoid(k2 * c * (1.0f + 0.044715f * c * c));
    a = g * s;
    slope = s * (1.0f + c * (1.0f - s) * k2 * (1.0f + 0.134145f * c * c));
  }
}

// 256 x 256: the most products a byte of LDS and of the caches; 128 accumulator registers a lane and two waves a SIMD, which
// fill each other's gaps (four waves of 128 x 128 each read a third less from LDS and were no faster forward; the gradients'
// registers spilled).  K in steps of 64 through rings of slots, copied straight into LDS.
// The tiles of one product, dealt to `blocks` blocks of which this is number `block`.  The blocks of an XCD take its run of
// tiles in turn, and the copies of a block's next tile are under way while the results of the last one are worked out and
// stored.
template <int MODE, int TP, int TQ, int SP, int SQ, int ACT>
__device__ __forceinline__ void run_tiles(const GemmArgs& a, char* smem, int block, int blocks) {
  constexpr bool kGated = gated_mode(MODE), kIsDx = MODE == kDx || MODE == kOneDx, kIsDw = MODE == kDw || MODE == kOneDw;
  constexpr bool kRowP = !kGated, kRowQ = kIsDw;
  constexpr int kTileP = TP, kTileQ = TQ, kBlocksP = TP / 32, QB = TQ / 64;   // blocks of a wave
  constexpr int kBytesP = kTileP * kStepK * 2, kBytesQ = kTileQ * kStepK * 2;
  using CopierP = Copier<kTileP, kRowP>;
  using CopierQ = Copier<kTileQ, kRowQ>;
  constexpr int kCopiesP = CopierP::kCopies, kCopiesQ = CopierQ::kCopies;   // a wave and step
  // With a slot more for P its copies go out in the other half of a step, into the slot of the step before, so that a wave has
  // a copy between two groups of products all the time.
  constexpr bool kSplit = SP != SQ;
  static_assert(!kSplit || SP == SQ + 1, "the waits of the loop");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int wp = wave >> 2, wq = wave & 3;
  const int wave_p = kGated ? wq : wave;   // gated: waves 0..3 copy gate rows, waves 4..7 the up rows behind them

  // Block b runs on XCD b % 8; every XCD gets a run of tiles, and within it panels of kPanel Q tiles, so that what is in
  // flight behind one L2 shares both operands.
  const int per_split = a.tiles_p * a.tiles_q, n = per_split * a.splits;
  const int xcd = block % kXcds;
  const int stride = blocks / kXcds + (xcd < blocks % kXcds ? 1 : 0);
  int id = xcd * (n / kXcds) + (xcd < n % kXcds ? xcd : n % kXcds);   // the run's first tile
  const int end = id + n / kXcds + (xcd < n % kXcds ? 1 : 0);
  id += block / kXcds;
  if (id >= end) return;

  const int seg_steps = (int)((a.depth + kStepK - 1) / kStepK);
  const int all_steps = MODE == kDx ? 2 * seg_steps : seg_steps;

  // Of the tile whose copies are issued.
  int split, p_row, step0, step1, placed_p, placed_q, turned = 0;   // p_row: first P row; gated: first feature
  int64_t q_row;
  const char *p_base0, *p_base1, *q_base;
  CopierP cp;
  CopierQ cq;
  auto begin = [&](int id) __attribute__((always_inline)) {
    split = id / per_split;
    const int tile = id - split * per_split;
    constexpr int kPanel = kGated ? 8 : 4;
    const int panel = tile / (kPanel * a.tiles_p);
    const int deep = a.tiles_q - panel * kPanel < kPanel ? a.tiles_q - panel * kPanel : kPanel;
    const int in_panel = tile - panel * kPanel * a.tiles_p;
    p_row = in_panel / deep * (kGated ? kTileP / 2 : kTileP);
    q_row = (int64_t)(panel * kPanel + in_panel % deep) * kTileQ;
    if constexpr (kGated) {   // waves 4..7 copy the up rows
      p_base0 = p_base1 = (wp == 0 ? a.p0 : a.p1) + p_row * a.ld_p;
    } else {
      p_base0 = a.p0 + (int64_t)p_row * 2;
      p_base1 = MODE == kDx ? a.p1 + (int64_t)p_row * 2 : p_base0;
    }
    q_base = kRowQ ? a.q + q_row * 2 : a.q + q_row * a.ld_q;
    cp.place(wave_p, lane, a.ld_p, a.rows_p - p_row, kStepK, MODE == kDw ? a.repeat : 0);
    cq.place(wave, lane, a.ld_q, a.rows_q - q_row, kStepK);
    placed_p = placed_q = kStepK;
    step0 = (int)((int64_t)all_steps * split / a.splits);
    step1 = (int)((int64_t)all_steps * (split + 1) / a.splits);
    // With one Q tile the time goes to the weights, which tiles read from their start: begun at different places of K they are
    // spread over the memory's channels, where rows a power of two apart would meet in few (32 rows of d 4096, F 12288: 44.6
    // us, so 41.2; d 3584, F 18944: 57.1 and 56.3).
    if (kGated) turned = a.tiles_q == 1 ? tile % all_steps : 0;
  };

  // Where an operand's copies come from, step after step.  What lies past the end of K comes as zeros, and so do steps past
  // the last, so that the loop has no end to look after.  Most steps only move the descriptor on: the full arithmetic in each
  // of them cost the small tiles a tenth.
  struct Walk { u32x4_t from; int plain; };   // plain: how many steps the descriptor only has to be moved on
  Walk walk_p, walk_q;
  auto find = [&](int step, int& seg, int64_t& k, Walk& w) __attribute__((always_inline)) {   // k there are in `step`
    seg = MODE == kDx && step >= seg_steps ? 1 : 0;
    const int full = (int)(a.depth / kStepK);
    int at = step - seg * seg_steps, end = step1 - seg * seg_steps;
    if (step >= step1) {
      k = 0;
      w.plain = 0x7fffffff;
      return 0;
    }
    if (kGated) {   // around K, from step `turned` on
      at += turned;
      if (at >= end) {
        at -= end;
        end = turned;
      }
    }
    k = (int64_t)at * kStepK;
    const int last = end < full ? end : full;
    w.plain = at < last ? last - 1 - at : 0;
    return at < full ? kStepK : (int)(a.depth - k);
  };
  auto locate_p = [&](int step) __attribute__((always_inline)) {
    int seg;
    int64_t k;
    const int left = find(step, seg, k, walk_p);
    if (!kRowP && left != placed_p && left != 0) {   // into or out of a last step of fewer k
      placed_p = left;
      cp.place(wave_p, lane, a.ld_p, a.rows_p - p_row, left);
    }
    const int rows = MODE == kDw && a.repeat != 0 && left != 0 ? a.repeat : left;   // across K: there are behind the base
    walk_p.from = buffer_from((seg ? p_base1 : p_base0) + (kRowP ? k * a.ld_p : k * 2),
                              kRowP ? rows * (uint32_t)a.ld_p : left == 0 ? 0 : kOutside);
  };
  auto locate_q = [&](int step) __attribute__((always_inline)) {
    int seg;
    int64_t k;
    const int left = find(step, seg, k, walk_q);
    if (!kRowQ && left != placed_q && left != 0) {
      placed_q = left;
      cq.place(wave, lane, a.ld_q, a.rows_q - q_row, left);
    }
    walk_q.from = buffer_from(q_base + (kRowQ ? k * a.ld_q : (k + (int64_t)seg * a.depth) * 2),
                              kRowQ ? left * (uint32_t)a.ld_q : left == 0 ? 0 : kOutside);
  };
  auto move = [&](Walk& w, uint32_t bytes) __attribute__((always_inline)) {
    const uint64_t b = ((uint64_t)w.from[1] << 32 | w.from[0]) + bytes;
    w.from[0] = (uint32_t)b;
    w.from[1] = (uint32_t)(b >> 32);
    --w.plain;
  };
  auto step_p = [&](int step) __attribute__((always_inline)) {   // to `step`, from the one before
    if (__builtin_expect(walk_p.plain > 0, 1)) move(walk_p, kRowP ? kStepK * (uint32_t)a.ld_p : kStepK * 2);
    else locate_p(step);
  };
  auto step_q = [&](int step) __attribute__((always_inline)) {
    if (__builtin_expect(walk_q.plain > 0, 1)) move(walk_q, kRowQ ? kStepK * (uint32_t)a.ld_q : kStepK * 2);
    else locate_q(step);
  };
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_ptr_t)smem;
  const uint32_t ring_p = lds0, ring_q = lds0 + SP * kBytesP;
  auto copy_p = [&](uint32_t to, int c) __attribute__((always_inline)) {
    cp.one(c, walk_p.from, kGated ? to + wp * (kBytesP / 2) : to, wave_p);
  };
  auto copy_q = [&](uint32_t to, int c) __attribute__((always_inline)) { cq.one(c, walk_q.from, to, wave); };

  // This wave's P blocks: gated, half of them gate blocks, then the up blocks of the same features.
  Reader<kTileP, kRowP> rp;
  Reader<kTileQ, kRowQ> rq;
  rp.place(ring_p, wp * (kGated ? kTileP / 4 : kTileP / 2), lane);
  rq.place(ring_q, wq * 16 * QB, lane);
  struct Half { bf16x8_t p[kBlocksP], q[QB]; };   // the fragments of half a step, 32 k
  constexpr int kReads = kBlocksP + QB;
  auto read = [&](Half& h, int kk, int c) __attribute__((always_inline)) {   // fragment c of them, Q first
    const int i = c - QB;
    if (c < QB) h.q[c] = rq.get(c, kk);
    else h.p[i] = rp.get(kGated && i >= kBlocksP / 2 ? i + kBlocksP / 2 : i, kk);
  };
  f32x4_t acc[kBlocksP][QB];
  // Where the registers hold it, the largest tile takes both halves of K of a block back to back: a product that adds to the
  // block of the one before it.  The card's power is what such a product runs at, and this order draws less of it: 16384 rows
  // of d 4096 x F 12288, both orders in turn on one card, forward in 2280 us for 2330, dx 2270 for 2314.  (dw, which reads both
  // operands by transposing, would spill 117 registers: eight times slower.)
  // fq: a step's Q fragments; fp: those of two pairs of P blocks.
  constexpr bool kPaired = TP == 256 && TQ == 256 && !kIsDw;
  static_assert(!kPaired || (kSplit && SQ == 2 && 2 * kCopiesP <= (kBlocksP / 2 - 1) * QB - 2 && kCopiesQ <= QB + 1),
                "P's copies before the meeting of a step, Q's behind it");
  bf16x8_t fq[2 * QB], fp[2][2][2];
  auto read_pair = [&](int i, int c) __attribute__((always_inline)) {   // half c % 2 of block i + c / 2; past the last, the next step's
    const int at = i % kBlocksP + c / 2;
    fp[i / 2 % 2][c / 2][c % 2] = rp.get(kGated && at >= kBlocksP / 2 ? at + kBlocksP / 2 : at, c % 2);
  };
  // Half a step: kBlocksP groups of QB products, with the other half's reads and some copies dealt out between them.  Products
  // come first, so that what they wait for was asked for half a step ago.
  struct Copies { int p, q; uint32_t to_p, to_q; };   // p, q: how many of each operand
  auto half_step = [&](const Half& use, Half& fill, int kk, const Copies& n) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kBlocksP; ++i) {
#pragma unroll
      for (int m = 0; m < QB; ++m) {
        const int j = i & 1 ? QB - 1 - m : m;   // to and fro: one operand of a product is always that of the last
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
  // The meeting of a step: its slots have been read by this wave, and its copies for the next have arrived (all but those issued
  // since may still be under way); so, then, for all waves.  On to the next step's slots.
  auto meet = [&]() __attribute__((always_inline)) {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((SP - 2) * kCopiesP + (SQ - 2) * kCopiesQ) : "memory");
    const uint32_t to_p = next_p(slot_p), to_q = next_q(slot_q);
    rp.move((int)(to_p - slot_p));
    rq.move((int)(to_q - slot_q));
    slot_p = to_p;
    slot_q = to_q;
  };

  int done_p = 0, done_split = 0;   // the tile whose results are in the accumulators
  int64_t done_q = -1;
  for (;;) {
    // The next tile's first copies, once all waves have read what the last half step read (zeros, for nobody).
    const bool more = id < end;
    if (more) {
      begin(id);
      uint32_t to_p = slot_p, to_q = slot_q;
#pragma unroll
      for (int n = 0; n < SQ; ++n) {
        if (n < SP - (kSplit ? 1 : 0)) {
          if (n == 0) locate_p(step0);
          else step_p(step0 + n);
#pragma unroll
          for (int c = 0; c < kCopiesP; ++c) copy_p(to_p, c);
          to_p = next_p(to_p);
        }
        if (n == 0) locate_q(step0);
        else step_q(step0 + n);
#pragma unroll
        for (int c = 0; c < kCopiesQ; ++c) copy_q(to_q, c);
        to_q = next_q(to_q);
      }
    }
    if (done_q >= 0) {
      // Accumulator register r of a lane: P row 4 (lane / 16) + r, Q row lane % 16 of the block.  Gathered, a lane has
      // 4 NB consecutive P rows from run on.
      constexpr int kHalf = kBlocksP / 2, NB = kGated ? (kHalf < 4 ? kHalf : 4) : 4;
      const int sub = 4 * (lane >> 4), run = first_of<NB>(lane);
      Quad grad[MODE == kRecompute ? QB : 1][NB];   // of the outputs, all asked for ahead of their use
      if constexpr (MODE == kRecompute) {
#pragma unroll
        for (int j = 0; j < QB; ++j) {
          const int64_t q = done_q + wq * 16 * QB + j * 16 + (lane & 15);
          load_quads(a.dout + q * a.ld_dout, done_p + wp * (kTileP / 4) + run, a.rows_p, q < a.rows_q, grad[j]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int j = 0; j < QB; ++j) {
        const int64_t q = done_q + wq * 16 * QB + j * 16 + (lane & 15);
        const bool in = q < a.rows_q;
        if constexpr (kGated) {
          const int f = done_p + wp * (kTileP / 4) + run;
          Quad o[NB];
          if constexpr (MODE == kForward) {
#pragma unroll
            for (int i = 0; i < NB; ++i) {
              float v[4];
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                float act, slope;
                activate<ACT>(acc[i][j][r], act, slope);
                v[r] = act * acc[i + kHalf][j][r];
              }
              pack(o[i], v);
            }
          } else {
            constexpr bool kLow = TQ == 64;   // the tiles that few rows take
            Quad g[NB], u[NB], gl[kLow ? NB : 1], ul[kLow ? NB : 1];
            scatter(grad[j]);
#pragma unroll
            for (int i = 0; i < NB; ++i) {
              const bf16x4_t dr = __builtin_bit_cast(bf16x4_t, uint2{grad[j][i][0], grad[j][i][1]});
              float vo[4], vg[4], vu[4];
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                float act, slope;
                const float up = acc[i + kHalf][j][r], x = (float)dr[r];
                activate<ACT>(acc[i][j][r], act, slope);
                vo[r] = act * up;
                vg[r] = x * up * slope;
                vu[r] = x * act;
              }
              pack(o[i], vo);
              // dg and du in 16 bits, once from 32, as the matrix products behind take them: it adds as much as the rounding
              // of the results does (a relative 0.0023 in the 2-norm, where that alone is 0.0017); few rows, in whose sums it
              // does not average out, carry what is left over in a second row.
              pack(g[i], vg);
              pack(u[i], vu);
              if constexpr (kLow) {
                pack_low(gl[i], g[i], vg);
                pack_low(ul[i], u[i], vu);
              }
            }
            gather(g);
            gather(u);
            if (in) {
              store_quads(a.out1 + q * a.ld_out1, f, a.rows_p, g);
              store_quads(a.out1 + q * a.ld_out1 + (int64_t)a.F * 2, f, a.rows_p, u);
            }
            if constexpr (kLow) {
              if (a.low != 0) {
                gather(gl);
                gather(ul);
                if (in) {
                  store_quads(a.out1 + a.low + q * a.ld_out1, f, a.rows_p, gl);
                  store_quads(a.out1 + a.low + q * a.ld_out1 + (int64_t)a.F * 2, f, a.rows_p, ul);
                }
              }
            }
          }
          gather(o);
          if (in && a.out0 != nullptr) store_quads(a.out0 + q * a.ld_out0, f, a.rows_p, o);
        } else {
          char* row;
          if constexpr (kIsDx) row = a.out0 + ((int64_t)done_split * a.rows_q + q) * a.ld_out0;
          else if constexpr (MODE == kOneDw) row = a.out0 + q * a.ld_out0;
          else row = q < a.F ? a.out0 + q * a.ld_out0 : a.out1 + (q - a.F) * a.ld_out0;
          const int c0 = done_p + wp * (kTileP / 2);
          if constexpr (MODE == kOneDw) {
            const int at = in && a.slot != nullptr ? a.slot[q] : -1;
            if (at >= 0) {
#pragma unroll
              for (int i = 0; i < kBlocksP; ++i) {
                const int c = c0 + i * 16 + sub;
                if (c < a.rows_p) acc[i][j] += *reinterpret_cast<const f32x4_t*>(a.extra + at * a.ld_extra + c);
              }
            }
          }
          if (a.f32) {
#pragma unroll
            for (int i = 0; i < kBlocksP; ++i) {
              const int c = c0 + i * 16 + sub;
              if (in && c < a.rows_p) {
                f32x4_t* to = reinterpret_cast<f32x4_t*>(row + (int64_t)c * 4);
                *to = a.accumulate ? *to + acc[i][j] : acc[i][j];
              }
            }
          } else {
#pragma unroll
            for (int i = 0; i < kBlocksP; i += 4) {
              Quad o[4];
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const float v[4] = {acc[i + k][j][0], acc[i + k][j][1], acc[i + k][j][2], acc[i + k][j][3]};
                pack(o[k], v);
              }
              gather(o);
              if (in) store_quads(row, c0 + i * 16 + run, a.rows_p, o);
            }
          }
        }
      }
      // Told by the builtin, the compiler knows that dout has arrived.  Where it did not, it waited for all copies in every step.
      if constexpr (MODE == kRecompute) __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0)
    }
    if (!more) break;
    // The first slots; with the last tile's stores behind them no count tells them from the others.
    constexpr int kLater = (SP - (kSplit ? 2 : 1)) * kCopiesP + (SQ - 1) * kCopiesQ;
    if (done_q < 0) asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(kLater) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
    for (int i = 0; i < kBlocksP; ++i) {
#pragma unroll
      for (int j = 0; j < QB; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    if constexpr (kPaired) {
#pragma unroll
      for (int c = 0; c < 2 * QB; ++c) fq[c] = rq.get(c % QB, c / QB);
#pragma unroll
      for (int c = 0; c < 4; ++c) read_pair(0, c);
      for (int step = step0; step < step1; ++step) {
        const uint32_t free_p = slot_p == ring_p ? ring_p + (SP - 1) * kBytesP : slot_p - kBytesP, free_q = slot_q;
        step_p(step + SP - 1);
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
              step_q(step + SQ);
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
      for (int step = step0; step < step1; ++step) {
        if constexpr (kSplit) step_p(step + SP - 1);
        half_step(h0, h1, 1, Copies{kSplit ? kCopiesP : 0, 0, slot_p == ring_p ? ring_p + (SP - 1) * kBytesP : slot_p - kBytesP, 0});
        const Copies n = {kSplit ? 0 : kCopiesP, kCopiesQ, slot_p, slot_q};
        meet();
        if constexpr (!kSplit) step_p(step + SP);
        step_q(step + SQ);
        half_step(h1, h0, 0, n);
      }
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    done_p = p_row;
    done_q = q_row;
    done_split = split;
    id += stride;
  }
}

template <int MODE, int TP, int TQ, int SP, int SQ, int ACT>
__global__ __launch_bounds__(kThreads) void ffn_gemm_kernel(const GemmArgs a) {
  __shared__ __attribute__((aligned(1024))) char smem[ring_bytes(TP, TQ, SP, SQ)];
  run_tiles<MODE, TP, TQ, SP, SQ, ACT>(a, smem, (int)blockIdx.x, (int)gridDim.x);
}

// Both gradients in one launch, a tile a block: the first `blocks_x` (a multiple of the XCDs) take dx, and as they end the
// others follow on the CUs that come free.  For sizes at which neither product fills the chip: 1237 rows of d 1024, F 4096 in
// 46 us, and 6 more to join dx; such sizes took 5 to 24% longer in two launches.
template <int TP, int TQ, int SP, int SQ>
__global__ __launch_bounds__(kThreads) void ffn_gradients_kernel(const GemmArgs x, const GemmArgs w, int blocks_x) {
  __shared__ __attribute__((aligned(1024))) char smem[ring_bytes(TP, TQ, SP, SQ)];
  if ((int)blockIdx.x < blocks_x) run_tiles<kDx, TP, TQ, SP, SQ, 0>(x, smem, (int)blockIdx.x, blocks_x);
  else run_tiles<kDw, TP, TQ, SP, SQ, 0>(w, smem, (int)blockIdx.x - blocks_x, (int)gridDim.x - blocks_x);
}

#ifdef __HIP_DEVICE_COMPILE__
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_at(const char* base) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, kOutside, 0x00020000);
}
__device__ __forceinline__ bf16x8_t load_at(__amdgpu_buffer_rsrc_t r, uint32_t offset, int from) {
  return __builtin_bit_cast(bf16x8_t, __builtin_amdgcn_raw_buffer_load_b128(r, offset, from, 0));
}
#endif

// A few rows, TB blocks of 16: the weights are read once, and that is all the time goes to.  A block takes 16 features of both
// projections; its four waves take the 64 k pieces of their rows in turn, straight into registers, so that 512 consecutive
// bytes of a row are asked for at once and no wave waits for another before the sums meet in LDS.  All of x is read by every
// block, from L2.
// 1 row of d 4096, F 12288: 34.2 to 34.5 us, the weights at 5.8 to 5.9 TB/s, as well with those of 24 layers in turn (4.8 GB, so
// that no cache holds them) as with one layer's; of 1024 x 4096, 32 rows 6.4 us and 64 rows 8.2, where tiles take 9.5.
// 32 features a block were slower throughout (1 row 48 us), fewer pieces under way at one row (2: 41 us).
constexpr int kFewThreads = 256;

template <int ACT, int TB>
__global__ __launch_bounds__(kFewThreads) void ffn_few_kernel(const GemmArgs a) {
#ifdef __HIP_DEVICE_COMPILE__
  constexpr int kDeep = 4;   // pieces under way
  __shared__ f32x4_t sums[4][2 * TB][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int f0 = (int)blockIdx.x * 16;
  const int row = lane & 15, part = (lane >> 4) * 8;
  const int d = (int)a.depth;
  // A lane's fragments of a piece: k = 32 h + part .. + 7 of its row, h = 0, 1.  What lies past the end of the rows or of K
  // is asked for outside the buffers and comes as zeros.
  const __amdgpu_buffer_rsrc_t gate = buffer_at(a.p0 + (int64_t)f0 * a.ld_p), up = buffer_at(a.p1 + (int64_t)f0 * a.ld_p);
  const __amdgpu_buffer_rsrc_t x = buffer_at(a.q);
  const uint32_t at_f = f0 + row < a.rows_p ? (uint32_t)(row * a.ld_p) + part * 2 : kOutside;
  uint32_t at_x[TB];
#pragma unroll
  for (int i = 0; i < TB; ++i) at_x[i] = 16 * i + row < a.rows_q ? (uint32_t)((16 * i + row) * a.ld_q) + part * 2 : kOutside;
  struct Piece { bf16x8_t g[2], u[2], x[2][TB]; };
  f32x4_t acc_g[TB], acc_u[TB];
#pragma unroll
  for (int t = 0; t < TB; ++t) acc_g[t] = acc_u[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  // Blocks begin at different places of K: side by side they would all ask for the same lines of x, and, rows lying a power of
  // two apart, for the same channels.
  const int rounds = (d + 4 * kStepK * kDeep - 1) / (4 * kStepK * kDeep);
  int turn = (int)blockIdx.x % rounds;
  for (int r = 0; r < rounds; ++r) {
    const int k0 = (turn * 4 * kDeep + wave) * kStepK;
    turn = turn + 1 == rounds ? 0 : turn + 1;
    Piece p[kDeep];
#pragma unroll
    for (int i = 0; i < kDeep; ++i) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = k0 + i * 4 * kStepK + 32 * h;
        const uint32_t past = k + part < d ? 0 : kOutside;
        p[i].g[h] = load_at(gate, at_f | past, k * 2);
        p[i].u[h] = load_at(up, at_f | past, k * 2);
#pragma unroll
        for (int t = 0; t < TB; ++t) p[i].x[h][t] = load_at(x, at_x[t] | past, k * 2);
      }
    }
    __builtin_amdgcn_sched_barrier(0);   // all of them under way: left to itself the compiler saves registers instead
#pragma unroll
    for (int i = 0; i < kDeep; ++i) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int t = 0; t < TB; ++t) {
          acc_g[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(p[i].g[h], p[i].x[h][t], acc_g[t], 0, 0, 0);
          acc_u[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(p[i].u[h], p[i].x[h][t], acc_u[t], 0, 0, 0);
        }
      }
    }
  }
#pragma unroll
  for (int t = 0; t < TB; ++t) {
    sums[wave][2 * t][lane] = acc_g[t];
    sums[wave][2 * t + 1][lane] = acc_u[t];
  }
  __syncthreads();
  const int f = f0 + 4 * (lane >> 4), q = 16 * wave + row;   // a wave, a block of rows
  if (wave >= TB || q >= a.rows_q || f >= a.rows_p) return;
  f32x4_t g = sums[0][2 * wave][lane], u = sums[0][2 * wave + 1][lane];
#pragma unroll
  for (int w = 1; w < 4; ++w) {
    g += sums[w][2 * wave][lane];
    u += sums[w][2 * wave + 1][lane];
  }
  bf16x4_t o;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    float act, slope;
    activate<ACT>(g[r], act, slope);
    o[r] = (__bf16)(act * u[r]);
  }
  *reinterpret_cast<bf16x4_t*>(a.out0 + q * a.ld_out0 + (int64_t)f * 2) = o;
#endif
}

// Adds the parts of dx in their order and rounds once.  Bound by its reads: six parts of 1237 x 1024 in 6 us, 5.4 TB/s; for few rows
// by their latency, so that eight parts are asked for at once: 32 parts of 1 x 512 in 3.8 us, one after another 9.4.
__global__ __launch_bounds__(256) void ffn_join_kernel(const float* __restrict__ partials, int splits, int64_t T, int d,
                                                       __bf16* __restrict__ dx, int64_t ld) {
  constexpr int kAtOnce = 8;
  const int per_row = d / 8;
  const int64_t all = T * per_row;
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < all; e += (int64_t)gridDim.x * 256) {
    const int64_t t = e / per_row;
    const int c = (int)(e - t * per_row) * 8;
    float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < splits; k += kAtOnce) {
      float v[kAtOnce][8];
#pragma unroll
      for (int n = 0; n < kAtOnce; ++n) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[n][i] = 0.f;
        if (k + n < splits) load8(partials + ((int64_t)(k + n) * T + t) * d + c, v[n]);
      }
      __builtin_amdgcn_sched_barrier(0);    // all of them under way
#pragma unroll
      for (int n = 0; n < kAtOnce; ++n) {
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] += v[n][i];
      }
    }
    store8(dx + t * ld + c, s);
  }
}

template <int MODE, int TILE, int SP, int SQ, int ACT>
int launch_tiles(GemmArgs a, hipStream_t stream) {
  const TileGrid g = tile_grid(MODE, TILE, a.rows_p, a.rows_q, a.splits);
  a.tiles_p = g.p;
  a.tiles_q = g.q;
  return launch_kernel(ffn_gemm_kernel<MODE, kTiles[TILE].p, kTiles[TILE].q, SP, SQ, ACT>, dim3((unsigned)g.blocks),
                       dim3(kThreads), stream, a);
}

template <int TILE, int SP, int SQ>
int launch_together(GemmArgs x, GemmArgs w, hipStream_t stream) {
  const TileGrid gx = tile_grid(kDx, TILE, x.rows_p, x.rows_q, x.splits), gw = tile_grid(kDw, TILE, w.rows_p, w.rows_q, 1);
  x.tiles_p = w.tiles_p = gx.p;
  x.tiles_q = gx.q;
  w.tiles_q = gw.q;
  const int blocks_x = (int)tiles(gx.n, kXcds) * kXcds;
  return launch_kernel(ffn_gradients_kernel<kTiles[TILE].p, kTiles[TILE].q, SP, SQ>, dim3((unsigned)(blocks_x + gw.n)),
                       dim3(kThreads), stream, x, w, blocks_x);
}

template <int MODE, int ACT>
int launch_gemm(const GemmArgs& a, hipStream_t stream) {
  const int tile = choose_tile(MODE, a.rows_p, a.rows_q, (MODE == kDx ? 2 : 1) * tiles(a.depth, kStepK), a.splits).tile;
  switch (tile) {
    case 0: return launch_tiles<MODE, 0, 3, 2, ACT>(a, stream);
    case 1: return launch_tiles<MODE, 1, 3, 3, ACT>(a, stream);
    case 2: return launch_tiles<MODE, 2, 3, 3, ACT>(a, stream);
    case 3: return launch_tiles<MODE, 3, 4, 4, ACT>(a, stream);
    case 4: return launch_tiles<MODE, 4, 4, 4, ACT>(a, stream);
    case 5: return launch_tiles<MODE, 5, 3, 3, ACT>(a, stream);
    case 6: return launch_tiles<MODE, 6, 6, 6, ACT>(a, stream);
  }
  if constexpr (gated_mode(MODE)) {
    switch (tile) {
      case 7: return launch_tiles<MODE, 7, 5, 5, ACT>(a, stream);
      case 8: return launch_tiles<MODE, 8, 4, 4, ACT>(a, stream);
      case 9: return launch_tiles<MODE, 9, 3, 2, ACT>(a, stream);
    }
  }
  return -1;
}

template <int ACT, int TB>
int launch_few_as(const GemmArgs& a, hipStream_t stream) {
  return launch_kernel(ffn_few_kernel<ACT, TB>, dim3((unsigned)tiles(a.rows_p, 16)), dim3(kFewThreads), stream, a);
}
template <int ACT>
int launch_few(const GemmArgs& a, hipStream_t stream) {
  switch (tiles(a.rows_q, 16)) {
    case 1: return launch_few_as<ACT, 1>(a, stream);
    case 2: return launch_few_as<ACT, 2>(a, stream);
    case 3: return launch_few_as<ACT, 3>(a, stream);
    default: return launch_few_as<ACT, 4>(a, stream);
  }
}
template <int MODE>
int launch_gated(const GemmArgs& a, int activation, hipStream_t stream) {
  return activation == MOSAIC_SILU ? launch_gemm<MODE, MOSAIC_SILU>(a, stream)
                                   : launch_gemm<MODE, MOSAIC_GELU_TANH>(a, stream);
}

}  // namespace

// Rows of dg | du with their low halves, and of 32-bit partial sums that dx may take, for up to T rows: no less for more rows, so
// that a workspace serves fewer too.
int64_t ffn_gradient_rows(int64_t T) {
  const int64_t halves = 2 * (T < kHalvesRows ? T : kHalvesRows);
  return T > halves ? T : halves;
}
int64_t ffn_partial_rows(int64_t T) {
  const int64_t halves = 2 * kMostParts * (T < kHalvesRows ? T : kHalvesRows), whole = T * kMostParts < kPartRows ? T * kMostParts : kPartRows;
  return whole > halves ? whole : halves;
}

int launch_gated_ffn_forward(const FfnForwardArgs& f, hipStream_t stream) {
  GemmArgs a = {};
  a.p0 = static_cast<const char*>(f.w_gate);
  a.p1 = static_cast<const char*>(f.w_up);
  a.ld_p = f.ld_w * 2;
  a.ld_q = f.ld_x * 2;
  a.rows_p = f.F;
  a.depth = f.d;
  a.splits = 1;
  a.F = f.F;
  a.ld_out0 = f.ld_out * 2;
  for (int64_t t = 0; t < f.T; t += kLaunchRows) {
    a.rows_q = f.T - t < kLaunchRows ? f.T - t : kLaunchRows;
    a.q = static_cast<const char*>(f.x) + t * a.ld_q;
    a.out0 = static_cast<char*>(f.out) + t * a.ld_out0;
    const int rc = !few_rows(f.T, f.F) ? launch_gated<kForward>(a, f.activation, stream)
                   : f.activation == MOSAIC_SILU ? launch_few<MOSAIC_SILU>(a, stream) : launch_few<MOSAIC_GELU_TANH>(a, stream);
    if (rc != 0) return -1;
  }
  return 0;
}

int64_t most_part_rows(int64_t rows) {
  const int64_t parts = rows * kMostParts < kPartRows ? rows * kMostParts : kPartRows;
  return parts > rows ? parts : rows;
}
ProductPlan plan_row_product(int64_t rows, int32_t cols, int64_t depth) {
  const int64_t steps = tiles(depth, kStepK);
  ProductPlan best = {1, 0.0};
  for (int32_t s = 1; s == 1 || (s <= kMostParts && s * rows <= kPartRows && s * 4 <= steps); ++s) {
    const double us = choose_tile(kOneDx, cols, rows, steps, s).us + (double)(rows * cols) * 8.0 * s / kJoinBytesPerUs;
    if (s == 1 || us < best.us) best = {s, us};
  }
  return best;
}

namespace {
GemmArgs product_args(const ProductArgs& f) {
  GemmArgs a = {};
  a.p0 = a.p1 = static_cast<const char*>(f.p);
  a.q = static_cast<const char*>(f.q);
  a.ld_p = f.ld_p * 2;
  a.ld_q = f.ld_q * 2;
  a.rows_q = f.rows;
  a.rows_p = f.cols;
  a.depth = f.depth;
  a.splits = f.splits;
  a.f32 = f.f32;
  a.accumulate = f.accumulate;
  a.out0 = static_cast<char*>(f.out);
  a.ld_out0 = f.ld_out * (f.f32 ? 4 : 2);
  a.slot = f.slot;
  a.extra = f.extra;
  a.ld_extra = f.ld_extra;
  return a;
}
}  // namespace

int launch_row_product(const ProductArgs& f, hipStream_t stream) {
  GemmArgs a = product_args(f);
  for (int64_t t = 0; t < f.rows; t += kLaunchRows) {   // (parts only where all rows are in one launch)
    a.rows_q = f.rows - t < kLaunchRows ? f.rows - t : kLaunchRows;
    a.q = static_cast<const char*>(f.q) + t * a.ld_q;
    a.out0 = static_cast<char*>(f.out) + t * a.ld_out0;
    if (launch_gemm<kOneDx, 0>(a, stream) != 0) return -1;
  }
  return 0;
}

int launch_column_product(const ProductArgs& f, hipStream_t stream) { return launch_gemm<kOneDw, 0>(product_args(f), stream); }

int launch_gated_ffn_backward(const FfnBackwardArgs& f, hipStream_t stream) {
  const int64_t ld_grads = (int64_t)f.F * 4;
  const bool halves = with_low_halves(f.T);
  const int64_t rows = halves ? 2 * f.T : f.T;   // of dg | du
  for (int64_t t = 0; t < f.T; t += kLaunchRows) {
    GemmArgs a = {};
    a.p0 = static_cast<const char*>(f.w_gate);
    a.p1 = static_cast<const char*>(f.w_up);
    a.ld_p = f.ld_w * 2;
    a.ld_q = f.ld_x * 2;
    a.rows_q = f.T - t < kLaunchRows ? f.T - t : kLaunchRows;
    a.q = static_cast<const char*>(f.x) + t * a.ld_q;
    a.rows_p = f.F;
    a.depth = f.d;
    a.splits = 1;
    a.F = f.F;
    a.ld_dout = f.ld_dout * 2;
    a.dout = static_cast<const char*>(f.dout) + t * a.ld_dout;
    a.ld_out0 = f.ld_out * 2;
    a.out0 = f.out == nullptr ? nullptr : static_cast<char*>(f.out) + t * a.ld_out0;
    a.ld_out1 = ld_grads;
    a.out1 = static_cast<char*>(f.grads) + t * ld_grads;
    a.low = halves ? f.T * ld_grads : 0;
    if (launch_gated<kRecompute>(a, f.activation, stream) != 0) return -1;
  }
  const GradientPlan plan = plan_gradients(f.T, f.d, f.F);
  GemmArgs x = {};
  x.p0 = static_cast<const char*>(f.w_gate);
  x.p1 = static_cast<const char*>(f.w_up);
  x.ld_p = f.ld_w * 2;
  x.ld_q = ld_grads;
  x.rows_p = f.d;
  x.depth = f.F;
  x.splits = plan.splits;
  const int parts = (int)plan.splits * (halves ? 2 : 1);   // of dx, added by the join: of every part of K the rows, then their low halves
  x.f32 = parts > 1;            // then all rows are in one launch
  x.ld_out0 = x.f32 ? (int64_t)f.d * 4 : f.ld_dx * 2;
  GemmArgs w = {};
  w.p0 = w.p1 = static_cast<const char*>(f.x);
  w.q = static_cast<const char*>(f.grads);
  w.ld_p = f.ld_x * 2;
  w.ld_q = ld_grads;
  w.rows_q = 2 * (int64_t)f.F;
  w.rows_p = f.d;
  w.depth = rows;
  w.repeat = halves ? (int32_t)f.T : 0;
  w.splits = 1;
  w.F = f.F;
  w.f32 = f.dw_f32;
  w.accumulate = f.accumulate;
  w.out0 = static_cast<char*>(f.dw_gate);
  w.out1 = static_cast<char*>(f.dw_up);
  w.ld_out0 = f.ld_dw * (f.dw_f32 ? 4 : 2);
  const bool together = plan.tile >= 0 && f.dx != nullptr && f.dw_gate != nullptr;
  for (int64_t t = 0; f.dx != nullptr && t < rows; t += kLaunchRows) {
    x.rows_q = rows - t < kLaunchRows ? rows - t : kLaunchRows;
    x.q = static_cast<const char*>(f.grads) + t * ld_grads;
    x.out0 = x.f32 ? reinterpret_cast<char*>(f.partials) : static_cast<char*>(f.dx) + t * x.ld_out0;
    const int rc = !together ? launch_gemm<kDx, 0>(x, stream)
                   : plan.tile == 0 ? launch_together<0, 3, 2>(x, w, stream)
                   : plan.tile == 1 ? launch_together<1, 3, 3>(x, w, stream)
                                    : launch_together<3, 4, 4>(x, w, stream);
    if (rc != 0) return -1;
  }
  if (f.dx != nullptr && parts > 1) {
    const int64_t blocks = tiles(f.T * (f.d / 8), 256);
    if (launch_kernel(ffn_join_kernel, dim3((unsigned)(blocks > 65536 ? 65536 : blocks)), dim3(256), stream, f.partials,
                      parts, f.T, f.d, static_cast<__bf16*>(f.dx), f.ld_dx) != 0)
      return -1;
  }
  if (f.dw_gate != nullptr && !together && launch_gemm<kDw, 0>(w, stream) != 0) return -1;
  return 0;
}

}  // namespace mosaic
