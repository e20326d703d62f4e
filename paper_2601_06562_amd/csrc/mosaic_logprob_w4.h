// Log probabilities of given tokens, and gradients at their logits, on the hand-scheduled K-loop of the mask-only pass
// (gen_w4_loop.py): four waves, one a SIMD, 128 ids by 16 NB rows each, whose logits stay in the accumulators until they are read, a
// column of 16 rows at a time.  Row tiles of 32 NB rows and parts of the vocabulary are chosen on the device from the rows found
// (mosaic_schedule.h), as there.
//
// Bound by the power of the matrix cores for many rows, by memory for few: 126464 x 4096, 4096 rows 2.61 to 2.81 ms (1.51 to 1.63
// PFLOP/s; the mask-only pass, which keeps no entropy, 2.55 to 2.59 beside it), with eight alternatives 4 to 5% more, one row 167 us
// (6.2 TB/s); gradients at the logits, 2048 rows by 63232 ids, 764 us (1.39 PFLOP/s).  Alternatives cost small tiles of work most (900
// rows of 32000 x 1024: 64 us, with five 117): a unit's first tiles bring the most candidates, and code that runs once a unit is
// fetched anew.  They are sorted in after 1, 2, 4, 8, ... tiles (every other schedule tried 2 to 8% slower at 4096 rows).
//
// It takes d that is a multiple of 64 and whole tiles of 256 ids, or a last tile over the vocabulary's last 256 ids, of which
// those of the tile before it are not counted again; mosaic_logprob.hip has the kernel for the rest.  Each of the four kernels is
// compiled by itself (mosaic_logprob_w4_*.hip), since one takes about a minute.
#ifndef MOSAIC_LOGPROB_W4_H_
#define MOSAIC_LOGPROB_W4_H_

#include <hip/hip_runtime.h>
#include <limits.h>
#include <stdint.h>

#include "mosaic_logprob_rows.h"

namespace mosaic {
namespace {

using namespace logprob;

typedef __attribute__((ext_vector_type(32))) float f32x32_t;
typedef const __attribute__((address_space(1))) void* gbl_ptr_t;

constexpr int kW4Threads = 256;
constexpr int64_t kStreamBytes = (int64_t)288 << 20;   // as the mask-only pass: a larger LM head passes the memory-side cache by
constexpr int kRowBytes = 128;
constexpr int kLmHeadSlot = 256 * kRowBytes;
constexpr int kLdsBytes = 160 * 1024;
#include "mosaic_w4_pieces.inc"

template <int N>
__device__ __forceinline__ void wait_vm() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ const char* scalar_pointer(const char* x) {
  const uint64_t a = (uint64_t)x;
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)a), hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32));
  return (const char*)((uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ uint32_t local_offset(uint32_t x) {
  asm volatile("" : "+v"(x));
  return x;
}

// The units of this workgroup.  `rows`: to be tiled; `found`: listed.
template <int MODE, int NB, bool STREAM>
__device__ __forceinline__ void w4_units(const LogitParams& p, const Schedule& sched, int rows, int found, int first, char* smem) {
  constexpr int kDepth = NB <= 2 ? 3 : 2;            // K-tiles under way, as the generator's depth()
  constexpr bool kPairs = NB >= kW4PairsFrom;        // the K-loop in pair order
  constexpr int kLatePieces = w4_late_pieces(NB);    // of eight LM-head copies, those a step issues behind its sync
  constexpr int NW = kDepth + 1, NH = kDepth;
  constexpr int kHiddenSlot = 32 * NB * kRowBytes;
  constexpr int kTokens = 32 * NB;
  constexpr int kAuxW = STREAM ? 2 : 0;              // the nt bit of the LM head's copies
  static_assert(NW * kLmHeadSlot + NH * kHiddenSlot <= kLdsBytes, "rings");

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wv = wave & 1;   // vocabulary half of the tile
  const int wt = wave >> 1;  // row half of the tile
  const bool odd_wave = (__builtin_amdgcn_readfirstlane(wave) & 1) != 0;
  const int l16 = lane & 15, q = lane >> 4;
  const int n_tt = sched.row_tiles, G = (int)p.sched.grid, S = sched.splits, n_units = n_tt * S;
  const int A = (int)panel_depth((uint32_t)n_tt, NB, 8);
  const int full_panel_units = A * S, n_panels = (n_tt + A - 1) / A;

  // Direct-to-LDS copy: instruction i of this wave fills rows first + 8 i + lane / 8 of the tile, first = 64 wave for the LM
  // head (i = 0..7), 8 NB wave for the hidden rows (i = 0..NB-1); 16-byte chunks are swizzled by row.
  const int sub = lane >> 3;
  auto chunk_of = [&](int row) { return (uint32_t)(((lane & 7) ^ ((row >> 1) & 7)) * 16); };
  const int nk = p.d / kTileK;
  const uint32_t w_row_bytes = (uint32_t)p.ld_w;
  uint32_t rdw[2], rdh[2], wlane[2];
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) {
    const uint32_t o = (uint32_t)(l16 * kRowBytes + (((4 * ks + q) ^ ((l16 >> 1) & 7)) * 16));
    rdw[ks] = o + (uint32_t)(wv * 128 * kRowBytes);
    rdh[ks] = o + (uint32_t)(NW * kLmHeadSlot + wt * (kTokens / 2) * kRowBytes);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) wlane[i] = (uint32_t)(wave * 64 + sub) * w_row_bytes + chunk_of(wave * 64 + 8 * i + sub);

  const uint32_t u_nk = (uint32_t)nk;
  const uint32_t u_wwrap = 256u * w_row_bytes - (uint32_t)(nk - 1) * 128u;
  const int ragged_rows = p.V % kVocab, ragged_tile = ragged_rows != 0 ? p.V / kVocab : -1;
  const uint32_t u_wwrap_ragged = (uint32_t)ragged_rows * w_row_bytes - (uint32_t)(nk - 1) * 128u;
  auto first_id = [&](int vt) { return vt == ragged_tile ? p.V - kVocab : vt * kVocab; };
  const uint32_t u_hwrap = (uint32_t)(nk - 1) * 128u;
  const uint32_t w_dst = (uint32_t)wave * 64u * kRowBytes, h_dst = (uint32_t)(wave * 8 * NB) * kRowBytes;

  Entry* const lists =
      MODE != kAlternatives ? nullptr : p.lists + ((int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(wave)) * (64 * NB) * kListRoom;

  for (int u = first; u < n_units; u += G) {
    int pnl = u / full_panel_units;
    if (pnl >= n_panels) pnl = n_panels - 1;
    const int ul = u - pnl * full_panel_units;
    const int hp = (n_tt - pnl * A) < A ? (n_tt - pnl * A) : A;
    const int sp = ul / hp;
    const int tt = pnl * A + ul % hp;
    const int vt0 = (int)(((int64_t)sp * p.sched.vocab_tiles) / S);
    const int vt1 = (int)(((int64_t)(sp + 1) * p.sched.vocab_tiles) / S);
    const int ntile = vt1 - vt0;
    const int total_steps = ntile * nk;
    const uint32_t u_total = (uint32_t)total_steps;

    // row tiles that share an LM-head tile copy its pieces in orders of their own, but for the widest
    const int turn = NB < 8 ? (tt & 1) * 4 + (tt & 2) : 0;
    uint32_t woff[8];
    auto w_source = [&](int gw) {   // past the end: the last one
      const int g = gw < total_steps ? gw : total_steps - 1;
      return p.w + (int64_t)first_id(vt0 + g / nk) * (int64_t)w_row_bytes + (g % nk) * kRowBytes;
    };
    auto copy_w = [&](int gw, int pieces = 8) {
      const char* src = scalar_pointer(w_source(gw));
      char* dst = smem + (gw % NW) * kLmHeadSlot + w_dst;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < pieces) __builtin_amdgcn_global_load_lds((gbl_ptr_t)(src + local_offset(woff[i])), (lds_ptr_t)(dst + (i ^ turn) * 1024), 16, 0, kAuxW);
    };
    wait_vm<0>();
    const int first_row = tt * kTokens + wt * (kTokens / 2);   // this wave's rows
    int trow[NB];
    [[maybe_unused]] int target[Rows<NB>::kOwn];
    if constexpr (!gradient_mode(MODE)) {
#pragma unroll
      for (int k = 0; k < Rows<NB>::kOwn; ++k) {
        const int row = first_row + 16 * (4 * k + q) + l16;
        target[k] = 4 * k + q < NB && p.targets != nullptr && row < rows ? in_memory(p.targets)[row] : -1;
      }
    }
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      int j = tt * kTokens + wave * 8 * NB + 8 * i + sub;
      if (j > rows - 1) j = rows - 1;
      trow[i] = p.idx != nullptr ? in_memory(p.idx)[j] : j;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) woff[i] = wlane[i & 1] + (uint32_t)(8 * (i ^ turn)) * w_row_bytes;
    copy_w(0);

    // Gather: 32-bit byte offsets of the NB rows this lane copies, from the lowest of those the wave copies (rows past the end
    // read the last one again; their results are never stored).
    int tmin = INT_MAX;
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      int t = trow[i];
      if (p.idx != nullptr) t = t < 0 ? 0 : (t > p.T - 1 ? p.T - 1 : t);   // a bad entry of a caller's list reads a valid row
      trow[i] = t;
      tmin = t < tmin ? t : tmin;
    }
#pragma unroll
    for (int x = 32; x >= 1; x >>= 1) {
      const int other = __shfl_xor(tmin, x, 64);
      tmin = other < tmin ? other : tmin;
    }
    tmin = __builtin_amdgcn_readfirstlane(tmin);
    const char* hidden_wave = p.x + (int64_t)tmin * p.ld_x;
    uint32_t hoff[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i)
      hoff[i] = (uint32_t)(trow[i] - tmin) * (uint32_t)p.ld_x + chunk_of(wave * 8 * NB + 8 * i + sub);
    auto copy_h = [&](int gh) {
      const char* src = scalar_pointer(hidden_wave + (gh % nk) * kRowBytes);
      char* dst = smem + NW * kLmHeadSlot + (gh % NH) * kHiddenSlot + h_dst;
#pragma unroll
      for (int i = 0; i < NB; ++i)
        __builtin_amdgcn_global_load_lds((gbl_ptr_t)(src + local_offset(hoff[i])), (lds_ptr_t)(dst + i * 1024), 16, 0, 0);
    };
    // What the rings hold.  In pair order the waves that copy a half's vocabulary blocks 4..7 run a K-tile behind the others, and
    // the copies that may be under way at the first sync, the eight youngest, are the LM head's.
    const int lead = kPairs && odd_wave ? NW - 1 : NW;   // K-tiles of the LM head ahead of the step
    copy_h(0);
    if constexpr (kPairs) {
      if (!odd_wave && total_steps > 1) copy_w(1);
      if (total_steps > 1) copy_h(1);
      copy_w(lead - 1, kLatePieces);   // the first step copies the others
      if (total_steps < NW) wait_vm<0>();
      else if (odd_wave) wait_vm<kLatePieces + NB>();
      else wait_vm<kLatePieces + 8 + NB>();
    } else {
#pragma unroll
      for (int g = 1; g < NW; ++g)
        if (g < total_steps) copy_w(g);
#pragma unroll
      for (int g = 1; g < NH; ++g)
        if (g < total_steps) copy_h(g);
      if (total_steps >= NW && total_steps >= NH) wait_vm<8 * (NW - 1) + NB * (NH - 1)>(); else wait_vm<0>();
    }
    __builtin_amdgcn_s_barrier();

    // State of the K-loop: next tiles to copy are W(gw) and H(NH).  Past the end never issued or, in pair order, into slots that
    // nobody reads any more.
    const int gw = kPairs ? lead - 1 : NW, gh = NH;
    const uint64_t wsrc0 = (uint64_t)(kPairs ? w_source(gw) : p.w + (int64_t)first_id(vt0 + gw / nk) * (int64_t)w_row_bytes + (gw % nk) * kRowBytes);
    const uint64_t hsrc0 = (uint64_t)(hidden_wave + (gh % nk) * kRowBytes);
    uint32_t st_wsrc_lo = (uint32_t)wsrc0, st_wsrc_hi = (uint32_t)(wsrc0 >> 32);
    uint32_t st_hsrc_lo = (uint32_t)hsrc0, st_hsrc_hi = (uint32_t)(hsrc0 >> 32);
    uint32_t st_wrd = 0, st_hrd = 0;
    uint32_t st_wdst = (uint32_t)((gw % NW) * kLmHeadSlot) + w_dst + (uint32_t)turn * 1024u;
    uint32_t st_hdst = (uint32_t)((gh % NH) * kHiddenSlot) + h_dst;
    uint32_t st_wk = (uint32_t)((kPairs && gw >= total_steps ? total_steps - 1 : gw) % nk), st_hk = (uint32_t)(gh % nk);
    uint32_t st_g = 0;

    [[maybe_unused]] Rows<NB> st;
    [[maybe_unused]] GradientRows<NB> of;
    if constexpr (gradient_mode(MODE)) of.read(p, first_row, found);
    else st.clear(first_row, rows);
    const int64_t of_half = (int64_t)(2 * sp + wv) * sched.stride;
    auto place = [&](int k, bool& in) __attribute__((always_inline)) {
      const int row = first_row + 16 * (4 * k + q) + l16;
      in = in && row < rows;
      return p.part_top + (of_half + (in ? row : 0)) * p.n_top;
    };

#pragma unroll 1
    for (int n = 0; n < ntile; ++n) {
      f32x32_t acc[NB];
      st_wsrc_lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)st_wsrc_lo);
      st_wsrc_hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)st_wsrc_hi);
      st_hsrc_lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)st_hsrc_lo);
      st_hsrc_hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)st_hsrc_hi);
      st_wrd = (uint32_t)__builtin_amdgcn_readfirstlane((int)st_wrd);
      st_hrd = (uint32_t)__builtin_amdgcn_readfirstlane((int)st_hrd);
      st_wdst = (uint32_t)__builtin_amdgcn_readfirstlane((int)st_wdst);
      st_hdst = (uint32_t)__builtin_amdgcn_readfirstlane((int)st_hdst);
      st_wk = (uint32_t)__builtin_amdgcn_readfirstlane((int)st_wk);
      st_hk = (uint32_t)__builtin_amdgcn_readfirstlane((int)st_hk);
      st_g = (uint32_t)__builtin_amdgcn_readfirstlane((int)st_g);
      {
        const uint32_t st_total = (uint32_t)__builtin_amdgcn_readfirstlane((int)u_total);
        const uint32_t st_nk = (uint32_t)__builtin_amdgcn_readfirstlane((int)u_nk);
        const uint32_t st_wwrap = (uint32_t)__builtin_amdgcn_readfirstlane((int)(vt0 + n + 1 == ragged_tile ? u_wwrap_ragged : u_wwrap));
        const uint32_t st_hwrap = (uint32_t)__builtin_amdgcn_readfirstlane((int)u_hwrap);
        [[maybe_unused]] const uint32_t st_wnext = (uint32_t)__builtin_amdgcn_readfirstlane(lead);
        uint32_t addr_tmp0, addr_tmp1;
        [[maybe_unused]] uint32_t addr_tmp2, addr_tmp3;
#include "mosaic_w4_products.inc"
      }
      auto load = [&](int j, float (&x)[32]) __attribute__((always_inline)) {
#include "mosaic_w4_columns.inc"
      };
      const int64_t v = first_id(vt0 + n) + wv * kHalf;
      if constexpr (gradient_mode(MODE)) {
        gradient_tile<NB, true, MODE == kGradientsLow>(load, of, v, first_row, found);
      } else {
        const int64_t from = vt0 + n == ragged_tile ? (int64_t)ragged_tile * kVocab : 0;
        reduce_tile<NB, true, MODE == kAlternatives, false>(load, st, v + 4 * q, from, p.V, target, first_row, lists, n == 0, sort_now(n + 1, ntile), place);
      }
    }
    if constexpr (!gradient_mode(MODE)) {
#pragma unroll
      for (int k = 0; k < Rows<NB>::kOwn; ++k) {
        const int row = first_row + 16 * (4 * k + q) + l16;
        if (4 * k + q < NB && row < rows) {
          p.part_e[of_half + row] = st.e[k];
          p.part_s[of_half + row] = st.s[k];
          p.part_t[of_half + row] = st.t[k];
        }
      }
    }
    if constexpr (kPairs) wait_vm<0>();   // the copies that the last steps made for nobody
    __syncthreads();                      // every wave is done with the rings
  }
}

template <int MODE, bool STREAM>
__device__ __forceinline__ void w4_units_of(const LogitParams& p, const Schedule& sched, int rows, int found, int first, char* smem) {
  switch (sched.width) {
    case 1: w4_units<MODE, 1, STREAM>(p, sched, rows, found, first, smem); break;
    case 2: w4_units<MODE, 2, STREAM>(p, sched, rows, found, first, smem); break;
    case 3: w4_units<MODE, 3, STREAM>(p, sched, rows, found, first, smem); break;
    case 4: w4_units<MODE, 4, STREAM>(p, sched, rows, found, first, smem); break;
    case 5: w4_units<MODE, 5, STREAM>(p, sched, rows, found, first, smem); break;
    case 6: w4_units<MODE, 6, STREAM>(p, sched, rows, found, first, smem); break;
    case 7: w4_units<MODE, 7, STREAM>(p, sched, rows, found, first, smem); break;
    default: w4_units<MODE, 8, STREAM>(p, sched, rows, found, first, smem); break;
  }
}

template <int MODE>
__global__ __launch_bounds__(kW4Threads) void logprob_kernel_w4(const LogitParams p, int stream_w) {
  __shared__ __attribute__((aligned(1024))) char smem[kLdsBytes];
  const int found = rows_found(p), rows = gradient_mode(MODE) ? p.max_rows : found;
  if (rows <= 0) return;
  const Schedule sched = choose_schedule_wave(p.sched, rows);
  if (!gradient_mode(MODE) && blockIdx.x == 0 && threadIdx.x == 0) {
    p.found[0] = 2 * sched.splits;
    p.found[1] = sched.stride;
  }
  const int units = sched.row_tiles * sched.splits, first = first_unit((int)blockIdx.x, (int)p.sched.grid, units);
  if (first >= units) return;
  if constexpr (!gradient_mode(MODE)) {
    if (stream_w != 0 && sched.row_tiles == 1) {
      w4_units_of<MODE, true>(p, sched, rows, found, first, smem);
      return;
    }
  }
  w4_units_of<MODE, false>(p, sched, rows, found, first, smem);
}

template <int MODE>
int launch(LogitParams p, hipStream_t stream) {
  p.sched.vocab_tiles = (uint32_t)(((int64_t)p.V + kVocab - 1) / kVocab);
  p.sched.k_tiles = (uint32_t)(p.d / kTileK);
  p.sched.widths = 0xff;
  // The mask-only pass's own rule, by its greedy reduction.  Each width forced in turn, 20 to 3000 rows of 8192 x 512, 32000 x 1024, 50257
  // x 704, 65536 x 2048, 126464 x 4096 and 152064 x 3584, 60 sizes: without alternatives its choice is 1.2% off the best width in the
  // mean and at most 13% (40 rows of 65536 x 2048, 57 us for 50); with one 1.9% and 18% (500 of 32000 x 1024, 71 for 60), five 1.8%
  // and 18% (79 for 67), 16 3.8% and 32% (500 of 50257 x 704, 160 for 122): candidates cost a wide tile more than the rule counts.
  p.sched.sampling = 0;
  p.sched.extra = 0;
  p.sched.grid = kCus;
  const int stream_w = (int64_t)p.V * p.d * 2 > kStreamBytes ? 1 : 0;
  return launch_kernel(logprob_kernel_w4<MODE>, dim3(kCus), dim3(kW4Threads), stream, p, stream_w);
}

}  // namespace
}  // namespace mosaic
#endif
