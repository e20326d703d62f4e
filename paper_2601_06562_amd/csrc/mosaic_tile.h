// What tiles on the matrix cores are built from: copies of operands into LDS, reads of fragments, and the order of results in
// the lanes.  Device code, for blocks of 8 waves.
#ifndef MOSAIC_TILE_H_
#define MOSAIC_TILE_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mosaic_layer_internal.h"

namespace mosaic {
namespace tile {

constexpr int kTileK = 64;   // K goes in steps of 64
typedef __attribute__((address_space(3))) void* lds_ptr_t;
typedef __attribute__((address_space(3))) bf16x4_t* lds_bf16x4_ptr_t;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;
typedef const __attribute__((address_space(3))) bf16x8_t* lds_bf16x8_ptr_t;

constexpr int kThreads = 512;   // 8 waves: 2 along P, 4 along Q
constexpr uint32_t kOutside = 0x80000000u;   // a buffer offset past every range here: such a lane's copy brings zeros
constexpr int kXcds = 8;

// Copies of one operand's K-step into LDS, 16 bytes a lane, through a buffer descriptor whose base moves with the step.
// Along K (rows of 64 consecutive k, 128 bytes): the eight 16-byte pieces of a row lie at piece ^ (row / 2 % 8), so that the
// 16 rows of a fragment read spread over the banks.
// Across K (KROW; rows of one k, ROWS consecutive columns): the 32-byte pieces (16 columns) of a row lie at piece ^ turn(k)
// for the transposing reads, of which 32 lanes take 8 k at once.
template <int ROWS, bool KROW>
struct Copier {
  static constexpr int kCopies = ROWS * 128 / (kThreads * 16);   // a wave and step
  uint32_t offset[kCopies];   // of this lane's piece within the step, or kOutside for one past the end

  static __device__ __forceinline__ int turn(int k) {
    if (ROWS >= 128) return (k & 3) | (k >> 3 & 1) << 2;
    return (k >> 1 & 1) | (k >> 3 & 1) << 1;   // rows of 128 bytes: two of them span the banks
  }

  // `valid`: rows there are; `left`: k there are, where rows lie along K (across K the descriptor's end cuts them).
  // `repeat`: across K, rows there are that come a second time behind themselves, or 0.
  __device__ __forceinline__ void place(int wave, int lane, int64_t ld, int64_t valid, int left, int repeat = 0) {
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      const int byte = (wave * kCopies + i) * 1024 + lane * 16;
      if constexpr (KROW) {
        const int k = byte / (ROWS * 2), piece = byte % (ROWS * 2) / 16;
        const int col = ((piece >> 1) ^ turn(k)) * 16 + (piece & 1) * 8;
        const int from = repeat != 0 && k >= repeat ? k - repeat : k;
        offset[i] = col < valid ? (uint32_t)(from * (uint32_t)ld + col * 2) : kOutside;
      } else {
        const int row = byte / 128, piece = byte % 128 / 16;
        const int k = (piece ^ (row >> 1 & 7)) * 8;
        offset[i] = row < valid && k < left ? (uint32_t)(row * (uint32_t)ld + k * 2) : kOutside;
      }
    }
  }

  // Copy i of the step that `r` begins at, to the operand's LDS address `to`.  Written as a statement because the compiler,
  // which cannot tell the slots apart, puts a wait for all copies under way ahead of every transposing read that follows a
  // copy it knows of.
  __device__ __forceinline__ void one(int i, u32x4_t r, uint32_t to, int wave) const {
    const uint32_t m0 = __builtin_amdgcn_readfirstlane((int)(to + (wave * kCopies + i) * 1024));
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 ::"s"(m0), "v"(offset[i]), "s"(r));   // nothing else in these kernels uses M0
  }
};

// Descriptor of `bytes` bytes from `base` on.
__device__ __forceinline__ u32x4_t buffer_from(const char* base, uint32_t bytes) {
  const uint64_t b = reinterpret_cast<uint64_t>(base);
  return u32x4_t{(uint32_t)__builtin_amdgcn_readfirstlane((int)b), (uint32_t)__builtin_amdgcn_readfirstlane((int)(b >> 32) & 0xffff),
                 (uint32_t)__builtin_amdgcn_readfirstlane((int)bytes), 0x00020000u};
}

// Reads of an operand's fragments: 16 rows, k = 32 kk + 8 (lane / 16) .. + 7.  A lane's addresses differ between blocks, halves
// and the two reads of a transposed fragment by constants that go into the instruction (and, across K, by one xor a block).
template <int ROWS, bool KROW>
struct Reader {
  uint32_t at[KROW ? 1 : 2];   // LDS address of block 0; along K: of each half

  __device__ __forceinline__ void place(uint32_t lds, int row, int lane) {   // row: a multiple of 16, across K of 128 or ROWS / 4
    const int g = lane >> 4, i = lane & 15;
    if constexpr (KROW) {
      const int k = 8 * g + (i >> 2);
      at[0] = lds + k * (ROWS * 2) + ((row >> 4) ^ Copier<ROWS, true>::turn(k)) * 32 + (i & 3) * 8;
    } else {
      at[0] = lds + (row + i) * 128 + ((g ^ (i >> 1)) * 16);
      at[1] = lds + (row + i) * 128 + (((4 + g) ^ (i >> 1)) * 16);
    }
  }
  __device__ __forceinline__ void move(int bytes) {   // to the other slot, a multiple of 1024 bytes on or back
    at[0] += bytes;
    if constexpr (!KROW) at[1] += bytes;
  }
  // Block `block` rows of 16 on; across K it is below the power of two that the first row is a multiple of.
  __device__ __forceinline__ bf16x8_t get(int block, int kk) const {
    if constexpr (KROW) {
      const uint32_t from = (at[0] ^ (block * 32)) + kk * 32 * (ROWS * 2);
      const bf16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_ptr_t)(uintptr_t)from);
      const bf16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_ptr_t)(uintptr_t)(from + 4 * ROWS * 2));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      return *(lds_bf16x8_ptr_t)(uintptr_t)(at[kk] + block * 2048);
    }
  }
};

// The four lanes that hold one Q row (16 apart) each have 4 consecutive P rows of every block; afterwards each has 4 NB
// consecutive ones, NB = 2 or 4 blocks, in order: what is stored, or was loaded, is 16 bytes a lane.  `scatter` takes
// gathered quads back.  Three blocks stay as they are, 8 bytes a lane.
typedef uint32_t Quad[2];   // four bf16
__device__ __forceinline__ void swap32(Quad& a, Quad& b) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const auto r = __builtin_amdgcn_permlane32_swap(a[h], b[h], false, false);
    a[h] = r[0];
    b[h] = r[1];
  }
}
__device__ __forceinline__ void swap16(Quad& a, Quad& b) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const auto r = __builtin_amdgcn_permlane16_swap(a[h], b[h], false, false);
    a[h] = r[0];
    b[h] = r[1];
  }
}
template <int NB>
__device__ __forceinline__ int first_of(int lane) { return (NB == 3 ? 4 : 4 * NB) * (lane >> 4); }   // a lane's first P row
template <int NB>
__device__ __forceinline__ void gather(Quad (&w)[NB]) {
  if constexpr (NB == 3) return;
  if constexpr (NB == 4) { swap32(w[0], w[2]); swap32(w[1], w[3]); swap16(w[2], w[3]); }
  else swap32(w[0], w[1]);
  swap16(w[0], w[1]);
}
template <int NB>
__device__ __forceinline__ void scatter(Quad (&w)[NB]) {
  if constexpr (NB == 3) return;
  swap16(w[0], w[1]);
  if constexpr (NB == 4) { swap16(w[2], w[3]); swap32(w[1], w[3]); swap32(w[0], w[2]); }
  else swap32(w[0], w[1]);
}
// Gathered quads to or from `row`, whose element `c` is the first of this lane's; `end`: elements there are, a multiple of 8.
template <int NB>
__device__ __forceinline__ void store_quads(char* row, int c, int end, const Quad (&w)[NB]) {
  if constexpr (NB == 3) {
#pragma unroll
    for (int i = 0; i < NB; ++i)
      if (c + 16 * i < end) *reinterpret_cast<uint2*>(row + (int64_t)(c + 16 * i) * 2) = uint2{w[i][0], w[i][1]};
    return;
  }
#pragma unroll
  for (int i = 0; i + 1 < NB; i += 2)
    if (c + 4 * i < end) *reinterpret_cast<u32x4_t*>(row + (int64_t)(c + 4 * i) * 2) = u32x4_t{w[i][0], w[i][1], w[i + 1][0], w[i + 1][1]};
}
template <int NB>
__device__ __forceinline__ void load_quads(const char* row, int c, int end, bool in, Quad (&w)[NB]) {
  if constexpr (NB == 3) {
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      uint2 v = {0u, 0u};
      if (in && c + 16 * i < end) v = *reinterpret_cast<const uint2*>(row + (int64_t)(c + 16 * i) * 2);
      w[i][0] = v.x; w[i][1] = v.y;
    }
    return;
  }
#pragma unroll
  for (int i = 0; i + 1 < NB; i += 2) {
    u32x4_t v = {0u, 0u, 0u, 0u};
    if (in && c + 4 * i < end) v = *reinterpret_cast<const u32x4_t*>(row + (int64_t)(c + 4 * i) * 2);
    w[i][0] = v[0]; w[i][1] = v[1]; w[i + 1][0] = v[2]; w[i + 1][1] = v[3];
  }
}
__device__ __forceinline__ void pack(Quad& w, const float (&v)[4]) {
  const bf16x4_t b = {(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
  const uint2 u = __builtin_bit_cast(uint2, b);
  w[0] = u.x;
  w[1] = u.y;
}
// What the rounding to `high` left of v, rounded in turn; zero beside what is no finite number.
__device__ __forceinline__ void pack_low(Quad& w, const Quad& high, const float (&v)[4]) {
  const bf16x4_t h = __builtin_bit_cast(bf16x4_t, uint2{high[0], high[1]});
  float low[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const float l = v[r] - (float)h[r];
    low[r] = __builtin_fabsf(l) < __builtin_inff() ? l : 0.f;
  }
  pack(w, low);
}

// LDS of a tile: a ring of SP slots for P, of SQ for Q.
constexpr int ring_bytes(int TP, int TQ, int SP, int SQ) { return (SP * TP + SQ * TQ) * kTileK * 2; }

}  // namespace tile
}  // namespace mosaic
#endif
