// Device helpers shared by the attention kernels: bf16 tiles in LDS, the two MFMA
// operand forms read from them, and their loads.
#pragma once

#include "common.hpp"

namespace flowmoe {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4i16 lds_v4i16_t;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.69314718055994531f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// the LDS stage of a double-buffered loop as a compile-time constant: the
// loops run their steps in pairs (stage 0, stage 1), so every LDS address of
// a step is a register base plus an immediate offset
template <int S>
struct Stage {
  static constexpr int value = S;
};

__device__ __forceinline__ bf16x8 zero8() { return __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0}); }

__device__ __forceinline__ floatx16 zero16() {
  floatx16 z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.0f;
  return z;
}

// LDS tiles hold rows of D bf16 (2D bytes); the 16-byte chunk c of row r
// sits at chunk c ^ sw(r). For D = 128 (a row is one pass over the 64 banks)
// sw is one-to-one on any 16 consecutive rows, so a row read (16 lanes on 16
// rows, one chunk each) touches 16 distinct bank groups; sw / 2 takes 4
// distinct values of one parity on 4 aligned rows, so a transposing read
// (4 aligned rows x two adjacent 32-byte column pairs per 32 lanes) does too.
// For D = 64 (two rows per pass) the same holds with the row parity as the
// extra bank bit.
template <int D>
__device__ __forceinline__ int sw(int r) {
  if constexpr (D == 128) return 4 * (r & 3) + ((r >> 2) & 3);
  else return 4 * ((r >> 1) & 1) + 2 * ((r >> 2) & 1) + ((r >> 3) & 1);
}
template <int D>
__device__ __forceinline__ int toff(int r, int c) {
  return r * (2 * D) + ((c ^ sw<D>(r)) << 4);
}

// Two MFMA operand forms are read from these tiles:
//   row operand (d contiguous): lane l supplies row r0 + l % 32 of a 32-row
//     block at d = 16 ks + 8 (l / 32) .. + 7, one 16-byte read of chunk
//     2 ks + l / 32 (row_base, frag_row_x);
//   transposed operand: lane l supplies column cb + l % 32 of the tile at
//     the 8 rows of its k-slots, slot 4 i + j (i = 0, 1; j = 0..3) being row
//     rb + 4 (l / 32) + 8 i + j, as two transposing reads (tr_base,
//     frag_tr_x). Each ds_read_b64_tr_b16 hands lane l' of a 16-lane group
//     element l' % 4 of the 4 values that lane 4 q + l' / 4 addressed, in
//     slot q; lanes aimed at rows r0 + s / 4, columns c0 + 4 (s % 4) give
//     lane l' column c0 + l' at rows r0 .. r0 + 3.

// The swizzle lets a lane's fragment addresses be formed from three per-lane
// bases: a row read of row r0 + lq (r0 a multiple of 32) at k step ks is at
// r0 * 2D + (row_base ^ 32 ks), and a transposing read at rows rb (a
// multiple of 16) and columns cb (a multiple of 32) at
// rb * 2D + (tr_base_i ^ 2 cb) for its two halves i. The loops rebuild the
// XORs in every step from bases they mark as changed (opaque()): the
// compiler would otherwise keep every combination live across the loop and,
// short of registers, spill them and reload one before each LDS read.
template <int D>
__device__ __forceinline__ int row_base(int lq, int h2) {
  return toff<D>(lq, h2);
}
template <int D>
__device__ __forceinline__ int tr_base(int lane, int i) {
  const int G = lane >> 4, sl = lane & 15;
  const int col = (G & 1) * 16 + 4 * (sl & 3);
  const int r = 4 * (G >> 1) + 8 * i + (sl >> 2);
  return toff<D>(r, col >> 3) + ((col & 7) << 1);
}
template <int D>
__device__ __forceinline__ bf16x8 frag_row_x(const char* t, int base, int r0, int ks) {
  return *reinterpret_cast<const bf16x8*>(t + r0 * 2 * D + (base ^ (ks << 5)));
}
template <int D>
__device__ __forceinline__ bf16x8 frag_tr_x(const char* t, int b0, int b1, int rb, int cb) {
  const v4i16 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_t*)(t + rb * 2 * D + (b0 ^ (2 * cb))));
  const v4i16 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_t*)(t + rb * 2 * D + (b1 ^ (2 * cb))));
  const short __attribute__((ext_vector_type(8))) s = {lo[0], lo[1], lo[2], lo[3],
                                                       hi[0], hi[1], hi[2], hi[3]};
  return __builtin_bit_cast(bf16x8, s);
}
__device__ __forceinline__ void opaque(int& a, int& b, int& c) {
  asm volatile("" : "+v"(a), "+v"(b), "+v"(c));
}

// Rows 16 s .. 16 s + 15 of a 32 x 32 accumulator (lane l: column l % 32,
// element 4 J + j = row 8 J + 4 (l / 32) + j) as an MFMA column operand in
// the transposed operand's slot order: slot 4 i + j <- element 8 s + 4 i + j.
__device__ __forceinline__ bf16x8 pfrag(const floatx16& a, int s) {
  bf16x8 r;
#pragma unroll
  for (int t = 0; t < 8; ++t) r[t] = (__bf16)a[8 * s + t];
  return r;
}

__device__ __forceinline__ floatx16 mfma(const bf16x8& a, const bf16x8& b, const floatx16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// store a 32-row block of a transposed accumulator (lane: column = token,
// rows = d) as bf16 row segments dst[8 J + 4 (l / 32) .. + 3] * scale
__device__ __forceinline__ void store_cols(bf16_t* dst, const floatx16& a, int h2, float scale) {
#pragma unroll
  for (int J = 0; J < 4; ++J) {
    uint2 v;
    v.x = pack_bf16x2(a[4 * J] * scale, a[4 * J + 1] * scale);
    v.y = pack_bf16x2(a[4 * J + 2] * scale, a[4 * J + 3] * scale);
    *reinterpret_cast<uint2*>(dst + 8 * J + 4 * h2) = v;
  }
}

// One operand's ROWS-row tiles of a (sequence, head) by LDS-DMA, in the layout
// above: wave w of NW fills 1 KB blocks w, w + NW, ... (64 / CPR rows each), every
// lane fetching the chunk that belongs at its place. Rows at or past N (every
// row of a tile past the last) load zeros without traffic.
template <int D, int ROWS, int NW>
struct TileDma {
  static constexpr int TB = ROWS * D * 2;        // bytes of a tile
  static constexpr int CPR = D / 8, RPB = 64 / CPR;  // chunks a row, rows a block
  static constexpr int NB = TB / 1024, LD = (NB + NW - 1) / NW;  // blocks, loads a wave
  static_assert(NB % NW == 0, "whole loads");
  static_assert(LD == 1 || LD == 2 || LD % 4 == 0, "loads of one, two or four blocks");
  unsigned lds0, ld2, full;  // this wave's first block in slot 0; bytes of a row step, of a tile
  unsigned off[LD];
  __device__ __forceinline__ TileDma(unsigned lds, int w, int lane, long ld)
      : lds0(lds + w * 1024), ld2((unsigned)(2 * ld)), full((ROWS - 1) * ld2 + 2 * D) {
#pragma unroll
    for (int u = 0; u < LD; ++u) {
      const int r = (w + NW * u) * RPB + lane / CPR, c = (lane % CPR) ^ sw<D>(r);
      off[u] = r * ld2 + 16 * c;
    }
  }
  // the tile whose first row is at g, of which `rows` are there
  __device__ __forceinline__ void load(const bf16_t* g, int rows, int slot) const {
    const unsigned n = rows >= ROWS ? full : rows <= 0 ? 0u : (rows - 1) * ld2 + 2 * D;
    const unsigned long a = reinterpret_cast<unsigned long>(g);
    const u32x4 rs = {(unsigned)a, (unsigned)(a >> 32) & 0xFFFFu, n, 0x00020000u};
    if constexpr (LD <= 4) {
      dma16_row<LD, NW * 1024>(rs, lds0 + slot, off);
    } else {
#pragma unroll
      for (int g = 0; g < LD; g += 4) {
        const unsigned o4[4] = {off[g], off[g + 1], off[g + 2], off[g + 3]};
        dma16_row<4, NW * 1024>(rs, lds0 + slot + g * NW * 1024, o4);
      }
    }
  }
};

// the maximum and the sum over a lane pair (l, l + 32)
__device__ __forceinline__ float pair_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float pair_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

}  // namespace
}  // namespace flowmoe
