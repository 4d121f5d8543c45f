// Operands of 16-bit numbers on their way through registers to LDS, with consecutive k or with rows of k.
#pragma once

#include "layer8.hpp"

namespace rsvd {

constexpr int kKnK = 64;                   // k of a k-tile

// Place of 32-byte piece c of row k of a [k][X] tile.
template <int X> __device__ __forceinline__ int krow_piece(int c, int k) {
  if (X >= 128) return c ^ ((k & 3) | ((k >> 1) & 4));
  return c ^ (((k >> 1) & 1) | ((k >> 2) & 2));            // (two rows of 64 columns share 256 bytes)
}

// What one of NT threads stages of a k-tile of X rows (consecutive k) or columns (KROWS): N pieces of 16 bytes.
template <int NT, int X, bool KROWS, int DEPTH> struct Staged {
  static constexpr int ROW = KROWS ? X * 2 : 128, PER = ROW / 16, STEP = NT / PER, N = X * 128 / 16 / NT;      // bytes of a row; pieces; rows between a thread's
  static_assert(X * 128 % (16 * NT) == 0 && STEP % 8 == 0, "whole rounds; a thread's rows have their pieces exchanged alike, but for bit 3 of k");
  u32x4 reg[DEPTH][N];
  uint32_t off[N];
  int pos, place;
  // left: rows (columns) of the tile that exist; others are read as one that does, and not stored
  __device__ __forceinline__ void init(int64_t ld, int64_t left, int tid) {
    const int row = tid / PER, last = (int)(left < X ? left : X) - 1;
    pos = tid % PER;
    place = row * ROW + (KROWS ? (krow_piece<X>(pos >> 1, row) << 5) + ((pos & 1) << 4) : (pos ^ (row & 7)) << 4);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = row + STEP * i;
      off[i] = KROWS ? (uint32_t)r * (uint32_t)ld + (8 * pos > last ? 0u : 16u * pos)
                     : (uint32_t)(r < last ? r : last) * (uint32_t)ld + 16u * pos;
      asm volatile("" : "+v"(off[i]));                   // (one register, not the pair that the product came in)
    }
  }
  // base: the tile in memory; k_left: k of it that exist.  Those that do not are read beyond the end of the buffer, which gives zeros: behind the
  // last row of a [k][x] tile, and a long way off where k is consecutive.
  __device__ __forceinline__ void load(int set, int i, const char *base, int64_t ld, int k_left) {
    const int bytes = KROWS ? (int)(k_left * (uint32_t)ld) : 0x7fffffff;
    const __amdgpu_buffer_rsrc_t all = __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, bytes, 0x00027000);
    const uint32_t o = KROWS || 8 * pos < k_left ? off[i] : 0x80000000u;
    reg[set][i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(all, o, 0, 0));
  }
  __device__ __forceinline__ void write(int set, int i, char *lds) const {
    *reinterpret_cast<u32x4 *>(lds + (place ^ (KROWS && STEP % 16 == 8 ? (i & 1) << 7 : 0)) + i * STEP * ROW) = reg[set][i];
  }
};

}  // namespace rsvd
