// Products of two matrices with consecutive k: 16-bit numbers, and codes of 8-bit floats with a power of two for 128 of them.
//
// Tiles of BM x BN by WGM x WGN wavefronts.  A k-tile is 128 bytes of every row of both operands (64 numbers, 128 codes); two of them (three of small tiles) have
// room in LDS, which is filled by loads that write there themselves, issued among the matrix instructions of the tile before.  LDS is written in the order of the
// lanes, 16 bytes each, so a lane fetches the piece that belongs to its place: piece ch of row r lies in place ch ^ (r mod 8), which lets the eight rows that are
// read together start at different banks.  What is behind the last k is written over with zeros once it has arrived: a load has no mask.
//
// Rows of B are the columns of C.  Two blocks of sixteen share 32 rows so that a lane ends with eight consecutive columns of each row in its registers, four from either,
// and stores them as they are: row r of block 2 p + b is row 32 p + 8 (r / 4) + 4 b + r mod 4 of the tile, and pieces of B are exchanged by r mod 4 and bit 3 of the row.
// gated: 32 rows of the gate and the 32 of the up projection that belong to them in turn (16, and blocks as they come, where a wavefront has no more than two blocks).
//
// Codes are multiplied with their powers by the scaled matrix instruction (one for 128 k).  It takes eight k at a time and cuts each product off, towards zero, below
// 2^-13 of the largest of them, as all instructions for 8-bit floats do: measured 1.4e-5 of a result of normal numbers, 1.5e-4 of the sum of
// magnitudes at the worst.  That is lost in the rounding of a 16-bit result; for fp32 results DK_F8_EXACT makes bf16 numbers of the codes and
// their powers, exactly, and multiplies those at half the rate.
//
// Measured: bf16 8192 x 4096 x 16384 890 us with its gate (1.23 PFLOP/s; the library's largest product 1.41), 8-bit floats 482 us (2.28 PFLOP/s, library 2.67), at the
// clocks that the power budget leaves (1.93 to 1.98 GHz, matrix pipe busy 55 to 59 %).  Small tiles are bound by what a wavefront issues beside its matrix instructions and by the
// time of its loads: 0.3 us a k-tile.  So what can be counted on from k-tile to k-tile is not worked out anew (36.8 to 31.6 us for 512 x 4096 x 8192).
#pragma once

#include <type_traits>

#include "dense_tile.hpp"

namespace rsvd {

template <int KIND, int PL, int BM, int BN> struct DenseNtCfg {
  static constexpr int POWERS = PL * (BM + BN) * 128, STAGE = POWERS + (KIND >= DK_F8 ? (BM + BN) * 4 : 0), RING = BM > 64 || PL == 2 ? 2 : 3;      // behind the codes, a word of powers a row
  static constexpr size_t lds = RING * (size_t)STAGE;      // (more than the wavefronts need in the end)
};

// What the exchange of a row's pieces goes by.  PAIRED: rows of B that share blocks as above.
template <bool PAIRED> __device__ __forceinline__ int dense_swizzle(int row) { return PAIRED ? (row & 3) | ((row >> 1) & 4) : row & 7; }

// The loads of ROWS rows of a k-tile by NT threads.  GROUP: rows of gate and of up in turn (0: one matrix).
template <int NT, int ROWS, bool PAIRED, int GROUP> struct DenseLoad {
  static constexpr int N = ROWS * 8 / NT;
  static_assert(ROWS * 8 % NT == 0 && NT % 64 == 0, "whole rounds");
  uint32_t off[N];
  static __device__ __forceinline__ int piece(int q) { return (q & 7) ^ dense_swizzle<PAIRED>(q >> 3); }      // of the k-tile, in place q
  __device__ __forceinline__ void init(int64_t ld, int64_t rows_left, int tid) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int q = tid + NT * i, r = q >> 3, wanted = GROUP ? r / (2 * (GROUP ? GROUP : 1)) * GROUP + r % (GROUP ? GROUP : 1) : r;
      const int row = wanted < rows_left ? wanted : (int)rows_left - 1;
      off[i] = (uint32_t)row * (uint32_t)ld + (uint32_t)(piece(q) << 4);
      asm volatile("" : "+v"(off[i]));                   // (one register, not the pair that the product came in)
    }
  }
  // Load i of a thread, from the tile's first row on (`up` bytes behind it for rows of the up projection; a wavefront has eight rows of one of
  // both).  left: pieces of the k-tile that exist; another one is read in the place of those that do not.
  __device__ __forceinline__ void issue(int i, const char *base, int64_t up, char *lds, int left, int wave, int tid) {
    uint32_t o = off[i];
    if (left < 8) {
      const int ch = piece(tid + NT * i);
      if (ch >= left) o -= (uint32_t)ch << 4;
    }
    if (GROUP && ((wave * 8 + NT / 8 * i) / (GROUP ? GROUP : 1) & 1)) base += up;
    const __amdgpu_buffer_rsrc_t all = __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, 0x7fffffff, 0x00027000);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(all, (__attribute__((address_space(3))) void *)(lds + (wave * 64 + NT * i) * 16), 16, o, 0, 0, 0);
  }
};

// Sixteen codes times a power of two as bf16 numbers (exactly, but for results below the least bf16 number).
__device__ __forceinline__ void f8_widen(u32x4 codes, float unit, u32x4 (&out)[2]) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const unsigned four = codes[w];
    out[w >> 1][2 * (w & 1)] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(four, unit, false));
    out[w >> 1][2 * (w & 1) + 1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(four, unit, true));
  }
}
// 2^e of the byte e + 127, NaN for 255.  (No branches: arithmetic on the bits; 0 is 2^-127.)
__device__ __forceinline__ float f8_unit(unsigned power) { return __uint_as_float(max(power << 23, 0x00400000u) + ((power + 1) >> 8 << 22)); }
__device__ __forceinline__ i32x8 f8_both(const u32x4 (&p)[2]) {
  return i32x8{(int)p[0][0], (int)p[0][1], (int)p[0][2], (int)p[0][3], (int)p[1][0], (int)p[1][1], (int)p[1][2], (int)p[1][3]};
}

// PL planes of both operands are multiplied while a k-tile of all is in LDS; 1: the products of planes are further k.
// KG: groups of wavefronts that have the whole tile and a half of every k-tile (2: two wavefronts a SIMD, one waits while the other multiplies; gated fp32
// 384 x 2048 -> 2048 59.8 us, with one group 70.0; updates of 1000 x 2000 in bf16 201 and 225; but gated bf16 384 x 2048 -> 2048 16.0 and 14.8, several workgroups a CU), or all of it (1).
template <int KIND, bool GATED, int PL, int BM, int BN, int WGM, int WGN, int KG>
__global__ __launch_bounds__(64 * WGM * WGN * KG, BM == 256 ? 1 : KG == 1 ? 2 : PL == 3 ? 2 : 4) void dense_nt_kernel(const DenseParams P) {
  static_assert(KG == 1 || (KG == 2 && BM == 64 && KIND < DK_F8), "halves of the k-tiles of small tiles");
  constexpr int NT = 64 * WGM * WGN * KG, WM = BM / WGM, WN = BN / WGN, TM = WM / 16, TN = WN / 16, STAGE = DenseNtCfg<KIND, PL, BM, BN>::STAGE, RING = DenseNtCfg<KIND, PL, BM, BN>::RING;
  constexpr bool CODES = KIND >= DK_F8;
  extern __shared__ __attribute__((aligned(16))) char dense_lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, kq = lane >> 4;
  const int group = KG == 1 ? 0 : wave / (WGM * WGN), wave_m = wave / WGN - group * WGM, wm0 = wave_m * WM, wn0 = (wave % WGN) * WN;
  const DenseWork work = dense_work<BM * BN>(P);
  const int tile_m = work.tile_m, tile_n = work.tile_n, batch = work.batch, kt_begin = work.kt_begin, nkt = work.nkt;
  const int64_t m0 = (int64_t)tile_m * BM, n0 = (int64_t)tile_n * (GATED ? BN / 2 : BN);

  f32x4 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      acc[i][j] = (f32x4)0.f;
      pin<BM == 256>(acc[i][j]);
    }

  constexpr bool PAIRED = !GATED || TN > 2;
  DenseLoad<NT, BM, false, 0> la;
  DenseLoad<NT, BN, PAIRED, !GATED ? 0 : PAIRED ? 32 : 16> lb;
  la.init(P.lda, P.M - m0, tid);
  lb.init(P.ldb, P.N - n0, tid);
  // of codes, too: the words that hold the powers of the tile's rows, one row a lane (small tiles: by two wavefronts each)
  constexpr int POWER_LOADS = !CODES ? 0 : BM + BN < NT ? 1 : (BM + BN) / NT, TILE_LOADS = decltype(la)::N + decltype(lb)::N, LOADS = PL * TILE_LOADS + POWER_LOADS;
  uint32_t pow_off[CODES ? POWER_LOADS : 1];
  if constexpr (CODES) {
#pragma unroll
    for (int i = 0; i < POWER_LOADS; ++i) {
      const int r = (tid + NT * i) & (BM + BN - 1);
      const int64_t m = m0 + r < P.M ? m0 + r : P.M - 1, n = n0 + r - BM < P.N ? n0 + r - BM : P.N - 1;
      pow_off[i] = r < BM ? (uint32_t)((m >> P.a_shift) * P.ld_apow) : (uint32_t)((n >> P.b_shift) * P.ld_bpow);
    }
  }
  const char *const a_row = P.A + batch * P.a_batch + m0 * P.lda, *const b_row = P.B + batch * P.b_batch + n0 * P.ldb;
  const int last_left = (int)((P.K * (CODES ? 1 : 2) - (int64_t)(P.ktiles - 1) * 128) >> 4);      // pieces of the last k-tile that exist

  // the k-tile that is loaded next: its part of k and its place there
  int next_seg = __builtin_amdgcn_readfirstlane(kt_begin / P.ktiles), next_kt = __builtin_amdgcn_readfirstlane(kt_begin - next_seg * P.ktiles), next = 0;
  const int first_kt = next_kt;
  const char *a_now, *b_now;
  int left;
  auto point = [&]() RSVD_INLINE {
    a_now = a_row + (PL > 1 || CODES ? 0 : (int64_t)(P.segs.a >> (4 * next_seg) & 15) * P.a_plane) + (int64_t)next_kt * 128;
    b_now = b_row + (PL > 1 || CODES ? 0 : (int64_t)(P.segs.b >> (4 * next_seg) & 15) * P.b_plane) + (int64_t)next_kt * 128;
  };
  auto remain = [&]() RSVD_INLINE { left = CODES ? 8 : next_kt == P.ktiles - 1 ? last_left : 8; };
  auto advance = [&]() RSVD_INLINE {                    // (behind the last tile that one again, where nobody reads it: no branches around loads)
    const int step = ++next < nkt ? 1 : 0;
    next_kt += step;
    a_now += 128 * step;
    b_now += 128 * step;
    if (PL == 1 && !CODES && next_kt == P.ktiles) {
      next_kt = 0;
      ++next_seg;
      point();
    }
    remain();
  };
  // (where a tile lies: `place` bytes into LDS)
  auto place = [&](int kt) RSVD_INLINE { return (kt % RING) * STAGE; };
  auto issue = [&](int at_lds, int l) RSVD_INLINE {
    char *st = dense_lds + at_lds;
    const int q = l / TILE_LOADS, at = l % TILE_LOADS;   // (planes: those of A and B in turn)
    if (q < PL && at < decltype(la)::N) {
      la.issue(at, a_now + q * P.a_plane, 0, st + q * (BM + BN) * 128, left, wave, tid);
    } else if (q < PL) {
      lb.issue(at - decltype(la)::N, b_now + q * P.b_plane, P.b_up, st + (q * (BM + BN) + BM) * 128, left, wave, tid);
    } else if constexpr (CODES) {
      const int i = l - TILE_LOADS, first = (wave * 64 + NT * i) & (BM + BN - 1);
      const uint8_t *base = (first < BM ? P.a_pow : P.b_pow) + (next_kt & ~3);
      const __amdgpu_buffer_rsrc_t all = __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, 0x7fffffff, 0x00027000);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(all, (__attribute__((address_space(3))) void *)(st + DenseNtCfg<KIND, PL, BM, BN>::POWERS + first * 4), 4, pow_off[i], 0, 0, 0);
    }
  };

  constexpr int AHEAD = TM >= 4 ? 3 : 1;               // rows of blocks read ahead, not all of them: registers
  constexpr int FIRST = KIND == DK_F8 || BM == 64 || LOADS < 2 * AHEAD ? LOADS : 2 * AHEAD;      // loads of a tile that are issued behind a meeting
  // (rows of a wavefront's blocks start at multiples of 32, or of 16 where they are not shared: what pieces are exchanged by is the lane's)
  const int b_first = PAIRED ? 8 * (r16 >> 2) + (r16 & 3) : r16, a_swz = dense_swizzle<false>(r16), b_swz = dense_swizzle<PAIRED>(b_first);
  const char *const a_lds = dense_lds + (wm0 + r16) * 128, *const b_lds = dense_lds + BM * 128 + (wn0 + b_first) * 128;
  auto piece_a = [&](int at_lds, int i, int h, int q = 0) RSVD_INLINE {
    return *reinterpret_cast<const u32x4 *>(a_lds + at_lds + q * (BM + BN) * 128 + i * 2048 + (((4 * h + kq) ^ a_swz) << 4));
  };
  auto piece_b = [&](int at_lds, int j, int h, int q = 0) RSVD_INLINE {
    return *reinterpret_cast<const u32x4 *>(b_lds + at_lds + q * (BM + BN) * 128 + (PAIRED ? j / 2 * 4096 + (j & 1) * 512 : j * 2048) + (((4 * h + kq) ^ b_swz) << 4));
  };
  // powers of the rows of a lane's blocks: in words of four k-tiles, and of the one that is multiplied
  unsigned words_a[CODES ? TM : 1], words_b[CODES ? TN : 1], pa[CODES ? TM : 1], pb[CODES ? TN : 1];
  const char *const pow_lds = dense_lds + DenseNtCfg<KIND, PL, BM, BN>::POWERS;
  auto read_powers = [&](int at_lds) RSVD_INLINE {
#pragma unroll
    for (int i = 0; i < (CODES ? TM : 0); ++i) words_a[i] = *reinterpret_cast<const unsigned *>(pow_lds + at_lds + (wm0 + 16 * i + r16) * 4);
#pragma unroll
    for (int j = 0; j < (CODES ? TN : 0); ++j)
      words_b[j] = *reinterpret_cast<const unsigned *>(pow_lds + at_lds + (BM + wn0 + 32 * (j / 2) + 4 * (j & 1) + b_first) * 4);
  };
  auto take_powers = [&](int kt) RSVD_INLINE {
    const int by = 8 * ((kt_begin + kt) & 3);
#pragma unroll
    for (int i = 0; i < (CODES ? TM : 0); ++i) pa[i] = words_a[i] >> by;
#pragma unroll
    for (int j = 0; j < (CODES ? TN : 0); ++j) pb[j] = words_b[j] >> by;
  };
  // Everybody has read its last of the tile before kt, and kt has arrived: `flying` loads are of later tiles.
  auto meet = [&](auto flying, int kt, int at_lds) RSVD_INLINE {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(tile_wait(decltype(flying)::value));
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if constexpr (!CODES) {
      if (last_left < 8 && (first_kt + kt + 1) % P.ktiles == 0) {      // zeros behind the last k
        for (int q = tid; q < (BM + BN) * 8; q += NT)
          if ((q < BM * 8 ? decltype(la)::piece(q) : decltype(lb)::piece(q - BM * 8)) >= last_left) {
#pragma unroll
            for (int p = 0; p < PL; ++p) *reinterpret_cast<u32x4 *>(dense_lds + at_lds + (p * (BM + BN) * 8 + q) * 16) = (u32x4)0u;
          }
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(tile_wait(63));
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
      }
    }
  };
  point();
  remain();
#pragma unroll
  for (int t = 0; t < RING - 1; ++t) {
#pragma unroll
    for (int l = 0; l < LOADS; ++l) issue(t * STAGE, l);
    advance();
  }
#pragma unroll
  for (int l = 0; l < FIRST; ++l) issue((RING - 1) * STAGE, l);
  meet(std::integral_constant<int, (RING - 2) * LOADS + FIRST>(), 0, 0);

  // Where the rows of blocks of a tile that are read ahead would be those of the next one, wavefronts meet, and go on with the next tile's: no wavefront
  // waits for LDS at the start of a tile.  (The loads of a tile go to the place of the one that is multiplied before, from the meeting on.)
  if constexpr (BM == 64) {
    // small tiles: all operands of the next tile are read while one is multiplied (LDS takes longer to answer than a row of blocks takes)
    u32x4 a[2][TM][2 / KG][PL], b[2][TN][2 / KG][PL];
    unsigned words[2][2][CODES ? TM : 1];
    static_assert(TM == TN, "square tiles");
    auto fetch = [&](auto to, int at_lds) RSVD_INLINE {
      constexpr int S = decltype(to)::value;
#pragma unroll
      for (int h = 0; h < 2 / KG; ++h)
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int q = PL - 1; q >= 0; --q) {
            a[S][i][h][q] = piece_a(at_lds, i, KG == 1 ? h : group, q);
            b[S][i][h][q] = piece_b(at_lds, i, KG == 1 ? h : group, q);
          }
      if constexpr (CODES) {
        read_powers(at_lds);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
          words[S][0][i] = words_a[i];
          words[S][1][i] = words_b[i];
        }
      }
    };
    auto multiply = [&](auto of, int kt) RSVD_INLINE {
      constexpr int S = decltype(of)::value;
      if constexpr (CODES) {
        const int by = 8 * ((kt_begin + kt) & 3);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
          pa[i] = words[S][0][i] >> by;
          pb[i] = words[S][1][i] >> by;
        }
      }
      if constexpr (KIND == DK_F8) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int j = 0; j < TN; ++j) {
            const u32x4 x[2] = {b[S][j][0][0], b[S][j][1][0]}, y[2] = {a[S][i][0][0], a[S][i][1][0]};
            acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(f8_both(x), f8_both(y), acc[i][j], 0, 0, 0, (int)pb[j], 0, (int)pa[i]);
          }
      } else if constexpr (KIND == DK_F8_EXACT) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          u32x4 x[TN][2], y[TM][2];
#pragma unroll
          for (int i = 0; i < TM; ++i) {
            f8_widen(b[S][i][h][0], f8_unit(pb[i] & 255u), x[i]);
            f8_widen(a[S][i][h][0], f8_unit(pa[i] & 255u), y[i]);
          }
#pragma unroll
          for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
              for (int j = 0; j < TN; ++j) acc[i][j] = mfma_bf16(x[j][q], y[i][q], acc[i][j]);
        }
      } else {
#pragma unroll
        for (int h = 0; h < 2 / KG; ++h)
          with_segs<PL>([&](auto qa, auto qb) RSVD_INLINE {
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
              for (int j = 0; j < TN; ++j) {
                const u32x4 x = b[S][j][h][decltype(qb)::value], y = a[S][i][h][decltype(qa)::value];
                acc[i][j] = KIND == DK_BF16 ? mfma_bf16(x, y, acc[i][j]) : mfma_f16(x, y, acc[i][j]);
              }
          });
      }
    };
    int here = 0, there = STAGE;                         // where a tile and the next one lie
    auto tile = [&](auto now, auto then, int kt) RSVD_INLINE {
      meet(std::integral_constant<int, (RING - 2) * LOADS>(), kt + 1, there);
      advance();
      fetch(then, there);
#pragma unroll
      for (int l = 0; l < LOADS; ++l) issue(here, l);
      here = there;
      there = there == (RING - 1) * STAGE ? 0 : there + STAGE;
      __builtin_amdgcn_sched_barrier(0);
      multiply(now, kt);
      __builtin_amdgcn_sched_barrier(0);
    };
    typedef std::integral_constant<int, 0> even;
    typedef std::integral_constant<int, 1> odd;
    fetch(even(), 0);
    for (int kt = 0; kt < nkt; kt += 2) {
      tile(even(), odd(), kt);
      if (kt + 1 < nkt) tile(odd(), even(), kt + 1);
    }
  } else if constexpr (KIND == DK_F8) {
    // a tile's last rows of blocks column by column, so that an operand of B is free for the next tile's as soon as it can be
    u32x4 a[AHEAD + 1][2], b[TN][2];
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) b[j][h] = piece_b(0, j, h);
#pragma unroll
    for (int h = 0; h < 2; ++h) a[0][h] = piece_a(0, 0, h);
    read_powers(0);
    for (int kt = 0; kt < nkt; ++kt) {
      take_powers(kt);
      auto multiply = [&](int i, int j) RSVD_INLINE {
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(f8_both(b[j]), f8_both(a[i % (AHEAD + 1)]), acc[i][j], 0, 0, 0, (int)pb[j], 0, (int)pa[i]);
      };
#pragma unroll
      for (int i = 1; i < AHEAD; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) a[i][h] = piece_a(place(kt), i, h);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < TM - AHEAD; ++i) {
#pragma unroll
        for (int h = 0; h < 2; ++h) a[(i + AHEAD) % (AHEAD + 1)][h] = piece_a(place(kt), i + AHEAD, h);
#pragma unroll
        for (int j = 0; j < TN; ++j) multiply(i, j);
        __builtin_amdgcn_sched_barrier(0);
      }
      meet(std::integral_constant<int, (RING - 2) * LOADS>(), kt + 1, place(kt + 1));
      advance();
#pragma unroll
      for (int h = 0; h < 2; ++h) a[0][h] = piece_a(place(kt + 1), 0, h);
      read_powers(place(kt + 1));
#pragma unroll
      for (int j = 0; j < TN; ++j) {
#pragma unroll
        for (int i = TM - AHEAD; i < TM; ++i) multiply(i, j);
#pragma unroll
        for (int l = 0; l < LOADS; ++l)
          if (l * TN / LOADS == j) issue(place(kt), l);
#pragma unroll
        for (int h = 0; h < 2; ++h) b[j][h] = piece_b(place(kt + 1), j, h);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  } else {
    // (of 8-bit floats as bf16 numbers: two steps of 32 k out of a piece)
    constexpr int Q = KIND == DK_F8_EXACT ? 2 : 1;
    u32x4 a[AHEAD + 1][PL], b[2][TN][PL];
#pragma unroll
    for (int q = 0; q < PL; ++q) {
#pragma unroll
      for (int j = 0; j < TN; ++j) b[0][j][q] = piece_b(0, j, 0, q);
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) a[i][q] = piece_a(0, i, 0, q);
    }
    if constexpr (CODES) read_powers(0);
    u32x4 wide[Q == 2 ? TN : 1][2];
    for (int kt = 0; kt < nkt; ++kt) {
      if constexpr (CODES) take_powers(kt);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int step = 0; step < 2 * TM; ++step) {
        const int h = step / TM, i = step % TM, ahead = step + AHEAD;
        if (step == 2 * TM - AHEAD) {
          meet(std::integral_constant<int, (RING - 2) * LOADS>(), kt + 1, place(kt + 1));
          advance();
          if constexpr (CODES) read_powers(place(kt + 1));
        }
        u32x4 now[PL];
#pragma unroll
        for (int q = 0; q < PL; ++q) {
          now[q] = a[step % (AHEAD + 1)][q];
          a[ahead % (AHEAD + 1)][q] = piece_a(place(ahead < 2 * TM ? kt : kt + 1), ahead % TM, ahead / TM % 2, q);
#pragma unroll
          for (int j = 0; j < TN; ++j) {
            if (h == 0 && i == j * TM / TN) b[1][j][q] = piece_b(place(kt), j, 1, q);
            if (step >= 2 * TM - AHEAD && (step - 2 * TM + AHEAD) == j * AHEAD / TN) b[0][j][q] = piece_b(place(kt + 1), j, 0, q);
          }
        }
        if constexpr (KIND == DK_F8_EXACT) {
          u32x4 wide_a[2];
          f8_widen(now[0], f8_unit(pa[i] & 255u), wide_a);
          if (i == 0) {
#pragma unroll
            for (int j = 0; j < TN; ++j) f8_widen(b[h][j][0], f8_unit(pb[j] & 255u), wide[j]);
          }
#pragma unroll
          for (int q = 0; q < Q; ++q)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = mfma_bf16(wide[j][q], wide_a[q], acc[i][j]);
        } else {
          with_segs<PL>([&](auto pa_, auto pb_) RSVD_INLINE {
#pragma unroll
            for (int j = 0; j < TN; ++j)
              acc[i][j] = KIND == DK_BF16 ? mfma_bf16(b[h][j][decltype(pb_)::value], now[decltype(pa_)::value], acc[i][j])
                                          : mfma_f16(b[h][j][decltype(pb_)::value], now[decltype(pa_)::value], acc[i][j]);
          });
        }
#pragma unroll
        for (int l = 0; l < LOADS; ++l) {
          // (FIRST of them behind the meeting; the others two a step, or as many as it takes to have them all before the next)
          constexpr int EACH = (LOADS - FIRST + 2 * TM - AHEAD - 1) / (2 * TM - AHEAD) > 2 ? (LOADS - FIRST + 2 * TM - AHEAD - 1) / (2 * TM - AHEAD) : 2;
          if (l < FIRST ? step == 2 * TM - AHEAD + l / 2 : step == (l - FIRST) / EACH) issue(place(l < FIRST ? kt : kt + RING - 1), l);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }

  int last_lane = lane;                                // (anew: what follows from it would be worked out before the main loop otherwise, and kept)
  asm volatile("" : "+v"(last_lane));
  const int64_t n1 = n0 + (GATED ? wn0 / 2 : wn0);
  float *const partial = work.partial != nullptr ? work.partial + wm0 * BN + wn0 : nullptr;
  // Of groups that have halves of k, each ends with one row of blocks: its own sums and the other's.
  constexpr int ROWS = TM / KG;
  f32x4 sums[ROWS][TN];
  if constexpr (KG == 2) {
    static_assert(TM == 2 && WGM * WGN * 2 * TN * 1024 <= RING * STAGE, "a row of blocks a group");
    __builtin_amdgcn_s_waitcnt(tile_wait(0));            // (nothing may land in LDS any more)
    __syncthreads();
    f32x4 *const mine = reinterpret_cast<f32x4 *>(dense_lds) + wave * TN * 64 + last_lane;
    f32x4 *const other = reinterpret_cast<f32x4 *>(dense_lds) + (wave + (group == 0 ? WGM * WGN : -WGM * WGN)) * TN * 64 + last_lane;
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      mine[j * 64] = group == 0 ? acc[1][j] : acc[0][j];
      sums[0][j] = group == 0 ? acc[0][j] : acc[1][j];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < TN; ++j) sums[0][j] += other[j * 64];
  } else {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) sums[i][j] = acc[i][j];
  }
  const int64_t m1 = m0 + wm0 + (KG == 1 ? 0 : 16 * group);
  dense_finish_rows<GATED, BN, ROWS, TN>(P, sums, KG == 1 || partial == nullptr ? partial : partial + 16 * group * BN, batch, m1, n1, last_lane);
  if constexpr (!GATED && !CODES) {
    if (P.symmetric && tile_m != tile_n && partial == nullptr) {
      __builtin_amdgcn_s_waitcnt(tile_wait(0));          // (nothing may land in LDS any more)
      __syncthreads();
      dense_finish_mirror<ROWS, TN>(P, sums, batch, m1, n1, last_lane, reinterpret_cast<float *>(dense_lds + wave * finish_lds<TN>()));
    }
  }
}

template <int KIND, bool GATED, int PL, int BM, int BN, int WGM, int WGN, int KG = 1> hipError_t dense_nt_run(hipStream_t s, const DenseParams &P) {
  hipLaunchKernelGGL((dense_nt_kernel<KIND, GATED, PL, BM, BN, WGM, WGN, KG>), dim3(dense_groups(P)), dim3(64 * WGM * WGN * KG), (DenseNtCfg<KIND, PL, BM, BN>::lds), s, P);
  return hipGetLastError();
}
// The planes that small tiles of a kind take at once: three of bf16 numbers, two of fp16 numbers of a plain product.
template <int KIND, bool GATED> constexpr int dense_nt_planes() { return KIND == DK_BF16 ? 3 : KIND == DK_F16 && !GATED ? 2 : 1; }
template <int KIND, bool GATED> hipError_t dense_nt_tile(hipStream_t s, const DenseParams &P, int b) {
  if (b == 256) return dense_nt_run<KIND, GATED, 1, 256, 256, 2, 2>(s, P);
  if (b == 128) return dense_nt_run<KIND, GATED, 1, 128, 128, 2, 2>(s, P);
  constexpr int PL = dense_nt_planes<KIND, GATED>();
  if (P.segs.count > 1) return dense_nt_run<KIND, GATED, PL, 64, 64, 2, 2, (PL > 1 ? 2 : 1)>(s, P);
  return dense_nt_run<KIND, GATED, 1, 64, 64, 2, 2, KIND == DK_F16 && !GATED ? 2 : 1>(s, P);
}
template <int KIND, bool GATED> hipError_t dense_nt_init() {
  constexpr int PL = dense_nt_planes<KIND, GATED>();
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&dense_nt_kernel<KIND, GATED, 1, 256, 256, 2, 2, 1>), hipFuncAttributeMaxDynamicSharedMemorySize,
                                           (int)DenseNtCfg<KIND, 1, 256, 256>::lds);
  if (e != hipSuccess || PL == 1) return e;
  return hipFuncSetAttribute(reinterpret_cast<const void *>(&dense_nt_kernel<KIND, GATED, PL, 64, 64, 2, 2, (PL > 1 ? 2 : 1)>), hipFuncAttributeMaxDynamicSharedMemorySize,
                             (int)DenseNtCfg<KIND, PL, 64, 64>::lds);
}
#define DENSE_NT(KIND, GATED)                                                                        \
  template hipError_t dense_nt_tile<KIND, GATED>(hipStream_t s, const DenseParams &P, int b);       \
  template hipError_t dense_nt_init<KIND, GATED>();

}  // namespace rsvd
