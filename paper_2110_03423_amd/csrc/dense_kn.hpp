// Products of 16-bit numbers where B has rows of n, and A rows of k or of m: gradients, and polynomials times a matrix.
//
// Tiles [k][x] in LDS are read with the transposing LDS load (sixteen lanes read four k of sixteen columns and get one column of four k each); rows of k
// lie with their 32-byte pieces exchanged by the low bits of k, so that the eight rows that half a wavefront reads start at different banks.  Both operands go
// from memory to registers and from there to LDS, among the matrix instructions of the tile before.
//
// Measured: bf16 8192 x 16384 x 4096 829 us (1.33 PFLOP/s, matrix pipe busy 69 % at 1.84 GHz: power; the library's product in this order 1.25), with rows of m 888 us (1.24; library 1.11).
// fp32 301 x 2820 x 2999 in tiles of 64 with all planes at once 47.3 us (fp32 numbers of B as they lie 55.3, without the 13 that laying them out takes), 2820 x 301 x 2999 in tiles of 128 45.4.
#pragma once

#include <type_traits>

#include "dense_tile.hpp"
#include "layer8_staged.hpp"

namespace rsvd {

template <int PL, int BM, int BN> struct DenseKnCfg {
  static constexpr int A = BM * 128, B = BN * 128, PLANE = A + B, STAGE = PL * PLANE, DEPTH = BM == 256 ? 1 : 2;
  static constexpr size_t lds = 2 * (size_t)STAGE;      // (more than the wavefronts need in the end)
};

// Rows of k of B that are fp32 numbers as they lie, for tiles of 64: eight numbers of a row a thread, which become three bf16 numbers each on the way to LDS.  A piece that ends
// behind the last column is read further to the left, and its numbers moved (at least four columns).
template <int NT, int DEPTH> struct WideStaged {
  static_assert(NT == 512, "a piece a thread");
  u32x4 reg[DEPTH][2];
  uint32_t off[2];
  int moved, place;
  // n0: the tile's first column; columns: how many there are
  __device__ __forceinline__ void init(int64_t ld, int64_t n0, int64_t columns, int tid) {
    const int row = tid >> 3, pos = tid & 7;
    place = row * 128 + (krow_piece<64>(pos >> 1, row) << 5) + ((pos & 1) << 4);
    moved = 0;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const int64_t first = n0 + 8 * pos + 4 * q;
      const int64_t from = first + 4 <= columns ? first : first < columns ? columns - 4 : 0;
      if (first + 4 > columns && first < columns) moved |= (int)(first - from) << (4 * q);
      off[q] = (uint32_t)row * (uint32_t)ld + (uint32_t)from * 4u;
      asm volatile("" : "+v"(off[q]));
    }
  }
  // base: the tile's first row; rows that do not exist are read beyond the end of the buffer, which gives zeros
  __device__ __forceinline__ void load(int set, const char *base, int64_t ld, int k_left) {
    const __amdgpu_buffer_rsrc_t all = __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, (int)(k_left * (uint32_t)ld), 0x00027000);
#pragma unroll
    for (int q = 0; q < 2; ++q) reg[set][q] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(all, off[q], 0, 0));
  }
  // whole: every column of the tile exists
  __device__ __forceinline__ void write(int set, char *lds, int plane, bool whole) const {
    Raw8<RSVD_X_F32> v = {{reg[set][0], reg[set][1]}};
    if (!whole) {
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int by = moved >> (4 * q) & 3;
        u32x4 w = v.w[q];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = by & 1 ? (e < 3 ? w[e < 3 ? e + 1 : 3] : 0u) : w[e];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = by & 2 ? (e < 2 ? w[e < 2 ? e + 2 : 3] : 0u) : w[e];
        v.w[q] = w;
      }
    }
    u32x4 x[3];
    unsigned top = 0u;                                   // (one question for all of what bf16 numbers round to infinity, or that is it)
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, v.w[e >> 2][e & 3] << 1);
    if (top < 0x7f7f8000u << 1) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        unsigned p[3];
        bf16_parts2<3, false>(__uint_as_float(v.w[e >> 1][2 * (e & 1)]), __uint_as_float(v.w[e >> 1][2 * (e & 1) + 1]), p);
#pragma unroll
        for (int q = 0; q < 3; ++q) x[q][e] = p[q];
      }
    } else {
      split_operand<RSVD_X_F32>(v, x);
    }
#pragma unroll
    for (int p = 0; p < 3; ++p) *reinterpret_cast<u32x4 *>(lds + p * plane + place) = x[p];
  }
};

// PL planes of both operands are multiplied while a k-tile of all is in LDS; 1: the products of planes are further k.
// KG: groups of wavefronts that have the whole tile and a half of every k-tile (2: two wavefronts a SIMD, one waits while the other multiplies), or all of it (1).
// WIDE: B is fp32 numbers as they lie.
template <int KIND, bool A_KROWS, int PL, int BM, int BN, int WGM, int WGN, int KG, bool WIDE>
__global__ __launch_bounds__(64 * WGM * WGN * KG, KG == 1 ? 2 : PL == 3 ? 2 : 4) void dense_kn_kernel(const DenseParams P) {
  static_assert(!WIDE || (KIND == DK_BF16 && PL == 3 && KG == 2), "three bf16 numbers of each");
  static_assert(KG == 1 || (KG == 2 && BM == 64), "halves of the k-tiles of small tiles");
  constexpr int NT = 64 * WGM * WGN * KG, WM = BM / WGM, WN = BN / WGN, TM = WM / 16, TN = WN / 16, DEPTH = DenseKnCfg<PL, BM, BN>::DEPTH;
  constexpr int STAGE = DenseKnCfg<PL, BM, BN>::STAGE, PLANE = DenseKnCfg<PL, BM, BN>::PLANE, B_LDS = DenseKnCfg<PL, BM, BN>::A;
  extern __shared__ __attribute__((aligned(16))) char dense_lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, kq = lane >> 4;
  const int group = KG == 1 ? 0 : wave / (WGM * WGN), wave_m = wave / WGN - group * WGM, wave_n = wave % WGN, wm0 = wave_m * WM, wn0 = wave_n * WN;
  const DenseWork work = dense_work<BM * BN>(P);
  const int tile_m = work.tile_m, tile_n = work.tile_n, batch = work.batch, kt_begin = work.kt_begin, nkt = work.nkt;
  const int64_t m0 = (int64_t)tile_m * BM, n0 = (int64_t)tile_n * BN;

  f32x4 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      acc[i][j] = (f32x4)0.f;
      pin<BM == 256>(acc[i][j]);
    }

  // the k-tile that is loaded next: its part of k, its place there, and how many k of it exist
  int next_seg = __builtin_amdgcn_readfirstlane(kt_begin / P.ktiles), next_kt = __builtin_amdgcn_readfirstlane(kt_begin - next_seg * P.ktiles);
  const char *const a_first = P.A + batch * P.a_batch + (A_KROWS ? m0 * 2 : m0 * P.lda), *const b_first = P.B + batch * P.b_batch + (WIDE ? 0 : n0 * 2);
  const char *a_now, *b_now;
  int left;
  auto point = [&]() RSVD_INLINE {
    const int64_t k = (int64_t)next_kt * kKnK;
    a_now = a_first + (PL > 1 ? 0 : (int64_t)(P.segs.a >> (4 * next_seg) & 15) * P.a_plane) + (A_KROWS ? k * P.lda : k * 2);
    b_now = b_first + (PL > 1 ? 0 : (int64_t)(P.segs.b >> (4 * next_seg) & 15) * P.b_plane) + k * P.ldb;
    left = (int)(P.K - k < kKnK ? P.K - k : kKnK);
  };
  const int64_t a_step = A_KROWS ? kKnK * P.lda : 2 * kKnK, b_step = kKnK * P.ldb;
  const int last_left = (int)(P.K - (int64_t)(P.ktiles - 1) * kKnK);
  auto advance = [&]() RSVD_INLINE {                    // (behind the last tile of this workgroup's range: loads stay inside the operands)
    a_now += a_step;
    b_now += b_step;
    if (++next_kt == P.ktiles) {
      next_kt = 0;
      if (PL == 1 && next_seg + 1 < P.segs.count) ++next_seg;
      point();
    }
    left = next_kt == P.ktiles - 1 ? last_left : kKnK;
  };
  Staged<NT, BM, A_KROWS, DEPTH * PL> sa;
  std::conditional_t<WIDE, WideStaged<NT, DEPTH>, Staged<NT, BN, true, DEPTH * PL>> sb;
  sa.init(P.lda, P.M - m0, tid);
  if constexpr (WIDE) sb.init(P.ldb, n0, P.N, tid);
  else sb.init(P.ldb, P.N - n0, tid);
  constexpr int NA = decltype(sa)::N, NB = Staged<NT, BN, true, DEPTH * PL>::N, EACH = WIDE ? NA : NA + NB, PIECES = PL * EACH + (WIDE ? 1 : 0);
  const bool b_whole = n0 + BN <= P.N;
  auto load = [&](int set, int piece) RSVD_INLINE {
    const int q = piece / EACH, p = piece % EACH;
    if constexpr (WIDE)
      if (piece == PL * NA) {
        sb.load(set, b_now, P.ldb, left);
        return;
      }
    if (p < NA) sa.load(PL * set + q, p, a_now + q * P.a_plane, P.lda, left);
    else if constexpr (!WIDE) sb.load(PL * set + q, p - NA, b_now + q * P.b_plane, P.ldb, left);
  };
  auto write = [&](int set, int piece, int buf) RSVD_INLINE {
    const int q = piece / EACH, p = piece % EACH;
    if constexpr (WIDE)
      if (piece == PL * NA) {
        sb.write(set, dense_lds + buf * STAGE + B_LDS, PLANE, b_whole);
        return;
      }
    if (p < NA) sa.write(PL * set + q, p, dense_lds + buf * STAGE + q * PLANE);
    else if constexpr (!WIDE) sb.write(PL * set + q, p - NA, dense_lds + buf * STAGE + q * PLANE + B_LDS);
  };

  // ---- operands of this lane
  constexpr int A_ROW = decltype(sa)::ROW;
  const int key_row = 8 * kq + (r16 >> 2), part = (r16 & 3) * 8;
  // (blocks of 16 columns differ from the first one of the wavefront in the bits that are exchanged)
  static_assert((TM == 8 || TM == 4 || TM == 2) && (TN == 8 || TN == 4 || TN == 2), "blocks of a power of two");
  const int a_at = A_KROWS ? key_row * A_ROW + (krow_piece<BM>(wm0 / 16, key_row) << 5) + part : (wm0 + r16) * 128;
  const int b_at = B_LDS + key_row * (BN * 2) + (krow_piece<BN>(wn0 / 16, key_row) << 5) + part;
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  auto transposed = [&](const char *p, int row_bytes) RSVD_INLINE {
    const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(p)));
    const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(p + 4 * row_bytes)));
    return u32x4{lo[0], lo[1], hi[0], hi[1]};
  };
  // A barrier that waits for what was written to LDS but not for loads.
  auto meet = [&]() RSVD_INLINE {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(tile_wait(63));
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };

  // The matrix instructions of a tile, with the next one going to LDS in step.  (Behind the last tile that is one that nobody reads: no branches.)
  auto body = [&](int buf, auto from) RSVD_INLINE {
    constexpr int SET = decltype(from)::value;
    const int a_lds = a_at + buf * STAGE, b_lds = b_at + buf * STAGE;
    constexpr int STEPS = 2 / KG * TM;                 // rows of blocks, for either half of k or for the group's
    auto read_a = [&](int step, int q) RSVD_INLINE {
      const int h = KG == 1 ? step / TM : group, i = step % TM;
      return A_KROWS ? transposed(dense_lds + q * PLANE + (a_lds ^ (i << 5)) + h * 32 * A_ROW, A_ROW)
                     : *reinterpret_cast<const u32x4 *>(dense_lds + q * PLANE + a_lds + i * 2048 + (((4 * h + kq) ^ (r16 & 7)) << 4));
    };
    auto read_b = [&](int of, int j, int q) RSVD_INLINE {
      const int h = KG == 1 ? of : group;
      return transposed(dense_lds + q * PLANE + (b_lds ^ (j << 5)) + h * 32 * BN * 2, BN * 2);
    };
    constexpr int AHEAD = TM >= 4 ? 3 : 1;             // rows of blocks read ahead, not all of them: registers
    u32x4 a[AHEAD + 1][PL], b[2 / KG][TN][PL];
#pragma unroll
    for (int q = 0; q < PL; ++q) {
#pragma unroll
      for (int j = 0; j < TN; ++j) b[0][j][q] = read_b(0, j, q);
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) a[i][q] = read_a(i, q);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int step = 0; step < STEPS; ++step) {
      const int h = step / TM, i = step % TM;
#pragma unroll
      for (int q = 0; q < PL; ++q) {
        if (step + AHEAD < STEPS) a[(step + AHEAD) % (AHEAD + 1)][q] = read_a(step + AHEAD, q);
#pragma unroll
        for (int j = 0; j < TN; ++j)
          if (KG == 1 && h == 0 && i == j * TM / TN) b[KG == 1][j][q] = read_b(1, j, q);
      }
      with_segs<PL>([&](auto pa, auto pb) RSVD_INLINE {
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          const u32x4 x = b[h][j][decltype(pb)::value], y = a[step % (AHEAD + 1)][decltype(pa)::value];
          acc[i][j] = KIND == DK_BF16 ? mfma_bf16(x, y, acc[i][j]) : mfma_f16(x, y, acc[i][j]);
        }
      });
#pragma unroll
      for (int p = 0; p < PIECES; ++p)
        if (p * STEPS / PIECES == step) {
          write(SET, p, buf ^ 1);
          load(SET, p);
        }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // Tile kt goes through register set kt mod DEPTH.
  point();
#pragma unroll
  for (int set = 0; set < DEPTH; ++set) {
#pragma unroll
    for (int p = 0; p < PIECES; ++p) load(set, p);
    advance();
  }
#pragma unroll
  for (int p = 0; p < PIECES; ++p) {
    write(0, p, 0);
    load(0, p);
  }
  advance();
  meet();
  auto tile = [&](int buf, auto from) RSVD_INLINE {
    body(buf, from);
    advance();
    meet();
  };
  // (the tile behind goes to LDS out of the set that holds it)
  if constexpr (DEPTH == 1) {
    for (int kt = 0; kt < nkt; ++kt) tile(kt & 1, std::integral_constant<int, 0>());
  } else {
    for (int kt = 0; kt < nkt; kt += 2) {
      tile(0, std::integral_constant<int, 1>());
      if (kt + 1 < nkt) tile(1, std::integral_constant<int, 0>());
    }
  }
  float *const partial = work.partial != nullptr ? work.partial + wm0 * BN + wn0 : nullptr;
  int last_lane = lane;                                // (anew: what follows from it would be worked out before the main loop otherwise, and kept)
  asm volatile("" : "+v"(last_lane));
  // Of groups that have halves of k, each ends with one row of blocks: its own sums and the other's, through LDS (behind what the end takes, where there is room).
  // (behind the last meeting nobody reads the tiles)
  constexpr int ROWS = TM / KG;
  f32x4 sums[ROWS][TN];
  if constexpr (KG == 2) {
    constexpr int END = WGM * WGN * KG * finish_lds<TN>(), EXCHANGE = WGM * WGN * 2 * TN * 1024;
    constexpr bool APART = END + EXCHANGE <= 2 * STAGE;
    constexpr int ROOM = APART ? END : 0;
    static_assert(TM == 2 && END % 16 == 0 && ROOM + EXCHANGE <= 2 * STAGE, "a row of blocks a group");
    f32x4 *const mine = reinterpret_cast<f32x4 *>(dense_lds + ROOM) + wave * TN * 64 + last_lane;
    f32x4 *const other = reinterpret_cast<f32x4 *>(dense_lds + ROOM) + (wave + (group == 0 ? WGM * WGN : -WGM * WGN)) * TN * 64 + last_lane;
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      mine[j * 64] = group == 0 ? acc[1][j] : acc[0][j];
      sums[0][j] = group == 0 ? acc[0][j] : acc[1][j];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < TN; ++j) sums[0][j] += other[j * 64];
    if constexpr (!APART) __syncthreads();
  } else {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) sums[i][j] = acc[i][j];
  }
  const int below = KG == 1 ? 0 : 16 * group;
  float by = 1.f;
  if constexpr (KIND == DK_F16)
    if (P.out.scale != nullptr) by = *P.out.scale;
  dense_finish<BN, ROWS, TN>(P, sums, partial == nullptr ? nullptr : partial + below * BN, batch, m0 + wm0 + below, n0 + wn0, P.symmetric && tile_m != tile_n, last_lane,
                             reinterpret_cast<float *>(dense_lds + wave * finish_lds<TN>()), by);
}

template <int KIND, bool A_KROWS, int PL, int BM, int BN, int WGM, int WGN, int KG = 1, bool WIDE = false> hipError_t dense_kn_run(hipStream_t s, const DenseParams &P) {
  hipLaunchKernelGGL((dense_kn_kernel<KIND, A_KROWS, PL, BM, BN, WGM, WGN, KG, WIDE>), dim3(dense_groups(P)), dim3(64 * WGM * WGN * KG), (DenseKnCfg<PL, BM, BN>::lds), s, P);
  return hipGetLastError();
}
// The planes that small tiles of a kind take at once.
template <int KIND> constexpr int dense_kn_planes() { return KIND == DK_BF16 ? 3 : 2; }
template <int KIND, bool A_KROWS> hipError_t dense_kn_tile(hipStream_t s, const DenseParams &P, int b, bool wide) {
  if constexpr (KIND == DK_BF16)
    if (wide) return b == 64 && P.segs.count == 6 ? dense_kn_run<KIND, A_KROWS, 3, 64, 64, 2, 2, 2, true>(s, P) : hipErrorInvalidValue;
  if (b == 256) return dense_kn_run<KIND, A_KROWS, 1, 256, 256, 2, 4>(s, P);
  if (b == 128) return dense_kn_run<KIND, A_KROWS, 1, 128, 128, 2, 2>(s, P);
  if (P.segs.count > 1) return dense_kn_run<KIND, A_KROWS, dense_kn_planes<KIND>(), 64, 64, 2, 2, 2>(s, P);
  return dense_kn_run<KIND, A_KROWS, 1, 64, 64, 2, 2, 2>(s, P);
}
template <int KIND, bool A_KROWS> hipError_t dense_kn_init() {
  constexpr int PL = dense_kn_planes<KIND>();
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&dense_kn_kernel<KIND, A_KROWS, 1, 256, 256, 2, 4, 1, false>), hipFuncAttributeMaxDynamicSharedMemorySize,
                                           (int)DenseKnCfg<1, 256, 256>::lds);
  if (e != hipSuccess) return e;
  if constexpr (KIND == DK_BF16) {
    const hipError_t e2 = hipFuncSetAttribute(reinterpret_cast<const void *>(&dense_kn_kernel<KIND, A_KROWS, PL, 64, 64, 2, 2, 2, true>), hipFuncAttributeMaxDynamicSharedMemorySize,
                                              (int)DenseKnCfg<PL, 64, 64>::lds);
    if (e2 != hipSuccess) return e2;
  }
  return hipFuncSetAttribute(reinterpret_cast<const void *>(&dense_kn_kernel<KIND, A_KROWS, PL, 64, 64, 2, 2, 2, false>), hipFuncAttributeMaxDynamicSharedMemorySize,
                             (int)DenseKnCfg<PL, 64, 64>::lds);
}
#define DENSE_KN(KIND, A_KROWS)                                                                      \
  template hipError_t dense_kn_tile<KIND, A_KROWS>(hipStream_t s, const DenseParams &P, int b, bool wide);     \
  template hipError_t dense_kn_init<KIND, A_KROWS>();

}  // namespace rsvd
