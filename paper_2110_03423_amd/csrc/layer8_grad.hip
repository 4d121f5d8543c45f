// Products of bf16 numbers for gradients, C = sum over k of A_p[m][k] B[k][n], in the orders that the operands lie in memory.
//
// B runs along n from k to k, and so does A in the gradient of a weight, where k counts tokens.  Neither is transposed in memory:
// tiles [k][x] of bf16 numbers in LDS are read with the transposing LDS load (sixteen lanes read four k of sixteen columns and get one column of
// four k each).  LDS rows of such a tile have their 32-byte pieces exchanged by the low bits of k, so that the eight rows that half a wavefront
// reads start at different banks; rows of consecutive k have their 16-byte pieces exchanged by the row.
// Both operands go from memory to registers and from there to LDS, among the matrix instructions of the tile before, and a register is loaded
// for the tile after next (or, of small tiles, which are done before a load arrives, the one behind) as soon as it has been written.  (Loads
// straight to LDS: the compiler lets the transposing loads wait for all of them, wherever they go.) Large products are bound by power like
// those of codes (60 % of the matrix pipe's cycles at 1.8 GHz): gradient of a weight 16384 x 4096 over 16384 tokens 1805 to 1933 us (1.14 to
// 1.22 PFLOP/s; the library takes 1932 for operands in these orders), 4096 tokens of 16384 to 4096 in two planes 840 to 970 us (1.13 to 1.31).  Eight
// wavefronts of 128 x 64: four of 128 x 128 would have no registers left for what they stage. Several planes of A are taken as further k, the
// smallest first; by small tiles together with each k-tile of B, which is then staged and read once for all of them (2048 x 2048 x 1024
// tokens, three planes: 60 -> 47 us; larger tiles would have no room for two workgroups on a CU). Where few rows of tiles need it, B is taken
// as the 8-bit codes that it comes from and made bf16 numbers on the way to LDS.
#include <type_traits>

#include "layer8_rows.hpp"
#include "layer8_tile.hpp"

namespace rsvd {

constexpr int kKnK = 64;                   // k of a k-tile

struct KnParams {
  const char *A; int64_t lda, plane;       // bytes
  int planes, ktiles;                      // k-tiles of a plane
  int64_t K;
  const char *B; int64_t ldb;              // bytes
  const uint8_t *powers; int64_t ldp;      // of codes in the place of B: their powers of two, or NULL
  float *sums; int sum_columns;            // A_KROWS: sums of A over k by ranges, [split][sum_columns][M], or NULL
  int sums_whole, sums_accumulate;         // they are one row, and what is wanted (added to it)
  TileParams T;
};

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

// The same for codes: N pieces of sixteen codes of a row, as bf16 numbers in LDS.  POWERS: multiplied by their powers of two.
// (No branch between the loads: where it ends the compiler would wait for all of them.)
template <int NT, int X, bool POWERS, int DEPTH> struct StagedCodes {
  static constexpr int ROW = X * 2, PER = X / 16, STEP = NT / PER, N = X * kKnK / 16 / NT;
  static_assert(X * kKnK % (16 * NT) == 0 && STEP % 16 == 0, "whole rounds; a thread's rows have their pieces exchanged alike");
  u32x4 reg[DEPTH][N];
  unsigned unit[DEPTH][POWERS ? N : 1];
  uint32_t off[N], unit_off[POWERS ? N : 1];
  int place, half;
  __device__ __forceinline__ void init(int64_t ld, int64_t left, int tid, int64_t ldp) {
    const int row = tid / PER, pos = tid % PER, col = 16 * pos < left ? 16 * pos : 0;
    half = (pos & 1) << 4;                               // (neighbours start with different halves of their pieces: other banks)
    place = row * ROW + (krow_piece<X>(pos, row) << 5);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t r = row + STEP * i;
      off[i] = r * (uint32_t)ld + (uint32_t)col;
      asm volatile("" : "+v"(off[i]));
      if constexpr (POWERS) {
        unit_off[i] = r * (uint32_t)ldp + (uint32_t)(col >> 5);
        asm volatile("" : "+v"(unit_off[i]));
      }
    }
  }
  // base, powers: of the tile's first k and column; what is behind the last row is read as zeros, codes and units
  __device__ __forceinline__ void load(int set, int i, const char *base, int64_t ld, int k_left, const uint8_t *powers, int64_t ldp) {
    const __amdgpu_buffer_rsrc_t all = __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, (int)(k_left * (uint32_t)ld), 0x00027000);
    reg[set][i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(all, off[i], 0, 0));
    if constexpr (POWERS) {
      const __amdgpu_buffer_rsrc_t u = __builtin_amdgcn_make_buffer_rsrc((void *)powers, 0, (int)(k_left * (uint32_t)ldp), 0x00027000);
      unit[set][i] = __builtin_amdgcn_raw_buffer_load_b8(u, unit_off[i], 0, 0);
    }
  }
  __device__ __forceinline__ void write(int set, int i, char *lds) const {
    float by = 1.f;
    if constexpr (POWERS) by = kept_unit(unit[set][i]);
    u32x4 p[2];
    widen16(reg[set][i], by, p);
    char *at = lds + place + i * STEP * ROW;
    *reinterpret_cast<u32x4 *>(at + half) = half ? p[1] : p[0];
    *reinterpret_cast<u32x4 *>(at + (half ^ 16)) = half ? p[0] : p[1];
  }
};

template <int BM, int BN, int PL> struct KnCfg {
  static constexpr int A = BM * 128, B = BN * 128, STAGE = PL * A + B, DEPTH = BM == 256 ? 1 : 2;
  static constexpr size_t lds = 2 * (size_t)STAGE;      // (more than the wavefronts need in the end)
};

// PL planes of A are multiplied by a k-tile of B while it is in LDS; 1: the planes are further k.
template <bool A_KROWS, bool CODES, int PL, int BM, int BN, int WGM, int WGN>
__global__ __launch_bounds__(64 * WGM * WGN, 2) void kn_kernel(const KnParams P) {
  constexpr int NT = 64 * WGM * WGN, WM = BM / WGM, WN = BN / WGN, TM = WM / 16, TN = WN / 16, DEPTH = KnCfg<BM, BN, PL>::DEPTH;
  constexpr int STAGE = KnCfg<BM, BN, PL>::STAGE, A_BYTES = KnCfg<BM, BN, PL>::A, B_LDS = PL * A_BYTES;
  extern __shared__ __attribute__((aligned(16))) char kn_lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, kq = lane >> 4;
  const int wave_m = wave / WGN, wave_n = wave % WGN, wm0 = wave_m * WM, wn0 = wave_n * WN;
  int tile_m, tile_n, split;
  tile_of(P.T, tile_m, tile_n, split);
  const int64_t m0 = (int64_t)tile_m * BM, n0 = (int64_t)tile_n * BN;
  const int kt_begin = split * P.T.kt_per_split;
  const int nkt = split == P.T.splits ? 0 : P.T.kt_all - kt_begin < P.T.kt_per_split ? P.T.kt_all - kt_begin : P.T.kt_per_split;

  f32x4 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      acc[i][j] = (f32x4)0.f;
      pin<BM == 256>(acc[i][j]);
    }

  // k-tiles of the planes one after the other, the smallest plane first; next: the one that is loaded next
  int next_kt = __builtin_amdgcn_readfirstlane(kt_begin % P.ktiles), next_plane = __builtin_amdgcn_readfirstlane(kt_begin / P.ktiles);
  int64_t next_k = (int64_t)next_kt * kKnK;
  int next_left = (int)(P.K - next_k < kKnK ? P.K - next_k : kKnK);      // k of it that exist
  const char *const a_first = P.A + (A_KROWS ? m0 * 2 : m0 * P.lda), *const b_first = P.B + n0 * (CODES ? 1 : 2);
  Staged<NT, BM, A_KROWS, DEPTH * PL> sa;
  std::conditional_t<CODES, StagedCodes<NT, BN, A_KROWS, DEPTH>, Staged<NT, BN, true, DEPTH>> sb;
  sa.init(P.lda, P.T.M - m0, tid);
  if constexpr (CODES) sb.init(P.ldb, P.T.N - n0, tid, P.ldp);
  else sb.init(P.ldb, P.T.N - n0, tid);
  constexpr int NA = decltype(sa)::N, PIECES = PL * NA + decltype(sb)::N;
  auto load = [&](int set, int p) RSVD_INLINE {
    if (p < PL * NA) {
      const int plane = PL > 1 ? p / NA : P.planes - 1 - next_plane;
      sa.load(PL * set + p / NA, p % NA, a_first + plane * P.plane + (A_KROWS ? next_k * P.lda : next_k * 2), P.lda, next_left);
    } else if constexpr (CODES) sb.load(set, p - PL * NA, b_first + next_k * P.ldb, P.ldb, next_left, P.powers + next_k * P.ldp + n0 / 32, P.ldp);
    else sb.load(set, p - PL * NA, b_first + next_k * P.ldb, P.ldb, next_left);
  };
  auto write = [&](int set, int p, int buf) RSVD_INLINE {
    if (p < PL * NA) sa.write(PL * set + p / NA, p % NA, kn_lds + buf * STAGE + p / NA * A_BYTES);
    else sb.write(set, p - PL * NA, kn_lds + buf * STAGE + B_LDS);
  };
  auto advance = [&]() RSVD_INLINE {                    // (behind the last tile of this workgroup's range: loads stay inside the operands)
    next_k += kKnK;
    if (++next_kt == P.ktiles) {
      next_kt = 0;
      next_k = 0;
      if (PL == 1 && next_plane + 1 < P.planes) ++next_plane;
    }
    next_left = (int)(P.K - next_k < kKnK ? P.K - next_k : kKnK);
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

  // ---- sums of A over k
  // Large tiles: k-tile kt is summed by the tiles of column kt mod sum_columns, each wavefront its share of the rows.  Small ones: by the tiles of the first
  // column (sum_columns is 1), as products with ones of what is in registers anyway.
  constexpr int SHARE = A_KROWS ? (TM + WGN - 1) / WGN : 1;
  const bool sums_here = A_KROWS && P.sums != nullptr && tile_n < P.sum_columns;
  f32x4 asum[SHARE][PL];                               // (of each plane: no chain of instructions that wait for each other)
#pragma unroll
  for (int i = 0; i < SHARE; ++i)
#pragma unroll
    for (int q = 0; q < PL; ++q) asum[i][q] = (f32x4)0.f;
  int now_column = __builtin_amdgcn_readfirstlane(kt_begin % P.sum_columns);      // of the tile that is multiplied
  auto sum_a = [&](int buf) RSVD_INLINE {
    const int at = a_at + buf * STAGE, first = wave_n * SHARE;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < SHARE; ++i)
        if (first + i < TM) {
          const u32x4 v = transposed(kn_lds + (at ^ ((first + i) << 5)) + h * 32 * A_ROW, A_ROW);
#pragma unroll
          for (int e = 0; e < 4; ++e) asum[i][0][0] += bf16_low(v[e]) + bf16_high(v[e]);
        }
  };

  // The matrix instructions of a tile, with the next one going to LDS in step.  (Behind the last tile that is one that nobody reads: no
  // branches.)
  auto body = [&](int buf, auto from, auto sums) RSVD_INLINE {
    constexpr int SET = decltype(from)::value;
    constexpr bool SUMS = decltype(sums)::value;
    const int a_now = a_at + buf * STAGE, b_now = b_at + buf * STAGE;
    auto read_a = [&](int step, u32x4 (&to)[PL]) RSVD_INLINE {
      const int h = step / TM, i = step % TM;
#pragma unroll
      for (int q = 0; q < PL; ++q)
        to[q] = A_KROWS ? transposed(kn_lds + q * A_BYTES + (a_now ^ (i << 5)) + h * 32 * A_ROW, A_ROW)
                        : *reinterpret_cast<const u32x4 *>(kn_lds + q * A_BYTES + a_now + i * 2048 + (((4 * h + kq) ^ (r16 & 7)) << 4));
    };
    auto read_b = [&](int h, int j) RSVD_INLINE { return transposed(kn_lds + (b_now ^ (j << 5)) + h * 32 * BN * 2, BN * 2); };
    constexpr int AHEAD = TM >= 4 ? 3 : 1;             // rows of blocks read ahead, not all of them: registers
    u32x4 a[AHEAD + 1][PL], b[2][TN];
#pragma unroll
    for (int j = 0; j < TN; ++j) b[0][j] = read_b(0, j);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) read_a(i, a[i]);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int step = 0; step < 2 * TM; ++step) {
      const int h = step / TM, i = step % TM;
      if (step + AHEAD < 2 * TM) read_a(step + AHEAD, a[(step + AHEAD) % (AHEAD + 1)]);
#pragma unroll
      for (int j = 0; j < TN; ++j)
        if (h == 0 && i == j * TM / TN) b[1][j] = read_b(1, j);
#pragma unroll
      for (int q = PL - 1; q >= 0; --q)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = mfma_bf16(b[h][j], a[step % (AHEAD + 1)][q], acc[i][j]);
      if (SUMS && i / SHARE == wave_n) {
        const u32x4 ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
#pragma unroll
        for (int q = PL - 1; q >= 0; --q) asum[i % SHARE][q] = mfma_bf16(ones, a[step % (AHEAD + 1)][q], asum[i % SHARE][q]);
      }
#pragma unroll
      for (int p = 0; p < PIECES; ++p)
        if (p * (2 * TM) / PIECES == step) {
          write(SET, p, buf ^ 1);
          load(SET, p);
        }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // Tile kt goes through register set kt mod DEPTH.
  if (nkt > 0) {
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
  }
  auto tile = [&](int buf, auto from, auto sums) RSVD_INLINE {
    if (BM > 64 && sums_here && now_column == tile_n) sum_a(buf);
    body(buf, from, sums);
    advance();
    if (++now_column == P.sum_columns) now_column = 0;
    meet();
  };
  auto all = [&](auto sums) RSVD_INLINE {
    if constexpr (DEPTH == 1) {
      for (int kt = 0; kt < nkt; ++kt) tile(kt & 1, std::integral_constant<int, 0>(), sums);
    } else {
      for (int kt = 0; kt < nkt; kt += 2) {
        tile(0, std::integral_constant<int, 1>(), sums);
        if (kt + 1 < nkt) tile(1, std::integral_constant<int, 0>(), sums);
      }
    }
  };
  if constexpr (A_KROWS && BM == 64) {
    if (sums_here) all(std::true_type());
    else all(std::false_type());
  } else {
    all(std::false_type());
  }
  if (sums_here) {      // (no low-rank term there: split is a range of k)
#pragma unroll
    for (int i = 0; i < SHARE; ++i) {
      float sum = asum[i][PL - 1][0];
#pragma unroll
      for (int q = PL - 2; q >= 0; --q) sum += asum[i][q][0];
      if (BM > 64) {
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
      }
      const int64_t m = m0 + wm0 + (wave_n * SHARE + i) * 16 + r16;
      if (lane < 16 && wave_n * SHARE + i < TM && m < P.T.M) {
        float *to = P.sums + ((int64_t)split * P.sum_columns + tile_n) * P.T.M + m;
        *to = P.sums_whole && P.sums_accumulate ? *to + sum : sum;
      }
    }
  }
  int last_lane = lane;                                // (anew: what follows from it would be worked out before the main loop otherwise, and kept)
  asm volatile("" : "+v"(last_lane));
  // (behind the last meeting nobody reads the tiles)
  finish_tile<TM, TN, BM == 256>(P.T, acc, split, m0 + wm0, n0 + wn0, last_lane, reinterpret_cast<float *>(kn_lds + wave * finish_lds<TN>()));
}

// What is left to add up: ranges of k, and behind them sums of A, sixteen columns a workgroup with sixteen threads for the rows of each.
struct SumsParams { const float *sums; int64_t blocks, n; float *out; int accumulate; };
__global__ __launch_bounds__(256) void kn_end_kernel(const ReduceParams R, const SumsParams P) {
  if ((int64_t)blockIdx.x < R.groups) {
    reduce_group<false>(R, blockIdx.x);
    return;
  }
  const int col = threadIdx.x & 15, part = threadIdx.x >> 4;
  const int64_t j = ((int64_t)blockIdx.x - R.groups) * 16 + col;
  __shared__ float parts[16][17];
  float sum = 0.f;
  if (j < P.n) {
    for (int64_t b = part; b < P.blocks; b += 64) {
      float v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = b + 16 * u < P.blocks ? P.sums[(b + 16 * u) * P.n + j] : 0.f;
      sum += (v[0] + v[1]) + (v[2] + v[3]);
    }
  }
  parts[part][col] = sum;
  __syncthreads();
  if (threadIdx.x >= 16 || j >= P.n) return;
  sum = 0.f;
#pragma unroll
  for (int p = 0; p < 16; ++p) sum += parts[p][col];
  P.out[j] = P.accumulate ? P.out[j] + sum : sum;
}

static TileChoice kn_choose(const rsvd_ctx *ctx, int64_t M, int64_t N, int64_t K, int planes, bool lowrank) {
  return tile_choose(ctx, M, N, ceil_div(K, kKnK), planes, lowrank);
}
size_t kn_partial_bytes(const rsvd_ctx *ctx, int64_t M, int64_t N, int64_t K, int planes, bool lowrank) {
  return tile_partial_bytes(kn_choose(ctx, M, N, K, planes, lowrank), M, N, lowrank);
}
// Columns of tiles that share the sums of A.  (Small tiles with one range of k need no launch to add them up: 1000 x 1000 x 1000 bf16 15.2 -> 13.5 us.  128
// rows and columns have no registers for it.)
static int64_t kn_sum_columns(const TileChoice &c, int64_t N) {
  const int64_t most = c.bm == 64 ? 1 : 8;
  return ceil_div(N, c.bn) < most ? ceil_div(N, c.bn) : most;
}
int64_t kn_sum_rows(const rsvd_ctx *ctx, int64_t M, int64_t N, int64_t K, int planes) {
  const TileChoice c = kn_choose(ctx, M, N, K, planes, false);
  return c.splits * kn_sum_columns(c, N);
}

template <bool A_KROWS, bool CODES, int PL, int BM, int BN, int WGM, int WGN> static hipError_t kn_run(hipStream_t s, const KnParams &P) {
  hipLaunchKernelGGL((kn_kernel<A_KROWS, CODES, PL, BM, BN, WGM, WGN>), dim3(tile_groups(P.T)), dim3(64 * WGM * WGN), (KnCfg<BM, BN, PL>::lds), s, P);
  return hipGetLastError();
}

template <bool A_KROWS, bool CODES> static hipError_t kn_run_small(hipStream_t s, const KnParams &P, int bm) {
  if (bm == 128) return kn_run<A_KROWS, CODES, 1, 128, 128, 2, 2>(s, P);
  if constexpr (A_KROWS)                                  // (the other's are two or three)
    if (P.planes == 1) return kn_run<A_KROWS, CODES, 1, 64, 64, 2, 2>(s, P);
  return P.planes == 2 ? kn_run<A_KROWS, CODES, 2, 64, 64, 2, 2>(s, P) : kn_run<A_KROWS, CODES, 3, 64, 64, 2, 2>(s, P);
}
template <bool A_KROWS> static hipError_t kn_run_tile(hipStream_t s, const KnParams &P, int bm, bool codes) {
  if (bm == 256) return kn_run<A_KROWS, false, 1, 256, 256, 2, 4>(s, P);
  return codes ? kn_run_small<A_KROWS, true>(s, P, bm) : kn_run_small<A_KROWS, false>(s, P, bm);
}

// Every row of tiles makes bf16 numbers of all the codes again, and so does every plane that is further k; a matrix of them is made once and read twice as
// long.  Rows of tiles (times such planes) up to which the codes are taken as they are, measured as codes / matrix.  Weight: 4096 x 4096 codes with
// 64 columns of dY in bf16 (1) 18 / 34 us, fp32 (1) 23 / 33, 256 of bf16 (4) 31 / 42, 512 (8) 49 / 51, 512 of fp16 (8) 68 / 66; 2048 x 2048 with 1024 of
// bf16 (16) 28 / 33.  X, where a launch before the product is needed anyway: 4096 x 4096 codes and 64 tokens (1) 20 / 34 us (bf16, fp16) and 22 / 35 (fp32),
// 128 (2) 25 / 34 and 30 / 38, 256 (4) 35 / 42 and 43 / 50; 128 tokens with 16384 x 4096 codes (2) 60 / 92 and 73 / 111.  (Not at its end: with 320
// (5) 44 / 50 and 55 / 61, 512 (8) 56 / 61 and 71 / 75, 301 tokens of 2000 x 1410 (5) 19 / 21 and 25 / 28.)
bool kn_takes_codes(const rsvd_ctx *ctx, bool a_krows, int64_t M, int64_t N, int64_t K, int planes, bool lowrank, int64_t ldc,
                    int64_t ldp) {
  const TileChoice c = kn_choose(ctx, M, N, K, planes, lowrank);
  return c.bm < 256 && ceil_div(M, c.bm) * (c.bm == 64 ? 1 : planes) <= (a_krows ? 16 : 4) && ldc <= kMaxLd && ldp <= kMaxLd;
}

hipError_t nt_init_device();
hipError_t layer8_init_device(rsvd_ctx *) {
  hipError_t e = nt_init_device();
  const void *wide[2] = {reinterpret_cast<const void *>(&kn_kernel<true, false, 1, 256, 256, 2, 4>),
                         reinterpret_cast<const void *>(&kn_kernel<false, false, 1, 256, 256, 2, 4>)};
  for (const void *k : wide)
    if (e == hipSuccess) e = hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, (int)KnCfg<256, 256, 1>::lds);
  return e;
}

hipError_t kn_launch(rsvd_ctx *ctx, hipStream_t s, const KnDesc &d) {
  const TileChoice c = kn_choose(ctx, d.M, d.N, d.K, d.planes, d.out.r > 0);
  const int64_t ktiles = ceil_div(d.K, kKnK), kt = c.kt;
  if (c.splits > 1 && (d.partial == nullptr || d.partial_bytes < tile_partial_bytes(c, d.M, d.N, d.out.r > 0))) return hipErrorInvalidValue;
  KnParams P;
  P.A = (const char *)d.A; P.lda = d.lda; P.plane = d.plane; P.planes = d.planes;
  P.ktiles = (int)ktiles; P.K = d.K;
  P.B = (const char *)d.B; P.ldb = d.ldb;
  const bool codes = d.codes != nullptr;
  if (codes) {
    if (!kn_takes_codes(ctx, d.a_krows, d.M, d.N, d.K, d.planes, d.out.r > 0, d.ldc, d.ldp)) return hipErrorInvalidValue;
    P.B = (const char *)d.codes; P.ldb = d.ldc;
  }
  P.powers = d.powers; P.ldp = d.ldp;
  P.sums = d.a_krows ? d.sums : nullptr;
  P.sum_columns = (int)kn_sum_columns(c, d.N);
  P.sums_whole = c.splits * P.sum_columns == 1;
  P.sums_accumulate = d.out.accumulate;
  if (P.sums != nullptr && P.sums_whole) P.sums = d.sums_out;
  P.T = tile_params(c, d.M, d.N, kt, d.partial, d.out);
  const hipError_t e = d.a_krows ? kn_run_tile<true>(s, P, c.bm, codes) : kn_run_tile<false>(s, P, c.bm, codes);
  const ReduceParams R = reduce_params(P.T);
  const SumsParams S = {P.sums, (int64_t)c.splits * P.sum_columns, d.M, d.sums_out, d.out.accumulate};
  const int64_t groups = R.groups + (P.sums != nullptr && !P.sums_whole ? ceil_div(d.M, 16) : 0);
  if (e != hipSuccess || groups == 0) return e;
  hipLaunchKernelGGL(kn_end_kernel, dim3((unsigned)groups), dim3(256), 0, s, R, S);
  return hipGetLastError();
}

}  // namespace rsvd
