// What the product kernels of the layer operators for many tokens have in common: tiles, ranges of k, and the end of a tile.
#pragma once

#include <type_traits>

#include "layer8_epilogue.hpp"

namespace rsvd {

struct TileParams {
  int64_t M, N;
  int tiles_m, tiles_n, splits, kt_all, kt_per_split;      // k-tiles
  float *partial;                          // splits > 1: [split][M][N], integers for codes; behind them the low-rank term [M][N] if there is one
  Layer8Epilogue E;
};

// Operand of s_waitcnt: at most n vector memory operations outstanding, no LDS operation.
constexpr int tile_wait(int n) { return (n & 15) | ((n >> 4) << 14) | 0x0070; }

// Tiles: a contiguous run for each of the eight XCDs (which have an L2 each), and within it strips of eight rows of tiles, column by column.
__device__ __forceinline__ void tile_of(const TileParams &P, int &tile_m, int &tile_n, int &split) {
  const int total = (int)gridDim.x, pid = (int)blockIdx.x;
  const int per = (total + 7) >> 3, tall = (total & 7) ? (total & 7) : 8, xcd = pid & 7, local = pid >> 3;
  int t = xcd < tall ? xcd * per + local : tall * per + (xcd - tall) * (per - 1) + local;
  const int grid_mn = P.tiles_m * P.tiles_n;
  // (the quotients are worked out in vector registers, where all that follows from them would stay)
  split = __builtin_amdgcn_readfirstlane(t / grid_mn);
  t -= split * grid_mn;
  const int strip = __builtin_amdgcn_readfirstlane(t / (8 * P.tiles_n)), first = strip * 8;
  const int high = P.tiles_m - first < 8 ? P.tiles_m - first : 8;
  t -= strip * 8 * P.tiles_n;
  tile_n = __builtin_amdgcn_readfirstlane(t / high);
  tile_m = first + t - tile_n * high;
}

// Bytes of LDS that a wavefront with TN blocks side by side needs to store them.
template <int TN> constexpr int finish_lds() { return 16 * (16 * TN + 4) * 4; }

// Stores a wavefront's blocks through LDS, sixteen rows at a time, so that lanes next to each other write what is next to each other.  The
// value of block (i, j) that lane L has are row 16 i + L % 16 and four columns from 16 j + 4 (L / 16) on.  Where all rows and columns exist, what
// sixteen rows hold is read at once and stored without a look at each.
template <int TYPE, int TM, int TN, typename vec_t>
__device__ __forceinline__ void store_blocks(const Layer8Epilogue &E, int64_t M, int64_t N, const vec_t (&val)[TM][TN], int64_t m1, int64_t n1,
                                             int lane, float *lds) {
  constexpr int PITCH = 16 * TN + 4, PER_ROW = 4 * TN, ROWS = 64 / PER_ROW, PASSES = 16 / ROWS, SIZE = TYPE == RSVD_X_F32 ? 4 : 2;
  const int r16 = lane & 15, kq = lane >> 4, row = lane / PER_ROW, col = 4 * (lane % PER_ROW);
  const int64_t n = n1 + col;
  const bool whole = m1 + 16 * TM <= M && n1 + 16 * TN <= N && E.accumulate == 0;
  char *const c = reinterpret_cast<char *>(E.C) + ((m1 + row) * E.ldc + n) * SIZE;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
#pragma unroll
    for (int j = 0; j < TN; ++j) *reinterpret_cast<vec_t *>(lds + r16 * PITCH + 16 * j + 4 * kq) = val[i][j];
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
    if (whole) {
      f32x4 v[PASSES];
#pragma unroll
      for (int p = 0; p < PASSES; ++p) v[p] = *reinterpret_cast<const f32x4 *>(lds + (p * ROWS + row) * PITCH + col);
#pragma unroll
      for (int p = 0; p < PASSES; ++p) {
        char *at = c + (int64_t)(16 * i + p * ROWS) * E.ldc * SIZE;
        if constexpr (TYPE == RSVD_X_F32) *reinterpret_cast<f32x4_any *>(at) = v[p];
        else *reinterpret_cast<u32x2_any *>(at) = halves4<TYPE>(v[p]);
      }
    } else {
#pragma unroll 1
      for (int p = 0; p < PASSES; ++p) {
        const int64_t m = m1 + 16 * i + p * ROWS + row;
        const f32x4 v = *reinterpret_cast<const f32x4 *>(lds + (p * ROWS + row) * PITCH + col);
        if (m < M && n < N) store4<TYPE>(E, m, n, N, v);
      }
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
  }
}

// Keeps sums in the accumulation registers, half of what a wavefront of the largest tiles has: among the others the compiler moves them about in the
// main loop, and spills.  (The ends of the 256 x 256 kernels still spill, 83 to 104 registers: operands of the low-rank term and of the stores, outside of the
// loop over k.)
template <bool PIN, typename vec_t> __device__ __forceinline__ void pin(vec_t &v) {
  if constexpr (PIN) {
    asm volatile("" : "+a"(v));
    __builtin_amdgcn_sched_barrier(0);                  // (one after the other, or they are all fetched at once)
  }
}

// The end of a wavefront's TM x TN blocks of 16 x 16, whose first is at (m1, n1).  lds: the wavefront's finish_lds<TN>() bytes; nobody
// reads them any more.
template <int TM, int TN, bool PIN, typename acc_t>
__device__ __forceinline__ void finish_tile(const TileParams &P, acc_t (&acc)[TM][TN], int split, int64_t m1, int64_t n1, int lane, float *lds) {
  const int r16 = lane & 15, kq = lane >> 4;
  const Layer8Epilogue &E = P.E;
  Layer8Epilogue W = E;
  f32x4 val[TM][TN];
  if (P.splits > 1) {
    // A part of the sums.  Those of codes stay integers, so that however k was divided the sum is exact; the low-rank term is a part of
    // its own, behind the others, by workgroups that have no k-tiles.
    W.C = P.partial + (int64_t)split * P.M * P.N;
    W.ldc = P.N;
    W.type = RSVD_X_F32;
    W.accumulate = 0;
    W.bias = nullptr;
    if (split < P.splits) W.rp = 0;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        val[i][j] = __builtin_bit_cast(f32x4, acc[i][j]);
        pin<PIN>(val[i][j]);
      }
  } else {
    float rs[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int64_t m = m1 + i * 16 + r16;
      rs[i] = E.rs != nullptr ? E.rs[m < P.M ? m : P.M - 1] : 1.f;
    }
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const f32x4 cs = column4(E.cs, n1 + j * 16 + 4 * kq, P.N, 1.f);
#pragma unroll
      for (int i = 0; i < TM; ++i) {
#pragma unroll
        for (int v = 0; v < 4; ++v) val[i][j][v] = (float)acc[i][j][v] * rs[i] * cs[v];
        pin<PIN>(val[i][j]);
      }
    }
  }
  // the low-rank term; the operands of a step are loaded during the one before
  const int steps = W.parts * W.rp / 32;
  if (steps > 0) {
    u32x4 a[2][TM], b[2][TN];
    auto fetch = [&](auto set, int step) RSVD_INLINE {
      constexpr int S = decltype(set)::value;
      const int p = 32 * step, pr = p % W.rp + 8 * kq;
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const int64_t n = n1 + j * 16 + r16;
        b[S][j] = factor8(E, n < P.N ? n : P.N - 1, pr);
      }
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const int64_t m = m1 + i * 16 + r16;
        a[S][i] = *reinterpret_cast<const u32x4 *>(E.t + (m < P.M ? m : P.M - 1) * E.parts * E.rp + p + 8 * kq);
      }
    };
    auto multiply = [&](auto set) RSVD_INLINE {
      constexpr int S = decltype(set)::value;
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) val[i][j] = mfma_bf16(b[S][j], a[S][i], val[i][j]);
    };
    fetch(std::integral_constant<int, 0>(), 0);
#pragma unroll 1
    for (int step = 0; step < steps; step += 2) {
      if (step + 1 < steps) fetch(std::integral_constant<int, 1>(), step + 1);
      __builtin_amdgcn_sched_barrier(0);
      multiply(std::integral_constant<int, 0>());
      __builtin_amdgcn_sched_barrier(0);
      if (step + 1 >= steps) break;
      if (step + 2 < steps) fetch(std::integral_constant<int, 0>(), step + 2);
      __builtin_amdgcn_sched_barrier(0);
      multiply(std::integral_constant<int, 1>());
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  if (W.bias != nullptr) {
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const f32x4 bias = column4(W.bias, n1 + j * 16 + 4 * kq, P.N, 0.f);
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        val[i][j] += bias;
        pin<PIN>(val[i][j]);
      }
    }
  }
  if (W.type == RSVD_X_F32) store_blocks<RSVD_X_F32>(W, P.M, P.N, val, m1, n1, lane, lds);
  else if (W.type == RSVD_X_BF16) store_blocks<RSVD_X_BF16>(W, P.M, P.N, val, m1, n1, lane, lds);
  else store_blocks<RSVD_X_F16>(W, P.M, P.N, val, m1, n1, lane, lds);
}

// The parts of sums over k, added in their order, and the rest of the epilogue.
struct ReduceParams {
  const float *partial; int splits;
  int64_t M, N, groups;            // groups: workgroups that share the work
  Layer8Epilogue E;
};
template <bool CODES> __device__ __forceinline__ void reduce_group(const ReduceParams &P, int64_t group) {
  const float *__restrict__ partial = P.partial;
  const Layer8Epilogue &E = P.E;
  const int64_t M = P.M, N = P.N;
  typedef typename std::conditional<CODES, i32x4, f32x4>::type acc_t;
  typedef typename std::conditional<CODES, int, float>::type one_t;
  const int64_t per_row = (N + 3) / 4, total = M * per_row;
  for (int64_t e = group * 256 + threadIdx.x; e < total; e += P.groups * 256) {
    const int64_t m = e / per_row, n = (e - m * per_row) * 4;
    auto part = [&](int s, auto zero) RSVD_INLINE {
      typedef decltype(zero) vec;
      vec v = zero;
      const float *p = partial + ((int64_t)s * M + m) * N + n;
      if (n + 4 <= N) {
        v = __builtin_bit_cast(vec, *reinterpret_cast<const f32x4_any *>(p));
      } else {
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (n + u < N) {
            if constexpr (std::is_same<vec, i32x4>::value) v[u] = reinterpret_cast<const int *>(p)[u];
            else v[u] = p[u];
          }
      }
      return v;
    };
    acc_t sum = (acc_t)(one_t)0;
#pragma unroll 4
    for (int s = 0; s < P.splits; ++s) sum += part(s, (acc_t)(one_t)0);
    const float rs = E.rs != nullptr ? E.rs[m] : 1.f;
    const f32x4 cs = column4(E.cs, n, N, 1.f);
    f32x4 val;
#pragma unroll
    for (int v = 0; v < 4; ++v) val[v] = (float)sum[v] * rs * cs[v];
    if (E.r > 0) val += part(P.splits, (f32x4)0.f);
    if (E.bias != nullptr) val += column4(E.bias, n, N, 0.f);
    store4(E, m, n, N, val);
  }
}


// Tile and ranges of k for kt k-tiles of each of `planes` matrices A.  Small tiles take a k-tile of all planes at once, others one after
// the other (TileChoice::kt in all).  lowrank: a low-rank term is added.
struct TileChoice { int bm, bn, splits; int64_t kt_per_split, kt; };
TileChoice tile_choose(const rsvd_ctx *ctx, int64_t M, int64_t N, int64_t kt, int planes, bool lowrank);
inline size_t tile_partial_bytes(const TileChoice &c, int64_t M, int64_t N, bool lowrank) {
  return c.splits > 1 ? (size_t)(c.splits + (lowrank ? 1 : 0)) * M * N * 4 : 0;
}
inline TileParams tile_params(const TileChoice &c, int64_t M, int64_t N, int64_t kt, float *partial, const Layer8Out &out) {
  TileParams P;
  P.M = M; P.N = N;
  P.tiles_m = (int)ceil_div(M, c.bm); P.tiles_n = (int)ceil_div(N, c.bn);
  P.splits = c.splits; P.kt_all = (int)kt; P.kt_per_split = (int)c.kt_per_split;
  P.partial = partial;
  P.E = layer8_epilogue(out);
  return P;
}
// Workgroups of a product.
inline unsigned tile_groups(const TileParams &P) {
  return (unsigned)((int64_t)P.tiles_m * P.tiles_n * (P.splits > 1 && P.E.r > 0 ? P.splits + 1 : P.splits));
}
// groups: 0 where there is one range of k, and nothing to add
inline ReduceParams reduce_params(const TileParams &P) {
  int64_t groups = P.splits <= 1 ? 0 : ceil_div(P.M * ceil_div(P.N, 4), 256);
  if (groups > 4096) groups = 4096;
  return ReduceParams{P.partial, P.splits, P.M, P.N, groups, P.E};
}

}  // namespace rsvd
