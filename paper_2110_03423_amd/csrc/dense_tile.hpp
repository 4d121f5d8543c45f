// What the product kernels of the gated block's operators have in common: places of tiles, and the end of a tile.
#pragma once

#include "dense.hpp"
#include "layer8_tile.hpp"

namespace rsvd {

struct DenseParams {
  const char *A, *B;
  int64_t lda, ldb, a_plane, b_plane, a_batch, b_batch;      // bytes
  int64_t b_up;                            // gated: bytes from a gate row to its up row
  const uint8_t *a_pow, *b_pow; int64_t ld_apow, ld_bpow; int a_shift, b_shift;
  DenseSegs segs;
  int64_t M, N, K;
  int ktiles, tiles_m, tiles_n, tiles, splits, kt_all, kt_per_split, batch;      // tiles: of a problem; k-tiles: of a part of k, and of all
  int symmetric;
  float *partial;                          // splits > 1: [batch][split][M][columns], of gated products gate and up side by side
  LinearOut out;
  GatedOut gate;
};

__device__ __forceinline__ f32x4 mfma_f16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Tiles: a contiguous run for each of the eight XCDs, which have an L2 each, problem by problem, range of k by range of k.  Within one, strips of eight rows of
// tiles, column by column; of symmetric results the tiles on and below the diagonal, row by row.
__device__ __forceinline__ void dense_tile_of(const DenseParams &P, int &tile_m, int &tile_n, int &split, int &batch) {
  const int total = (int)gridDim.x, pid = (int)blockIdx.x;
  const int per = (total + 7) >> 3, tall = (total & 7) ? (total & 7) : 8, xcd = pid & 7, local = pid >> 3;
  int t = xcd < tall ? xcd * per + local : tall * per + (xcd - tall) * (per - 1) + local;
  batch = __builtin_amdgcn_readfirstlane(t / (P.tiles * P.splits));
  t -= batch * P.tiles * P.splits;
  split = __builtin_amdgcn_readfirstlane(t / P.tiles);
  t -= split * P.tiles;
  if (P.symmetric) {
    int row = (int)((__builtin_sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
    while (row * (row + 1) / 2 > t) --row;                // (the root is rounded)
    while ((row + 1) * (row + 2) / 2 <= t) ++row;
    tile_m = __builtin_amdgcn_readfirstlane(row);
    tile_n = __builtin_amdgcn_readfirstlane(t - row * (row + 1) / 2);
    return;
  }
  const int strip = __builtin_amdgcn_readfirstlane(t / (8 * P.tiles_n)), first = strip * 8;
  const int high = P.tiles_m - first < 8 ? P.tiles_m - first : 8;
  t -= strip * 8 * P.tiles_n;
  tile_n = __builtin_amdgcn_readfirstlane(t / high);
  tile_m = first + t - tile_n * high;
}

// ---------------------------------------------------------------- four consecutive results
template <int TYPE> __device__ __forceinline__ f32x4 load4(const void *p, int64_t at, int left) {
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if constexpr (TYPE == RSVD_X_F32) {
    const float *c = reinterpret_cast<const float *>(p) + at;
    if (left >= 4) v = *reinterpret_cast<const f32x4_any *>(c);
    else
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = e < left ? c[e] : 0.f;
  } else {
    const uint16_t *c = reinterpret_cast<const uint16_t *>(p) + at;
    u32x2 w = {0u, 0u};
    if (left >= 4) w = *reinterpret_cast<const u32x2_any *>(c);
    else
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (e < left) w[e >> 1] |= (unsigned)c[e] << (16 * (e & 1));
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const unsigned pair = w[h];
      if constexpr (TYPE == RSVD_X_BF16) {
        v[2 * h] = bf16_low(pair);
        v[2 * h + 1] = bf16_high(pair);
      } else {
        const f16x2 f = __builtin_bit_cast(f16x2, pair);
        v[2 * h] = (float)f[0];
        v[2 * h + 1] = (float)f[1];
      }
    }
  }
  return v;
}
template <int TYPE> __device__ __forceinline__ void put4(void *p, int64_t at, int left, f32x4 v) {
  if constexpr (TYPE == RSVD_X_F32) {
    float *c = reinterpret_cast<float *>(p) + at;
    if (left >= 4) *reinterpret_cast<f32x4_any *>(c) = v;
    else
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (e < left) c[e] = v[e];
  } else {
    uint16_t *c = reinterpret_cast<uint16_t *>(p) + at;
    const u32x2 w = halves4<TYPE>(v);
    if (left >= 4) *reinterpret_cast<u32x2_any *>(c) = w;
    else
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (e < left) c[e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
  }
}
__device__ __forceinline__ f32x4 load4(int type, const void *p, int64_t at, int left) {
  return type == RSVD_X_F32 ? load4<RSVD_X_F32>(p, at, left) : type == RSVD_X_BF16 ? load4<RSVD_X_BF16>(p, at, left) : load4<RSVD_X_F16>(p, at, left);
}
__device__ __forceinline__ void put4(int type, void *p, int64_t at, int left, f32x4 v) {
  if (type == RSVD_X_F32) put4<RSVD_X_F32>(p, at, left, v);
  else if (type == RSVD_X_BF16) put4<RSVD_X_BF16>(p, at, left, v);
  else put4<RSVD_X_F16>(p, at, left, v);
}
__device__ __forceinline__ int left_of(int64_t n, int64_t N) { return N - n >= 4 ? 4 : (int)(N - n); }

// Columns n to n + 3 of row m, of which those before `width` are stored and those from N on are zeros.
__device__ __forceinline__ void linear_end(const LinearOut &O, int64_t N, int batch, int64_t m, int64_t n, f32x4 v) {
  const int have = left_of(n, N), left = left_of(n, O.width);
  v *= O.alpha;
  if (O.D != nullptr) {
    const uint16_t *d = O.D + batch * O.d_batch;
    f32x4 sum = load4<RSVD_X_F16>(d, m * O.ldd + n, have);
    if (O.d_planes == 2) sum += load4<RSVD_X_F16>(d + O.d_plane / 2, m * O.ldd + n, have);
    v += O.beta * sum;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = e < have ? v[e] : 0.f;
  const int64_t at = batch * O.c_batch + m * O.ldc + n;
  if (O.planes == 2) {
    put4<RSVD_X_F16>(O.C, at, left, v);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] -= (float)(_Float16)v[e];
    put4<RSVD_X_F16>(reinterpret_cast<char *>(O.C) + O.c_plane, at, left, v);
    return;
  }
  if (O.accumulate) v += load4(O.type, O.C, at, left);
  put4(O.type, O.C, at, left, v);
}

// The activation (g times a share of it) and its derivative.  The shares are written so that none is a difference of numbers near one: 1 / 2 + erf / 2 as a
// complement, 1 / 2 + tanh(y) / 2 as 1 / (1 + exp(-2 y)).
__device__ __forceinline__ float act_share(int act, float g) {
  if (act == GATED_SILU) return 1.f / (1.f + __expf(-g));
  if (act == GATED_GELU) return 0.5f * erfcf(-0.70710678f * g);
  return 1.f / (1.f + __expf(-1.5957691f * (g + 0.044715f * g * g * g)));
}
__device__ __forceinline__ float act_value(int act, float g) {
  if (act == GATED_RELU) return g > 0.f ? g : g != g ? g : 0.f;
  return g * act_share(act, g);
}
__device__ __forceinline__ float act_slope(int act, float g, float &value) {
  if (act == GATED_RELU) {
    value = g > 0.f ? g : g != g ? g : 0.f;
    return g > 0.f ? 1.f : 0.f;
  }
  const float s = act_share(act, g);
  value = g * s;
  if (act == GATED_SILU) return s + value * (1.f - s);
  if (act == GATED_GELU) return s + g * __expf(-0.5f * g * g) * 0.39894228f;
  return s + value * (1.f - s) * 1.5957691f * (1.f + 0.134145f * g * g);
}

// Gradients of gate and up, four columns from n on, to the planes of D (gate from column 0 on, up from column m on).
__device__ __forceinline__ void slope_end(const GatedOut &O, int64_t N, int64_t m, int64_t n, f32x4 g, f32x4 u) {
  const int left = left_of(n, N);
  const f32x4 dh = load4(O.type, O.dH, m * O.lddh + n, left);
  f32x4 dg, du;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float value;
    const float slope = act_slope(O.act, g[e], value);
    dg[e] = dh[e] * u[e] * slope;
    du[e] = dh[e] * value;
  }
  const int64_t at = m * O.ldD + n;
  if (n + 4 >= N)                                        // (the zeros behind them)
    for (int64_t c = 2 * N; c < O.ldD; ++c)
      for (int q = 0; q < (O.type == RSVD_X_F32 ? 3 : 1); ++q) O.D[q * (O.plane / 2) + m * O.ldD + c] = 0;
  if (O.type == RSVD_X_F16) {
    put4<RSVD_X_F16>(O.D, at, left, dg);
    put4<RSVD_X_F16>(O.D, at + N, left, du);
  } else if (O.type == RSVD_X_BF16) {
    put4<RSVD_X_BF16>(O.D, at, left, dg);
    put4<RSVD_X_BF16>(O.D, at + N, left, du);
  } else {
    unsigned p[2][2][3];
    bf16_parts2<3>(dg[0], dg[1], p[0][0]);
    bf16_parts2<3>(dg[2], dg[3], p[0][1]);
    bf16_parts2<3>(du[0], du[1], p[1][0]);
    bf16_parts2<3>(du[2], du[3], p[1][1]);
#pragma unroll
    for (int q = 0; q < 3; ++q)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint16_t *c = O.D + q * (O.plane / 2) + at + h * N;
        if (left >= 4) *reinterpret_cast<u32x2_any *>(c) = u32x2{p[h][0][q], p[h][1][q]};
        else
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (e < left) c[e] = (uint16_t)(p[h][e >> 1][q] >> (16 * (e & 1)));
      }
  }
}

__device__ __forceinline__ void gated_end(const GatedOut &O, int64_t N, int64_t m, int64_t n, f32x4 g, f32x4 u) {
  if (O.dH != nullptr) {
    slope_end(O, N, m, n, g, u);
    return;
  }
  const int left = left_of(n, N);
  f32x4 h;
#pragma unroll
  for (int e = 0; e < 4; ++e) h[e] = act_value(O.act, g[e]) * u[e];
  put4(O.type, O.H, m * O.ldh + n, left, h);
  if (O.kept != nullptr) {
    put4(O.type, O.kept, m * O.ldk + n, left, g);
    put4(O.type, O.kept, m * O.ldk + N + n, left, u);
  }
}

// ---------------------------------------------------------------- the end of a wavefront's TM x TN blocks of 16 x 16
// Through LDS, sixteen rows at a time, so that lanes next to each other write what is next to each other: block (i, j) of lane L holds row 16 i + L % 16 and
// four columns from 16 j + 4 (L / 16) on.  gated: blocks are gate and up in turn, (m1, n1) counts outputs.  lds: the wavefront's finish_lds<TN>() bytes.
template <bool GATED, int TM, int TN>
__device__ __forceinline__ void dense_finish(const DenseParams &P, f32x4 (&acc)[TM][TN], int split, int batch, int64_t m1, int64_t n1, bool mirror, int lane, float *lds) {
  constexpr int PITCH = 16 * TN + 4, PER_ROW = (GATED ? 2 : 4) * TN, ROWS = 64 / PER_ROW, PASSES = 16 / ROWS;
  const int r16 = lane & 15, kq = lane >> 4, row = lane / PER_ROW, col = 4 * (lane % PER_ROW);
  const int at = GATED ? 32 * (col / 16) + col % 16 : col;
  const int64_t columns = GATED ? 2 * P.N : P.N, n = n1 + col;
  float *const partial = P.partial + ((int64_t)batch * P.splits + split) * P.M * columns;
  const int64_t width = GATED || P.splits > 1 ? P.N : P.out.width;
#pragma unroll 1
  for (int i = 0; i < TM; ++i) {                        // (one copy of what follows, not one for each row of blocks)
#pragma unroll
    for (int x = 0; x < TM; ++x)
      if (i == x) {
#pragma unroll
        for (int j = 0; j < TN; ++j) *reinterpret_cast<f32x4 *>(lds + r16 * PITCH + 16 * j + 4 * kq) = acc[x][j];
      }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
#pragma unroll 1
    for (int p = 0; p < PASSES; ++p) {
      const float *from = lds + (p * ROWS + row) * PITCH + at;
      const int64_t m = m1 + 16 * i + p * ROWS + row;
      const f32x4 v = *reinterpret_cast<const f32x4 *>(from);
      if (m < P.M && n < width) {
        if constexpr (GATED) {
          const f32x4 u = *reinterpret_cast<const f32x4 *>(from + 16);
          if (P.splits > 1) {
            put4<RSVD_X_F32>(partial, m * columns + n, left_of(n, P.N), v);
            put4<RSVD_X_F32>(partial, m * columns + P.N + n, left_of(n, P.N), u);
          } else {
            gated_end(P.gate, P.N, m, n, v, u);
          }
        } else if (P.splits > 1) {
          put4<RSVD_X_F32>(partial, m * columns + n, left_of(n, P.N), v);
        } else {
          linear_end(P.out, P.N, batch, m, n, v);
        }
      }
    }
    if (!GATED && mirror) {                             // rows and columns exchanged: lane e has column e / 4 and four of the rows
#pragma unroll 1
      for (int e = lane; e < 64 * TN; e += 64) {
        const int c = e >> 2, q = 4 * (e & 3);
        f32x4 v;
#pragma unroll
        for (int x = 0; x < 4; ++x) v[x] = lds[(q + x) * PITCH + c];
        const int64_t mm = n1 + c, nn = m1 + 16 * i + q;
        if (mm < P.M && nn < width) {
          if (P.splits > 1) put4<RSVD_X_F32>(partial, mm * columns + nn, left_of(nn, P.N), v);
          else linear_end(P.out, P.N, batch, mm, nn, v);
        }
      }
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
  }
}

// Ranges of k added up, in their order.
template <bool GATED> __global__ __launch_bounds__(256) void dense_reduce_kernel(const DenseParams P, int64_t width) {
  const int64_t columns = GATED ? 2 * P.N : P.N, per_row = (width + 3) / 4, total = (int64_t)P.batch * P.M * per_row;
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < total; e += (int64_t)gridDim.x * 256) {
    const int64_t row = e / per_row, n = (e - row * per_row) * 4, batch = row / P.M, m = row - batch * P.M;
    const float *p = P.partial + (batch * P.splits * P.M + m) * columns + n;
    f32x4 v = {0.f, 0.f, 0.f, 0.f}, u = v;
    const int left = left_of(n, P.N);
#pragma unroll 4
    for (int s = 0; s < P.splits; ++s, p += P.M * columns) {
      v += load4<RSVD_X_F32>(p, 0, left);
      if constexpr (GATED) u += load4<RSVD_X_F32>(p + P.N, 0, left);
    }
    if constexpr (GATED) gated_end(P.gate, P.N, m, n, v, u);
    else linear_end(P.out, P.N, (int)batch, m, n, v);
  }
}

// ---------------------------------------------------------------- host
// (the same for all products; TileChoice::bn counts rows of B)
TileChoice dense_choose(const rsvd_ctx *ctx, const DenseDesc &d);
DenseParams dense_params(const TileChoice &c, const DenseDesc &d);
hipError_t dense_reduce_launch(hipStream_t s, const DenseParams &P, bool gated);
inline unsigned dense_groups(const DenseParams &P) { return (unsigned)((int64_t)P.batch * P.splits * P.tiles); }
inline int dense_k(int kind) { return kind >= DK_F8 ? 128 : 64; }      // k of a k-tile: 128 bytes

}  // namespace rsvd
