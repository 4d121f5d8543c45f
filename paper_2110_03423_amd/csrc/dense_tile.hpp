// What the product kernels of the gated block's operators have in common: places of tiles, and the end of a tile.
#pragma once

#include <type_traits>

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
  int ktiles, tiles_m, tiles_n, tiles, batch;      // k-tiles of a part of k; tiles of a problem
  int kt_all;                              // k-tiles
  int whole, rest, splits, kt_per_split;   // tiles of all problems that are worked out at once, and behind them those whose k is in `splits` ranges
  int symmetric;
  float *partial;                          // [rest][splits][tile], fp32
  LinearOut out;
  GatedOut gate;
};

__device__ __forceinline__ f32x4 mfma_f16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Where tile t of a problem lies: strips of eight rows of tiles, column by column; of symmetric results the tiles on and below the diagonal, row by row.
__device__ __forceinline__ void dense_place(const DenseParams &P, int t, int &tile_m, int &tile_n) {
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

// What a workgroup works out.
struct DenseWork {
  int tile_m, tile_n, batch, kt_begin, nkt;
  float *partial;                          // the tile's place for a range of k, or NULL
};
// Workgroups of the whole tiles first, then range of k by range of k those of the rest; in each a contiguous run for each of the eight XCDs, which have an L2 each.
template <int SIZE> __device__ __forceinline__ DenseWork dense_work(const DenseParams &P) {
  DenseWork w;
  const bool part = (int)blockIdx.x >= P.whole;
  const int total = part ? P.rest * P.splits : P.whole, pid = (int)blockIdx.x - (part ? P.whole : 0);
  const int per = (total + 7) >> 3, tall = (total & 7) ? (total & 7) : 8, xcd = pid & 7, local = pid >> 3;
  int t = xcd < tall ? xcd * per + local : tall * per + (xcd - tall) * (per - 1) + local;
  w.kt_begin = 0;
  w.nkt = P.kt_all;
  w.partial = nullptr;
  if (part) {
    const int split = __builtin_amdgcn_readfirstlane(t / P.rest);
    t -= split * P.rest;
    w.partial = P.partial + ((int64_t)t * P.splits + split) * SIZE;
    w.kt_begin = split * P.kt_per_split;
    w.nkt = P.kt_all - w.kt_begin < P.kt_per_split ? P.kt_all - w.kt_begin : P.kt_per_split;
    t += P.whole;
  }
  w.batch = __builtin_amdgcn_readfirstlane(t / P.tiles);
  dense_place(P, __builtin_amdgcn_readfirstlane(t - w.batch * P.tiles), w.tile_m, w.tile_n);
  return w;
}

// f with the planes of both operands in each product of numbers of PL planes, in the order of dense_segs.
template <int PL, typename F> __device__ __forceinline__ void with_segs(F f) {
  using std::integral_constant;
  if constexpr (PL == 3) {
    f(integral_constant<int, 2>(), integral_constant<int, 0>());
    f(integral_constant<int, 1>(), integral_constant<int, 1>());
    f(integral_constant<int, 0>(), integral_constant<int, 2>());
  }
  if constexpr (PL >= 2) {
    f(integral_constant<int, 1>(), integral_constant<int, 0>());
    f(integral_constant<int, 0>(), integral_constant<int, 1>());
  }
  f(integral_constant<int, 0>(), integral_constant<int, 0>());
}

// Eight numbers as fp32.
template <int XT> __device__ __forceinline__ void x_values(const Raw8<XT> &r, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if constexpr (XT == RSVD_X_F32) v[e] = __uint_as_float(r.w[e >> 2][e & 3]);
    else if constexpr (XT == RSVD_X_BF16) v[e] = e & 1 ? bf16_high(r.w[0][e >> 1]) : bf16_low(r.w[0][e >> 1]);
    else {
      const unsigned pair = r.w[0][e >> 1];
      v[e] = (float)__builtin_bit_cast(f16x2, pair)[e & 1];
    }
  }
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
// V times four columns from n on that exist.
template <int V = 1> __device__ __forceinline__ int left_of(int64_t n, int64_t N) { return N - n >= 4 * V ? 4 * V : (int)(N - n); }

// V times four numbers, of which `left` exist.
template <int TYPE, int V> __device__ __forceinline__ void load_row(const void *p, int64_t at, int left, f32x4 (&v)[V]) {
  if constexpr (V == 2 && TYPE != RSVD_X_F32) {
    if (left >= 8) {
      const u32x4 w = *reinterpret_cast<const u32x4_any *>(reinterpret_cast<const uint16_t *>(p) + at);
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const unsigned pair = w[h];
        if constexpr (TYPE == RSVD_X_BF16) {
          v[h >> 1][2 * (h & 1)] = bf16_low(pair);
          v[h >> 1][2 * (h & 1) + 1] = bf16_high(pair);
        } else {
          const f16x2 f = __builtin_bit_cast(f16x2, pair);
          v[h >> 1][2 * (h & 1)] = (float)f[0];
          v[h >> 1][2 * (h & 1) + 1] = (float)f[1];
        }
      }
      return;
    }
  }
#pragma unroll
  for (int x = 0; x < V; ++x) v[x] = load4<TYPE>(p, at + 4 * x, left - 4 * x);
}
template <int TYPE, int V> __device__ __forceinline__ void put_row(void *p, int64_t at, int left, const f32x4 (&v)[V]) {
  if constexpr (V == 2 && TYPE != RSVD_X_F32) {
    if (left >= 8) {
      const u32x2 a = halves4<TYPE>(v[0]), b = halves4<TYPE>(v[1]);
      *reinterpret_cast<u32x4_any *>(reinterpret_cast<uint16_t *>(p) + at) = u32x4{a[0], a[1], b[0], b[1]};
      return;
    }
  }
#pragma unroll
  for (int x = 0; x < V; ++x) put4<TYPE>(p, at + 4 * x, left - 4 * x, v[x]);
}

// f with the type, or the activation, as a constant.
template <typename F> __device__ __forceinline__ void with_type(int type, F f) {
  if (type == RSVD_X_BF16) f(std::integral_constant<int, RSVD_X_BF16>());
  else if (type == RSVD_X_F16) f(std::integral_constant<int, RSVD_X_F16>());
  else f(std::integral_constant<int, RSVD_X_F32>());
}
template <typename F> __device__ __forceinline__ void with_act(int act, F f) {
  if (act == GATED_SILU) f(std::integral_constant<int, GATED_SILU>());
  else if (act == GATED_GELU) f(std::integral_constant<int, GATED_GELU>());
  else if (act == GATED_GELU_TANH) f(std::integral_constant<int, GATED_GELU_TANH>());
  else f(std::integral_constant<int, GATED_RELU>());
}

// Eight numbers of each of C groups of D as they lie, both planes, and rows_m.
template <int C> struct DRows { u32x4 high[C], low[C]; float row; };

// The end of C groups of V times four columns.  Group c has row m[c] (if it is there) and columns from n[c] on, of which those before `width` are stored and those from N on are
// zeros.  All loads come before the stores.  WHOLE: all rows and columns exist (no branches between loads).  AHEAD: D, rows and columns
// (a vector of them for each of v's) were loaded before (V = 2).
template <int C, int V, bool WHOLE, bool AHEAD = false>
__device__ __forceinline__ void linear_end(const LinearOut &O, int64_t N, int batch, const int64_t (&m)[C], const int64_t (&n)[C], const bool (&there)[C], f32x4 (&v)[C][V],
                                           const DRows<AHEAD ? C : 1> ahead = {}, const f32x4 (*ahead_columns)[V] = nullptr) {
  // (one by one, in scalar registers: arguments of the kernel that are read together and under conditions would go through memory)
  float alpha = O.alpha, beta = O.beta, gamma = O.gamma;
  const uint16_t *d = O.D;
  asm volatile("" : "+s"(alpha), "+s"(beta), "+s"(gamma), "+s"(d));
  const int64_t ldd = O.ldd, d_plane = O.d_plane / 2;
  const bool has_d = d != nullptr, two = O.d_planes == 2;
  d += batch * O.d_batch;
  const float *const rows = O.rows, *const columns = O.columns;
  float *const diagonal = O.diagonal;
  const int64_t v_first = batch * O.v_batch, width = O.width;
  auto have = [&](int c) RSVD_INLINE { return WHOLE ? 4 * V : there[c] ? left_of<V>(n[c], N) : 0; };
  auto left = [&](int c) RSVD_INLINE { return WHOLE ? 4 * V : there[c] ? left_of<V>(n[c], width) : 0; };
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int x = 0; x < V; ++x) v[c][x] *= alpha;
  if (has_d) {
    f32x4 sum[C][V], low[C][V];
    if constexpr (AHEAD) {
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          const unsigned high2 = ahead.high[c][h], low2 = two ? ahead.low[c][h] : 0u;
          const f16x2 x = __builtin_bit_cast(f16x2, high2), y = __builtin_bit_cast(f16x2, low2);
          sum[c][h >> 1][2 * (h & 1)] = (float)x[0] + (float)y[0];
          sum[c][h >> 1][2 * (h & 1) + 1] = (float)x[1] + (float)y[1];
        }
    } else {
#pragma unroll
      for (int c = 0; c < C; ++c) load_row<RSVD_X_F16, V>(d, m[c] * ldd + n[c], have(c), sum[c]);
      if (two) {
#pragma unroll
        for (int c = 0; c < C; ++c) load_row<RSVD_X_F16, V>(d + d_plane, m[c] * ldd + n[c], have(c), low[c]);
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int x = 0; x < V; ++x) sum[c][x] += low[c][x];
      }
    }
    f32x4 by[C][V];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float row = beta;
      if constexpr (AHEAD) row += gamma * ahead.row;
      else if (rows != nullptr && (WHOLE || there[c])) row += gamma * rows[v_first + m[c]];
#pragma unroll
      for (int x = 0; x < V; ++x) {
        by[c][x] = (f32x4)row;
        if constexpr (AHEAD) by[c][x] += gamma * ahead_columns[c][x];
        else if (columns != nullptr) by[c][x] += gamma * load4<RSVD_X_F32>(columns + v_first, n[c] + 4 * x, have(c) - 4 * x);
      }
    }
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int x = 0; x < V; ++x) v[c][x] += by[c][x] * sum[c][x];
  }
  if (diagonal != nullptr) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int at = (int)(m[c] - n[c]);                 // (the value on the diagonal, if the group has it)
      if ((WHOLE || there[c]) && at >= 0 && at < 4 * V) {
        float own = 0.f;
        if (rows != nullptr) own = rows[v_first + m[c]];
        float value = own * (beta + gamma * own);
#pragma unroll
        for (int x = 0; x < V; ++x) {
          const f32x4 old = v[c][x];
          f32x4 rest;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            value += at == 4 * x + e ? old[e] : 0.f;
            rest[e] = at == 4 * x + e ? 0.f : old[e];
          }
          v[c][x] = rest;
        }
        diagonal[v_first + m[c]] = value;
      }
    }
  }
  if constexpr (!WHOLE) {
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int e = 0; e < 4 * V; ++e) v[c][e >> 2][e & 3] = e < have(c) ? v[c][e >> 2][e & 3] : 0.f;
  }
  const int64_t at = batch * O.c_batch;
  if (O.planes == 2) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      put_row<RSVD_X_F16, V>(O.C, at + m[c] * O.ldc + n[c], left(c), v[c]);
#pragma unroll
      for (int e = 0; e < 4 * V; ++e) v[c][e >> 2][e & 3] -= (float)(_Float16)v[c][e >> 2][e & 3];
      put_row<RSVD_X_F16, V>(reinterpret_cast<char *>(O.C) + O.c_plane, at + m[c] * O.ldc + n[c], left(c), v[c]);
    }
    return;
  }
  with_type(O.type, [&](auto type) RSVD_INLINE {
    constexpr int TYPE = decltype(type)::value;
    if constexpr (TYPE == RSVD_X_F32)
      if (O.accumulate) {
        f32x4 old[C][V];
#pragma unroll
        for (int c = 0; c < C; ++c) load_row<TYPE, V>(O.C, at + m[c] * O.ldc + n[c], left(c), old[c]);
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int x = 0; x < V; ++x) v[c][x] += old[c][x];
      }
#pragma unroll
    for (int c = 0; c < C; ++c) put_row<TYPE, V>(O.C, at + m[c] * O.ldc + n[c], left(c), v[c]);
  });
}
__device__ __forceinline__ void linear_end1(const LinearOut &O, int64_t N, int batch, int64_t m, int64_t n, f32x4 v) {
  const int64_t row[1] = {m}, column[1] = {n};
  const bool there[1] = {true};
  f32x4 vs[1][1] = {{v}};
  linear_end<1, 1, false>(O, N, batch, row, column, there, vs);
}

// The activation (g times a share of it) and its derivative.  The shares are written so that none is a difference of numbers near one: 1 / 2 + erf / 2 as a
// complement, 1 / 2 + tanh(y) / 2 as 1 / (1 + exp(-2 y)).
template <int ACT> __device__ __forceinline__ float act_share(float g) {
  if constexpr (ACT == GATED_SILU) return 1.f / (1.f + __expf(-g));
  else if constexpr (ACT == GATED_GELU) return 0.5f * erfcf(-0.70710678f * g);
  else return 1.f / (1.f + __expf(-1.5957691f * (g + 0.044715f * g * g * g)));
}
template <int ACT> __device__ __forceinline__ float act_value(float g) {
  if constexpr (ACT == GATED_RELU) return g > 0.f ? g : g != g ? g : 0.f;
  else return g * act_share<ACT>(g);
}
template <int ACT> __device__ __forceinline__ float act_slope(float g, float &value) {
  if constexpr (ACT == GATED_RELU) {
    value = g > 0.f ? g : g != g ? g : 0.f;
    return g > 0.f ? 1.f : 0.f;
  } else {
    const float s = act_share<ACT>(g);
    value = g * s;
    if constexpr (ACT == GATED_SILU) return s + value * (1.f - s);
    else if constexpr (ACT == GATED_GELU) return s + g * __expf(-0.5f * g * g) * 0.39894228f;
    else return s + value * (1.f - s) * 1.5957691f * (1.f + 0.134145f * fminf(g * g, 1e30f));      // (0, not 0 times infinity, where the share is 0 or 1)
  }
}
// Gradients of gate and up, V times four columns from n on, to the planes of D (gate from column 0 on, up from column N on, zeros behind both).
template <int TYPE, int V> __device__ __forceinline__ void slope_put(const GatedOut &O, int64_t N, int64_t m, int64_t n, int left, const f32x4 (&dg)[V], const f32x4 (&du)[V]) {
  constexpr int PLANES = TYPE == RSVD_X_F32 ? 3 : 1;
  const int64_t at = m * O.ldD + n;
  if (2 * N != O.ldD && n < N && n + 4 * V >= N)
    for (int64_t c = 2 * N; c < O.ldD; ++c)
      for (int q = 0; q < PLANES; ++q) O.D[q * (O.plane / 2) + m * O.ldD + c] = 0;
  if constexpr (TYPE != RSVD_X_F32) {
    put_row<TYPE, V>(O.D, at, left, dg);
    put_row<TYPE, V>(O.D, at + N, left, du);
  } else {
#pragma unroll
    for (int x = 0; x < V; ++x) {
      unsigned p[2][2][3];
      bf16_parts2<3>(dg[x][0], dg[x][1], p[0][0]);
      bf16_parts2<3>(dg[x][2], dg[x][3], p[0][1]);
      bf16_parts2<3>(du[x][0], du[x][1], p[1][0]);
      bf16_parts2<3>(du[x][2], du[x][3], p[1][1]);
#pragma unroll
      for (int q = 0; q < 3; ++q)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint16_t *c = O.D + q * (O.plane / 2) + at + 4 * x + h * N;
          if (left >= 4 * x + 4) *reinterpret_cast<u32x2_any *>(c) = u32x2{p[h][0][q], p[h][1][q]};
          else
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (4 * x + e < left) c[e] = (uint16_t)(p[h][e >> 1][q] >> (16 * (e & 1)));
        }
    }
  }
}

// The end of C groups of V times four outputs, as linear_end: all loads, then all activations, then the stores.
template <int C, int V, bool WHOLE>
__device__ __forceinline__ void gated_end(const GatedOut &O, int64_t N, const int64_t (&m)[C], const int64_t (&n)[C], const bool (&there)[C], f32x4 (&g)[C][V], f32x4 (&u)[C][V]) {
  auto left = [&](int c) RSVD_INLINE { return WHOLE ? 4 * V : there[c] ? left_of<V>(n[c], N) : 0; };
  with_type(O.type, [&](auto type) RSVD_INLINE {
    constexpr int TYPE = decltype(type)::value;
    if (O.dH != nullptr) {
      const float by = TYPE == RSVD_X_F16 ? *O.scale : 1.f;
      f32x4 dh[C][V];
#pragma unroll
      for (int c = 0; c < C; ++c) load_row<TYPE, V>(O.dH, m[c] * O.lddh + n[c], left(c), dh[c]);
      with_act(O.act, [&](auto act) RSVD_INLINE {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int x = 0; x < V; ++x)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              float value;
              const float slope = act_slope<decltype(act)::value>(g[c][x][e], value);
              g[c][x][e] = dh[c][x][e] * u[c][x][e] * slope * by;
              u[c][x][e] = dh[c][x][e] * value * by;
            }
      });
#pragma unroll
      for (int c = 0; c < C; ++c)
        if (WHOLE || there[c]) slope_put<TYPE, V>(O, N, m[c], n[c], left(c), g[c], u[c]);
    } else {
      if (O.kept != nullptr) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
          put_row<TYPE, V>(O.kept, m[c] * O.ldk + n[c], left(c), g[c]);
          put_row<TYPE, V>(O.kept, m[c] * O.ldk + N + n[c], left(c), u[c]);
        }
      }
      with_act(O.act, [&](auto act) RSVD_INLINE {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int x = 0; x < V; ++x)
#pragma unroll
            for (int e = 0; e < 4; ++e) g[c][x][e] = act_value<decltype(act)::value>(g[c][x][e]) * u[c][x][e];
      });
#pragma unroll
      for (int c = 0; c < C; ++c) put_row<TYPE, V>(O.H, m[c] * O.ldh + n[c], left(c), g[c]);
    }
  });
}
__device__ __forceinline__ void gated_end1(const GatedOut &O, int64_t N, int64_t m, int64_t n, f32x4 g, f32x4 u) {
  const int64_t row[1] = {m}, column[1] = {n};
  const bool there[1] = {true};
  f32x4 gs[1][1] = {{g}}, us[1][1] = {{u}};
  gated_end<1, 1, false>(O, N, row, column, there, gs, us);
}

// ---------------------------------------------------------------- the end of a wavefront's TM x TN blocks of 16 x 16
// (m1, n1): the first row and column of the wavefront's.  partial: where its first sum goes if it has a range of k, rows of BN sums; or NULL.

// Sixteen rows of a wavefront's blocks in LDS, with their rows and columns exchanged: group e of four has column e / 4 and four of the rows.
template <int TN> __device__ __forceinline__ void mirror_rows(const DenseParams &P, int batch, int64_t m2, int64_t n1, int lane, const float *lds) {
  constexpr int PITCH = 16 * TN + 4, C = TN < 4 ? TN : 4;
  const bool whole = n1 + 16 * TN <= P.M && m2 + 16 <= P.N;
#pragma unroll 1
  for (int e0 = lane; e0 < 64 * TN; e0 += 64 * C) {
    f32x4 v[C][1];
    int64_t m[C], n[C];
    bool there[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int e = e0 + 64 * c, col = e >> 2, q = 4 * (e & 3);
#pragma unroll
      for (int x = 0; x < 4; ++x) v[c][0][x] = lds[(q + x) * PITCH + col];
      m[c] = n1 + col;
      n[c] = m2 + q;
      there[c] = m[c] < P.M && n[c] < P.out.width;
    }
    if (whole) linear_end<C, 1, true>(P.out, P.N, batch, m, n, there, v);
    else linear_end<C, 1, false>(P.out, P.N, batch, m, n, there, v);
  }
}

// Block (i, j) of lane L holds row 16 i + L % 16 and four columns from 16 j + 4 (L / 16) on: through LDS, sixteen rows at a time, so that lanes next to each
// other write what is next to each other.  mirror: and the same with rows and columns exchanged.  lds: the wavefront's finish_lds<TN>() bytes.  by: what all
// sums are multiplied by.
template <int BN, int TM, int TN>
__device__ __forceinline__ void dense_finish(const DenseParams &P, f32x4 (&acc)[TM][TN], float *partial, int batch, int64_t m1, int64_t n1, bool mirror, int lane, float *lds,
                                             float by) {
  constexpr int PITCH = 16 * TN + 4, PER_ROW = 4 * TN, ROWS = 64 / PER_ROW, PASSES = 16 / ROWS, C = PASSES < 4 ? PASSES : 4;
  const int r16 = lane & 15, kq = lane >> 4, row = lane / PER_ROW, col = 4 * (lane % PER_ROW);
  const bool whole = m1 + 16 * TM <= P.M && n1 + 16 * TN <= P.N;
#pragma unroll 1
  for (int i = 0; i < TM; ++i) {                        // (one copy of what follows, not one for each row of blocks)
#pragma unroll
    for (int x = 0; x < TM; ++x)
      if (i == x) {
#pragma unroll
        for (int j = 0; j < TN; ++j) *reinterpret_cast<f32x4 *>(lds + r16 * PITCH + 16 * j + 4 * kq) = acc[x][j] * by;
      }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
#pragma unroll 1
    for (int p = 0; p < PASSES; p += C) {
      f32x4 v[C][1];
      int64_t m[C], n[C];
      bool there[C];
#pragma unroll
      for (int c = 0; c < C; ++c) {
        v[c][0] = *reinterpret_cast<const f32x4 *>(lds + ((p + c) * ROWS + row) * PITCH + col);
        m[c] = m1 + 16 * i + (p + c) * ROWS + row;
        n[c] = n1 + col;
        there[c] = m[c] < P.M && n[c] < P.out.width;
      }
      if (partial != nullptr) {
#pragma unroll
        for (int c = 0; c < C; ++c) *reinterpret_cast<f32x4 *>(partial + (16 * i + (p + c) * ROWS + row) * BN + col) = v[c][0];
      } else if (whole) {
        linear_end<C, 1, true>(P.out, P.N, batch, m, n, there, v);
      } else {
        linear_end<C, 1, false>(P.out, P.N, batch, m, n, there, v);
      }
    }
    if (mirror && partial == nullptr) mirror_rows<TN>(P, batch, m1 + 16 * i, n1, lane, lds);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
  }
}

// The mirrored half for blocks in the order of dense_finish_rows.
template <int TM, int TN> __device__ __forceinline__ void dense_finish_mirror(const DenseParams &P, f32x4 (&acc)[TM][TN], int batch, int64_t m1, int64_t n1, int lane, float *lds) {
  constexpr int PITCH = 16 * TN + 4;
  const int r16 = lane & 15, kq = lane >> 4;
#pragma unroll 1
  for (int i = 0; i < TM; ++i) {
#pragma unroll
    for (int x = 0; x < TM; ++x)
      if (i == x) {
#pragma unroll
        for (int j = 0; j < TN; ++j) *reinterpret_cast<f32x4 *>(lds + r16 * PITCH + 32 * (j / 2) + 8 * kq + 4 * (j & 1)) = acc[x][j];
      }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
    mirror_rows<TN>(P, batch, m1 + 16 * i, n1, lane, lds);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
  }
}

// Blocks (i, 2 p) and (i, 2 p + 1) of lane L hold row 16 i + L % 16 and eight columns from 32 p + 8 (L / 16) on: stored as they are.  gated: p even is the gate and p odd the
// up projection of 32 outputs; with two blocks, these are the gate and the up projection of sixteen, four of them a lane.
template <bool GATED, int BN, int TM, int TN> __device__ __forceinline__ void dense_finish_rows(const DenseParams &P, f32x4 (&acc)[TM][TN], float *partial, int batch, int64_t m1, int64_t n1,
                                                                                               int lane) {
  constexpr int V = GATED && TN == 2 ? 1 : 2, C = GATED ? TN / (2 * V) : TN / 2;      // groups of a row, and vectors of four in each
  const bool whole = m1 + 16 * TM <= P.M && n1 + 4 * V * 4 * C <= P.N;
  int64_t m[C], n[C];
  bool there[C];
#pragma unroll
  for (int c = 0; c < C; ++c) n[c] = n1 + 16 * V * c + 4 * V * (lane >> 4);
  // (D of the next row of blocks is under way while this one ends: 8 to 10 % of the time of a product of 4096 k with D)
  constexpr bool AHEAD = !GATED && V == 2;
  const uint16_t *d_first = P.out.D;
  asm volatile("" : "+s"(d_first));
  const bool d_ahead = AHEAD && whole && partial == nullptr && d_first != nullptr;
  const uint16_t *const d_high = d_first + batch * P.out.d_batch, *const d_low = P.out.d_planes == 2 ? d_high + P.out.d_plane / 2 : d_high;
  const int64_t ldd = P.out.ldd;
  DRows<AHEAD ? C : 1> next = {};
  const float *const rows = P.out.rows, *const columns = P.out.columns;
  const int64_t v_first = batch * P.out.v_batch;
  f32x4 column[C][V];
#pragma unroll
  for (int c = 0; c < (AHEAD ? C : 0); ++c)
#pragma unroll
    for (int x = 0; x < V; ++x) column[c][x] = d_ahead && columns != nullptr ? *reinterpret_cast<const f32x4_any *>(columns + v_first + n[c] + 4 * x) : (f32x4)0.f;
  auto load_next = [&](int i) RSVD_INLINE {
    if constexpr (AHEAD) {
      const int64_t row = m1 + 16 * (i < TM ? i : TM - 1) + (lane & 15), at = row * ldd;
      if (rows != nullptr) next.row = rows[v_first + row];
#pragma unroll
      for (int c = 0; c < C; ++c) next.high[c] = *reinterpret_cast<const u32x4_any *>(d_high + at + n[c]);
#pragma unroll
      for (int c = 0; c < C; ++c) next.low[c] = *reinterpret_cast<const u32x4_any *>(d_low + at + n[c]);
    }
  };
  if (d_ahead) load_next(0);
#pragma unroll 1
  for (int i = 0; i < TM; ++i) {                        // (one copy of what follows, not one for each row of blocks)
    f32x4 v[C][V], u[C][V];
#pragma unroll
    for (int x = 0; x < TM; ++x)
      if (i == x) {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int y = 0; y < V; ++y) {
            v[c][y] = acc[x][(GATED ? 2 * V : V) * c + y];
            if constexpr (GATED) u[c][y] = acc[x][2 * V * c + V + y];
          }
      }
#pragma unroll
    for (int c = 0; c < C; ++c) {
      m[c] = m1 + 16 * i + (lane & 15);
      there[c] = m[c] < P.M && n[c] < (GATED ? P.N : P.out.width);
    }
    if (partial != nullptr) {
      float *to = partial + (16 * i + (lane & 15)) * BN + 4 * V * (lane >> 4);
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int y = 0; y < V; ++y) {
          *reinterpret_cast<f32x4 *>(to + (GATED ? 32 * V : 16 * V) * c + 4 * y) = v[c][y];
          if constexpr (GATED) *reinterpret_cast<f32x4 *>(to + 32 * V * c + 16 * V + 4 * y) = u[c][y];
        }
    } else if constexpr (GATED) {
      if (whole) gated_end<C, V, true>(P.gate, P.N, m, n, there, v, u);
      else gated_end<C, V, false>(P.gate, P.N, m, n, there, v, u);
    } else {
      if (d_ahead) {
        if constexpr (AHEAD) {
          const DRows<C> now = next;
          load_next(i + 1);
          linear_end<C, V, true, true>(P.out, P.N, batch, m, n, there, v, now, column);
        }
      } else if (whole) {
        linear_end<C, V, true>(P.out, P.N, batch, m, n, there, v);
      } else {
        linear_end<C, V, false>(P.out, P.N, batch, m, n, there, v);
      }
    }
  }
}

// Ranges of k added up, in their order: 32 x 32 sums a workgroup, four a thread.  GROUP: outputs whose gate stands before their up projection (0: no gate).
template <int GROUP> __global__ __launch_bounds__(256) void dense_reduce_kernel(const DenseParams P, int b) {
  const int across = (GROUP ? b / 2 : b) / 32, shares = across * (b / 32), q = (int)blockIdx.x / shares, share = (int)blockIdx.x - q * shares;
  const int t = P.whole + q, batch = t / P.tiles, tid = threadIdx.x;
  int tile_m, tile_n;
  dense_place(P, t - batch * P.tiles, tile_m, tile_n);
  const int64_t size = (int64_t)b * b;
  const int row0 = share / across * 32, col0 = share % across * 32, row = row0 + (tid >> 3), col = col0 + 4 * (tid & 7);
  const int64_t m0 = (int64_t)tile_m * b, n0 = (int64_t)tile_n * (GROUP ? b / 2 : b), width = GROUP ? P.N : P.out.width;
  const bool mirror = GROUP == 0 && P.symmetric && tile_m != tile_n;
  if (m0 + row0 >= P.M || (n0 + col0 >= width && !mirror)) return;
  auto add = [&](int at) RSVD_INLINE {
    const float *p = P.partial + (int64_t)q * P.splits * size + at;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < P.splits; s += 8) {
      f32x4 v[8];                                        // (eight loads in flight)
#pragma unroll
      for (int x = 0; x < 8; ++x) v[x] = *reinterpret_cast<const f32x4 *>(p + (s + x < P.splits ? s + x : s) * size);
#pragma unroll
      for (int x = 0; x < 8; ++x)
        if (s + x < P.splits) sum += v[x];
    }
    return sum;
  };
  const int64_t m = m0 + row, n = n0 + col;
  if constexpr (GROUP) {
    const int at = row * b + col / GROUP * 2 * GROUP + col % GROUP;
    const f32x4 g = add(at), u = add(at + GROUP);
    if (m < P.M && n < width) gated_end1(P.gate, P.N, m, n, g, u);
  } else {
    const f32x4 v = add(row * b + col);
    if (m < P.M && n < width) linear_end1(P.out, P.N, batch, m, n, v);
    if (!mirror) return;
    __shared__ __attribute__((aligned(16))) float block[32][36];
    *reinterpret_cast<f32x4 *>(&block[tid >> 3][4 * (tid & 7)]) = v;
    __syncthreads();
    f32x4 w;                                             // a column and four of its rows
#pragma unroll
    for (int x = 0; x < 4; ++x) w[x] = block[4 * (tid & 7) + x][tid >> 3];
    const int64_t mm = n0 + col0 + (tid >> 3), nn = m0 + row0 + 4 * (tid & 7);
    if (mm < P.M && nn < P.out.width) linear_end1(P.out, P.N, batch, mm, nn, w);
  }
}

// ---------------------------------------------------------------- host
// Tiles of b rows and columns (of gated products: of B), and which of them have their k in ranges.
struct DenseChoice { int b; int64_t tiles, whole, rest, splits, kt, kt_per_split; };
inline unsigned dense_groups(const DenseParams &P) { return (unsigned)(P.whole + P.rest * P.splits); }
inline int dense_k(int kind) { return kind >= DK_F8 ? 128 : 64; }      // k of a k-tile: 128 bytes

}  // namespace rsvd
