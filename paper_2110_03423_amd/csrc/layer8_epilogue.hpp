// What becomes of a sum over k in the products of the layer operators: scales, the low-rank term, the bias, and the store.
#pragma once

#include "layer8.hpp"

namespace rsvd {

// Matrix instructions of gfx950 with operands of 16 bytes a lane.  Lane L supplies row (column) L % 16 of both operands, k from
// 16 (L / 16) on (codes) or 8 (L / 16) on (bf16); register v of the accumulator holds row 4 (L / 16) + v of the first operand's
// index and column L % 16 of the second's.
__device__ __forceinline__ i32x4 mfma_codes(u32x4 a, u32x4 b, i32x4 c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma_bf16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

struct Layer8Epilogue {
  const float *rs, *cs, *bias;
  const uint16_t *t, *G;
  int64_t ldg;
  int r, rp, parts;
  void *C;
  int64_t ldc;
  int type, accumulate;
};

inline Layer8Epilogue layer8_epilogue(const Layer8Out &o) {
  Layer8Epilogue e;
  e.rs = o.rs; e.cs = o.cs; e.bias = o.bias;
  e.t = o.t; e.G = o.G; e.ldg = o.ldg;
  e.r = o.r; e.rp = (int)rank_places(o.r);
  e.parts = o.parts;
  e.C = o.C; e.ldc = o.ldc; e.type = o.type; e.accumulate = o.accumulate;
  return e;
}

// Eight bf16 numbers of row i of G from p on, zeros from r on.
__device__ __forceinline__ u32x4 factor8(const Layer8Epilogue &E, int64_t i, int p) { return halves8(E.G + i * E.ldg + p, E.r - p); }

// Four values for the columns from n on, for columns that do not exist those of the last one; `all` for p = NULL.
__device__ __forceinline__ f32x4 column4(const float *p, int64_t n, int64_t N, float all) {
  f32x4 v = {all, all, all, all};
  if (p != nullptr) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = p[n + e < N ? n + e : N - 1];
  }
  return v;
}

// Four numbers rounded to a 16-bit type.
template <int TYPE> __device__ __forceinline__ u32x2 halves4(f32x4 v) {
  if constexpr (TYPE == RSVD_X_BF16) return u32x2{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
  else return u32x2{__builtin_bit_cast(unsigned, __builtin_convertvector(f32x2{v[0], v[1]}, f16x2)),
                    __builtin_bit_cast(unsigned, __builtin_convertvector(f32x2{v[2], v[3]}, f16x2))};
}

// Four consecutive results of row m from column n on, of which those before column N exist.
template <int TYPE> __device__ __forceinline__ void store4(const Layer8Epilogue &E, int64_t m, int64_t n, int64_t N, f32x4 v) {
  const int64_t at = m * E.ldc + n;
  const bool whole = n + 4 <= N;
  if constexpr (TYPE == RSVD_X_F32) {
    float *c = reinterpret_cast<float *>(E.C) + at;
    if (whole) {
      if (E.accumulate) v += *reinterpret_cast<const f32x4_any *>(c);
      *reinterpret_cast<f32x4_any *>(c) = v;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (n + e < N) c[e] = E.accumulate ? c[e] + v[e] : v[e];
    }
  } else {
    const u32x2 p = halves4<TYPE>(v);
    uint16_t *c = reinterpret_cast<uint16_t *>(E.C) + at;
    if (whole) {
      *reinterpret_cast<u32x2_any *>(c) = p;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (n + e < N) c[e] = (uint16_t)(p[e >> 1] >> (16 * (e & 1)));
    }
  }
}
__device__ __forceinline__ void store4(const Layer8Epilogue &E, int64_t m, int64_t n, int64_t N, f32x4 v) {
  if (E.type == RSVD_X_F32) store4<RSVD_X_F32>(E, m, n, N, v);
  else if (E.type == RSVD_X_BF16) store4<RSVD_X_BF16>(E, m, n, N, v);
  else store4<RSVD_X_F16>(E, m, n, N, v);
}

}  // namespace rsvd
