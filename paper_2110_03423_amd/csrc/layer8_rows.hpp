// One row of X to 8 bits with a scale, by a workgroup of 256 threads.
#pragma once

#include "layer8.hpp"

namespace rsvd {

__device__ __forceinline__ unsigned magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// Eight integers in [-127, 127], given as floats, as bytes.
__device__ __forceinline__ u32x2 pack8(const float (&q)[8]) {
  u32x2 w;
#pragma unroll
  for (int h = 0; h < 2; ++h)
    w[h] = ((unsigned)(int)q[4 * h] & 255u) | (((unsigned)(int)q[4 * h + 1] & 255u) << 8) | (((unsigned)(int)q[4 * h + 2] & 255u) << 16) |
           ((unsigned)(int)q[4 * h + 3] << 24);
  return w;
}

// Four places of t: the sums over ranges of k added up, as `parts` (2 or 3) bf16 numbers.  e counts quadruples, rp / 4 a token.
__device__ __forceinline__ void join_lowrank(const float *sums, int splits, int64_t tokens, int rp, int parts, uint16_t *t, int64_t e) {
  const int64_t token = e / (rp / 4);
  const int p = (int)(e - token * (rp / 4)) * 4;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < splits; s += 8) {
    f32x4 v[8];                                       // (eight loads in flight)
#pragma unroll
    for (int u = 0; u < 8; ++u)
      v[u] = s + u < splits ? *reinterpret_cast<const f32x4 *>(sums + ((int64_t)(s + u) * tokens + token) * rp + p) : (f32x4)0.f;
#pragma unroll
    for (int u = 0; u < 8; ++u) sum += v[u];
  }
  uint16_t *out = t + token * parts * rp + p;
  unsigned a[3], b[3];
  if (parts == 3) {
    bf16_parts2<3>(sum[0], sum[1], a);
    bf16_parts2<3>(sum[2], sum[3], b);
  } else {
    unsigned c[2], d[2];
    bf16_parts2<2>(sum[0], sum[1], c);
    bf16_parts2<2>(sum[2], sum[3], d);
    a[0] = c[0]; a[1] = c[1]; a[2] = 0u;
    b[0] = d[0]; b[1] = d[1]; b[2] = 0u;
  }
#pragma unroll
  for (int q = 0; q < 3; ++q)
    if (q < parts) *reinterpret_cast<u32x2 *>(out + q * rp) = u32x2{a[q], b[q]};
}

struct Rows8Params {
  const char *X; int64_t ldx, rows; int n;
  int8_t *codes; int64_t ldq; int width;      // a row of codes is written up to `width` (>= n, a multiple of 8) with zeros behind n
  float *scale;
  const float *sums; int splits, rp, parts;   // sums != NULL: the row's places of t are joined as well
  uint16_t *t;
};

// Memory is the bound: X is read once and the codes are written.  16384 x 16384 fp16 155 us (5.3 TB/s), 2048 x 4096 bf16 8 us (a launch of many rows).
// The largest magnitude is found among the bit patterns (as integers they are ordered like the magnitudes, infinity and NaN on
// top).  CH chunks of 8 elements stay in a thread's registers between the maximum and the codes; longer rows are read twice.
template <int XT, int CH> __device__ __forceinline__ void rows8_row(const Rows8Params &P, int64_t row) {
  __shared__ unsigned part[4];
  const int tid = threadIdx.x, n = P.n;
  const char *x = P.X + row * P.ldx * XTraits<XT>::SIZE;
  const int chunks = (P.width + 7) / 8;
  if (P.sums != nullptr) {
    for (int e = tid; e < P.rp / 4; e += 256) join_lowrank(P.sums, P.splits, P.rows, P.rp, P.parts, P.t, row * (P.rp / 4) + e);
  }
  float v[CH][8];
  unsigned top = 0u;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int j = 8 * (tid + 256 * c);
    x_load8<XT>(x + (int64_t)j * XTraits<XT>::SIZE, n - j, v[c]);
  }
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, magnitude(v[c][e]));
  for (int c = tid + 256 * CH; c < chunks; c += 256) {
    float w[8];
    x_load8<XT>(x + (int64_t)8 * c * XTraits<XT>::SIZE, n - 8 * c, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, magnitude(w[e]));
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) top = max(top, (unsigned)__shfl_xor((int)top, d));
  if ((tid & 63) == 0) part[tid >> 6] = top;
  __syncthreads();
  top = max(max(part[0], part[1]), max(part[2], part[3]));
  const float a = __uint_as_float(top);
  const bool bad = top >= 0x7f800000u, none = bad || a < 0x1p-116f;
  const float per = none ? 0.f : 127.f * (1.f / a);
  if (tid == 0) P.scale[row] = bad ? __uint_as_float(0x7fc00000u) : none ? 0.f : a / 127.f;
  auto store = [&](int c, const float (&w)[8]) RSVD_INLINE {
    float q[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e] = none ? 0.f : __builtin_rintf(w[e] * per);
    *reinterpret_cast<u32x2 *>(P.codes + row * P.ldq + 8 * c) = pack8(q);
  };
#pragma unroll
  for (int c = 0; c < CH; ++c)
    if (tid + 256 * c < chunks) store(tid + 256 * c, v[c]);
  for (int c = tid + 256 * CH; c < chunks; c += 256) {
    float w[8];
    x_load8<XT>(x + (int64_t)8 * c * XTraits<XT>::SIZE, n - 8 * c, w);
    store(c, w);
  }
}

// The value of code q of a block with power byte b: exact in bf16.
__device__ __forceinline__ float kept_unit(unsigned b) { return b == 255u ? __uint_as_float(0x7fc00000u) : __uint_as_float(b << 23); }

// ---------------------------------------------------------------- operands of the gradients
// Row and place in it of piece group * 256 + thread, per_row pieces a row.  (One long division for the workgroup, a short one for the thread.)
__device__ __forceinline__ void piece_of(int64_t group, int per_row, int64_t &row, int &place) {
  const int64_t first = group * 256, row0 = first / per_row;
  const unsigned at = (unsigned)(first - row0 * per_row) + threadIdx.x, more = at / (unsigned)per_row;
  row = row0 + more;
  place = (int)(at - more * (unsigned)per_row);
}

// planes[q][row][0 .. width): the bf16 parts of X_rj, or with SCALED of X_rj factor_j, zeros from n on; width: a multiple of 8.
struct SplitParams {
  const char *X; int64_t ldx, rows, n;
  const float *factor;
  uint16_t *planes; int64_t width;
  int64_t groups;                  // workgroups: 256 pieces of eight each
};
template <int XT, bool SCALED> __device__ __forceinline__ void split_rows_group(const SplitParams &P, int64_t group) {
  constexpr int PARTS = SCALED && XT == RSVD_X_BF16 ? 2 : XTraits<XT>::PARTS;
  int64_t row;
  int place;
  piece_of(group, (int)(P.width / 8), row, place);
  const int64_t j = 8 * (int64_t)place;
  if (row >= P.rows) return;
  const int64_t left = P.n - j;
  const char *x = P.X + (row * P.ldx + j) * XTraits<XT>::SIZE;
  u32x4 out[PARTS];
  if constexpr (SCALED) {
    float v[8], f[8];
    x_load8<XT>(x, left, v);
    x_load8<RSVD_X_F32>(reinterpret_cast<const char *>(P.factor + j), left, f);
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] *= f[u];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      unsigned p[PARTS];
      bf16_parts2<PARTS>(v[2 * u], v[2 * u + 1], p);
#pragma unroll
      for (int q = 0; q < PARTS; ++q) out[q][u] = p[q];
    }
  } else {
    split_operand<XT>(raw_load8<XT>(x, left), out);
  }
#pragma unroll
  for (int q = 0; q < PARTS; ++q) *reinterpret_cast<u32x4 *>(P.planes + q * P.rows * P.width + row * P.width + j) = out[q];
}

// Sixteen codes times `unit` as bf16 numbers.
__device__ __forceinline__ void widen16(const u32x4 &w, float unit, u32x4 (&p)[2]) {
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const unsigned d = w[2 * h + (u >> 1)];
      const float a = (float)((int)(d << (24 - 16 * (u & 1))) >> 24) * unit, b = (float)((int)(d << (16 - 16 * (u & 1))) >> 24) * unit;
      p[h][u] = bf16_pair(a, b);
    }
}

// plane[row][0 .. width): the codes of a row as bf16 numbers, multiplied by the powers of two of kept activations (NULL: as they are); width: n up to
// a multiple of 8.
struct WidenParams {
  const int8_t *codes; int64_t ldc;
  const uint8_t *powers; int64_t ldp;
  int64_t rows, n;
  uint16_t *plane; int64_t width;
  int64_t groups;                  // workgroups: 256 pieces of sixteen each
};
__device__ __forceinline__ void widen_group(const WidenParams &P, int64_t group) {
  int64_t row;
  int place;
  piece_of(group, (int)((P.n + 15) / 16), row, place);
  const int64_t j = 16 * (int64_t)place;
  if (row >= P.rows) return;
  const u32x4 w = *reinterpret_cast<const u32x4 *>(P.codes + row * P.ldc + j);
  const float unit = P.powers != nullptr ? kept_unit(P.powers[row * P.ldp + (j >> 5)]) : 1.f;
  u32x4 p[2];
  widen16(w, unit, p);
#pragma unroll
  for (int h = 0; h < 2; ++h)
    if (j + 8 * h < P.width) *reinterpret_cast<u32x4 *>(P.plane + row * P.width + j + 8 * h) = p[h];
}

}  // namespace rsvd
