// The products of a few tokens, and the first product of the low-rank term.  Memory is the bound: the weight passes once, in
// sixteen rows a workgroup, straight from memory into the matrix instructions; eight wavefronts take the pieces of k in turn and
// add up at the end.
#include "layer8_epilogue.hpp"

namespace rsvd {

constexpr int kFewWaves = 8;

struct FewParams {
  const char *A, *B;
  int64_t lda, ldb, M, N;
  int steps;                       // of 64 k
  Layer8Epilogue E;
};

// TB blocks of sixteen tokens.
template <int TB> __global__ __launch_bounds__(64 * kFewWaves) void few_kernel(const FewParams P) {
  __shared__ i32x4 part[kFewWaves][TB][64];
  __shared__ f32x4 part_low[kFewWaves][TB][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, kq = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * 16;
  const Layer8Epilogue &E = P.E;
  const int64_t row = n0 + r16 < P.N ? n0 + r16 : P.N - 1;
  const char *b = P.B + row * P.ldb, *a[TB];
#pragma unroll
  for (int i = 0; i < TB; ++i) {
    const int64_t m = 16 * i + r16;
    a[i] = P.A + (m < P.M ? m : P.M - 1) * P.lda + 16 * kq;
  }
  // (pieces behind the row of codes: the first of the row, where the tokens' codes are zero)
  const int pieces = (int)(P.ldb / 16);
  i32x4 acc[TB];
#pragma unroll
  for (int i = 0; i < TB; ++i) acc[i] = (i32x4)0;
  constexpr int U = TB > 2 ? 2 : 4;                     // k-steps in flight
  for (int s0 = wave; s0 < P.steps; s0 += kFewWaves * U) {
    u32x4 x[U], y[U][TB];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int s = s0 + kFewWaves * u;
      if (s < P.steps) {
        x[u] = *reinterpret_cast<const u32x4 *>(b + (4 * s + kq < pieces ? 64 * s + 16 * kq : 0));
#pragma unroll
        for (int i = 0; i < TB; ++i) y[u][i] = *reinterpret_cast<const u32x4 *>(a[i] + 64 * s);
      } else {
        x[u] = (u32x4)0u;
#pragma unroll
        for (int i = 0; i < TB; ++i) y[u][i] = (u32x4)0u;
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < TB; ++i) acc[i] = mfma_codes(x[u], y[u][i], acc[i]);
  }
  // the wavefronts' integers are added before they are scaled: the sum is exact
  f32x4 low[TB];
#pragma unroll
  for (int i = 0; i < TB; ++i) low[i] = (f32x4)0.f;
  for (int p = 32 * wave; p < 2 * E.rp; p += 32 * kFewWaves) {
    const u32x4 g = factor8(E, row, (p < E.rp ? p : p - E.rp) + 8 * kq);
#pragma unroll
    for (int i = 0; i < TB; ++i) {
      const int64_t m = 16 * i + r16;
      const u32x4 t = *reinterpret_cast<const u32x4 *>(E.t + (m < P.M ? m : P.M - 1) * 2 * E.rp + p + 8 * kq);
      low[i] = mfma_bf16(g, t, low[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < TB; ++i) {
    part[wave][i][lane] = acc[i];
    part_low[wave][i][lane] = low[i];
  }
  __syncthreads();
  for (int i = wave; i < TB; i += kFewWaves) {
    i32x4 sum = part[0][i][lane];
    f32x4 val = part_low[0][i][lane];
#pragma unroll
    for (int w = 1; w < kFewWaves; ++w) {
      sum += part[w][i][lane];
      val += part_low[w][i][lane];
    }
    const int64_t m = 16 * i + r16, n = n0 + 4 * kq;
    if (m >= P.M || n >= P.N) continue;
    const float rs = E.rs != nullptr ? E.rs[m] : 1.f;
    const f32x4 cs = column4(E.cs, n, P.N, 1.f);
#pragma unroll
    for (int v = 0; v < 4; ++v) val[v] += (float)sum[v] * rs * cs[v];
    if (E.bias != nullptr) val += column4(E.bias, n, P.N, 0.f);
    store4(E, m, n, P.N, val);
  }
}

hipError_t few_launch(rsvd_ctx *, hipStream_t s, const FewDesc &d) {
  if (d.M < 1 || d.M > kFewTokens) return hipErrorInvalidValue;
  FewParams P;
  P.A = (const char *)d.A; P.B = (const char *)d.B;
  P.lda = d.lda; P.ldb = d.ldb; P.M = d.M; P.N = d.N;
  P.steps = (int)(d.k / 64);
  P.E = layer8_epilogue(d.out);
  const dim3 grid((unsigned)ceil_div(d.N, 16)), block(64 * kFewWaves);
  if (d.M <= 16) hipLaunchKernelGGL(few_kernel<1>, grid, block, 0, s, P);
  else if (d.M <= 32) hipLaunchKernelGGL(few_kernel<2>, grid, block, 0, s, P);
  else hipLaunchKernelGGL(few_kernel<4>, grid, block, 0, s, P);
  return hipGetLastError();
}

// ---------------------------------------------------------------- t = X F^T
struct LowrankParams {
  const char *X; int64_t ldx, tokens, n;
  const uint16_t *F; int64_t ldf; int r, rp;
  uint16_t *t;
  int x_vec, f_vec;
};

// 16 TB tokens and sixteen rows of F a workgroup; X is split into bf16 numbers on the way from memory to the matrix instructions.
template <int XT, int TB> __global__ __launch_bounds__(64 * kFewWaves) void lowrank_kernel(const LowrankParams P) {
  constexpr int PARTS = XTraits<XT>::PARTS;
  __shared__ f32x4 part[kFewWaves][TB][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, kq = lane >> 4;
  const int p0 = (int)blockIdx.x * 16;
  const int64_t t0 = (int64_t)blockIdx.y * (16 * TB);
  const int row = p0 + r16 < P.r ? p0 + r16 : P.r - 1;
  const uint16_t *f = P.F + row * P.ldf;
  f32x4 acc[TB];
#pragma unroll
  for (int i = 0; i < TB; ++i) acc[i] = (f32x4)0.f;
  for (int64_t k0 = 32 * wave; k0 < P.n; k0 += 32 * kFewWaves) {
    const int64_t k = k0 + 8 * kq, left = P.n - k;
    u32x4 g = {0u, 0u, 0u, 0u};
    if (P.f_vec && left >= 8) {
      g = *reinterpret_cast<const u32x4 *>(f + k);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < left) g[e >> 1] |= (unsigned)f[k + e] << (16 * (e & 1));
    }
#pragma unroll
    for (int i = 0; i < TB; ++i) {
      const int64_t m = t0 + 16 * i + r16;
      float v[8];
      x_load8<XT>(P.X + ((m < P.tokens ? m : P.tokens - 1) * P.ldx + k) * XTraits<XT>::SIZE, left, P.x_vec != 0, v);
      u32x4 x[PARTS];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        unsigned p[PARTS];
        bf16_parts2<PARTS>(v[2 * e], v[2 * e + 1], p);
#pragma unroll
        for (int q = 0; q < PARTS; ++q) x[q][e] = p[q];
      }
#pragma unroll
      for (int q = PARTS - 1; q >= 0; --q) acc[i] = mfma_bf16(g, x[q], acc[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < TB; ++i) part[wave][i][lane] = acc[i];
  __syncthreads();
  for (int i = wave; i < TB; i += kFewWaves) {
    f32x4 sum = part[0][i][lane];
#pragma unroll
    for (int w = 1; w < kFewWaves; ++w) sum += part[w][i][lane];
    const int64_t m = t0 + 16 * i + r16;
    const int p = p0 + 4 * kq;
    if (m >= P.tokens) continue;
    u32x2 hi, lo;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float a = p + 2 * h < P.r ? sum[2 * h] : 0.f, b = p + 2 * h + 1 < P.r ? sum[2 * h + 1] : 0.f;
      unsigned q[2];
      bf16_parts2<2>(a, b, q);
      hi[h] = q[0];
      lo[h] = q[1];
    }
    uint16_t *t = P.t + m * 2 * P.rp + p;
    *reinterpret_cast<u32x2 *>(t) = hi;
    *reinterpret_cast<u32x2 *>(t + P.rp) = lo;
  }
}

template <int XT> static void lowrank_typed(hipStream_t s, const LowrankParams &P) {
  const int tb = P.tokens <= 16 ? 1 : P.tokens <= 2048 ? 2 : 4;
  const dim3 grid((unsigned)(P.rp / 16), (unsigned)ceil_div(P.tokens, 16 * tb)), block(64 * kFewWaves);
  if (tb == 1) hipLaunchKernelGGL((lowrank_kernel<XT, 1>), grid, block, 0, s, P);
  else if (tb == 2) hipLaunchKernelGGL((lowrank_kernel<XT, 2>), grid, block, 0, s, P);
  else hipLaunchKernelGGL((lowrank_kernel<XT, 4>), grid, block, 0, s, P);
}

hipError_t lowrank_launch(hipStream_t s, rsvd_xtype type, int64_t tokens, int64_t n, int64_t r, const void *X, int64_t ldx, const void *F,
                          int64_t ldf, uint16_t *t) {
  LowrankParams P = {(const char *)X, ldx, tokens, n, (const uint16_t *)F, ldf, (int)r, (int)rank_places(r), t,
                     rows_aligned(X, ldx, xtype_size(type)) ? 1 : 0, rows_aligned(F, ldf, 2) ? 1 : 0};
  // (the grid's second extent ends at 65535)
  const int64_t chunk = 65535 * 64, size = xtype_size(type);
  for (int64_t t0 = 0; t0 < tokens; t0 += chunk) {
    LowrankParams Q = P;
    Q.X = P.X + t0 * ldx * size;
    Q.t = P.t + t0 * 2 * P.rp;
    Q.tokens = tokens - t0 < chunk ? tokens - t0 : chunk;
    if (type == RSVD_X_BF16) lowrank_typed<RSVD_X_BF16>(s, Q);
    else if (type == RSVD_X_F16) lowrank_typed<RSVD_X_F16>(s, Q);
    else lowrank_typed<RSVD_X_F32>(s, Q);
  }
  return hipGetLastError();
}

}  // namespace rsvd
