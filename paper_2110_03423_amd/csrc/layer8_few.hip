// The product of codes for a few tokens.  Memory is the bound: the weight passes once, in
// sixteen rows a workgroup, straight from memory into the matrix instructions; four or eight wavefronts take the pieces of k in turn and
// add up at the end.  (One token, 4096 x 4096: 6.9 us, 2.4 TB/s; 7 tokens, 2000 x 10000: 9.4 us, 2.1 TB/s.  All loads of a workgroup are under way at
// once, and all workgroups fit on the chip, so what is left is a launch, one round of memory, and the end.)
#include "layer8_epilogue.hpp"

namespace rsvd {

struct FewParams {
  const char *A, *B;
  int64_t lda, ldb, M, N;
  int steps;                       // of 64 k
  int b_pieces;                    // 16-byte pieces of a row of B that may be read
  const float *sums; int splits;             // the low-rank sums over ranges of k, or NULL: E.t
  Layer8Epilogue E;
};

// TB blocks of sixteen tokens, WAVES wavefronts.
template <int TB, int WAVES> __global__ __launch_bounds__(64 * WAVES) void few_kernel(const FewParams P) {
  __shared__ i32x4 part[WAVES][TB][64];
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
  i32x4 acc[TB];
  f32x4 low[TB];
#pragma unroll
  for (int i = 0; i < TB; ++i) {
    acc[i] = (i32x4)0;
    low[i] = (f32x4)0.f;
  }
  // The loads of several steps are issued together, those of the low-rank term and of the weight ahead of the first matrix instruction.
  constexpr int LU = TB == 1 ? 2 : 1, U = TB == 1 ? 8 : TB == 2 ? 4 : 2;
  // low-rank term; sums over ranges of k need not be joined: the second product is linear
  const int low_steps = (P.sums != nullptr ? P.splits : E.parts) * E.rp / 32;
  u32x4 g[LU];
  Raw8<RSVD_X_F32> t[LU][TB];
  auto load_low = [&](int c0) RSVD_INLINE {
#pragma unroll
    for (int u = 0; u < LU; ++u) {
      const int c = c0 + WAVES * u < low_steps ? c0 + WAVES * u : c0;
      const int which = 32 * c / E.rp, p = 32 * c - which * E.rp + 8 * kq;
      g[u] = factor8(E, row, p);
      const bool none = c0 + WAVES * u >= low_steps;      // (zeros on both sides: sums may be infinite)
      if (none) g[u] = (u32x4)0u;
#pragma unroll
      for (int i = 0; i < TB; ++i) {
        const int64_t m = 16 * i + r16 < P.M ? 16 * i + r16 : P.M - 1;
        if (P.sums != nullptr) t[u][i] = raw_load8<RSVD_X_F32>(reinterpret_cast<const char *>(P.sums + ((int64_t)which * P.M + m) * E.rp + p), 8);
        else t[u][i].w[0] = *reinterpret_cast<const u32x4 *>(E.t + (m * E.parts + which) * E.rp + p);
        if (none) t[u][i].w[0] = t[u][i].w[1] = (u32x4)0u;
      }
    }
  };
  auto multiply_low = [&]() RSVD_INLINE {
#pragma unroll
    for (int u = 0; u < LU; ++u)
#pragma unroll
      for (int i = 0; i < TB; ++i) {
        if (P.sums != nullptr) {
          u32x4 x[3];
          split_operand<RSVD_X_F32>(t[u][i], x);
#pragma unroll
          for (int q = 2; q >= 0; --q) low[i] = mfma_bf16(g[u], x[q], low[i]);
        } else {
          low[i] = mfma_bf16(g[u], t[u][i].w[0], low[i]);
        }
      }
  };
  u32x4 x[U], y[U][TB];
  auto load = [&](int s0) RSVD_INLINE {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int s = s0 + WAVES * u;
      if (s < P.steps) {
        x[u] = *reinterpret_cast<const u32x4 *>(b + (4 * s + kq < P.b_pieces ? 64 * s + 16 * kq : 0));      // (behind those: the first, the tokens' codes are zero)
#pragma unroll
        for (int i = 0; i < TB; ++i) y[u][i] = *reinterpret_cast<const u32x4 *>(a[i] + 64 * s);
      } else {
        x[u] = (u32x4)0u;
#pragma unroll
        for (int i = 0; i < TB; ++i) y[u][i] = (u32x4)0u;
      }
    }
  };
  load(wave);
  for (int c = wave; c < low_steps; c += WAVES * LU) {
    load_low(c);
    multiply_low();
  }
  for (int s0 = wave; s0 < P.steps;) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < TB; ++i) acc[i] = mfma_codes(x[u], y[u][i], acc[i]);
    s0 += WAVES * U;
    if (s0 < P.steps) load(s0);
  }
#pragma unroll
  for (int i = 0; i < TB; ++i) part[wave][i][lane] = acc[i];
  __syncthreads();
  i32x4 sum = (i32x4)0;                                // (of block `wave` of the tokens)
  if (wave < TB) {
#pragma unroll
    for (int w = 0; w < WAVES; ++w) sum += part[w][wave][lane];
  }
  if (E.r > 0) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < TB; ++i) part[wave][i][lane] = __builtin_bit_cast(i32x4, low[i]);
    __syncthreads();
  }
  if (wave < TB) {
    const int i = wave;
    f32x4 val = (f32x4)0.f;
    if (E.r > 0) {
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        const i32x4 bits = part[w][i][lane];
        val += __builtin_bit_cast(f32x4, bits);
      }
    }
    const int64_t m = 16 * i + r16, n = n0 + 4 * kq;
    if (m >= P.M || n >= P.N) return;
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
  P.b_pieces = (int)(d.b_bytes / 16);
  P.E = layer8_epilogue(d.out);
  P.sums = d.sums; P.splits = d.splits;
  const dim3 grid((unsigned)ceil_div(d.N, 16));
  // one load of the weight's rows is all that a wavefront has to do, where eight of them can hold a row
  const bool wide = P.steps > 32;
  const dim3 block(wide ? 512 : 256);
#define FEW(TB)                                                              \
  if (wide) hipLaunchKernelGGL((few_kernel<TB, 8>), grid, block, 0, s, P);   \
  else hipLaunchKernelGGL((few_kernel<TB, 4>), grid, block, 0, s, P)
  if (d.M <= 16) { FEW(1); }
  else if (d.M <= 32) { FEW(2); }
  else { FEW(4); }
#undef FEW
  return hipGetLastError();
}

}  // namespace rsvd
