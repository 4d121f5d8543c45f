// A gated block beside its large products: a few tokens, gradients of kept products, operands in the order that the products want.
#include "dense_tile.hpp"
#include "layer8_rows.hpp"

namespace rsvd {

// ---------------------------------------------------------------- a few tokens
// Memory is the bound: the weight passes once, sixteen outputs a workgroup (their rows of gate and of up), straight from memory into the matrix instructions;
// the wavefronts take the steps of 32 k in turn and add up at the end.  One token of bf16, 2048 -> 4096: 7.3 us, 4.6 TB/s; 4096 -> 8192: 5.4 TB/s.
struct GatedFewParams {
  const char *X, *W;
  int64_t ldx, ldw, tokens, n, m;
  int steps;                       // of 32 k
  GatedOut out;
};

template <int XT> __device__ __forceinline__ f32x4 few_multiply(const Raw8<XT> &w, const Raw8<XT> &x, f32x4 acc) {
  if constexpr (XT == RSVD_X_BF16) {
    return mfma_bf16(w.w[0], x.w[0], acc);
  } else if constexpr (XT == RSVD_X_F16) {
    return mfma_f16(w.w[0], x.w[0], acc);
  } else {                                             // (the products that dense_segs names)
    u32x4 a[3], b[3];
    split_operand<XT>(w, a);
    split_operand<XT>(x, b);
    acc = mfma_bf16(a[2], b[0], acc);
    acc = mfma_bf16(a[1], b[1], acc);
    acc = mfma_bf16(a[0], b[2], acc);
    acc = mfma_bf16(a[1], b[0], acc);
    acc = mfma_bf16(a[0], b[1], acc);
    return mfma_bf16(a[0], b[0], acc);
  }
}

// TB blocks of sixteen tokens, WAVES wavefronts.
template <int XT, int TB, int WAVES> __global__ __launch_bounds__(64 * WAVES) void gated_few_kernel(const GatedFewParams P) {
  constexpr int SIZE = XTraits<XT>::SIZE, U = TB == 1 ? (SIZE == 2 ? 8 : 4) : TB == 2 ? (SIZE == 2 ? 4 : 2) : 2;      // steps whose loads are issued together
  __shared__ f32x4 part[WAVES][2][TB][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, kq = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * 16;
  const int64_t row = n0 + r16 < P.m ? n0 + r16 : P.m - 1;
  const char *w[2] = {P.W + row * P.ldw * SIZE, P.W + (P.m + row) * P.ldw * SIZE}, *x[TB];
#pragma unroll
  for (int i = 0; i < TB; ++i) {
    const int64_t t = 16 * i + r16;
    x[i] = P.X + (t < P.tokens ? t : P.tokens - 1) * P.ldx * SIZE;
  }
  f32x4 acc[2][TB];
#pragma unroll
  for (int i = 0; i < TB; ++i) acc[0][i] = acc[1][i] = (f32x4)0.f;
  Raw8<XT> a[U][2], b[U][TB];
  auto load = [&](int s0) RSVD_INLINE {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t k = 32 * (int64_t)(s0 + WAVES * u) + 8 * kq, left = s0 + WAVES * u < P.steps ? P.n - k : 0;
#pragma unroll
      for (int h = 0; h < 2; ++h) a[u][h] = raw_load8<XT>(w[h] + k * SIZE, left);
#pragma unroll
      for (int i = 0; i < TB; ++i) b[u][i] = raw_load8<XT>(x[i] + k * SIZE, left);
    }
  };
  for (int s0 = wave; s0 < P.steps; s0 += WAVES * U) {
    load(s0);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < TB; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) acc[h][i] = few_multiply<XT>(a[u][h], b[u][i], acc[h][i]);
  }
#pragma unroll
  for (int i = 0; i < TB; ++i) {
    part[wave][0][i][lane] = acc[0][i];
    part[wave][1][i][lane] = acc[1][i];
  }
  __syncthreads();
  if (wave >= TB) return;
  f32x4 g = (f32x4)0.f, u = g;
#pragma unroll
  for (int v = 0; v < WAVES; ++v) {
    g += part[v][0][wave][lane];
    u += part[v][1][wave][lane];
  }
  const int64_t t = 16 * wave + r16, n = n0 + 4 * kq;
  if (t < P.tokens && n < P.m) gated_end1(P.out, P.m, t, n, g, u);
}

template <int XT> static void gated_few_run(hipStream_t s, const GatedFewParams &P, dim3 grid, bool wide) {
#define FEW(TB)                                                                        \
  if (wide) hipLaunchKernelGGL((gated_few_kernel<XT, TB, 8>), grid, dim3(512), 0, s, P); \
  else hipLaunchKernelGGL((gated_few_kernel<XT, TB, 4>), grid, dim3(256), 0, s, P)
  if (P.tokens <= 16) { FEW(1); }
  else if (P.tokens <= 32) { FEW(2); }
  else if constexpr (XT == RSVD_X_F32) { FEW(4); }
#undef FEW
}

hipError_t gated_few_launch(rsvd_ctx *, hipStream_t s, const GatedFewDesc &d) {
  if (d.tokens < 1 || d.tokens > (d.type == RSVD_X_F32 ? 64 : 32)) return hipErrorInvalidValue;
  const GatedFewParams P = {(const char *)d.X, (const char *)d.W, d.ldx, d.ldw, d.tokens, d.n, d.m, (int)ceil_div(d.n, 32), d.out};
  const dim3 grid((unsigned)ceil_div(d.m, 16));
  const bool wide = P.steps > 32;
  if (d.type == RSVD_X_BF16) gated_few_run<RSVD_X_BF16>(s, P, grid, wide);
  else if (d.type == RSVD_X_F16) gated_few_run<RSVD_X_F16>(s, P, grid, wide);
  else gated_few_run<RSVD_X_F32>(s, P, grid, wide);
  return hipGetLastError();
}

// ---------------------------------------------------------------- the range of a gradient in fp16
// D = (dH u act', dH act) of fp16 tokens is held in fp16 times a power of two.  As it is it would leave the range on either side where neither gradient does: dH of 1e-5 lost 4.3e-3 of dW (2.1e-4 now, as with dH of 1e-2), and dH u
// above 65504 was an infinity.  With |act'| <= 1.13, |act| <= |g| and |g|, |u| <= G, |D| <= 1.13 max |dH| G; that, with room for rounding, is brought to 2^15 or more.  G is the largest
// product that was kept or, of those that are computed again, the largest norm of a row of X times that of a row of W.  What is not finite does not count: it stays what it is.
// Memory is the bound: 8192 x 4096 -> 8192 kept, 403 MB 84 us (4.8 TB/s), computed again, 335 MB 68 us, of a gradient of 2930; the second launch, one workgroup, takes 2 to 5.
struct RangeOf { const char *p; int64_t ld, rows, cols; bool norm; };

// Magnitudes of eight fp16 numbers, the largest that is finite.
__device__ __forceinline__ unsigned range_top8(u32x4 w, unsigned top) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const unsigned v = (w[e >> 1] >> (16 * (e & 1))) & 0x7fffu;
    top = max(top, v < 0x7c00u ? v : 0u);
  }
  return top;
}
__device__ __forceinline__ float range_squares8(u32x4 w, float sum) {
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    const unsigned pair = w[h];
    const f16x2 f = __builtin_bit_cast(f16x2, pair);
    sum += (float)f[0] * (float)f[0] + (float)f[1] * (float)f[1];
  }
  return sum;
}
// The largest magnitude of a matrix, or the largest sum of squares of a row, by parts.
__global__ __launch_bounds__(256) void range_kernel(const RangeOf first, const RangeOf second, const RangeOf third, float *parts) {
  const RangeOf M = blockIdx.y == 0 ? first : blockIdx.y == 1 ? second : third;
  __shared__ float wave_top[4];
  const int tid = threadIdx.x, lane = tid & 63, per_row = (int)((M.cols + 7) / 8);
  constexpr int U = 4;                                   // loads in flight
  float most = 0.f;
  auto finite = [](float v) RSVD_INLINE { return v < __uint_as_float(0x7f800000u) ? v : 0.f; };
  if (!M.norm) {
    const int64_t total = M.rows * per_row;
    unsigned top = 0u;
    for (int64_t group = blockIdx.x; group * 256 < total; group += U * gridDim.x) {
      u32x4 v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        int64_t r;
        int c;
        piece_of(group + u * gridDim.x, per_row, r, c);
        v[u] = halves8(reinterpret_cast<const uint16_t *>(M.p) + r * M.ld + 8 * c, r < M.rows ? M.cols - 8 * c : 0);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) top = range_top8(v[u], top);
    }
    most = (float)__builtin_bit_cast(_Float16, (uint16_t)top);
  } else {
    // a row by 64 lanes, or by as many of a power of two as have a piece of it
    int lanes = 64;
    while (lanes > 1 && lanes / 2 >= per_row) lanes >>= 1;
    const int at_once = 64 / lanes, place = lane & (lanes - 1);
    const int64_t wave = (int64_t)blockIdx.x * 4 + (tid >> 6), step = (int64_t)gridDim.x * 4 * at_once;
    for (int64_t row = wave * at_once + lane / lanes; row - lane / lanes < M.rows; row += U * step) {
      float sum[U] = {0.f, 0.f, 0.f, 0.f};
      for (int c = place; c - place < per_row; c += lanes) {
        u32x4 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int64_t r = row + u * step;
          v[u] = halves8(reinterpret_cast<const uint16_t *>(M.p) + r * M.ld + 8 * c, r < M.rows ? M.cols - 8 * c : 0);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) sum[u] = range_squares8(v[u], sum[u]);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        for (int d = 1; d < lanes; d <<= 1) sum[u] += __shfl_xor(sum[u], d);
        most = fmaxf(most, finite(sum[u]));
      }
    }
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) most = fmaxf(most, __shfl_xor(most, d));
  if (lane == 0) wave_top[tid >> 6] = most;
  __syncthreads();
  if (tid == 0) parts[blockIdx.y * gridDim.x + blockIdx.x] = fmaxf(fmaxf(wave_top[0], wave_top[1]), fmaxf(wave_top[2], wave_top[3]));
}
__global__ __launch_bounds__(256) void range_scale_kernel(const float *parts, int count, int norms, float *scale) {
  __shared__ float wave_top[3][4];
  const int tid = threadIdx.x;
  float top[3] = {0.f, 0.f, 0.f};
#pragma unroll
  for (int q = 0; q < 3; ++q) {
    if (q == 2 && norms == 0) break;
#pragma unroll
    for (int x = 0; x < kRangeParts; x += 256) top[q] = fmaxf(top[q], x + tid < count ? parts[q * count + x + tid] : 0.f);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top[q] = fmaxf(top[q], __shfl_xor(top[q], d));
  }
  if ((tid & 63) == 0)
#pragma unroll
    for (int q = 0; q < 3; ++q) wave_top[q][tid >> 6] = top[q];
  __syncthreads();
  if (tid > 0) return;
#pragma unroll
  for (int q = 0; q < 3; ++q) top[q] = fmaxf(fmaxf(wave_top[q][0], wave_top[q][1]), fmaxf(wave_top[q][2], wave_top[q][3]));
  // (the norms' sums, and the products', are off by up to 1 % of themselves for 2^17 numbers added in turn)
  const float bound = 1.14f * top[0] * (norms ? 1.02f * sqrtf(top[1]) * sqrtf(top[2]) : top[1]);
  const int up = bound > 0.f ? 15 - ilogbf(bound) : 0;   // (bounds: 2^-72 to 2^66)
  scale[0] = ldexpf(1.f, up);
  scale[1] = ldexpf(1.f, -up);
}
hipError_t range_launch(hipStream_t s, int64_t tokens, int64_t n, int64_t m, const void *dH, int64_t lddh, const void *kept, int64_t ldk, const void *X, int64_t ldx, const void *W,
                        int64_t ldw, float *parts, float *scale) {
  const bool norms = kept == nullptr;
  const RangeOf dh = {(const char *)dH, lddh, tokens, m, false};
  const RangeOf second = norms ? RangeOf{(const char *)X, ldx, tokens, n, true} : RangeOf{(const char *)kept, ldk, tokens, 2 * m, false}, third = {(const char *)W, ldw, 2 * m, n, true};
  const int64_t pieces = (norms ? (tokens + 2 * m) * ceil_div(n, 8) : tokens * ceil_div(2 * m, 8)) + tokens * ceil_div(m, 8);
  const int count = pieces >= 1024 * kRangeParts ? kRangeParts : (int)ceil_div(pieces, 1024);
  hipLaunchKernelGGL(range_kernel, dim3((unsigned)count, norms ? 3 : 2), dim3(256), 0, s, dh, second, third, parts);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(range_scale_kernel, dim3(1), dim3(256), 0, s, parts, count, (int)norms, scale);
  return hipGetLastError();
}

// ---------------------------------------------------------------- operands
// Gradients of gate and up from the kept products, and matrices as the products want them; memory is the bound (301 x 2999 -> 1410 in fp32 with its weight: 106 MB in 17.6 us).  One launch: workgroups of the one, then of the others.
template <int TYPE> __device__ __forceinline__ void slope_group(const GatedOut &O, int64_t tokens, int64_t m, int64_t group) {
  int64_t t[1], n[1];
  int place;
  piece_of(group, (int)((m + 7) / 8), t[0], place);
  n[0] = 8 * (int64_t)place;
  const bool there[1] = {t[0] < tokens};
  if (!there[0]) return;
  const int left = left_of<2>(n[0], m);
  f32x4 g[1][2], u[1][2];
  load_row<TYPE, 2>(O.kept, t[0] * O.ldk + n[0], left, g[0]);
  load_row<TYPE, 2>(O.kept, t[0] * O.ldk + m + n[0], left, u[0]);
  gated_end<1, 2, false>(O, m, t, n, there, g, u);
}
template <int XT> __device__ __forceinline__ void planes_group(const LayOut &L, int64_t n, int64_t width, int64_t group) {
  constexpr int SIZE = XTraits<XT>::SIZE;
  int64_t r;
  int place;
  piece_of(group, (int)(width / 8), r, place);
  if (r >= L.rows) return;
  const int64_t c = 8 * (int64_t)place;
  const Raw8<XT> v = raw_load8<XT>(reinterpret_cast<const char *>(L.X) + (r * L.ldx + c) * SIZE, n - c);
  uint16_t *to = L.out + r * width + c;
  if constexpr (XT == RSVD_X_F32) {
    u32x4 p[3];
    split_operand<XT>(v, p);
#pragma unroll
    for (int q = 0; q < 3; ++q) *reinterpret_cast<u32x4 *>(to + q * (L.plane / 2)) = p[q];
  } else {
    *reinterpret_cast<u32x4 *>(to) = v.w[0];
  }
}
struct LayOutGroups { int64_t slope, x, w; };
template <int XT> __global__ __launch_bounds__(256) void lay_out_kernel(const LayOutGroups G, int64_t n, int64_t width, const LayOut X, const LayOut W, int64_t tokens, int64_t m,
                                                                       const GatedOut O) {
  for (int64_t group = blockIdx.x; group < G.slope + G.x + G.w; group += gridDim.x) {
    if (group < G.slope) slope_group<XT>(O, tokens, m, group);
    else if (group < G.slope + G.x) planes_group<XT>(X, n, width, group - G.slope);
    else planes_group<XT>(W, n, width, group - G.slope - G.x);
  }
}
hipError_t lay_out_launch(hipStream_t s, rsvd_xtype type, int64_t n, int64_t width, const LayOut &x, const LayOut &w, int64_t tokens, int64_t m, const GatedOut &slope) {
  const LayOutGroups G = {ceil_div(tokens * ceil_div(m, 8), 256), ceil_div(x.rows * (width / 8), 256), ceil_div(w.rows * (width / 8), 256)};
  int64_t groups = G.slope + G.x + G.w;
  if (groups == 0) return hipSuccess;
  if (groups > 65536) groups = 65536;
  const dim3 grid((unsigned)groups);
  if (type == RSVD_X_F32) hipLaunchKernelGGL((lay_out_kernel<RSVD_X_F32>), grid, dim3(256), 0, s, G, n, width, x, w, tokens, m, slope);
  else if (type == RSVD_X_F16) hipLaunchKernelGGL((lay_out_kernel<RSVD_X_F16>), grid, dim3(256), 0, s, G, n, width, x, w, tokens, m, slope);
  else hipLaunchKernelGGL((lay_out_kernel<RSVD_X_BF16>), grid, dim3(256), 0, s, G, n, width, x, w, tokens, m, slope);
  return hipGetLastError();
}

// ---------------------------------------------------------------- the gradient of no tokens
template <typename T> __global__ __launch_bounds__(256) void zero_kernel(T *C, int64_t ldc, int64_t rows, int64_t n) {
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < rows * n; e += (int64_t)gridDim.x * 256) C[e / n * ldc + e % n] = 0;
}
hipError_t zero_launch(hipStream_t s, rsvd_xtype type, int64_t rows, int64_t n, void *C, int64_t ldc) {
  int64_t groups = ceil_div(rows * n, 256);
  if (groups > 16384) groups = 16384;
  if (type == RSVD_X_F32) hipLaunchKernelGGL((zero_kernel<uint32_t>), dim3((unsigned)groups), dim3(256), 0, s, (uint32_t *)C, ldc, rows, n);
  else hipLaunchKernelGGL((zero_kernel<uint16_t>), dim3((unsigned)groups), dim3(256), 0, s, (uint16_t *)C, ldc, rows, n);
  return hipGetLastError();
}

}  // namespace rsvd
