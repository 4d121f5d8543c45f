// Orthogonalising an update: its norm, and the first iterate.
#include "dense_tile.hpp"
#include "layer8_rows.hpp"

namespace rsvd {

// Sums of squares of a matrix in fp64, in kNormParts parts, added by whoever needs the norm, always in the same order.  (fp32 squares would leave its range for
// gradients of 1e-20 or 1e20.)  Memory is the bound: 2 of 8192 x 4096 in bf16 34 us, 3.9 TB/s; the first iterate, 403 MB, 70 us.
template <int XT> __global__ __launch_bounds__(256) void norm_kernel(const char *G, int64_t ldg, int64_t stride, int64_t m, int64_t n, double *parts) {
  constexpr int SIZE = XTraits<XT>::SIZE;
  __shared__ double wave_sum[4];
  const int tid = threadIdx.x;
  const char *g = G + (int64_t)blockIdx.y * stride * SIZE;
  const int per_row = (int)((n + 7) / 8);
  const int64_t total = m * per_row;
  double sum = 0.0;
  constexpr int U = 4;                                   // loads in flight
  for (int64_t group = blockIdx.x; group * 256 < total; group += U * kNormParts) {
    Raw8<XT> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      int64_t r;
      int c;
      piece_of(group + u * kNormParts, per_row, r, c);
      v[u] = raw_load8<XT>(g + (r * ldg + 8 * c) * SIZE, r < m ? n - 8 * c : 0);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float x[8];
      x_values<XT>(v[u], x);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += (double)x[e] * (double)x[e];
    }
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) sum += __shfl_down(sum, d);
  if ((tid & 63) == 0) wave_sum[tid >> 6] = sum;
  __syncthreads();
  if (tid == 0) parts[(int64_t)blockIdx.y * kNormParts + blockIdx.x] = (wave_sum[0] + wave_sum[1]) + (wave_sum[2] + wave_sum[3]);
}

template <int XT> __global__ __launch_bounds__(256) void unit_kernel(const char *G, int64_t ldg, int64_t stride, int64_t m, int64_t n, const double *parts,
                                                                    uint16_t *X, int64_t width, int64_t plane) {
  constexpr int SIZE = XTraits<XT>::SIZE;
  static_assert(kNormParts == 256, "one a thread");
  __shared__ double wave_sum[4];
  const int tid = threadIdx.x;
  double sum = parts[(int64_t)blockIdx.y * kNormParts + tid];
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) sum += __shfl_down(sum, d);
  if ((tid & 63) == 0) wave_sum[tid >> 6] = sum;
  __syncthreads();
  sum = (wave_sum[0] + wave_sum[1]) + (wave_sum[2] + wave_sum[3]);
  const double norm = sqrt(sum);
  // (a matrix of zeros stays one; with an infinity or NaN everything is NaN)
  const double scale = norm > 0.0 ? (norm < 1e300 ? 8192.0 / norm : (double)__uint_as_float(0x7fc00000u)) : norm == 0.0 ? 0.0 : norm;
  const char *g = G + (int64_t)blockIdx.y * stride * SIZE;
  uint16_t *x = X + (int64_t)blockIdx.y * m * width;
  const int per_row = (int)(width / 8);
  const int64_t total = m * per_row;
  for (int64_t group = blockIdx.x; group * 256 < total; group += gridDim.x) {
    int64_t r;
    int c;
    piece_of(group, per_row, r, c);
    if (r >= m) continue;
    const int64_t left = n - 8 * c;
    float v[8];
    x_values<XT>(raw_load8<XT>(g + (r * ldg + 8 * c) * SIZE, left), v);
    u32x4 high, low;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      f32x2 y;
#pragma unroll
      for (int h = 0; h < 2; ++h) y[h] = 2 * q + h < left ? (float)((double)v[2 * q + h] * scale) : 0.f;
      const f16x2 f = __builtin_convertvector(y, f16x2);
      high[q] = __builtin_bit_cast(unsigned, f);
      low[q] = __builtin_bit_cast(unsigned, __builtin_convertvector(y - __builtin_convertvector(f, f32x2), f16x2));
    }
    uint16_t *to = x + r * width + 8 * c;
    *reinterpret_cast<u32x4 *>(to) = high;
    *reinterpret_cast<u32x4 *>(reinterpret_cast<char *>(to) + plane) = low;
  }
}

hipError_t norm_launch(hipStream_t s, rsvd_xtype type, int batch, int64_t m, int64_t n, const void *G, int64_t ldg, int64_t stride, double *parts) {
  const dim3 grid(kNormParts, (unsigned)batch);
  const char *g = (const char *)G;
  if (type == RSVD_X_BF16) hipLaunchKernelGGL((norm_kernel<RSVD_X_BF16>), grid, dim3(256), 0, s, g, ldg, stride, m, n, parts);
  else if (type == RSVD_X_F16) hipLaunchKernelGGL((norm_kernel<RSVD_X_F16>), grid, dim3(256), 0, s, g, ldg, stride, m, n, parts);
  else hipLaunchKernelGGL((norm_kernel<RSVD_X_F32>), grid, dim3(256), 0, s, g, ldg, stride, m, n, parts);
  return hipGetLastError();
}

hipError_t unit_launch(hipStream_t s, rsvd_xtype type, int batch, int64_t m, int64_t n, const void *G, int64_t ldg, int64_t stride, const double *parts,
                       uint16_t *X, int64_t width, int64_t plane) {
  int64_t groups = ceil_div(m * (width / 8), 256);
  if (groups > 2048) groups = 2048;
  const dim3 grid((unsigned)groups, (unsigned)batch);
  const char *g = (const char *)G;
  if (type == RSVD_X_BF16) hipLaunchKernelGGL((unit_kernel<RSVD_X_BF16>), grid, dim3(256), 0, s, g, ldg, stride, m, n, parts, X, width, plane);
  else if (type == RSVD_X_F16) hipLaunchKernelGGL((unit_kernel<RSVD_X_F16>), grid, dim3(256), 0, s, g, ldg, stride, m, n, parts, X, width, plane);
  else hipLaunchKernelGGL((unit_kernel<RSVD_X_F32>), grid, dim3(256), 0, s, g, ldg, stride, m, n, parts, X, width, plane);
  return hipGetLastError();
}

}  // namespace rsvd
