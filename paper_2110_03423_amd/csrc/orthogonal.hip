// Orthogonalising an update: its norm, and the first iterate.
#include "dense_tile.hpp"

namespace rsvd {

// Sums of squares of a matrix in fp64, kNormParts parts of it, added by whoever needs the norm in their order.  (fp32 squares would leave its range for gradients of
// 1e-20 or 1e20.)
template <int XT> __global__ __launch_bounds__(256) void norm_kernel(const char *G, int64_t ldg, int64_t stride, int64_t m, int64_t n, double *parts) {
  constexpr int SIZE = XTraits<XT>::SIZE;
  __shared__ double wave_sum[4];
  const int tid = threadIdx.x;
  const char *g = G + (int64_t)blockIdx.y * stride * SIZE;
  const int64_t per_row = (n + 7) / 8, total = m * per_row;
  double sum = 0.0;
  for (int64_t e = (int64_t)blockIdx.x * 256 + tid; e < total; e += (int64_t)kNormParts * 256) {
    const int64_t r = e / per_row, c = (e - r * per_row) * 8;
    float v[8];
    x_load8<XT>(g + (r * ldg + c) * SIZE, n - c, v);
#pragma unroll
    for (int x = 0; x < 8; ++x) sum += (double)v[x] * (double)v[x];
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) sum += __shfl_down(sum, d);
  if ((tid & 63) == 0) wave_sum[tid >> 6] = sum;
  __syncthreads();
  if (tid == 0) parts[(int64_t)blockIdx.y * kNormParts + blockIdx.x] = (wave_sum[0] + wave_sum[1]) + (wave_sum[2] + wave_sum[3]);
}

template <int XT> __global__ __launch_bounds__(256) void unit_kernel(const char *G, int64_t ldg, int64_t stride, int64_t m, int64_t n, const double *parts,
                                                                    uint16_t *X, int64_t width, int64_t plane, int planes) {
  constexpr int SIZE = XTraits<XT>::SIZE;
  const double *p = parts + (int64_t)blockIdx.y * kNormParts;
  double sum = 0.0;
  for (int i = 0; i < kNormParts; ++i) sum += p[i];
  const double norm = sqrt(sum);
  // (a matrix of zeros stays one; with an infinity or NaN everything is NaN)
  const double scale = norm > 0.0 ? (norm < 1e300 ? 8192.0 / norm : (double)__uint_as_float(0x7fc00000u)) : norm == 0.0 ? 0.0 : norm;
  const char *g = G + (int64_t)blockIdx.y * stride * SIZE;
  uint16_t *x = X + (int64_t)blockIdx.y * m * width;
  const int64_t per_row = width / 4, total = m * per_row;
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < total; e += (int64_t)gridDim.x * 256) {
    const int64_t r = e / per_row, c = (e - r * per_row) * 4;
    const int left = left_of(c, n);
    f32x4 v = load4<XT>(g, r * ldg + c, left);
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = q < left ? (float)((double)v[q] * scale) : 0.f;
    put4<RSVD_X_F16>(x, r * width + c, 4, v);
    if (planes == 2) {
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] -= (float)(_Float16)v[q];
      put4<RSVD_X_F16>(reinterpret_cast<char *>(x) + plane, r * width + c, 4, v);
    }
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
                       uint16_t *X, int64_t width, int64_t plane, int planes) {
  int64_t groups = ceil_div(m * (width / 4), 256);
  if (groups > 2048) groups = 2048;
  const dim3 grid((unsigned)groups, (unsigned)batch);
  const char *g = (const char *)G;
  if (type == RSVD_X_BF16) hipLaunchKernelGGL((unit_kernel<RSVD_X_BF16>), grid, dim3(256), 0, s, g, ldg, stride, m, n, parts, X, width, plane, planes);
  else if (type == RSVD_X_F16) hipLaunchKernelGGL((unit_kernel<RSVD_X_F16>), grid, dim3(256), 0, s, g, ldg, stride, m, n, parts, X, width, plane, planes);
  else hipLaunchKernelGGL((unit_kernel<RSVD_X_F32>), grid, dim3(256), 0, s, g, ldg, stride, m, n, parts, X, width, plane, planes);
  return hipGetLastError();
}

}  // namespace rsvd
