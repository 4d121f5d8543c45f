// Numbers to 8 bits and back, and the operand planes of the bf16 products of the layer operators.
#include "layer8_rows.hpp"

namespace rsvd {

// ---------------------------------------------------------------- rows with a scale each
template <int XT, int CH> __global__ __launch_bounds__(256) void rows8_kernel(const Rows8Params P) { rows8_row<XT, CH>(P, blockIdx.x); }

template <int XT> static void rows8_typed(hipStream_t s, const Rows8Params &P) {
  const int64_t chunks = ceil_div(P.width, 8);
  const dim3 grid((unsigned)P.rows);
  if (chunks <= 256) hipLaunchKernelGGL((rows8_kernel<XT, 1>), grid, dim3(256), 0, s, P);
  else if (chunks <= 512) hipLaunchKernelGGL((rows8_kernel<XT, 2>), grid, dim3(256), 0, s, P);
  else if (chunks <= 1024) hipLaunchKernelGGL((rows8_kernel<XT, 4>), grid, dim3(256), 0, s, P);
  else hipLaunchKernelGGL((rows8_kernel<XT, 8>), grid, dim3(256), 0, s, P);
}

hipError_t rows8_launch(hipStream_t s, rsvd_xtype type, int64_t rows, int64_t n, const void *X, int64_t ldx, int8_t *codes, int64_t ldq,
                        int64_t width, float *scale, const float *sums, int splits, int64_t r, int parts, uint16_t *t) {
  // (a launch has fewer than 2^32 threads; with sums there are kMaxTokens rows at the most, and one launch)
  for (int64_t row = 0; row < rows; row += kMaxTokens) {
    const int64_t some = rows - row < kMaxTokens ? rows - row : kMaxTokens;
    const Rows8Params P = {(const char *)X + row * ldx * xtype_size(type), ldx, some, (int)n, codes + row * ldq, ldq, (int)width, scale + row, sums,
                           splits, (int)rank_places(r), parts, t};
    if (type == RSVD_X_BF16) rows8_typed<RSVD_X_BF16>(s, P);
    else if (type == RSVD_X_F16) rows8_typed<RSVD_X_F16>(s, P);
    else rows8_typed<RSVD_X_F32>(s, P);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  return hipSuccess;
}

// ---------------------------------------------------------------- blocks of 32 with a power of two
// Memory is the bound.  16384 x 4096 bf16: 42 us to save (203 MB, 4.8 TB/s), 31 us to load; 1001 x 2999 fp32 4.4 and 6.4 us.
// Eight features a thread, so four lanes share a block.  A workgroup covers `lanes` chunks (a power of two, at least 4) of 256 / lanes rows.
__device__ __forceinline__ unsigned quad_max(unsigned x) {
  x = max(x, (unsigned)__builtin_amdgcn_mov_dpp((int)x, 0xb1, 0xf, 0xf, true));      // lanes 1 0 3 2
  return max(x, (unsigned)__builtin_amdgcn_mov_dpp((int)x, 0x4e, 0xf, 0xf, true));   // lanes 2 3 0 1
}

template <int XT>
__global__ __launch_bounds__(256) void keep8_save_kernel(const char *__restrict__ X, int64_t ldx, int64_t tokens, int n,
                                                         int8_t *__restrict__ codes, int64_t ldc, uint8_t *__restrict__ powers, int64_t ldp,
                                                         int shift) {
  const int c = (int)(blockIdx.x << shift) + (int)(threadIdx.x & ((1u << shift) - 1u));
  const int rows = 256 >> shift;
  if ((c >> 2) * 32 >= n) return;                       // (whole blocks only: the quads stay together)
  for (int64_t t = (int64_t)blockIdx.y * rows + (threadIdx.x >> shift); t < tokens; t += (int64_t)gridDim.y * rows) {
    float v[8], q[8];
    x_load8<XT>(X + (t * ldx + 8 * c) * XTraits<XT>::SIZE, n - 8 * c, v);
    unsigned top = 0u;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, magnitude(v[e]));
    top = quad_max(top);
    const bool bad = top >= 0x7f800000u;
    // a = f 2^E in [2^(E-1), 2^E): its biased exponent is E + 126 (0 below 2^-126), and e + 127 = E + 120
    int byte = (int)(top >> 23) - 6;
    byte = byte < 1 ? 1 : byte;
    const float per = __uint_as_float((unsigned)(254 - byte) << 23);      // 2^-e: 2^126 at the most, 2^-121 at the least
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float y = __builtin_rintf(v[e] * per);
      q[e] = bad ? 0.f : y > 127.f ? 127.f : y < -127.f ? -127.f : y;
    }
    if (8 * c < (n + 15) / 16 * 16) *reinterpret_cast<u32x2 *>(codes + t * ldc + 8 * c) = pack8(q);
    if ((c & 3) == 0) powers[t * ldp + (c >> 2)] = (uint8_t)(bad ? 255 : byte);
  }
}

template <int XT>
__global__ __launch_bounds__(256) void keep8_load_kernel(const int8_t *__restrict__ codes, int64_t ldc, const uint8_t *__restrict__ powers,
                                                         int64_t ldp, int64_t tokens, int n, char *__restrict__ X, int64_t ldx, int shift) {
  const int c = (int)(blockIdx.x << shift) + (int)(threadIdx.x & ((1u << shift) - 1u));
  const int rows = 256 >> shift;
  if (8 * c >= n) return;
  for (int64_t t = (int64_t)blockIdx.y * rows + (threadIdx.x >> shift); t < tokens; t += (int64_t)gridDim.y * rows) {
    const u32x2 w = *reinterpret_cast<const u32x2 *>(codes + t * ldc + 8 * c);
    const float unit = kept_unit(powers[t * ldp + (c >> 2)]);
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)((int)(w[e >> 2] << (24 - 8 * (e & 3))) >> 24) * unit;
    char *x = X + (t * ldx + 8 * c) * XTraits<XT>::SIZE;
    if constexpr (XT == RSVD_X_F32) {
      if (n - 8 * c >= 8) {
        reinterpret_cast<f32x4_any *>(x)[0] = f32x4{v[0], v[1], v[2], v[3]};
        reinterpret_cast<f32x4_any *>(x)[1] = f32x4{v[4], v[5], v[6], v[7]};
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (8 * c + e < n) reinterpret_cast<float *>(x)[e] = v[e];
      }
    } else {
      u32x4 p;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (XT == RSVD_X_BF16) p[e] = bf16_pair(v[2 * e], v[2 * e + 1]);
        else p[e] = __builtin_bit_cast(unsigned, __builtin_convertvector(f32x2{v[2 * e], v[2 * e + 1]}, f16x2));
      }
      if (n - 8 * c >= 8) {
        *reinterpret_cast<u32x4_any *>(x) = p;
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (8 * c + e < n) reinterpret_cast<uint16_t *>(x)[e] = (uint16_t)(p[e >> 1] >> (16 * (e & 1)));
      }
    }
  }
}

// Lanes along a row (log2) and grid of the two kernels above.
static dim3 keep8_grid(int64_t tokens, int64_t n, int &shift) {
  const int64_t chunks = ceil_div(n, 32) * 4;
  shift = 2;
  while (shift < 8 && (1 << shift) < chunks) ++shift;
  int64_t groups = ceil_div(tokens, 256 >> shift);
  if (groups > 65535) groups = 65535;
  return dim3((unsigned)ceil_div(chunks, 1 << shift), (unsigned)groups);
}

hipError_t keep8_save_launch(hipStream_t s, rsvd_xtype type, int64_t tokens, int64_t n, const void *X, int64_t ldx, int8_t *codes,
                             int64_t ldc, uint8_t *powers, int64_t ldp) {
  int shift;
  const dim3 grid = keep8_grid(tokens, n, shift);
#define SAVE(XT)                                                                                                                        \
  hipLaunchKernelGGL(keep8_save_kernel<XT>, grid, dim3(256), 0, s, (const char *)X, ldx, tokens, (int)n, codes, ldc, powers, ldp, shift)
  if (type == RSVD_X_BF16) SAVE(RSVD_X_BF16);
  else if (type == RSVD_X_F16) SAVE(RSVD_X_F16);
  else SAVE(RSVD_X_F32);
#undef SAVE
  return hipGetLastError();
}

hipError_t keep8_load_launch(hipStream_t s, rsvd_xtype type, int64_t tokens, int64_t n, const int8_t *codes, int64_t ldc,
                             const uint8_t *powers, int64_t ldp, void *X, int64_t ldx) {
  int shift;
  const dim3 grid = keep8_grid(tokens, n, shift);
#define LOAD(XT)                                                                                                                    \
  hipLaunchKernelGGL(keep8_load_kernel<XT>, grid, dim3(256), 0, s, codes, ldc, powers, ldp, tokens, (int)n, (char *)X, ldx, shift)
  if (type == RSVD_X_BF16) LOAD(RSVD_X_BF16);
  else if (type == RSVD_X_F16) LOAD(RSVD_X_F16);
  else LOAD(RSVD_X_F32);
#undef LOAD
  return hipGetLastError();
}

// ---------------------------------------------------------------- zeros
__global__ __launch_bounds__(256) void fill_zero_kernel(float *__restrict__ out, int64_t rows, int64_t cols, int64_t ld) {
  for (int64_t r = blockIdx.y; r < rows; r += gridDim.y)
    for (int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x; c < cols; c += (int64_t)gridDim.x * 256) out[r * ld + c] = 0.f;
}

hipError_t fill_zero_launch(hipStream_t s, int64_t rows, int64_t cols, float *out, int64_t ld) {
  const int64_t gx = ceil_div(cols, 256), gy = rows < 4096 ? rows : 4096;
  hipLaunchKernelGGL(fill_zero_kernel, dim3((unsigned)(gx < 64 ? gx : 64), (unsigned)gy), dim3(256), 0, s, out, rows, cols, ld);
  return hipGetLastError();
}

}  // namespace rsvd
