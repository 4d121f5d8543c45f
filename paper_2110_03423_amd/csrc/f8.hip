// 8-bit floats (e4m3) in blocks of 128 that share a power of two: rounding to them, and the product of a few tokens.
//
// With a = max |x| of a block, its power 2^e is the least with a <= 448 2^e (448 is the largest code), e at least -126; held as the byte e + 127.  With a = 1.f 2^E
// that is E - 8, and one more where 1.f > 1.75: read off the bits.  x 2^-e is exact, the rounding to a code (nearest, ties to even) is the conversion instruction's.
// A block with an infinity or NaN has the byte 255 and codes that are NaN.
#include "dense_nt.hpp"
#include "layer8_rows.hpp"

namespace rsvd {

__device__ __forceinline__ unsigned f8_magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }
// The power byte of a block whose largest magnitude has these bits, and the factor for its numbers.
__device__ __forceinline__ unsigned f8_power(unsigned top) {
  const unsigned expo = top >> 23, more = (top & 0x7fffffu) > 0x600000u ? 1u : 0u;
  if (expo == 255u) return 255u;
  return expo + more > 9u ? expo + more - 8u : 1u;
}
__device__ __forceinline__ float f8_factor(unsigned power) { return power == 255u ? __uint_as_float(0x7fc00000u) : __uint_as_float((254u - power) << 23); }
// Four codes.  (A NaN: what the conversion makes of one.)
__device__ __forceinline__ unsigned f8_codes4(float a, float b, float c, float d, float by) {
  const int low = __builtin_amdgcn_cvt_pk_fp8_f32(a * by, b * by, 0, false);
  return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c * by, d * by, low, true);
}
__device__ __forceinline__ u32x2 f8_codes8(const float (&v)[8], float by) { return u32x2{f8_codes4(v[0], v[1], v[2], v[3], by), f8_codes4(v[4], v[5], v[6], v[7], by)}; }
__device__ __forceinline__ unsigned f8_top8(const float (&v)[8], unsigned top) {
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, f8_magnitude(v[e]));
  return top;
}
// (As integers the magnitudes' bits are ordered like them, infinity and NaN on top.)
__device__ __forceinline__ unsigned f8_shared(unsigned top, int mask) { return max(top, (unsigned)__shfl_xor((int)top, mask)); }

// Blocks of a row: eight lanes a block, sixteen numbers each.  Memory is the bound: 8192 x 16384 in bf16 70 us, 5.7 TB/s.
template <int XT> __global__ __launch_bounds__(256) void f8_rows_kernel(const char *X, int64_t ldx, int64_t rows, int64_t n, uint8_t *codes, int64_t width,
                                                                       uint8_t *powers, int64_t ldp) {
  constexpr int SIZE = XTraits<XT>::SIZE;
  const int per_row = (int)(width / 16);
  const int64_t total = rows * per_row;
  // (whole blocks end together: eight lanes have one)
  for (int64_t group = blockIdx.x; group * 256 < total; group += gridDim.x) {
    int64_t r;
    int place;
    piece_of(group, per_row, r, place);
    if (r >= rows) continue;
    const int64_t c = 16 * (int64_t)place;
    float v[2][8];
    unsigned top = 0u;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      x_load8<XT>(X + (r * ldx + c + 8 * h) * SIZE, n - c - 8 * h, v[h]);
      top = f8_top8(v[h], top);
    }
#pragma unroll
    for (int d = 1; d < 8; d <<= 1) top = f8_shared(top, d);
    const unsigned power = f8_power(top);
    const float by = f8_factor(power);
    const u32x2 a = f8_codes8(v[0], by), b = f8_codes8(v[1], by);
    *reinterpret_cast<u32x4 *>(codes + r * width + c) = u32x4{a[0], a[1], b[0], b[1]};
    if ((threadIdx.x & 7) == 0) powers[r * ldp + c / 128] = (uint8_t)power;
  }
}

// Blocks of 128 rows, 64 columns a workgroup: through LDS, a column a thread and then a row of codes.  Memory is the bound: 16384 x 12288 in bf16 132 us, 4.6 TB/s.
// Two matrices of the same rows in one launch, one behind the other (block by block of rows in turn, 16384 x 8192 and 4096 took a product of them 3 % more).
struct F8Columns { const char *X; int64_t ldx, n; uint8_t *codes, *powers; };
template <int XT> __global__ __launch_bounds__(256) void f8_columns_kernel(const F8Columns A, const F8Columns B, int a_groups, int64_t rows, int64_t width, int64_t ldp) {
  constexpr int SIZE = XTraits<XT>::SIZE, PITCH = 65, OUT = 144;
  __shared__ __attribute__((aligned(16))) float tile[128 * PITCH];
  __shared__ unsigned tops[4][64];
  const int tid = threadIdx.x, c = tid & 63, q = tid >> 6;
  const int row_blocks = (int)((rows + 127) / 128);
  const bool first = (int)blockIdx.x < a_groups * row_blocks;
  const int at = (int)blockIdx.x - (first ? 0 : a_groups * row_blocks);
  const char *const X = first ? A.X : B.X;
  const int64_t ldx = first ? A.ldx : B.ldx, n = first ? A.n : B.n;
  uint8_t *const codes = first ? A.codes : B.codes, *const powers = first ? A.powers : B.powers;
  const int across = (int)((n + 63) / 64), row_block = at / across;
  const int64_t r0 = (int64_t)row_block * 128, c0 = (int64_t)(at - row_block * across) * 64;
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    const int row = (tid >> 3) + 32 * p, col = 8 * (tid & 7);
    float v[8];
    x_load8<XT>(X + ((r0 + row) * ldx + c0 + col) * SIZE, r0 + row < rows ? n - c0 - col : 0, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) tile[row * PITCH + col + e] = v[e];
  }
  __syncthreads();
  float v[4][8];
  unsigned top = 0u;
#pragma unroll
  for (int p = 0; p < 4; ++p) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[p][e] = tile[(32 * q + 8 * p + e) * PITCH + c];
    top = f8_top8(v[p], top);
  }
  tops[q][c] = top;
  __syncthreads();
  top = max(max(tops[0][c], tops[1][c]), max(tops[2][c], tops[3][c]));
  const unsigned power = f8_power(top);
  const float by = f8_factor(power);
  if (q == 0 && c0 + c < n) powers[(c0 + c) * ldp + row_block] = (uint8_t)power;
  char *const out = reinterpret_cast<char *>(tile);      // (everybody has read the tile)
#pragma unroll
  for (int p = 0; p < 4; p += 2) {
    const u32x2 a = f8_codes8(v[p], by), b = f8_codes8(v[p + 1], by);
    *reinterpret_cast<u32x4 *>(out + c * OUT + 32 * q + 8 * p) = u32x4{a[0], a[1], b[0], b[1]};
  }
  __syncthreads();
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const int row = (tid >> 3) + 32 * p, at = 16 * (tid & 7);
    if (c0 + row < n) *reinterpret_cast<u32x4 *>(codes + (c0 + row) * width + r0 + at) = *reinterpret_cast<const u32x4 *>(out + row * OUT + at);
  }
}

// Blocks of 128 x 128, one a workgroup, in both orders; the other one through LDS, in words of four codes that a thread exchanges for those of four rows.  Memory is the bound:
// 16384 x 4096 in bf16 51 us, 5.3 TB/s (two threads a row, 64 numbers each, and bytes gathered one by one: 138).
template <int XT> __global__ __launch_bounds__(256) void f8_weight_kernel(const char *W, int64_t ldw, int64_t m, int64_t n, uint8_t *codes, int64_t ldq, uint8_t *powers,
                                                                         int64_t ldp, uint8_t *codes_t, int64_t ldqt, uint8_t *powers_t, int64_t ldpt) {
  constexpr int SIZE = XTraits<XT>::SIZE, PITCH = 33, SHIFT = 8;      // words of a row, and more behind each sixteen rows: the rows that are read together start at different banks
  __shared__ unsigned tile[128 * PITCH + 8 * SHIFT];
  __shared__ unsigned tops[4];
  const int tid = threadIdx.x, line = tid >> 4, col = 8 * (tid & 15);
  const int64_t r0 = (int64_t)blockIdx.y * 128, c0 = (int64_t)blockIdx.x * 128;
  float v[8][8];
  unsigned top = 0u;
#pragma unroll
  for (int p = 0; p < 8; ++p) x_load8<XT>(W + ((r0 + line + 16 * p) * ldw + c0 + col) * SIZE, r0 + line + 16 * p < m ? n - c0 - col : 0, v[p]);
#pragma unroll
  for (int p = 0; p < 8; ++p) top = f8_top8(v[p], top);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) top = f8_shared(top, d);
  if ((tid & 63) == 0) tops[tid >> 6] = top;
  __syncthreads();
  top = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
  const unsigned power = f8_power(top);
  const float by = f8_factor(power);
  if (tid == 0) {
    powers[blockIdx.y * ldp + blockIdx.x] = (uint8_t)power;
    if (powers_t != nullptr) powers_t[blockIdx.x * ldpt + blockIdx.y] = (uint8_t)power;
  }
#pragma unroll
  for (int p = 0; p < 8; ++p) {
    const u32x2 a = f8_codes8(v[p], by);
    const int row = line + 16 * p;
    if (r0 + row < m) *reinterpret_cast<u32x2 *>(codes + (r0 + row) * ldq + c0 + col) = a;
    unsigned *to = tile + row * PITCH + p * SHIFT + (col >> 2);
    to[0] = a[0];
    to[1] = a[1];
  }
  if (codes_t == nullptr) return;
  __syncthreads();
  const int group = tid & 7, word = tid >> 3;            // sixteen rows, four columns
  u32x4 out[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    unsigned w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = tile[(16 * group + 4 * q + e) * PITCH + group * SHIFT + word];
    // (bytes 0 and 1, and 2 and 3, of two rows in turn, and then of all four)
    const unsigned a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), b = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u);
    const unsigned c = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u), d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
    out[0][q] = __builtin_amdgcn_perm(c, a, 0x05040100u);
    out[1][q] = __builtin_amdgcn_perm(c, a, 0x07060302u);
    out[2][q] = __builtin_amdgcn_perm(d, b, 0x05040100u);
    out[3][q] = __builtin_amdgcn_perm(d, b, 0x07060302u);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (c0 + 4 * word + e < n) *reinterpret_cast<u32x4 *>(codes_t + (c0 + 4 * word + e) * ldqt + r0 + 16 * group) = out[e];
}

hipError_t f8_rows_launch(hipStream_t s, rsvd_xtype type, int64_t rows, int64_t n, const void *X, int64_t ldx, uint8_t *codes, int64_t width, uint8_t *powers,
                          int64_t ldp) {
  int64_t groups = ceil_div(rows * (width / 16), 256);
  if (groups > 65536) groups = 65536;
  const dim3 grid((unsigned)groups);
  const char *x = (const char *)X;
  if (type == RSVD_X_BF16) hipLaunchKernelGGL((f8_rows_kernel<RSVD_X_BF16>), grid, dim3(256), 0, s, x, ldx, rows, n, codes, width, powers, ldp);
  else if (type == RSVD_X_F16) hipLaunchKernelGGL((f8_rows_kernel<RSVD_X_F16>), grid, dim3(256), 0, s, x, ldx, rows, n, codes, width, powers, ldp);
  else hipLaunchKernelGGL((f8_rows_kernel<RSVD_X_F32>), grid, dim3(256), 0, s, x, ldx, rows, n, codes, width, powers, ldp);
  return hipGetLastError();
}

hipError_t f8_columns_launch(hipStream_t s, rsvd_xtype type, int64_t rows, int64_t m, const void *Y, int64_t ldy, uint8_t *y_codes, uint8_t *y_powers, int64_t n, const void *X,
                             int64_t ldx, uint8_t *x_codes, uint8_t *x_powers, int64_t width, int64_t ldp) {
  const F8Columns A = {(const char *)Y, ldy, m, y_codes, y_powers}, B = {(const char *)X, ldx, n, x_codes, x_powers};
  const int a_groups = (int)ceil_div(m, 64);
  const dim3 grid((unsigned)((a_groups + ceil_div(n, 64)) * ceil_div(rows, 128)));
  if (type == RSVD_X_BF16) hipLaunchKernelGGL((f8_columns_kernel<RSVD_X_BF16>), grid, dim3(256), 0, s, A, B, a_groups, rows, width, ldp);
  else if (type == RSVD_X_F16) hipLaunchKernelGGL((f8_columns_kernel<RSVD_X_F16>), grid, dim3(256), 0, s, A, B, a_groups, rows, width, ldp);
  else hipLaunchKernelGGL((f8_columns_kernel<RSVD_X_F32>), grid, dim3(256), 0, s, A, B, a_groups, rows, width, ldp);
  return hipGetLastError();
}

hipError_t f8_weight_launch(hipStream_t s, rsvd_xtype type, int64_t m, int64_t n, const void *W, int64_t ldw, uint8_t *codes, int64_t ldq, uint8_t *powers, int64_t ldp,
                            uint8_t *codes_t, int64_t ldqt, uint8_t *powers_t, int64_t ldpt) {
  const dim3 grid((unsigned)ceil_div(n, 128), (unsigned)ceil_div(m, 128));
  const char *w = (const char *)W;
#define WEIGHT(XT) hipLaunchKernelGGL((f8_weight_kernel<XT>), grid, dim3(256), 0, s, w, ldw, m, n, codes, ldq, powers, ldp, codes_t, ldqt, powers_t, ldpt)
  if (type == RSVD_X_BF16) WEIGHT(RSVD_X_BF16);
  else if (type == RSVD_X_F16) WEIGHT(RSVD_X_F16);
  else WEIGHT(RSVD_X_F32);
#undef WEIGHT
  return hipGetLastError();
}

// ---------------------------------------------------------------- a few tokens
// Memory is the bound: the weight passes once, sixteen rows a workgroup, straight from memory into the matrix instructions; the wavefronts take the steps of
// 128 k in turn and add up at the end.  Every workgroup rounds the tokens again: a lane has 32 numbers of a token's block, and their codes are its operand as they are.
struct F8FewParams {
  const char *X; int64_t ldx, tokens, n, m;
  const uint8_t *codes, *powers; int64_t ldq, ldp;
  int steps;                       // of 128 k
  void *Y; int64_t ldy;
};

template <int XT, int WAVES> __global__ __launch_bounds__(64 * WAVES, 4) void f8_few_kernel(const F8FewParams P) {
  constexpr int SIZE = XTraits<XT>::SIZE, U = 2;        // steps whose weights are under way together (four: more registers than two workgroups on a CU allow, 10.9 for 10.1 us at 4096 -> 8192)
  __shared__ f32x4 part[WAVES][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, kq = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * 16;
  const int64_t row = n0 + r16 < P.m ? n0 + r16 : P.m - 1;
  const uint8_t *const w = P.codes + row * P.ldq + 32 * kq, *const powers = P.powers + (n0 >> 7) * P.ldp;
  const char *const x = P.X + (r16 < P.tokens ? r16 : P.tokens - 1) * P.ldx * SIZE;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  u32x4 b[U][2], y[U][2];
  unsigned pb[U], power[U];
  Raw8<XT> a[2][4];
  auto load_tokens = [&](int set, int s) RSVD_INLINE {
    const int64_t k = 128 * (int64_t)s + 32 * kq, left = s < P.steps ? P.n - k : 0;      // (behind the last step: none, zeros)
#pragma unroll
    for (int q = 0; q < 4; ++q) a[set][q] = raw_load8<XT>(x + (k + 8 * q) * SIZE, left - 8 * q);
  };
  for (int s0 = wave; s0 < P.steps; s0 += WAVES * U) {
    load_tokens(0, s0);
    load_tokens(1, s0 + WAVES);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int s = s0 + WAVES * u < P.steps ? s0 + WAVES * u : s0;      // (behind the last step: the first one again, unused)
      pb[u] = powers[s];
#pragma unroll
      for (int h = 0; h < 2; ++h) b[u][h] = *reinterpret_cast<const u32x4 *>(w + (int64_t)128 * s + 16 * h);
    }
    // tokens, out of a cache, are rounded while weights come
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float v[4][8];
      unsigned top = 0u;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        x_values<XT>(a[u & 1][q], v[q]);
        top = f8_top8(v[q], top);
      }
      if (u + 2 < U) load_tokens(u & 1, s0 + WAVES * (u + 2));
      top = f8_shared(f8_shared(top, 16), 32);
      power[u] = f8_power(top);
      const float by = f8_factor(power[u]);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const u32x2 c = f8_codes8(v[2 * h], by), d = f8_codes8(v[2 * h + 1], by);
        y[u][h] = u32x4{c[0], c[1], d[0], d[1]};
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (s0 + WAVES * u >= P.steps) break;
      if constexpr (XT == RSVD_X_F32) {
        const float ub = f8_unit(pb[u]), ua = f8_unit(power[u]);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          u32x4 bw[2], aw[2];
          f8_widen(b[u][h], ub, bw);
          f8_widen(y[u][h], ua, aw);
#pragma unroll
          for (int z = 0; z < 2; ++z) acc = mfma_bf16(bw[z], aw[z], acc);
        }
      } else {
        acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(f8_both(b[u]), f8_both(y[u]), acc, 0, 0, 0, (int)pb[u], 0, (int)power[u]);
      }
    }
  }
  part[wave][lane] = acc;
  __syncthreads();
  if (wave > 0) return;
  acc = part[0][lane];
#pragma unroll
  for (int v = 1; v < WAVES; ++v) acc += part[v][lane];
  const int64_t n = n0 + 4 * kq;
  if (r16 < P.tokens && n < P.m) put4<XT>(P.Y, r16 * P.ldy + n, left_of(n, P.m), acc);
}

// Up to 32 tokens that were rounded before (rounding 32 tokens again would take every workgroup as long as its weights).
struct F8CodesParams {
  const uint8_t *x, *x_powers; int64_t ldx, ldxp, tokens, m;
  const uint8_t *codes, *powers; int64_t ldq, ldp;
  int steps;                       // of 128 k
  void *Y; int64_t ldy;
};
template <int XT, int WAVES> __global__ __launch_bounds__(64 * WAVES, 4) void f8_codes_kernel(const F8CodesParams P) {
  constexpr int U = 2, TB = 2;
  __shared__ f32x4 part[WAVES][TB][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, kq = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * 16;
  const int64_t row = n0 + r16 < P.m ? n0 + r16 : P.m - 1;
  const uint8_t *const w = P.codes + row * P.ldq + 32 * kq, *const powers = P.powers + (n0 >> 7) * P.ldp;
  const uint8_t *x[TB], *x_powers[TB];
#pragma unroll
  for (int i = 0; i < TB; ++i) {
    const int64_t t = 16 * i + r16 < P.tokens ? 16 * i + r16 : P.tokens - 1;
    x[i] = P.x + t * P.ldx + 32 * kq;
    x_powers[i] = P.x_powers + t * P.ldxp;
  }
  f32x4 acc[TB];
#pragma unroll
  for (int i = 0; i < TB; ++i) acc[i] = (f32x4)0.f;
  for (int s0 = wave; s0 < P.steps; s0 += WAVES * U) {
    u32x4 b[U][2], y[U][TB][2];
    unsigned pb[U], pa[U][TB];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int s = s0 + WAVES * u < P.steps ? s0 + WAVES * u : s0;      // (behind the last step: the first one again, unused)
      pb[u] = powers[s];
#pragma unroll
      for (int h = 0; h < 2; ++h) b[u][h] = *reinterpret_cast<const u32x4 *>(w + (int64_t)128 * s + 16 * h);
#pragma unroll
      for (int i = 0; i < TB; ++i) {
        pa[u][i] = x_powers[i][s];
#pragma unroll
        for (int h = 0; h < 2; ++h) y[u][i][h] = *reinterpret_cast<const u32x4 *>(x[i] + (int64_t)128 * s + 16 * h);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (s0 + WAVES * u >= P.steps) break;
      if constexpr (XT == RSVD_X_F32) {
        const float ub = f8_unit(pb[u]);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          u32x4 bw[2], aw[2];
          f8_widen(b[u][h], ub, bw);
#pragma unroll
          for (int i = 0; i < TB; ++i) {
            f8_widen(y[u][i][h], f8_unit(pa[u][i]), aw);
#pragma unroll
            for (int z = 0; z < 2; ++z) acc[i] = mfma_bf16(bw[z], aw[z], acc[i]);
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < TB; ++i)
          acc[i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(f8_both(b[u]), f8_both(y[u][i]), acc[i], 0, 0, 0, (int)pb[u], 0, (int)pa[u][i]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < TB; ++i) part[wave][i][lane] = acc[i];
  __syncthreads();
  if (wave >= TB) return;
  f32x4 sum = part[0][wave][lane];
#pragma unroll
  for (int v = 1; v < WAVES; ++v) sum += part[v][wave][lane];
  const int64_t t = 16 * wave + r16, n = n0 + 4 * kq;
  if (t < P.tokens && n < P.m) put4<XT>(P.Y, t * P.ldy + n, left_of(n, P.m), sum);
}

template <int XT> static void f8_codes_run(hipStream_t s, const F8CodesParams &P, dim3 grid) {
  if (P.steps > 16) hipLaunchKernelGGL((f8_codes_kernel<XT, 16>), grid, dim3(1024), 0, s, P);
  else if (P.steps > 8) hipLaunchKernelGGL((f8_codes_kernel<XT, 8>), grid, dim3(512), 0, s, P);
  else hipLaunchKernelGGL((f8_codes_kernel<XT, 4>), grid, dim3(256), 0, s, P);
}

hipError_t f8_codes_launch(rsvd_ctx *, hipStream_t s, const F8FewDesc &d, const uint8_t *x, int64_t ldx, const uint8_t *x_powers, int64_t ldxp) {
  if (d.tokens < 1 || d.tokens > 32) return hipErrorInvalidValue;
  const F8CodesParams P = {x, x_powers, ldx, ldxp, d.tokens, d.m, d.codes, d.powers, d.ldq, d.ldp, (int)ceil_div(d.n, 128), d.Y, d.ldy};
  const dim3 grid((unsigned)ceil_div(d.m, 16));
  if (d.type == RSVD_X_BF16) f8_codes_run<RSVD_X_BF16>(s, P, grid);
  else if (d.type == RSVD_X_F16) f8_codes_run<RSVD_X_F16>(s, P, grid);
  else f8_codes_run<RSVD_X_F32>(s, P, grid);
  return hipGetLastError();
}

template <int XT> static void f8_few_run(hipStream_t s, const F8FewParams &P, dim3 grid) {
  // (16 wavefronts: 4096 -> 8192 one token of bf16 10.1 us, 8: 11.3; 16384 -> 4096 18.4 and 21.0)
  if (P.steps > 16) hipLaunchKernelGGL((f8_few_kernel<XT, 16>), grid, dim3(1024), 0, s, P);
  else if (P.steps > 8) hipLaunchKernelGGL((f8_few_kernel<XT, 8>), grid, dim3(512), 0, s, P);
  else hipLaunchKernelGGL((f8_few_kernel<XT, 4>), grid, dim3(256), 0, s, P);
}

hipError_t f8_few_launch(rsvd_ctx *, hipStream_t s, const F8FewDesc &d) {
  if (d.tokens < 1 || d.tokens > 16) return hipErrorInvalidValue;
  const F8FewParams P = {(const char *)d.X, d.ldx, d.tokens, d.n, d.m, d.codes, d.powers, d.ldq, d.ldp, (int)ceil_div(d.n, 128), d.Y, d.ldy};
  const dim3 grid((unsigned)ceil_div(d.m, 16));
  if (d.type == RSVD_X_BF16) f8_few_run<RSVD_X_BF16>(s, P, grid);
  else if (d.type == RSVD_X_F16) f8_few_run<RSVD_X_F16>(s, P, grid);
  else f8_few_run<RSVD_X_F32>(s, P, grid);
  return hipGetLastError();
}

}  // namespace rsvd
