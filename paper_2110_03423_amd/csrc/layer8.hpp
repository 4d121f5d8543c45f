// Shared declarations of the layer operators: products with 8-bit weights and low-rank factors, activations kept in 8 bits.
#pragma once

#include "common.hpp"

namespace rsvd {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
// (memory takes any alignment of the elements; one instruction all the same)
typedef unsigned u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef unsigned u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

#define RSVD_INLINE __attribute__((always_inline))

inline int64_t xtype_size(rsvd_xtype t) { return t == RSVD_X_F32 ? 4 : 2; }
// bf16 numbers whose sum is exactly a number of the type.
inline int xtype_parts(rsvd_xtype t) { return t == RSVD_X_BF16 ? 1 : t == RSVD_X_F16 ? 2 : 3; }
// bf16 numbers that hold such a number times an fp32 scale: to 2^-17 of it (two; results of 16 bits), or as fp32 has it (three).  One, with the scale
// rounded into the weight, would be half the product, and was not kept: an error of 1.24 to 1.4 times the rounding of a bf16 result.
inline int scaled_parts(rsvd_xtype t) { return t == RSVD_X_F32 ? 3 : 2; }
// Rows that may be read and written in 16-byte pieces.
inline bool rows_aligned(const void *p, int64_t ld, int64_t size) { return ((uintptr_t)p & 15) == 0 && ld * size % 16 == 0; }

#ifdef __HIPCC__
template <int XT> struct XTraits;
template <> struct XTraits<RSVD_X_BF16> { static constexpr int SIZE = 2, PARTS = 1; };
template <> struct XTraits<RSVD_X_F16> { static constexpr int SIZE = 2, PARTS = 2; };
template <> struct XTraits<RSVD_X_F32> { static constexpr int SIZE = 4, PARTS = 3; };

// Element i behind p, as fp32.
template <int XT> __device__ __forceinline__ float x_value(const char *p, int64_t i) {
  if constexpr (XT == RSVD_X_F32) return reinterpret_cast<const float *>(p)[i];
  else if constexpr (XT == RSVD_X_F16) return (float)reinterpret_cast<const _Float16 *>(p)[i];
  else return __uint_as_float((unsigned)reinterpret_cast<const uint16_t *>(p)[i] << 16);
}

// Eight consecutive elements from p on, `left` of which exist (the others are zero).
template <int XT> __device__ __forceinline__ void x_load8(const char *p, int64_t left, float (&v)[8]) {
  if (left >= 8) {
    if constexpr (XT == RSVD_X_F32) {
      const f32x4 a = reinterpret_cast<const f32x4_any *>(p)[0], b = reinterpret_cast<const f32x4_any *>(p)[1];
#pragma unroll
      for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[4 + e] = b[e]; }
    } else {
      const u32x4 a = *reinterpret_cast<const u32x4_any *>(p);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (XT == RSVD_X_BF16) {
          v[2 * e] = __uint_as_float(a[e] << 16);
          v[2 * e + 1] = __uint_as_float(a[e] & 0xffff0000u);
        } else {
          const unsigned pair = a[e];      // (a copy: the cast of a vector's element takes its first one)
          const f16x2 h = __builtin_bit_cast(f16x2, pair);
          v[2 * e] = (float)h[0];
          v[2 * e + 1] = (float)h[1];
        }
      }
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < left ? x_value<XT>(p, e) : 0.f;
  }
}

// Eight consecutive bf16 numbers from p on, as they are.
__device__ __forceinline__ u32x4 halves8(const uint16_t *p, int64_t left) {
  u32x4 v = {0u, 0u, 0u, 0u};
  if (left >= 8) {
    v = *reinterpret_cast<const u32x4_any *>(p);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < left) v[e >> 1] |= (unsigned)p[e] << (16 * (e & 1));
  }
  return v;
}

// The same of any type.
template <int XT> struct Raw8 { u32x4 w[XTraits<XT>::SIZE / 2]; };
template <int XT> __device__ __forceinline__ Raw8<XT> raw_load8(const char *p, int64_t left) {
  Raw8<XT> v;
  if constexpr (XT == RSVD_X_F32) {
    if (left >= 8) {
      v.w[0] = reinterpret_cast<const u32x4_any *>(p)[0];
      v.w[1] = reinterpret_cast<const u32x4_any *>(p)[1];
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v.w[e >> 2][e & 3] = e < left ? reinterpret_cast<const unsigned *>(p)[e] : 0u;
    }
  } else {
    v.w[0] = halves8(reinterpret_cast<const uint16_t *>(p), left);
  }
  return v;
}

__device__ __forceinline__ unsigned bf16_pair(float a, float b) {      // rounded to nearest even
  return __builtin_bit_cast(unsigned, __builtin_convertvector(f32x2{a, b}, bf16x2));
}
__device__ __forceinline__ float bf16_low(unsigned pair) { return __uint_as_float(pair << 16); }
__device__ __forceinline__ float bf16_high(unsigned pair) { return __uint_as_float(pair & 0xffff0000u); }

// The parts of two numbers as bf16 numbers, the largest first, each the rounded rest of the ones before: three hold every fp32
// number, two every fp16 number and any other to 2^-17 of itself.  Numbers that round to infinity are cut off instead; an infinity
// or NaN has zeros behind its first part.
// CHECK = false: an infinity has NaN behind its first part, and no finite number may round to one.
template <int PARTS, bool CHECK = true> __device__ __forceinline__ void bf16_parts2(float a, float b, unsigned (&p)[PARTS]) {
#pragma unroll
  for (int s = 0; s < PARTS; ++s) {
    p[s] = bf16_pair(a, b);
    if (s + 1 < PARTS) {
      float ra = a - bf16_low(p[s]), rb = b - bf16_high(p[s]);
      if (CHECK && s == 0 && ((p[0] & 0x7f80u) == 0x7f80u || (p[0] & 0x7f800000u) == 0x7f800000u)) {
        const unsigned ua = __float_as_uint(a), ub = __float_as_uint(b);
        if ((p[0] & 0x7f80u) == 0x7f80u) {
          const bool finite = (ua & 0x7f800000u) != 0x7f800000u;
          if (finite) p[0] = (p[0] & 0xffff0000u) | (ua >> 16);
          ra = finite ? a - __uint_as_float(ua & 0xffff0000u) : 0.f;
        }
        if ((p[0] & 0x7f800000u) == 0x7f800000u) {
          const bool finite = (ub & 0x7f800000u) != 0x7f800000u;
          if (finite) p[0] = (p[0] & 0x0000ffffu) | (ub & 0xffff0000u);
          rb = finite ? b - __uint_as_float(ub & 0xffff0000u) : 0.f;
        }
      }
      a = ra;
      b = rb;
    }
  }
}

// Operands of the bf16 matrix instruction out of eight numbers, the largest part first.
template <int XT, bool CHECK = true> __device__ __forceinline__ void split_operand(const Raw8<XT> &v, u32x4 (&x)[XTraits<XT>::PARTS]) {
  constexpr int PARTS = XTraits<XT>::PARTS;
  if constexpr (XT == RSVD_X_BF16) {
    x[0] = v.w[0];
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      unsigned p[PARTS];
      if constexpr (XT == RSVD_X_F32) {
        bf16_parts2<PARTS>(__uint_as_float(v.w[e >> 1][2 * (e & 1)]), __uint_as_float(v.w[e >> 1][2 * (e & 1) + 1]), p);
      } else {
        const unsigned pair = v.w[0][e];
        const f16x2 h = __builtin_bit_cast(f16x2, pair);
        bf16_parts2<PARTS, CHECK>((float)h[0], (float)h[1], p);
      }
#pragma unroll
      for (int q = 0; q < PARTS; ++q) x[q][e] = p[q];
    }
  }
}
#endif

// Leading dimensions that rows in tiles may have: 32-bit offsets inside a tile.
constexpr int64_t kMaxLd = (int64_t)1 << 23;
// (sums over tokens, indexes of workgroups, threads of a launch of one workgroup a token)
constexpr int64_t kMaxTokens = (int64_t)1 << 22;

// ---------------------------------------------------------------- layer8_rows.hip
// Rows of X (rows x n) to codes with a scale each; a row of codes is written up to `width` (>= n, a multiple of 8) with zeros behind n.
// sums != NULL: t is joined on the way (lowrank_join_launch).
hipError_t rows8_launch(hipStream_t s, rsvd_xtype type, int64_t rows, int64_t n, const void *X, int64_t ldx, int8_t *codes,
                        int64_t ldq, int64_t width, float *scale, const float *sums = nullptr, int splits = 0, int64_t r = 0, int parts = 0,
                        uint16_t *t = nullptr);
hipError_t keep8_save_launch(hipStream_t s, rsvd_xtype type, int64_t tokens, int64_t n, const void *X, int64_t ldx, int8_t *codes,
                             int64_t ldc, uint8_t *powers, int64_t ldp);
hipError_t keep8_load_launch(hipStream_t s, rsvd_xtype type, int64_t tokens, int64_t n, const int8_t *codes, int64_t ldc,
                             const uint8_t *powers, int64_t ldp, void *X, int64_t ldx);
hipError_t fill_zero_launch(hipStream_t s, int64_t rows, int64_t cols, float *out, int64_t ld);

// ---------------------------------------------------------------- layer8_lowrank.hip
constexpr int64_t kMaxRank = 1024, kFewTokens = 64;
inline int64_t rank_places(int64_t r) { return align_up((size_t)r, 32); }
// bf16 numbers that hold a number of t between the two products: 2^-17 of it is left out with two, nothing with three.
inline int lowrank_parts(rsvd_xtype type) { return type == RSVD_X_F32 ? 3 : 2; }
// sums [splits][tokens][rank_places(r)]: the products of X (tokens x n) with the rows of F (r x n, bf16) over ranges of k; zeros from r on.
int lowrank_splits(const rsvd_ctx *ctx, int64_t tokens, int64_t n, int64_t r);
hipError_t lowrank_launch(rsvd_ctx *ctx, hipStream_t s, rsvd_xtype type, int64_t tokens, int64_t n, int64_t r, const void *X, int64_t ldx,
                          const void *F, int64_t ldf, float *sums);
// The same for up to kFewTokens tokens, together with rows8_launch.
hipError_t front_launch(rsvd_ctx *ctx, hipStream_t s, rsvd_xtype type, int64_t tokens, int64_t n, int64_t r, const void *X, int64_t ldx,
                        const void *F, int64_t ldf, float *sums, int8_t *codes, int64_t ldq, int64_t width, float *scale);
// The operands of kn_launch for a gradient, and lowrank_launch for dY (r = 0: without): planes[q][token][0 .. planes_width) the bf16 parts of dY
// (tokens x m), or of dY_tj dy_factor_j (scaled_parts() of them), zeros from m on (planes NULL: not wanted); plane[row][0 .. width) the codes (rows x n) as
// bf16 numbers, multiplied by the powers of two of kept activations (NULL: as they are; plane NULL: not wanted).  Widths are m and n up to a multiple of 8.
hipError_t grad_front_launch(rsvd_ctx *ctx, hipStream_t s, rsvd_xtype type, int64_t tokens, int64_t m, int64_t r, const void *dY, int64_t lddy,
                             const void *F, int64_t ldf, float *sums, const float *dy_factor, uint16_t *planes, int64_t planes_width,
                             int64_t rows, int64_t n, const int8_t *codes, int64_t ldc, const uint8_t *powers, int64_t ldp, uint16_t *plane,
                             int64_t width);
// Whether the operands of that many elements (planes of dY, codes; 0: not wanted) are few enough for a launch, which has fewer than 2^32 threads, eight elements
// of dY or sixteen codes each.  (2^28 of them are more than the low-rank sums take.)
inline bool grad_front_fits(int64_t tokens, int64_t planes_width, int64_t rows, int64_t n) {
  return tokens * (planes_width / 8) + rows * ceil_div(n, 16) < ((int64_t)1 << 32) - ((int64_t)1 << 28);
}
// t [tokens][parts][rank_places(r)]: the sums added up, as bf16 numbers, the largest first.
hipError_t lowrank_join_launch(hipStream_t s, const float *sums, int splits, int64_t tokens, int64_t r, int parts, uint16_t *t);

// What becomes of a sum over k: value_ti = rs_t cs_i sum + sum_p t_tp G_ip + bias_i
struct Layer8Out {
  const float *rs = nullptr, *cs = nullptr, *bias = nullptr;      // NULL: ones, ones, zeros
  const uint16_t *t = nullptr; int parts = 2;                     // as lowrank_join_launch leaves it
  const uint16_t *G = nullptr; int64_t ldg = 0; int r = 0;        // bf16, N x r
  void *C = nullptr; int64_t ldc = 0; int type = RSVD_X_F32;      // M x N
  int accumulate = 0;                                             // (fp32)
};

// ---------------------------------------------------------------- layer8_gemm.hip
// C (M x N) out of the integer sums over k of codes A (M rows) and B (N rows), both with consecutive k, in k-tiles of 128.  Both start at 16-byte
// addresses and have row lengths of a multiple of 16 bytes.
struct NtDesc {
  int64_t M = 0, N = 0;
  int64_t ktiles = 0;                    // every row of A has that many whole k-tiles, zeros behind the last k
  const int8_t *A = nullptr; int64_t lda = 0;
  const int8_t *B = nullptr; int64_t ldb = 0;
  int64_t b_bytes = 0;                   // bytes of a row of B that may be read (a multiple of 16)
  Layer8Out out;
  float *partial = nullptr; size_t partial_bytes = 0;      // for sums over k in several ranges
};
size_t nt_partial_bytes(const rsvd_ctx *ctx, int64_t M, int64_t N, int64_t ktiles, bool lowrank);
hipError_t nt_launch(rsvd_ctx *ctx, hipStream_t s, const NtDesc &d);

// ---------------------------------------------------------------- layer8_grad.hip
// C (M x N) = sum over k < K of A_mk B_kn of bf16 numbers, A a sum of `planes` matrices (`plane` bytes apart, the largest first), B with rows of n.
// a_krows: A is stored K x M, else M x K.  Rows of both may be read in 16-byte pieces as far as these hold an element.
struct KnDesc {
  int64_t M = 0, N = 0, K = 0;
  bool a_krows = false;
  const uint16_t *A = nullptr; int64_t lda = 0;            // bytes
  int planes = 1; int64_t plane = 0;
  const uint16_t *B = nullptr; int64_t ldb = 0;            // bytes
  const int8_t *codes = nullptr; int64_t ldc = 0;          // in the place of B, where kn_takes_codes(): codes (K x N)
  const uint8_t *powers = nullptr; int64_t ldp = 0;        // a_krows: their powers of two (row k, blocks of 32 columns)
  float *sums = nullptr, *sums_out = nullptr;              // a_krows: place for kn_sum_rows() parts of the sums of A over k, M each, and for the sums; or NULL
  Layer8Out out;
  float *partial = nullptr; size_t partial_bytes = 0;
};
size_t kn_partial_bytes(const rsvd_ctx *ctx, int64_t M, int64_t N, int64_t K, int planes, bool lowrank);
int64_t kn_sum_rows(const rsvd_ctx *ctx, int64_t M, int64_t N, int64_t K, int planes);
bool kn_takes_codes(const rsvd_ctx *ctx, bool a_krows, int64_t M, int64_t N, int64_t K, int planes, bool lowrank, int64_t ldc, int64_t ldp);
hipError_t kn_launch(rsvd_ctx *ctx, hipStream_t s, const KnDesc &d);

// ---------------------------------------------------------------- layer8_few.hip
// The product of codes for up to kFewTokens tokens.
struct FewDesc {
  int64_t M = 0, N = 0, k = 0;           // k: a multiple of 64, zeros in A behind the last
  const int8_t *A = nullptr; int64_t lda = 0;
  const int8_t *B = nullptr; int64_t ldb = 0;
  int64_t b_bytes = 0;                   // bytes of a row of B that may be read (a multiple of 16)
  const float *sums = nullptr; int splits = 0;      // the low-rank sums as they are, in the place of out.t (NULL: out.t)
  Layer8Out out;
};
hipError_t few_launch(rsvd_ctx *ctx, hipStream_t s, const FewDesc &d);

}  // namespace rsvd
