// Shared declarations of the operators of a gated block: products of 16-bit numbers and of 8-bit floats.
#pragma once

#include "layer8.hpp"

namespace rsvd {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// What the operands of a product are: 16-bit numbers, or codes of 8-bit floats (e4m3) with a power of two for 128 of them along k.
// DK_F8 multiplies codes as they are; DK_F8_EXACT makes bf16 numbers of codes and powers first, see dense_nt.hpp.
enum DenseKind { DK_BF16 = 0, DK_F16 = 1, DK_F8 = 2, DK_F8_EXACT = 3 };

// Products of planes: numbers that are sums of several 16-bit numbers, whose products are taken as further k, the smallest first.  Nibble s of
// `a` and `b`: planes of the two operands in part s of k.
struct DenseSegs { int count; uint32_t a, b; };
// (Small tiles take all planes of a k-tile at once and multiply them there, in this order.)
inline DenseSegs dense_segs(int planes) {
  if (planes == 3) return {6, 0x001012u, 0x010210u};       // (2,0) (1,1) (0,2) (1,0) (0,1) (0,0): 2^-24 of the largest is left out
  if (planes == 2) return {3, 0x001u, 0x010u};             // (1,0) (0,1) (0,0): 2^-22
  return {1, 0u, 0u};
}

// value = alpha sum + (beta + gamma (rows_m + columns_n)) D, stored in `type`, or as two fp16 numbers c_plane bytes apart (planes = 2).  D: fp16 numbers, d_planes of them.
// diagonal: the values of row m = column m go there in fp32, with rows_m (beta + gamma rows_m) added (rows are then the diagonal of D, which has zeros), and zeros to C.
struct LinearOut {
  float alpha = 1.f, beta = 0.f;
  const uint16_t *D = nullptr; int64_t ldd = 0, d_plane = 0, d_batch = 0;      // (elements, bytes, elements)
  int d_planes = 1;
  float gamma = 0.f;
  const float *rows = nullptr, *columns = nullptr; float *diagonal = nullptr; int64_t v_batch = 0;      // (NULL: zeros, not wanted; elements from problem to problem, of all three)
  void *C = nullptr; int64_t ldc = 0, c_plane = 0, c_batch = 0;               // (elements, bytes, elements)
  int type = RSVD_X_F32, planes = 1, accumulate = 0;
  int64_t width = 0;                       // columns stored, zeros from N on (0: N)
  const float *scale = nullptr;            // a power of two that sums are multiplied by first (dense_kn_launch of fp16 numbers; NULL: 1)
};

enum GatedAct { GATED_SILU = 0, GATED_GELU = 1, GATED_GELU_TANH = 2, GATED_RELU = 3, GATED_ACTS = 4 };

// gate, up -> act(gate) up, and both of them as they are (kept: N columns of gate, N of up); or, with dH, their gradients to `planes` planes of D.
struct GatedOut {
  int act = GATED_SILU, type = RSVD_X_BF16;
  void *H = nullptr; int64_t ldh = 0;
  void *kept = nullptr; int64_t ldk = 0;
  const void *dH = nullptr; int64_t lddh = 0;
  uint16_t *D = nullptr; int64_t ldD = 0, plane = 0;      // (elements, bytes)
  const float *scale = nullptr;            // fp16: D is held times this power of two, see range_launch
};

// ---------------------------------------------------------------- products
// C (M x N) = sum over k < K of A_mk B_kn, for each of `batch` problems.
// Strides in bytes.  gated: B has 2 N rows, gate and up, and N counts the outputs.
struct DenseDesc {
  int kind = DK_BF16, batch = 1;
  int64_t M = 0, N = 0, K = 0;
  bool rows_of_n = false;                  // B has rows of n: for dense_kn_launch
  bool gated = false, symmetric = false;   // symmetric (M = N): the tiles on and below the diagonal are computed, and stored twice
  const void *A = nullptr; int64_t lda = 0, a_plane = 0, a_batch = 0;
  const void *B = nullptr; int64_t ldb = 0, b_plane = 0, b_batch = 0;
  int planes = 1;                          // of both
  bool b_wide = false;                     // B is fp32 numbers, rows of n at any address of a number (dense_kn_launch, where dense_takes_wide)
  // 8-bit floats: powers, row (index >> shift), a byte for 128 k; rows are a multiple of 4 bytes from a 4-byte aligned address
  const uint8_t *a_pow = nullptr, *b_pow = nullptr; int64_t ld_apow = 0, ld_bpow = 0; int a_shift = 0, b_shift = 0;
  LinearOut out;
  GatedOut gate;
  float *partial = nullptr; size_t partial_bytes = 0;
};
// Workgroups of a launch: fewer than this (a grid has fewer than 2^32 threads).  Tiles of 256 have to be fewer; others are taken where they are.
constexpr int64_t kDenseGroups = (int64_t)1 << 22;
size_t dense_partial_bytes(const rsvd_ctx *ctx, const DenseDesc &d);

// Both operands with consecutive k (M rows, N or 2 N rows), rows of whole 16-byte pieces from 16-byte aligned addresses.  (8-bit floats: rows of whole k-tiles of 128,
// zeros behind the last k.)
hipError_t dense_nt_launch(rsvd_ctx *ctx, hipStream_t s, const DenseDesc &d);
// B with rows of n (K x N); A with rows of k, or with rows of m (a_krows: K x M).  Rows as above; zeros from k = K to the next multiple of 8 in A.
hipError_t dense_kn_launch(rsvd_ctx *ctx, hipStream_t s, const DenseDesc &d, bool a_krows);
// Whether small tiles will be chosen, which make three bf16 numbers of fp32 ones on the way.
bool dense_takes_wide(const rsvd_ctx *ctx, const DenseDesc &d);
hipError_t dense_init_device(rsvd_ctx *ctx);

// ---------------------------------------------------------------- gated.hip
hipError_t zero_launch(hipStream_t s, rsvd_xtype type, int64_t rows, int64_t n, void *C, int64_t ldc);
// Whether a few tokens go by the weight as it lies.  In tiles a weight is read once, too; every workgroup of sixteen outputs reads all tokens, and few outputs leave CUs without one.
// bf16 4096 -> 4096 32 tokens 18.6 us (33 in tiles: 19.3), 4096 -> 8192 17 tokens 34.2, 32: 40.0 (35.2), 8192 -> 2048 8 tokens 22.4, 32: 33.0 (19.0), 8192 -> 8192 16
// tokens 60.7 (70.6), 24: 69.9 (69.9).  fp32 weights would be laid
// out before: 4096 -> 8192 64 tokens 166 (65 in tiles: 256), 1024 -> 1024 17 tokens 21, 64: 36 (22).
inline bool gated_few(rsvd_xtype type, int64_t tokens, int64_t n, int64_t m, bool w_lies) {
  if (type == RSVD_X_F32) return tokens <= (m >= 2048 ? 64 : 16);
  if (!w_lies && m >= 4096) return tokens <= 32;       // (it would be laid out before)
  return m >= 8192 ? tokens <= 20 && tokens * n <= 3 << 16 : tokens <= 32 && tokens * n <= 3 << 15;
}
struct GatedFewDesc {
  rsvd_xtype type; int64_t tokens, n, m;
  const void *X; int64_t ldx;
  const void *W; int64_t ldw;
  GatedOut out;
};
hipError_t gated_few_launch(rsvd_ctx *ctx, hipStream_t s, const GatedFewDesc &d);
// What has to be laid out before the products, in one launch: matrices of `n` columns as 16-bit numbers in rows of `width` (a multiple of 8) with zeros behind n, fp32 as three
// bf16 planes `plane` bytes apart (rows = 0: none); and D from kept products (slope.kept; tokens = 0: none).
struct LayOut { const void *X; int64_t ldx, rows; uint16_t *out; int64_t plane; };
hipError_t lay_out_launch(hipStream_t s, rsvd_xtype type, int64_t n, int64_t width, const LayOut &x, const LayOut &w, int64_t tokens, int64_t m, const GatedOut &slope);

// What D of fp16 tokens is held times: scale[0], a power of two, and scale[1], which takes it out of sums again.  From dH, and the products that were kept or (kept NULL) X and W.
// parts: kRangeParts * 3 floats.
constexpr int kRangeParts = 1024;
hipError_t range_launch(hipStream_t s, int64_t tokens, int64_t n, int64_t m, const void *dH, int64_t lddh, const void *kept, int64_t ldk, const void *X, int64_t ldx, const void *W,
                        int64_t ldw, float *parts, float *scale);

// ---------------------------------------------------------------- f8.hip
// Whether each workgroup rounds the tokens itself, and whether a weight is read straight from memory for tokens that were rounded before; tiles are faster for more tokens and for
// large weights, whose tokens come out of a cache again for every sixteen rows.  4096 -> 4096 in bf16 16 tokens 8.6 us, 17 rounded before 11.0, in tiles 13.7, 32: 12.7 and 14.1;
// 4096 -> 16384 8 tokens 21.9, 16: 29.0, in tiles 19.3; fp32 4096 -> 8192 8 tokens 17.6, 12: 20.5, in tiles 21.2.
// (Fewer than 4096 outputs leave CUs without a workgroup: each takes as long.)
inline int64_t f8_rounded(int64_t tokens, int64_t n, int64_t m) { return tokens * n * (m > 4096 ? m : 4096); }
inline bool f8_few(rsvd_xtype type, int64_t tokens, int64_t n, int64_t m) {
  return tokens <= 16 && f8_rounded(tokens, n, m) <= (type == RSVD_X_F32 ? (int64_t)3 << 26 : (int64_t)1 << 29);
}
inline bool f8_few_codes(int64_t tokens, int64_t n, int64_t m) { return tokens <= 32 && f8_rounded(tokens, n, m) <= (int64_t)1 << 29; }
// X (rows x n) to codes in blocks of 128 of a row (codes: rows x width, powers rows x ldp), zeros behind the last number; Y (rows x m) and X (rows x n) to codes in blocks of 128
// rows (m x width and n x width, powers of rows of ldp; width = rows up to a multiple of 128).
hipError_t f8_rows_launch(hipStream_t s, rsvd_xtype type, int64_t rows, int64_t n, const void *X, int64_t ldx, uint8_t *codes, int64_t width, uint8_t *powers, int64_t ldp);
hipError_t f8_columns_launch(hipStream_t s, rsvd_xtype type, int64_t rows, int64_t m, const void *Y, int64_t ldy, uint8_t *y_codes, uint8_t *y_powers, int64_t n, const void *X,
                             int64_t ldx, uint8_t *x_codes, uint8_t *x_powers, int64_t width, int64_t ldp);
// W (m x n) to codes in blocks of 128 x 128, and the same in the other order (NULL: not wanted).
hipError_t f8_weight_launch(hipStream_t s, rsvd_xtype type, int64_t m, int64_t n, const void *W, int64_t ldw, uint8_t *codes, int64_t ldq, uint8_t *powers, int64_t ldp,
                            uint8_t *codes_t, int64_t ldqt, uint8_t *powers_t, int64_t ldpt);
// The product of a few tokens, X rounded on the way.
struct F8FewDesc {
  rsvd_xtype type; int64_t tokens, n, m;
  const void *X; int64_t ldx;
  const uint8_t *codes; int64_t ldq;
  const uint8_t *powers; int64_t ldp;
  void *Y; int64_t ldy;
};
hipError_t f8_few_launch(rsvd_ctx *ctx, hipStream_t s, const F8FewDesc &d);
// The same of up to 32 tokens, rounded before.
hipError_t f8_codes_launch(rsvd_ctx *ctx, hipStream_t s, const F8FewDesc &d, const uint8_t *x, int64_t ldx, const uint8_t *x_powers, int64_t ldxp);

// ---------------------------------------------------------------- orthogonal.hip
// |G| of every matrix by parts (kNormParts doubles each), and G / |G| times 2^13 as two fp16 planes with zeros up to `width`.
constexpr int kNormParts = 256;
hipError_t norm_launch(hipStream_t s, rsvd_xtype type, int batch, int64_t m, int64_t n, const void *G, int64_t ldg, int64_t stride, double *parts);
hipError_t unit_launch(hipStream_t s, rsvd_xtype type, int batch, int64_t m, int64_t n, const void *G, int64_t ldg, int64_t stride, const double *parts,
                       uint16_t *X, int64_t width, int64_t plane);

}  // namespace rsvd
