// C entry points of the layer operators: argument checks, workspace layout, sequence of launches.  Host code only.
#include <stdio.h>

#include "layer8.hpp"

using namespace rsvd;

namespace {

int fail_hip(rsvd_ctx *ctx, hipError_t e, const char *where) {
  snprintf(ctx->hip_error, sizeof(ctx->hip_error), "%s: %s", where, hipGetErrorString(e));
  return RSVD_ERR_HIP;
}

#define RSVD_TRY(expr, where)                                   \
  do {                                                          \
    hipError_t e_ = (expr);                                     \
    if (e_ != hipSuccess) return fail_hip(ctx, e_, where);      \
  } while (0)

bool valid_xtype(rsvd_xtype t) { return t == RSVD_X_BF16 || t == RSVD_X_F16 || t == RSVD_X_F32; }
bool valid_codes(const void *p) { return p != nullptr && ((uintptr_t)p & 15) == 0; }
bool element_aligned(const void *p, int64_t size) { return ((uintptr_t)p & (uintptr_t)(size - 1)) == 0; }

// Sums over ranges of k times ranks up to which the product of a few tokens takes them as they are (eight pieces of 32 for each of its
// wavefronts); beyond, a launch that joins them first is less.
constexpr int64_t kFewUnjoined = 2048;

struct Take {
  size_t off = 0;
  size_t operator()(size_t bytes) { const size_t o = off; off = align_up(off + bytes, 256); return o; }
};

// codes of X, their scales, the sums with Vt before and after they are joined, parts of sums
struct ProductLayout { size_t codes, scale, sums, t, partial, partial_bytes, total; int64_t width; int splits; };

ProductLayout product_layout(const rsvd_ctx *ctx, rsvd_xtype type, int64_t tokens, int64_t n, int64_t m, int64_t r) {
  ProductLayout L;
  Take take;
  L.width = (int64_t)align_up((size_t)n, 128);
  L.codes = take((size_t)tokens * L.width);
  L.scale = take((size_t)tokens * 4);
  L.splits = r > 0 ? lowrank_splits(ctx, tokens, n, r) : 0;
  L.sums = take((size_t)L.splits * tokens * rank_places(r) * 4);
  L.t = take((size_t)tokens * rank_places(r) * 2 * lowrank_parts(type));
  L.partial_bytes = tokens > kFewTokens ? nt_partial_bytes(ctx, tokens, m, L.width / 128, r > 0) : 0;
  L.partial = take(L.partial_bytes);
  L.total = take.off;
  return L;
}

// Whether rows of bf16 numbers can be taken as they are by kn_launch (as a matrix M x K, or K x M): no byte is read that is not theirs.
bool takes_rows(rsvd_xtype type, const void *p, int64_t cols, int64_t ld) {
  return type == RSVD_X_BF16 && cols % 8 == 0 && rows_aligned(p, ld, 2) && ld <= kMaxLd / 4;
}

// planes of dY (of a weight gradient: where it cannot be taken as it is), codes as bf16 numbers, low-rank sums before and after they are joined, or column sums of dY, parts of sums
struct GradLayout { size_t a, b, sums, t, partial, partial_bytes, total; int64_t width, b_width; int planes, splits; };

GradLayout product_grad_layout(const rsvd_ctx *ctx, rsvd_xtype type, int64_t tokens, int64_t n, int64_t m, int64_t r) {
  GradLayout L;
  Take take;
  L.planes = scaled_parts(type);
  L.width = (int64_t)align_up((size_t)m, 8);
  L.b_width = (int64_t)align_up((size_t)n, 8);
  L.a = take((size_t)L.planes * tokens * L.width * 2);
  L.b = take((size_t)m * L.b_width * 2);
  L.splits = r > 0 ? lowrank_splits(ctx, tokens, m, r) : 0;
  L.sums = take((size_t)L.splits * tokens * rank_places(r) * 4);
  L.t = take((size_t)tokens * rank_places(r) * 2 * lowrank_parts(type));
  L.partial_bytes = kn_partial_bytes(ctx, tokens, n, m, L.planes, r > 0);
  L.partial = take(L.partial_bytes);
  L.total = take.off;
  return L;
}

GradLayout keep8_grad_layout(const rsvd_ctx *ctx, rsvd_xtype type, int64_t tokens, int64_t n, int64_t m) {
  GradLayout L;
  Take take;
  L.planes = xtype_parts(type);
  L.width = (int64_t)align_up((size_t)m, 8);
  L.b_width = (int64_t)align_up((size_t)n, 8);
  L.a = take((size_t)L.planes * tokens * L.width * 2);
  L.b = take((size_t)tokens * L.b_width * 2);
  L.sums = take((size_t)kn_sum_rows(ctx, m, n, tokens, L.planes) * m * 4);
  L.t = L.sums;
  L.splits = 0;
  L.partial_bytes = kn_partial_bytes(ctx, m, n, tokens, L.planes, false);
  L.partial = take(L.partial_bytes);
  L.total = take.off;
  return L;
}

}  // namespace

extern "C" {

int rsvd_q8_rows(rsvd_ctx *ctx, void *stream, rsvd_xtype type, int64_t rows, int64_t n, const void *X, int64_t ldx, int8_t *codes,
                 int64_t ldq, float *scale) {
  if (ctx == nullptr) return -1;
  if (!valid_xtype(type)) return -3;
  if (rows < 0) return -4;
  if (n < 1) return -5;
  if (rows == 0) return RSVD_OK;
  if (X == nullptr || !element_aligned(X, xtype_size(type))) return -6;
  if (ldx < n) return -7;
  if (!valid_codes(codes)) return -8;
  if (ldq < n || ldq % 16 != 0) return -9;
  if (scale == nullptr || !element_aligned(scale, 4)) return -10;
  if (n > kMaxLd || rows > 0x7fffffff) return RSVD_ERR_UNSUPPORTED;
  if (ctx->device < 0) return RSVD_ERR_NO_DEVICE;
  ProfScope ps(ctx, (hipStream_t)stream, PK_SMALL);
  RSVD_TRY(rows8_launch((hipStream_t)stream, type, rows, n, X, ldx, codes, ldq, (int64_t)align_up((size_t)n, 16), scale), "rows to 8 bits");
  return RSVD_OK;
}

// Checks that the sizes of a product have in common; 0 or the error.
static int check_sizes(rsvd_xtype type, int64_t tokens, int64_t n, int64_t m, int64_t r, int first) {
  if (!valid_xtype(type)) return -first;
  if (tokens < 0) return -(first + 1);
  if (n < 1) return -(first + 2);
  if (m < 1) return -(first + 3);
  if (r < 0) return -(first + 4);
  return 0;
}
static bool sizes_supported(int64_t tokens, int64_t n, int64_t m, int64_t r) {
  return tokens <= kMaxTokens && n <= RSVD_Q8_MAX_FEATURES && m <= RSVD_Q8_MAX_FEATURES && r <= kMaxRank;
}

int rsvd_q8_product_bytes(rsvd_ctx *ctx, rsvd_xtype type, int64_t tokens, int64_t n, int64_t m, int64_t r, size_t *bytes) {
  if (ctx == nullptr) return -1;
  if (const int rc = check_sizes(type, tokens, n, m, r, 2)) return rc;
  if (bytes == nullptr) return -7;
  if (!sizes_supported(tokens, n, m, r)) return RSVD_ERR_UNSUPPORTED;
  *bytes = tokens > 0 ? product_layout(ctx, type, tokens, n, m, r).total : 0;
  return RSVD_OK;
}

int rsvd_q8_product_grad_bytes(rsvd_ctx *ctx, rsvd_xtype type, int64_t tokens, int64_t n, int64_t m, int64_t r, size_t *bytes) {
  if (ctx == nullptr) return -1;
  if (const int rc = check_sizes(type, tokens, n, m, r, 2)) return rc;
  if (bytes == nullptr) return -7;
  if (!sizes_supported(tokens, n, m, r)) return RSVD_ERR_UNSUPPORTED;
  *bytes = tokens > 0 ? product_grad_layout(ctx, type, tokens, n, m, r).total : 0;
  return RSVD_OK;
}

int rsvd_keep8_grad_bytes(rsvd_ctx *ctx, rsvd_xtype type, int64_t tokens, int64_t n, int64_t m, size_t *bytes) {
  if (ctx == nullptr) return -1;
  if (const int rc = check_sizes(type, tokens, n, m, 0, 2)) return rc;
  if (bytes == nullptr) return -6;
  if (!sizes_supported(tokens, n, m, 0)) return RSVD_ERR_UNSUPPORTED;
  *bytes = tokens > 0 ? keep8_grad_layout(ctx, type, tokens, n, m).total : 0;
  return RSVD_OK;
}

int rsvd_q8_product(rsvd_ctx *ctx, void *stream, rsvd_xtype type, int64_t tokens, int64_t n, int64_t m, int64_t r, const void *X,
                    int64_t ldx, const int8_t *codes, int64_t ldq, const float *scale, const void *U, int64_t ldu, const void *Vt,
                    int64_t ldvt, const float *bias, void *Y, int64_t ldy, void *workspace, size_t workspace_bytes) {
  if (ctx == nullptr) return -1;
  if (const int rc = check_sizes(type, tokens, n, m, r, 3)) return rc;
  if (tokens == 0) return RSVD_OK;
  const int64_t es = xtype_size(type);
  if (X == nullptr || !element_aligned(X, es)) return -8;
  if (ldx < n) return -9;
  if (!valid_codes(codes)) return -10;
  if (ldq < n || ldq % 16 != 0) return -11;
  if (scale == nullptr || !element_aligned(scale, 4)) return -12;
  if (r > 0 && (U == nullptr || !element_aligned(U, 2))) return -13;
  if (r > 0 && ldu < r) return -14;
  if (r > 0 && (Vt == nullptr || !element_aligned(Vt, 2))) return -15;
  if (r > 0 && ldvt < n) return -16;
  if (!element_aligned(bias, 4)) return -17;
  if (Y == nullptr || !element_aligned(Y, es)) return -18;
  if (ldy < m) return -19;
  if (!sizes_supported(tokens, n, m, r) || ldq > kMaxLd) return RSVD_ERR_UNSUPPORTED;
  const ProductLayout L = product_layout(ctx, type, tokens, n, m, r);
  if (workspace == nullptr || ((uintptr_t)workspace & 255) != 0) return -20;
  if (workspace_bytes < L.total) return -21;
  if (ctx->device < 0) return RSVD_ERR_NO_DEVICE;
  hipStream_t s = (hipStream_t)stream;
  char *ws = (char *)workspace;
  int8_t *q = (int8_t *)(ws + L.codes);
  float *rs = (float *)(ws + L.scale);
  uint16_t *t = (uint16_t *)(ws + L.t);
  float *sums = r > 0 ? (float *)(ws + L.sums) : nullptr;
  const int parts = lowrank_parts(type);
  const bool few = tokens <= kFewTokens, unjoined = few && L.splits * rank_places(r) <= kFewUnjoined;
  {
    ProfScope ps(ctx, s, PK_SMALL);
    if (few) {
      RSVD_TRY(front_launch(ctx, s, type, tokens, n, r, X, ldx, Vt, ldvt, sums, q, L.width, L.width, rs), "rows to 8 bits, low-rank term");
      if (r > 0 && !unjoined) RSVD_TRY(lowrank_join_launch(s, sums, L.splits, tokens, r, parts, t), "low-rank term");
    } else {
      if (r > 0) RSVD_TRY(lowrank_launch(ctx, s, type, tokens, n, r, X, ldx, Vt, ldvt, sums), "low-rank term");
      RSVD_TRY(rows8_launch(s, type, tokens, n, X, ldx, q, L.width, L.width, rs, sums, L.splits, r, parts, t), "rows to 8 bits");
    }
  }
  Layer8Out o;
  o.rs = rs; o.cs = scale; o.bias = bias;
  o.t = t; o.parts = parts; o.G = (const uint16_t *)U; o.ldg = ldu; o.r = (int)r;
  o.C = Y; o.ldc = ldy; o.type = type;
  ProfScope ps(ctx, s, PK_GEMM_AX);
  if (few) {
    FewDesc d;
    d.sums = unjoined ? sums : nullptr; d.splits = L.splits;
    d.M = tokens; d.N = m; d.k = L.width;
    d.A = q; d.lda = L.width; d.B = codes; d.ldb = ldq; d.b_bytes = (int64_t)align_up((size_t)n, 16);
    d.out = o;
    RSVD_TRY(few_launch(ctx, s, d), "product of a few tokens");
    return RSVD_OK;
  }
  NtDesc d;
  d.M = tokens; d.N = m; d.ktiles = L.width / 128;
  d.A = q; d.lda = L.width; d.B = codes; d.ldb = ldq; d.b_bytes = (int64_t)align_up((size_t)n, 16);
  d.out = o;
  d.partial = (float *)(ws + L.partial); d.partial_bytes = L.partial_bytes;
  RSVD_TRY(nt_launch(ctx, s, d), "product of codes");
  return RSVD_OK;
}

int rsvd_q8_product_grad(rsvd_ctx *ctx, void *stream, rsvd_xtype type, int64_t tokens, int64_t n, int64_t m, int64_t r, const void *dY,
                         int64_t lddy, const int8_t *codes, int64_t ldq, const float *scale, const void *Ut, int64_t ldut, const void *V,
                         int64_t ldv, void *dX, int64_t lddx, void *workspace, size_t workspace_bytes) {
  if (ctx == nullptr) return -1;
  if (const int rc = check_sizes(type, tokens, n, m, r, 3)) return rc;
  if (tokens == 0) return RSVD_OK;
  const int64_t es = xtype_size(type);
  if (dY == nullptr || !element_aligned(dY, es)) return -8;
  if (lddy < m) return -9;
  if (!valid_codes(codes)) return -10;
  if (ldq < n || ldq % 16 != 0) return -11;
  if (scale == nullptr || !element_aligned(scale, 4)) return -12;
  if (r > 0 && (Ut == nullptr || !element_aligned(Ut, 2))) return -13;
  if (r > 0 && ldut < m) return -14;
  if (r > 0 && (V == nullptr || !element_aligned(V, 2))) return -15;
  if (r > 0 && ldv < r) return -16;
  if (dX == nullptr || !element_aligned(dX, es)) return -17;
  if (lddx < n) return -18;
  if (!sizes_supported(tokens, n, m, r) || ldq > kMaxLd) return RSVD_ERR_UNSUPPORTED;
  const GradLayout L = product_grad_layout(ctx, type, tokens, n, m, r);
  if (workspace == nullptr || ((uintptr_t)workspace & 255) != 0) return -19;
  if (workspace_bytes < L.total) return -20;
  // (the scale goes to dY before that is split, and the codes stay exact)
  const bool as_codes = kn_takes_codes(ctx, false, tokens, n, m, L.planes, r > 0, ldq, 0);
  if (!grad_front_fits(tokens, L.width, as_codes ? 0 : m, n)) return RSVD_ERR_UNSUPPORTED;
  if (ctx->device < 0) return RSVD_ERR_NO_DEVICE;
  hipStream_t s = (hipStream_t)stream;
  char *ws = (char *)workspace;
  uint16_t *a = (uint16_t *)(ws + L.a), *b = (uint16_t *)(ws + L.b), *t = (uint16_t *)(ws + L.t);
  {
    ProfScope ps(ctx, s, PK_SMALL);
    float *sums = (float *)(ws + L.sums);
    RSVD_TRY(grad_front_launch(ctx, s, type, tokens, m, r, dY, lddy, Ut, ldut, sums, scale, a, L.width, m, n, codes, ldq, nullptr, 0,
                               as_codes ? nullptr : b, L.b_width),
             "operands of the gradient");
    if (r > 0) RSVD_TRY(lowrank_join_launch(s, sums, L.splits, tokens, r, lowrank_parts(type), t), "low-rank term");
  }
  KnDesc d;
  d.M = tokens; d.N = n; d.K = m;
  d.A = a; d.lda = L.width * 2; d.planes = L.planes; d.plane = tokens * L.width * 2;
  d.B = b; d.ldb = L.b_width * 2;
  if (as_codes) d.codes = codes;
  d.ldc = ldq;
  d.out.t = t; d.out.parts = lowrank_parts(type); d.out.G = (const uint16_t *)V; d.out.ldg = ldv; d.out.r = (int)r;
  d.out.C = dX; d.out.ldc = lddx; d.out.type = type;
  d.partial = (float *)(ws + L.partial); d.partial_bytes = L.partial_bytes;
  ProfScope ps(ctx, s, PK_GEMM_ATX);
  RSVD_TRY(kn_launch(ctx, s, d), "gradient of a product of codes");
  return RSVD_OK;
}

int rsvd_keep8_save(rsvd_ctx *ctx, void *stream, rsvd_xtype type, int64_t tokens, int64_t n, const void *X, int64_t ldx, int8_t *codes,
                    int64_t ldc, uint8_t *powers, int64_t ldp) {
  if (ctx == nullptr) return -1;
  if (!valid_xtype(type)) return -3;
  if (tokens < 0) return -4;
  if (n < 1) return -5;
  if (tokens == 0) return RSVD_OK;
  if (X == nullptr || !element_aligned(X, xtype_size(type))) return -6;
  if (ldx < n) return -7;
  if (!valid_codes(codes)) return -8;
  if (ldc < n || ldc % 16 != 0) return -9;
  if (powers == nullptr) return -10;
  if (ldp < ceil_div(n, 32)) return -11;
  if (n > kMaxLd) return RSVD_ERR_UNSUPPORTED;
  if (ctx->device < 0) return RSVD_ERR_NO_DEVICE;
  ProfScope ps(ctx, (hipStream_t)stream, PK_SMALL);
  RSVD_TRY(keep8_save_launch((hipStream_t)stream, type, tokens, n, X, ldx, codes, ldc, powers, ldp), "keep in 8 bits");
  return RSVD_OK;
}

int rsvd_keep8_load(rsvd_ctx *ctx, void *stream, rsvd_xtype type, int64_t tokens, int64_t n, const int8_t *codes, int64_t ldc,
                    const uint8_t *powers, int64_t ldp, void *X, int64_t ldx) {
  if (ctx == nullptr) return -1;
  if (!valid_xtype(type)) return -3;
  if (tokens < 0) return -4;
  if (n < 1) return -5;
  if (tokens == 0) return RSVD_OK;
  if (!valid_codes(codes)) return -6;
  if (ldc < n || ldc % 16 != 0) return -7;
  if (powers == nullptr) return -8;
  if (ldp < ceil_div(n, 32)) return -9;
  if (X == nullptr || !element_aligned(X, xtype_size(type))) return -10;
  if (ldx < n) return -11;
  if (n > kMaxLd) return RSVD_ERR_UNSUPPORTED;
  if (ctx->device < 0) return RSVD_ERR_NO_DEVICE;
  ProfScope ps(ctx, (hipStream_t)stream, PK_SMALL);
  RSVD_TRY(keep8_load_launch((hipStream_t)stream, type, tokens, n, codes, ldc, powers, ldp, X, ldx), "kept numbers");
  return RSVD_OK;
}

int rsvd_keep8_grad(rsvd_ctx *ctx, void *stream, rsvd_xtype type, int64_t tokens, int64_t n, int64_t m, const void *dY, int64_t lddy,
                    const int8_t *codes, int64_t ldc, const uint8_t *powers, int64_t ldp, float *dW, int64_t lddw, float *db,
                    int accumulate, void *workspace, size_t workspace_bytes) {
  if (ctx == nullptr) return -1;
  if (const int rc = check_sizes(type, tokens, n, m, 0, 3)) return rc;
  if (tokens > 0) {
    if (dY == nullptr || !element_aligned(dY, xtype_size(type))) return -7;
    if (lddy < m) return -8;
    if (!valid_codes(codes)) return -9;
    if (ldc < n || ldc % 16 != 0) return -10;
    if (powers == nullptr) return -11;
    if (ldp < ceil_div(n, 32)) return -12;
  }
  if (dW == nullptr || !element_aligned(dW, 4)) return -13;
  if (lddw < n) return -14;
  if (!element_aligned(db, 4)) return -15;
  if (!sizes_supported(tokens, n, m, 0)) return RSVD_ERR_UNSUPPORTED;
  hipStream_t s = (hipStream_t)stream;
  if (tokens == 0) {
    if (ctx->device < 0) return RSVD_ERR_NO_DEVICE;
    if (accumulate) return RSVD_OK;
    RSVD_TRY(fill_zero_launch(s, m, n, dW, lddw), "zeros");
    if (db != nullptr) RSVD_TRY(fill_zero_launch(s, 1, m, db, m), "zeros");
    return RSVD_OK;
  }
  const GradLayout L = keep8_grad_layout(ctx, type, tokens, n, m);
  if (workspace == nullptr || ((uintptr_t)workspace & 255) != 0) return -17;
  if (workspace_bytes < L.total) return -18;
  const bool direct = takes_rows(type, dY, m, lddy), as_codes = kn_takes_codes(ctx, true, m, n, tokens, L.planes, false, ldc, ldp);
  if (!grad_front_fits(direct ? 0 : tokens, L.width, as_codes ? 0 : tokens, n)) return RSVD_ERR_UNSUPPORTED;
  if (ctx->device < 0) return RSVD_ERR_NO_DEVICE;
  char *ws = (char *)workspace;
  uint16_t *a = (uint16_t *)(ws + L.a), *b = (uint16_t *)(ws + L.b);
  float *sums = db != nullptr ? (float *)(ws + L.sums) : nullptr;
  {
    ProfScope ps(ctx, s, PK_SMALL);
    RSVD_TRY(grad_front_launch(ctx, s, type, tokens, m, 0, dY, lddy, nullptr, 0, nullptr, nullptr, direct ? nullptr : a, L.width, tokens, n, codes,
                               ldc, powers, ldp, as_codes ? nullptr : b, L.b_width),
             "operands of the gradient");
  }
  KnDesc d;
  d.M = m; d.N = n; d.K = tokens;
  d.a_krows = true;
  d.A = direct ? (const uint16_t *)dY : a; d.lda = (direct ? lddy : L.width) * 2; d.planes = L.planes; d.plane = tokens * L.width * 2;
  d.B = b; d.ldb = L.b_width * 2;
  if (as_codes) d.codes = codes;
  d.ldc = ldc; d.powers = powers; d.ldp = ldp;
  d.sums = sums; d.sums_out = db;
  d.out.C = dW; d.out.ldc = lddw; d.out.type = RSVD_X_F32; d.out.accumulate = accumulate;
  d.partial = (float *)(ws + L.partial); d.partial_bytes = L.partial_bytes;
  ProfScope ps(ctx, s, PK_GEMM_ATX);
  RSVD_TRY(kn_launch(ctx, s, d), "gradient of a weight");
  return RSVD_OK;
}

}  // extern "C"
