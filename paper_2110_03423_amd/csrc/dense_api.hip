// C entry points of the gated block, of products in 8-bit floats and of orthogonalised updates: argument checks, workspace layout, sequence of launches.  Host code only.
#include <math.h>
#include <stdio.h>

#include "dense.hpp"

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
bool valid_act(rsvd_act a) { return (int)a >= 0 && (int)a < GATED_ACTS; }
bool element_aligned(const void *p, int64_t size) { return ((uintptr_t)p & (uintptr_t)(size - 1)) == 0; }
bool valid(const void *p, int64_t size) { return p != nullptr && element_aligned(p, size); }
int kind_of(rsvd_xtype t) { return t == RSVD_X_F16 ? DK_F16 : DK_BF16; }
int planes_of(rsvd_xtype t) { return t == RSVD_X_F32 ? 3 : 1; }

struct Take {
  size_t off = 0;
  size_t operator()(size_t bytes) { const size_t o = off; off = align_up(off + bytes, 256); return o; }
};

// A matrix in memory: rows of `width` bytes, `step` bytes apart (p = NULL: none).
struct Span { const void *p; int64_t rows, width, step; };
Span span(const void *p, int64_t rows, int64_t cols, int64_t ld, int64_t size) { return {p, rows, cols * size, ld * size}; }
// Whether two have a byte in common; columns of one wider matrix have none.
bool overlap(const Span &a, const Span &b) {
  if (a.p == nullptr || b.p == nullptr || a.rows < 1 || b.rows < 1) return false;
  const uintptr_t at = (uintptr_t)a.p, bt = (uintptr_t)b.p;
  const uintptr_t a_end = at + (uintptr_t)((a.rows - 1) * a.step + a.width), b_end = bt + (uintptr_t)((b.rows - 1) * b.step + b.width);
  if (a_end <= bt || b_end <= at) return false;
  if ((a.rows == 1 && b.rows == 1) || (a.rows > 1 && b.rows > 1 && a.step != b.step)) return true;
  const int64_t step = a.rows > 1 ? a.step : b.step, d = at <= bt ? (int64_t)((bt - at) % (uintptr_t)step) : (step - (int64_t)((at - bt) % (uintptr_t)step)) % step;
  return !(d >= a.width && d + b.width <= step);
}
template <int N> bool overlap(const Span &a, const Span (&others)[N]) {
  for (const Span &b : others)
    if (overlap(a, b)) return true;
  return false;
}

// The context's device while a call launches: the null stream is the current device's.
struct OnDevice {
  int back = -1;
  hipError_t error;
  explicit OnDevice(const rsvd_ctx *ctx) {
    int now = -1;
    error = hipGetDevice(&now);
    if (error != hipSuccess || now == ctx->device) return;
    error = hipSetDevice(ctx->device);
    if (error == hipSuccess) back = now;
  }
  ~OnDevice() {
    if (back >= 0) (void)hipSetDevice(back);
  }
};
#define RSVD_ON_DEVICE()                                        \
  if (ctx->device < 0) return RSVD_ERR_NO_DEVICE;               \
  const OnDevice on(ctx);                                       \
  RSVD_TRY(on.error, "the context's device")

// Whether a matrix of n columns can be an operand as it lies.
bool laid_out(rsvd_xtype type, int64_t n, const void *p, int64_t ld) {
  return type != RSVD_X_F32 && n % 8 == 0 && rows_aligned(p, ld, 2) && ld <= kMaxLd / 2;
}

int check_sizes(rsvd_xtype type, int64_t tokens, int64_t n, int64_t m, int first) {
  if (!valid_xtype(type)) return -first;
  if (tokens < 0) return -(first + 1);
  if (n < 1) return -(first + 2);
  if (m < 1) return -(first + 3);
  return 0;
}
// (2^34 numbers: the grids of the products stay within a launch)
bool sizes_supported(int64_t tokens, int64_t n, int64_t m) {
  const int64_t most = (int64_t)1 << 34;
  return tokens <= kMaxTokens && n <= RSVD_Q8_MAX_FEATURES && m <= RSVD_Q8_MAX_FEATURES && tokens * m <= most && tokens * n <= most && n * m <= most;
}

// An operand of 16-bit numbers: where it lies, or in the workspace in planes.
struct Operand { const void *p; int64_t ld, plane; };
Operand in_place(const void *p, int64_t ld) { return {p, ld * 2, 0}; }
Operand in_planes(const void *p, int64_t rows, int64_t width) { return {p, width * 2, rows * width * 2}; }
int64_t width_of(int64_t n) { return (int64_t)align_up((size_t)n, 8); }
size_t planes_bytes(rsvd_xtype type, int64_t rows, int64_t n) { return (size_t)planes_of(type) * rows * width_of(n) * 2; }

DenseDesc gated_desc(rsvd_xtype type, int64_t tokens, int64_t n, int64_t m) {
  DenseDesc d;
  d.kind = kind_of(type); d.planes = planes_of(type);
  d.M = tokens; d.N = m; d.K = width_of(n);
  d.gated = true;
  return d;
}
// dX = D W: k counts the 2 m columns of D
DenseDesc slope_x_desc(rsvd_xtype type, int64_t tokens, int64_t n, int64_t m) {
  DenseDesc d;
  d.kind = kind_of(type); d.planes = planes_of(type);
  d.M = tokens; d.N = n; d.K = 2 * m;
  d.rows_of_n = true;
  return d;
}
// dW = D^T X: k counts tokens
DenseDesc slope_w_desc(rsvd_xtype type, int64_t tokens, int64_t n, int64_t m) {
  DenseDesc d;
  d.kind = kind_of(type); d.planes = planes_of(type);
  d.M = 2 * m; d.N = n; d.K = tokens;
  d.rows_of_n = true;
  return d;
}

struct GatedLayout { size_t x, w, D, range, partial, partial_bytes, total; };
size_t most(size_t a, size_t b) { return a > b ? a : b; }
GatedLayout gated_layout(const rsvd_ctx *ctx, rsvd_xtype type, int64_t tokens, int64_t n, int64_t m, bool x_lies, bool w_lies, bool grad, bool kept) {
  GatedLayout L;
  Take take;
  L.x = take(x_lies ? 0 : planes_bytes(type, tokens, n));
  L.w = take(w_lies ? 0 : planes_bytes(type, 2 * m, n));
  L.D = take(grad ? planes_bytes(type, tokens, 2 * m) : 0);
  L.range = take(grad && type == RSVD_X_F16 ? (3 * kRangeParts + 2) * sizeof(float) : 0);
  L.partial_bytes = kept ? 0 : dense_partial_bytes(ctx, gated_desc(type, tokens, n, m));
  if (grad) {
    L.partial_bytes = most(L.partial_bytes, dense_partial_bytes(ctx, slope_x_desc(type, tokens, n, m)));
    L.partial_bytes = most(L.partial_bytes, dense_partial_bytes(ctx, slope_w_desc(type, tokens, n, m)));
  }
  L.partial = take(L.partial_bytes);
  L.total = take.off;
  return L;
}

// ---- 8-bit floats
int64_t f8_width(int64_t n) { return (int64_t)align_up((size_t)n, 128); }
int64_t f8_powers(int64_t n) { return (int64_t)align_up((size_t)ceil_div(n, 128), 4); }
// (1024 rows of powers within the 31 bits that loads count bytes in)
constexpr int64_t kMaxPowersLd = (int64_t)1 << 20;
bool valid_codes8(const void *p) { return p != nullptr && ((uintptr_t)p & 15) == 0; }
bool valid_powers(const void *p) { return p != nullptr && ((uintptr_t)p & 3) == 0; }

// (what is added up for an fp32 result is added in fp32)
DenseDesc f8_desc(bool f32, int64_t M, int64_t N, int64_t K) {
  DenseDesc d;
  d.kind = f32 ? DK_F8_EXACT : DK_F8;
  d.M = M; d.N = N; d.K = K;
  return d;
}
struct F8Layout { size_t a, a_pow, b, b_pow, partial, partial_bytes, total; };
F8Layout f8_product_layout(const rsvd_ctx *ctx, rsvd_xtype type, int64_t tokens, int64_t n, int64_t m) {
  F8Layout L = {};
  Take take;
  if (!f8_few(type, tokens, n, m)) {
    L.a = take((size_t)tokens * f8_width(n));
    L.a_pow = take((size_t)tokens * f8_powers(n));
    L.partial_bytes = f8_few_codes(tokens, n, m) ? 0 : dense_partial_bytes(ctx, f8_desc(type == RSVD_X_F32, tokens, m, n));
    L.partial = take(L.partial_bytes);
  }
  L.total = take.off;
  return L;
}
F8Layout f8_weight_grad_layout(const rsvd_ctx *ctx, bool f32, int64_t tokens, int64_t n, int64_t m) {
  F8Layout L;
  Take take;
  L.a = take((size_t)m * f8_width(tokens));
  L.a_pow = take((size_t)m * f8_powers(tokens));
  L.b = take((size_t)n * f8_width(tokens));
  L.b_pow = take((size_t)n * f8_powers(tokens));
  L.partial_bytes = dense_partial_bytes(ctx, f8_desc(f32, m, n, tokens));
  L.partial = take(L.partial_bytes);
  L.total = take.off;
  return L;
}

// Y (tokens x m) = X^ times codes^T (m rows); `first`: the position of X among the arguments, behind which codes, powers, Y and the workspace stand.
int f8_product(rsvd_ctx *ctx, void *stream, rsvd_xtype type, int64_t tokens, int64_t n, int64_t m, const void *X, int64_t ldx, const uint8_t *codes, int64_t ldq,
               const uint8_t *powers, int64_t ldp, void *Y, int64_t ldy, void *workspace, size_t workspace_bytes, int prof) {
  const int64_t es = xtype_size(type);
  if (!valid(X, es)) return -7;
  if (ldx < n) return -8;
  if (!valid_codes8(codes)) return -9;
  if (ldq < f8_width(n) || ldq % 16 != 0) return -10;
  if (!valid_powers(powers)) return -11;
  if (ldp < f8_powers(n) || ldp % 4 != 0) return -12;
  if (!valid(Y, es)) return -13;
  if (ldy < m) return -14;
  if (!sizes_supported(tokens, n, m) || ldq > kMaxLd || ldp > kMaxPowersLd) return RSVD_ERR_UNSUPPORTED;
  if (overlap(span(Y, tokens, m, ldy, es), {span(X, tokens, n, ldx, es), span(codes, m, f8_width(n), ldq, 1), span(powers, ceil_div(m, 128), f8_powers(n), ldp, 1)})) return -13;
  const F8Layout L = f8_product_layout(ctx, type, tokens, n, m);
  if (L.total > 0 && (workspace == nullptr || ((uintptr_t)workspace & 255) != 0)) return -15;
  if (workspace_bytes < L.total) return -16;
  RSVD_ON_DEVICE();
  hipStream_t s = (hipStream_t)stream;
  if (f8_few(type, tokens, n, m)) {
    const F8FewDesc d = {type, tokens, n, m, X, ldx, codes, ldq, powers, ldp, Y, ldy};
    ProfScope ps(ctx, s, prof);
    RSVD_TRY(f8_few_launch(ctx, s, d), "product of a few tokens");
    return RSVD_OK;
  }
  char *ws = (char *)workspace;
  uint8_t *q = (uint8_t *)(ws + L.a), *p = (uint8_t *)(ws + L.a_pow);
  {
    ProfScope ps(ctx, s, PK_SMALL);
    RSVD_TRY(f8_rows_launch(s, type, tokens, n, X, ldx, q, f8_width(n), p, f8_powers(n)), "tokens to 8-bit floats");
  }
  if (f8_few_codes(tokens, n, m)) {
    const F8FewDesc d = {type, tokens, n, m, X, ldx, codes, ldq, powers, ldp, Y, ldy};
    ProfScope ps(ctx, s, prof);
    RSVD_TRY(f8_codes_launch(ctx, s, d, q, f8_width(n), p, f8_powers(n)), "product of a few tokens");
    return RSVD_OK;
  }
  DenseDesc d = f8_desc(type == RSVD_X_F32, tokens, m, n);
  d.A = q; d.lda = f8_width(n); d.a_pow = p; d.ld_apow = f8_powers(n);
  d.B = codes; d.ldb = ldq; d.b_pow = powers; d.ld_bpow = ldp; d.b_shift = 7;
  d.out.C = Y; d.out.ldc = ldy; d.out.type = type;
  d.partial = (float *)(ws + L.partial); d.partial_bytes = L.partial_bytes;
  ProfScope ps(ctx, s, prof);
  RSVD_TRY(dense_nt_launch(ctx, s, d), "product of 8-bit floats");
  return RSVD_OK;
}

// ---- orthogonalised updates
// What is held of an iteration.  An iterate X is two fp16 numbers (2^-22 left out): what a rounding of X adds in directions of small singular values would be taken for a part
// of them and grow with them (four large singular values among hundreds, a hundred times the others: 4 % of a result, 0.15 % with two numbers until the last two steps).  The square A and the
// polynomial B = b A + c A^2 are fp16 numbers off their diagonals, which are held in fp32: near the end B is close to -2.7 times the unit matrix and a I + B to 0.7 of it.
// bf16 results: products take the first number of each (what that leaves out is a relative error of A and B alone, 4 to 9e-4 of a result beside the 1.7e-3 of its
// rounding); others take two of each, and three products, for 2^-22.
int iterate_planes(rsvd_xtype type) { return type == RSVD_X_BF16 ? 1 : 2; }

struct OrthogonalLayout { size_t parts, X[2], A, B, a_diagonal, b_diagonal, partial, partial_bytes, total; int64_t small, x_ld, a_ld, x_plane, a_plane; };

DenseDesc gram_desc(rsvd_xtype type, int batch, int64_t m, int64_t n) {
  DenseDesc d;
  d.kind = DK_F16; d.planes = iterate_planes(type); d.batch = batch;
  d.M = d.N = m <= n ? m : n;
  d.K = m <= n ? width_of(n) : m;
  d.rows_of_n = m > n;
  d.symmetric = true;
  return d;
}
DenseDesc square_desc(rsvd_xtype type, int batch, int64_t small) {
  DenseDesc d;
  d.kind = DK_F16; d.planes = iterate_planes(type); d.batch = batch;
  d.M = d.N = small; d.K = width_of(small);
  d.symmetric = true;
  return d;
}
DenseDesc apply_desc(rsvd_xtype type, int batch, int64_t m, int64_t n) {
  DenseDesc d;
  d.kind = DK_F16; d.planes = iterate_planes(type); d.batch = batch;
  d.M = m; d.N = n;
  d.K = m <= n ? m : width_of(n);
  d.rows_of_n = m <= n;
  return d;
}

OrthogonalLayout orthogonal_layout(const rsvd_ctx *ctx, rsvd_xtype type, int batch, int64_t m, int64_t n) {
  OrthogonalLayout L;
  Take take;
  const int planes = iterate_planes(type);
  L.small = m <= n ? m : n;
  L.x_ld = (int64_t)align_up((size_t)n, 64);
  L.a_ld = (int64_t)align_up((size_t)L.small, 64);
  L.x_plane = (int64_t)batch * m * L.x_ld * 2;
  L.a_plane = (int64_t)batch * L.small * L.a_ld * 2;
  L.parts = take((size_t)batch * kNormParts * 8);
  for (int i = 0; i < 2; ++i) L.X[i] = take((size_t)2 * L.x_plane);
  L.A = take((size_t)planes * L.a_plane);
  L.B = take((size_t)planes * L.a_plane);
  L.a_diagonal = take((size_t)batch * L.small * 4);
  L.b_diagonal = take((size_t)batch * L.small * 4);
  L.partial_bytes = most(dense_partial_bytes(ctx, gram_desc(type, batch, m, n)), dense_partial_bytes(ctx, square_desc(type, batch, L.small)));
  L.partial_bytes = most(L.partial_bytes, dense_partial_bytes(ctx, apply_desc(type, batch, m, n)));
  L.partial = take(L.partial_bytes);
  L.total = take.off;
  return L;
}

// Whether singular values that start in [0, 1] stay where fp16 numbers times 2^13 hold them, their squares and the polynomials.  What a step makes of an interval is an interval again, whose
// ends are values at the old ones and where the derivative is zero; it is followed, not single values: between any two of those an iteration may have one that leaves.  Only what is off the diagonals of A and
// of b A + c A^2 is held in fp16, and is at most half of what their eigenvalues spread by.
// Every step's interval is widened by what rounding moves: `slack` of the magnitudes that are added up.  For bf16 results, whose products take 11 bits of each number, 2^-10: matrices of one
// magnitude round all entries alike, and 2^-12 too much at the end of a range that the next steps stretch tenfold each made NaN of them.  Others keep 22 bits: 2^-18, or
// what a sum in fp32 of as many equal numbers as the long side has may be off by: 2^-24 for each 32 that an instruction adds.
bool stays_in_range(rsvd_xtype type, int64_t longer, int steps, const float *c) {
  const double slack = type == RSVD_X_BF16 ? 0x1p-10 : fmax(0x1p-18, 0x1p-29 * (double)longer);
  double low = 0.0, high = 1.0;                          // of singular values, whose sign a step may change
  for (int s = 0; s < steps; ++s) {
    const double a = c[3 * s], b = c[3 * s + 1], g = c[3 * s + 2];
    if (!isfinite(a) || !isfinite(b) || !isfinite(g)) return false;
    auto p = [&](double y) { return y * (b + y * g); };
    auto f = [&](double x) { return x * (a + p(x * x)); };
    const double reach = fmax(fabs(low), fabs(high)), y_high = reach * reach, y_low = low <= 0.0 && high >= 0.0 ? 0.0 : fmin(low * low, high * high);
    double p_low = fmin(p(y_low), p(y_high)), p_high = fmax(p(y_low), p(y_high));
    if (g != 0.0 && -b / (2.0 * g) > y_low && -b / (2.0 * g) < y_high) {
      p_low = fmin(p_low, p(-b / (2.0 * g)));
      p_high = fmax(p_high, p(-b / (2.0 * g)));
    }
    double f_low = fmin(f(low), f(high)), f_high = fmax(f(low), f(high));
    auto turn = [&](double y) {                          // (where a + 3 b y + 5 g y^2 = 0 for y = x^2)
      if (!(y > 0.0) || !isfinite(y)) return;
      for (const double x : {sqrt(y), -sqrt(y)})
        if (x > low && x < high) {
          f_low = fmin(f_low, f(x));
          f_high = fmax(f_high, f(x));
        }
    };
    const double disc = 9.0 * b * b - 20.0 * a * g;
    if (disc >= 0.0) {                                   // (both roots without a difference of numbers that may be near each other)
      const double q = -0.5 * (3.0 * b + copysign(sqrt(disc), b));
      if (g != 0.0) turn(q / (5.0 * g));
      if (q != 0.0) turn(a / q);
    }
    const double moved = slack * reach * (fabs(a) + fmax(fabs(p_low), fabs(p_high)));
    low = f_low - moved;
    high = f_high + moved;
    if (!(p_high - p_low <= 15.0) || !(fmax(fabs(low), fabs(high)) <= 2.7)) return false;
  }
  return true;
}

}  // namespace

extern "C" {

int rsvd_gated_product_bytes(rsvd_ctx *ctx, rsvd_xtype type, int64_t tokens, int64_t n, int64_t m, int lie, size_t *bytes) {
  if (ctx == nullptr) return -1;
  if (const int rc = check_sizes(type, tokens, n, m, 2)) return rc;
  if (bytes == nullptr) return -7;
  if (!sizes_supported(tokens, n, m)) return RSVD_ERR_UNSUPPORTED;
  // (a weight that is not known to lie may do so all the same, and may then go in tiles where it would not)
  const bool can = type != RSVD_X_F32 && n % 8 == 0, x_lies = can && (lie & 1);
  *bytes = 0;
  for (const bool w_lies : {can && (lie & 2), can})
    if (!gated_few(type, tokens, n, m, w_lies)) *bytes = most(*bytes, gated_layout(ctx, type, tokens, n, m, x_lies, w_lies, false, false).total);
  return RSVD_OK;
}

int rsvd_gated_product(rsvd_ctx *ctx, void *stream, rsvd_xtype type, rsvd_act act, int64_t tokens, int64_t n, int64_t m, const void *X, int64_t ldx, const void *W,
                       int64_t ldw, void *H, int64_t ldh, void *kept, int64_t ldk, void *workspace, size_t workspace_bytes) {
  if (ctx == nullptr) return -1;
  if (!valid_xtype(type)) return -3;
  if (!valid_act(act)) return -4;
  if (tokens < 0) return -5;
  if (n < 1) return -6;
  if (m < 1) return -7;
  if (tokens == 0) return RSVD_OK;
  const int64_t es = xtype_size(type);
  if (!valid(X, es)) return -8;
  if (ldx < n) return -9;
  if (!valid(W, es)) return -10;
  if (ldw < n) return -11;
  if (!valid(H, es)) return -12;
  if (ldh < m) return -13;
  if (!element_aligned(kept, es)) return -14;
  if (kept != nullptr && ldk < 2 * m) return -15;
  if (!sizes_supported(tokens, n, m)) return RSVD_ERR_UNSUPPORTED;
  const Span x_span = span(X, tokens, n, ldx, es), w_span = span(W, 2 * m, n, ldw, es), h_span = span(H, tokens, m, ldh, es);
  if (overlap(h_span, {x_span, w_span})) return -12;
  if (overlap(span(kept, tokens, 2 * m, ldk, es), {x_span, w_span, h_span})) return -14;
  const bool x_lies = laid_out(type, n, X, ldx), w_lies = laid_out(type, n, W, ldw), few = gated_few(type, tokens, n, m, w_lies);
  const GatedLayout L = few ? GatedLayout{} : gated_layout(ctx, type, tokens, n, m, x_lies, w_lies, false, false);
  if (L.total > 0 && (workspace == nullptr || ((uintptr_t)workspace & 255) != 0)) return -16;
  if (workspace_bytes < L.total) return -17;
  RSVD_ON_DEVICE();
  hipStream_t s = (hipStream_t)stream;
  GatedOut o;
  o.act = act; o.type = type;
  o.H = H; o.ldh = ldh; o.kept = kept; o.ldk = ldk;
  if (few) {
    const GatedFewDesc d = {type, tokens, n, m, X, ldx, W, ldw, o};
    ProfScope ps(ctx, s, PK_GEMM_AX);
    RSVD_TRY(gated_few_launch(ctx, s, d), "gated product of a few tokens");
    return RSVD_OK;
  }
  char *ws = (char *)workspace;
  const int64_t width = width_of(n);
  Operand x = in_place(X, ldx), w = in_place(W, ldw);
  if (!x_lies || !w_lies) {
    if (!x_lies) x = in_planes(ws + L.x, tokens, width);
    if (!w_lies) w = in_planes(ws + L.w, 2 * m, width);
    ProfScope ps(ctx, s, PK_SMALL);
    RSVD_TRY(lay_out_launch(s, type, n, width, {X, ldx, x_lies ? 0 : tokens, (uint16_t *)(ws + L.x), x.plane},
                            {W, ldw, w_lies ? 0 : 2 * m, (uint16_t *)(ws + L.w), w.plane}, 0, m, o), "operands of the gated product");
  }
  DenseDesc d = gated_desc(type, tokens, n, m);
  d.A = x.p; d.lda = x.ld; d.a_plane = x.plane;
  d.B = w.p; d.ldb = w.ld; d.b_plane = w.plane;
  d.gate = o;
  d.partial = (float *)(ws + L.partial); d.partial_bytes = L.partial_bytes;
  ProfScope ps(ctx, s, PK_GEMM_AX);
  RSVD_TRY(dense_nt_launch(ctx, s, d), "gated product");
  return RSVD_OK;
}

int rsvd_gated_product_grad_bytes(rsvd_ctx *ctx, rsvd_xtype type, int64_t tokens, int64_t n, int64_t m, int lie, size_t *bytes) {
  if (ctx == nullptr) return -1;
  if (const int rc = check_sizes(type, tokens, n, m, 2)) return rc;
  if (bytes == nullptr) return -7;
  if (!sizes_supported(tokens, n, m)) return RSVD_ERR_UNSUPPORTED;
  const bool can = type != RSVD_X_F32 && n % 8 == 0;
  *bytes = tokens > 0 ? gated_layout(ctx, type, tokens, n, m, can && (lie & 1), can && (lie & 2), true, (lie & 4) != 0).total : 0;
  return RSVD_OK;
}

int rsvd_gated_product_grad(rsvd_ctx *ctx, void *stream, rsvd_xtype type, rsvd_act act, int64_t tokens, int64_t n, int64_t m, const void *dH, int64_t lddh, const void *X,
                            int64_t ldx, const void *W, int64_t ldw, const void *kept, int64_t ldk, void *dX, int64_t lddx, void *dW, int64_t lddw, int dw_f32,
                            int accumulate, void *workspace, size_t workspace_bytes) {
  if (ctx == nullptr) return -1;
  if (!valid_xtype(type)) return -3;
  if (!valid_act(act)) return -4;
  if (tokens < 0) return -5;
  if (n < 1) return -6;
  if (m < 1) return -7;
  const int64_t es = xtype_size(type);
  const rsvd_xtype wtype = dw_f32 ? RSVD_X_F32 : type;
  const bool recompute = kept == nullptr;
  if (tokens > 0) {
    if (!valid(dH, es)) return -8;
    if (lddh < m) return -9;
    if ((recompute || dW != nullptr) && X == nullptr) return -10;
    if (!element_aligned(X, es)) return -10;
    if (X != nullptr && ldx < n) return -11;
    if ((recompute || dX != nullptr) && W == nullptr) return -12;
    if (!element_aligned(W, es)) return -12;
    if (W != nullptr && ldw < n) return -13;
    if (!element_aligned(kept, es)) return -14;
    if (kept != nullptr && ldk < 2 * m) return -15;
    if (!element_aligned(dX, es)) return -16;
    if (dX != nullptr && lddx < n) return -17;
  }
  if (!element_aligned(dW, xtype_size(wtype))) return -18;
  if (dW != nullptr && lddw < n) return -19;
  if (accumulate && wtype != RSVD_X_F32) return -21;
  if (!sizes_supported(tokens, n, m)) return RSVD_ERR_UNSUPPORTED;
  hipStream_t s = (hipStream_t)stream;
  if (tokens == 0) {
    RSVD_ON_DEVICE();
    if (dW != nullptr && !accumulate) RSVD_TRY(zero_launch(s, wtype, 2 * m, n, dW, lddw), "zeros");
    return RSVD_OK;
  }
  const Span inputs[4] = {span(dH, tokens, m, lddh, es), span(X, tokens, n, ldx, es), span(W, 2 * m, n, ldw, es), span(kept, tokens, 2 * m, ldk, es)};
  const Span dx_span = span(dX, tokens, n, lddx, es), dw_span = span(dW, 2 * m, n, lddw, xtype_size(wtype));
  if (overlap(dx_span, inputs)) return -16;
  if (overlap(dw_span, inputs) || overlap(dw_span, dx_span)) return -18;
  const bool x_needed = recompute || dW != nullptr, w_needed = recompute || dX != nullptr;
  const bool x_lies = !x_needed || laid_out(type, n, X, ldx), w_lies = !w_needed || laid_out(type, n, W, ldw);
  const GatedLayout L = gated_layout(ctx, type, tokens, n, m, x_lies, w_lies, true, !recompute);
  if (workspace == nullptr || ((uintptr_t)workspace & 255) != 0) return -22;
  if (workspace_bytes < L.total) return -23;
  RSVD_ON_DEVICE();
  if (dX == nullptr && dW == nullptr) return RSVD_OK;
  char *ws = (char *)workspace;
  const int64_t width = width_of(n);
  Operand x = in_place(X, ldx), w = in_place(W, ldw);
  const Operand D = in_planes(ws + L.D, tokens, width_of(2 * m));
  GatedOut o;
  o.act = act; o.type = type;
  o.kept = (void *)kept; o.ldk = ldk;
  o.dH = dH; o.lddh = lddh;
  o.D = (uint16_t *)(ws + L.D); o.ldD = width_of(2 * m); o.plane = D.plane;
  float *const range = (float *)(ws + L.range), *const scale = type == RSVD_X_F16 ? range + 3 * kRangeParts : nullptr;
  o.scale = scale;
  if (scale != nullptr) {
    ProfScope ps(ctx, s, PK_SMALL);
    RSVD_TRY(range_launch(s, tokens, n, m, dH, lddh, kept, ldk, X, ldx, W, ldw, range, scale), "range of the gated gradient");
  }
  // (fp32 operands of small tiles are read as they lie)
  const bool x_wide = type == RSVD_X_F32 && !recompute && dW != nullptr && ldx <= kMaxLd / 4 && dense_takes_wide(ctx, slope_w_desc(type, tokens, n, m));
  const bool w_wide = type == RSVD_X_F32 && !recompute && dX != nullptr && ldw <= kMaxLd / 4 && dense_takes_wide(ctx, slope_x_desc(type, tokens, n, m));
  const bool lay_x = !x_lies && !x_wide, lay_w = !w_lies && !w_wide;
  if (x_wide) x = {X, ldx * 4, 0};
  if (w_wide) w = {W, ldw * 4, 0};
  if (lay_x || lay_w || !recompute) {
    if (lay_x) x = in_planes(ws + L.x, tokens, width);
    if (lay_w) w = in_planes(ws + L.w, 2 * m, width);
    ProfScope ps(ctx, s, PK_SMALL);
    RSVD_TRY(lay_out_launch(s, type, n, width, {X, ldx, lay_x ? tokens : 0, (uint16_t *)(ws + L.x), x.plane},
                            {W, ldw, lay_w ? 2 * m : 0, (uint16_t *)(ws + L.w), w.plane}, recompute ? 0 : tokens, m, o), "operands of the gated gradient");
  }
  float *partial = (float *)(ws + L.partial);
  if (recompute) {
    DenseDesc d = gated_desc(type, tokens, n, m);
    d.A = x.p; d.lda = x.ld; d.a_plane = x.plane;
    d.B = w.p; d.ldb = w.ld; d.b_plane = w.plane;
    d.gate = o;
    d.partial = partial; d.partial_bytes = L.partial_bytes;
    ProfScope ps(ctx, s, PK_GEMM_AX);
    RSVD_TRY(dense_nt_launch(ctx, s, d), "gated product");
  }
  ProfScope ps(ctx, s, PK_GEMM_ATX);
  if (dX != nullptr) {
    DenseDesc d = slope_x_desc(type, tokens, n, m);
    d.A = D.p; d.lda = D.ld; d.a_plane = D.plane;
    d.B = w.p; d.ldb = w.ld; d.b_plane = w.plane; d.b_wide = w_wide;
    d.out.C = dX; d.out.ldc = lddx; d.out.type = type;
    if (scale != nullptr) d.out.scale = scale + 1;
    d.partial = partial; d.partial_bytes = L.partial_bytes;
    RSVD_TRY(dense_kn_launch(ctx, s, d, false), "gradient of tokens");
  }
  if (dW != nullptr) {
    DenseDesc d = slope_w_desc(type, tokens, n, m);
    d.A = D.p; d.lda = D.ld; d.a_plane = D.plane;
    d.B = x.p; d.ldb = x.ld; d.b_plane = x.plane; d.b_wide = x_wide;
    d.out.C = dW; d.out.ldc = lddw; d.out.type = wtype; d.out.accumulate = accumulate;
    if (scale != nullptr) d.out.scale = scale + 1;
    d.partial = partial; d.partial_bytes = L.partial_bytes;
    RSVD_TRY(dense_kn_launch(ctx, s, d, true), "gradient of a weight");
  }
  return RSVD_OK;
}

int rsvd_f8_weight(rsvd_ctx *ctx, void *stream, rsvd_xtype type, int64_t m, int64_t n, const void *W, int64_t ldw, uint8_t *codes, int64_t ldq, uint8_t *powers,
                   int64_t ldp, uint8_t *codes_t, int64_t ldqt, uint8_t *powers_t, int64_t ldpt) {
  if (ctx == nullptr) return -1;
  if (!valid_xtype(type)) return -3;
  if (m < 1) return -4;
  if (n < 1) return -5;
  if (!valid(W, xtype_size(type))) return -6;
  if (ldw < n) return -7;
  if (!valid_codes8(codes)) return -8;
  if (ldq < f8_width(n) || ldq % 16 != 0) return -9;
  if (!valid_powers(powers)) return -10;
  if (ldp < f8_powers(n) || ldp % 4 != 0) return -11;
  if (codes_t != nullptr && !valid_codes8(codes_t)) return -12;
  if (codes_t != nullptr && (ldqt < f8_width(m) || ldqt % 16 != 0)) return -13;
  if (codes_t != nullptr && !valid_powers(powers_t)) return -14;
  if (codes_t != nullptr && (ldpt < f8_powers(m) || ldpt % 4 != 0)) return -15;
  if (!sizes_supported(1, n, m)) return RSVD_ERR_UNSUPPORTED;
  const Span w_span = span(W, m, n, ldw, xtype_size(type)), q_span = span(codes, m, f8_width(n), ldq, 1);
  if (overlap(q_span, w_span)) return -8;
  const Span qt_span = span(codes_t, n, f8_width(m), ldqt, 1);
  if (overlap(qt_span, {w_span, q_span})) return -12;
  RSVD_ON_DEVICE();
  // (behind the question for a device: a plan may name one place for the powers and what is read)
  const Span p_span = span(powers, ceil_div(m, 128), ceil_div(n, 128), ldp, 1);
  const Span pt_span = span(codes_t != nullptr ? powers_t : nullptr, ceil_div(n, 128), ceil_div(m, 128), ldpt, 1);
  if (overlap(p_span, {w_span, q_span})) return -10;
  if (overlap(qt_span, p_span)) return -12;
  if (overlap(pt_span, {w_span, q_span, qt_span, p_span})) return -14;
  ProfScope ps(ctx, (hipStream_t)stream, PK_SMALL);
  RSVD_TRY(f8_weight_launch((hipStream_t)stream, type, m, n, W, ldw, codes, ldq, powers, ldp, codes_t, ldqt, codes_t != nullptr ? powers_t : nullptr, ldpt),
           "weight to 8-bit floats");
  return RSVD_OK;
}

int rsvd_f8_product_bytes(rsvd_ctx *ctx, rsvd_xtype type, int64_t tokens, int64_t n, int64_t m, size_t *bytes) {
  if (ctx == nullptr) return -1;
  if (const int rc = check_sizes(type, tokens, n, m, 2)) return rc;
  if (bytes == nullptr) return -6;
  if (!sizes_supported(tokens, n, m)) return RSVD_ERR_UNSUPPORTED;
  *bytes = f8_product_layout(ctx, type, tokens, n, m).total;
  return RSVD_OK;
}

int rsvd_f8_product(rsvd_ctx *ctx, void *stream, rsvd_xtype type, int64_t tokens, int64_t n, int64_t m, const void *X, int64_t ldx, const uint8_t *codes, int64_t ldq,
                    const uint8_t *powers, int64_t ldp, void *Y, int64_t ldy, void *workspace, size_t workspace_bytes) {
  if (ctx == nullptr) return -1;
  if (const int rc = check_sizes(type, tokens, n, m, 3)) return rc;
  if (tokens == 0) return RSVD_OK;
  return f8_product(ctx, stream, type, tokens, n, m, X, ldx, codes, ldq, powers, ldp, Y, ldy, workspace, workspace_bytes, PK_GEMM_AX);
}

int rsvd_f8_product_grad_bytes(rsvd_ctx *ctx, rsvd_xtype type, int64_t tokens, int64_t n, int64_t m, size_t *bytes) {
  if (ctx == nullptr) return -1;
  if (const int rc = check_sizes(type, tokens, n, m, 2)) return rc;
  if (bytes == nullptr) return -6;
  if (!sizes_supported(tokens, n, m)) return RSVD_ERR_UNSUPPORTED;
  *bytes = f8_product_layout(ctx, type, tokens, m, n).total;
  return RSVD_OK;
}

int rsvd_f8_product_grad(rsvd_ctx *ctx, void *stream, rsvd_xtype type, int64_t tokens, int64_t n, int64_t m, const void *dY, int64_t lddy, const uint8_t *codes_t,
                         int64_t ldqt, const uint8_t *powers_t, int64_t ldpt, void *dX, int64_t lddx, void *workspace, size_t workspace_bytes) {
  if (ctx == nullptr) return -1;
  if (const int rc = check_sizes(type, tokens, n, m, 3)) return rc;
  if (tokens == 0) return RSVD_OK;
  return f8_product(ctx, stream, type, tokens, m, n, dY, lddy, codes_t, ldqt, powers_t, ldpt, dX, lddx, workspace, workspace_bytes, PK_GEMM_ATX);
}

int rsvd_f8_weight_grad_bytes(rsvd_ctx *ctx, rsvd_xtype type, int64_t tokens, int64_t n, int64_t m, int dw_f32, size_t *bytes) {
  if (ctx == nullptr) return -1;
  if (const int rc = check_sizes(type, tokens, n, m, 2)) return rc;
  if (bytes == nullptr) return -7;
  if (!sizes_supported(tokens, n, m)) return RSVD_ERR_UNSUPPORTED;
  *bytes = tokens > 0 ? f8_weight_grad_layout(ctx, dw_f32 || type == RSVD_X_F32, tokens, n, m).total : 0;
  return RSVD_OK;
}

int rsvd_f8_weight_grad(rsvd_ctx *ctx, void *stream, rsvd_xtype type, int64_t tokens, int64_t n, int64_t m, const void *dY, int64_t lddy, const void *X, int64_t ldx,
                        void *dW, int64_t lddw, int dw_f32, int accumulate, void *workspace, size_t workspace_bytes) {
  if (ctx == nullptr) return -1;
  if (const int rc = check_sizes(type, tokens, n, m, 3)) return rc;
  const int64_t es = xtype_size(type);
  const rsvd_xtype wtype = dw_f32 ? RSVD_X_F32 : type;
  if (tokens > 0) {
    if (!valid(dY, es)) return -7;
    if (lddy < m) return -8;
    if (!valid(X, es)) return -9;
    if (ldx < n) return -10;
  }
  if (!valid(dW, xtype_size(wtype))) return -11;
  if (lddw < n) return -12;
  if (accumulate && wtype != RSVD_X_F32) return -14;
  if (!sizes_supported(tokens, n, m)) return RSVD_ERR_UNSUPPORTED;
  hipStream_t s = (hipStream_t)stream;
  if (tokens == 0) {
    RSVD_ON_DEVICE();
    if (!accumulate) RSVD_TRY(zero_launch(s, wtype, m, n, dW, lddw), "zeros");
    return RSVD_OK;
  }
  if (overlap(span(dW, m, n, lddw, xtype_size(wtype)), {span(dY, tokens, m, lddy, es), span(X, tokens, n, ldx, es)})) return -11;
  const F8Layout L = f8_weight_grad_layout(ctx, wtype == RSVD_X_F32, tokens, n, m);
  if (workspace == nullptr || ((uintptr_t)workspace & 255) != 0) return -15;
  if (workspace_bytes < L.total) return -16;
  RSVD_ON_DEVICE();
  char *ws = (char *)workspace;
  uint8_t *a = (uint8_t *)(ws + L.a), *a_pow = (uint8_t *)(ws + L.a_pow), *b = (uint8_t *)(ws + L.b), *b_pow = (uint8_t *)(ws + L.b_pow);
  const int64_t width = f8_width(tokens), ldp = f8_powers(tokens);
  {
    ProfScope ps(ctx, s, PK_SMALL);
    RSVD_TRY(f8_columns_launch(s, type, tokens, m, dY, lddy, a, a_pow, n, X, ldx, b, b_pow, width, ldp), "gradients and tokens to 8-bit floats");
  }
  DenseDesc d = f8_desc(wtype == RSVD_X_F32, m, n, tokens);
  d.A = a; d.lda = width; d.a_pow = a_pow; d.ld_apow = ldp;
  d.B = b; d.ldb = width; d.b_pow = b_pow; d.ld_bpow = ldp;
  d.out.C = dW; d.out.ldc = lddw; d.out.type = wtype; d.out.accumulate = accumulate;
  d.partial = (float *)(ws + L.partial); d.partial_bytes = L.partial_bytes;
  ProfScope ps(ctx, s, PK_GEMM_ATX);
  RSVD_TRY(dense_nt_launch(ctx, s, d), "gradient of a weight");
  return RSVD_OK;
}

static int check_matrices(rsvd_xtype type, int batch, int64_t m, int64_t n, int first) {
  if (!valid_xtype(type)) return -first;
  if (batch < 0) return -(first + 1);
  if (m < 1) return -(first + 2);
  if (n < 1) return -(first + 3);
  return 0;
}
static bool matrices_supported(int batch, int64_t m, int64_t n) {
  return batch <= 65535 && m <= RSVD_Q8_MAX_FEATURES && n <= RSVD_Q8_MAX_FEATURES && (int64_t)batch * m * n <= (int64_t)1 << 34 &&
         batch * ceil_div(m, 256) * ceil_div(n, 256) < kDenseGroups;
}

int rsvd_orthogonalize_bytes(rsvd_ctx *ctx, rsvd_xtype type, int batch, int64_t m, int64_t n, size_t *bytes) {
  if (ctx == nullptr) return -1;
  if (const int rc = check_matrices(type, batch, m, n, 2)) return rc;
  if (bytes == nullptr) return -6;
  if (!matrices_supported(batch, m, n)) return RSVD_ERR_UNSUPPORTED;
  *bytes = batch > 0 ? orthogonal_layout(ctx, type, batch, m, n).total : 0;
  return RSVD_OK;
}

int rsvd_orthogonalize(rsvd_ctx *ctx, void *stream, rsvd_xtype type, int batch, int64_t m, int64_t n, const void *G, int64_t ldg, int64_t stride_g, int steps,
                       const float *coefficients, void *O, int64_t ldo, int64_t stride_o, void *workspace, size_t workspace_bytes) {
  if (ctx == nullptr) return -1;
  if (const int rc = check_matrices(type, batch, m, n, 3)) return rc;
  if (batch == 0) return RSVD_OK;
  const int64_t es = xtype_size(type);
  if (!valid(G, es)) return -7;
  if (ldg < n) return -8;
  if (batch > 1 && stride_g < 0) return -9;
  if (steps < 1 || steps > 64) return -10;
  if (coefficients == nullptr) return -11;
  if (!valid(O, es)) return -12;
  if (ldo < n) return -13;
  if (batch > 1 && stride_o < (m - 1) * ldo + n) return -14;
  if (!matrices_supported(batch, m, n)) return RSVD_ERR_UNSUPPORTED;
  if (!stays_in_range(type, m > n ? m : n, steps, coefficients)) return RSVD_ERR_UNSUPPORTED;
  const OrthogonalLayout L = orthogonal_layout(ctx, type, batch, m, n);
  if (workspace == nullptr || ((uintptr_t)workspace & 255) != 0) return -15;
  if (workspace_bytes < L.total) return -16;
  RSVD_ON_DEVICE();
  hipStream_t s = (hipStream_t)stream;
  char *ws = (char *)workspace;
  const int planes = iterate_planes(type);
  const bool wide = m <= n;
  {
    ProfScope ps(ctx, s, PK_SMALL);
    RSVD_TRY(norm_launch(s, type, batch, m, n, G, ldg, stride_g, (double *)(ws + L.parts)), "norm");
    RSVD_TRY(unit_launch(s, type, batch, m, n, G, ldg, stride_g, (const double *)(ws + L.parts), (uint16_t *)(ws + L.X[0]), L.x_ld, L.x_plane), "first iterate");
  }
  ProfScope ps(ctx, s, PK_GRAM);
  float *partial = (float *)(ws + L.partial);
  constexpr float kUnit = 8192.f;                     // what iterates, their squares and polynomials are held times
  auto half = [&](LinearOut &o, size_t at, int n) {
    o.C = ws + at; o.type = RSVD_X_F16; o.planes = n;
  };
  float *const a_diagonal = (float *)(ws + L.a_diagonal), *const b_diagonal = (float *)(ws + L.b_diagonal);
  // (how much what is lost of an iterate may grow until the last: from 16 times on, bf16 results need both numbers, too)
  float grows[65];
  grows[steps] = 1.f;
  for (int step = steps - 1; step >= 0; --step) grows[step] = grows[step + 1] * fmaxf(1.f, fabsf(coefficients[3 * step]));
  auto numbers = [&](int step) { return planes == 2 || grows[step] >= 16.f ? 2 : 1; };
  for (int step = 0; step < steps; ++step) {
    const char *X = ws + L.X[step & 1];
    DenseDesc g = gram_desc(type, batch, m, n);
    g.A = g.B = X; g.lda = g.ldb = L.x_ld * 2; g.a_plane = g.b_plane = L.x_plane; g.a_batch = g.b_batch = m * L.x_ld * 2;
    g.out.alpha = 1.f / kUnit;
    half(g.out, L.A, planes);
    g.out.diagonal = a_diagonal; g.out.v_batch = L.small;
    g.out.ldc = L.a_ld; g.out.c_plane = L.a_plane; g.out.c_batch = L.small * L.a_ld; g.out.width = width_of(L.small);
    g.partial = partial; g.partial_bytes = L.partial_bytes;
    if (wide) RSVD_TRY(dense_nt_launch(ctx, s, g), "square of an iterate");
    else RSVD_TRY(dense_kn_launch(ctx, s, g, true), "square of an iterate");

    DenseDesc p = square_desc(type, batch, L.small);
    p.A = p.B = ws + L.A; p.lda = p.ldb = L.a_ld * 2; p.a_plane = p.b_plane = L.a_plane; p.a_batch = p.b_batch = L.small * L.a_ld * 2;
    p.out = g.out;
    p.out.C = ws + L.B;
    p.out.alpha = coefficients[3 * step + 2] / kUnit; p.out.beta = coefficients[3 * step + 1];
    p.out.D = (const uint16_t *)(ws + L.A); p.out.ldd = L.a_ld; p.out.d_plane = L.a_plane; p.out.d_batch = L.small * L.a_ld; p.out.d_planes = planes;
    // (with A = O + diag d:  A^2 = O^2 + d_m O + O d_n off the diagonal, and d^2 on it)
    p.out.gamma = p.out.alpha; p.out.rows = p.out.columns = a_diagonal; p.out.diagonal = b_diagonal;
    p.partial = partial; p.partial_bytes = L.partial_bytes;
    RSVD_TRY(dense_nt_launch(ctx, s, p), "polynomial of an iterate");

    DenseDesc a = apply_desc(type, batch, m, n);
    const bool last = step == steps - 1;
    if (wide) { a.A = ws + L.B; a.B = X; } else { a.A = X; a.B = ws + L.B; }
    const int64_t x_batch = m * L.x_ld * 2, b_batch = L.small * L.a_ld * 2;
    a.lda = wide ? L.a_ld * 2 : L.x_ld * 2; a.a_plane = wide ? L.a_plane : L.x_plane; a.a_batch = wide ? b_batch : x_batch;
    a.ldb = wide ? L.x_ld * 2 : L.a_ld * 2; a.b_plane = wide ? L.x_plane : L.a_plane; a.b_batch = wide ? x_batch : b_batch;
    a.out.alpha = last ? 1.f / (kUnit * kUnit) : 1.f / kUnit;
    a.out.beta = last ? coefficients[3 * step] / kUnit : coefficients[3 * step];
    a.out.D = (const uint16_t *)X; a.out.ldd = L.x_ld; a.out.d_plane = L.x_plane; a.out.d_batch = m * L.x_ld; a.out.d_planes = numbers(step);
    a.out.gamma = a.out.alpha; a.out.v_batch = L.small;
    if (wide) a.out.rows = b_diagonal; else a.out.columns = b_diagonal;
    if (last) {
      a.out.C = O; a.out.ldc = ldo; a.out.c_batch = stride_o; a.out.type = type;
    } else {
      half(a.out, L.X[(step + 1) & 1], numbers(step + 1));
      a.out.ldc = L.x_ld; a.out.c_plane = L.x_plane; a.out.c_batch = m * L.x_ld; a.out.width = width_of(n);
    }
    a.partial = partial; a.partial_bytes = L.partial_bytes;
    if (wide) RSVD_TRY(dense_kn_launch(ctx, s, a, false), "next iterate");
    else RSVD_TRY(dense_nt_launch(ctx, s, a), "next iterate");
  }
  return RSVD_OK;
}

}  // extern "C"
