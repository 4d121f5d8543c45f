// Products of the gated block's operators: choice of tile and of the ranges of k, launches, and the sums over ranges.
#include "dense_tile.hpp"

namespace rsvd {

template <int KIND, bool GATED> hipError_t dense_nt_tile(hipStream_t s, const DenseParams &P, int b);
template <int KIND, bool GATED> hipError_t dense_nt_init();
template <int KIND, bool A_KROWS> hipError_t dense_kn_tile(hipStream_t s, const DenseParams &P, int b, bool wide);
template <int KIND, bool A_KROWS> hipError_t dense_kn_init();

static int64_t dense_tiles(const DenseDesc &d, int b) {
  const int64_t rows = ceil_div(d.M, b), columns = ceil_div(d.gated ? 2 * d.N : d.N, b);
  return d.symmetric ? rows * (rows + 1) / 2 : rows * columns;
}

// The time of each tile and number of ranges is estimated, and the least taken.  What bounds a k-tile (128 bytes of a row) of the smaller tiles is what a CU gets out of the
// L2 caches, 55 to 86 GB/s: 0.22 (0.3 where operands go through registers, 0.19 of fp16 numbers that do not) and 0.5 us for each workgroup of 64 and 128 rows and columns on a CU, but 0.3 and 0.7 us where there are not as many as CUs; tiles of 256 take
// 1.7 us, near the rate of the matrix instructions (1.4 where CUs are idle and operands do not go through registers).  Small tiles take a k-tile of all planes at once (two 0.55 us, three 1.0; 0.9 and 0.95).  Beside that 3, 5 and
// 8 us for each workgroup that a CU has behind another.  Tiles that fill the chip a number of times are worked out whole; of what is left k may be in ranges, for all CUs to
// have a part: a second launch, and their sums are written and read (5 bytes / ps).  Measured for 130 products of 80 to 3000 tokens (bf16 and fp32; gated, both gradients, 8-bit floats
// and their weights' gradients) with all tiles and one to sixteen ranges: what is chosen takes 0.3 % more than the best of them in the median, 3 % on the average, and fifteen times more than 6 %.  Four of those, 1.2 to 2.0
// times, are dX in fp32 of 128 to 256 tokens of wide layers: small tiles read the weight as it lies (dense_takes_wide), and that it need not be laid out then is not part of the estimate.
static DenseChoice dense_choose(const rsvd_ctx *ctx, const DenseDesc &d) {
  const int products = dense_segs(d.planes).count;
  const bool through = d.rows_of_n;                      // operands through registers
  const double small = d.planes == 3 ? 1.0 : d.planes == 2 ? 0.55 : through ? 0.3 : d.gated || d.kind >= DK_F8 ? 0.22 : 0.19, alone = d.planes == 3 ? 0.95 : d.planes == 2 ? 0.9 : 0.3;
  const struct { int b, at_once; double step, alone, more; } tile[3] = {{64, d.planes == 3 ? 1 : d.planes == 2 ? 2 : 3, small, alone, 3.0}, {128, 2, 0.5, 0.7, 5.0},
                                                                         {256, 1, 1.7, through ? 1.55 : 1.4, 8.0}};
  static const int ranges[9] = {1, 2, 3, 4, 6, 8, 12, 16, 24};
  const int64_t ktiles = ceil_div(d.K, dense_k(d.kind)), cu = ctx->cu_count;
  DenseChoice best = {};
  double least = 1e300;
  for (const auto &t : tile) {
    const int64_t kt = t.b == 64 ? ktiles : ktiles * products;
    const int64_t tiles = dense_tiles(d, t.b) * d.batch, full = cu * t.at_once;
    auto time = [&](int64_t groups, int64_t k) {
      const double each = groups < cu ? t.alone : (double)ceil_div(groups, cu) * t.step;
      return groups == 0 ? 0.0 : (double)ceil_div(groups, full) * t.more + (double)k * (each > t.alone ? each : t.alone);
    };
    for (const int r : ranges) {
      if (r > 1 && kt < 2 * r) break;
      const int64_t per = ceil_div(kt, r), used = ceil_div(kt, per);
      if (r > 1 && used < 2) continue;
      const int64_t whole = used > 1 ? tiles / full * full : tiles, rest = tiles - whole;
      if ((used > 1 && rest == 0) || whole + rest * used >= kDenseGroups) continue;
      double us = time(whole, kt) + time(rest * used, per);
      if (used > 1) us += 4.0 + (double)used * (double)rest * t.b * t.b * 8.0 / 5e6;
      if (us < least) {
        least = us;
        best = DenseChoice{t.b, dense_tiles(d, t.b), whole, rest, used, kt, per};
      }
    }
  }
  return best;
}

static size_t partial_bytes(const DenseChoice &c) { return c.splits > 1 ? (size_t)(c.rest * c.splits) * c.b * c.b * 4 : 0; }
size_t dense_partial_bytes(const rsvd_ctx *ctx, const DenseDesc &d) { return partial_bytes(dense_choose(ctx, d)); }

// (Every row of tiles makes its three bf16 numbers of an fp32 one, where laying out makes them once and writes and reads 12 bytes of each: gradients of 100 tokens, 4096 -> 1000 37.0 to
// 27.3 us, 301, 2999 -> 1410 61.2 to 56.4, 777, 1410 -> 512 36.9 to 36.4, 1500, 1000 -> 500 44.5 and 45.8.)
bool dense_takes_wide(const rsvd_ctx *ctx, const DenseDesc &d) { return d.planes == 3 && d.N >= 4 && d.M <= 640 && dense_choose(ctx, d).b == 64; }

static DenseParams dense_params(const DenseChoice &c, const DenseDesc &d) {
  DenseParams P;
  P.A = (const char *)d.A; P.B = (const char *)d.B;
  P.lda = d.lda; P.ldb = d.ldb; P.a_plane = d.a_plane; P.b_plane = d.b_plane; P.a_batch = d.a_batch; P.b_batch = d.b_batch;
  P.b_up = d.N * d.ldb;
  P.a_pow = d.a_pow; P.b_pow = d.b_pow; P.ld_apow = d.ld_apow; P.ld_bpow = d.ld_bpow; P.a_shift = d.a_shift; P.b_shift = d.b_shift;
  P.segs = dense_segs(d.planes);
  P.M = d.M; P.N = d.N; P.K = d.K;
  P.ktiles = (int)ceil_div(d.K, dense_k(d.kind));
  if (d.kind >= DK_F8) P.K = (int64_t)P.ktiles * 128;
  P.tiles_m = (int)ceil_div(d.M, c.b); P.tiles_n = (int)ceil_div(d.gated ? 2 * d.N : d.N, c.b);
  P.tiles = (int)c.tiles; P.batch = d.batch;
  P.kt_all = (int)c.kt;
  P.whole = (int)c.whole; P.rest = (int)c.rest; P.splits = (int)c.splits; P.kt_per_split = (int)c.kt_per_split;
  P.symmetric = d.symmetric;
  P.partial = d.partial;
  P.out = d.out; P.gate = d.gate;
  if (P.out.width == 0) P.out.width = d.N;
  return P;
}

static hipError_t dense_reduce_launch(hipStream_t s, const DenseParams &P, int b, bool gated) {
  const int across = (gated ? b / 2 : b) / 32;
  const dim3 grid((unsigned)(P.rest * across * (b / 32)));
  if (!gated) hipLaunchKernelGGL((dense_reduce_kernel<0>), grid, dim3(256), 0, s, P, b);
  else if (b > 64) hipLaunchKernelGGL((dense_reduce_kernel<32>), grid, dim3(256), 0, s, P, b);
  else hipLaunchKernelGGL((dense_reduce_kernel<16>), grid, dim3(256), 0, s, P, b);
  return hipGetLastError();
}

// Whether the operands, the room for parts and the grid are what the kernels take.
static bool fits(const DenseChoice &c, const DenseDesc &d) {
  if (c.splits > 1 && (d.partial == nullptr || d.partial_bytes < partial_bytes(c))) return false;
  if (d.symmetric && (d.M != d.N || d.gated)) return false;
  const auto pieces = [](const void *p, int64_t ld) { return p != nullptr && ((uintptr_t)p & 15) == 0 && ld % 16 == 0 && ld <= kMaxLd; };
  if (d.b_wide && (((uintptr_t)d.B & 3) != 0 || d.ldb % 4 != 0 || d.ldb > kMaxLd || d.N < 4)) return false;
  return pieces(d.A, d.lda) && (d.b_wide || pieces(d.B, d.ldb)) && c.b != 0 && c.whole + c.rest * c.splits < kDenseGroups;
}

hipError_t dense_nt_launch(rsvd_ctx *ctx, hipStream_t s, const DenseDesc &d) {
  const DenseChoice c = dense_choose(ctx, d);
  if (!fits(c, d) || d.b_wide || d.rows_of_n || (d.kind < DK_F8 && d.K % 8 != 0)) return hipErrorInvalidValue;
  const DenseParams P = dense_params(c, d);
  hipError_t e = hipErrorInvalidValue;
  if (d.kind == DK_BF16 && d.gated) e = dense_nt_tile<DK_BF16, true>(s, P, c.b);
  else if (d.kind == DK_F16 && d.gated) e = dense_nt_tile<DK_F16, true>(s, P, c.b);
  else if (d.kind == DK_F16) e = dense_nt_tile<DK_F16, false>(s, P, c.b);
  else if (d.kind == DK_F8 && !d.gated) e = dense_nt_tile<DK_F8, false>(s, P, c.b);
  else if (d.kind == DK_F8_EXACT && !d.gated) e = dense_nt_tile<DK_F8_EXACT, false>(s, P, c.b);
  return e == hipSuccess && c.splits > 1 ? dense_reduce_launch(s, P, c.b, d.gated) : e;
}

hipError_t dense_kn_launch(rsvd_ctx *ctx, hipStream_t s, const DenseDesc &d, bool a_krows) {
  const DenseChoice c = dense_choose(ctx, d);
  if (!fits(c, d) || !d.rows_of_n || d.kind >= DK_F8 || d.gated || (d.b_wide && d.kind != DK_BF16)) return hipErrorInvalidValue;
  const DenseParams P = dense_params(c, d);
  hipError_t e;
  if (d.kind == DK_BF16) e = a_krows ? dense_kn_tile<DK_BF16, true>(s, P, c.b, d.b_wide) : dense_kn_tile<DK_BF16, false>(s, P, c.b, d.b_wide);
  else e = a_krows ? dense_kn_tile<DK_F16, true>(s, P, c.b, false) : dense_kn_tile<DK_F16, false>(s, P, c.b, false);
  return e == hipSuccess && c.splits > 1 ? dense_reduce_launch(s, P, c.b, false) : e;
}

hipError_t dense_init_device(rsvd_ctx *) {
  hipError_t e = dense_nt_init<DK_BF16, true>();
  if (e == hipSuccess) e = dense_nt_init<DK_F16, true>();
  if (e == hipSuccess) e = dense_nt_init<DK_F16, false>();
  if (e == hipSuccess) e = dense_nt_init<DK_F8, false>();
  if (e == hipSuccess) e = dense_nt_init<DK_F8_EXACT, false>();
  if (e == hipSuccess) e = dense_kn_init<DK_BF16, false>();
  if (e == hipSuccess) e = dense_kn_init<DK_BF16, true>();
  if (e == hipSuccess) e = dense_kn_init<DK_F16, false>();
  if (e == hipSuccess) e = dense_kn_init<DK_F16, true>();
  return e;
}

}  // namespace rsvd
