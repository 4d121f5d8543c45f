// The first product of the low-rank term, t = X F^T (X tokens x n, F r x n in bf16), and the rows of X in 8 bits that go with it.
//
// X is read once and is most of what there is to read, so a workgroup takes all ranks (up to 128 at a time) of its tokens.  X goes straight
// from memory into the matrix instructions, split into bf16 numbers on the way (one for bf16, two for fp16, three for fp32: exact); F goes
// through LDS, once for the four wavefronts.  Sums over ranges of k are left in fp32 for whoever needs t next to add up.
// Memory and matrix instructions are near each other: 16384 x 16384 fp16 with 128 ranks takes 162 us, 537 MB (3.3 TB/s; a copy would take 104) and two
// products of bf16 numbers (0.85 PFLOP/s); 2048 x 4096 bf16 with 64 ranks 7.5 us.
#include <type_traits>

#include "layer8_epilogue.hpp"
#include "layer8_rows.hpp"

namespace rsvd {

struct LowrankParams {
  const char *X; int64_t ldx, tokens, n;
  const uint16_t *F; int64_t ldf; int r, rp;
  float *sums;                     // [split][token][rp]
  int splits; int64_t k_per_split; // a multiple of 64
  int rank_tiles;                  // of 128 ranks
};

// ---------------------------------------------------------------- many tokens
// 64 TB tokens a workgroup, sixteen TB a wavefront, 16 RB ranks; k-steps of 64; those of F are loaded one ahead, those of X, which come
// from further away, two.  CHECK: whether infinities are looked for, which a product of rows that are NaN with one need not.
template <int XT, int RB, int TB, bool CHECK> __device__ __forceinline__ void lowrank_group(const LowrankParams &P, int group, char (*tile)[16 * RB * 128]) {
  constexpr int PARTS = XTraits<XT>::PARTS, ROWS = 16 * RB, NF = (ROWS * 8 + 255) / 256;      // 16-byte pieces of a k-step of F per thread
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, kq = lane >> 4;
  const int p0 = group % P.rank_tiles * 128;
  group /= P.rank_tiles;
  const int split = group % P.splits;      // (workgroups of an XCD share a range of F where there are eight)
  const int64_t t0 = (int64_t)(group / P.splits) * (64 * TB) + 16 * TB * wave;
  const int64_t k0 = split * P.k_per_split, k1 = k0 + P.k_per_split < P.n ? k0 + P.k_per_split : P.n;
  const char *x[TB];
#pragma unroll
  for (int i = 0; i < TB; ++i) {
    const int64_t token = t0 + 16 * i + r16;
    x[i] = P.X + (token < P.tokens ? token : P.tokens - 1) * P.ldx * XTraits<XT>::SIZE;
  }
  f32x4 acc[TB][RB];
#pragma unroll
  for (int i = 0; i < TB; ++i)
#pragma unroll
    for (int j = 0; j < RB; ++j) acc[i][j] = (f32x4)0.f;

  Raw8<XT> xa[TB][2], xb[TB][2];
  u32x4 fv[NF];
  // (whole k-steps without a look at each lane's end: a branch for every load would keep them from being under way together)
  auto load_x = [&](int64_t k, Raw8<XT> (&v)[TB][2]) RSVD_INLINE {
    auto all = [&](auto whole) RSVD_INLINE {
#pragma unroll
      for (int i = 0; i < TB; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int64_t at = k + 16 * kq + 8 * h;
          v[i][h] = raw_load8<XT>(x[i] + at * XTraits<XT>::SIZE, decltype(whole)::value ? 8 : k1 - at);
        }
    };
    if (k + 64 <= k1) all(std::true_type());
    else all(std::false_type());
  };
  auto load_f = [&](int64_t k) RSVD_INLINE {
    auto all = [&](auto whole) RSVD_INLINE {
#pragma unroll
      for (int i = 0; i < NF; ++i) {
        const int q = tid + 256 * i, row = p0 + (q >> 3);
        if (ROWS * 8 % 256 == 0 || q < ROWS * 8)
          fv[i] = halves8(P.F + (int64_t)(row < P.r ? row : P.r - 1) * P.ldf + k + 8 * (q & 7), decltype(whole)::value ? 8 : k1 - k - 8 * (q & 7));
      }
    };
    if (k + 64 <= k1) all(std::true_type());
    else all(std::false_type());
  };
  auto place = [&](int buf) RSVD_INLINE {
#pragma unroll
    for (int i = 0; i < NF; ++i) {
      const int q = tid + 256 * i, row = q >> 3;
      if (ROWS * 8 % 256 == 0 || q < ROWS * 8) *reinterpret_cast<u32x4 *>(&tile[buf][row * 128 + (((q & 7) ^ (row & 7)) << 4)]) = fv[i];
    }
  };
  auto step = [&](int64_t k, int buf, Raw8<XT> (&v)[TB][2]) RSVD_INLINE {
    u32x4 a[TB][2][PARTS];
#pragma unroll
    for (int i = 0; i < TB; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) split_operand<XT, CHECK>(v[i][h], a[i][h]);
    // (a barrier that leaves the loads in flight, which __syncthreads() would not)
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xc07f);                  // LDS
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (k + 64 < k1) load_f(k + 64);
    if (k + 128 < k1) load_x(k + 128, v);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < RB; ++j) {
        const u32x4 f = *reinterpret_cast<const u32x4 *>(&tile[buf][(16 * j + r16) * 128 + (((2 * kq + h) ^ (r16 & 7)) << 4)]);
#pragma unroll
        for (int q = PARTS - 1; q >= 0; --q)
#pragma unroll
          for (int i = 0; i < TB; ++i) acc[i][j] = mfma_bf16(f, a[i][h][q], acc[i][j]);
      }
    if (k + 64 < k1) place(buf ^ 1);
  };
  if (k0 < k1) {
    load_f(k0);
    load_x(k0, xa);
    if (k0 + 64 < k1) load_x(k0 + 64, xb);
    place(0);
  }
  for (int64_t k = k0; k < k1; k += 128) {
    step(k, 0, xa);
    if (k + 64 < k1) step(k + 64, 1, xb);
  }
#pragma unroll
  for (int i = 0; i < TB; ++i) {
    const int64_t token = t0 + 16 * i + r16;
    if (token >= P.tokens) continue;
    float *out = P.sums + ((int64_t)split * P.tokens + token) * P.rp + p0;
#pragma unroll
    for (int j = 0; j < RB; ++j) {
      const int p = 16 * j + 4 * kq;
      if (p0 + p >= P.rp) continue;
      f32x4 v = acc[i][j];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = p0 + p + e < P.r ? v[e] : 0.f;
      *reinterpret_cast<f32x4 *>(out + p) = v;
    }
  }
}

template <int XT, int RB, int TB> __global__ __launch_bounds__(256, 2) void lowrank_kernel(const LowrankParams P) {
  __shared__ __attribute__((aligned(16))) char tile[2][16 * RB * 128];
  lowrank_group<XT, RB, TB, XT == RSVD_X_F32>(P, (int)blockIdx.x, tile);
}

// The same, and behind it the operands of the gradients: three things that have nothing to do with each other, in one launch.  (4096 x 16384 bf16 with 64
// ranks, to two planes, beside 16384 x 4096 codes: 136 us for 330 MB read and 412 written, 5.5 TB/s.)
struct GradFrontParams {
  LowrankParams L; int64_t lowrank_groups;
  SplitParams S;
  WidenParams W;
};
template <int XT, int RB> __global__ __launch_bounds__(256, 2) void grad_front_kernel(const GradFrontParams P) {
  __shared__ __attribute__((aligned(16))) char tile[2][16 * RB * 128];
  int64_t group = blockIdx.x;
  if (group < P.lowrank_groups) {
    lowrank_group<XT, RB, 1, true>(P.L, (int)group, tile);
    return;
  }
  group -= P.lowrank_groups;
  if (group < P.W.groups) {
    widen_group(P.W, group);
    return;
  }
  group -= P.W.groups;
  if (P.S.factor != nullptr) split_rows_group<XT, true>(P.S, group);
  else split_rows_group<XT, false>(P.S, group);
}

// ---------------------------------------------------------------- a few tokens
// Up to 16 TB tokens and sixteen ranks a workgroup; its four wavefronts take the steps of a range of k in turn.  The workgroups behind the
// first `rank_groups` put one row of X each into 8 bits.
struct FrontParams {
  LowrankParams L;
  int rank_groups;                 // splits x rp / 16
  Rows8Params R;
};

template <int XT, int TB> __global__ __launch_bounds__(256) void front_kernel(const FrontParams F) {
  constexpr int PARTS = XTraits<XT>::PARTS;
  if ((int)blockIdx.x >= F.rank_groups) {
    rows8_row<XT, 2>(F.R, (int64_t)blockIdx.x - F.rank_groups);
    return;
  }
  const LowrankParams &P = F.L;
  __shared__ f32x4 part[4][TB][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, kq = lane >> 4;
  const int split = (int)blockIdx.x % P.splits, p0 = (int)blockIdx.x / P.splits * 16;
  const int64_t k0 = split * P.k_per_split, k1 = k0 + P.k_per_split < P.n ? k0 + P.k_per_split : P.n;
  const uint16_t *f = P.F + (int64_t)(p0 + r16 < P.r ? p0 + r16 : P.r - 1) * P.ldf;
  f32x4 acc[TB];
#pragma unroll
  for (int i = 0; i < TB; ++i) acc[i] = (f32x4)0.f;
#pragma unroll 4
  for (int64_t k = k0 + 32 * wave; k < k1; k += 128) {
    const int64_t at = k + 8 * kq;
    const u32x4 g = halves8(f + at, k1 - at);
#pragma unroll
    for (int i = 0; i < TB; ++i) {
      const int64_t m = 16 * i + r16;
      u32x4 a[PARTS];
      split_operand<XT>(raw_load8<XT>(P.X + ((m < P.tokens ? m : P.tokens - 1) * P.ldx + at) * XTraits<XT>::SIZE, k1 - at), a);
#pragma unroll
      for (int q = PARTS - 1; q >= 0; --q) acc[i] = mfma_bf16(g, a[q], acc[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < TB; ++i) part[wave][i][lane] = acc[i];
  __syncthreads();
  for (int i = wave; i < TB; i += 4) {
    const int64_t m = 16 * i + r16;
    const int p = p0 + 4 * kq;
    if (m >= P.tokens) continue;
    f32x4 sum = (part[0][i][lane] + part[1][i][lane]) + (part[2][i][lane] + part[3][i][lane]);
#pragma unroll
    for (int v = 0; v < 4; ++v) sum[v] = p + v < P.r ? sum[v] : 0.f;
    *reinterpret_cast<f32x4 *>(P.sums + ((int64_t)split * P.tokens + m) * P.rp + p) = sum;
  }
}

// ---------------------------------------------------------------- ranges of k
// Many tokens: four workgroups of four wavefronts for every CU, but at least four k-steps each.  A few: up to eight
// ranges that leave each wavefront of a workgroup four k-steps.
int lowrank_splits(const rsvd_ctx *ctx, int64_t tokens, int64_t n, int64_t r) {
  int64_t s;
  if (tokens <= kFewTokens) {
    s = ceil_div(n, 512);
    if (s > 8) s = 8;
  } else {
    s = 4 * ctx->cu_count / (ceil_div(tokens, 64) * ceil_div(r, 128));
    if (s > ceil_div(n, 256)) s = ceil_div(n, 256);
    if (s > 16) s = 16;
  }
  return s < 1 ? 1 : (int)s;
}

static LowrankParams lowrank_params(const rsvd_ctx *ctx, int64_t tokens, int64_t n, int64_t r, const void *X, int64_t ldx, const void *F,
                                    int64_t ldf, float *sums) {
  LowrankParams P;
  P.X = (const char *)X; P.ldx = ldx; P.tokens = tokens; P.n = n;
  P.F = (const uint16_t *)F; P.ldf = ldf; P.r = (int)r; P.rp = (int)rank_places(r);
  P.sums = sums;
  P.splits = lowrank_splits(ctx, tokens, n, r);
  P.k_per_split = (int64_t)align_up((size_t)ceil_div(n, P.splits), 64);
  P.rank_tiles = (int)ceil_div(r, 128);
  return P;
}

static int64_t lowrank_groups(const LowrankParams &P, int tb) { return ceil_div(P.tokens, 64 * tb) * P.splits * P.rank_tiles; }

// Two blocks of tokens a wavefront read F half as often, where that leaves every CU two workgroups: 16384 x 16384 fp16, 128 ranks, takes 165 us
// with two and 179 with one.
template <int XT, int TB> static void lowrank_typed(hipStream_t s, const LowrankParams &P) {
  const dim3 grid((unsigned)lowrank_groups(P, TB));
  if (P.r <= 32) hipLaunchKernelGGL((lowrank_kernel<XT, 2, TB>), grid, dim3(256), 0, s, P);
  else if (P.r <= 64) hipLaunchKernelGGL((lowrank_kernel<XT, 4, TB>), grid, dim3(256), 0, s, P);
  else hipLaunchKernelGGL((lowrank_kernel<XT, 8, TB>), grid, dim3(256), 0, s, P);
}
template <int XT> static void lowrank_blocks(rsvd_ctx *ctx, hipStream_t s, const LowrankParams &P) {
  if (lowrank_groups(P, 2) >= 2 * ctx->cu_count) lowrank_typed<XT, 2>(s, P);
  else lowrank_typed<XT, 1>(s, P);
}

hipError_t lowrank_launch(rsvd_ctx *ctx, hipStream_t s, rsvd_xtype type, int64_t tokens, int64_t n, int64_t r, const void *X, int64_t ldx,
                          const void *F, int64_t ldf, float *sums) {
  const LowrankParams P = lowrank_params(ctx, tokens, n, r, X, ldx, F, ldf, sums);
  if (type == RSVD_X_BF16) lowrank_blocks<RSVD_X_BF16>(ctx, s, P);
  else if (type == RSVD_X_F16) lowrank_blocks<RSVD_X_F16>(ctx, s, P);
  else lowrank_blocks<RSVD_X_F32>(ctx, s, P);
  return hipGetLastError();
}

template <int XT> static void grad_front_typed(hipStream_t s, const GradFrontParams &P) {
  const dim3 grid((unsigned)(P.lowrank_groups + P.W.groups + P.S.groups));
  if (P.L.r <= 32) hipLaunchKernelGGL((grad_front_kernel<XT, 2>), grid, dim3(256), 0, s, P);
  else if (P.L.r <= 64) hipLaunchKernelGGL((grad_front_kernel<XT, 4>), grid, dim3(256), 0, s, P);
  else hipLaunchKernelGGL((grad_front_kernel<XT, 8>), grid, dim3(256), 0, s, P);
}

hipError_t grad_front_launch(rsvd_ctx *ctx, hipStream_t s, rsvd_xtype type, int64_t tokens, int64_t m, int64_t r, const void *dY, int64_t lddy,
                             const void *F, int64_t ldf, float *sums, const float *dy_factor, uint16_t *planes, int64_t planes_width,
                             int64_t rows, int64_t n, const int8_t *codes, int64_t ldc, const uint8_t *powers, int64_t ldp, uint16_t *plane,
                             int64_t width) {
  GradFrontParams P;
  P.L = lowrank_params(ctx, tokens, m, r < 1 ? 1 : r, dY, lddy, F, ldf, sums);
  P.lowrank_groups = r > 0 ? lowrank_groups(P.L, 1) : 0;
  P.S = SplitParams{(const char *)dY, lddy, tokens, m, dy_factor, planes, planes_width, 0};
  if (planes != nullptr) P.S.groups = ceil_div(tokens * (planes_width / 8), 256);
  P.W = WidenParams{codes, ldc, powers, ldp, rows, n, plane, width, plane != nullptr ? ceil_div(rows * ceil_div(n, 16), 256) : 0};
  if (P.lowrank_groups + P.S.groups + P.W.groups == 0) return hipSuccess;
  if (type == RSVD_X_BF16) grad_front_typed<RSVD_X_BF16>(s, P);
  else if (type == RSVD_X_F16) grad_front_typed<RSVD_X_F16>(s, P);
  else grad_front_typed<RSVD_X_F32>(s, P);
  return hipGetLastError();
}

template <int XT> static void front_typed(hipStream_t s, const FrontParams &F) {
  const dim3 grid((unsigned)(F.rank_groups + F.R.rows));
  if (F.L.tokens <= 16) hipLaunchKernelGGL((front_kernel<XT, 1>), grid, dim3(256), 0, s, F);
  else if (F.L.tokens <= 32) hipLaunchKernelGGL((front_kernel<XT, 2>), grid, dim3(256), 0, s, F);
  else hipLaunchKernelGGL((front_kernel<XT, 4>), grid, dim3(256), 0, s, F);
}

hipError_t front_launch(rsvd_ctx *ctx, hipStream_t s, rsvd_xtype type, int64_t tokens, int64_t n, int64_t r, const void *X, int64_t ldx,
                        const void *F, int64_t ldf, float *sums, int8_t *codes, int64_t ldq, int64_t width, float *scale) {
  if (tokens < 1 || tokens > kFewTokens) return hipErrorInvalidValue;
  FrontParams P;
  P.L = lowrank_params(ctx, tokens, n, r < 1 ? 1 : r, X, ldx, F, ldf, sums);
  P.rank_groups = r > 0 ? P.L.splits * (P.L.rp / 16) : 0;
  P.R = Rows8Params{(const char *)X, ldx, tokens, (int)n, codes, ldq, (int)width, scale, nullptr, 0, 0, 0, nullptr};
  if (type == RSVD_X_BF16) front_typed<RSVD_X_BF16>(s, P);
  else if (type == RSVD_X_F16) front_typed<RSVD_X_F16>(s, P);
  else front_typed<RSVD_X_F32>(s, P);
  return hipGetLastError();
}

// t out of the sums over ranges of k: [token][parts][rp]
__global__ __launch_bounds__(256) void lowrank_join_kernel(const float *__restrict__ sums, int splits, int64_t tokens, int rp, int parts,
                                                           uint16_t *__restrict__ t) {
  const int64_t total = tokens * (rp / 4);
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < total; e += (int64_t)gridDim.x * 256) join_lowrank(sums, splits, tokens, rp, parts, t, e);
}

hipError_t lowrank_join_launch(hipStream_t s, const float *sums, int splits, int64_t tokens, int64_t r, int parts, uint16_t *t) {
  const int64_t rp = rank_places(r);
  int64_t blocks = ceil_div(tokens * (rp / 4), 256);
  if (blocks > 2048) blocks = 2048;
  hipLaunchKernelGGL(lowrank_join_kernel, dim3((unsigned)blocks), dim3(256), 0, s, sums, splits, tokens, (int)rp, parts, t);
  return hipGetLastError();
}

}  // namespace rsvd
