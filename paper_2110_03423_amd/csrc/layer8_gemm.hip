// Products of two matrices with consecutive k (8-bit codes, or bf16 numbers) for many tokens.
//
// Tiles of BM x BN outputs by WGM x WGN wavefronts.  A k-tile is 128 bytes of every row of both operands; a ring of S k-tiles in LDS is
// filled by loads that write there themselves.  LDS is written in the order of the lanes, 16 bytes each, so a lane fetches
// the piece that belongs to its place: piece ch of row r lies in place ch ^ (r mod 8), which lets the sixteen rows that an operand
// of a matrix instruction takes start at different banks.
// The first operand of the instruction is B, so that a lane ends with four consecutive columns of C in its registers.
// bf16 sums of several planes of A take the planes as further k, the smallest first.
#include <type_traits>

#include "layer8_epilogue.hpp"

namespace rsvd {

struct NtParams {
  const char *A, *B;
  int64_t lda, ldb, M, N, plane;
  int planes, ktiles, b_pieces;            // b_pieces: 16-byte pieces of a row of B that may be read
  int tiles_m, tiles_n, splits, kt_per_split;
  float *partial;                          // splits > 1: [split][M][N], integers for codes; behind them the low-rank term [M][N] if there is one
  Layer8Epilogue E;
};

// Operand of s_waitcnt: at most n vector memory operations outstanding, no LDS operation.
constexpr int nt_wait(int n) { return (n & 15) | ((n >> 4) << 14) | 0x0070; }

template <int BM, int BN, int S> struct NtCfg {
  static constexpr int STAGE = (BM + BN) * 128;
  static constexpr size_t lds = (size_t)S * STAGE;
};

// The loads of ROWS rows of a k-tile by NT threads.
template <int NT, int ROWS> struct NtLoad {
  static constexpr int N = ROWS * 8 / NT;
  static_assert(ROWS * 8 % NT == 0, "whole rounds");
  uint32_t off[N];
  // pieces: pieces of a row that may be read, counted from the first of this k range
  __device__ __forceinline__ void init(int64_t ld, int64_t rows_left, int tid) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int q = tid + NT * i, r = q >> 3;
      const int row = r < rows_left ? r : (int)rows_left - 1;
      off[i] = (uint32_t)row * (uint32_t)ld + (uint32_t)(((q & 7) ^ (r & 7)) << 4);
    }
  }
  // left: pieces of the k-tile that may be read; another one is read in the place of those that may not (the other operand is zero there)
  __device__ __forceinline__ void issue(const char *base, char *lds, int left, int wave, int tid) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      uint32_t o = off[i];
      if (left < 8) {
        const int q = tid + NT * i, ch = (q & 7) ^ ((q >> 3) & 7);
        if (ch >= left) o -= (uint32_t)ch << 4;
      }
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(base + o),
                                       (__attribute__((address_space(3))) void *)(lds + (wave * 64 + NT * i) * 16), 16, 0, 0);
    }
  }
};

template <bool CODES, int BM, int BN, int WGM, int WGN, int S, int PERSIMD>
__global__ __launch_bounds__(64 * WGM * WGN, PERSIMD) void nt_kernel(const NtParams P) {
  constexpr int NT = 64 * WGM * WGN, WM = BM / WGM, WN = BN / WGN, TM = WM / 16, TN = WN / 16, STAGE = NtCfg<BM, BN, S>::STAGE;
  extern __shared__ __attribute__((aligned(16))) char nt_lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, kq = lane >> 4;
  const int wm0 = (wave / WGN) * WM, wn0 = (wave % WGN) * WN;

  // Tiles: a contiguous run for each of the eight XCDs (which have an L2 each), and within it strips of eight rows of tiles, column by column.
  int tile_m, tile_n, split;
  {
    const int total = (int)gridDim.x, pid = (int)blockIdx.x;
    const int per = (total + 7) >> 3, tall = (total & 7) ? (total & 7) : 8, xcd = pid & 7, local = pid >> 3;
    int t = xcd < tall ? xcd * per + local : tall * per + (xcd - tall) * (per - 1) + local;
    const int grid_mn = P.tiles_m * P.tiles_n;
    split = t / grid_mn;
    t -= split * grid_mn;
    const int strip = t / (8 * P.tiles_n), first = strip * 8;
    const int high = P.tiles_m - first < 8 ? P.tiles_m - first : 8;
    t -= strip * 8 * P.tiles_n;
    tile_n = t / high;
    tile_m = first + t - tile_n * high;
  }
  const int64_t m0 = (int64_t)tile_m * BM, n0 = (int64_t)tile_n * BN;
  const int kt_all = P.ktiles * P.planes;
  const int kt_begin = split * P.kt_per_split;
  int nkt = kt_all - kt_begin < P.kt_per_split ? kt_all - kt_begin : P.kt_per_split;
  if (nkt < 0) nkt = 0;

  typedef typename std::conditional<CODES, i32x4, f32x4>::type acc_t;
  acc_t acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = (acc_t)0;

  NtLoad<NT, BM> la;
  NtLoad<NT, BN> lb;
  la.init(P.lda, P.M - m0, tid);
  lb.init(P.ldb, P.N - n0, tid);
  constexpr int LOADS = decltype(la)::N + decltype(lb)::N;
  static_assert((S - 2) * LOADS < 64, "the counter of outstanding loads ends at 63");
  // the k-tile that is loaded next: its plane counted from the smallest, and its place inside
  int load_plane = kt_begin / P.ktiles, load_kt = kt_begin - load_plane * P.ktiles, issued = 0;
  const char *const a_row = P.A + m0 * P.lda, *const b_row = P.B + n0 * P.ldb;
  auto issue = [&]() RSVD_INLINE {
    if (issued < nkt) {
      char *st = nt_lds + (issued % S) * STAGE;
      la.issue(a_row + (P.planes - 1 - load_plane) * P.plane + (int64_t)load_kt * 128, st, 8, wave, tid);
      lb.issue(b_row + (int64_t)load_kt * 128, st + BM * 128, P.b_pieces - load_kt * 8, wave, tid);
      if (++load_kt == P.ktiles) { load_kt = 0; ++load_plane; }
    }
    ++issued;
  };
#pragma unroll
  for (int s = 0; s < S - 1; ++s) issue();

  const int swz = r16 & 7;                       // (rows of a wavefront's blocks start at multiples of 16)
  const char *const a_lds = nt_lds + (wm0 + r16) * 128, *const b_lds = nt_lds + BM * 128 + (wn0 + r16) * 128;
  for (int kt = 0; kt < nkt; ++kt) {
    // tile kt has landed once at most the loads of the S - 2 tiles behind it are outstanding
    asm volatile("" ::: "memory");
    if (S > 2 && kt + S - 1 <= nkt) __builtin_amdgcn_s_waitcnt(nt_wait((S - 2) * LOADS));
    else __builtin_amdgcn_s_waitcnt(nt_wait(0));
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    issue();
    const int at = (kt % S) * STAGE;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int piece = ((4 * h + kq) ^ swz) << 4;
      u32x4 a[TM], b[TN];
#pragma unroll
      for (int j = 0; j < TN; ++j) b[j] = *reinterpret_cast<const u32x4 *>(b_lds + at + j * 2048 + piece);
#pragma unroll
      for (int i = 0; i < TM; ++i) a[i] = *reinterpret_cast<const u32x4 *>(a_lds + at + i * 2048 + piece);
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          if constexpr (CODES) acc[i][j] = mfma_codes(b[j], a[i], acc[i][j]);
          else acc[i][j] = mfma_bf16(b[j], a[i], acc[i][j]);
        }
    }
  }

  const Layer8Epilogue &E = P.E;
  // Parts of sums of codes stay integers, so that however k was divided the sum is exact.
  auto write_part = [&](int plane, const auto &v) RSVD_INLINE {
    Layer8Epilogue W = E;
    W.C = P.partial + (int64_t)plane * P.M * P.N;
    W.ldc = P.N;
    W.type = RSVD_X_F32;
    W.accumulate = 0;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int64_t m = m0 + wm0 + i * 16 + r16;
      if (m < P.M)
#pragma unroll
        for (int j = 0; j < TN; ++j) store4(W, m, n0 + wn0 + j * 16 + 4 * kq, P.N, __builtin_bit_cast(f32x4, v[i][j]));
    }
  };
  if (P.splits > 1) write_part(split, acc);
  if (P.splits > 1 && (E.r == 0 || split != 0)) return;

  f32x4 val[TM][TN];
  if (P.splits > 1) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) val[i][j] = (f32x4)0.f;
  } else {
    float rs[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int64_t m = m0 + wm0 + i * 16 + r16;
      rs[i] = E.rs != nullptr && m < P.M ? E.rs[m] : 1.f;
    }
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const f32x4 cs = column4(E.cs, n0 + wn0 + j * 16 + 4 * kq, P.N, 1.f);
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int v = 0; v < 4; ++v) val[i][j][v] = (float)acc[i][j][v] * rs[i] * cs[v];
    }
  }
  for (int p = 0, pr = 8 * kq; p < E.parts * E.rp; p += 32, pr = pr + 32 < E.rp ? pr + 32 : 8 * kq) {
    u32x4 a[TM], b[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const int64_t n = n0 + wn0 + j * 16 + r16;
      b[j] = factor8(E, n < P.N ? n : P.N - 1, pr);
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int64_t m = m0 + wm0 + i * 16 + r16;
      a[i] = *reinterpret_cast<const u32x4 *>(E.t + (m < P.M ? m : P.M - 1) * E.parts * E.rp + p + 8 * kq);
    }
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) val[i][j] = mfma_bf16(b[j], a[i], val[i][j]);
  }
  if (P.splits > 1) {
    write_part(P.splits, val);
    return;
  }
#pragma unroll
  for (int j = 0; j < TN; ++j) {
    const int64_t n = n0 + wn0 + j * 16 + 4 * kq;
    const f32x4 bias = column4(E.bias, n, P.N, 0.f);
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int64_t m = m0 + wm0 + i * 16 + r16;
      if (m < P.M) store4(E, m, n, P.N, E.bias != nullptr ? val[i][j] + bias : val[i][j]);
    }
  }
}

// The parts of sums over k, added in their order, and the rest of the epilogue.
template <bool CODES>
__global__ __launch_bounds__(256) void nt_reduce_kernel(const float *__restrict__ partial, int splits, int64_t M, int64_t N, Layer8Epilogue E) {
  typedef typename std::conditional<CODES, i32x4, f32x4>::type acc_t;
  typedef typename std::conditional<CODES, int, float>::type one_t;
  const int64_t per_row = (N + 3) / 4, total = M * per_row;
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < total; e += (int64_t)gridDim.x * 256) {
    const int64_t m = e / per_row, n = (e - m * per_row) * 4;
    auto part = [&](int s, auto zero) RSVD_INLINE {
      typedef decltype(zero) vec;
      vec v = zero;
      const float *p = partial + ((int64_t)s * M + m) * N + n;
      if (n + 4 <= N) {
        v = __builtin_bit_cast(vec, *reinterpret_cast<const f32x4_any *>(p));
      } else {
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (n + u < N) {
            if constexpr (std::is_same<vec, i32x4>::value) v[u] = reinterpret_cast<const int *>(p)[u];
            else v[u] = p[u];
          }
      }
      return v;
    };
    acc_t sum = (acc_t)(one_t)0;
    for (int s = 0; s < splits; ++s) sum += part(s, (acc_t)(one_t)0);
    const float rs = E.rs != nullptr ? E.rs[m] : 1.f;
    const f32x4 cs = column4(E.cs, n, N, 1.f);
    f32x4 val;
#pragma unroll
    for (int v = 0; v < 4; ++v) val[v] = (float)sum[v] * rs * cs[v];
    if (E.r > 0) val += part(splits, (f32x4)0.f);
    if (E.bias != nullptr) val += column4(E.bias, n, N, 0.f);
    store4(E, m, n, N, val);
  }
}

// ---------------------------------------------------------------- choice of tile and of the parts of k
struct NtChoice { int bm, bn, splits; int64_t kt_per_split; };

static NtChoice nt_choose(const rsvd_ctx *ctx, int64_t M, int64_t N, int64_t kt) {
  NtChoice c = {64, 64, 1, kt};
  const int64_t cus = ctx->cu_count;
  if (ceil_div(M, 256) * ceil_div(N, 256) >= cus / 2) c.bm = c.bn = 256;
  else if (ceil_div(M, 128) * ceil_div(N, 128) >= cus / 2) c.bm = c.bn = 128;
  const int64_t tiles = ceil_div(M, c.bm) * ceil_div(N, c.bn);
  const int64_t want = c.bm == 64 ? 2 * cus : cus;
  int64_t splits = want / tiles;
  if (splits > kt / 8) splits = kt / 8;
  if (splits > 16) splits = 16;
  if (splits > 1 && c.bm < 256) {
    c.kt_per_split = ceil_div(kt, splits);
    c.splits = (int)ceil_div(kt, c.kt_per_split);
  }
  return c;
}

size_t nt_partial_bytes(const rsvd_ctx *ctx, int64_t M, int64_t N, int64_t kt, bool lowrank) {
  const NtChoice c = nt_choose(ctx, M, N, kt);
  return c.splits > 1 ? (size_t)(c.splits + (lowrank ? 1 : 0)) * M * N * 4 : 0;
}

template <bool CODES, int BM, int BN, int WGM, int WGN, int S, int PERSIMD> static hipError_t nt_run(hipStream_t s, const NtParams &P) {
  hipLaunchKernelGGL((nt_kernel<CODES, BM, BN, WGM, WGN, S, PERSIMD>), dim3((unsigned)((int64_t)P.tiles_m * P.tiles_n * P.splits)),
                     dim3(64 * WGM * WGN), (NtCfg<BM, BN, S>::lds), s, P);
  return hipGetLastError();
}

template <bool CODES> static hipError_t nt_run_tile(hipStream_t s, const NtParams &P, int bm) {
  if (bm == 256) return nt_run<CODES, 256, 256, 2, 4, 2, 2>(s, P);
  if (bm == 128) return nt_run<CODES, 128, 128, 2, 2, 2, 2>(s, P);
  return nt_run<CODES, 64, 64, 2, 2, 4, 2>(s, P);
}

hipError_t layer8_init_device(rsvd_ctx *) {
  hipError_t e = hipSuccess;
  const void *wide[2] = {reinterpret_cast<const void *>(&nt_kernel<true, 256, 256, 2, 4, 2, 2>),
                         reinterpret_cast<const void *>(&nt_kernel<false, 256, 256, 2, 4, 2, 2>)};
  for (const void *k : wide)
    if (e == hipSuccess) e = hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, (int)NtCfg<256, 256, 2>::lds);
  return e;
}

hipError_t nt_launch(rsvd_ctx *ctx, hipStream_t s, const NtDesc &d) {
  const int64_t kt = d.ktiles * d.planes;
  const NtChoice c = nt_choose(ctx, d.M, d.N, kt);
  NtParams P;
  P.A = (const char *)d.A; P.B = (const char *)d.B;
  P.lda = d.lda; P.ldb = d.ldb; P.M = d.M; P.N = d.N; P.plane = d.plane;
  P.planes = d.planes; P.ktiles = (int)d.ktiles; P.b_pieces = (int)(d.b_bytes / 16);
  P.tiles_m = (int)ceil_div(d.M, c.bm); P.tiles_n = (int)ceil_div(d.N, c.bn);
  P.splits = c.splits; P.kt_per_split = (int)c.kt_per_split;
  P.partial = d.partial;
  P.E = layer8_epilogue(d.out);
  if (c.splits > 1 && (d.partial == nullptr || d.partial_bytes < nt_partial_bytes(ctx, d.M, d.N, kt, d.out.r > 0))) return hipErrorInvalidValue;
  hipError_t e = d.codes ? nt_run_tile<true>(s, P, c.bm) : nt_run_tile<false>(s, P, c.bm);
  if (e == hipSuccess && c.splits > 1) {
    int64_t blocks = ceil_div(d.M * ceil_div(d.N, 4), 256);
    if (blocks > 4096) blocks = 4096;
    if (d.codes) hipLaunchKernelGGL(nt_reduce_kernel<true>, dim3((unsigned)blocks), dim3(256), 0, s, d.partial, c.splits, d.M, d.N, P.E);
    else hipLaunchKernelGGL(nt_reduce_kernel<false>, dim3((unsigned)blocks), dim3(256), 0, s, d.partial, c.splits, d.M, d.N, P.E);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace rsvd
