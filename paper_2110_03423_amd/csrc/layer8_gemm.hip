// Products of two matrices of 8-bit codes with consecutive k, for many tokens.
//
// Tiles of BM x BN outputs by WGM x WGN wavefronts.  A k-tile is 128 codes of every row of both operands; two of them (three of small tiles, which
// are done before a load arrives: 333 x 2999 x 1410 26 -> 21 us) have room in LDS, which is
// filled by loads that write there themselves, issued over the first half of the matrix instructions of the tile before.  LDS is written in the
// order of the lanes, 16 bytes each, so a lane fetches the piece that belongs to its place: piece ch of row r lies in place ch ^ (r mod 8), which
// lets the eight rows that are read together start at different banks.
// Large products are bound by the power that the card may take (59 % of the matrix pipe's cycles at 1.9 GHz): 16384 x 4096 x 16384 939 to 986
// us (2.23 to 2.34 POP/s, a large product of the library 2.06), 2048 x 16384 x 4096 141 us (1.96, two tiles a CU and the stores of both).  256
// rows and columns by four wavefronts of 128 x 128 read LDS least (14 % busy) and have the room for it in the accumulation registers. The
// first operand of the instruction is B, so that a lane ends with four consecutive columns of C in its registers.
#include "layer8_tile.hpp"

namespace rsvd {

struct NtParams {
  const char *A, *B;
  int64_t lda, ldb;
  int b_pieces;                            // 16-byte pieces of a row of B that may be read
  TileParams T;
};

template <int BM, int BN> struct NtCfg {
  static constexpr int STAGE = (BM + BN) * 128, RING = BM == 64 ? 3 : 2;
  static constexpr size_t lds = RING * (size_t)STAGE;      // (more than the wavefronts need in the end)
};

// The loads of ROWS rows of a k-tile by NT threads.
template <int NT, int ROWS> struct NtLoad {
  static constexpr int N = ROWS * 8 / NT;
  static_assert(ROWS * 8 % NT == 0, "whole rounds");
  uint32_t off[N];
  __device__ __forceinline__ void init(int64_t ld, int64_t rows_left, int tid) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int q = tid + NT * i, r = q >> 3;
      const int row = r < rows_left ? r : (int)rows_left - 1;
      off[i] = (uint32_t)row * (uint32_t)ld + (uint32_t)(((q & 7) ^ (r & 7)) << 4);
      asm volatile("" : "+v"(off[i]));                   // (one register, not the pair that the product came in)
    }
  }
  // Load i of a thread, from `at` bytes behind the base.  left: pieces of the k-tile that may be read; another one is read in the place of those that
  // may not (the other operand is zero there).  (The buffer form: a load to LDS with a flat address would make the compiler wait for all reads
  // of LDS at once.)
  __device__ __forceinline__ void issue(int i, __amdgpu_buffer_rsrc_t base, int at, char *lds, int left, int wave, int tid) {
    uint32_t o = off[i];
    if (left < 8) {
      const int q = tid + NT * i, ch = (q & 7) ^ ((q >> 3) & 7);
      if (ch >= left) o -= (uint32_t)ch << 4;
    }
    __builtin_amdgcn_raw_ptr_buffer_load_lds(base, (__attribute__((address_space(3))) void *)(lds + (wave * 64 + NT * i) * 16), 16, o, at, 0, 0);
  }
};

template <int BM, int BN, int WGM, int WGN>
__global__ __launch_bounds__(64 * WGM * WGN, BM == 256 ? 1 : 2) void nt_kernel(const NtParams P) {
  constexpr int NT = 64 * WGM * WGN, WM = BM / WGM, WN = BN / WGN, TM = WM / 16, TN = WN / 16, STAGE = NtCfg<BM, BN>::STAGE, RING = NtCfg<BM, BN>::RING;
  extern __shared__ __attribute__((aligned(16))) char nt_lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, kq = lane >> 4;
  const int wm0 = (wave / WGN) * WM, wn0 = (wave % WGN) * WN;
  int tile_m, tile_n, split;
  tile_of(P.T, tile_m, tile_n, split);
  const int64_t m0 = (int64_t)tile_m * BM, n0 = (int64_t)tile_n * BN;
  const int kt_begin = split * P.T.kt_per_split;
  const int nkt = split == P.T.splits ? 0 : P.T.kt_all - kt_begin < P.T.kt_per_split ? P.T.kt_all - kt_begin : P.T.kt_per_split;

  i32x4 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      acc[i][j] = (i32x4)0;
      pin<BM == 256>(acc[i][j]);
    }

  NtLoad<NT, BM> la;
  NtLoad<NT, BN> lb;
  la.init(P.lda, P.T.M - m0, tid);
  lb.init(P.ldb, P.T.N - n0, tid);
  constexpr int LOADS = decltype(la)::N + decltype(lb)::N;
  const char *const a_row = P.A + m0 * P.lda + (int64_t)kt_begin * 128, *const b_row = P.B + n0 * P.ldb + (int64_t)kt_begin * 128;
  // (a buffer of 2 GiB from the tile on: its 256 rows reach that far at the most)
  const __amdgpu_buffer_rsrc_t a_all = __builtin_amdgcn_make_buffer_rsrc((void *)a_row, 0, 0x7fffffff, 0x00027000);
  const __amdgpu_buffer_rsrc_t b_all = __builtin_amdgcn_make_buffer_rsrc((void *)b_row, 0, 0x7fffffff, 0x00027000);
  auto issue = [&](int kt, int l) RSVD_INLINE {
    const int k = kt < nkt ? kt : nkt - 1;              // (behind the last tile that one again, where nobody reads it: no branches)
    char *st = nt_lds + (kt % RING) * STAGE;
    if (l < decltype(la)::N) la.issue(l, a_all, k * 128, st, 8, wave, tid);
    else lb.issue(l - decltype(la)::N, b_all, k * 128, st + BM * 128, P.b_pieces - (kt_begin + k) * 8, wave, tid);
  };
  if (nkt > 0) {
#pragma unroll
    for (int t = 0; t < RING - 1; ++t)
#pragma unroll
      for (int l = 0; l < LOADS; ++l) issue(t, l);
  }
  const int swz = r16 & 7;                       // (rows of a wavefront's blocks start at multiples of 16)
  const char *const a_lds = nt_lds + (wm0 + r16) * 128, *const b_lds = nt_lds + BM * 128 + (wn0 + r16) * 128;
  for (int kt = 0; kt < nkt; ++kt) {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(tile_wait((RING - 2) * LOADS));
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    const int at = (kt % RING) * STAGE;
    auto read_a = [&](int step) RSVD_INLINE {
      return *reinterpret_cast<const u32x4 *>(a_lds + at + step % TM * 2048 + (((4 * (step / TM) + kq) ^ swz) << 4));
    };
    auto read_b = [&](int h, int j) RSVD_INLINE { return *reinterpret_cast<const u32x4 *>(b_lds + at + j * 2048 + (((4 * h + kq) ^ swz) << 4)); };
    constexpr int AHEAD = TM >= 4 ? 3 : 1;             // rows of blocks read ahead, not all of them: registers
    u32x4 a[AHEAD + 1], b[2][TN];
#pragma unroll
    for (int j = 0; j < TN; ++j) b[0][j] = read_b(0, j);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) a[i] = read_a(i);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int step = 0; step < 2 * TM; ++step) {
      const int h = step / TM, i = step % TM;
      if (step + AHEAD < 2 * TM) a[(step + AHEAD) % (AHEAD + 1)] = read_a(step + AHEAD);
#pragma unroll
      for (int j = 0; j < TN; ++j)
        if (h == 0 && i == j * TM / TN) b[1][j] = read_b(1, j);
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = mfma_codes(b[h][j], a[step % (AHEAD + 1)], acc[i][j]);
#pragma unroll
      for (int l = 0; l < LOADS; ++l)
        if (l * TM / LOADS == step) issue(kt + RING - 1, l);
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  __builtin_amdgcn_s_waitcnt(tile_wait(0));            // (nothing may land in LDS any more)
  __syncthreads();
  int last_lane = lane;                                // (anew: what follows from it would be worked out before the main loop otherwise, and kept)
  asm volatile("" : "+v"(last_lane));
  finish_tile<TM, TN, BM == 256>(P.T, acc, split, m0 + wm0, n0 + wn0, last_lane, reinterpret_cast<float *>(nt_lds + wave * finish_lds<TN>()));
}

__global__ __launch_bounds__(256) void nt_reduce_kernel(const ReduceParams P) { reduce_group<true>(P, blockIdx.x); }

// ---------------------------------------------------------------- choice of tile and of the ranges of k
// The time of each tile and number of ranges is estimated, and the least taken.  Measured with both product kernels (4096 to 8192 k, one to four
// workgroups on a CU): a k-tile takes a CU 0.22, 0.55 and 2.05 us for each workgroup of 64, 128 and 256 rows and columns, but no less than 0.33,
// 0.78 and 1.8 us, and small tiles 0.15 us more for each further plane of A; a launch 5 us beside that; ranges of k a second launch, and their sums
// and those of a low-rank term are written and read (5 bytes / ps).  What that decides:
// 2048 x 2048, 64 k-tiles: 128 in 55 us, 256 and four ranges in 64, 64 in 65; 2048 x 1024: 128 and four ranges in 36, one in 46, 64 in 38;
// 512 x 2048: 128 and four ranges in 24, 64 in 25; 4096 x 64, 128 k-tiles: 64 and four ranges in 19, sixteen in 23.  Three planes (gradients of
// fp32), 64 k-tiles each: 256 x 4096 with a low-rank term 64 and one range in 55, two ranges in 69; 512 x 4096: 64 in 81, 128 and four in 103.
TileChoice tile_choose(const rsvd_ctx *ctx, int64_t M, int64_t N, int64_t kt, int planes, bool lowrank) {
  const struct { int b; double step, least; } tile[3] = {{64, 0.07 + 0.15 * planes, 0.18 + 0.15 * planes}, {128, 0.55, 0.78}, {256, 2.05, 1.8}};
  static const int ranges[8] = {1, 2, 3, 4, 6, 8, 12, 16};
  TileChoice best = {64, 64, 1, kt, kt};
  double least = 1e300;
  for (const auto &t : tile) {
    const int64_t all = t.b == 64 ? kt : kt * planes;
    for (const int r : ranges) {
      if (r > 1 && all < 4 * r) break;
      const int64_t per = ceil_div(all, r), used = ceil_div(all, per);
      const int64_t groups = ceil_div(ceil_div(M, t.b) * ceil_div(N, t.b) * used, ctx->cu_count);
      const double step = (double)groups * t.step;
      double us = (double)per * (step > t.least ? step : t.least);
      if (used > 1) us += 3.0 + (double)(used + (lowrank ? 1 : 0)) * (double)M * (double)N * 8.0 / 5e6;
      if (us < least) {
        least = us;
        best = TileChoice{t.b, t.b, (int)used, per, all};
      }
    }
  }
  return best;
}

size_t nt_partial_bytes(const rsvd_ctx *ctx, int64_t M, int64_t N, int64_t kt, bool lowrank) {
  return tile_partial_bytes(tile_choose(ctx, M, N, kt, 1, lowrank), M, N, lowrank);
}

template <int BM, int BN, int WGM, int WGN> static hipError_t nt_run(hipStream_t s, const NtParams &P) {
  hipLaunchKernelGGL((nt_kernel<BM, BN, WGM, WGN>), dim3(tile_groups(P.T)), dim3(64 * WGM * WGN), (NtCfg<BM, BN>::lds), s, P);
  return hipGetLastError();
}

hipError_t nt_init_device() {
  return hipFuncSetAttribute(reinterpret_cast<const void *>(&nt_kernel<256, 256, 2, 2>), hipFuncAttributeMaxDynamicSharedMemorySize,
                             (int)NtCfg<256, 256>::lds);
}

hipError_t nt_launch(rsvd_ctx *ctx, hipStream_t s, const NtDesc &d) {
  const TileChoice c = tile_choose(ctx, d.M, d.N, d.ktiles, 1, d.out.r > 0);
  if (c.splits > 1 && (d.partial == nullptr || d.partial_bytes < tile_partial_bytes(c, d.M, d.N, d.out.r > 0))) return hipErrorInvalidValue;
  const NtParams P = {(const char *)d.A, (const char *)d.B, d.lda, d.ldb, (int)(d.b_bytes / 16),
                      tile_params(c, d.M, d.N, d.ktiles, d.partial, d.out)};
  hipError_t e;
  if (c.bm == 256) e = nt_run<256, 256, 2, 2>(s, P);
  else if (c.bm == 128) e = nt_run<128, 128, 2, 2>(s, P);
  else e = nt_run<64, 64, 2, 2>(s, P);
  const ReduceParams R = reduce_params(P.T);
  if (e != hipSuccess || R.groups == 0) return e;
  hipLaunchKernelGGL(nt_reduce_kernel, dim3((unsigned)R.groups), dim3(256), 0, s, R);
  return hipGetLastError();
}

}  // namespace rsvd
