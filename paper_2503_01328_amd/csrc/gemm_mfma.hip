// bf16 GEMM on the CDNA4 matrix cores (v_mfma_f32_32x32x16_bf16), fp32 accumulate: the kernels around the tile of gemm_wide_tile.h, and
// the choice among its forms.
#include <stdint.h>
#include <stdlib.h>
#include <string.h>

#include "gemm_wide_tile.h"

namespace po {

// ---- the kernels -----------------------------------------------------------------
// One tile per block.  XCD-aware remap: ids equal modulo 8 share an XCD; each XCD gets a contiguous run of tiles.
template <int WTM, int WTN, bool TA, bool TB, int EPI, bool EDGE>
__device__ __forceinline__ void gemm_block(int M, int N, int K, const bf16* __restrict__ A, int lda,
                                           const bf16* __restrict__ B, int ldb, const Epilogue& ep, int tiles_m,
                                           int tiles_n) {
  extern __shared__ __align__(16) char smem[];
  int n_tiles = tiles_m * tiles_n;
  int pid = blockIdx.x;
  int lin = (n_tiles % 8 == 0) ? (pid % 8) * (n_tiles / 8) + pid / 8 : pid;
  int tile_m, tile_n;
  tile_of(lin, tiles_m, tiles_n, tile_m, tile_n);
  gemm_tile<WTM, WTN, TA, TB, EPI, EDGE>(M, N, K, A, lda, B, ldb, ep, tile_m, tile_n, smem);
}

template <int WTM, int WTN, bool TA, bool TB, int EPI>
__global__ __launch_bounds__(256) void gemm_mfma_kernel(int K, const bf16* __restrict__ A, int lda,
                                                        const bf16* __restrict__ B, int ldb, Epilogue ep,
                                                        int tiles_m, int tiles_n) {
  gemm_block<WTM, WTN, TA, TB, EPI, false>(0, 0, K, A, lda, B, ldb, ep, tiles_m, tiles_n);
}
template <int WTM, int WTN, bool TA, bool TB, int EPI>
__global__ __launch_bounds__(256) void gemm_edge_kernel(int M, int N, int K, const bf16* __restrict__ A, int lda,
                                                        const bf16* __restrict__ B, int ldb, Epilogue ep,
                                                        int tiles_m, int tiles_n) {
  gemm_block<WTM, WTN, TA, TB, EPI, true>(M, N, K, A, lda, B, ldb, ep, tiles_m, tiles_n);
}

// Several independent GEMMs of one form in one launch: the 256 x 256 tiles of all problems are numbered one
// problem after the other and the blocks (at most one per CU) take them round by round, so that a round is full
// as long as tiles are left, whatever the shape of a single problem (a 2048 x 2048 result alone has 64 tiles,
// a 2048 x 6144 one 192), and a block's epilogue no longer marks the end of a launch.
constexpr int kMaxGroupedGemms = 4;
struct GroupedProblem {
  const bf16* A;
  const bf16* B;
  Epilogue ep;
  int M, N, K, lda, ldb, tiles_m, tiles_n, first_tile;
};
struct GroupedArgs {
  GroupedProblem p[kMaxGroupedGemms];
  int n, total_tiles;
};

template <bool TA, bool TB, int EPI, bool EDGE>
__device__ __forceinline__ void gemm_grouped_blocks(const GroupedArgs& g) {
  extern __shared__ __align__(16) char smem[];
  int pid = blockIdx.x, nb = gridDim.x;
  int slot = (nb % 8 == 0) ? (pid % 8) * (nb / 8) + pid / 8 : pid;  // an XCD's blocks take a run of tile numbers
  for (int base = 0; base < g.total_tiles; base += nb) {
    int lin = base + slot;
    if (lin < g.total_tiles) {  // the same for every thread of the block
      // The problem that owns tile `lin`, picked with constant indices only: a run-time index into the argument
      // block would send it through private memory and the compiler would no longer know that K, the strides
      // and the LDS addresses derived from them are the same in every lane.
      GroupedProblem P = g.p[0];
#pragma unroll
      for (int i = 1; i < kMaxGroupedGemms; ++i)
        if (i < g.n && lin >= g.p[i].first_tile) P = g.p[i];
      int tile_m, tile_n;
      tile_of(lin - P.first_tile, P.tiles_m, P.tiles_n, tile_m, tile_n);
      gemm_tile<4, 4, TA, TB, EPI, EDGE>(uniform(P.M), uniform(P.N), uniform(P.K), uniform(P.A), uniform(P.lda), uniform(P.B), uniform(P.ldb), P.ep,
                                   uniform(tile_m), uniform(tile_n), smem);
    }
    __syncthreads();  // the next tile's operand loads overwrite the epilogue strips of every wave
  }
}

template <bool TA, bool TB, int EPI>
__global__ __launch_bounds__(256) void gemm_mfma_grouped_kernel(GroupedArgs g) {
  gemm_grouped_blocks<TA, TB, EPI, false>(g);
}
template <bool TA, bool TB, int EPI>
__global__ __launch_bounds__(256) void gemm_edge_grouped_kernel(GroupedArgs g) {
  gemm_grouped_blocks<TA, TB, EPI, true>(g);
}

// ---- host side ------------------------------------------------------------------
// 256 x 256 tiles once they fill three quarters of the 256 CUs in one round (measured: 192 big tiles beat 768
// small ones, 58 against 63 us at M = 2048, N = 6144, K = 2048); below that the 128 x 128 tile.  Where N is a
// multiple of 192 the 256 x 192 tile takes over when its rounds cost less: a round is as long as its slowest
// block, so 256 narrower tiles in one round beat 192 big ones with a quarter of the CUs idle, and 512 in two
// rounds beat 384 big ones (a narrow tile's round takes about 0.8 of a big tile's: 3/4 of the flops at
// slightly more operand bytes per flop).
static int tile_threshold() { return 192; }
static int64_t rounds(int64_t tiles) { return (tiles + 255) / 256; }
static void pick_tile(int M, int N, int& wtm, int& wtn) {
  wtm = wtn = 0;
  if (M % 256 == 0 && N % 256 == 0 && (int64_t)(M / 256) * (N / 256) >= tile_threshold()) {
    wtm = wtn = 4;
  } else if (M % 128 == 0 && N % 128 == 0) {
    wtm = wtn = 2;
  }
  if (M % 256 == 0 && N % 192 == 0 && (int64_t)(M / 256) * (N / 192) >= tile_threshold()) {
    int64_t narrow = 8 * rounds((int64_t)(M / 256) * (N / 192));  // in tenths of a big tile's round
    int64_t other = wtm == 4 ? 10 * rounds((int64_t)(M / 256) * (N / 256))
                             : (wtm == 2 ? 4 * rounds((int64_t)(M / 128) * (N / 128)) : INT64_MAX);
    if (narrow < other) {
      wtm = 4;
      wtn = 3;
    }
  }
}

void gemm_mfma_tile(int M, int N, int* bm, int* bn) {
  int wtm = 0, wtn = 0;
  if (M > 0 && N > 0) pick_tile(M, N, wtm, wtn);
  *bm = 64 * wtm;
  *bn = 64 * wtn;
}

bool gemm_mfma_supported(int trans_a, int trans_b, int M, int N, int K, int lda, int ldb, int ldc) {
  (void)trans_a;
  (void)trans_b;
  int wtm, wtn;
  pick_tile(M, N, wtm, wtn);
  return wtm != 0 && K > 0 && K % kBK == 0 && lda % 8 == 0 && ldb % 8 == 0 && ldc % 8 == 0;
}

template <int WTM, int WTN, bool TA, bool TB, int EPI, bool EDGE = false>
static bool launch_mfma_epi(int M, int N, int K, const bf16* A, int lda, const bf16* B, int ldb, const Epilogue& ep,
                            hipStream_t stream) {
  constexpr int BM = 64 * WTM, BN = 64 * WTN;
  constexpr int smem_ops = stages_of(WTM, WTN) * (BM + BN) * 128;
  constexpr int smem_epi = 4 * 32 * (WTN * 32 + 4) * 4;
  constexpr int smem = smem_ops > smem_epi ? smem_ops : smem_epi;
  const void* kern;
  if constexpr (EDGE) kern = reinterpret_cast<const void*>(gemm_edge_kernel<WTM, WTN, TA, TB, EPI>);
  else kern = reinterpret_cast<const void*>(gemm_mfma_kernel<WTM, WTN, TA, TB, EPI>);
  static LdsLimit lds;  // per instantiation
  if (!lds.allow(kern, smem)) return false;
  int tiles_m = ceil_div(M, BM), tiles_n = ceil_div(N, BN);
  if constexpr (EDGE)
    gemm_edge_kernel<WTM, WTN, TA, TB, EPI><<<tiles_m * tiles_n, 256, smem, stream>>>(M, N, K, A, lda, B, ldb, ep,
                                                                                   tiles_m, tiles_n);
  else
    gemm_mfma_kernel<WTM, WTN, TA, TB, EPI><<<tiles_m * tiles_n, 256, smem, stream>>>(K, A, lda, B, ldb, ep, tiles_m,
                                                                                   tiles_n);
  return launch_ok("gemm_mfma_kernel");
}

template <int WTM, int WTN, bool TA, bool TB>
static bool launch_mfma(int M, int N, int K, const bf16* A, int lda, const bf16* B, int ldb, const Epilogue& ep,
                        hipStream_t stream) {
  if (ep.acc_f32) return launch_mfma_epi<WTM, WTN, TA, TB, kEpiAccumulate>(M, N, K, A, lda, B, ldb, ep, stream);
  if (ep.gelu_u) return launch_mfma_epi<WTM, WTN, TA, TB, kEpiGeluBackward>(M, N, K, A, lda, B, ldb, ep, stream);
  if (ep.gelu_out) return launch_mfma_epi<WTM, WTN, TA, TB, kEpiStoreGelu>(M, N, K, A, lda, B, ldb, ep, stream);
  return launch_mfma_epi<WTM, WTN, TA, TB, kEpiStore>(M, N, K, A, lda, B, ldb, ep, stream);
}

template <int WTM, int WTN>
static bool dispatch_trans(int ta, int tb, int M, int N, int K, const bf16* A, int lda, const bf16* B, int ldb,
                           const Epilogue& ep, hipStream_t stream) {
  // kernel flag TB means "B is n-contiguous", i.e. the API's trans_b == 0
  if (!ta && !tb) return launch_mfma<WTM, WTN, false, true>(M, N, K, A, lda, B, ldb, ep, stream);
  if (!ta && tb) return launch_mfma<WTM, WTN, false, false>(M, N, K, A, lda, B, ldb, ep, stream);
  if (ta && !tb) return launch_mfma<WTM, WTN, true, true>(M, N, K, A, lda, B, ldb, ep, stream);
  return launch_mfma<WTM, WTN, true, false>(M, N, K, A, lda, B, ldb, ep, stream);
}

bool gemm_mfma_bf16(int trans_a, int trans_b, int M, int N, int K, const void* A, int lda, const void* B, int ldb,
                    const Epilogue& ep, hipStream_t stream) {
  if (!gemm_mfma_supported(trans_a, trans_b, M, N, K, lda, ldb, ep.ldc)) {
    set_error("gemm_mfma: unsupported shape M=%d N=%d K=%d lda=%d ldb=%d ldc=%d", M, N, K, lda, ldb, ep.ldc);
    return false;
  }
  int need_lda = trans_a ? M : K, need_ldb = trans_b ? K : N;
  if (lda < need_lda || ldb < need_ldb || ep.ldc < N || !A || !B || (!ep.out && !ep.acc_f32) ||
      (ep.gelu_u && !ep.out)) {
    set_error("gemm_mfma: bad operands (lda=%d ldb=%d ldc=%d)", lda, ldb, ep.ldc);
    return false;
  }
  uintptr_t al = (uintptr_t)A | (uintptr_t)B | (uintptr_t)ep.out | (uintptr_t)ep.gelu_out | (uintptr_t)ep.gelu_u |
                 (uintptr_t)ep.residual | (uintptr_t)ep.acc_f32 | (uintptr_t)ep.bias;
  if (al % 16 != 0) {
    set_error("gemm_mfma: operands must be 16-byte aligned");
    return false;
  }
  int wtm, wtn;
  pick_tile(M, N, wtm, wtn);
  const bf16* a = (const bf16*)A;
  const bf16* b = (const bf16*)B;
  if (wtm == 4 && wtn == 3) return dispatch_trans<4, 3>(trans_a, trans_b, M, N, K, a, lda, b, ldb, ep, stream);
  if (wtm == 4) return dispatch_trans<4, 4>(trans_a, trans_b, M, N, K, a, lda, b, ldb, ep, stream);
  return dispatch_trans<2, 2>(trans_a, trans_b, M, N, K, a, lda, b, ldb, ep, stream);
}

// ---- results of any size ----
// Time of a launch in us, from timings over M 100 .. 4000, N 1024 .. 16384, K 1024 .. 16384 (k-contiguous and k-major B
// alike): rounds of `slots` blocks, each a fixed cost and one per K slice that grows from `low` for a lone block to
// `full` where every CU has one (the clock falls).  Within 10 % of what was measured, e.g. 1733 x 6144, K 2048: 256 x 256
// 47.5, 256 x 192 42.4, 128 x 128 54.9 us, 64 x 64 73.5; 300 x 1024, K 4096: 73, 57, 25.5 us, 64 x 64 with four waves 13.6.
static double launch_us(int M, int N, int K, int bm, int bn, int slots, double fixed, double low, double full) {
  const int64_t tiles = (int64_t)ceil_div(M, bm) * ceil_div(N, bn), rest = tiles % slots;
  const double slices = ceil_div(K, kBK);
  double us = (double)(tiles / slots) * (fixed + slices * full);
  if (rest) us += fixed + slices * (low + (full - low) * (double)rest / slots);
  return us;
}
static double tile_us(int M, int N, int K, int wtm, int wtn) {
  if (wtn == 4) return launch_us(M, N, K, 256, 256, 256, 8.0, 1.04, 1.44);
  if (wtm == 4) return launch_us(M, N, K, 256, 192, 256, 6.5, 0.79, 1.12);
  return launch_us(M, N, K, 128, 128, 256, 4.3, 0.34, 0.44);
}
static double pick_edge_tile(int M, int N, int K, int& wtm, int& wtn) {
  static constexpr int forms[3][2] = {{4, 4}, {4, 3}, {2, 2}};
  double best = 0.;
  for (const auto& f : forms) {
    const double us = tile_us(M, N, K, f[0], f[1]);
    if (wtm && us >= best) continue;
    best = us;
    wtm = f[0];
    wtn = f[1];
  }
  return best;
}

bool gemm_small_is_faster(int M, int N, int K) {
  int wtm, wtn;
  pick_tile(M, N, wtm, wtn);
  // Whole large tiles whose few slices are all on their way at once win, which the estimates below do not see.  512 x 1024,
  // K 64 / 128 / 192 / 256, GeLU epilogue, us: large 5.5 / 5.7 / 6.3 / 6.6, small 6.2 / 6.8 / 7.3 / 5.6; 2048 x 2048, K 128:
  // 5.4 and 7.1.
  if (wtm && K % kBK == 0 && K < 4 * kBK) return false;
  const double big = wtm && K % kBK == 0 ? tile_us(M, N, K, wtm, wtn) : pick_edge_tile(M, N, K, wtm = 0, wtn);
  const double small4 = launch_us(M, N, K, 64, 64, 256, 4.0, 0.17, 0.17);  // a tile's K over four waves
  const double small1 = launch_us(M, N, K, 64, 64, 1024, 3.5, 0.6, 0.75);
  return (small4 < small1 ? small4 : small1) < big;
}

bool gemm_mfma_edge_supported(int ta, int tb, int M, int N, int K, const void* A, int lda, const void* B, int ldb,
                              const Epilogue& ep) {
  if (M <= 0 || N <= 0 || K <= 0 || !A || !B || (!ep.out && !ep.acc_f32) || (ep.gelu_u && !ep.out) || ep.ldc < N ||
      lda < (ta ? M : K) || ldb < (tb ? K : N))
    return false;
  if (ta ? (tb || !ep.acc_f32 || M % 8 != 0) : (ep.acc_f32 != nullptr || K % kBK != 0)) return false;  // the forms below
  if (ep.gelu_u && (!tb || ep.bias || ep.residual)) return false;  // the GeLU-backward epilogue adds neither
  if (tb && ep.gelu_out && !ep.gelu_u) return false;
  const uintptr_t al = (uintptr_t)A | (uintptr_t)B | (uintptr_t)ep.out | (uintptr_t)ep.gelu_out | (uintptr_t)ep.gelu_u |
                       (uintptr_t)ep.residual | (uintptr_t)ep.acc_f32 | (uintptr_t)ep.bias;
  // offsets and sizes of the buffer descriptors fit 31 bits: 256 rows of a k-contiguous operand, all of a k-major one and at
  // least the rows of a whole slice, whose offsets a lane forms also where K ends before
  const int64_t k_rows = K > kBK ? K : kBK;
  const int64_t a_bytes = 2 * (ta ? k_rows * lda : (int64_t)256 * lda + K);
  const int64_t b_bytes = 2 * (tb ? (int64_t)256 * ldb + K : k_rows * ldb);
  const int64_t limit = (int64_t)1 << 31;
  return N % 8 == 0 && lda % 8 == 0 && ldb % 8 == 0 && ep.ldc % 8 == 0 && al % 16 == 0 && a_bytes < limit &&
         b_bytes < limit;
}

// The forms a layer uses: forward (A k-contiguous, B not), input gradients (both k-contiguous), weight gradients (neither,
// accumulated; there K need not be whole slices either).
template <int WTM, int WTN>
static bool launch_edge(int ta, int tb, int M, int N, int K, const bf16* A, int lda, const bf16* B, int ldb,
                        const Epilogue& ep, hipStream_t stream) {
  if (ta) return launch_mfma_epi<WTM, WTN, true, true, kEpiAccumulate, true>(M, N, K, A, lda, B, ldb, ep, stream);
  if (!tb) {
    if (ep.gelu_out) return launch_mfma_epi<WTM, WTN, false, true, kEpiStoreGelu, true>(M, N, K, A, lda, B, ldb, ep, stream);
    return launch_mfma_epi<WTM, WTN, false, true, kEpiStore, true>(M, N, K, A, lda, B, ldb, ep, stream);
  }
  if (ep.gelu_u) return launch_mfma_epi<WTM, WTN, false, false, kEpiGeluBackward, true>(M, N, K, A, lda, B, ldb, ep, stream);
  return launch_mfma_epi<WTM, WTN, false, false, kEpiStore, true>(M, N, K, A, lda, B, ldb, ep, stream);
}

bool gemm_mfma_edge(int ta, int tb, int M, int N, int K, const void* A, int lda, const void* B, int ldb,
                    const Epilogue& ep, hipStream_t stream) {
  if (!gemm_mfma_edge_supported(ta, tb, M, N, K, A, lda, B, ldb, ep)) {
    set_error("gemm_mfma_edge: unsupported M=%d N=%d K=%d lda=%d ldb=%d ldc=%d", M, N, K, lda, ldb, ep.ldc);
    return false;
  }
  int wtm = 0, wtn = 0;
  pick_edge_tile(M, N, K, wtm, wtn);
  const bf16* a = (const bf16*)A;
  const bf16* b = (const bf16*)B;
  if (wtn == 4) return launch_edge<4, 4>(ta, tb, M, N, K, a, lda, b, ldb, ep, stream);
  if (wtn == 3) return launch_edge<4, 3>(ta, tb, M, N, K, a, lda, b, ldb, ep, stream);
  return launch_edge<2, 2>(ta, tb, M, N, K, a, lda, b, ldb, ep, stream);
}

// ---- grouped launch ---------------------------------------------------------------
bool gemm_mfma_grouped_supported(int n, const GemmProblem* p) {
  if (n < 1 || n > kMaxGroupedGemms || !p) return false;
  for (int i = 0; i < n; ++i) {
    const GemmProblem& q = p[i];
    if (q.M <= 0 || q.N <= 0 || q.K <= 0 || q.M % 256 != 0 || q.N % 256 != 0 || q.K % kBK != 0 || q.lda % 8 != 0 ||
        q.ldb % 8 != 0 || q.ldc % 8 != 0 || q.lda < q.M || q.ldb < q.N || q.ldc < q.N || !q.A || !q.B || !q.acc_f32 ||
        ((uintptr_t)q.A | (uintptr_t)q.B | (uintptr_t)q.acc_f32) % 16 != 0)
      return false;
  }
  return true;
}

template <bool EDGE>
static bool launch_grouped(GroupedArgs& g, hipStream_t stream) {
  constexpr int smem = stages_of(4, 4) * (256 + 256) * 128;
  auto kern = EDGE ? gemm_edge_grouped_kernel<true, true, kEpiAccumulate>
                   : gemm_mfma_grouped_kernel<true, true, kEpiAccumulate>;
  static LdsLimit lds;
  if (!lds.allow(kern, smem)) return false;
  int blocks = g.total_tiles < 256 ? g.total_tiles : 256;  // one block per CU; more tiles mean more rounds per block
  kern<<<blocks, 256, smem, stream>>>(g);
  return launch_ok("gemm_mfma_grouped_kernel");
}

static void grouped_args(int n, const GemmProblem* p, GroupedArgs& g) {
  memset(&g, 0, sizeof(g));
  g.n = n;
  int total = 0;
  for (int i = 0; i < n; ++i) {
    GroupedProblem& q = g.p[i];
    q.A = static_cast<const bf16*>(p[i].A);
    q.B = static_cast<const bf16*>(p[i].B);
    q.ep.acc_f32 = p[i].acc_f32;
    q.ep.ldc = p[i].ldc;
    q.M = p[i].M;
    q.N = p[i].N;
    q.K = p[i].K;
    q.lda = p[i].lda;
    q.ldb = p[i].ldb;
    q.tiles_m = ceil_div(p[i].M, 256);
    q.tiles_n = ceil_div(p[i].N, 256);
    q.first_tile = total;
    total += q.tiles_m * q.tiles_n;
  }
  g.total_tiles = total;
}

bool gemm_mfma_grouped_accumulate(int n, const GemmProblem* p, hipStream_t stream) {
  if (!gemm_mfma_grouped_supported(n, p)) {
    set_error("gemm_mfma_grouped: %d problems, or a shape, stride or pointer the grouped kernel does not take", n);
    return false;
  }
  GroupedArgs g;
  grouped_args(n, p, g);
  return launch_grouped<false>(g, stream);
}

// The same for M, N that are multiples of 8 and any K.
bool gemm_mfma_grouped_edge_supported(int n, const GemmProblem* p) {
  if (n < 1 || n > kMaxGroupedGemms || !p) return false;
  for (int i = 0; i < n; ++i) {
    Epilogue ep;
    memset(&ep, 0, sizeof(ep));
    ep.acc_f32 = p[i].acc_f32;
    ep.ldc = p[i].ldc;
    if (!gemm_mfma_edge_supported(1, 0, p[i].M, p[i].N, p[i].K, p[i].A, p[i].lda, p[i].B, p[i].ldb, ep)) return false;
  }
  return true;
}

bool gemm_mfma_grouped_edge_accumulate(int n, const GemmProblem* p, hipStream_t stream) {
  if (!gemm_mfma_grouped_edge_supported(n, p)) {
    set_error("gemm_mfma_grouped_edge: %d problems, or a shape, stride or pointer the grouped kernel does not take", n);
    return false;
  }
  GroupedArgs g;
  grouped_args(n, p, g);
  return launch_grouped<true>(g, stream);
}

// The four weight-gradient products of a layer of width h over s rows, us with 256 x 256 tiles / 64 x 64 tiles:
//   h  512 ( 48 tiles of 256): s 100  13.1 /  9.0, s 1733   40 /  25, s 4000   75 /  45
//   h 1024 (192):              s 100  23.9 / 26.3, s  700 34.6 / 43.4, s 4000   97 / 144
//   h 2048 (768):              s 100    73 /   90, s 1733  184 /  290, s 4000  341 / 623
//   h 4096 (3072):             s 100   323 /  518, s 1733  721 / 1277
// The line between, half a round, is where the small tiles' time, in proportion to the work, meets one round of large ones.
bool gemm_small_group_is_faster(int n, const GemmProblem* p) {
  int64_t tiles = 0;
  for (int i = 0; i < n; ++i) tiles += (int64_t)ceil_div(p[i].M, 256) * ceil_div(p[i].N, 256);
  return tiles <= 128;
}

}  // namespace po
