// One output tile of the bf16 GEMM on the CDNA4 matrix cores, the wide form: what gemm_mfma.hip's kernels and the weight gradients from
// 8-bit checkpoints share.
//
// One 256-thread block (4 waves, 2 x 2) owns a (64*WTM) x (64*WTN) tile of C; a
// wave owns WTM x WTN MFMA tiles of 32 x 32, i.e. up to 128 x 128 with 256 fp32
// accumulators per lane.  K is walked in slices of 64 through a ring of LDS stages: two for the
// 256 x 256 and 256 x 192 tiles, four for the 128 x 128 tile, whose slices are too short to cover a
// memory round trip.  The 256 x 192 tile exists for outputs whose 256 x 256 tiles would leave a
// quarter of the chip idle (192 of them where 256 of the narrower ones fit).
//
// A wave is alone on its SIMD, so its one instruction stream has to keep the matrix core fed: the
// HBM -> LDS loads of a later slice, the LDS reads of the fragments three k-steps ahead and the
// MFMAs of the current k-step are woven together by hand, one load (three instructions: M0, a
// wait state, the load with a scalar base and a 32-bit lane offset) and one fragment read per two
// MFMAs, with a single barrier per slice placed where no MFMA waits for what follows it.
//
// Operand slices travel HBM -> LDS directly (global_load_lds_dwordx4: lane L of
// a wave deposits its 16 bytes at LDS base + 16 L), so no registers and no
// ds_write instructions are spent on staging.  Because the LDS side of such a
// load is fixed, the bank-conflict swizzle is applied on the global side: each
// lane fetches the 16-byte chunk that belongs at its LDS position.
//
// Two LDS layouts, chosen by how the operand lies in memory:
//   k-contiguous operand (A of forward/dgrad, B of dgrad): "row tile"
//     [rows][64] bf16, 128 bytes per row, 16-byte chunk c stored at c ^ (row & 7);
//     an MFMA fragment is one ds_read_b128.
//   operand whose contiguous index is m or n (B of forward, both of wgrad):
//     "k-major tile" [64][rows] bf16, 32-byte unit u of a row stored at
//     u ^ (k & 7) (u ^ (k & 3) when a row has 12 units); an MFMA fragment is two transposing reads (ds_read_b64_tr_b16),
//     arranged so that a lane receives k = 16 kk + 8 half + 0..7 exactly as the
//     ds_read_b128 path does, which lets the two kinds be mixed in one MFMA.
// Nothing is transposed in registers.
//
// The MFMA is issued with the B fragment in the first operand slot, so a lane holds
// four consecutive n of one row m per accumulator quad.  The epilogue moves each
// 32-row strip of a wave through LDS and then touches global memory row-wise, 16
// bytes per lane, whole 128-byte lines per row: bias, residual, GeLU, GeLU-backward
// and the fp32 accumulate all happen on that coalesced side.
//
// Results that are no whole tiles use a second form of the same kernel, EDGE: loads through buffer descriptors, guarded
// stores.  A stage of C2's widths at 1733 rows: forward products 101, 133 and 73 us with the 64 x 64 tiles of
// gemm_small.hip -> 54, 68 and 52 us, the four weight gradients 345 -> 195 us (261 with every tile guarded), the step
// 5.18 -> 3.68 ms.
//
// Workgroup ids are remapped so that the blocks that land on one XCD (ids equal
// modulo 8) work on neighbouring tiles and share operand slices in that XCD's L2.
#pragma once

#include <type_traits>

#include "mfma_common.h"

namespace po {

#define PO_LDS3(p) ((void __attribute__((address_space(3)))*)(p))
#define PO_GLB1(p) ((const void __attribute__((address_space(1)))*)(p))
#define PO_LDS_S16X4(p) ((s16x4 __attribute__((address_space(3)))*)(p))

constexpr int kBK = 64;

enum EpiKind : int { kEpiStore = 0, kEpiStoreGelu = 1, kEpiGeluBackward = 2, kEpiAccumulate = 3, kEpiStoreF32 = 4 };

// ---- HBM -> LDS, one operand slice -----------------------------------------------
// KMAJOR == false: operand is [R rows][K], slice = R rows x 64 k, row tile in LDS.
// KMAJOR == true : operand is [K][R], slice = 64 k x R, k-major tile in LDS.
// Swizzle of the k-major tile: row k keeps unit u at position u ^ (k & mask).  The position must stay inside
// the row, so a row of 12 units (R = 192) swaps only within groups of four; the fragment reads of four
// consecutive k and two neighbouring units still fall into eight different 32-byte bank groups.
template <int R>
__device__ __forceinline__ int kmajor_unit(int u, int k) {
  static_assert(R % 64 == 0, "rows of the k-major tile are whole groups of four units");
  constexpr int MASK = (R % 128 == 0) ? 7 : 3;
  return u ^ (k & MASK);
}

// The slice is R * 128 bytes = R / 8 wave-wide loads of 1 KiB; wave w issues pieces w, w + 4, w + 8, ...
// What a lane fetches for piece u never changes from slice to slice except for a step that is the same for every
// lane, so the lane keeps one 32-bit byte offset per piece and the wave one 64-bit slice pointer in scalar
// registers: a load costs its own instruction and the M0 set-up, no address arithmetic.
// EDGE: the loads go through a buffer descriptor that starts at the slice pointer and ends with the operand, so rows of
// a k-contiguous operand past its last one and k of the other kind past K read as zero; what a k-major slice reads past
// its rows is the next k's (or zero) and ends up in results that are not stored.
template <int R, bool KMAJOR, bool EDGE>
struct SliceLoader {
  static constexpr int N_INST = R * 128 / 1024;
  static constexpr int PER_WAVE = N_INST / 4;
  static_assert(N_INST % 4 == 0 && PER_WAVE >= 4, "tile too small for four waves");
  unsigned voff[PER_WAVE];  // this lane's byte offset from the slice pointer, per piece
  const char* slice;        // first byte of the next slice to request (same in every lane)
  unsigned step;            // bytes from one slice to the next
  int left;                 // EDGE: bytes from the slice pointer to the end of the operand (may fall below zero)

  // `base` points at (first row of the tile, k = 0); rows: how many the operand has from there on.
  __device__ __forceinline__ void init(const bf16* base, int ld, int rows, int K, int wave, int lane) {
#pragma unroll
    for (int u = 0; u < PER_WAVE; ++u) {
      int g = u * 4 + wave;  // which 1 KiB piece of the tile
      unsigned elem;
      if (!KMAJOR) {
        int row = 8 * g + (lane >> 3);
        int c = (lane & 7) ^ (row & 7);
        elem = (unsigned)row * (unsigned)ld + c * 8;
      } else {
        constexpr int ROW_BYTES = 2 * R;
        int byte = g * 1024 + lane * 16;
        int k = byte / ROW_BYTES;
        int pos16 = (byte % ROW_BYTES) >> 4;
        int unit = kmajor_unit<R>(pos16 >> 1, k);
        elem = (unsigned)k * (unsigned)ld + (unit * 2 + (pos16 & 1)) * 8;
      }
      voff[u] = elem * 2;
    }
    slice = reinterpret_cast<const char*>(base);
    step = KMAJOR ? 128u * (unsigned)ld : 128u;
    if (EDGE) left = KMAJOR ? ((K - 1) * ld + rows) * 2 : ((min(rows, R) - 1) * ld + K) * 2;
  }
  // Piece u of the slice at `slice` -> LDS at lds_wave + 4096 u (lds_wave: the LDS address of this wave's piece 0
  // in the target stage).  Issued as inline assembly on purpose: through the builtin the compiler treats every
  // later LDS read as dependent on the load and waits for it at once, which would undo the double buffering.
  // The caller waits (wait_loads) before the barrier that publishes the slice.
  __device__ __forceinline__ void issue(int u, unsigned lds_wave) const {
    unsigned dst = lds_wave + 4096u * u;
    if constexpr (EDGE) buffer_to_lds(dst, voff[u], buffer_of(slice, (unsigned)max(left, 0)));
    else asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(dst), "v"(voff[u]), "s"(slice)
                 : "memory");
  }
  __device__ __forceinline__ void advance() {
    slice += step;
    if (EDGE) left -= (int)step;
  }
};

// Eight codes with one scale as bf16, exactly.
__device__ __forceinline__ u32x4 widen8(uint2 codes, unsigned byte) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const float scale = __uint_as_float(byte << 23);
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes.x, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes.x, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes.y, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes.y, scale, true);
  return u32x4{__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b), __builtin_bit_cast(unsigned, c), __builtin_bit_cast(unsigned, d)};
}

// ---- codes -> LDS, one operand slice of an 8-bit checkpoint --------------------------
// The operand is [K][R columns] as saved8.h has it; a slice becomes the same k-major tile in LDS.  Its codes have to be scaled on the way, so they
// go through registers: sixteen columns of a k (one unit, one scale) at a time, loaded a whole slice before they are converted.  Four units of a
// thread are 32 conversions and eight LDS writes a slice, beside 64 MFMAs of a wave; converting fragments instead, where a lane's eight k
// have eight scales, would take ten times as many.
struct Saved8Operand {
  const uint8_t *codes, *scales;
  int padded, rows;  // codes in a row; rows (K)
};
template <int R>
struct Saved8SliceLoader {
  static constexpr int PER_WAVE = 0;  // direct loads
  static constexpr int UNITS = R * kBK / 16 / 256;
  static_assert(R % 128 == 0, "a thread's units are whole k apart");
  u32x4 codes[UNITS];
  unsigned byte[UNITS];
  unsigned at[UNITS], scale_at[UNITS], lds_at[UNITS];
  const uint8_t *slice, *scale_slice;
  int64_t left;  // codes from the slice on
  int step;

  __device__ __forceinline__ void init(const Saved8Operand& x, int column0, int tid) {
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      const int q = u * 256 + tid, k = q / (R / 16), unit = q % (R / 16);
      at[u] = (unsigned)k * (unsigned)x.padded + column0 + 16 * unit;
      scale_at[u] = at[u] >> 5;
      lds_at[u] = k * (2 * R) + (kmajor_unit<R>(unit, k) << 5);
    }
    slice = x.codes;
    scale_slice = x.scales;
    left = (int64_t)x.rows * x.padded;
    step = kBK * x.padded;
  }
  // Codes behind the last row are zero, as a load past its buffer is; columns past a row's end are the next row's and end up in
  // results that are not stored.
  __device__ __forceinline__ void load(int u) {
    const unsigned bytes = (unsigned)min(max(left, (int64_t)0), (int64_t)0xffffffe0);
    codes[u] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(buffer_resource(slice, bytes), (int)at[u], 0, 0));
    byte[u] = __builtin_amdgcn_raw_buffer_load_b8(buffer_resource(scale_slice, bytes >> 5), (int)scale_at[u], 0, 0);
  }
  __device__ __forceinline__ void advance() {
    slice += step;
    scale_slice += step >> 5;
    left -= step;
  }
  __device__ __forceinline__ void put(int u, char* stage) const {
    *reinterpret_cast<u32x4*>(stage + lds_at[u]) = widen8(make_uint2(codes[u][0], codes[u][1]), byte[u]);
    *reinterpret_cast<u32x4*>(stage + lds_at[u] + 16) = widen8(make_uint2(codes[u][2], codes[u][3]), byte[u]);
  }
};

// ---- LDS -> MFMA fragment: 32 rows (row0 + lane % 32), k = 16 kk + 8 (lane / 32) + 0..7 ----
template <int R, bool KMAJOR>
__device__ __forceinline__ bf16x8 read_fragment(const char* lds, int row0, int kk, int lane) {
  if (!KMAJOR) {
    int row = row0 + (lane & 31);
    int c = (2 * kk + (lane >> 5)) ^ (row & 7);
    return *reinterpret_cast<const bf16x8*>(lds + row * 128 + (c << 4));
  } else {
    // Transposing read: within a group of 16 lanes, lane i receives element (i % 4) of the
    // addresses supplied by lanes i / 4, 4 + i / 4, 8 + i / 4, 12 + i / 4.  Lane r of the group
    // supplies row k = kbase + r / 4, columns m0 + 4 (r % 4) .. + 3; lane i then holds
    // k = kbase .. kbase + 3 of column m0 + i.
    constexpr int ROW_BYTES = 2 * R;
    int i = lane & 15, grp = lane >> 4;
    int m = row0 + 16 * (grp & 1) + 4 * (i & 3);
    int k = 16 * kk + 8 * (grp >> 1) + (i >> 2);
    int unit = m >> 4;
    int inner = (m & 15) * 2;
    const char* p0 = lds + k * ROW_BYTES + (kmajor_unit<R>(unit, k) << 5) + inner;
    const char* p1 = lds + (k + 4) * ROW_BYTES + (kmajor_unit<R>(unit, k + 4) << 5) + inner;
    s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(PO_LDS_S16X4(p0));
    s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(PO_LDS_S16X4(p1));
    union {
      struct {
        s16x4 a, b;
      } s;
      bf16x8 v;
    } u;
    u.s.a = lo;
    u.s.b = hi;
    return u.v;
  }
}

// ---- epilogue on one row-contiguous piece ----------------------------------------
// v[0..N) are consecutive n of row m starting at n.  bf16 kinds use N = 8 (16-byte accesses),
// the fp32 accumulate uses N = 4.
struct __attribute__((aligned(16))) bf16x8_t {
  bf16 v[8];
};

// `aux` is the piece of the auxiliary operand at the same place, loaded by the caller ahead of time:
// u for the GeLU backward kind, the residual (if any) for the store kinds.
template <int EPI>
__device__ __forceinline__ void epilogue_row_piece(const Epilogue& e, int m, int n, const float* v,
                                                   const bf16x8_t& aux) {
  size_t idx = (size_t)m * e.ldc + n;
  float a[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) a[i] = v[i];
  if (EPI == kEpiGeluBackward) {
    const bf16x8_t& u = aux;
    bf16x8_t o, g;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float gf, dgf;
      gelu_and_grad_f((float)u.v[i], gf, dgf);
      g.v[i] = (bf16)gf;
      o.v[i] = (bf16)(a[i] * dgf);
    }
    if (e.gelu_out) *reinterpret_cast<bf16x8_t*>(static_cast<bf16*>(e.gelu_out) + idx) = g;
    *reinterpret_cast<bf16x8_t*>(static_cast<bf16*>(e.out) + idx) = o;
    return;
  }
  if (e.bias) {
    bf16x8_t b = *reinterpret_cast<const bf16x8_t*>(static_cast<const bf16*>(e.bias) + n);
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] += (float)b.v[i];
  }
  if (e.residual) {
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] += (float)aux.v[i];
  }
  bf16x8_t o;
#pragma unroll
  for (int i = 0; i < 8; ++i) o.v[i] = (bf16)a[i];
  *reinterpret_cast<bf16x8_t*>(static_cast<bf16*>(e.out) + idx) = o;
  if (EPI == kEpiStoreGelu) {
    bf16x8_t g;
#pragma unroll
    for (int i = 0; i < 8; ++i) g.v[i] = (bf16)gelu_f((float)o.v[i]);
    *reinterpret_cast<bf16x8_t*>(static_cast<bf16*>(e.gelu_out) + idx) = g;
  }
}

// LDS stages of a tile: what fits into 160 KiB at (BM + BN) * 128 bytes per stage.
constexpr int stages_of(int wtm, int wtn) { return wtm * wtn >= 12 ? 2 : 4; }

// Tiles are walked in groups of 4 tile rows, so that a run of consecutive tile numbers is compact in both
// dimensions (the blocks of one XCD take such a run and share operand slices in that XCD's L2).
__device__ __forceinline__ void tile_of(int lin, int tiles_m, int tiles_n, int& tile_m, int& tile_n) {
  constexpr int GROUP = 4;
  int width = GROUP * tiles_n;
  int group_id = lin / width;
  int first_m = group_id * GROUP;
  int gsize = min(tiles_m - first_m, GROUP);
  tile_m = first_m + (lin % width) % gsize;
  tile_n = (lin % width) / gsize;
}

// Tells the compiler that a value is the same in every lane (it is: it derives from the block id and the kernel
// arguments only), so that it stays in scalar registers.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ const bf16* uniform(const bf16* p) {
  uintptr_t v = reinterpret_cast<uintptr_t>(p);
  unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)v), hi = __builtin_amdgcn_readfirstlane((unsigned)(v >> 32));
  return reinterpret_cast<const bf16*>(((uintptr_t)hi << 32) | lo);
}

// ---- one output tile -----------------------------------------------------------
// TA: A is [K, M] (m-contiguous).  TB: B is [K, N] (n-contiguous).  All 256 threads of the block call it with
// the same arguments; `smem` is the block's dynamic LDS (stages, then reused by the epilogue strips).
// EDGE: M x N need not be whole tiles (N a multiple of 8), nor K whole slices where TA and TB.
// OperandA: a bf16 matrix, or a Saved8Operand (TA, EDGE, two stages; lda is not used).
template <int WTM, int WTN, bool TA, bool TB, int EPI, bool EDGE, typename OperandA = const bf16*>
__device__ __forceinline__ void gemm_tile(int M, int N, int K, OperandA A, int lda,
                                          const bf16* __restrict__ B, int ldb, const Epilogue& ep, int tile_m,
                                          int tile_n, char* smem) {
  constexpr int BM = 64 * WTM, BN = 64 * WTN;
  constexpr int A_BYTES = BM * 128, B_BYTES = BN * 128;
  constexpr int STAGE = A_BYTES + B_BYTES;

  int tid = threadIdx.x, lane = tid & 63;
  int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int wm = wave >> 1, wn = wave & 1;
  int m0 = tile_m * BM, n0 = tile_n * BN;

  constexpr bool SAVED = std::is_same<OperandA, Saved8Operand>::value;
  static_assert(!SAVED || (TA && EDGE), "the form that a checkpoint's slices are woven into");
  const bf16* a_base = nullptr;
  if constexpr (!SAVED) a_base = TA ? A + m0 : A + (size_t)m0 * lda;
  const bf16* b_base = TB ? B + n0 : B + (size_t)n0 * ldb;

  f32x16 acc[WTM][WTN];
#pragma unroll
  for (int i = 0; i < WTM; ++i)
#pragma unroll
    for (int j = 0; j < WTN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

  // Pipeline.  Three streams feed the MFMAs, each running ahead of them by a fixed distance:
  //   HBM -> LDS   slice kt + NSTAGE is requested during slice kt, into the stage slice kt occupies, from the
  //                moment every wave is done reading it (the barrier below);
  //   LDS -> regs  the fragments of a k-step are read three k-steps (most of a slice) before their MFMAs, into a
  //                ring of four register buffers, so an LDS round trip is never waited for;
  //   barrier      one per slice, before k-step 1: it publishes slice kt + 1 (whose first fragments are read
  //                from k-step 1 on) and releases stage kt % NSTAGE (whose last fragments were read in k-step 0).
  // The big tiles have room for two stages, the small tile (a slice is four times shorter) gets four.
  constexpr int NSTAGE = SAVED ? 2 : stages_of(WTM, WTN);
  using LoaderA = typename std::conditional<SAVED, Saved8SliceLoader<SAVED ? BM : 128>, SliceLoader<BM, TA, EDGE>>::type;
  using LoaderB = SliceLoader<BN, TB, EDGE>;
  constexpr int PER_SLICE = LoaderA::PER_WAVE + LoaderB::PER_WAVE;  // load instructions of one wave per slice
  int nk = EDGE ? (K + kBK - 1) / kBK : K / kBK;
  LoaderA la;
  LoaderB lb;
  if constexpr (SAVED) la.init(A, m0, tid);
  else la.init(a_base, lda, M - m0, K, wave, lane);
  lb.init(b_base, ldb, N - n0, K, wave, lane);
  const unsigned lds0 = uniform((int)lds_byte(smem)) + 1024u * wave;  // this wave's piece 0 of stage 0, operand A
  // Load q (0 .. PER_SLICE - 1, A's pieces first) of the slice the loaders point at, into stage `st`.
  auto issue_load = [&](int q, unsigned st) {
    unsigned base = lds0 + st * STAGE;
    if constexpr (!SAVED) {
      if (q < LoaderA::PER_WAVE) {
        la.issue(q, base);
        return;
      }
    }
    lb.issue(q - LoaderA::PER_WAVE, base + A_BYTES);
  };
  auto next_slice = [&]() {
    la.advance();
    lb.advance();
  };
  if constexpr (SAVED) {  // slices 0 and 1 of the checkpoint, with slice 2 under way; past the end they are zeros
    LoaderA second = la;
    second.advance();
#pragma unroll
    for (int u = 0; u < LoaderA::UNITS; ++u) la.load(u);
#pragma unroll
    for (int u = 0; u < LoaderA::UNITS; ++u) second.load(u);
#pragma unroll
    for (int u = 0; u < LoaderA::UNITS; ++u) la.put(u, smem);
#pragma unroll
    for (int u = 0; u < LoaderA::UNITS; ++u) second.put(u, smem + STAGE);
    la = second;
    la.advance();
#pragma unroll
    for (int u = 0; u < LoaderA::UNITS; ++u) la.load(u);
  }
#ifdef PO_PHASE_TIMING  // measurement build only (gemm_phases.py): cycle counts of the three phases of tile (0, 0)
  const long long tim0 = __builtin_readcyclecounter(), wal0 = wall_clock64();
#endif
  {
    int ahead = min(nk, NSTAGE);
    for (int t = 0; t < ahead; ++t) {
#pragma unroll
      for (int q = 0; q < PER_SLICE; ++q) issue_load(q, t);
      if constexpr (SAVED) lb.advance();
      else next_slice();
    }
    // slice 0 has landed when at most ahead - 1 slices are still in flight
    if (ahead >= 4) wait_loads<3 * PER_SLICE>();
    else if (ahead == 3) wait_loads<2 * PER_SLICE>();
    else if (ahead == 2) wait_loads<PER_SLICE>();
    else wait_loads<0>();
  }
  __syncthreads();
#ifdef PO_PHASE_TIMING
  const long long tim1 = __builtin_readcyclecounter();
#endif

  bf16x8 fa[4][WTM], fb[4][WTN];
  // Fragments are fetched in the order a0 b0 a1 b1 ... and the MFMAs of a k-step walk the
  // (i, j) grid as a growing square, so the first MFMAs need only the first fragments fetched
  // and the fragment fetched last is needed last.
  constexpr int NFRAG = WTM + WTN;
  auto load_fragment = [&](const char* stage, int kk, int r) {  // r-th fragment of k-step kk, into buffer kk
    // (with WTM != WTN the longer operand's surplus fragments come last)
    constexpr int PAIRS = WTM < WTN ? WTM : WTN;
    bool is_a;
    int t;
    if (r < 2 * PAIRS) {
      is_a = (r & 1) == 0;
      t = r >> 1;
    } else {
      is_a = WTM > WTN;
      t = PAIRS + (r - 2 * PAIRS);
    }
    if (is_a) fa[kk][t] = read_fragment<BM, TA>(stage, wm * (WTM * 32) + t * 32, kk, lane);
    else fb[kk][t] = read_fragment<BN, TB>(stage + A_BYTES, wn * (WTN * 32) + t * 32, kk, lane);
  };
#pragma unroll
  for (int kk = 0; kk < 3; ++kk)
#pragma unroll
    for (int r = 0; r < NFRAG; ++r) load_fragment(smem, kk, r);

  // One slice: MFMAs on the fragments of stage kt % NSTAGE.  ISSUE: slice kt + NSTAGE is requested meanwhile.
  // MORE: a slice follows.  The tail slices are peeled off so that the steady-state loop body has no branches.
  //
  // Inside a k-step the three instruction streams are woven by hand, and scheduling barriers keep the compiler
  // from undoing it: behind every few MFMAs one LDS fragment read and, in k-steps 1 .. kLoadSteps, one
  // HBM -> LDS load.  A wave has a single MFMA pipe to keep busy and no other wave on its SIMD to fill in, so
  // anything issued in a clump (sixteen loads with their scalar set-up back to back) is time the matrix core
  // stands still.
  constexpr int NMFMA = WTM * WTN;
  constexpr int kLoadSteps = NSTAGE == 4 ? 3 : 2;  // measured: the small tile's eight loads spread thinner
  constexpr int LOADS_PER_STEP = (PER_SLICE + kLoadSteps - 1) / kLoadSteps;
  auto slice = [&](int kt, auto issue_tag, auto more_tag) {
    constexpr bool ISSUE = decltype(issue_tag)::value;
    constexpr bool MORE = decltype(more_tag)::value;
    unsigned st_cur = (unsigned)(kt % NSTAGE);
    char* cur = smem + st_cur * STAGE;
    char* nxt = smem + ((kt + 1) % NSTAGE) * STAGE;
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      if (MORE && kk == 1) {
        // slice kt + 1 complete (in steady state NSTAGE - 2 younger slices may stay in flight; the tail slices
        // simply wait for everything), own reads of stage kt % NSTAGE complete, then the barrier
        wait_loads<(ISSUE ? NSTAGE - 2 : 0) * PER_SLICE>();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __syncthreads();
        __builtin_amdgcn_sched_barrier(0);
      }
      int n = 0;  // MFMAs issued in this k-step
      auto after_mfma = [&]() {
        ++n;
        // the share of the other two streams that belongs behind MFMA n of NMFMA
        bool any = false;
        if (kk == 0) {
          // the last reads of this stage: all in the first half of the k-step, so that they have come back
          // when the wave waits for them at the barrier
#pragma unroll
          for (int r = (n - 1) * NFRAG * 2 / NMFMA; r < n * NFRAG * 2 / NMFMA; ++r)
            if (r < NFRAG) {
              load_fragment(cur, 3, r);
              any = true;
            }
        } else if (MORE) {
#pragma unroll
          for (int r = (n - 1) * NFRAG / NMFMA; r < n * NFRAG / NMFMA; ++r) {
            load_fragment(nxt, kk - 1, r);
            any = true;
          }
        }
        if constexpr (SAVED) {
          // A checkpoint's units first: the compiler, which knows their loads alone, waits before it uses them until no more are under way
          // than it has seen since, and the direct loads, which it does not see, must not be among those.
          constexpr int UNITS = LoaderA::UNITS, EARLY = NMFMA / 2, HALF = PER_SLICE / 2;
          if (ISSUE && kk == 1) {
            if (n == 1) la.advance();  // (the registers hold slice kt + 2; what is loaded now is kt + 3)
#pragma unroll
            for (int u = (n - 1) * UNITS / EARLY; u < n * UNITS / EARLY; ++u)
              if (u < UNITS) {
                la.put(u, cur);
                la.load(u);
                any = true;
              }
#pragma unroll
            for (int q = (n - 1 - EARLY) * HALF / (NMFMA - EARLY); q < (n - EARLY) * HALF / (NMFMA - EARLY); ++q)
              if (n > EARLY) {
                issue_load(q, st_cur);
                any = true;
              }
          } else if (ISSUE && kk == 2) {
#pragma unroll
            for (int q = (n - 1) * HALF / NMFMA; q < n * HALF / NMFMA; ++q) {
              issue_load(HALF + q, st_cur);
              any = true;
            }
          }
        } else if (ISSUE && kk >= 1 && kk <= kLoadSteps) {
#pragma unroll
          for (int q = (n - 1) * LOADS_PER_STEP / NMFMA; q < n * LOADS_PER_STEP / NMFMA; ++q) {
            int ql = (kk - 1) * LOADS_PER_STEP + q;
            if (ql < PER_SLICE) {
              issue_load(ql, st_cur);
              any = true;
            }
          }
        }
        if (any) __builtin_amdgcn_sched_barrier(0);
      };
#pragma unroll
      for (int t = 0; t < (WTM > WTN ? WTM : WTN); ++t) {  // ring t of the growing square
#pragma unroll
        for (int j = 0; j < t && j < WTN; ++j)
          if (t < WTM) {
            acc[t][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[kk][j], fa[kk][t], acc[t][j], 0, 0, 0);
            after_mfma();
          }
#pragma unroll
        for (int i = 0; i <= t && i < WTM; ++i)
          if (t < WTN) {
            acc[i][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[kk][t], fa[kk][i], acc[i][t], 0, 0, 0);
            after_mfma();
          }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if (ISSUE) {
      if constexpr (SAVED) lb.advance();
      else next_slice();
    }
  };
  {
    using T = std::true_type;
    using F = std::false_type;
    int kt = 0;
    for (; kt + NSTAGE < nk; ++kt) slice(kt, T{}, T{});
    for (; kt + 1 < nk; ++kt) slice(kt, F{}, T{});  // nothing left to request
    slice(nk - 1, F{}, F{});
  }
  __syncthreads();  // the epilogue strips reuse the operand stages
#ifdef PO_PHASE_TIMING
  const long long tim2 = __builtin_readcyclecounter();
#endif

  // Epilogue.  acc[i][j][4q + r] = C[m][n], m = strip row (lane & 31), n = 32 j + 8 q + 4 (lane >> 5) + r.
  // Each wave owns a private [32][WTN*32 + 4] fp32 strip in LDS (the operand buffers are free now).
  constexpr int STRIP_N = WTN * 32;
  constexpr int STRIP_LD = STRIP_N + 4;  // floats; the 16-byte pad staggers rows over the banks
  float* strip = reinterpret_cast<float*>(smem) + wave * (32 * STRIP_LD);
  int col = lane & 31, half = lane >> 5;
  auto inside = [&](int m, int n) { return m < M && n < N; };
  auto epilogue = [&](auto guard_tag) __attribute__((always_inline)) {
    constexpr bool GUARD = decltype(guard_tag)::value;  // the tile ends outside the result
#pragma unroll
    for (int i = 0; i < WTM; ++i) {
#pragma unroll
      for (int j = 0; j < WTN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          f32x4 v = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
          *reinterpret_cast<f32x4*>(strip + col * STRIP_LD + 32 * j + 8 * q + 4 * half) = v;
        }
      // (a wave reads back only what it wrote itself: program order is enough, no barrier)
      int mrow0 = m0 + wm * (WTM * 32) + i * 32;
      int ncol0 = n0 + wn * STRIP_N;
      if (EPI == kEpiAccumulate || EPI == kEpiStoreF32) {
        // fp32 read-modify-write of the strip: all loads of the old values are issued before the first
        // add, so that a wave keeps 16 KiB in flight instead of one access at a time.
        constexpr int LPR = STRIP_N / 4;       // lanes per row, 4 floats each
        constexpr int NIT = 32 * LPR / 64;     // wave-wide accesses per strip; piece it * 64 + lane of the strip
        static_assert(32 * LPR % 64 == 0, "strip is a whole number of wave-wide accesses");
        f32x4 old[NIT];
        float* cbase = ep.acc_f32 + (size_t)mrow0 * ep.ldc + ncol0;
#pragma unroll
        for (int it = 0; it < NIT && EPI == kEpiAccumulate; ++it) {
          int piece = it * 64 + lane;
          if (GUARD && !inside(mrow0 + piece / LPR, ncol0 + (piece % LPR) * 4)) continue;
          old[it] = *reinterpret_cast<const f32x4*>(cbase + (size_t)(piece / LPR) * ep.ldc + (piece % LPR) * 4);
        }
#pragma unroll
        for (int it = 0; it < NIT; ++it) {
          int piece = it * 64 + lane;
          int r = piece / LPR;
          int c = (piece % LPR) * 4;
          if (GUARD && !inside(mrow0 + r, ncol0 + c)) continue;
          f32x4 v = *reinterpret_cast<const f32x4*>(strip + r * STRIP_LD + c);
          *reinterpret_cast<f32x4*>(cbase + (size_t)r * ep.ldc + c) = EPI == kEpiAccumulate ? old[it] + v : v;
        }
      } else {
        constexpr int LPR = STRIP_N / 8;  // lanes per row, 8 values each
        constexpr int NIT = 32 * LPR / 64;
        static_assert(32 * LPR % 64 == 0, "strip is a whole number of wave-wide accesses");
        // the strip's pieces of u (GeLU backward) or of the residual are all requested before the first use
        bf16x8_t aux[NIT];
        const bf16* aux_src = EPI == kEpiGeluBackward ? static_cast<const bf16*>(ep.gelu_u)
                                                      : static_cast<const bf16*>(ep.residual);
        if (aux_src) {
          const bf16* abase = aux_src + (size_t)mrow0 * ep.ldc + ncol0;
#pragma unroll
          for (int it = 0; it < NIT; ++it) {
            int piece = it * 64 + lane;
            if (GUARD && !inside(mrow0 + piece / LPR, ncol0 + (piece % LPR) * 8)) continue;
            aux[it] = *reinterpret_cast<const bf16x8_t*>(abase + (size_t)(piece / LPR) * ep.ldc + (piece % LPR) * 8);
          }
        }
#pragma unroll
        for (int it = 0; it < NIT; ++it) {
          int piece = it * 64 + lane;
          int r = piece / LPR;
          int c = (piece % LPR) * 8;
          if (GUARD && !inside(mrow0 + r, ncol0 + c)) continue;
          f32x4 v0 = *reinterpret_cast<const f32x4*>(strip + r * STRIP_LD + c);
          f32x4 v1 = *reinterpret_cast<const f32x4*>(strip + r * STRIP_LD + c + 4);
          float vv[8] = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
          epilogue_row_piece<EPI>(ep, mrow0 + r, ncol0 + c, vv, aux[it]);
        }
      }
    }
  };
  if (!EDGE || (m0 + BM <= M && n0 + BN <= N)) epilogue(std::false_type());
  else epilogue(std::true_type());
#ifdef PO_PHASE_TIMING  // overwrites the first 16 bytes of the result: prologue, main loop, epilogue cycles, cycles per 10 ns
  __syncthreads();
  if (tile_m == 0 && tile_n == 0 && threadIdx.x == 0 && ep.out) {
    const long long tim3 = __builtin_readcyclecounter();
    float* dbg = reinterpret_cast<float*>(ep.out);
    dbg[0] = (float)(tim1 - tim0); dbg[1] = (float)(tim2 - tim1); dbg[2] = (float)(tim3 - tim2);
    dbg[3] = (float)(tim3 - tim0) / (float)(wall_clock64() - wal0);
  }
#endif
}

}  // namespace po
