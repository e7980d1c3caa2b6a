// A weight's gradient from the 8-bit checkpoint of its input:  dW [k, n] (+)= X^T dY,  X [rows, k] restored (saved8.h), dY [rows, n].
//
// A restored value is exact in bf16, so that the product belongs on the bf16 matrix cores whatever type dY has: in bf16 as it is, in
// fp32 as the sum of three bf16 terms (8 + 8 + 8 significant bits, cut off rather than rounded; bits under 2^-133, bf16's smallest number, are lost, so that the
// sum is exact for magnitudes from 2^-110 on), three products of exact operands with fp32 accumulators; the matrix cores take subnormal terms as they are.  X never exists in 16 bits outside LDS.
//
// The contraction is over rows, the slow index of both operands: slices of 64 rows go through registers into LDS as [64][columns] bf16 (codes are
// scaled on the way: a row's neighbouring columns have one scale), and the fragments come out of it by transposing reads.
//
// Large and long bf16 results: gemm_wide_tile.h's pipeline in tiles of 256 x 256 and 128 x 256, bound by the matrix cores (4096 rows, 4096 x 16384: 457 us, 1.20
// PFLOP/s, a plain product of 8192^3 1.34; 4096 x 2048: 71 us, 0.97).  Others: tiles of 128 and 64, bound by LDS, which a slice of 128 x 128 keeps busy for half of its 0.77 us (1733 rows, 2048 x 2048: 30 us; fp32 59), small
// ones by the chain of slices (16384 rows, 640 x 256: 18 us and 4 for the sum of the splits).
#include <algorithm>

#include "gemm_tile.h"
#include "gemm_wide_tile.h"
#include "saved8.h"

namespace po {

namespace {

struct WeightGrad {
  const uint8_t *codes, *scales;
  const void* dy;
  float* dw;
  float* partials;  // splits > 1: [splits][k][n]
  int rows, k, n, padded, ldy, ldc, accumulate;
  int tiles_m, tiles_n, split_rows;
  int vec_w;  // rows of dw start on 16-byte boundaries
};

constexpr int kSlice = 64;

// x as the sum of three bf16 numbers: its upper half, the upper half of what that leaves, and the rest.  What is not finite goes into the
// first alone.
__device__ __forceinline__ void three_terms(float x, unsigned (&t)[3]) {
  const unsigned bits = __float_as_uint(x);
  const bool finite = (bits & 0x7f800000u) != 0x7f800000u;
  t[0] = x != x ? 0x7fc0u : bits >> 16;
  const float rest = x - __uint_as_float(bits & 0xffff0000u);
  const unsigned more = __float_as_uint(rest);
  const float last = rest - __uint_as_float(more & 0xffff0000u);
  t[1] = finite ? more >> 16 : 0u;
  t[2] = finite ? __float_as_uint(last) >> 16 : 0u;
}

template <typename T>
struct Planes {
  static constexpr int N = 1;
};
template <>
struct Planes<float> {
  static constexpr int N = 3;
};

// Eight columns of a row of dY in registers, and from there into their planes.  VEC: 16-byte pieces that are all there or not at all; loads go through
// a buffer that ends with the slice's rows, and a piece that is not there is asked for past its end.
template <typename T, bool VEC>
struct Eight {
  static constexpr int V = 8 * sizeof(T) / 16;  // 16-byte pieces
  u32x4 v[V];
  // at: bytes from the slice's first; held: columns that there are
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t slice, int at, int held) {
    constexpr int E = 16 / sizeof(T);
#pragma unroll
    for (int i = 0; i < V; ++i)
      v[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(slice, i * E < held ? at + 16 * i : (int)kOutOfBuffer, 0, 0));
  }
  // From rows on no 16-byte boundaries: whole vectors from wherever they start, past the end of a row too (what is there meets only results that are not
  // written), and single values at the end of the last row (1512 rows, 7824 x 285: 33 us, with single values everywhere 69).
  // there: whether dY has the row and the first column; left: bytes from the slice's first to dY's last.
  __device__ __forceinline__ void load(const uint8_t* slice, int at, int held, bool there, int64_t left) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = u32x4{0u, 0u, 0u, 0u};
    if (!there) return;
    if (at + (int64_t)(8 * sizeof(T)) <= left) {
      __builtin_memcpy(v, slice + at, 8 * sizeof(T));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < held) {
          if constexpr (sizeof(T) == 4) v[i / 4][i % 4] = reinterpret_cast<const unsigned*>(slice + at)[i];
          else v[0][i / 2] |= (unsigned)reinterpret_cast<const uint16_t*>(slice + at)[i] << (16 * (i % 2));
        }
    }
  }
  // plane pl's 16 bytes
  __device__ __forceinline__ void planes(u32x4 (&out)[Planes<T>::N]) const {
    if constexpr (sizeof(T) == 2) {
      out[0] = v[0];
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        unsigned a[3], b[3];
        three_terms(__uint_as_float(v[i / 2][2 * (i % 2)]), a);
        three_terms(__uint_as_float(v[i / 2][2 * (i % 2) + 1]), b);
#pragma unroll
        for (int pl = 0; pl < 3; ++pl) out[pl][i] = a[pl] | b[pl] << 16;
      }
    }
  }
};

template <int TILE>
__device__ __forceinline__ int eight_at(int row, int eight) {  // byte of eight columns in a slice, as fragment() reads it
  constexpr int MASK = TILE >= 128 ? 7 : TILE / 16 - 1;
  return row * (2 * TILE) + (((eight >> 1) ^ (row & MASK)) << 5) + ((eight & 1) << 4);
}

// TILE x TILE results a block, WAVES waves in two rows (128: eight of 64 x 32, two to a SIMD; 1733 rows, 2048 x 2048, with four of 64 x 64 35 us, so 32).
// AHEAD slices are on their way into registers while one is computed: a slice is
// 512 cycles of MFMAs (TILE 128), memory a thousand and more away.
template <typename T, int TILE, bool VEC, int AHEAD, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void weight_grad_saved8_kernel(WeightGrad p) {
  extern __shared__ __align__(16) char smem[];
  constexpr int PLANES = Planes<T>::N, EIGHTS = TILE / 8, PER = kSlice * EIGHTS / (64 * WAVES);
  constexpr int WM = TILE / 64, WN = 2 * TILE / (32 * WAVES);  // MFMA tiles of a wave
  constexpr int X_BYTES = kSlice * TILE * 2, STAGE = X_BYTES * (1 + PLANES);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave / (WAVES / 2), wn = wave % (WAVES / 2);
  int tile_m, tile_n;
  place_of_tile(tile_of_block(), p.tiles_m, p.tiles_n, tile_m, tile_n);
  const int m0 = tile_m * TILE, n0 = tile_n * TILE;
  const int first = blockIdx.y * p.split_rows, end = min(p.rows, first + p.split_rows);

  // Neighbouring lanes take neighbouring eights: sixteen bytes each into LDS, next to each other (sixteen columns a lane, 32 bytes apart, cost 16
  // cycles of bank conflicts a write).
  uint2 codes[AHEAD][PER];
  unsigned byte[AHEAD][PER];
  Eight<T, VEC> y[AHEAD][PER];
  int x_at[PER], y_at[PER], y_held[PER], lds_at[PER];
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int q = u * (64 * WAVES) + tid, row = q / EIGHTS, eight = q % EIGHTS, m = m0 + 8 * eight, n = n0 + 8 * eight;
    x_at[u] = m < p.padded ? row * p.padded + m : -1;
    y_at[u] = (row * p.ldy + n) * (int)sizeof(T);
    y_held[u] = p.n - n;
    lds_at[u] = eight_at<TILE>(row, eight);
  }
  auto load = [&](int slot, int r0) {  // rows from `end` on read as zeros
    const int rows = max(0, min(kSlice, end - r0));
    const int64_t at = (int64_t)r0 * p.padded;
    const __amdgpu_buffer_rsrc_t x = buffer_resource(p.codes + at, rows * p.padded);
    const __amdgpu_buffer_rsrc_t scale = buffer_resource(p.scales + (at >> 5), rows * p.padded >> 5);
    const uint8_t* dy = (const uint8_t*)p.dy + (int64_t)r0 * p.ldy * (int)sizeof(T);
    const __amdgpu_buffer_rsrc_t slice = buffer_resource(dy, rows * p.ldy * (int)sizeof(T));
    const int64_t left = ((int64_t)(p.rows - 1 - r0) * p.ldy + p.n) * (int)sizeof(T);
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const auto q = __builtin_amdgcn_raw_buffer_load_b64(x, x_at[u] >= 0 ? x_at[u] : (int)kOutOfBuffer, 0, 0);
      codes[slot][u] = make_uint2(q[0], q[1]);
      byte[slot][u] = __builtin_amdgcn_raw_buffer_load_b8(scale, x_at[u] >= 0 ? x_at[u] >> 5 : (int)kOutOfBuffer, 0, 0);
      if constexpr (VEC)
        y[slot][u].load(slice, y_at[u], y_held[u]);
      else
        y[slot][u].load(dy, y_at[u], y_held[u], (u * (64 * WAVES) + tid) / EIGHTS < rows && y_held[u] > 0, left);
    }
  };
  auto stage = [&](int slot, int u, char* lds) {
    u32x4 planes[PLANES];
    y[slot][u].planes(planes);
    *reinterpret_cast<u32x4*>(lds + lds_at[u]) = widen8(codes[slot][u], byte[slot][u]);
#pragma unroll
    for (int pl = 0; pl < PLANES; ++pl) *reinterpret_cast<u32x4*>(lds + X_BYTES * (1 + pl) + lds_at[u]) = planes[pl];
  };
  bf16x8 a[2][WM], b[2][PLANES][WN];
  auto fragments = [&](int kk, const char* lds) {
#pragma unroll
    for (int w = 0; w < WM; ++w) a[kk % 2][w] = fragment<TILE, true>((const bf16*)nullptr, lds, 32 * (wm * WM + w), kk, lane);
#pragma unroll
    for (int pl = 0; pl < PLANES; ++pl)
#pragma unroll
      for (int w = 0; w < WN; ++w)
        b[kk % 2][pl][w] = fragment<TILE, true>((const bf16*)nullptr, lds + X_BYTES * (1 + pl), 32 * (wn * WN + w), kk, lane);
  };

  f32x16 acc[WM][WN];
#pragma unroll
  for (int i = 0; i < WM; ++i)
#pragma unroll
    for (int j = 0; j < WN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

  // Slice s lies in LDS stage s % 2 while it is computed; slot s % AHEAD holds a later one on its way.
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) load(i, first + i * kSlice);
#pragma unroll
  for (int u = 0; u < PER; ++u) stage(0, u, smem);
  load(0, first + AHEAD * kSlice);
  int turn = 0;
  // (whole rounds of slices: a way out between them would make the compiler wait for all loads at each; behind `end` come zeros)
  for (int r0 = first; r0 < end; r0 += AHEAD * kSlice) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int at = r0 + i * kSlice;
      __syncthreads();
      const char* lds = smem + turn * STAGE;
      turn ^= 1;
      const int slot = (i + 1) % AHEAD;
      fragments(0, lds);
#pragma unroll
      for (int kk = 0; kk < kSlice / 16; ++kk) {  // the next step's fragments, this step's products, a share of the next slice
        if (kk + 1 < kSlice / 16) fragments(kk + 1, lds);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int pl = PLANES - 1; pl >= 0; --pl)  // the smallest terms first
#pragma unroll
          for (int w = 0; w < WM; ++w)
#pragma unroll
            for (int j = 0; j < WN; ++j) acc[w][j] = multiply(b[kk % 2][pl][j], a[kk % 2][w], acc[w][j]);
        if (kk < PER) stage(slot, kk, smem + turn * STAGE);  // (behind the last slice zeros, which nothing reads)
        __builtin_amdgcn_sched_barrier(0);
      }
      load(slot, at + (1 + AHEAD) * kSlice);
    }
  }
  __syncthreads();  // the strips reuse the stages

  // acc[i][j][4 q + r] = dW[m][n], m = strip row lane % 32, n = 32 j + 8 q + 4 (lane / 32) + r: strips of 32 rows through LDS, so that a row of
  // results is written by neighbouring lanes.
  constexpr int WIDE = 32 * WN, LD = WIDE + 4, LANES = WIDE / 4, STEPS = 32 * LANES / 64;
  float* strip = reinterpret_cast<float*>(smem) + wave * (32 * LD);
  const bool split = gridDim.y > 1;
  float* out = split ? p.partials + (int64_t)blockIdx.y * p.k * p.n : p.dw;
  const int ld = split ? p.n : p.ldc;
  const bool vec = split ? p.n % 4 == 0 : p.vec_w, add = !split && p.accumulate;
#pragma unroll
  for (int i = 0; i < WM; ++i) {
#pragma unroll
    for (int j = 0; j < WN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4 v = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        *reinterpret_cast<f32x4*>(strip + (lane & 31) * LD + 32 * j + 8 * q + 4 * (lane >> 5)) = v;
      }
    // (a wave reads back only what it wrote itself: program order is enough, no barrier)
    // What is added to is read first, all of it, so that its round trips are one.
    f32x4 old[STEPS];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int piece = s * 64 + lane, m = m0 + 32 * (wm * WM + i) + piece / LANES, n = n0 + wn * WIDE + piece % LANES * 4;
      old[s] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (!add || m >= p.k || n >= p.n) continue;
      const float* from = out + (int64_t)m * ld + n;
      if (vec && n + 4 <= p.n) {
        old[s] = *reinterpret_cast<const f32x4*>(from);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (n + e < p.n) old[s][e] = from[e];
      }
    }
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int piece = s * 64 + lane, r = piece / LANES, c = piece % LANES * 4;
      const int m = m0 + 32 * (wm * WM + i) + r, n = n0 + wn * WIDE + c;
      if (m >= p.k || n >= p.n) continue;
      const f32x4 v = old[s] + *reinterpret_cast<const f32x4*>(strip + r * LD + c);
      float* to = out + (int64_t)m * ld + n;
      if (vec && n + 4 <= p.n) {
        *reinterpret_cast<f32x4*>(to) = v;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (n + e < p.n) to[e] = v[e];
      }
    }
  }
}

// 64 WTM x 64 WTN results a block, in gemm_tile's pipeline: dY's slices straight into LDS, the checkpoint's through registers.
template <int WTM, int WTN, int EPI>
__global__ __launch_bounds__(256) void weight_grad_saved8_wide_kernel(WeightGrad p) {
  extern __shared__ __align__(16) char smem[];
  const int n_tiles = p.tiles_m * p.tiles_n, pid = blockIdx.x;
  const int lin = n_tiles % 8 == 0 ? (pid % 8) * (n_tiles / 8) + pid / 8 : pid;
  int tile_m, tile_n;
  tile_of(lin, p.tiles_m, p.tiles_n, tile_m, tile_n);
  const int first = blockIdx.y * p.split_rows, rows = min(p.rows - first, p.split_rows);
  const int64_t at = (int64_t)first * p.padded;
  const Saved8Operand x{p.codes + at, p.scales + (at >> 5), p.padded, rows};
  Epilogue ep = {};
  ep.acc_f32 = gridDim.y > 1 ? p.partials + (int64_t)blockIdx.y * p.k * p.n : p.dw;
  ep.ldc = gridDim.y > 1 ? p.n : p.ldc;
  gemm_tile<WTM, WTN, true, true, EPI, true>(p.k, p.n, rows, x, 0, (const bf16*)p.dy + (int64_t)first * p.ldy, p.ldy, ep, tile_m, tile_n, smem);
}

// dW (+)= the splits' partial results, in a fixed order: GROUPS threads share four results, each every GROUPS-th split's, four loads under way.
// One for up to eight splits (4096 rows, 2048 x 1024, two splits: 37 us, eight threads 41), eight for more (16384 rows, 256 x 256, 32 splits: 16.3 us, one
// thread, a load at a time, 31).
template <bool VEC, int GROUPS>  // VEC: the splits start on 16-byte boundaries
__global__ __launch_bounds__(256) void weight_grad_sum_kernel(WeightGrad p, int splits) {
  constexpr int LANES = 256 / GROUPS;
  __shared__ f32x4 part[GROUPS][LANES];
  const int64_t total = (int64_t)p.k * p.n;
  const int x = threadIdx.x % LANES, y = threadIdx.x / LANES;
  const int64_t i = ((int64_t)blockIdx.x * LANES + x) * 4;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  auto value = [&](int k) {
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (k >= splits || i >= total) return v;
    const float* from = p.partials + k * total + i;
    if (VEC) return *reinterpret_cast<const f32x4*>(from);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = i + e < total ? from[e] : 0.f;
    return v;
  };
  for (int k = y; k < splits; k += 4 * GROUPS) {
    f32x4 v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = value(k + GROUPS * u);
    sum += (v[0] + v[1]) + (v[2] + v[3]);
  }
  if (GROUPS > 1) {
    part[y][x] = sum;
    __syncthreads();
    if (y) return;
#pragma unroll
    for (int g = 1; g < GROUPS; ++g) sum += part[g][x];
  }
  if (i >= total) return;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (i + e < total) {
      const int64_t m = (i + e) / p.n, n = i + e - m * p.n;
      float* to = p.dw + m * p.ldc + n;
      *to = p.accumulate ? *to + sum[e] : sum[e];
    }
}

constexpr int kMaxRows = 1 << 25, kMaxWidth = 1 << 20, kMaxPitch = 1 << 22;  // a slice's offsets fit 31 bits
constexpr int64_t kMaxTiles = 1 << 21;

// The tiles there are: rows of dW (k), columns, whether of the wide kernel, blocks of a round, us a slice of a full round in bf16 and fp32 (measured).
// 4096 rows, 4096 x 2048: 128 x 256 73 us, 128 x 128 94 (256 x 128, which the checkpoint's conversions slow down, 80).
struct Tile {
  int m, n;
  bool wide;
  int round;
  double slice_bf16, slice_f32;
};
constexpr Tile kTiles[] = {{64, 64, false, 512, 0.55, 1.5}, {128, 128, false, 256, 0.77, 1.9}, {128, 256, true, 256, 1.05, 0}, {256, 256, true, 256, 1.7, 0}};
struct Form {
  int tile, tiles_m, tiles_n, splits, split_rows;  // tile: of kTiles
};
int64_t tiles_of(const Tile& t, int k, int n) { return (int64_t)ceil_div(k, t.m) * ceil_div(n, t.n); }
// At most so many splits: a round of blocks, four slices each at least.
int most_splits(const Tile& t, int rows, int k, int n) {
  return (int)std::max<int64_t>(1, std::min<int64_t>(ceil_div(rows, 4 * kSlice), t.round / tiles_of(t, k, n)));
}
// The tile and the splits that should take least: rounds of blocks, each its slices one after another, a split's partial results written and
// read again (the sum 3 us and 8 bytes a partial result at 5 TB/s).
Form form_of(int dtype, int rows, int k, int n, bool wide) {
  Form best = {};
  double least = 0;
  for (int tile = 0; tile < 4; ++tile) {
    const Tile& t = kTiles[tile];
    if (t.wide && !wide) continue;
    const int64_t tiles = tiles_of(t, k, n);
    for (int splits = most_splits(t, rows, k, n);; splits /= 2) {
      const int each = ceil_div(ceil_div(rows, splits), kSlice);  // slices
      const double time = (double)ceil_div64(tiles * splits, t.round) * (each + 4) * (dtype == kF32 ? t.slice_f32 : t.slice_bf16) +
                          (splits > 1 ? 3 + splits * (double)k * n * 8 / 5e6 : 0);
      if (least == 0 || time < least) {
        least = time;
        best = Form{tile, ceil_div(k, t.m), ceil_div(n, t.n), ceil_div(rows, each * kSlice), each * kSlice};
      }
      if (splits <= 1) break;
    }
  }
  return best;
}
bool sizes_ok(int rows, int k, int n) {
  return rows >= 1 && rows <= kMaxRows && k >= 1 && k <= kMaxWidth && n >= 1 && n <= kMaxWidth &&
         (int64_t)ceil_div(k, 128) * ceil_div(n, 128) <= kMaxTiles && saved8_codes(rows, k) / 8 <= kMaxSaved8Chunks;
}

template <typename T, int TILE, bool VEC>
bool launch(const WeightGrad& p, const Form& f, hipStream_t stream) {
  constexpr int BYTES = 2 * kSlice * TILE * 2 * (1 + Planes<T>::N), AHEAD = 2, WAVES = TILE == 128 ? 8 : 4;
  static LdsLimit limit;
  if (!limit.allow(weight_grad_saved8_kernel<T, TILE, VEC, AHEAD, WAVES>, BYTES)) return false;
  weight_grad_saved8_kernel<T, TILE, VEC, AHEAD, WAVES><<<dim3((unsigned)(f.tiles_m * f.tiles_n), (unsigned)f.splits), 64 * WAVES, BYTES, stream>>>(p);
  return launch_ok("weight_grad_saved8_kernel");
}
template <typename T>
bool launch(const WeightGrad& p, const Form& f, bool vec, hipStream_t stream) {
  return (f.tile == 1 ? (vec ? launch<T, 128, true> : launch<T, 128, false>) : (vec ? launch<T, 64, true> : launch<T, 64, false>))(p, f, stream);
}
template <int WTM, int WTN, int EPI>
bool launch_wide(const WeightGrad& p, const Form& f, hipStream_t stream) {
  constexpr int BYTES = 2 * 64 * (WTM + WTN) * 128;
  static LdsLimit limit;
  if (!limit.allow(weight_grad_saved8_wide_kernel<WTM, WTN, EPI>, BYTES)) return false;
  weight_grad_saved8_wide_kernel<WTM, WTN, EPI><<<dim3((unsigned)(f.tiles_m * f.tiles_n), (unsigned)f.splits), 256, BYTES, stream>>>(p);
  return launch_ok("weight_grad_saved8_wide_kernel");
}
template <int EPI>
bool launch_wide(const WeightGrad& p, const Form& f, hipStream_t stream) {
  return (f.tile == 2 ? launch_wide<2, 4, EPI> : launch_wide<4, 4, EPI>)(p, f, stream);
}

}  // namespace

size_t weight_grad_saved8_workspace(int dtype, int rows, int k, int n) {
  if (!sizes_ok(rows, k, n)) return 0;
  // for the most splits that any tile may take, so that a workspace for more rows serves fewer
  int most = 1;
  for (const Tile& t : kTiles)
    if (!t.wide || dtype == kBF16) most = std::max(most, most_splits(t, rows, k, n));
  return most > 1 ? (size_t)most * k * n * sizeof(float) : 0;
}

bool weight_grad_saved8(int dtype, const void* saved_x, const void* dy, int ldy, float* dw, int ldc, int accumulate, void* workspace, int rows,
                        int k, int n, hipStream_t stream) {
  const char* what = "weight_grad_saved8";
  const int size = dtype == kF32 ? 4 : 2;
  if (!sizes_ok(rows, k, n) || ldy < n || ldy > kMaxPitch || ldc < n || (accumulate != 0 && accumulate != 1)) {
    set_error("%s: rows=%d k=%d n=%d ldy=%d ldc=%d accumulate=%d (1 to %d rows, k and n 1 to %d, rows x k at most %lld, at most %lld tiles of 128 x 128, ldy and "
              "ldc at least n, ldy at most %d, accumulate 0 or 1)", what, rows, k, n, ldy, ldc, accumulate, kMaxRows, kMaxWidth,
              (long long)kMaxSaved8Chunks * 8, (long long)kMaxTiles, kMaxPitch);
    return false;
  }
  const size_t needed = weight_grad_saved8_workspace(dtype, rows, k, n);
  if (!saved_x || !dy || !dw || (uintptr_t)saved_x % 16 != 0 || (uintptr_t)dy % size != 0 || (uintptr_t)dw % 4 != 0 ||
      (needed > 0 && (!workspace || (uintptr_t)workspace % 16 != 0))) {
    set_error("%s: saved_x=%p dy=%p dw=%p workspace=%p (a NULL pointer, or one not aligned: 16 bytes, workspace too, dy and dw to their type)",
              what, saved_x, dy, (void*)dw, workspace);
    return false;
  }
  const uint64_t x_bytes = saved8_bytes(rows, k), y_bytes = ((uint64_t)(rows - 1) * ldy + n) * size, w_bytes = ((uint64_t)(k - 1) * ldc + n) * 4;
  if (overlap(dw, w_bytes, saved_x, x_bytes) || overlap(dw, w_bytes, dy, y_bytes) ||
      (needed > 0 && (overlap(workspace, needed, saved_x, x_bytes) || overlap(workspace, needed, dy, y_bytes) || overlap(workspace, needed, dw, w_bytes)))) {
    set_error("%s: dw or workspace overlaps what is read or the other", what);
    return false;
  }
  const bool vec_y = (uintptr_t)dy % 16 == 0 && (rows == 1 || (int64_t)ldy * size % 16 == 0);
  const bool vec_w = (uintptr_t)dw % 16 == 0 && (k == 1 || ldc % 4 == 0);
  // The wide kernel: bf16, whole eights of columns on 16-byte boundaries, dy within 2 GiB.
  const bool wide = dtype == kBF16 && vec_y && vec_w && n % 8 == 0 && ((int64_t)rows + 256) * ldy * 2 <= INT32_MAX;
  const Form f = form_of(dtype, rows, k, n, wide);
  WeightGrad p = {};
  p.codes = (const uint8_t*)saved_x;
  p.scales = p.codes + saved8_codes(rows, k);
  p.dy = dy;
  p.dw = dw;
  p.partials = (float*)workspace;
  p.rows = rows;
  p.k = k;
  p.n = n;
  p.padded = (int)saved8_cols(k);
  p.ldy = ldy;
  p.ldc = ldc;
  p.accumulate = accumulate;
  p.tiles_m = f.tiles_m;
  p.tiles_n = f.tiles_n;
  p.split_rows = f.split_rows;
  p.vec_w = vec_w;
  const bool done = kTiles[f.tile].wide ? (accumulate && f.splits == 1 ? launch_wide<kEpiAccumulate>(p, f, stream) : launch_wide<kEpiStoreF32>(p, f, stream))
                    : dtype == kF32     ? launch<float>(p, f, vec_y && n % 4 == 0, stream)
                                        : launch<bf16>(p, f, vec_y && n % 8 == 0, stream);
  if (!done) return false;
  if (f.splits == 1) return true;
  const bool many = f.splits > 8, whole = (int64_t)k * n % 4 == 0;
  const unsigned blocks = (unsigned)ceil_div64((int64_t)k * n, many ? 128 : 1024);
  auto sum = many ? (whole ? weight_grad_sum_kernel<true, 8> : weight_grad_sum_kernel<false, 8>)
                  : (whole ? weight_grad_sum_kernel<true, 1> : weight_grad_sum_kernel<false, 1>);
  sum<<<blocks, 256, 0, stream>>>(p, f.splits);
  return launch_ok("weight_grad_sum_kernel");
}

}  // namespace po
