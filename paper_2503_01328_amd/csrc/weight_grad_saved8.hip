// A weight's gradient from the 8-bit checkpoint of its input:  dW [k, n] (+)= X^T dY,  X [rows, k] restored (saved8.h), dY [rows, n].
//
// A restored value is exact in bf16, so that the product belongs on the bf16 matrix cores whatever type dY has: in bf16 as it is, in
// fp32 as the sum of three bf16 terms (8 + 8 + 8 significant bits, cut off rather than rounded, which makes the sum exact), three products of
// exact operands with fp32 accumulators.  X never exists in 16 bits outside LDS.
//
// The contraction is over rows, the slow index of both operands: slices of 64 rows go through registers into LDS as [64][columns] bf16 (codes are
// scaled on the way, sixteen columns of a row have one scale), and the fragments come out of it by transposing reads.
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
  int vec_y, vec_w;  // rows of dy, of dw start on 16-byte boundaries
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

// Sixteen columns of a row of dY in registers, and from there into their planes.
template <typename T>
struct Sixteen {
  static constexpr int V = 16 * sizeof(T) / 16;  // 16-byte pieces
  u32x4 v[V];
  __device__ __forceinline__ void load(const T* p, int held, bool vec) {
    if (vec && held >= 16) {
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(p) + 16 * i);
    } else {
      union {
        T e[16];
        u32x4 u[V];
      } w;
#pragma unroll
      for (int i = 0; i < 16; ++i) w.e[i] = i < held ? p[i] : (T)0.f;
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = w.u[i];
    }
  }
  // plane pl's 32 bytes
  __device__ __forceinline__ void planes(u32x4 (&out)[Planes<T>::N][2]) const {
    if constexpr (sizeof(T) == 2) {
      out[0][0] = v[0];
      out[0][1] = v[1];
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        unsigned a[3], b[3];
        three_terms(__uint_as_float(v[i / 2][2 * (i % 2)]), a);
        three_terms(__uint_as_float(v[i / 2][2 * (i % 2) + 1]), b);
#pragma unroll
        for (int pl = 0; pl < 3; ++pl) out[pl][i / 4][i % 4] = a[pl] | b[pl] << 16;
      }
    }
  }
};

template <int TILE>
__device__ __forceinline__ int unit_at(int row, int unit) {  // byte of a unit of sixteen columns in a slice, as fragment() reads it
  constexpr int MASK = TILE >= 128 ? 7 : TILE / 16 - 1;
  return row * (2 * TILE) + ((unit ^ (row & MASK)) << 5);
}

// TILE x TILE results a block, four waves of TILE / 2 x TILE / 2.
template <typename T, int TILE>
__global__ __launch_bounds__(256) void weight_grad_saved8_kernel(WeightGrad p) {
  extern __shared__ __align__(16) char smem[];
  constexpr int PLANES = Planes<T>::N, UNITS = TILE / 16, PER = kSlice * UNITS / 256, WT = TILE / 64;
  constexpr int X_BYTES = kSlice * TILE * 2, STAGE = X_BYTES * (1 + PLANES);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave >> 1, wn = wave & 1;
  int tile_m, tile_n;
  place_of_tile(tile_of_block(), p.tiles_m, p.tiles_n, tile_m, tile_n);
  const int m0 = tile_m * TILE, n0 = tile_n * TILE;
  const int first = blockIdx.y * p.split_rows, end = min(p.rows, first + p.split_rows);

  u32x4 codes[PER];
  unsigned byte[PER];
  Sixteen<T> y[PER];
  auto load = [&](int r0) {
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const int q = u * 256 + tid, row = r0 + q / UNITS, unit = q % UNITS;
      const bool there = row < end;
      const int m = m0 + 16 * unit, n = n0 + 16 * unit;
      codes[u] = u32x4{0, 0, 0, 0};
      byte[u] = 127;
      if (there && m < p.padded) {
        const int64_t at = (int64_t)row * p.padded + m;
        codes[u] = *reinterpret_cast<const u32x4*>(p.codes + at);
        byte[u] = p.scales[at >> 5];
      }
      y[u].load((const T*)p.dy + (int64_t)row * p.ldy + n, there ? p.n - n : 0, p.vec_y);
    }
  };
  auto stage = [&](char* lds) {
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const int q = u * 256 + tid, at = unit_at<TILE>(q / UNITS, q % UNITS);
      u32x4 w[2], planes[PLANES][2];
      Saved8SliceLoader<128>::widen16(codes[u], byte[u], w);
      y[u].planes(planes);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        *reinterpret_cast<u32x4*>(lds + at + 16 * h) = w[h];
#pragma unroll
        for (int pl = 0; pl < PLANES; ++pl) *reinterpret_cast<u32x4*>(lds + X_BYTES * (1 + pl) + at + 16 * h) = planes[pl][h];
      }
    }
  };

  f32x16 acc[WT][WT];
#pragma unroll
  for (int i = 0; i < WT; ++i)
#pragma unroll
    for (int j = 0; j < WT; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

  load(first);
  stage(smem);
  int turn = 0;
  for (int r0 = first; r0 < end; r0 += kSlice) {
    const bool more = r0 + kSlice < end;
    if (more) load(r0 + kSlice);
    __syncthreads();
    const char* lds = smem + turn * STAGE;
#pragma unroll
    for (int kk = 0; kk < kSlice / 16; ++kk) {
      bf16x8 a[WT], b[WT];
#pragma unroll
      for (int i = 0; i < WT; ++i) a[i] = fragment<TILE, true>((const bf16*)nullptr, lds, wm * (TILE / 2) + 32 * i, kk, lane);
#pragma unroll
      for (int pl = PLANES - 1; pl >= 0; --pl) {  // the smallest terms first
#pragma unroll
        for (int j = 0; j < WT; ++j)
          b[j] = fragment<TILE, true>((const bf16*)nullptr, lds + X_BYTES * (1 + pl), wn * (TILE / 2) + 32 * j, kk, lane);
#pragma unroll
        for (int i = 0; i < WT; ++i)
#pragma unroll
          for (int j = 0; j < WT; ++j) acc[i][j] = multiply(b[j], a[i], acc[i][j]);
      }
    }
    turn ^= 1;
    if (more) stage(smem + turn * STAGE);
  }
  __syncthreads();  // the strips reuse the stages

  // acc[i][j][4 q + r] = dW[m][n], m = strip row lane % 32, n = 32 j + 8 q + 4 (lane / 32) + r: strips of 32 rows through LDS, so that a row of
  // results is written by neighbouring lanes.
  constexpr int WIDE = TILE / 2, LD = WIDE + 4, LANES = WIDE / 4, STEPS = 32 * LANES / 64;
  float* strip = reinterpret_cast<float*>(smem) + wave * (32 * LD);
  const bool split = gridDim.y > 1;
  float* out = split ? p.partials + (int64_t)blockIdx.y * p.k * p.n : p.dw;
  const int ld = split ? p.n : p.ldc;
  const bool vec = split ? p.n % 4 == 0 : p.vec_w, add = !split && p.accumulate;
#pragma unroll
  for (int i = 0; i < WT; ++i) {
#pragma unroll
    for (int j = 0; j < WT; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4 v = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        *reinterpret_cast<f32x4*>(strip + (lane & 31) * LD + 32 * j + 8 * q + 4 * (lane >> 5)) = v;
      }
    // (a wave reads back only what it wrote itself: program order is enough, no barrier)
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int piece = s * 64 + lane, r = piece / LANES, c = piece % LANES * 4;
      const int m = m0 + wm * WIDE + 32 * i + r, n = n0 + wn * WIDE + c;
      if (m >= p.k || n >= p.n) continue;
      const f32x4 v = *reinterpret_cast<const f32x4*>(strip + r * LD + c);
      float* to = out + (int64_t)m * ld + n;
      if (vec && n + 4 <= p.n) {
        f32x4* t = reinterpret_cast<f32x4*>(to);
        *t = add ? *t + v : v;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (n + e < p.n) to[e] = add ? to[e] + v[e] : v[e];
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

// dW (+)= the splits' partial results, in their order.
__global__ __launch_bounds__(256) void weight_grad_sum_kernel(WeightGrad p, int splits) {
  const int64_t total = (int64_t)p.k * p.n;
  for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < total; i += (int64_t)gridDim.x * 1024) {
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    const bool whole = total % 4 == 0;  // then every split's start is a 16-byte boundary
    for (int k = 0; k < splits; ++k) {
      const float* from = p.partials + k * total + i;
      if (whole) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(from);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] += v[e];
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] += i + e < total ? from[e] : 0.f;
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + e < total) {
        const int64_t m = (i + e) / p.n, n = i + e - m * p.n;
        float* to = p.dw + m * p.ldc + n;
        *to = p.accumulate ? *to + s[e] : s[e];
      }
  }
}

constexpr int kMaxRows = 1 << 25, kMaxWidth = 1 << 20;
constexpr int64_t kMaxTiles = 1 << 23;

struct Form {
  int tile, tiles_m, tiles_n, splits, split_rows;  // tile: 64, 128, or 256: the wide kernel
};
Form form_of(int rows, int k, int n, bool wide) {
  Form f;
  if (wide && (int64_t)ceil_div(k, 256) * ceil_div(n, 256) >= 128) {
    f = Form{256, ceil_div(k, 256), ceil_div(n, 256), 1, rows};
    return f;
  }
  f.tile = (int64_t)ceil_div(k, 128) * ceil_div(n, 128) >= 128 ? 128 : 64;
  f.tiles_m = ceil_div(k, f.tile);
  f.tiles_n = ceil_div(n, f.tile);
  const int64_t tiles = (int64_t)f.tiles_m * f.tiles_n;
  f.splits = (int)std::max<int64_t>(1, std::min<int64_t>(ceil_div(rows, 4 * kSlice), 512 / std::max<int64_t>(tiles, 1)));
  f.split_rows = ceil_div(ceil_div(rows, f.splits), kSlice) * kSlice;
  f.splits = ceil_div(rows, f.split_rows);
  return f;
}
bool sizes_ok(int rows, int k, int n) {
  return rows >= 1 && rows <= kMaxRows && k >= 1 && k <= kMaxWidth && n >= 1 && n <= kMaxWidth &&
         (int64_t)ceil_div(k, 128) * ceil_div(n, 128) <= kMaxTiles;
}

template <typename T, int TILE>
bool launch(const WeightGrad& p, const Form& f, hipStream_t stream) {
  constexpr int BYTES = 2 * kSlice * TILE * 2 * (1 + Planes<T>::N);
  static LdsLimit limit;
  if (!limit.allow(weight_grad_saved8_kernel<T, TILE>, BYTES)) return false;
  weight_grad_saved8_kernel<T, TILE><<<dim3((unsigned)(f.tiles_m * f.tiles_n), (unsigned)f.splits), 256, BYTES, stream>>>(p);
  return launch_ok("weight_grad_saved8_kernel");
}
template <int EPI>
bool launch_wide(const WeightGrad& p, const Form& f, hipStream_t stream) {
  constexpr int BYTES = stages_of(4, 4) * (256 + 256) * 128;
  static LdsLimit limit;
  if (!limit.allow(weight_grad_saved8_wide_kernel<4, 4, EPI>, BYTES)) return false;
  weight_grad_saved8_wide_kernel<4, 4, EPI><<<dim3((unsigned)(f.tiles_m * f.tiles_n), (unsigned)f.splits), 256, BYTES, stream>>>(p);
  return launch_ok("weight_grad_saved8_wide_kernel");
}

}  // namespace

size_t weight_grad_saved8_workspace(int dtype, int rows, int k, int n) {
  if (!sizes_ok(rows, k, n)) return 0;
  const Form f = form_of(rows, k, n, false);
  return f.splits > 1 ? (size_t)f.splits * k * n * sizeof(float) : 0;
}

bool weight_grad_saved8(int dtype, const void* saved_x, const void* dy, int ldy, float* dw, int ldc, int accumulate, void* workspace, int rows,
                        int k, int n, hipStream_t stream) {
  const char* what = "weight_grad_saved8";
  const int size = dtype == kF32 ? 4 : 2;
  if (!sizes_ok(rows, k, n) || ldy < n || ldc < n || (accumulate != 0 && accumulate != 1)) {
    set_error("%s: rows=%d k=%d n=%d ldy=%d ldc=%d accumulate=%d (1 to %d rows, k and n 1 to %d, %lld tiles of 128 x 128, ldy and ldc at "
              "least n, accumulate 0 or 1)", what, rows, k, n, ldy, ldc, accumulate, kMaxRows, kMaxWidth, (long long)kMaxTiles);
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
  const Form f = form_of(rows, k, n, wide);
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
  p.vec_y = vec_y;
  p.vec_w = vec_w;
  if (f.tile == 256) return accumulate ? launch_wide<kEpiAccumulate>(p, f, stream) : launch_wide<kEpiStoreF32>(p, f, stream);
  auto run = dtype == kF32 ? (f.tile == 128 ? launch<float, 128> : launch<float, 64>) : (f.tile == 128 ? launch<bf16, 128> : launch<bf16, 64>);
  if (!run(p, f, stream)) return false;
  if (f.splits == 1) return true;
  const int64_t blocks = std::min<int64_t>(ceil_div64((int64_t)k * n, 1024), 2048);
  weight_grad_sum_kernel<<<(unsigned)blocks, 256, 0, stream>>>(p, f.splits);
  return launch_ok("weight_grad_sum_kernel");
}

}  // namespace po
