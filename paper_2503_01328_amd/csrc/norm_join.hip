// A block's output on its way back into the residual stream, and the norm in front of the next block:
//
//   z = N(f) gain2 + shift2 (or f),  y = skip x + branch g z (g: none, one for each column, one for each value),  n = N(y) gain + shift
// N: LayerNorm, (v - mean) / sqrt(var + eps), or the RMS norm, v / sqrt(mean(v^2) + eps).  The forward leaves 8-bit checkpoints of f and y
// (saved8.h), y's of y as it is stored.  Backward, from dy and dn, f and y (checkpoints or tensors):
//   a = dn gain,  t = dy + r (a - mean(a) - yh mean(a yh))  (yh = N(y), r its root; RMS: without mean(a)),  dx = skip t
//   w = branch t,  dg = w z,  dz = w g,  b = dz gain2,  df = r2 (b - mean(b) - fh mean(b fh))
//   dgain += sum dn yh, dshift += sum dn, dgain2 += sum dz fh, dshift2 += sum dz, and dg's sum where g is one for each column
// n can be had again beside: it is the input of the weight gradient that follows.  Everything between the loads and the one rounding of a
// store is fp32, variances are those of centred values.
//
// Bound by memory: every tensor once.  A block of as many waves as a row of eights needs takes a row, values stay in registers from
// the load to the store, sums go over the lanes by lane exchanges and over the waves through LDS.  Backward blocks take rows one after another and
// hold their columns' sums of the parameter gradients in registers; a second launch adds the blocks' in a fixed order: no atomics.
// bf16: forward of 2048 rows of 2048 with both RMS norms, a gate and both checkpoints 9.8 us; backward of 4096 rows of 4096, LayerNorm, with n 39 us and 5
// for the sums (4.7 TB/s), of 16384 rows of 5120 with both RMS norms and a gate for each value 212 and 6 (5.4 TB/s).
#include <algorithm>

#include "norm_join.h"

namespace po {

using namespace norm_join;

namespace {

// v becomes N(v); held: columns of each eight that there are (VEC: eight or none).  ZEROS: behind them v stays zero where the root is not finite too (a zero
// times it is NaN, and a checkpoint's codes behind the last column are zeros).  Where nothing behind is stored it may be NaN (4096 rows of 4097: 0.3 us).
template <bool VEC, bool ZEROS, int C>
__device__ __forceinline__ void normalise(float (&v)[C][8], const int (&held)[C], const Join& p, BlockSums& sums) {
  float s[1] = {0.f};
  const float over_h = 1.f / (float)p.h;
  if (p.layer) {
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) s[0] += v[c][i];
    sums(s);
    const float mean = s[0] * over_h;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) v[c][i] = i < held[c] ? v[c][i] - mean : 0.f;
    s[0] = 0.f;
  }
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) s[0] = fmaf(v[c][i], v[c][i], s[0]);
  sums(s);
  const float r = rsqrtf(s[0] * over_h + p.eps);
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) v[c][i] *= !ZEROS || (VEC ? 0 : i) < held[c] ? r : 0.f;
}
template <typename P, int C>
__device__ __forceinline__ void affine(float (&v)[C][8], const P (&gain)[C], const P (&shift)[C]) {
  float g[8], a[8];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    gain[c].get(g);
    shift[c].get(a);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[c][i] = fmaf(v[c][i], g[i], a[i]);
  }
}
template <int C>
__device__ __forceinline__ void save_row(uint8_t* codes, const float (&v)[C][8], const unsigned (&col)[C], int64_t row, const Join& p) {
  uint8_t* scales = codes + (int64_t)p.rows * p.padded;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    unsigned byte;
    const uint2 q = saved8_encode(v[c], byte);
    if ((int)col[c] < p.padded) {
      const int64_t at = row * p.padded + col[c];
      store_past(codes + at, q);
      if (threadIdx.x % 4 == 0) scales[at / 32] = (uint8_t)byte;
    }
  }
}

// VEC: rows of whole eights on 16-byte boundaries.
template <typename T, int C, bool VEC>
__global__ __launch_bounds__(64 * kMaxWaves) void norm_join_forward_kernel(Join p) {
  __shared__ float room[2][2][16];
  const int64_t row = blockIdx.x;
  unsigned col[C];
  int held[C];
  Packed<T, VEC> f_in[C], x_in[C], g_in[C], post_gain[C], post_shift[C], pre_gain[C], pre_shift[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    col[c] = (c * blockDim.x + threadIdx.x) * 8;
    held[c] = p.h - (int)col[c];
    f_in[c].load(p.f, row, p.h, true, col[c]);
    x_in[c].load(p.x, row, p.h, true, col[c]);
    g_in[c].load(p.gate, p.gate_per_value ? row : 0, p.h, p.gate, col[c]);
    post_gain[c].load(p.post_gain, 0, p.h, p.post_gain, col[c]);
    post_shift[c].load(p.post_shift, 0, p.h, p.post_shift, col[c]);
    pre_gain[c].load(p.pre_gain, 0, p.h, p.pre_gain, col[c]);
    pre_shift[c].load(p.pre_shift, 0, p.h, p.pre_shift, col[c]);
  }
  BlockSums sums(room);
  float f[C][8], x[C][8];
#pragma unroll
  for (int c = 0; c < C; ++c) f_in[c].get(f[c]);
  if (p.f_codes_out) save_row(p.f_codes_out, f, col, row, p);
  if (p.post_gain) {
    normalise<VEC, true>(f, held, p, sums);
    affine(f, post_gain, post_shift);
  }
#pragma unroll
  for (int c = 0; c < C; ++c) {
    float g[8];
    x_in[c].get(x[c]);
    g_in[c].get(g);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float z = p.gate ? f[c][i] * g[i] : f[c][i];
      x[c][i] = fmaf(p.skip, x[c][i], p.branch * z);
    }
    Packed<T, VEC> stored;
    stored.set(x[c]);
    stored.store(p.y, row, p.h, col[c]);
    stored.get(f[c]);  // y as it is stored
  }
  if (p.y_codes_out) save_row(p.y_codes_out, f, col, row, p);
  if (!p.pre_gain) return;
  normalise<VEC, false>(x, held, p, sums);
  affine(x, pre_gain, pre_shift);
#pragma unroll
  for (int c = 0; c < C; ++c) store_chunk<T, VEC>(p.n, x[c], row, p.h, col[c]);
}

// += the blocks' partial sums [blocks][n_sums h]: a block 32 columns, a thread every 32nd block's value of one, eight loads under way.
__global__ __launch_bounds__(1024) void norm_join_sum_kernel(const float* __restrict__ partials, int blocks, int h, int n_sums, SumTargets targets) {
  __shared__ float part[32][33];
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
  const int64_t width = (int64_t)n_sums * h, e = (int64_t)blockIdx.x * 32 + x;
  float v = 0.f;
  if (e < width) {
    for (int b = y; b < blocks; b += 256) {
      float u[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) u[k] = b + 32 * k < blocks ? partials[(b + 32 * k) * width + e] : 0.f;
      v += ((u[0] + u[1]) + (u[2] + u[3])) + ((u[4] + u[5]) + (u[6] + u[7]));
    }
  }
  part[y][x] = v;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    __syncthreads();
    if (y < o) part[y][x] += part[y + o][x];
  }
  if (y || e >= width) return;
  const int which = (int)(e / h);
  float* to = targets.to[0];
#pragma unroll
  for (int k = 1; k < kSums; ++k)
    if (which == k) to = targets.to[k];
  to[e - (int64_t)which * h] += part[0][x];
}

int forward_chunks(int h) { return h <= 64 * 8 ? 1 : h <= kMaxWaves * 64 * 8 * 2 ? 2 : 4; }

// row_waves: waves of a launch for each row, none where blocks take rows one after another; saved: whether a checkpoint is read or written.
bool check(const char* what, int norm, int rows, int h, int row_waves, bool saved, float skip, float branch, float eps) {
  if ((norm != kNormLayer && norm != kNormRms) || rows < 1 || rows > kMaxRows || h < 1 || h > kMaxWidth || !(fabsf(skip) < 3e38f) ||
      !(fabsf(branch) < 3e38f) || !(eps >= 0.f) || eps > 3e38f) {
    set_error("%s: norm=%d rows=%d h=%d skip=%g branch=%g eps=%g (norm 0 or 1, 1 to %d rows, h 1 to %d, scales finite, eps finite and not "
              "negative)", what, norm, rows, h, skip, branch, eps, kMaxRows, kMaxWidth);
    return false;
  }
  if ((int64_t)rows * 64 * row_waves > UINT32_MAX || (saved && saved8_codes(rows, h) / 8 > kMaxSaved8Chunks)) {
    set_error("%s: rows=%d h=%d are too many for a launch, or for a checkpoint (%lld values)", what, rows, h, (long long)kMaxSaved8Chunks * 8);
    return false;
  }
  return true;
}
// One tensor of a call: where it is, how long, whether it is written, which input it may be.
struct Range {
  const char* name;
  const void* p;
  uint64_t bytes;
  int align;
  bool written;
  const void* may_be;
  bool rows = false;  // an input [rows, h] of dtype: a row is read before any of it is written, as a parameter, which every row reads anew, is not
};
bool check_ranges(const char* what, const Range* r, int n) {
  for (int i = 0; i < n; ++i) {
    if ((uintptr_t)r[i].p % r[i].align != 0) {
      set_error("%s: %s=%p is not aligned to %d bytes", what, r[i].name, r[i].p, r[i].align);
      return false;
    }
    for (int j = 0; j < n; ++j) {
      if (i == j || !r[i].written || !overlap(r[i].p, r[i].bytes, r[j].p, r[j].bytes)) continue;
      if (r[j].rows && r[i].p == r[j].p && r[i].may_be == r[j].p) continue;
      set_error("%s: %s is written and overlaps %s", what, r[i].name, r[j].name);
      return false;
    }
  }
  return true;
}

template <typename T, bool VEC>
void launch_forward(const Join& p, hipStream_t stream) {
  const int chunks = forward_chunks(p.h), threads = 64 * waves_of(p.h, chunks);
  if (chunks == 1) norm_join_forward_kernel<T, 1, VEC><<<p.rows, threads, 0, stream>>>(p);
  else if (chunks == 2) norm_join_forward_kernel<T, 2, VEC><<<p.rows, threads, 0, stream>>>(p);
  else norm_join_forward_kernel<T, 4, VEC><<<p.rows, threads, 0, stream>>>(p);
}

}  // namespace

bool norm_join_forward(int dtype, const NormJoin& a, const void* x, const void* f, void* y, void* n, void* saved_f, void* saved_y,
                       hipStream_t stream) {
  const char* what = "norm_join_forward";
  if (!check(what, a.norm, a.rows, a.h, waves_of(a.h, forward_chunks(a.h)), saved_f || saved_y, a.skip, a.branch, a.eps)) return false;
  if (!x || !f || !y || (a.pre_gain == nullptr) != (n == nullptr) || (!a.pre_gain && a.pre_shift) || (!a.post_gain && a.post_shift) ||
      (a.norm == kNormRms && (a.pre_shift || a.post_shift)) || (a.gate_per_value != 0 && a.gate_per_value != 1)) {
    set_error("%s: x=%p f=%p y=%p n=%p pre_gain=%p pre_shift=%p post_gain=%p post_shift=%p gate_per_value=%d (x, f and y given, n with "
              "pre_gain, shifts with their gain and not with the RMS norm)", what, x, f, y, n, a.pre_gain, a.pre_shift, a.post_gain, a.post_shift,
              a.gate_per_value);
    return false;
  }
  const int size = dtype == kF32 ? 4 : 2;
  const uint64_t one = (uint64_t)a.rows * a.h * size, row = (uint64_t)a.h * size, saved = saved8_bytes(a.rows, a.h);
  const Range ranges[] = {{"y", y, one, size, true, x},           {"n", n, one, size, true, f},
                          {"saved_f", saved_f, saved, 16, true, nullptr}, {"saved_y", saved_y, saved, 16, true, nullptr},
                          {"x", x, one, size, false, nullptr, true}, {"f", f, one, size, false, nullptr, true},
                          {"gate", a.gate, a.gate_per_value ? one : row, size, false, nullptr, a.gate_per_value != 0}, {"pre_gain", a.pre_gain, row, size, false, nullptr},
                          {"pre_shift", a.pre_shift, row, size, false, nullptr}, {"post_gain", a.post_gain, row, size, false, nullptr},
                          {"post_shift", a.post_shift, row, size, false, nullptr}};
  if (!check_ranges(what, ranges, sizeof(ranges) / sizeof(ranges[0]))) return false;
  Join p = {};
  p.x = x;
  p.f = f;
  p.gate = a.gate;
  p.post_gain = a.post_gain;
  p.post_shift = a.post_shift;
  p.pre_gain = a.pre_gain;
  p.pre_shift = a.pre_shift;
  p.y = y;
  p.n = n;
  p.f_codes_out = (uint8_t*)saved_f;
  p.y_codes_out = (uint8_t*)saved_y;
  p.rows = a.rows;
  p.h = a.h;
  p.padded = (int)saved8_cols(a.h);
  uintptr_t all = (uintptr_t)row;
  for (const Range& r : ranges) all |= (uintptr_t)r.p;
  p.vec = all % 16 == 0 && a.h % 8 == 0;
  p.gate_per_value = a.gate_per_value;
  p.layer = a.norm == kNormLayer;
  p.skip = a.skip;
  p.branch = a.branch;
  p.eps = a.eps;
  (dtype == kF32 ? (p.vec ? launch_forward<float, true> : launch_forward<float, false>)
                 : (p.vec ? launch_forward<bf16, true> : launch_forward<bf16, false>))(p, stream);
  return launch_ok("norm_join_forward_kernel");
}

size_t norm_join_backward_workspace(int rows, int h) {
  if (rows < 1 || rows > kMaxRows || h < 1 || h > kMaxWidth) return 0;
  return (size_t)blocks_of(rows, h) * kSums * h * sizeof(float);
}

bool norm_join_backward(int dtype, const NormJoin& a, const NormJoinBackward& b, hipStream_t stream) {
  const char* what = "norm_join_backward";
  if (!check(what, a.norm, a.rows, a.h, 0, (b.dn && b.y_saved8) || ((a.post_gain || a.gate) && b.f_saved8), a.skip, a.branch, a.eps)) return false;
  const bool pre = b.dn != nullptr, post = a.post_gain != nullptr, gate = a.gate != nullptr, rms = a.norm == kNormRms;
  if (!b.dx || !b.df || (!b.dy && !pre) || pre != (a.pre_gain != nullptr) || (pre && !b.y) || ((post || gate) && !b.f) || (b.n && !pre) ||
      (a.gate_per_value != 0 && a.gate_per_value != 1) || (!pre && a.pre_shift) || (!post && a.post_shift) ||
      (rms && (a.pre_shift || a.post_shift))) {
    set_error("%s: dy=%p dn=%p y=%p f=%p dx=%p df=%p n=%p pre_gain=%p pre_shift=%p post_gain=%p post_shift=%p gate_per_value=%d (dx, df and dy or "
              "dn given, dn and pre_gain both or none, y with dn, f with post_gain or gate, n only with dn, shifts with their gain and not with "
              "the RMS norm)", what, b.dy, b.dn, b.y, b.f, b.dx, b.df, b.n, a.pre_gain, a.pre_shift, a.post_gain, a.post_shift, a.gate_per_value);
    return false;
  }
  const bool columns = gate && !a.gate_per_value;
  if (gate != (b.dgate != nullptr) || pre != (b.dpre_gain != nullptr) || (a.pre_shift != nullptr) != (b.dpre_shift != nullptr) ||
      post != (b.dpost_gain != nullptr) || (a.post_shift != nullptr) != (b.dpost_shift != nullptr) || ((pre || post || columns) && !b.workspace)) {
    set_error("%s: dgate=%p dpre_gain=%p dpre_shift=%p dpost_gain=%p dpost_shift=%p workspace=%p (a gradient for every parameter that is given and "
              "no other, a workspace for their sums)", what, b.dgate, (void*)b.dpre_gain, (void*)b.dpre_shift, (void*)b.dpost_gain,
              (void*)b.dpost_shift, (void*)b.workspace);
    return false;
  }
  const int size = dtype == kF32 ? 4 : 2;
  const uint64_t one = (uint64_t)a.rows * a.h * size, row = (uint64_t)a.h * size, saved = saved8_bytes(a.rows, a.h), sum = (uint64_t)a.h * 4;
  const Range ranges[] = {{"dx", b.dx, one, size, true, b.dy},
                          {"df", b.df, one, size, true, b.dn},
                          {"dgate", b.dgate, columns ? sum : one, columns ? 4 : size, true, nullptr},
                          {"dpre_gain", b.dpre_gain, sum, 4, true, nullptr},
                          {"dpre_shift", b.dpre_shift, sum, 4, true, nullptr},
                          {"dpost_gain", b.dpost_gain, sum, 4, true, nullptr},
                          {"dpost_shift", b.dpost_shift, sum, 4, true, nullptr},
                          {"n", b.n, one, size, true, nullptr},
                          {"workspace", b.workspace, norm_join_backward_workspace(a.rows, a.h), 16, true, nullptr},
                          {"dy", b.dy, one, size, false, nullptr, true},
                          {"dn", b.dn, one, size, false, nullptr, true},
                          {"y", pre ? b.y : nullptr, b.y_saved8 ? saved : one, b.y_saved8 ? 16 : size, false, nullptr, !b.y_saved8},
                          {"f", post || gate ? b.f : nullptr, b.f_saved8 ? saved : one, b.f_saved8 ? 16 : size, false, nullptr, !b.f_saved8},
                          {"gate", a.gate, a.gate_per_value ? one : row, size, false, nullptr, a.gate_per_value != 0},
                          {"pre_gain", a.pre_gain, row, size, false, nullptr},
                          {"pre_shift", a.pre_shift, row, size, false, nullptr},
                          {"post_gain", a.post_gain, row, size, false, nullptr},
                          {"post_shift", a.post_shift, row, size, false, nullptr}};
  if (!check_ranges(what, ranges, sizeof(ranges) / sizeof(ranges[0]))) return false;
  Join p = {};
  p.gate = a.gate;
  p.post_gain = a.post_gain;
  p.post_shift = a.post_shift;
  p.pre_gain = a.pre_gain;
  p.pre_shift = a.pre_shift;
  p.dy = b.dy;
  p.dn = b.dn;
  if (b.y_saved8) p.y_codes = (const uint8_t*)b.y;
  else p.y_in = b.y;
  if (b.f_saved8) p.f_codes = (const uint8_t*)b.f;
  else p.f = b.f;
  p.n = b.n;
  p.dx = b.dx;
  p.df = b.df;
  p.dgate = b.dgate;
  const bool any = pre || post || columns;
  p.partials = any ? (float*)b.workspace : nullptr;
  p.rows = a.rows;
  p.h = a.h;
  p.padded = (int)saved8_cols(a.h);
  uintptr_t all = (uintptr_t)row;
  for (const Range& r : ranges)
    if (r.align != 4 || size == 4) all |= (uintptr_t)r.p;
  p.vec = all % 16 == 0 && a.h % 8 == 0;
  p.gate_per_value = a.gate_per_value;
  p.layer = !rms;
  p.skip = a.skip;
  p.branch = a.branch;
  p.eps = a.eps;
  p.n_sums = pre + (a.pre_shift != nullptr) + post + (a.post_shift != nullptr) + columns;
  const int blocks = blocks_of(a.rows, a.h);
  (dtype == kF32 ? launch_backward_f32 : launch_backward_bf16)(p, stream);
  if (!launch_ok("norm_join_backward_kernel")) return false;
  if (!any) return true;
  SumTargets targets = {};
  int n = 0;
  if (pre) targets.to[n++] = b.dpre_gain;
  if (a.pre_shift) targets.to[n++] = b.dpre_shift;
  if (post) targets.to[n++] = b.dpost_gain;
  if (a.post_shift) targets.to[n++] = b.dpost_shift;
  if (columns) targets.to[n++] = (float*)b.dgate;
  norm_join_sum_kernel<<<(unsigned)ceil_div64((int64_t)n * a.h, 32), 1024, 0, stream>>>((const float*)b.workspace, blocks, a.h, n, targets);
  return launch_ok("norm_join_sum_kernel");
}

}  // namespace po
