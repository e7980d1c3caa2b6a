// Queries and keys of a layer on their way from the projection to attention: every head normed by its root mean square and rotated by
// its row's positions, one pass over q | k | v, forward and backward.
//
//   r = 1 / sqrt(mean(x^2) + eps), y = x r g (one gain for all query heads, one for all key heads; no norm: y = x)
//   pair p = elements (a, b) of y, angle t = position[axis of p] inv_freq[p]:  (a cos t - b sin t, a sin t + b cos t)
// backward, d the gradient of the output: u = the rotation by -t of d,
//   dg += sum over rows and heads of u x r,  w = u g,  dx = r (w - x r mean(w x r))
// Everything between the load and the one rounding of the store is fp32; angles are formed in fp64 and reduced to a turn there: in
// fp32 position 10^6 would be a twentieth of a radian off.
//
// Bound by memory: each element is read (backward with gains: with its input) and written once.  A wave takes a row at a time, or shares
// one with others (waves_of_a_row): lane p forms the cosine and sine of pair p once for all heads, which read them back from LDS; then
// 64 / LANES heads at a time, a lane holding 16 elements (eight pairs) of one head.  bf16, from HBM: 16384 rows, 40 heads of 128 over 8:
// forward 91 us, backward 145 us (a large copy reaches 4.9 TB/s); 2048 rows, 16 heads: 13.6 us, and 24.0 us.
// The gains' gradients stay in registers over all rows of a wave, are added over the lanes and waves of a block in a fixed order, and a
// second launch adds the blocks: no atomics.  Half of those blocks take the queries and half the keys and values, so that a lane has one
// gain's gradient to hold, not two, and twice the waves fit: 189 us without, 140 with.
#include <algorithm>

#include "kernels.h"

namespace po {

namespace {

constexpr int kBlocks = 1024;  // for queries and for keys at most in the backward; each leaves a partial sum of a gain's gradient
constexpr int kMaxPairs = 128;
constexpr int kMaxRows = 1 << 25, kMaxBlocks = 1 << 23;  // 2^31 threads

struct Axes {
  int end[kMaxRotaryAxes];  // the pairs [end[i - 1], end[i]) turn by axis i
};

// A lane's 16 elements of a head as eight pairs.  Halves: chunk l of the first half and of the second; behind the rotated part two chunks
// in a row.  Neighbours: two chunks in a row.
template <typename T>
__device__ __forceinline__ void load8(float (&v)[8], const T* p) {
  constexpr int V = Vec16<T>::N;
#pragma unroll
  for (int k = 0; k < 8; k += V) {
    const Vec16<T> x = load16(p + k);
#pragma unroll
    for (int i = 0; i < V; ++i) v[k + i] = to_f32(x.v[i]);
  }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&v)[8]) {
  constexpr int V = Vec16<T>::N;
#pragma unroll
  for (int k = 0; k < 8; k += V) {
    Vec16<T> x;
#pragma unroll
    for (int i = 0; i < V; ++i) x.v[i] = from_f32<T>(v[k + i]);
    store16(p + k, x);
  }
}
template <typename T, bool NEIGHBOURS>
__device__ __forceinline__ void load_pairs(float (&a)[8], float (&b)[8], const T* head, int at_a, int at_b) {
  float x[8], y[8];
  load8(x, head + at_a);
  load8(y, head + at_b);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    a[i] = NEIGHBOURS ? (i < 4 ? x[2 * i] : y[2 * i - 8]) : x[i];
    b[i] = NEIGHBOURS ? (i < 4 ? x[2 * i + 1] : y[2 * i - 7]) : y[i];
  }
}
template <typename T, bool NEIGHBOURS>
__device__ __forceinline__ void store_pairs(T* head, int at_a, int at_b, const float (&a)[8], const float (&b)[8]) {
  float x[8], y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    x[i] = NEIGHBOURS ? (i & 1 ? b[i / 2] : a[i / 2]) : a[i];
    y[i] = NEIGHBOURS ? (i & 1 ? b[4 + i / 2] : a[4 + i / 2]) : b[i];
  }
  store8(head + at_a, x);
  store8(head + at_b, y);
}
template <int LANES>
__device__ __forceinline__ float sum_over_head(float v) {
#pragma unroll
  for (int o = 1; o < LANES; o <<= 1) v += __shfl_xor(v, o, 64);
  return v;
}

__device__ __forceinline__ void rotate(float (&a)[8], float (&b)[8], const float (&c)[8], const float (&sn)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float y = a[i] * c[i] - b[i] * sn[i];
    b[i] = a[i] * sn[i] + b[i] * c[i];
    a[i] = y;
  }
}
// What the lanes of this wave left in LDS before is there for all of them after.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

struct Shape {
  int rows, h, hkv, dh, pairs, n_heads, n_kv_heads;
  float eps;
};

// BACKWARD: x_in is the input of the forward (null: no norm), in the gradient of its output, out that of its input.
template <typename T, int LANES, bool NEIGHBOURS, bool BACKWARD>
__global__ __launch_bounds__(256) void qk_norm_rotary_kernel(const T* in, const T* __restrict__ x_in, const T* __restrict__ gain_q,
                                                             const T* __restrict__ gain_k, const int* __restrict__ positions,
                                                             const float* __restrict__ inv_freq, Axes axes, T* out,
                                                             float* __restrict__ partials, Shape s, int split) {
  __shared__ float2 turns[4][kMaxPairs];
  __shared__ __align__(16) float gains[2 * LANES][16];  // for queries, for keys
  __shared__ float sums[BACKWARD ? 4 : 1][BACKWARD ? 16 * LANES : 1];
  constexpr int HEADS = 64 / LANES;  // of a wave at a time
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane & (LANES - 1);
  const int ld = s.h + 2 * s.hkv;
  const bool held = 16 * l < s.dh, rotated = 8 * l < s.pairs, norm = gain_q != nullptr;
  const int at_a = NEIGHBOURS || !rotated ? 16 * l : 8 * l, at_b = NEIGHBOURS || !rotated ? 16 * l + 8 : s.pairs + 8 * l;
  if (norm) {  // a lane's sixteen gains next to each other
    if (threadIdx.x < 2 * LANES) {
      float a[8] = {}, b[8] = {};  // lanes without elements add zeros to a head's sums
      if (held) load_pairs<T, NEIGHBOURS>(a, b, threadIdx.x < LANES ? gain_q : gain_k, at_a, at_b);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        gains[threadIdx.x][i] = a[i];
        gains[threadIdx.x][8 + i] = b[i];
      }
    }
    __syncthreads();
  }
  float dg_a[8], dg_b[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) dg_a[i] = dg_b[i] = 0.f;
  // Gradients of gains: the first half of the blocks takes the queries, the second the keys and values.
  const bool parts = BACKWARD && norm;
  const int blocks = parts ? gridDim.x / 2 : gridDim.x, part = (int)blockIdx.x >= blocks, block = blockIdx.x - part * blocks;
  const int head_first = part ? s.n_heads : 0, head_end = parts && !part ? s.n_heads : s.n_heads + s.n_kv_heads;

  const int share = wave & (split - 1), shared = 4 / split;  // `split` waves share a row, `shared` rows a block
  for (int row = block * shared + wave / split; row < s.rows; row += blocks * shared) {
    if (positions[row] < 0) continue;  // no token there
    for (int p = lane; p < s.pairs; p += 64) {
      int axis = 0;
#pragma unroll
      for (int i = 0; i + 1 < kMaxRotaryAxes; ++i) axis += p >= axes.end[i];
      const double turn = (double)positions[(size_t)axis * s.rows + row] * (double)inv_freq[p] * 0.15915494309189533577;
      float2 cs;
      sincospif(2.f * (float)(turn - rint(turn)), &cs.y, &cs.x);
      turns[wave][p] = cs;
    }
    wave_sync();
    float c[8], sn[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 cs = rotated ? turns[wave][8 * l + i] : make_float2(1.f, 0.f);
      c[i] = cs.x;
      sn[i] = BACKWARD ? -cs.y : cs.y;
    }
    wave_sync();
    for (int head0 = head_first + share * HEADS; head0 < head_end; head0 += split * HEADS) {
      const int head = head0 + lane / LANES;
      const bool mine = held && head < head_end;
      const size_t at = (size_t)row * ld + (size_t)head * s.dh;
      const float* gain = gains[(head < s.n_heads ? 0 : LANES) + l];
      float a[8], b[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) a[i] = b[i] = 0.f;
      if (mine) load_pairs<T, NEIGHBOURS>(a, b, in + at, at_a, at_b);
      if constexpr (!BACKWARD) {
        if (norm) {
          float sq = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) sq = fmaf(a[i], a[i], fmaf(b[i], b[i], sq));
          const float r = rsqrtf(sum_over_head<LANES>(sq) / (float)s.dh + s.eps);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            a[i] *= r * gain[i];
            b[i] *= r * gain[8 + i];
          }
        }
        if (rotated) rotate(a, b, c, sn);
      } else {
        if (rotated) rotate(a, b, c, sn);
        if (norm) {
          float x[8], y[8], sq = 0.f, dot = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = y[i] = 0.f;
          if (mine) load_pairs<T, NEIGHBOURS>(x, y, x_in + at, at_a, at_b);
#pragma unroll
          for (int i = 0; i < 8; ++i) sq = fmaf(x[i], x[i], fmaf(y[i], y[i], sq));
          // The normed x from here on: its products stay in range wherever its own squares did, r^3 does not
          const float r = rsqrtf(sum_over_head<LANES>(sq) / (float)s.dh + s.eps);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            x[i] *= r;
            y[i] *= r;
            if (mine) {
              dg_a[i] = fmaf(a[i], x[i], dg_a[i]);
              dg_b[i] = fmaf(b[i], y[i], dg_b[i]);
            }
            a[i] *= gain[i];
            b[i] *= gain[8 + i];
            dot = fmaf(a[i], x[i], fmaf(b[i], y[i], dot));
          }
          const float mean = sum_over_head<LANES>(dot) / (float)s.dh;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            a[i] = r * (a[i] - x[i] * mean);
            b[i] = r * (b[i] - y[i] * mean);
          }
        }
      }
      if (mine) store_pairs<T, NEIGHBOURS>(out + at, at_a, at_b, a, b);
    }
    if (in != out && (!parts || part)) {  // the values pass
      constexpr int V = Vec16<T>::N;
      const size_t v0 = (size_t)row * ld + s.h + s.hkv;
      for (int e = (share * 64 + lane) * V; e < s.hkv; e += split * 64 * V) store16(out + v0 + e, load16(in + v0 + e));
    }
  }
  if constexpr (BACKWARD) {
    if (!norm) return;
    // element order of the gain: what a lane's pair i is at
    float* mine = sums[wave];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float v[2] = {dg_a[i], dg_b[i]};
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int o = LANES; o < 64; o <<= 1) v[k] += __shfl_xor(v[k], o, 64);
      if (lane < LANES && held) {
        mine[NEIGHBOURS ? 16 * l + 2 * i : at_a + i] = v[0];
        mine[NEIGHBOURS ? 16 * l + 2 * i + 1 : at_b + i] = v[1];
      }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < s.dh; e += 256)
      partials[(size_t)blockIdx.x * s.dh + e] = (sums[0][e] + sums[1][e]) + (sums[2][e] + sums[3][e]);
  }
}

// dgain_q, dgain_k [dh] += the blocks' partial sums [2][blocks][dh]: a block eight columns, a thread every 32nd row of one, eight loads
// under way: 5.3 us for 1024 blocks (sixteen columns and every sixteenth row, a load at a time: 25.4).
__global__ __launch_bounds__(256) void rotary_gain_sum_kernel(const float* __restrict__ partials, int blocks, int dh,
                                                              float* __restrict__ dgain_q, float* __restrict__ dgain_k) {
  __shared__ float sums[32][9];
  const int x = threadIdx.x & 7, y = threadIdx.x >> 3, e = blockIdx.x * 8 + x;  // dh is a multiple of 8
  const float* p = partials + (e < dh ? e : (size_t)blocks * dh + e - dh);
  float v = 0.f;
  for (int b = y; b < blocks; b += 32 * 8) {
    float u[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) u[k] = b + 32 * k < blocks ? p[(size_t)(b + 32 * k) * dh] : 0.f;
    v += ((u[0] + u[1]) + (u[2] + u[3])) + ((u[4] + u[5]) + (u[6] + u[7]));
  }
  sums[y][x] = v;
  __syncthreads();
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    if (y < o) sums[y][x] += sums[y + o][x];
    __syncthreads();
  }
  if (y) return;
  float* to = e < dh ? dgain_q + e : dgain_k + (e - dh);
  *to += sums[0][x];
}

bool check(const char* what, const QkNormRotary& a, const void* in, const void* x_in, const void* out, Axes& axes, Shape& s) {
  const int dh = a.n_heads > 0 ? a.h / a.n_heads : 0;
  if (a.rows <= 0 || a.rows > kMaxRows || a.h <= 0 || a.n_heads <= 0 || a.h % a.n_heads != 0 || a.n_kv_heads <= 0 ||
      a.n_heads % a.n_kv_heads != 0 || dh % 16 != 0 || dh < 16 || dh > 256) {
    set_error("%s: rows=%d h=%d heads=%d kv_heads=%d (1 to %d rows, head size h / heads a multiple of 16 up to 256, kv_heads a divisor of "
              "heads)", what, a.rows, a.h, a.n_heads, a.n_kv_heads, kMaxRows);
    return false;
  }
  if ((int64_t)a.h + 2 * (int64_t)a.n_kv_heads * dh > INT32_MAX) {
    set_error("%s: a row of h=%d and %d key/value heads is too long", what, a.h, a.n_kv_heads);
    return false;
  }
  if (a.n_axes < 1 || a.n_axes > kMaxRotaryAxes || !a.axis_pairs) {
    set_error("%s: n_axes=%d axis_pairs=%p (1 to %d axes)", what, a.n_axes, (const void*)a.axis_pairs, kMaxRotaryAxes);
    return false;
  }
  int64_t pairs = 0;
  for (int i = 0; i < kMaxRotaryAxes; ++i) {
    if (i < a.n_axes && a.axis_pairs[i] < 0) pairs = -1;
    if (i < a.n_axes && pairs >= 0) pairs += a.axis_pairs[i];
    axes.end[i] = i + 1 < a.n_axes ? (int)std::min<int64_t>(pairs, INT32_MAX) : INT32_MAX;
    if (pairs < 0) break;
  }
  if (pairs < 0 || pairs > dh / 2 || pairs % 8 != 0 || (a.layout != kRotaryHalves && a.layout != kRotaryNeighbours)) {
    set_error("%s: %lld pairs of heads of %d, layout %d (pairs per axis not negative, together a multiple of 8 and at most half the "
              "head size; layout 0 or 1)", what, (long long)pairs, dh, a.layout);
    return false;
  }
  if (!(a.eps >= 0.f) || a.eps > 3e38f || (a.gain_q == nullptr) != (a.gain_k == nullptr)) {
    set_error("%s: eps=%g gain_q=%p gain_k=%p (eps finite and not negative, both gains or none)", what, a.eps, a.gain_q, a.gain_k);
    return false;
  }
  if (!in || !out || !a.positions || (pairs > 0 && !a.inv_freq) ||
      ((uintptr_t)in | (uintptr_t)x_in | (uintptr_t)out | (uintptr_t)a.gain_q | (uintptr_t)a.gain_k) % 16 != 0 ||
      ((uintptr_t)a.positions | (uintptr_t)a.inv_freq) % 4 != 0) {
    set_error("%s: a NULL pointer, or one that is not 16-byte aligned", what);
    return false;
  }
  s = Shape{a.rows, a.h, a.n_kv_heads * dh, dh, (int)pairs, a.n_heads, a.n_kv_heads, a.eps};
  return true;
}

int lanes_of_a_head(int dh) { return dh <= 32 ? 2 : dh <= 64 ? 4 : dh <= 128 ? 8 : 16; }

template <typename T, int LANES, bool BACKWARD>
void launch(const QkNormRotary& a, const void* in, const void* x_in, void* out, float* partials, const Axes& axes, const Shape& s,
            int blocks, int split, hipStream_t stream) {
  auto k = a.layout == kRotaryNeighbours ? qk_norm_rotary_kernel<T, LANES, true, BACKWARD> : qk_norm_rotary_kernel<T, LANES, false, BACKWARD>;
  k<<<blocks, 256, 0, stream>>>((const T*)in, (const T*)x_in, (const T*)a.gain_q, (const T*)a.gain_k, a.positions, a.inv_freq, axes,
                                (T*)out, partials, s, split);
}
template <bool BACKWARD>
void launch(int dtype, const QkNormRotary& a, const void* in, const void* x_in, void* out, float* partials, const Axes& axes,
            const Shape& s, int blocks, int split, hipStream_t stream) {
  const int lanes = lanes_of_a_head(s.dh);
  auto k = lanes == 2   ? (dtype == kF32 ? launch<float, 2, BACKWARD> : launch<bf16, 2, BACKWARD>)
           : lanes == 4 ? (dtype == kF32 ? launch<float, 4, BACKWARD> : launch<bf16, 4, BACKWARD>)
           : lanes == 8 ? (dtype == kF32 ? launch<float, 8, BACKWARD> : launch<bf16, 8, BACKWARD>)
                        : (dtype == kF32 ? launch<float, 16, BACKWARD> : launch<bf16, 16, BACKWARD>);
  k(a, in, x_in, out, partials, axes, s, blocks, split, stream);
}
// How many waves share a row of `heads` heads.  Few rows: the wave's chain of loads, heads after heads, is what such a launch waits for.
// Many: two waves to a row still leave less of the card idle towards the end where a row has three steps of heads, angles formed twice cost
// more than that where it has fewer.  With gains' gradients a launch has two kinds of blocks and its partial sums grow with the blocks.
// bf16 from HBM, us, one wave / two / four: 40 heads of 128 over 8, forward 128 rows 8.9 6.1 5.4, 1000 rows 14.0 10.5 10.5, 2048 rows 16.7
// 15.6 17.2, 16384 rows 97 91 91; 16 heads of 64 over 4 (two steps) 5.3 4.5 4.6 (500 rows), 9.9 11.8 14.6 (4096).  Backward with gains: 128
// rows 14.5 11.4 10.3, 500 rows 18.3 15.1 14.5, 1000 rows 20.0 18.5 23.9, 2048 rows 25.9 30.5 35.0; 16 heads of 64 (one step), 500
// rows 9.4 9.5 11.7.
int waves_of_a_row(int rows, int dh, int heads, bool gains) {
  const int steps = ceil_div(heads, 64 / lanes_of_a_head(dh)), most = steps > 2 ? 4 : steps;
  if (gains) return rows <= 512 ? most : rows <= 1024 ? std::min(most, 2) : 1;
  return rows <= 1024 ? most : steps > 2 ? 2 : 1;
}
// (split is at most 4: no more blocks than rows)
int blocks_of(int rows, int split, int most) { return (int)std::min<int64_t>(ceil_div64((int64_t)rows * split, 4), most); }

}  // namespace

// What any count of rows up to `rows` needs, for a program that keeps one workspace for its largest batch: fewer rows can make more
// blocks, as more waves share each, but never more than rows.
size_t qk_norm_rotary_backward_workspace(int rows, int h, int n_heads) {
  return (size_t)std::min(rows, kBlocks) * 2 * (h / n_heads) * sizeof(float);
}

bool qk_norm_rotary_forward(int dtype, const QkNormRotary& a, const void* qkv, void* out, hipStream_t stream) {
  Axes axes;
  Shape s;
  if (!check("qk_norm_rotary_forward", a, qkv, nullptr, out, axes, s)) return false;
  const int split = waves_of_a_row(a.rows, s.dh, a.n_heads + a.n_kv_heads, false);
  launch<false>(dtype, a, qkv, nullptr, out, nullptr, axes, s, blocks_of(a.rows, split, kMaxBlocks), split, stream);
  return launch_ok("qk_norm_rotary_kernel");
}

bool qk_norm_rotary_backward(int dtype, const QkNormRotary& a, const void* d_out, const void* qkv, void* dqkv, float* dgain_q,
                             float* dgain_k, float* workspace, hipStream_t stream) {
  Axes axes;
  Shape s;
  if (!check("qk_norm_rotary_backward", a, d_out, qkv, dqkv, axes, s)) return false;
  if (a.gain_q && (!qkv || !dgain_q || !dgain_k || !workspace || ((uintptr_t)dgain_q | (uintptr_t)dgain_k | (uintptr_t)workspace) % 4 != 0)) {
    set_error("qk_norm_rotary_backward: with gains, qkv=%p dgain_q=%p dgain_k=%p and workspace=%p are needed", qkv, (void*)dgain_q,
              (void*)dgain_k, (void*)workspace);
    return false;
  }
  if (qkv == dqkv && a.gain_q) {
    set_error("qk_norm_rotary_backward: dqkv may be d_out, but not qkv");
    return false;
  }
  const int split = waves_of_a_row(a.rows, s.dh, a.gain_q ? a.n_heads : a.n_heads + a.n_kv_heads, a.gain_q != nullptr);
  const int blocks = blocks_of(a.rows, split, a.gain_q ? kBlocks : kMaxBlocks);
  launch<true>(dtype, a, d_out, qkv, dqkv, workspace, axes, s, a.gain_q ? 2 * blocks : blocks, split, stream);
  // one gain for both: the partial sums of queries and of keys are one array of twice the blocks, and its columns added to once
  const bool shared = dgain_q == dgain_k;
  if (a.gain_q)
    rotary_gain_sum_kernel<<<(shared ? 1 : 2) * s.dh / 8, 256, 0, stream>>>(workspace, shared ? 2 * blocks : blocks, s.dh, dgain_q, dgain_k);
  return launch_ok("qk_norm_rotary_kernel");
}

}  // namespace po
