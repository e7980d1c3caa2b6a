// A feed-forward's activation with the checkpoint of its input, and its backward pass from that checkpoint.
//
//   out = act(u), or gated, u = a | b:  out = act(a) b;  act(a) = a s(a): SiLU, s = 1 / (1 + exp(-a)); GeLU in its tanh form,
//   s = (1 + tanh z) / 2 = 1 / (1 + exp(-2 z)), z = c (a + 0.044715 a^3), c = sqrt(2 / pi)
// backward, d the gradient of out:  du = d act'(u), or  da = d b act'(a), db = d act(a);
//   act' = s (1 + a (1 - s) w'), w' = 1 for SiLU, 2 z'(a) for GeLU.
// The backward makes out again beside: the weight gradient behind it needs it, and no value more has to be read for that.
//
// Bound by memory: forward u in, out and u's checkpoint out, backward the checkpoint and d in, du and out out.  A lane takes eight columns
// (gated: eight of a and eight of b), four lanes a block of the checkpoint.  Gated columns that are no whole blocks (f not a multiple of
// 32: b's blocks begin inside eights of a) go a value at a time, behind a launch that makes the checkpoint.
// bf16, 4096 rows of 2 x 8192, SiLU: forward 55 us (4.9 TB/s), backward 60 (5.6); 128 rows of 1024, fp32: 3.0 and 3.1.  A value at a time, 2 x 8200: forward 86
// (3.1), backward 165 (2.1), bound by instructions: a division and an access for every value.
#include <algorithm>

#include "saved8.h"

namespace po {

namespace {

struct Act {
  const void* u;             // [rows, cols] (backward: null where there is a checkpoint)
  const uint8_t *codes, *scales;
  const void* d_out;
  void *out, *du;
  uint8_t *codes_out, *scales_out;
  uint32_t chunks, row_chunks;  // eights of columns of out, padded to blocks, altogether and in a row
  int rows, f, cols;            // columns of out, of u
  int padded;                   // codes in a row
};

// The activation and its slope in terms of the gate keep = e r, r = 1 / (1 + e): e = exp(2 z) for GeLU, exp(a) for SiLU, r = 1 - keep.  As e r
// the gate has its relative precision where it is near zero, which 1 - r has not.  Far out the gate is 0 or 1 and a enters it cut, so
// that no square and no product with an infinity makes a NaN there (a NaN stays one).
template <bool SILU>
__device__ __forceinline__ void act_and_slope(float a, float& v, float& slope) {
  constexpr float kMost = SILU ? 150.f : 30.f, kC = 0.7978845608028654f, kLog2e = 1.4426950408889634f;
  const float x = fabsf(a) > kMost ? copysignf(kMost, a) : a;
  const float z = SILU ? x * kLog2e : x * (2.f * kC * kLog2e + 2.f * kC * kLog2e * 0.044715f * x * x);
  const float e = __builtin_amdgcn_exp2f(z > 120.f ? 120.f : z);
  const float r = __builtin_amdgcn_rcpf(1.f + e), keep = e * r;
  v = keep > 0.f ? a * keep : keep;  // keep is 0 far out, or NaN
  slope = keep * (1.f + x * r * (SILU ? 1.f : 2.f * kC + 6.f * 0.044715f * kC * x * x));
}
template <bool SILU>
__device__ __forceinline__ float act_of(float a) {
  float v, slope;
  act_and_slope<SILU>(a, v, slope);
  return v;
}

// Eight columns at a time.  GATED: f is a multiple of 32.
template <typename T, bool SILU, bool GATED, int UNROLL>
__global__ __launch_bounds__(256) void activation_forward_kernel(Act p) {
  const uint32_t base = blockIdx.x * (256u * UNROLL) + threadIdx.x;
  float a[UNROLL][8], b[GATED ? UNROLL : 1][8];
  uint32_t row[UNROLL], col[UNROLL];
  const int b_at = GATED ? p.f : 0;
#pragma unroll
  for (int k = 0; k < UNROLL; ++k) {
    const uint32_t i = base + 256u * k;
    row[k] = i / p.row_chunks;
    col[k] = (i - row[k] * p.row_chunks) * 8;
    const int held = i < p.chunks ? p.f - (int)col[k] : 0;
    const T* u = (const T*)p.u + (size_t)row[k] * p.cols + col[k];
    load_eight(a[k], u, held);
    if (GATED) load_eight(b[k], u + b_at, held);
  }
#pragma unroll
  for (int k = 0; k < UNROLL; ++k) {
    const uint32_t i = base + 256u * k;
    const bool there = i < p.chunks;
    const int held = there ? p.f - (int)col[k] : 0;
    if (p.codes_out) {
      unsigned byte;
      const uint2 codes = saved8_encode(a[k], byte);
      const size_t at = (size_t)row[k] * p.padded + col[k];
      if (there) {
        store_past(p.codes_out + at, codes);
        if (i % 4 == 0) p.scales_out[at / 32] = (uint8_t)byte;
      }
      if (GATED) {
        const uint2 more = saved8_encode(b[k], byte);
        if (there) {
          store_past(p.codes_out + at + b_at, more);
          if (i % 4 == 0) p.scales_out[(at + b_at) / 32] = (uint8_t)byte;
        }
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      a[k][e] = act_of<SILU>(a[k][e]);
      if (GATED) a[k][e] *= b[k][e];
    }
    if (there) store_eight((T*)p.out + (size_t)row[k] * p.f + col[k], a[k], held);
  }
}

template <typename T, bool SILU, bool GATED, bool SAVED, int UNROLL>
__global__ __launch_bounds__(256) void activation_backward_kernel(Act p) {
  const uint32_t base = blockIdx.x * (256u * UNROLL) + threadIdx.x;
  const int b_at = GATED ? p.f : 0;
  float a[UNROLL][8], b[GATED ? UNROLL : 1][8], d[UNROLL][8];
#pragma unroll
  for (int k = 0; k < UNROLL; ++k) {
    const uint32_t i = base + 256u * k, row = i / p.row_chunks, col = (i - row * p.row_chunks) * 8;
    const int held = i < p.chunks ? p.f - (int)col : 0;
    if (SAVED) {
      const size_t at = (size_t)row * p.padded + col;
      uint2 ca = make_uint2(0, 0), cb = ca;
      unsigned ba = 127, bb = 127;
      if (i < p.chunks) {
        ca = *(const uint2*)(p.codes + at);
        ba = p.scales[at / 32];
        if (GATED) {
          cb = *(const uint2*)(p.codes + at + b_at);
          bb = p.scales[(at + b_at) / 32];
        }
      }
      saved8_decode(ca, ba, a[k]);
      if (GATED) saved8_decode(cb, bb, b[k]);
    } else {
      const T* u = (const T*)p.u + (size_t)row * p.cols + col;
      load_eight(a[k], u, held);
      if (GATED) load_eight(b[k], u + b_at, held);
    }
    load_eight(d[k], (const T*)p.d_out + (size_t)row * p.f + col, held);
  }
#pragma unroll
  for (int k = 0; k < UNROLL; ++k) {
    const uint32_t i = base + 256u * k, row = i / p.row_chunks, col = (i - row * p.row_chunks) * 8;
    if (i >= p.chunks) continue;
    const int held = p.f - (int)col;
    T* du = (T*)p.du + (size_t)row * p.cols + col;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float v, slope;
      act_and_slope<SILU>(a[k][e], v, slope);
      if (GATED) {
        a[k][e] = v * b[k][e];
        b[k][e] *= d[k][e] * slope;
        d[k][e] *= v;
      } else {
        a[k][e] = v;
        d[k][e] *= slope;
      }
    }
    if (p.out) store_eight((T*)p.out + (size_t)row * p.f + col, a[k], held);
    if (GATED) {
      store_eight(du, b[k], held);
      store_eight(du + b_at, d[k], held);
    } else {
      store_eight(du, d[k], held);
    }
  }
}

// Gated columns that are no whole blocks, one value a thread.
__device__ __forceinline__ float saved8_at(const Act& p, size_t row, int col) {
  const size_t at = row * p.padded + col;
  return __builtin_amdgcn_cvt_f32_fp8((int)p.codes[at], 0) * saved8_scale(p.scales[at / 32]);
}
template <typename T, bool SILU, bool BACKWARD>
__global__ __launch_bounds__(256) void activation_ragged_kernel(Act p) {
  const size_t n = (size_t)p.rows * p.f;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) {
    const size_t row = i / (unsigned)p.f;
    const int col = (int)(i - row * p.f);
    const T* u = (const T*)p.u + row * p.cols + col;
    const bool saved = BACKWARD && p.codes;
    const float a = saved ? saved8_at(p, row, col) : to_f32(u[0]);
    const float b = saved ? saved8_at(p, row, p.f + col) : to_f32(u[p.f]);
    float v, slope;
    act_and_slope<SILU>(a, v, slope);
    if (!BACKWARD) v = act_of<SILU>(a);
    const float d = BACKWARD ? to_f32(((const T*)p.d_out)[i]) : 0.f;
    if (p.out) ((T*)p.out)[i] = from_f32<T>(v * b);
    if (BACKWARD) {
      T* du = (T*)p.du + row * p.cols + col;
      du[0] = from_f32<T>(b * (d * slope));
      du[p.f] = from_f32<T>(d * v);
    }
  }
}

template <typename T, bool SILU, bool GATED>
void launch_forward(const Act& p, hipStream_t stream) {
  // Two chunks a thread, both loads under way, where that still leaves every CU eight blocks.
  if (p.chunks >= 2u * 256 * 2048)
    activation_forward_kernel<T, SILU, GATED, 2><<<(unsigned)ceil_div64(p.chunks, 512), 256, 0, stream>>>(p);
  else
    activation_forward_kernel<T, SILU, GATED, 1><<<(unsigned)ceil_div64(p.chunks, 256), 256, 0, stream>>>(p);
}
template <typename T, bool SILU, bool GATED>
void launch_backward(const Act& p, hipStream_t stream) {
  const bool many = p.chunks >= 2u * 256 * 2048;
  const unsigned blocks = (unsigned)ceil_div64(p.chunks, many ? 512 : 256);
  if (p.codes) {
    if (many) activation_backward_kernel<T, SILU, GATED, true, 2><<<blocks, 256, 0, stream>>>(p);
    else activation_backward_kernel<T, SILU, GATED, true, 1><<<blocks, 256, 0, stream>>>(p);
  } else {
    if (many) activation_backward_kernel<T, SILU, GATED, false, 2><<<blocks, 256, 0, stream>>>(p);
    else activation_backward_kernel<T, SILU, GATED, false, 1><<<blocks, 256, 0, stream>>>(p);
  }
}
template <typename T, bool BACKWARD>
void launch_ragged(const Act& p, bool silu, hipStream_t stream) {
  const unsigned blocks = (unsigned)std::min<int64_t>(ceil_div64((int64_t)p.rows * p.f, 256), 1 << 14);
  if (silu) activation_ragged_kernel<T, true, BACKWARD><<<blocks, 256, 0, stream>>>(p);
  else activation_ragged_kernel<T, false, BACKWARD><<<blocks, 256, 0, stream>>>(p);
}

bool check(const char* what, int dtype, int act, int gated, int rows, int f) {
  if ((act != kActGelu && act != kActSilu) || (gated != 0 && gated != 1) || rows < 1 || f < 1 || f > (1 << 28) ||
      saved8_codes(rows, gated ? 2 * f : f) / 8 > kMaxSaved8Chunks) {
    set_error("%s: act=%d gated=%d rows=%d f=%d (act 0 or 1, gated 0 or 1, at least one row and column, at most %lld values)", what, act, gated,
              rows, f, (long long)kMaxSaved8Chunks * 8);
    return false;
  }
  return true;
}
Act shape_of(int dtype, int gated, int rows, int f) {
  Act p = {};
  p.rows = rows;
  p.f = f;
  p.cols = gated ? 2 * f : f;
  p.padded = (int)saved8_cols(p.cols);
  p.row_chunks = (uint32_t)(saved8_cols(f) / 8);
  p.chunks = p.row_chunks * (uint32_t)rows;
  return p;
}

}  // namespace

bool activation_forward(int dtype, int act, int gated, const void* u, void* out, void* saved_u, int rows, int f, hipStream_t stream) {
  if (!check("activation_forward", dtype, act, gated, rows, f)) return false;
  Act p = shape_of(dtype, gated, rows, f);
  const int size = dtype == kF32 ? 4 : 2;
  const uint64_t u_bytes = (uint64_t)rows * p.cols * size, out_bytes = (uint64_t)rows * f * size, saved_bytes = saved8_bytes(rows, p.cols);
  if (!u || !out || (uintptr_t)u % size != 0 || (uintptr_t)out % size != 0 || (uintptr_t)saved_u % 16 != 0) {
    set_error("activation_forward: u=%p out=%p saved_u=%p (u and out given and aligned to their type, saved_u to 16 bytes)", u, out, saved_u);
    return false;
  }
  if (overlap(u, u_bytes, saved_u, saved_bytes) || overlap(out, out_bytes, saved_u, saved_bytes) ||
      (overlap(u, u_bytes, out, out_bytes) && (gated || u != out))) {
    set_error("activation_forward: what is written overlaps what is read or written (out may be u where there is no gate)");
    return false;
  }
  p.u = u;
  p.out = out;
  const bool silu = act == kActSilu, ragged = gated && f % kSaved8Block != 0;
  if (ragged) {
    if (saved_u && !save8(dtype, 1, &u, &rows, &p.cols, &p.cols, &saved_u, stream)) return false;
    (dtype == kF32 ? launch_ragged<float, false> : launch_ragged<bf16, false>)(p, silu, stream);
    return launch_ok("activation_ragged_kernel");
  }
  if (saved_u) {
    p.codes_out = (uint8_t*)saved_u;
    p.scales_out = p.codes_out + saved8_codes(rows, p.cols);
  }
  auto k = dtype == kF32 ? (silu ? (gated ? launch_forward<float, true, true> : launch_forward<float, true, false>)
                                 : (gated ? launch_forward<float, false, true> : launch_forward<float, false, false>))
                         : (silu ? (gated ? launch_forward<bf16, true, true> : launch_forward<bf16, true, false>)
                                 : (gated ? launch_forward<bf16, false, true> : launch_forward<bf16, false, false>));
  k(p, stream);
  return launch_ok("activation_forward_kernel");
}

bool activation_backward(int dtype, int act, int gated, const void* u, int u_saved8, const void* d_out, void* du, void* out, int rows, int f,
                         hipStream_t stream) {
  if (!check("activation_backward", dtype, act, gated, rows, f)) return false;
  Act p = shape_of(dtype, gated, rows, f);
  const int size = dtype == kF32 ? 4 : 2;
  const uint64_t f_bytes = (uint64_t)rows * f * size, du_bytes = (uint64_t)rows * p.cols * size;
  const uint64_t u_bytes = u_saved8 ? saved8_bytes(rows, p.cols) : du_bytes;
  if (!u || !d_out || !du || (uintptr_t)u % (u_saved8 ? 16 : size) != 0 ||
      ((uintptr_t)d_out | (uintptr_t)du | (uintptr_t)out) % size != 0) {
    set_error("activation_backward: u=%p d_out=%p du=%p out=%p (u, d_out and du given, aligned to their type, a checkpoint to 16 bytes)", u, d_out,
              du, out);
    return false;
  }
  const bool in_place = du == d_out && !gated;
  if (overlap(du, du_bytes, u, u_bytes) || overlap(out, f_bytes, u, u_bytes) || overlap(out, f_bytes, d_out, f_bytes) ||
      overlap(out, f_bytes, du, du_bytes) || (overlap(du, du_bytes, d_out, f_bytes) && !in_place)) {
    set_error("activation_backward: what is written overlaps what is read or written (du may be d_out where there is no gate)");
    return false;
  }
  if (u_saved8) {
    p.codes = (const uint8_t*)u;
    p.scales = p.codes + saved8_codes(rows, p.cols);
  } else {
    p.u = u;
  }
  p.d_out = d_out;
  p.du = du;
  p.out = out;
  const bool silu = act == kActSilu;
  if (gated && f % kSaved8Block != 0) {
    (dtype == kF32 ? launch_ragged<float, true> : launch_ragged<bf16, true>)(p, silu, stream);
    return launch_ok("activation_ragged_kernel");
  }
  auto k = dtype == kF32 ? (silu ? (gated ? launch_backward<float, true, true> : launch_backward<float, true, false>)
                                 : (gated ? launch_backward<float, false, true> : launch_backward<float, false, false>))
                         : (silu ? (gated ? launch_backward<bf16, true, true> : launch_backward<bf16, true, false>)
                                 : (gated ? launch_backward<bf16, false, true> : launch_backward<bf16, false, false>));
  k(p, stream);
  return launch_ok("activation_backward_kernel");
}

}  // namespace po
