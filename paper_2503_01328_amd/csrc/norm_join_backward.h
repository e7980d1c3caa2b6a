// The backward of norm_join.hip for one type, compiled in a file for each.
//
// A block takes rows one after another.  Each tensor's registers are loaded with the next row's values, packed as they lie in memory, as soon as
// this row's have been used, so that a row's loads are under way while the row before is computed; parameters stay in registers.
// Loads and stores go through buffers that end with the row: columns behind it, tensors that are not there and rows behind the last read
// as zeros without a branch: branches around loads made the compiler wait for each at once (16384 rows of 5120, both norms and a gate: 435 us, without 228).
// What bounds it: memory, 5.4 TB/s in that case with the blocks that the chip holds at once (212 us).
#pragma once

#include "norm_join.h"

namespace po {
namespace norm_join {

// Which kernel: y and f from checkpoints, or both from tensors, with rows of whole eights on 16-byte boundaries; or anything: one from a checkpoint and one from a
// tensor, rows on no such boundaries (whole eights as vectors from wherever they start, a row's last columns a value at a time).  It branches around its
// loads, and takes sixteen waves and scratch from 4097 columns on: bf16, both LayerNorms and a gate for each column, 4096 rows of 4096: both saved 53 us, both
// tensors 57, one of each 81; of 8192: 101, 107, 265.
enum Form { kFromSaved, kFromTensors, kAny };

// Eight columns of y or f.
template <typename T, Form FORM>
struct Source {
  Packed<T, FORM != kAny> raw;
  uint2 codes;
  unsigned byte;
  __device__ __forceinline__ void load(const void* tensor, const uint8_t* saved, int64_t row, const Join& p, bool there, unsigned col) {
    if (FORM != kFromSaved) raw.load(tensor, row, p.h, there && tensor, col);
    if (FORM != kFromTensors) {
      const bool from_saved = there && (FORM == kFromSaved || saved);
      const auto q = __builtin_amdgcn_raw_buffer_load_b64(row_buffer(saved, row * p.padded, from_saved ? p.padded : 0), (int)col, 0, 0);
      codes = make_uint2(q[0], q[1]);
      byte = __builtin_amdgcn_raw_buffer_load_b8(row_buffer(saved, ((int64_t)p.rows * p.padded) + (row * p.padded >> 5), from_saved ? p.padded >> 5 : 0),
                                                 (int)(col >> 5), 0, 0);
    }
  }
  __device__ __forceinline__ void get(float (&x)[8], bool saved, int held) const {
    if (FORM == kFromSaved || (FORM == kAny && saved)) saved8_decode(codes, byte, x);
    else raw.get(x);
    if (FORM == kAny) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i >= held) x[i] = 0.f;
    }
  }
};

// v - mean where there is a column, zero elsewhere; a lane's eight are all there or none of them, but in kAny.
template <Form FORM>
__device__ __forceinline__ void centre_eight(float (&v)[8], float mean, int held) {
  const float m = held > 0 ? mean : 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = FORM != kAny || i < held ? v[i] - m : 0.f;
}

// The parameter sums that a launch makes: all of them, but for rows that take two eights a lane and more than eight waves, whose 128
// registers a lane do not hold them all: there each kind has a launch of its own, of which the last writes the outputs.  What does not fit still spills, 20 bytes a lane
// (bf16, RMS norm alone) to 820 (fp32, anything): 4096 rows of 12288, bf16, RMS norm 92 us, LayerNorm 172, both LayerNorms and a gate for each column 830.
enum { kSumPre = 1, kSumPost = 2, kSumGate = 4 };

// LAYER: not the RMS norm.  POST: there is a norm of f.  (kAny asks the arguments for both.)  SUMS: what is summed.  OUT: whether dx, df, dgate and n are written.
// WAVES: of a block at most.
template <typename T, int C, int WAVES, Form FORM, bool LAYER_, bool POST_, int SUMS, bool OUT>
__global__ __launch_bounds__(64 * WAVES) void norm_join_backward_kernel(Join p) {
  __shared__ float room[2][2][16];
  constexpr bool VEC = FORM != kAny, PRE_SUM = SUMS & kSumPre, POST_SUM = SUMS & kSumPost, GATE_SUM = SUMS & kSumGate;
  const bool LAYER = FORM == kAny ? p.layer : LAYER_, POST = FORM == kAny ? p.post_gain != nullptr : POST_;
  BlockSums sums(room);
  const float over_h = 1.f / (float)p.h;
  const bool pre = p.dn, gate = p.gate, uses_f = POST || gate, per_value = p.gate_per_value;
  unsigned col[C];
  int held[C];
  float dpre_gain[C][8], dpre_shift[C][8], dpost_gain[C][8], dpost_shift[C][8], dgate[C][8];
  Packed<T, VEC> pre_gain[C], post_gain[C], gates[C], dy[C], dn[C];
  Source<T, FORM> y_source[C], f_source[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    col[c] = (c * blockDim.x + threadIdx.x) * 8;
    held[c] = p.h - (int)col[c];
#pragma unroll
    for (int i = 0; i < 8; ++i) dpre_gain[c][i] = dpre_shift[c][i] = dpost_gain[c][i] = dpost_shift[c][i] = dgate[c][i] = 0.f;
    pre_gain[c].load(p.pre_gain, 0, p.h, pre, col[c]);
    if (POST) post_gain[c].load(p.post_gain, 0, p.h, true, col[c]);
    gates[c].load(p.gate, gate && per_value ? (int64_t)blockIdx.x : 0, p.h, gate, col[c]);
    y_source[c].load(p.y_in, p.y_codes, blockIdx.x, p, pre, col[c]);
    dn[c].load(p.dn, blockIdx.x, p.h, pre, col[c]);
    f_source[c].load(p.f, p.f_codes, blockIdx.x, p, uses_f, col[c]);
    dy[c].load(p.dy, blockIdx.x, p.h, p.dy, col[c]);
  }
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
    const int64_t next = row + gridDim.x;
    const bool more = next < p.rows;
    float y[C][8], t[C][8], d[C][8], w[8], s[2] = {0.f, 0.f}, m[2] = {0.f, 0.f};
    // both norms' statistics
    float mean_f = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      y_source[c].get(y[c], p.y_codes, held[c]);
      y_source[c].load(p.y_in, p.y_codes, next, p, pre && more, col[c]);
    }
    if (LAYER) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        if (POST) f_source[c].get(w, p.f_codes, held[c]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          s[0] += y[c][i];
          if (POST) s[1] += w[i];
        }
      }
      sums(s);
      mean_f = s[1] * over_h;
#pragma unroll
      for (int c = 0; c < C; ++c) centre_eight<FORM>(y[c], s[0] * over_h, held[c]);
    }
    s[0] = s[1] = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (POST) {
        f_source[c].get(w, p.f_codes, held[c]);
        if (LAYER) centre_eight<FORM>(w, mean_f, held[c]);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        s[0] = fmaf(y[c][i], y[c][i], s[0]);
        if (POST) s[1] = fmaf(w[i], w[i], s[1]);
      }
    }
    sums(s);
    const float root = rsqrtf(s[0] * over_h + p.eps), root_f = rsqrtf(s[1] * over_h + p.eps);
    if (pre) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        dn[c].get(d[c]);
        dn[c].load(p.dn, next, p.h, more, col[c]);
        pre_gain[c].get(w);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          y[c][i] *= root;
          if (PRE_SUM) dpre_gain[c][i] = fmaf(d[c][i], y[c][i], dpre_gain[c][i]);
          if (PRE_SUM && LAYER) dpre_shift[c][i] += d[c][i];
          d[c][i] *= w[i];
          if (LAYER) m[0] += d[c][i];
          m[1] = fmaf(d[c][i], y[c][i], m[1]);
        }
      }
      sums(m);
    }
    // t, and d: what f's branch gets
#pragma unroll
    for (int c = 0; c < C; ++c) {
      dy[c].get(t[c]);
      dy[c].load(p.dy, next, p.h, p.dy && more, col[c]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (pre) t[c][i] = fmaf(root, d[c][i] - m[0] * over_h - y[c][i] * (m[1] * over_h), t[c][i]);
        d[c][i] = p.branch * t[c][i];
        t[c][i] *= p.skip;
      }
      if (OUT) store_chunk<T, VEC>(p.dx, t[c], row, p.h, col[c]);
      if (OUT && p.n) {
        pre_gain[c].get(w);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[c][i] *= w[i];
        if (LAYER && p.pre_shift) {
          Packed<T, VEC> shift;
          shift.load(p.pre_shift, 0, p.h, true, col[c]);
          shift.get(w);
#pragma unroll
          for (int i = 0; i < 8; ++i) y[c][i] += w[i];
        }
        store_chunk<T, VEC>(p.n, y[c], row, p.h, col[c]);
      }
    }
    m[0] = m[1] = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (!uses_f) continue;
      f_source[c].get(y[c], p.f_codes, held[c]);
      f_source[c].load(p.f, p.f_codes, next, p, more, col[c]);
      if (POST) {
        if (LAYER) centre_eight<FORM>(y[c], mean_f, held[c]);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[c][i] *= root_f;
      }
      if (gate) {
        float z[8];
        if (POST) post_gain[c].get(w);
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = POST ? y[c][i] * w[i] : y[c][i];
        if (POST && LAYER && p.post_shift) {
          Packed<T, VEC> shift;
          shift.load(p.post_shift, 0, p.h, true, col[c]);
          shift.get(w);
#pragma unroll
          for (int i = 0; i < 8; ++i) z[i] += w[i];
        }
        gates[c].get(w);
        if (per_value) gates[c].load(p.gate, next, p.h, more, col[c]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          z[i] *= d[c][i];
          if (GATE_SUM) dgate[c][i] += z[i];
          d[c][i] *= w[i];
        }
        if (OUT && per_value) store_chunk<T, VEC>(p.dgate, z, row, p.h, col[c]);
      }
      if (POST) {
        post_gain[c].get(w);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (POST_SUM) dpost_gain[c][i] = fmaf(d[c][i], y[c][i], dpost_gain[c][i]);
          if (POST_SUM && LAYER) dpost_shift[c][i] += d[c][i];
          d[c][i] *= w[i];
          if (LAYER) m[0] += d[c][i];
          m[1] = fmaf(d[c][i], y[c][i], m[1]);
        }
      }
    }
    if (!OUT) continue;
    if (POST) sums(m);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (POST) {
#pragma unroll
        for (int i = 0; i < 8; ++i) d[c][i] = root_f * (d[c][i] - m[0] * over_h - y[c][i] * (m[1] * over_h));
      }
      store_chunk<T, VEC>(p.df, d[c], row, p.h, col[c]);
    }
  }
  if (!p.partials) return;
  // [blocks][the sums of the whole call][h]: this launch's at their place
  int64_t at = (int64_t)blockIdx.x * p.n_sums;
  auto leave = [&](const float (&v)[C][8], bool mine) {
    if (mine) {
#pragma unroll
      for (int c = 0; c < C; ++c) store_chunk<float, VEC>(p.partials, v[c], at, p.h, col[c]);
    }
    ++at;
  };
  if (pre) leave(dpre_gain, PRE_SUM);
  if (pre && p.pre_shift) leave(dpre_shift, PRE_SUM);
  if (POST) leave(dpost_gain, POST_SUM);
  if (POST && p.post_shift) leave(dpost_shift, POST_SUM);
  if (gate && !per_value) leave(dgate, GATE_SUM);
}

template <typename T, int C, Form FORM, bool LAYER, bool POST>
void launch_all(const Join& p, hipStream_t stream) {
  constexpr int NORMS = kSumPre | (POST ? kSumPost : 0);
  const int blocks = blocks_of(p.rows, p.h), threads = 64 * waves_of(p.h, C);
  if (p.gate && !p.gate_per_value) norm_join_backward_kernel<T, C, 8, FORM, LAYER, POST, NORMS | kSumGate, true><<<blocks, threads, 0, stream>>>(p);
  else norm_join_backward_kernel<T, C, 8, FORM, LAYER, POST, NORMS, true><<<blocks, threads, 0, stream>>>(p);
}
// Sixteen waves: each kind of sums in a launch of its own, the outputs with the last (dx may be dy, df dn).
template <typename T, Form FORM, bool LAYER, bool POST>
void launch_wide(const Join& p, hipStream_t stream) {
  const int blocks = blocks_of(p.rows, p.h), threads = 64 * waves_of(p.h, 2);
  if (p.gate && !p.gate_per_value) norm_join_backward_kernel<T, 2, 16, FORM, LAYER, POST, kSumGate, false><<<blocks, threads, 0, stream>>>(p);
  if (p.post_gain) norm_join_backward_kernel<T, 2, 16, FORM, LAYER, POST, kSumPost, false><<<blocks, threads, 0, stream>>>(p);
  norm_join_backward_kernel<T, 2, 16, FORM, LAYER, POST, kSumPre, true><<<blocks, threads, 0, stream>>>(p);
}
template <typename T, Form FORM, bool LAYER, bool POST>
void launch_form(const Join& p, hipStream_t stream) {
  if (p.h <= 64 * 8) launch_all<T, 1, FORM, LAYER, POST>(p, stream);
  else if (p.h <= 8 * 64 * 8 * 2) launch_all<T, 2, FORM, LAYER, POST>(p, stream);
  else launch_wide<T, FORM, LAYER, POST>(p, stream);
}
template <typename T, Form FORM>
void launch_form(const Join& p, hipStream_t stream) {
  if (p.post_gain) (p.layer ? launch_form<T, FORM, true, true> : launch_form<T, FORM, false, true>)(p, stream);
  else (p.layer ? launch_form<T, FORM, true, false> : launch_form<T, FORM, false, false>)(p, stream);
}
template <typename T>
void launch_any(const Join& p, hipStream_t stream) {
  constexpr int ALL = kSumPre | kSumPost | kSumGate;
  const int blocks = blocks_of(p.rows, p.h), threads = 64 * waves_of(p.h, 1);
  if (p.h <= 8 * 64 * 8) norm_join_backward_kernel<T, 1, 8, kAny, true, true, ALL, true><<<blocks, threads, 0, stream>>>(p);
  else if (p.h <= 16 * 64 * 8) norm_join_backward_kernel<T, 1, 16, kAny, true, true, ALL, true><<<blocks, threads, 0, stream>>>(p);
  else launch_wide<T, kAny, true, true>(p, stream);
}
template <typename T>
void launch_backward(const Join& p, hipStream_t stream) {
  const bool uses_f = p.post_gain || p.gate, pre = p.dn;
  const bool saved = (!pre || p.y_codes) && (!uses_f || p.f_codes), tensors = (!pre || p.y_in) && (!uses_f || p.f);
  if (!p.vec || (!saved && !tensors)) return launch_any<T>(p, stream);
  (saved ? launch_form<T, kFromSaved> : launch_form<T, kFromTensors>)(p, stream);
}

}  // namespace norm_join
}  // namespace po
