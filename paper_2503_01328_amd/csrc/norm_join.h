// What the kernels of norm_join.hip and norm_join_backward.h share: a call's tensors, sums over a row, which parameter sums there are.
#pragma once

#include <algorithm>

#include "mfma_common.h"
#include "saved8.h"

namespace po {
namespace norm_join {

// Eight waves a row, two eights of columns a lane; the widest rows take four a lane (forward) or sixteen waves (backward).  One eight a lane and
// twice the waves is as fast (5120 columns, backward: 221 and 235 us, 4096: 49 and 48), but a row of 8192 then leaves a lane 128 registers.
constexpr int kMaxWaves = 8, kMaxWidth = kMaxWaves * 64 * 8 * 4, kMaxRows = 1 << 25;

struct Join {
  const void *x, *f, *gate, *post_gain, *post_shift, *pre_gain, *pre_shift;
  const void *dy, *dn, *y_in;
  const uint8_t *f_codes, *y_codes;  // backward: the checkpoints, where f and y_in are null
  uint8_t *f_codes_out, *y_codes_out;
  void *y, *n, *dx, *df, *dgate;
  float* partials;
  int rows, h, padded, vec, gate_per_value, layer, n_sums;
  float skip, branch, eps;
};

// Sums over a row of sixteen lanes and over a wave, the same in every lane: lane exchanges, then the wave's four rows.
__device__ __forceinline__ float sum_of_sixteen(float v) {
#define PO_ADD_DPP(ctrl) v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), ctrl, 0xf, 0xf, true))
  PO_ADD_DPP(0xb1);   // neighbours
  PO_ADD_DPP(0x4e);   // pairs of four
  PO_ADD_DPP(0x141);  // half rows mirrored
  PO_ADD_DPP(0x140);  // rows mirrored
#undef PO_ADD_DPP
  return v;
}
__device__ __forceinline__ float sum_of_wave(float v) {
  v = sum_of_sixteen(v);
  auto row = [&](int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane)); };
  return (row(0) + row(16)) + (row(32) + row(48));
}
// Sums of N values over the block: every wave leaves its own in LDS, every lane takes one of them, and a row of sixteen lanes adds them up.  Two buffers
// in turn: who writes one has passed the barrier behind the other's reads.
struct BlockSums {
  float (*room)[2][16];
  int turn = 0, waves;
  __device__ __forceinline__ BlockSums(float (*r)[2][16]) : room(r), waves((int)blockDim.x >> 6) {
    if (waves == 1) return;
    for (int i = threadIdx.x; i < 2 * 2 * 16; i += blockDim.x) (&room[0][0][0])[i] = 0.f;
    __syncthreads();
  }
  template <int N>
  __device__ __forceinline__ void operator()(float (&v)[N]) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = sum_of_wave(v[k]);
    if (waves == 1) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float(*r)[16] = room[turn];
    turn ^= 1;
    if (lane == 0) {
#pragma unroll
      for (int k = 0; k < N; ++k) r[k][wave] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = sum_of_sixteen(r[k][lane & 15]);
  }
};

// Rows are read and written through buffers that end with them: columns behind a row and tensors that are not there read as zeros, without a
// branch.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t row_buffer(const void* p, int64_t at, int bytes) {
  return buffer_resource((const char*)p + at, (unsigned)bytes);
}

constexpr int kStorePast = 2;  // a buffer store's non-temporal bit

// Eight columns as they lie in memory.  VEC: rows start on 16-byte boundaries and are whole eights.  Others: whole eights from wherever they start, a row's
// last a value at a time (backward of 4096 rows of 5001, RMS norm: 128 us, with single values everywhere 198; of 1001, fp32: 20.5, so 44).
template <typename T, bool VEC>
struct Packed {
  u32x4 v[sizeof(T) / 2];
  // p: the tensor; row: bytes = 0 for one that is not there
  __device__ __forceinline__ void load(const void* p, int64_t row, int h, bool there, unsigned col) {
    const int at = (int)(col * sizeof(T));
    if constexpr (!VEC) {
#pragma unroll
      for (int k = 0; k < (int)sizeof(T) / 2; ++k) v[k] = u32x4{0u, 0u, 0u, 0u};
      if (!there) return;
      if ((int)col + 8 <= h) {
        __builtin_memcpy(v, (const char*)p + row * h * (int64_t)sizeof(T) + at, sizeof(v));
        return;
      }
    }
    const __amdgpu_buffer_rsrc_t b = row_buffer(p, row * h * (int64_t)sizeof(T), there ? h * (int)sizeof(T) : 0);
    if constexpr (VEC) {
#pragma unroll
      for (int k = 0; k < (int)sizeof(T) / 2; ++k) v[k] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(b, at + 16 * k, 0, 0));
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i / 4][i % 4] = __builtin_amdgcn_raw_buffer_load_b32(b, at + 4 * i, 0, 0);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        v[0][i] = (unsigned)(uint16_t)__builtin_amdgcn_raw_buffer_load_b16(b, at + 4 * i, 0, 0) |
                  (unsigned)(uint16_t)__builtin_amdgcn_raw_buffer_load_b16(b, at + 4 * i + 2, 0, 0) << 16;
    }
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (sizeof(T) == 4) x[i] = __uint_as_float(v[i / 4][i % 4]);
      else x[i] = __uint_as_float(i % 2 ? v[0][i / 2] & 0xffff0000u : v[0][i / 2] << 16);
    }
  }
  __device__ __forceinline__ void set(const float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (sizeof(T) == 4) {
        v[i / 4][i % 4] = __float_as_uint(x[i]);
      } else if (i % 2 == 0) {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        const bf16x2 pair = {(bf16)x[i], (bf16)x[i + 1]};
        v[0][i / 2] = __builtin_bit_cast(unsigned, pair);
      }
    }
  }
  __device__ __forceinline__ void store(void* p, int64_t row, int h, unsigned col) const {
    const int at = (int)(col * sizeof(T));
    if constexpr (!VEC)
      if ((int)col + 8 <= h) {
        __builtin_memcpy((char*)p + row * h * (int64_t)sizeof(T) + at, v, sizeof(v));
        return;
      }
    const __amdgpu_buffer_rsrc_t b = row_buffer(p, row * h * (int64_t)sizeof(T), h * (int)sizeof(T));
    typedef unsigned raw __attribute__((ext_vector_type(4)));
    if constexpr (VEC) {
#pragma unroll
      for (int k = 0; k < (int)sizeof(T) / 2; ++k) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(raw, v[k]), b, at + 16 * k, 0, kStorePast);
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 8; ++i) __builtin_amdgcn_raw_buffer_store_b32(v[i / 4][i % 4], b, at + 4 * i, 0, 0);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) __builtin_amdgcn_raw_buffer_store_b16((unsigned short)(v[0][i / 2] >> (16 * (i % 2))), b, at + 2 * i, 0, 0);
    }
  }
};
template <typename T, bool VEC>
__device__ __forceinline__ void store_chunk(void* p, const float (&x)[8], int64_t row, int h, unsigned col) {
  Packed<T, VEC> w;
  w.set(x);
  w.store(p, row, h, col);
}

// Which sums a block leaves, in this order.
enum Sum { kPreGain, kPreShift, kPostGain, kPostShift, kGate, kSums };
struct SumTargets {
  float* to[kSums];  // null: not among the partial sums
};

// Waves that a row of h columns takes, `chunks` eights a lane.
inline int waves_of(int h, int chunks) { return ceil_div((int)(saved8_cols(h) / 8), 64 * chunks); }
// Blocks of the backward, each of which leaves a partial sum of every parameter's gradient: what the chip holds at once, at most 1024.
// bf16, us with the sums, 256 / 512 / 768 blocks: 4096 rows of 4096 (four waves a row) 62 49 51, 16384 rows of 5120 (five) 221 234 241.
inline int blocks_of(int rows, int h) {
  const int most = std::min(1024, 256 * std::max(1, kMaxWaves / waves_of(h, h <= 64 * 8 ? 1 : 2)));
  return rows < most ? rows : most;
}

// norm_join_backward_f32.hip, norm_join_backward_bf16.hip: dx, df, dgate, n and the blocks' partial sums.
void launch_backward_f32(const Join& p, hipStream_t stream);
void launch_backward_bf16(const Join& p, hipStream_t stream);

}  // namespace norm_join
}  // namespace po
