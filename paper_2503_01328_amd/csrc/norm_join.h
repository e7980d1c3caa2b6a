// What the kernels of norm_join.hip and norm_join_backward.h share: a call's tensors, sums over a row, which parameter sums there are.
#pragma once

#include "mfma_common.h"
#include "saved8.h"

namespace po {
namespace norm_join {

constexpr int kMaxWaves = 8, kMaxWidth = kMaxWaves * 64 * 8 * 4, kMaxRows = 1 << 25;
constexpr int kMaxBlocks = 512;  // of the backward: each leaves a partial sum of every parameter's gradient

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

// Which sums a block leaves, in this order.
enum Sum { kPreGain, kPreShift, kPostGain, kPostShift, kGate, kSums };
struct SumTargets {
  float* to[kSums];  // null: not among the partial sums
};

// Waves that a row of h columns takes, `chunks` eights a lane.
inline int waves_of(int h, int chunks) { return ceil_div((int)(saved8_cols(h) / 8), 64 * chunks); }
inline int blocks_of(int rows) { return rows < kMaxBlocks ? rows : kMaxBlocks; }

// norm_join_backward_f32.hip, norm_join_backward_bf16.hip: dx, df, dgate, n and the blocks' partial sums.
void launch_backward_f32(const Join& p, hipStream_t stream);
void launch_backward_bf16(const Join& p, hipStream_t stream);

}  // namespace norm_join
}  // namespace po
