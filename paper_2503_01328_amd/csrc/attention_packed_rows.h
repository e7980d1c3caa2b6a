// Rows of packed sequences one by one, for the matrix-core kernels' results that are not finite (attention_rows.h): row and key indexes
// are those of the packed batch, a row's sequence comes from the plan.
#pragma once

#include "attention_rows.h"
#include "packed_plan.h"

namespace po {

template <typename T, int DH>
__device__ __forceinline__ void redo_packed_forward_rows(uint32_t redo, int row0, PackedPlan plan, const T* __restrict__ qkv,
                                                         T* __restrict__ o, float* __restrict__ lse, int h, int hkv, int group,
                                                         int head, float scale) {
  while (redo) {
    const int i = row0 + __builtin_ctz(redo), first = __builtin_amdgcn_readfirstlane(plan.first()[i]);
    redo &= redo - 1;
    redo_forward_rows<T, DH>(1u, i - first, qkv + (size_t)first * (h + 2 * hkv), o + (size_t)first * h, lse + first, plan.rows, h, hkv,
                             group, head, scale);
  }
}
template <typename T, int DH>
__device__ __forceinline__ void redo_packed_dq_rows(uint32_t redo, int row0, PackedPlan plan, const T* __restrict__ qkv,
                                                    const T* __restrict__ d_o, const float* __restrict__ lse,
                                                    const float* __restrict__ delta, T* __restrict__ dqkv, int h, int hkv, int group,
                                                    int head, float scale) {
  while (redo) {
    const int i = row0 + __builtin_ctz(redo), first = __builtin_amdgcn_readfirstlane(plan.first()[i]);
    redo &= redo - 1;
    const size_t at = (size_t)first * (h + 2 * hkv);
    redo_dq_rows<T, DH>(1u, i - first, qkv + at, d_o + (size_t)first * h, lse + first, delta + first, dqkv + at, plan.rows, h, hkv,
                        group, head, scale);
  }
}
// Key rows; the heads of the group begin at `head`.
template <typename T, int DH>
__device__ __forceinline__ void redo_packed_key_rows(uint32_t redo, int row0, PackedPlan plan, const T* __restrict__ qkv,
                                                     const T* __restrict__ d_o, const float* __restrict__ lse,
                                                     const float* __restrict__ delta, T* __restrict__ dk, T* __restrict__ dv, int ld_out,
                                                     int h, int hkv, int group, int n_heads, int head, float scale) {
  while (redo) {
    const int j = row0 + __builtin_ctz(redo), last = __builtin_amdgcn_readfirstlane(plan.end()[j]) - 1, ld = h + 2 * hkv;
    redo &= redo - 1;
    int dh = DH, lane = (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
    asm volatile("" : "+s"(dh));  // a loop, not DH times its body
    const T* k = qkv + (size_t)j * ld + h + head / group * DH;
    const HeldRow<DH> key(k, scale, lane), value(k + hkv, 1.f, lane);
    attention_key_row<T, (DH + kWave - 1) / kWave, 8>(
        [&](int e) { return key.broadcast(e); }, [&](int e) { return value.broadcast(e); }, qkv + head * DH, d_o + head * DH, ld, h,
        lse + (size_t)head * plan.rows, delta + (size_t)head * plan.rows, plan.rows, n_heads, j, last, dh, lane, scale,
        dk + (size_t)j * ld_out, dv + (size_t)j * ld_out);
  }
}

}  // namespace po
