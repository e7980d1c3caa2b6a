// Rows of packed sequences one by one, for the matrix-core kernels' results that are not finite (attention_rows.h): row and key indexes
// are those of the packed batch, a row's sequence comes from the plan.  sign: 1, or -1 if the negative of delta stands in memory.
#pragma once

#include "attention_rows.h"
#include "packed_plan.h"

namespace po {

// Whether every element of a row is NaN.  All lanes call it.
template <typename T, int DH>
__device__ __forceinline__ bool all_nan(const T* __restrict__ row, int lane) {
  bool nan = is_nan(to_f32(row[lane]));
  if constexpr (DH > kWave) nan = nan && is_nan(to_f32(row[lane + kWave]));
  return __builtin_amdgcn_ballot_w64(nan) == ~(uint64_t)0;
}
template <typename T, int DH>
__device__ __forceinline__ void write_nan(T* __restrict__ row, int lane) {
  row[lane] = from_f32<T>(NAN);
  if constexpr (DH > kWave) row[lane + kWave] = from_f32<T>(NAN);
}

// o of these rows; their lse is right as it is, the scores of what a row does not see having been replaced.
template <typename T, int DH>
__device__ __forceinline__ void redo_packed_forward_rows(uint32_t redo, int row0, PackedPlan plan, const T* __restrict__ qkv,
                                                         T* __restrict__ o, int h, int hkv, int group, int head, float scale) {
  while (redo) {
    const int i = row0 + __builtin_ctz(redo), first = __builtin_amdgcn_readfirstlane(plan.first()[i]), ld = h + 2 * hkv;
    redo &= redo - 1;
    int dh = DH, lane = (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
    asm volatile("" : "+s"(dh));  // a loop, not DH times its body
    const T* k = qkv + (size_t)first * ld + h + head / group * DH;
    T* o_row = o + (size_t)i * h + head * DH;
    // a batch whose values have all become NaN is not computed row by row: a row sees its own value
    if (all_nan<T, DH>(k + hkv + (size_t)(i - first) * ld, lane)) {
      write_nan<T, DH>(o_row, lane);
      continue;
    }
    const HeldRow<DH> q(qkv + (size_t)i * ld + head * DH, scale, lane);
    float lse;
    attention_forward_row<T, (DH + kWave - 1) / kWave, 8>([&](int e) { return q.broadcast(e); }, k, k + hkv, ld, i - first, dh, lane, o_row,
                                                          &lse);
  }
}
template <typename T, int DH>
__device__ __forceinline__ void redo_packed_dq_rows(uint32_t redo, int row0, PackedPlan plan, const T* __restrict__ qkv,
                                                    const T* __restrict__ d_o, const float* __restrict__ lse,
                                                    const float* __restrict__ delta, T* __restrict__ dqkv, int h, int hkv, int group,
                                                    int head, float scale, float sign) {
  while (redo) {
    const int i = row0 + __builtin_ctz(redo), first = __builtin_amdgcn_readfirstlane(plan.first()[i]), ld = h + 2 * hkv;
    redo &= redo - 1;
    int dh = DH, lane = (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
    asm volatile("" : "+s"(dh));  // a loop, not DH times its body
    const HeldRow<DH> q(qkv + (size_t)i * ld + head * DH, scale, lane), g(d_o + (size_t)i * h + head * DH, 1.f, lane);
    const T* k = qkv + (size_t)first * ld + h + head / group * DH;
    attention_dq_row<T, (DH + kWave - 1) / kWave, 8>(
        [&](int e) { return q.broadcast(e); }, [&](int e) { return g.broadcast(e); }, k, k + hkv, ld, lse[(size_t)head * plan.rows + i],
        sign * delta[(size_t)head * plan.rows + i], i - first, dh, lane, scale, dqkv + (size_t)i * ld + head * DH);
  }
}
// Which of the key rows that have elements of dK (of dV) that are not finite are to be redone: not those that are NaN altogether, because a query
// row's own lse is, or for dK its delta.  lse and delta: those of row `key` of the first of the n heads, `rows` apart.
__device__ __forceinline__ uint32_t keys_to_redo(uint32_t bad_k, uint32_t bad_v, const float* __restrict__ lse,
                                                 const float* __restrict__ delta, int key, int n, int rows) {
  if (!(bad_k | bad_v)) return 0;
  bool lse_nan = false, delta_nan = false;
  for (int g = 0; g < n; ++g) {
    lse_nan = lse_nan || is_nan(lse[(size_t)g * rows + key]);
    delta_nan = delta_nan || is_nan(delta[(size_t)g * rows + key]);
  }
  return (bad_k & ~rows_to_redo(lse_nan || delta_nan, 32)) | (bad_v & ~rows_to_redo(lse_nan, 32));
}
// Key rows; the heads of the group begin at `head`.
template <typename T, int DH>
__device__ __forceinline__ void redo_packed_key_rows(uint32_t redo, int row0, PackedPlan plan, const T* __restrict__ qkv,
                                                     const T* __restrict__ d_o, const float* __restrict__ lse,
                                                     const float* __restrict__ delta, T* __restrict__ dk, T* __restrict__ dv, int ld_out,
                                                     int h, int hkv, int group, int n_heads, int head, float scale, float sign) {
  while (redo) {
    const int j = row0 + __builtin_ctz(redo), last = __builtin_amdgcn_readfirstlane(plan.end()[j]) - 1, ld = h + 2 * hkv;
    redo &= redo - 1;
    int dh = DH, lane = (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
    asm volatile("" : "+s"(dh));  // a loop, not DH times its body
    bool nan = false;  // a row of d_o that is NaN: its own key's gradients are NaN too
    for (int g = 0; g < n_heads; ++g) nan = nan || all_nan<T, DH>(d_o + (size_t)j * h + (head + g) * DH, lane);
    if (nan) {
      write_nan<T, DH>(dk + (size_t)j * ld_out, lane);
      write_nan<T, DH>(dv + (size_t)j * ld_out, lane);
      continue;
    }
    const T* k = qkv + (size_t)j * ld + h + head / group * DH;
    const HeldRow<DH> key(k, scale, lane), value(k + hkv, 1.f, lane);
    attention_key_row<T, (DH + kWave - 1) / kWave, 8>(
        [&](int e) { return key.broadcast(e); }, [&](int e) { return value.broadcast(e); }, qkv + head * DH, d_o + head * DH, ld, h,
        lse + (size_t)head * plan.rows, delta + (size_t)head * plan.rows, plan.rows, n_heads, j, last, dh, lane, scale, sign,
        dk + (size_t)j * ld_out, dv + (size_t)j * ld_out);
  }
}

}  // namespace po
