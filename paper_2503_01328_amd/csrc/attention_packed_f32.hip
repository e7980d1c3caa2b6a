// fp32 causal attention of packed sequences on the matrix cores (full fp32 products and sums), forward and backward.
//
// Masks and block order are those of attention_packed.hip, tiles, operand layouts and the four waves that split a block's tiles those of
// attention_f32.hip: a block owns 32 rows, wave w takes every fourth tile and reads its own copy of it, partial results are added in wave
// order.  Bound by the chain of tiles of the longest sequence while the launch does not fill the chip: 12 heads of 64 over 4, 1000 rows of
// 4 sequences, forward 22 us, backward 54 with its sums, against 13 us of products at the rate of a large one.
// Eight waves for heads of 64, which LDS has room for, gain where chains of tiles are long for the launch (this shape's backward with
// whole groups 61.1 -> 55.9 us) and lose elsewhere (16 heads, 4000 rows of 60 sequences 111 -> 158, 32 heads, 3000 rows 1090 -> 1176).
#include <algorithm>

#include "attention_f32_tile.h"
#include "attention_packed_rows.h"

namespace po {

template <int DH>
__global__ __launch_bounds__(256, 2) void packed_f32_fwd_kernel(const float* __restrict__ qkv, const int* words, float* __restrict__ o,
                                                                float* __restrict__ lse, int rows, int h, int hkv, int group,
                                                                float scale) {
  constexpr int DT = DH / 32, PART = 2 * kTileBytes<DH> / 4;
  // per wave a tile of K and one of V, later its partial output; then the waves' maxima and row sums, rows to redo
  extern __shared__ __align__(16) float lds[];
  const PackedPlan plan{words, rows};
  const int total = plan.total();
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  const int n_heads = h / DH, head = blockIdx.x % n_heads, at = blockIdx.x / n_heads;
  if (total == 0) return;
  const int q0 = plan.key_order()[at >> 2].x * kPlanBlock + (3 - (at & 3)) * 32;
  if (q0 >= total) return;
  const int q = q0 + (lane & 31), ld = h + 2 * hkv, last = total - 1;
  const int first = plan.first()[q], first_lo = plan.first()[q0], first_hi = plan.first()[min(q0 + 31, last)];
  const int t0 = first_lo / 32, t_end = q0 / 32 + 1;
  const float* kbase = qkv + h + (head / group) * DH;
  const float* vbase = kbase + hkv;
  const char* bytes = reinterpret_cast<const char*>(lds);
  const LaneReads<DH> reads(wave * PART * 4, lane);
  const unsigned k_lds = __builtin_amdgcn_readfirstlane((int)lds_byte(lds + wave * PART)), v_lds = k_lds + kTileBytes<DH>;
  auto request = [&](int t) {
    request_tile<DH>(k_lds, kbase, ld, 32 * t, last, lane);
    request_tile<DH>(v_lds, vbase, ld, 32 * t, last, lane);
  };
  if (t0 + wave < t_end) request(t0 + wave);
  f32x4 qf[DH / 8];
  load_pieces<DH>(qf, qkv + (size_t)min(q, last) * ld + head * DH, half);
  f32x16 acc[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d) acc[d] = zero16();
  float m_run = -INFINITY, l_run = 0.f;
  for (int t = t0 + wave; t < t_end; t += 4) {
    wait_loads<0>();
    f32x16 p = dot_tile<DH, 0>(bytes, reads, qf);
    if (t == t_end - 1 || 32 * t < first_hi) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int key = 32 * t + 8 * (e >> 2) + 4 * half + (e & 3);
        if (key > q || key < first) p[e] = -INFINITY;
      }
    }
    float mx = m_run;
#pragma unroll
    for (int e = 0; e < 16; ++e) mx = fmaxf(mx, p[e]);
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    const float ref = mx == -INFINITY ? 0.f : mx;  // a tile that the row does not see adds nothing
    float alpha = exp_scaled(m_run - ref, scale), sum = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      p[e] = exp_scaled(p[e] - ref, scale);
      sum += p[e];
    }
    m_run = mx;
    l_run = l_run * alpha + sum;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[d][e] *= alpha;
    accumulate_rows<DH, 1>(acc, bytes, reads, p);
    wait_lds_reads();
    if (t + 4 < t_end) request(t + 4);
  }
  put_partial<DT>(lds + wave * PART, acc, lane);
  float* stat = lds + 4 * PART;
  uint32_t* redo_of = reinterpret_cast<uint32_t*>(stat + 8 * 64);
  const uint32_t redo_mine = rows_to_redo(not_finite<DT>(acc), total - q0);
  if (lane == 0) redo_of[wave] = redo_mine;
  stat[wave * 64 + lane] = m_run;
  stat[(4 + wave) * 64 + lane] = l_run + __shfl_xor(l_run, 32, 64);
  __syncthreads();
  // Wave w finishes registers 4 w .. 4 w + 3 (columns 32 d + 8 w + 4 half ..) of every lane's row.
  float m = stat[lane], f[4], l = 0.f;
#pragma unroll
  for (int w = 1; w < 4; ++w) m = fmaxf(m, stat[w * 64 + lane]);  // the wave of the diagonal has seen the row's own key
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    f[w] = exp_scaled(stat[w * 64 + lane] - m, scale);
    l += stat[(4 + w) * 64 + lane] * f[w];
  }
  const uint32_t redo = all_redo(redo_of) & rows_to_redo(!is_nan(l), 32);
  if (q <= last && !(redo >> (lane & 31) & 1)) {
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      f32x4 v;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float x = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) x += lds[w * PART + (d * 16 + 4 * wave + r) * 64 + lane] * f[w];
        v[r] = x / l;
      }
      *reinterpret_cast<f32x4*>(o + (size_t)q * h + head * DH + 32 * d + 8 * wave + 4 * half) = v;
    }
  }
  if (wave == 0 && half == 0 && q <= last) lse[(size_t)head * rows + q] = fmaf(m, scale, __logf(l));
  if (redo) redo_packed_forward_rows<float, DH>(share_of(redo, wave), q0, plan, qkv, o, h, hkv, group, head, scale);
}

// 32 query rows of a head from q0 on.
template <int DH>
__device__ __forceinline__ void packed_f32_dq_block(float* lds, int q0, int head, PackedPlan plan, int total,
                                                    const float* __restrict__ qkv, const float* __restrict__ d_o,
                                                    const float* __restrict__ lse, const float* __restrict__ delta,
                                                    float* __restrict__ dqkv, int h, int hkv, int group, float scale) {
  constexpr int DT = DH / 32, PART = 2 * kTileBytes<DH> / 4;  // a wave's tiles of K and V, later its partial result
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  const int q = q0 + (lane & 31), ld = h + 2 * hkv, last = total - 1, qc = min(q, last);
  const int first = plan.first()[q], first_lo = plan.first()[q0], first_hi = plan.first()[min(q0 + 31, last)];
  const int t0 = first_lo / 32, t_end = q0 / 32 + 1;
  const float* kbase = qkv + h + (head / group) * DH;
  const float* vbase = kbase + hkv;
  const char* bytes = reinterpret_cast<const char*>(lds);
  const LaneReads<DH> reads(wave * PART * 4, lane);
  const unsigned k_lds = __builtin_amdgcn_readfirstlane((int)lds_byte(lds + wave * PART)), v_lds = k_lds + kTileBytes<DH>;
  auto request = [&](int t) {
    request_tile<DH>(k_lds, kbase, ld, 32 * t, last, lane);
    request_tile<DH>(v_lds, vbase, ld, 32 * t, last, lane);
  };
  if (t0 + wave < t_end) request(t0 + wave);
  f32x4 qf[DH / 8], dof[DH / 8];
  load_pieces<DH>(qf, qkv + (size_t)qc * ld + head * DH, half);
  load_pieces<DH>(dof, d_o + (size_t)qc * h + head * DH, half);
  const float lse_q = lse[(size_t)head * plan.rows + qc], delta_q = delta[(size_t)head * plan.rows + qc];
  f32x16 dq[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d) dq[d] = zero16();
  for (int t = t0 + wave; t < t_end; t += 4) {
    wait_loads<0>();
    f32x16 p = dot_tile<DH, 0>(bytes, reads, qf);
    f32x16 ds = dot_tile<DH, 1>(bytes, reads, dof);
    const bool masked = t == t_end - 1 || 32 * t < first_hi;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int key = 32 * t + 8 * (e >> 2) + 4 * half + (e & 3);
      ds[e] = __builtin_amdgcn_exp2f(fmaf(p[e], scale, -lse_q) * kLog2e) * (ds[e] - delta_q);
      if (masked && (key > q || key < first)) ds[e] = 0.f;
    }
    accumulate_rows<DH, 0>(dq, bytes, reads, ds);
    wait_lds_reads();
    if (t + 4 < t_end) request(t + 4);
  }
  put_partial<DT>(lds + wave * PART, dq, lane);
  uint32_t* redo_of = reinterpret_cast<uint32_t*>(lds + 4 * PART);
  const uint32_t redo_mine = rows_to_redo(not_finite<DT>(dq) && !is_nan(lse_q + delta_q), total - q0);
  if (lane == 0) redo_of[wave] = redo_mine;
  __syncthreads();
  const uint32_t redo = all_redo(redo_of);
  if (q <= last && !(redo >> (lane & 31) & 1)) {
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      f32x4 v;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float x = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) x += lds[w * PART + (d * 16 + 4 * wave + r) * 64 + lane];
        v[r] = x * scale;
      }
      *reinterpret_cast<f32x4*>(dqkv + (size_t)q * ld + head * DH + 32 * d + 8 * wave + 4 * half) = v;
    }
  }
  if (redo) redo_packed_dq_rows<float, DH>(share_of(redo, wave), q0, plan, qkv, d_o, lse, delta, dqkv, h, hkv, group, head, scale, 1.f);
}

// 32 keys from k0 on of the key/value head that `heads` query heads from head0 on read; its waves walk the query tiles of those.  `out`:
// column 0 of dK of row 0, dV hkv columns further, rows ld_out apart.
template <int DH>
__device__ __forceinline__ void packed_f32_dkv_block(float* lds, int k0, int head0, int heads, PackedPlan plan, int total,
                                                     const float* __restrict__ qkv, const float* __restrict__ d_o,
                                                     const float* __restrict__ lse, const float* __restrict__ delta,
                                                     float* __restrict__ out, int ld_out, int h, int hkv, int group, float scale) {
  constexpr int DT = DH / 32, PART = kTileBytes<DH> / 4;  // a wave's tiles of Q and dO, later its partial results
  int lane = threadIdx.x & 63, half = lane >> 5, key = k0 + (lane & 31);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), ld = h + 2 * hkv, last = total - 1, kv_head = head0 / group;
  const int end = plan.end()[key], end_lo = plan.end()[k0], end_hi = plan.end()[min(k0 + 31, last)];
  const int t0 = k0 / 32, n_q = (end_hi - 1) / 32 + 1 - t0, n_it = heads * n_q;
  const char* bytes = reinterpret_cast<const char*>(lds);
  const LaneReads<DH> reads(wave * 2 * PART * 4, lane);
  const unsigned q_lds = __builtin_amdgcn_readfirstlane((int)lds_byte(lds + wave * 2 * PART)), do_lds = q_lds + kTileBytes<DH>;
  auto request = [&](int it) {
    const int g = it / n_q, q0 = (t0 + it - g * n_q) * 32, head = head0 + g;
    request_tile<DH>(q_lds, qkv + head * DH, ld, q0, last, lane);
    request_tile<DH>(do_lds, d_o + head * DH, h, q0, last, lane);
  };
  if (wave < n_it) request(wave);
  f32x4 kf[DH / 8], vf[DH / 8];
  const float* krow = qkv + (size_t)min(key, last) * ld + h + kv_head * DH;
  load_pieces<DH>(kf, krow, half);
  load_pieces<DH>(vf, krow + hkv, half);
  f32x16 dk[DT], dv[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d) dk[d] = dv[d] = zero16();
  for (int it = wave; it < n_it; it += 4) {
    const int g = it / n_q, q0 = (t0 + it - g * n_q) * 32, head = head0 + g;
    // lse of row lane % 32 in the lower half-wave, its delta in the upper
    const float stat = (half ? delta : lse)[(size_t)head * plan.rows + min(q0 + (lane & 31), last)];
    wait_loads<0>();
    f32x16 p = dot_tile<DH, 0>(bytes, reads, kf);
    f32x16 ds = dot_tile<DH, 1>(bytes, reads, vf);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int row = 8 * (e >> 2) + 4 * half + (e & 3);
      p[e] = __builtin_amdgcn_exp2f(fmaf(p[e], scale, -__shfl(stat, row, 64)) * kLog2e);
      ds[e] = p[e] * (ds[e] - __shfl(stat, 32 + row, 64));
    }
    if (q0 == k0 || q0 + 32 > end_lo) {  // the diagonal, or rows past the end of a sequence
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int q = q0 + 8 * (e >> 2) + 4 * half + (e & 3);
        if (key > q || q >= end) p[e] = ds[e] = 0.f;  // dS too: 0 times the dP of a row that is not finite is no 0
      }
    }
    accumulate_rows<DH, 1>(dv, bytes, reads, p);
    accumulate_rows<DH, 0>(dk, bytes, reads, ds);
    wait_lds_reads();
    if (it + 4 < n_it) request(it + 4);
  }
  // rebuilt rather than kept (and, for heads of 128, spilled) across the loop
  lane = (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
  half = lane >> 5;
  key = k0 + (lane & 31);
  put_partial<DT>(lds + wave * 2 * PART, dk, lane);
  put_partial<DT>(lds + wave * 2 * PART + PART, dv, lane);
  uint32_t* redo_of = reinterpret_cast<uint32_t*>(lds + 8 * PART);
  const uint32_t bad_k = rows_to_redo(not_finite<DT>(dk), total - k0), bad_v = rows_to_redo(not_finite<DT>(dv), total - k0);
  if (lane == 0) redo_of[wave] = bad_k, redo_of[4 + wave] = bad_v;
  __syncthreads();
  const size_t stat_at = (size_t)head0 * plan.rows;
  const uint32_t redo = keys_to_redo(all_redo(redo_of), all_redo(redo_of + 4), lse + stat_at,
                                     delta + stat_at, min(key, last), heads, plan.rows);
  if (key <= last && !(redo >> (lane & 31) & 1)) {
    float* to = out + (size_t)key * ld_out + 8 * wave + 4 * half;
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      f32x4 vk, vv;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float x = 0.f, y = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          x += lds[w * 2 * PART + (d * 16 + 4 * wave + r) * 64 + lane];
          y += lds[w * 2 * PART + PART + (d * 16 + 4 * wave + r) * 64 + lane];
        }
        vk[r] = x * scale;
        vv[r] = y;
      }
      *reinterpret_cast<f32x4*>(to + 32 * d) = vk;
      *reinterpret_cast<f32x4*>(to + hkv + 32 * d) = vv;
    }
  }
  if (redo)
    redo_packed_key_rows<float, DH>(share_of(redo, wave), k0, plan, qkv, d_o, lse, delta, out, out + hkv, ld_out, h, hkv, group, heads, head0,
                                    scale, 1.f);
}

template <int DH>
__global__ __launch_bounds__(256, DH > 64 ? 1 : 2) void packed_f32_bwd_kernel(const float* __restrict__ qkv, const int* words,
                                                                              const float* __restrict__ d_o,
                                                                              const float* __restrict__ lse,
                                                                              const float* __restrict__ delta, float* __restrict__ dqkv,
                                                                              float* __restrict__ partials, int heads, int rows, int h,
                                                                              int hkv, int group, float scale, int dkv_blocks) {
  extern __shared__ __align__(16) float lds[];
  const PackedPlan plan{words, rows};
  const int total = plan.total();
  if (total == 0) return;
  const bool dkv = (int)blockIdx.x < dkv_blocks;
  const int x = dkv ? blockIdx.x : blockIdx.x - dkv_blocks, n_x = dkv ? h / DH / heads : h / DH, head = x % n_x, at = x / n_x;
  // of a block of 128 rows the first keys and the last queries meet the most
  const int row0 = dkv ? plan.query_order()[at >> 2].x * kPlanBlock + (at & 3) * 32
                       : plan.key_order()[at >> 2].x * kPlanBlock + (3 - (at & 3)) * 32;
  if (row0 >= total) return;
  if (dkv) {
    const int head0 = head * heads, part = head0 % group / heads, column = head0 / group * DH;
    float* out = partials ? partials + (size_t)part * rows * 2 * hkv + column : dqkv + h + column;
    packed_f32_dkv_block<DH>(lds, row0, head0, heads, plan, total, qkv, d_o, lse, delta, out, partials ? 2 * hkv : h + 2 * hkv, h, hkv, group,
                             scale);
  } else
    packed_f32_dq_block<DH>(lds, row0, head, plan, total, qkv, d_o, lse, delta, dqkv, h, hkv, group, scale);
}

// dK and dV of every row of a sequence: the sum of the query heads' partial results [parts][rows][2 hkv], in their order.
__global__ __launch_bounds__(256) void packed_f32_sum_kernel(const float* __restrict__ partials, const int* words, float* __restrict__ dqkv,
                                                             int parts, int rows, int h, int hkv) {
  const PackedPlan plan{words, rows};
  const int per_row = hkv / 2;  // vectors
  const size_t at = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= (size_t)plan.total() * per_row) return;
  const size_t row = at / per_row, c = (at - row * per_row) * 4;
  f32x4 v = *reinterpret_cast<const f32x4*>(partials + row * 2 * hkv + c);
  for (int p = 1; p < parts; ++p) v += *reinterpret_cast<const f32x4*>(partials + ((size_t)p * rows + row) * 2 * hkv + c);
  *reinterpret_cast<f32x4*>(dqkv + row * (h + 2 * hkv) + h + c) = v;
}

// ---- host side -------------------------------------------------------------------------------------------------
// Heads that share keys: a dK/dV block a query head, added up afterwards, while the blocks of whole groups, whose chains are that much
// longer, would fill half of the CUs at most.  Backward, us, whole groups / by heads: 12 heads of 64 over 4, 1000 rows of 4 sequences (128
// blocks) 61 / 45; 16 heads of 128 over 4, 2000 rows (252) 263 / 272; 32 heads of 128 over 8, 2048 rows (512) 1184 / 1249.
static int rows_by_heads(int n_heads, int n_kv_heads) {  // up to how many rows
  return n_heads > n_kv_heads ? 128 / n_kv_heads * 32 : 0;
}
static bool by_heads(int rows, int n_heads, int n_kv_heads) { return rows <= rows_by_heads(n_heads, n_kv_heads); }
// What any count of rows up to `rows` needs: a workspace for a program's largest batch serves its smaller ones.
size_t attention_packed_f32_partials(int rows, int h, int n_heads, int n_kv_heads) {
  return (size_t)std::min(rows, rows_by_heads(n_heads, n_kv_heads)) * 2 * h;  // group * 2 hkv columns
}

template <int DH>
static bool forward_f32(const float* qkv, const int* plan, float* o, float* lse, int rows, int h, int n_heads, int n_kv_heads,
                        hipStream_t stream) {
  constexpr int smem = 8 * kTileBytes<DH> + (8 * 64 + 4) * 4;
  static LdsLimit lds;
  if (!lds.allow(packed_f32_fwd_kernel<DH>, smem)) return false;
  packed_f32_fwd_kernel<DH><<<n_heads * ceil_div(rows, kPlanBlock) * 4, 256, smem, stream>>>(
      qkv, plan, o, lse, rows, h, n_kv_heads * DH, n_heads / n_kv_heads, 1.0f / sqrtf((float)DH));
  return launch_ok("packed_f32_fwd_kernel");
}

template <int DH>
static bool backward_f32(const float* qkv, const int* plan, const float* lse, const float* delta, const float* d_o, float* dqkv,
                         float* partials, int rows, int h, int n_heads, int n_kv_heads, hipStream_t stream) {
  constexpr int smem = 8 * kTileBytes<DH> + 32;
  static LdsLimit lds;
  if (!lds.allow(packed_f32_bwd_kernel<DH>, smem)) return false;
  const int tiles = ceil_div(rows, kPlanBlock) * 4, group = n_heads / n_kv_heads, hkv = n_kv_heads * DH;
  const bool split = by_heads(rows, n_heads, n_kv_heads);
  const int heads = split ? 1 : group, dkv_blocks = n_heads / heads * tiles;
  packed_f32_bwd_kernel<DH><<<dkv_blocks + n_heads * tiles, 256, smem, stream>>>(qkv, plan, d_o, lse, delta, dqkv, split ? partials : nullptr,
                                                                                heads, rows, h, hkv, group, 1.0f / sqrtf((float)DH),
                                                                                dkv_blocks);
  if (split)
    packed_f32_sum_kernel<<<(unsigned)(((size_t)rows * hkv / 2 + 255) / 256), 256, 0, stream>>>(partials, plan, dqkv, group, rows, h, hkv);
  return launch_ok("packed_f32_bwd_kernel");
}

bool attention_packed_forward_f32(const float* qkv, const int* plan, float* o, float* lse, int rows, int h, int n_heads,
                                  int n_kv_heads, hipStream_t stream) {
  auto launch = h / n_heads == 128 ? forward_f32<128> : forward_f32<64>;
  return launch(qkv, plan, o, lse, rows, h, n_heads, n_kv_heads, stream);
}

bool attention_packed_backward_f32(const float* qkv, const int* plan, const float* lse, const float* delta, const float* d_o,
                                   float* dqkv, float* partials, int rows, int h, int n_heads, int n_kv_heads, hipStream_t stream) {
  auto launch = h / n_heads == 128 ? backward_f32<128> : backward_f32<64>;
  return launch(qkv, plan, lse, delta, d_o, dqkv, partials, rows, h, n_heads, n_kv_heads, stream);
}

}  // namespace po
