// bf16 causal attention of packed sequences on the matrix cores, forward and backward: rows of many sequences back to back, row i sees
// keys first(i) .. i, where first(i) is the first row of its sequence (packed_plan.h).
//
// Blocks and tiles are cut from the packed axis, not from each sequence: a block of rows may hold the end of one sequence and several
// whole ones, and walks the tiles from the first key that any of its rows sees to the diagonal.  That wastes no rows of a block on
// short sequences, and the bounds first(i), end(j) of a row, one integer per lane, do all of the masking; tiles that every row sees whole pay
// nothing for it.  Operand layouts are those of attention_mfma.hip.
//
// P and dS are rounded to bf16 once on their way into the second product, as the inputs of every product here are; sums, maxima and
// accumulators are fp32.
// A key or value that is not finite reaches the rows that see it and no other, nor does a row of d_o reach another sequence: results that
// are not finite are redone row by row (attention_packed_rows.h).  Rows behind the last sequence read as zeros and are never written.
#include "attention_few_tile.h"
#include "attention_packed_rows.h"

namespace po {

template <int DH>
__global__ __launch_bounds__((64 * Few<DH, true>::W)) void packed_few_fwd_kernel(const bf16* __restrict__ qkv, const int* words,
                                                                                bf16* __restrict__ o, float* __restrict__ lse,
                                                                                int rows, int h, int hkv, int group, float scale) {
  using F = Few<DH, true>;
  constexpr int DT = DH / 32, W = F::W, PART = F::NS * F::STAGE / 4;
  extern __shared__ __align__(16) char smem[];
  const PackedPlan plan{words, rows};
  const int total = plan.total();
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  const int n_heads = h / DH, head = blockIdx.x % n_heads, at = blockIdx.x / n_heads;
  if (total == 0) return;
  const int q0 = plan.key_order()[at >> 2] * kPlanBlock + (3 - (at & 3)) * kRows;
  if (q0 >= total) return;
  const int q = q0 + (lane & 31), ld = h + 2 * hkv, last = total - 1;
  const int first = plan.first()[q], first_lo = plan.first()[q0], first_hi = plan.first()[min(q0 + kRows - 1, last)];
  const int t0 = first_lo / kRows, t_end = q0 / kRows + 1;
  const float c = scale * kLog2e;
  const bf16* kbase = qkv + h + (head / group) * DH;
  const bf16* vbase = kbase + hkv;
  char* stages = smem + wave * F::NS * F::STAGE;
  const unsigned stages_lds = __builtin_amdgcn_readfirstlane((int)lds_byte(stages));
  const TileLoads<DH> loads(ld, lane);
  auto request = [&](int i, int t) {
    loads.request(stages_lds + i % F::NS * F::STAGE, kbase, ld, kRows * t, total);
    loads.request(stages_lds + i % F::NS * F::STAGE + F::TILE, vbase, ld, kRows * t, total);
  };
#pragma unroll
  for (int i = 0; i < F::NS; ++i)
    if (t0 + wave + i * W < t_end) request(i, t0 + wave + i * W);
  bf16x8 qf[DH / 16];
  load_row<DH>(qf, qkv + (size_t)min(q, last) * ld + head * DH, half);  // (rows past the end: computed, not stored)
  f32x16 acc[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d) acc[d] = zero16();
  float m_run = -INFINITY, mc_run = -INFINITY, l_run = 0.f;
  for (int t = t0 + wave, i = 0; t < t_end; t += W, ++i) {
    const bool more = t + W < t_end;
    if (F::NS == 1) wait_loads<F::LOADS>();  // K is there, V may be on its way
    else if (more) wait_loads<2 * F::LOADS>();
    else wait_loads<0>();
    const char* ktile = stages + i % F::NS * F::STAGE;
    f32x16 p = dot_tile<DH>(ktile, qf, zero16(), lane);
    if (F::NS == 1 && more) {
      wait_lds_reads();
      loads.request(stages_lds, kbase, ld, kRows * (t + W), total);
    }
    if (t == t_end - 1 || kRows * t < first_hi) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int key = kRows * t + 8 * (e >> 2) + 4 * half + (e & 3);
        if (key > q || key < first) p[e] = -INFINITY;
      }
    }
    float mx = m_run;
#pragma unroll
    for (int e = 0; e < 16; ++e) mx = fmaxf(mx, p[e]);
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    const float mc_new = exponent_of(mx, c), mc = mx == -INFINITY ? 0.f : mc_new;  // a tile that the row does not see adds nothing
    const float alpha = fast_exp2(mc_run - mc);
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      p[e] = fast_exp2(fmaf(p[e], c, -mc));
      sum += p[e];
    }
    m_run = mx;
    mc_run = mc_new;
    l_run = l_run * alpha + sum;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[d][e] *= alpha;
    if (F::NS == 1) {
      if (more) wait_loads<F::LOADS>();
      else wait_loads<0>();
    }
    accumulate_tile<DH, false>(acc, ktile + F::TILE, p, lane);
    if (F::NS == 1 && more) {
      wait_lds_reads();
      loads.request(stages_lds + F::TILE, vbase, ld, kRows * (t + W), total);
    } else if (t + F::NS * W < t_end) {
      wait_lds_reads();
      request(i, t + F::NS * W);
    }
  }
  float* part = reinterpret_cast<float*>(smem);
  put_partial<DT>(part + wave * PART, acc, lane);
  float* stat = reinterpret_cast<float*>(smem + F::AFTER);
  uint32_t* redo_of = reinterpret_cast<uint32_t*>(stat + 2 * W * 64);
  stat[wave * 64 + lane] = m_run;
  stat[(W + wave) * 64 + lane] = l_run + __shfl_xor(l_run, 32, 64);
  const uint32_t mine = rows_to_redo(not_finite<DT>(acc), total - q0);
  if (lane == 0) redo_of[wave] = mine;
  __syncthreads();
  // Wave w finishes register groups w, w + W, ..: group g is columns 32 (g / 4) + 8 (g % 4) + 4 half .. of every lane's row.
  float m = stat[lane], f[W], l = 0.f;
#pragma unroll
  for (int w = 1; w < W; ++w) m = fmaxf(m, stat[w * 64 + lane]);  // the wave of the diagonal has seen the row's own key
  const float mc = exponent_of(m, c);
#pragma unroll
  for (int w = 0; w < W; ++w) {
    f[w] = fast_exp2(exponent_of(stat[w * 64 + lane], c) - mc);
    l += stat[(W + w) * 64 + lane] * f[w];
  }
  const uint32_t redo = all_redo<W>(redo_of) & rows_to_redo(!is_nan(l), 32);
  if (redo) redo_packed_forward_rows<bf16, DH>(share_of<W>(redo, wave), q0, plan, qkv, o, lse, h, hkv, group, head, scale);
  if (q > last || (redo >> (lane & 31) & 1)) return;
  const float inv = 1.0f / l;
#pragma unroll
  for (int g = wave; g < 4 * DT; g += W) {
    f32x4 v;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float x = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) x += part[w * PART + (4 * g + r) * 64 + lane] * f[w];
      v[r] = x * inv;
    }
    store4(o + (size_t)q * h + head * DH + 8 * g + 4 * half, v);
  }
  if (wave == 0 && half == 0) {
    // by whichever constant is the more exact: 1 / 8, or c ln 2, whose two roundings all but cancel
    const float log_l = __logf(l), ln2 = 0.6931471805599453f;
    lse[(size_t)head * rows + q] = DH == 64 ? m * scale + fmaf(fmaf(-m, c, mc), ln2, log_l) : fmaf(mc, ln2, log_l);
  }
}

// 32 query rows of a head from q0 on.
template <int DH>
__device__ __forceinline__ void packed_few_dq_block(char* smem, int q0, int head, PackedPlan plan, int total,
                                                    const bf16* __restrict__ qkv, const bf16* __restrict__ d_o,
                                                    const float* __restrict__ lse, const float* __restrict__ delta,
                                                    bf16* __restrict__ dqkv, int h, int hkv, int group, float scale) {
  using F = Few<DH>;
  constexpr int DT = DH / 32, W = F::W, PART = F::NS * F::STAGE / 4;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  const int q = q0 + (lane & 31), ld = h + 2 * hkv, last = total - 1, qc = min(q, last);
  const int first = plan.first()[q], first_lo = plan.first()[q0], first_hi = plan.first()[min(q0 + kRows - 1, last)];
  const int t0 = first_lo / kRows, t_end = q0 / kRows + 1;
  const float c = scale * kLog2e;
  const bf16* kbase = qkv + h + (head / group) * DH;
  const bf16* vbase = kbase + hkv;
  char* stages = smem + wave * F::NS * F::STAGE;
  const unsigned stages_lds = __builtin_amdgcn_readfirstlane((int)lds_byte(stages));
  const TileLoads<DH> loads(ld, lane);
  auto request = [&](int i, int t) {
    loads.request(stages_lds + i % F::NS * F::STAGE, kbase, ld, kRows * t, total);
    loads.request(stages_lds + i % F::NS * F::STAGE + F::TILE, vbase, ld, kRows * t, total);
  };
#pragma unroll
  for (int i = 0; i < F::NS; ++i)
    if (t0 + wave + i * W < t_end) request(i, t0 + wave + i * W);
  bf16x8 qf[DH / 16], dof[DH / 16];
  load_row<DH>(qf, qkv + (size_t)qc * ld + head * DH, half);
  load_row<DH>(dof, d_o + (size_t)qc * h + head * DH, half);
  const float lse_q = lse[(size_t)head * plan.rows + qc] * kLog2e, delta_q = delta[(size_t)head * plan.rows + qc];
  f32x16 dq[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d) dq[d] = zero16();
  for (int t = t0 + wave, i = 0; t < t_end; t += W, ++i) {
    if (t + W < t_end) wait_loads<2 * F::LOADS>();
    else wait_loads<0>();
    const char* ktile = stages + i % F::NS * F::STAGE;
    f32x16 p = dot_tile<DH>(ktile, qf, zero16(), lane);
    f32x16 ds = dot_tile<DH>(ktile + F::TILE, dof, zero16(), lane);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      p[e] = fast_exp2(p[e] * c - lse_q);
      ds[e] = p[e] * (ds[e] - delta_q);
    }
    if (t == t_end - 1 || kRows * t < first_hi) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int key = kRows * t + 8 * (e >> 2) + 4 * half + (e & 3);
        if (key > q || key < first) ds[e] = 0.f;
      }
    }
    accumulate_tile<DH, false>(dq, ktile, ds, lane);
    wait_lds_reads();
    if (t + F::NS * W < t_end) request(i, t + F::NS * W);
  }
  float* part = reinterpret_cast<float*>(smem);
  put_partial<DT>(part + wave * PART, dq, lane);
  uint32_t* redo_of = reinterpret_cast<uint32_t*>(smem + F::AFTER);
  const uint32_t mine = rows_to_redo(not_finite<DT>(dq) && !is_nan(lse_q + delta_q), total - q0);
  if (lane == 0) redo_of[wave] = mine;
  __syncthreads();
  const uint32_t redo = all_redo<W>(redo_of);
  if (redo) redo_packed_dq_rows<bf16, DH>(share_of<W>(redo, wave), q0, plan, qkv, d_o, lse, delta, dqkv, h, hkv, group, head, scale);
  if (q > last || (redo >> (lane & 31) & 1)) return;
#pragma unroll
  for (int g = wave; g < 4 * DT; g += W) {
    f32x4 v;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float x = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) x += part[w * PART + (4 * g + r) * 64 + lane];
      v[r] = x * scale;
    }
    store4(dqkv + (size_t)q * ld + head * DH + 8 * g + 4 * half, v);
  }
}

// 32 keys of a key/value head from k0 on; its waves walk the query tiles of every query head that reads it.
template <int DH>
__device__ __forceinline__ void packed_few_dkv_block(char* smem, int k0, int kv_head, PackedPlan plan, int total,
                                                     const bf16* __restrict__ qkv, const bf16* __restrict__ d_o,
                                                     const float* __restrict__ lse, const float* __restrict__ delta,
                                                     bf16* __restrict__ dqkv, int h, int hkv, int group, float scale) {
  using F = Few<DH>;
  constexpr int DT = DH / 32, W = F::W, PART = F::NS * F::STAGE / 4;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  const int key = k0 + (lane & 31), ld = h + 2 * hkv, last = total - 1, head0 = kv_head * group;
  const int end = plan.end()[key], end_lo = plan.end()[k0], end_hi = plan.end()[min(k0 + kRows - 1, last)];
  const int t0 = k0 / kRows, n_q = (end_hi - 1) / kRows + 1 - t0, n_it = group * n_q;
  const float c = scale * kLog2e, from_lse = -1.0f / scale;
  char* stages = smem + wave * F::NS * F::STAGE;
  char* stats = smem + F::AFTER + wave * F::NS * 256;  // per stage lse and delta of the tile's 32 rows
  const unsigned stages_lds = __builtin_amdgcn_readfirstlane((int)lds_byte(stages));
  const unsigned stats_lds = __builtin_amdgcn_readfirstlane((int)lds_byte(stats));
  const TileLoads<DH> q_loads(ld, lane), do_loads(h, lane);
  const float* stat_of = half ? delta : lse;
  auto request = [&](int i, int it) {
    const int g = it / n_q, q0 = (t0 + it - g * n_q) * kRows, head = head0 + g;
    q_loads.request(stages_lds + i % F::NS * F::STAGE, qkv + head * DH, ld, q0, total);
    do_loads.request(stages_lds + i % F::NS * F::STAGE + F::TILE, d_o + head * DH, h, q0, total);
    float_to_lds(stats_lds + i % F::NS * 256, stat_of + (size_t)head * plan.rows + min(q0 + (lane & 31), last));
  };
#pragma unroll
  for (int i = 0; i < F::NS; ++i)
    if (wave + i * W < n_it) request(i, wave + i * W);
  bf16x8 kf[DH / 16], vf[DH / 16];
  const bf16* krow = qkv + (size_t)min(key, last) * ld + h + kv_head * DH;  // (keys past the end: computed, not stored)
  load_row<DH>(kf, krow, half);
  load_row<DH>(vf, krow + hkv, half);
  f32x16 dk[DT], dv[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d) dk[d] = dv[d] = zero16();
  for (int it = wave, i = 0; it < n_it; it += W, ++i) {
    const int g = it / n_q, q0 = (t0 + it - g * n_q) * kRows;
    if (it + W < n_it) wait_loads<2 * F::LOADS + 1>();
    else wait_loads<0>();
    const char* qtile = stages + i % F::NS * F::STAGE;
    const float* stat = reinterpret_cast<const float*>(stats + i % F::NS * 256);
    f32x16 p, ds;  // the row statistics are the initial value: S - lse / scale and dP - delta
#pragma unroll
    for (int b = 0; b < 4; ++b) {  // register 4 b + r is query row 8 b + 4 half + r
      const f32x4 vl = *reinterpret_cast<const f32x4*>(stat + 8 * b + 4 * half);
      const f32x4 vd = *reinterpret_cast<const f32x4*>(stat + 32 + 8 * b + 4 * half);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        p[4 * b + r] = vl[r] * from_lse;
        ds[4 * b + r] = -vd[r];
      }
    }
    p = dot_tile<DH>(qtile, kf, p, lane);
    ds = dot_tile<DH>(qtile + F::TILE, vf, ds, lane);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      p[e] = fast_exp2(p[e] * c);
      ds[e] *= p[e];
    }
    if (q0 == k0 || q0 + kRows > end_lo) {  // the diagonal, or rows past the end of a sequence
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int q = q0 + 8 * (e >> 2) + 4 * half + (e & 3);
        if (key > q || q >= end) p[e] = ds[e] = 0.f;  // dS too: 0 times the dP of a row that is not finite is no 0
      }
    }
    accumulate_tile<DH, false>(dv, qtile + F::TILE, p, lane);
    accumulate_tile<DH, false>(dk, qtile, ds, lane);
    wait_lds_reads();
    if (it + F::NS * W < n_it) request(i, it + F::NS * W);
  }
  float* part = reinterpret_cast<float*>(smem);
  put_partial<DT>(part + wave * PART, dk, lane);
  put_partial<DT>(part + wave * PART + PART / 2, dv, lane);
  uint32_t* redo_of = reinterpret_cast<uint32_t*>(smem + F::AFTER + W * F::NS * 256);
  const uint32_t mine = rows_to_redo(not_finite<DT>(dk) || not_finite<DT>(dv), total - k0);
  if (lane == 0) redo_of[wave] = mine;
  __syncthreads();
  bf16* out = dqkv + h + kv_head * DH;
  const uint32_t redo = all_redo<W>(redo_of);
  if (redo)
    redo_packed_key_rows<bf16, DH>(share_of<W>(redo, wave), k0, plan, qkv, d_o, lse, delta, out, out + hkv, ld, h, hkv, group, group,
                                   head0, scale);
  if (key > last || (redo >> (lane & 31) & 1)) return;
  out += (size_t)key * ld + 4 * half;
#pragma unroll
  for (int g = wave; g < 4 * DT; g += W) {
    f32x4 vk, vv;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float x = 0.f, y = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) {
        x += part[w * PART + (4 * g + r) * 64 + lane];
        y += part[w * PART + PART / 2 + (4 * g + r) * 64 + lane];
      }
      vk[r] = x * scale;
      vv[r] = y;
    }
    store4(out + 8 * g, vk);
    store4(out + hkv + 8 * g, vv);
  }
}

template <int DH>
__global__ __launch_bounds__(64 * Few<DH>::W) void packed_few_bwd_kernel(const bf16* __restrict__ qkv, const int* words,
                                                                        const bf16* __restrict__ d_o, const float* __restrict__ lse,
                                                                        const float* __restrict__ delta, bf16* __restrict__ dqkv,
                                                                        int rows, int h, int hkv, int group, float scale,
                                                                        int dkv_blocks) {
  extern __shared__ __align__(16) char smem[];
  const PackedPlan plan{words, rows};
  const int total = plan.total();
  if (total == 0) return;
  const bool dkv = (int)blockIdx.x < dkv_blocks;
  const int x = dkv ? blockIdx.x : blockIdx.x - dkv_blocks, n_x = dkv ? hkv / DH : h / DH, head = x % n_x, at = x / n_x;
  // of a block of 128 rows the first keys and the last queries meet the most
  const int row0 = dkv ? plan.query_order()[at >> 2] * kPlanBlock + (at & 3) * kRows
                       : plan.key_order()[at >> 2] * kPlanBlock + (3 - (at & 3)) * kRows;
  if (row0 >= total) return;
  if (dkv)
    packed_few_dkv_block<DH>(smem, row0, head, plan, total, qkv, d_o, lse, delta, dqkv, h, hkv, group, scale);
  else
    packed_few_dq_block<DH>(smem, row0, head, plan, total, qkv, d_o, lse, delta, dqkv, h, hkv, group, scale);
}

// ---- host side -------------------------------------------------------------------------------------------------
template <int DH>
static bool few_forward(const bf16* qkv, const int* plan, bf16* o, float* lse, int rows, int h, int n_heads, int n_kv_heads,
                        hipStream_t stream) {
  using F = Few<DH, true>;
  constexpr int smem = F::AFTER + 2 * F::W * 256 + F::W * 4;
  static LdsLimit lds;
  if (!lds.allow(packed_few_fwd_kernel<DH>, smem)) return false;
  packed_few_fwd_kernel<DH><<<n_heads * ceil_div(rows, kPlanBlock) * 4, 64 * F::W, smem, stream>>>(
      qkv, plan, o, lse, rows, h, n_kv_heads * DH, n_heads / n_kv_heads, 1.0f / sqrtf((float)DH));
  return launch_ok("packed_few_fwd_kernel");
}

template <int DH>
static bool few_backward(const bf16* qkv, const int* plan, const float* lse, const float* delta, const bf16* d_o, bf16* dqkv, int rows,
                         int h, int n_heads, int n_kv_heads, hipStream_t stream) {
  using F = Few<DH>;
  constexpr int smem = F::AFTER + F::W * F::NS * 256 + F::W * 4;
  static LdsLimit lds;
  if (!lds.allow(packed_few_bwd_kernel<DH>, smem)) return false;
  const int tiles = ceil_div(rows, kPlanBlock) * 4;
  packed_few_bwd_kernel<DH><<<(n_kv_heads + n_heads) * tiles, 64 * F::W, smem, stream>>>(
      qkv, plan, d_o, lse, delta, dqkv, rows, h, n_kv_heads * DH, n_heads / n_kv_heads, 1.0f / sqrtf((float)DH), n_kv_heads * tiles);
  return launch_ok("packed_few_bwd_kernel");
}

static bool check(const char* what, int dtype, int rows, int h, int n_heads, int n_kv_heads, const void* plan, uintptr_t tensors,
                  bool null, uintptr_t floats) {
  const int size = dtype == kBF16 ? 2 : 4;
  if (rows <= 0 || !packed_plan_bytes(rows) || h <= 0 || n_heads <= 0 || h % n_heads != 0 || n_kv_heads <= 0 ||
      n_heads % n_kv_heads != 0 || (h / n_heads != 64 && h / n_heads != 128)) {
    set_error("%s: rows=%d h=%d heads=%d kv_heads=%d (rows as a plan takes them, head size h / heads 64 or 128, kv_heads a divisor of "
              "heads)", what, rows, h, n_heads, n_kv_heads);
    return false;
  }
  // a lane's offset in a tile of 64 rows fits 32 bits, the blocks of 32 rows of forward or backward a grid
  if (((int64_t)h + 2 * (int64_t)n_kv_heads * (h / n_heads)) * (64 * size) > (int64_t)1 << 32 ||
      ((int64_t)n_heads + n_kv_heads) * ceil_div(rows, kPlanBlock) * 4 >= (int64_t)1 << 23) {
    set_error("%s: rows=%d h=%d heads=%d kv_heads=%d: too long a row, or too many rows and heads", what, rows, h, n_heads, n_kv_heads);
    return false;
  }
  if (null || tensors % 16 != 0 || (uintptr_t)plan % 16 != 0 || floats % 4 != 0) {
    set_error("%s: a NULL pointer, or a tensor or plan that is not 16-byte aligned", what);
    return false;
  }
  return true;
}

bool attention_packed_forward(int dtype, const void* qkv, const int* plan, void* o, float* lse, int rows, int h, int n_heads,
                              int n_kv_heads, hipStream_t stream) {
  if (!check("attention_packed_forward", dtype, rows, h, n_heads, n_kv_heads, plan, (uintptr_t)qkv | (uintptr_t)o,
             !qkv || !plan || !o || !lse, (uintptr_t)lse))
    return false;
  if (dtype == kF32)
    return attention_packed_forward_f32((const float*)qkv, plan, (float*)o, lse, rows, h, n_heads, n_kv_heads, stream);
  auto launch = h / n_heads == 128 ? few_forward<128> : few_forward<64>;
  return launch((const bf16*)qkv, plan, (bf16*)o, lse, rows, h, n_heads, n_kv_heads, stream);
}

size_t attention_packed_backward_workspace(int dtype, int rows, int h, int n_heads, int n_kv_heads) {
  (void)dtype, (void)h, (void)n_kv_heads;
  return (size_t)n_heads * rows * sizeof(float);  // delta
}

bool attention_packed_backward(int dtype, const void* qkv, const int* plan, const void* o, const float* lse, const void* d_o,
                               void* dqkv, void* workspace, int rows, int h, int n_heads, int n_kv_heads, hipStream_t stream) {
  if (!check("attention_packed_backward", dtype, rows, h, n_heads, n_kv_heads, plan,
             (uintptr_t)qkv | (uintptr_t)o | (uintptr_t)d_o | (uintptr_t)dqkv | (uintptr_t)workspace,
             !qkv || !plan || !o || !lse || !d_o || !dqkv || !workspace, (uintptr_t)lse))
    return false;
  float* delta = (float*)workspace;
  if (dtype == kF32)
    return attention_delta_f32((const float*)o, (const float*)d_o, delta, rows, h, n_heads, stream) &&
           attention_packed_backward_f32((const float*)qkv, plan, lse, delta, (const float*)d_o, (float*)dqkv, rows, h, n_heads,
                                         n_kv_heads, stream);
  if (!attention_delta_bf16((const bf16*)o, (const bf16*)d_o, delta, rows, h, n_heads, stream)) return false;
  auto launch = h / n_heads == 128 ? few_backward<128> : few_backward<64>;
  return launch((const bf16*)qkv, plan, lse, delta, (const bf16*)d_o, (bf16*)dqkv, rows, h, n_heads, n_kv_heads, stream);
}

}  // namespace po
