// bf16 causal attention of packed sequences on the matrix cores, forward and backward: rows of many sequences back to back, row i sees
// keys first(i) .. i, where first(i) is the first row of its sequence (packed_plan.h).
//   O = softmax(Q K^T scale) V, lse = log of the softmax's sum; P = exp(S scale - lse), dP = dO V^T, delta = dO . O,
//   dS = P (dP - delta), dQ = dS K scale, dK = dS^T Q scale, dV = P^T dO, the last two summed over the heads of a group.
//
// Blocks and tiles are cut from the packed axis, not from each sequence: a block of rows may hold the end of one sequence and several
// whole ones, and walks the tiles from the first key that any of its rows sees to the diagonal.  That wastes no rows of a block on
// short sequences, and the bounds first(i), end(j) of a row, one integer per lane, do all of the masking; tiles that every row sees
// whole pay nothing for it.  Blocks start in the order of falling work, which the plan holds: the last to start are the shortest.
// Operand layouts are those of attention_mfma.hip.
//
// Three forms, by how much there is to share out (the rules stand at the entry points): "few", blocks of 32 rows whose eight (or four)
// waves take a tile each; "wide" with SPLIT = 2, blocks of 64 rows by two pairs of waves that take half of the keys each; "wide" with
// SPLIT = 1, blocks of 128 rows, 32 a wave, all waves against the same tiles.
//
// What bounds them: long sequences the matrix cores' issue (16384 rows in 3 sequences, 40 heads of 128: forward 986 us, 982 TFLOP/s of
// the 1135 that a large product reaches on this card; one sequence of 4096 rows, 32 heads of 128: forward 139 us, 988 TFLOP/s, backward
// 497 us, 553 TFLOP/s, of which two terms of dS are 50 us); short ones what a block does besides its products: its place in the plan, first
// tiles, masks and results, and the longest sequence's chain of tiles (4096 rows in 21 sequences, 32 heads of 128 over 8: 30 and 93 us; 8192
// rows in 170, 40 heads of 64 over 8: 29 and 78; 2048 rows in 6, 16 heads of 128: 23 and 48).  Blocks of 32 rows alone took 2870 us for the
// first of these and 88 and 188, 135 and 226, 31 and 84 for the last three.
//
// P and dS are rounded to bf16 once on their way into the second product, as the inputs of every product here are (dS for dQ in two
// terms: TwoTerms); sums, maxima and accumulators are fp32.  Each such rounding is as large as that of the result itself: against 64 bits o is 1.07
// to 1.31 times as far off as fp32 arithmetic rounded once at the end, the gradient 1.36 to 1.40 times.  Three terms, which are the fp32 value,
// took 2 to 35 % longer.
// A key or value that is not finite reaches the rows that see it and no other, nor does a row of d_o reach another sequence: results that
// are not finite are redone row by row (attention_packed_rows.h).  Rows behind the last sequence read as zeros and are never written.
#include <algorithm>

#include "attention_few_tile.h"
#include "attention_packed_rows.h"

namespace po {
template <int BEGIN, int END, typename F>
__device__ __forceinline__ void static_for(F&& f) {
  if constexpr (BEGIN < END) {
    f(std::integral_constant<int, BEGIN>());
    static_for<BEGIN + 1, END>(f);
  }
}

// Waits for all loads in a way that the compiler sees.  It counts the loads of its own that may be outstanding (a kernel's rows, read
// into registers), cannot see those requested by text, and would guard every use of such a register in the loop with a wait that is
// really one for the tiles under way: backward of 4096 rows, 32 heads of 128, 575 us so, 455 with one wait before the loop.
__device__ __forceinline__ void wait_loads_visibly() {
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0), the other counters left alone (expcnt 7, lgkmcnt 15)
  asm volatile("" ::: "memory");
}

// ==================================================================================
// Few blocks: 32 rows each, every wave with tiles and a ring of its own; merged through LDS at the end.
// ==================================================================================

// The running maximum and sum of a softmax, per row in lanes l and l + 32.  128 rows in 5 sequences, 8 heads of 64: 5.8 us, nearly all
// of it latency (launch, plan, rows, tile, merge).
template <int DH>
__global__ __launch_bounds__((64 * Few<DH, true>::W)) void packed_few_fwd_kernel(
    const bf16* __restrict__ qkv, const int* words, bf16* __restrict__ o, float* __restrict__ lse, int rows, int h, int hkv, int group,
    float scale) {
  using F = Few<DH, true>;
  constexpr int DT = DH / 32, W = F::W, PART = F::NS * F::STAGE / 4;
  extern __shared__ __align__(16) char smem[];
  const PackedPlan plan{words, rows};
  const int total = plan.total();
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  const int n_heads = h / DH, head = blockIdx.x % n_heads, at = blockIdx.x / n_heads;
  if (total == 0) return;
  const int q0 = plan.key_order()[at >> 2].x * kPlanBlock + (3 - (at & 3)) * kRows;
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
  wait_loads_visibly();
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
  if (q <= last && !(redo >> (lane & 31) & 1)) {
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
  }
  if (wave == 0 && half == 0 && q <= last) {
    // by whichever constant is the more exact: 1 / 8, or c ln 2, whose two roundings all but cancel
    const float log_l = __logf(l), ln2 = 0.6931471805599453f;
    lse[(size_t)head * rows + q] = DH == 64 ? m * scale + fmaf(fmaf(-m, c, mc), ln2, log_l) : fmaf(mc, ln2, log_l);
  }
  if (redo) redo_packed_forward_rows<bf16, DH>(share_of<W>(redo, wave), q0, plan, qkv, o, h, hkv, group, head, scale);
}

// A tile's dS as the operands of dQ: rounded to bf16, and what that leaves rounded again, 16 bits in all.  dQ is the cheapest place to
// keep an error down (a fragment of K feeds both MFMAs): with one term it was 1.53 to 1.62 times that of results computed in fp32 and
// rounded at the end, of which delta's error, from the rounded o, is a third; with two it is 1.14 to 1.27, and the whole gradient 1.36 to
// 1.40 instead of 1.46 to 1.50.  Backward, us, one term / two: 4096 rows, 32 heads of 128 over 8, 21 sequences 100 / 107; one sequence,
// 32 heads 450 / 502; 8192 rows, 40 heads of 64 over 8, 170 sequences 90 / 94.  The second term for dK or dV instead: 111 and 116, 498
// and 498, 95 and 107.
struct TwoTerms {
  bf16x8 first[2], rest[2];
  __device__ __forceinline__ explicit TwoTerms(f32x16 ds) {
#pragma unroll
    for (int st = 0; st < 2; ++st) {
      first[st] = pack_bf16x8(ds, 8 * st);
#pragma unroll
      for (int e = 0; e < 8; ++e) ds[8 * st + e] -= (float)first[st][e];
      rest[st] = pack_bf16x8(ds, 8 * st);
    }
  }
};

// 32 query rows of a head from q0 on.
template <int DH>
__device__ __forceinline__ void packed_few_dq_block(char* smem, int q0, int head, PackedPlan plan, int total,
                                                    const bf16* __restrict__ qkv, const bf16* __restrict__ d_o,
                                                    const float* __restrict__ lse, const float* __restrict__ from_lse,
                                                    const float* __restrict__ from_delta, bf16* __restrict__ dqkv, int h, int hkv,
                                                    int group, float scale) {
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
  const float lse_q = from_lse[(size_t)head * plan.rows + qc] * -c, delta_q = -from_delta[(size_t)head * plan.rows + qc];
  wait_loads_visibly();
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
    const TwoTerms w(ds);
#pragma unroll
    for (int st = 0; st < 2; ++st)
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const bf16x8 k = read_tr_fragment<DH>(ktile, 16 * st, 32 * d, lane);
        dq[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, w.rest[st], dq[d], 0, 0, 0);
        dq[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, w.first[st], dq[d], 0, 0, 0);
      }
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
  if (q <= last && !(redo >> (lane & 31) & 1)) {
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
  if (redo)
    redo_packed_dq_rows<bf16, DH>(share_of<W>(redo, wave), q0, plan, qkv, d_o, lse, from_delta, dqkv, h, hkv, group, head, scale, -1.f);
}

// 32 keys of a key/value head from k0 on; its waves walk the query tiles of every query head that reads it.
template <int DH>
__device__ __forceinline__ void packed_few_dkv_block(char* smem, int k0, int kv_head, PackedPlan plan, int total,
                                                     const bf16* __restrict__ qkv, const bf16* __restrict__ d_o,
                                                     const float* __restrict__ lse, const float* __restrict__ from_lse,
                                                     const float* __restrict__ from_delta, bf16* __restrict__ dqkv, int h, int hkv,
                                                     int group, float scale) {
  using F = Few<DH>;
  constexpr int DT = DH / 32, W = F::W, PART = F::NS * F::STAGE / 4;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  const int key = k0 + (lane & 31), ld = h + 2 * hkv, last = total - 1, head0 = kv_head * group;
  const int end = plan.end()[key], end_lo = plan.end()[k0], end_hi = plan.end()[min(k0 + kRows - 1, last)];
  const int t0 = k0 / kRows, n_q = (end_hi - 1) / kRows + 1 - t0, n_it = group * n_q;
  const float c = scale * kLog2e;
  char* stages = smem + wave * F::NS * F::STAGE;
  char* stats = smem + F::AFTER + wave * F::NS * 256;  // per stage the statistics of the tile's 32 rows
  const unsigned stages_lds = __builtin_amdgcn_readfirstlane((int)lds_byte(stages));
  const unsigned stats_lds = __builtin_amdgcn_readfirstlane((int)lds_byte(stats));
  const TileLoads<DH> q_loads(ld, lane), do_loads(h, lane);
  const float* stat_of = half ? from_delta : from_lse;
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
  wait_loads_visibly();
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
        p[4 * b + r] = vl[r];
        ds[4 * b + r] = vd[r];
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
  const uint32_t bad_k = rows_to_redo(not_finite<DT>(dk), total - k0), bad_v = rows_to_redo(not_finite<DT>(dv), total - k0);
  if (lane == 0) redo_of[wave] = bad_k, redo_of[W + wave] = bad_v;
  __syncthreads();
  bf16* out = dqkv + h + kv_head * DH;
  const size_t stat_at = (size_t)head0 * plan.rows;
  const uint32_t redo = keys_to_redo(all_redo<W>(redo_of), all_redo<W>(redo_of + W), lse + stat_at, from_delta + stat_at,
                                     min(key, last), group, plan.rows);
  if (key <= last && !(redo >> (lane & 31) & 1)) {
    bf16* to = out + (size_t)key * ld + 4 * half;
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
      store4(to + 8 * g, vk);
      store4(to + hkv + 8 * g, vv);
    }
  }
  if (redo)
    redo_packed_key_rows<bf16, DH>(share_of<W>(redo, wave), k0, plan, qkv, d_o, lse, from_delta, out, out + hkv, ld, h, hkv, group, group,
                                   head0, scale, -1.f);
}

template <int DH>
__global__ __launch_bounds__(64 * Few<DH>::W) void packed_few_bwd_kernel(
    const bf16* __restrict__ qkv, const int* words, const bf16* __restrict__ d_o, const float* __restrict__ lse,
    const float* __restrict__ from_lse, const float* __restrict__ from_delta, bf16* __restrict__ dqkv, int rows, int h, int hkv, int group,
    float scale, int dkv_blocks) {
  extern __shared__ __align__(16) char smem[];
  const PackedPlan plan{words, rows};
  const int total = plan.total();
  if (total == 0) return;
  const bool dkv = (int)blockIdx.x < dkv_blocks;
  const int x = dkv ? blockIdx.x : blockIdx.x - dkv_blocks, n_x = dkv ? hkv / DH : h / DH, head = x % n_x, at = x / n_x;
  // of a block of 128 rows the first keys and the last queries meet the most
  const int row0 = dkv ? plan.query_order()[at >> 2].x * kPlanBlock + (at & 3) * kRows
                       : plan.key_order()[at >> 2].x * kPlanBlock + (3 - (at & 3)) * kRows;
  if (row0 >= total) return;
  if (dkv)
    packed_few_dkv_block<DH>(smem, row0, head, plan, total, qkv, d_o, lse, from_lse, from_delta, dqkv, h, hkv, group, scale);
  else
    packed_few_dq_block<DH>(smem, row0, head, plan, total, qkv, d_o, lse, from_lse, from_delta, dqkv, h, hkv, group, scale);
}

// ==================================================================================
// Forward: four waves, each 32 rows against 32 keys at a time.
// ==================================================================================

// Consecutive blocks go to the eight XCDs in turn, each with an L2 of its own: heads that share keys and values go to the same one, next
// to each other.  Forward of 16384 rows in 300 sequences, 40 heads of 128 over 8: 149 us by consecutive heads, 128 so; 4096 rows in 21, 32
// heads, 36.2 and 33.4.
__device__ __forceinline__ int head_of_block(int block, int n_heads, int group) {
  const int x = block % n_heads;
  return n_heads % 8 == 0 && group > 1 ? (x & 7) * (n_heads >> 3) + (x >> 3) : x;
}

// Rows row0 .. row0 + ROWS - 1 of the matrix at m into the tile at `tile`, by the four waves of a block; rows from `total` on become zeros.
template <int DH, int ROWS>
struct BlockLoads {
  static constexpr int N = ROWS * DH * 2 / 4096;  // loads of a wave
  unsigned off;
  __device__ __forceinline__ BlockLoads(int ld, int wave, int lane) {
    const int byte = wave * 1024 + lane * 16, row = byte / (DH * 2), c = (byte % (DH * 2) >> 4) ^ swz<DH>(row);
    off = (unsigned)row * (unsigned)ld * 2u + c * 16;
  }
  __device__ __forceinline__ void request(char* tile, const bf16* m, int ld, int row0, int total, int wave) const {
    const int left = min(total - row0, ROWS);
    const i32x4 buf = buffer_of(m + (size_t)row0 * ld, left > 0 ? ((unsigned)(left - 1) * (unsigned)ld + DH) * 2u : 0u);
    const unsigned lds = __builtin_amdgcn_readfirstlane((int)lds_byte(tile + wave * 1024));
#pragma unroll
    for (int u = 0; u < N; ++u) buffer_to_lds(lds + 4096u * u, off + (unsigned)(u * (4096 / (DH * 2))) * (unsigned)ld * 2u, buf);
  }
};

// Where a lane reads fragments in a tile of 32 rows, as LDS bytes from the tile on: row fragments (contraction over the head dimension),
// step kk: row lane % 32; transposing ones (contraction over the rows), block d of 32 columns: rows 4 (lane / 32) + .., the second half 8
// rows further.  A step or block on is an XOR of the chunk's bits: of the KEEP first steps (half blocks) kept in a register each, of the
// others formed at every read; everything else is a constant of the instruction.
template <int DH, int KEEP_ROW, int KEEP_COL>
struct TileReads {
  int row[KEEP_ROW], col[KEEP_COL];
  __device__ __forceinline__ TileReads(int lane, int at) {
    const int i = lane & 15, grp = lane >> 4, c = 16 * (grp & 1) + 4 * (i & 3);
    const int k = at + tile_offset<DH>(lane & 31, lane >> 5), v = at + tile_offset<DH>(4 * (grp >> 1) + (i >> 2), c >> 3) + (c & 7) * 2;
#pragma unroll
    for (int x = 0; x < KEEP_ROW; ++x) row[x] = k ^ (x << 5);
#pragma unroll
    for (int x = 0; x < KEEP_COL; ++x) col[x] = v ^ (x << 5);  // 2 d + half: rows 8 further have their chunks 2 places on
  }
  template <int KEEP>
  static __device__ __forceinline__ unsigned at(const int (&kept)[KEEP], int x) {
    if (x < KEEP) return kept[x];
    unsigned a;  // as text, or the compiler would keep it
    asm volatile("v_xor_b32 %0, %1, %2" : "=v"(a) : "i"((x & -KEEP) << 5), "v"(kept[x & (KEEP - 1)]));
    return a;
  }
  // `tile`: a constant number of bytes
  __device__ __forceinline__ bf16x8 row_fragment(int tile, int kk) const {
    typedef const __attribute__((address_space(3))) bf16x8* lds_ptr;
    return *(lds_ptr)(size_t)(at(row, kk) + tile);
  }
  __device__ __forceinline__ bf16x8 col_fragment(int tile, int step, int d) const {
    typedef __attribute__((address_space(3))) s16x4* lds_ptr;
    union {
      s16x4 half[2];
      bf16x8 v;
    } u;
    u.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(size_t)(at(col, 2 * d) + tile + step * 16 * DH * 2));
    u.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(size_t)(at(col, 2 * d + 1) + tile + (step * 16 + 8) * DH * 2));
    return u.v;
  }
};

// A row's columns 16 k + 8 b + 4 half + 0 .. 3 of a result, b = 0 in v0 and 1 in v1, to `to` = column 16 k.  The half-waves exchange half of
// theirs, so that a lane writes 16 bytes, not twice 8: forward and backward of 16384 rows in 300 sequences, 40 heads of 128 over 8, 127 and
// 350 us so far, 111 and 328 with it; 2048 rows in 6, 16 heads of 128, backward 42 and 38.  Whole lines, by more exchanges, took the same.
__device__ __forceinline__ void store_pair(bf16* to, const f32x4& v0, const f32x4& v1, int half) {
  union {
    bf16x4 v;
    unsigned u[2];
  } a, b;
#pragma unroll
  for (int r = 0; r < 4; ++r) a.v[r] = (bf16)v0[r], b.v[r] = (bf16)v1[r];
  union {
    unsigned u[4];
    bf16x8 v;
  } x;
#pragma unroll
  for (int r = 0; r < 2; ++r) {  // the upper half of a against the lower half of b
    const auto swapped = __builtin_amdgcn_permlane32_swap(a.u[r], b.u[r], false, false);
    x.u[r] = swapped[0];
    x.u[2 + r] = swapped[1];
  }
  *reinterpret_cast<bf16x8*>(to + 8 * half) = x.v;
}

// SPLIT = 2: blocks of 64 rows, waves w and w + 2 own the same 32 and take one half of each stage's keys; merged through LDS at the end.
// Stages of SUB tiles a wave, two in LDS (three measured the same).  A row's 2^S are taken against a reference that follows the maximum
// only when that has outgrown it by 8: P stays below 2^8, the accumulators are rescaled in few tiles.  RING fragments are read ahead of
// the MFMAs that take them, across the softmax, and hold the loop's reads in that order.
template <int DH, int SPLIT, int SUB>
__global__ __launch_bounds__(256, DH == 128 ? 3 : 4) void packed_wide_fwd_kernel(
    const bf16* __restrict__ qkv, const int* words, bf16* __restrict__ o, float* __restrict__ lse, int rows, int h, int hkv, int group,
    float scale) {
  constexpr int DT = DH / 32, KS = DH / 16, KT = 32 * SPLIT * SUB, BQ = 128 / SPLIT, TBYTES = KT * DH * 2, STAGE = 2 * TBYTES;
  constexpr int RING = DH == 64 ? 8 : 4;  // fragments read ahead
  using Loads = BlockLoads<DH, KT>;
  extern __shared__ __align__(16) char smem[];
  const PackedPlan plan{words, rows};
  const int total = plan.total();
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n_heads = h / DH;
  if (total == 0) return;
  const int head = head_of_block(blockIdx.x, n_heads, group), at = blockIdx.x / n_heads;
  const int2 block = plan.key_order()[at / SPLIT];
  const int q0 = block.x * kPlanBlock + (SPLIT - 1 - at % SPLIT) * BQ;
  if (q0 >= total) return;
  const int last = total - 1, ld = h + 2 * hkv, half = lane >> 5, slice = wave / (4 / SPLIT);
  const int qw0 = q0 + 32 * (wave % (4 / SPLIT)), q = qw0 + (lane & 31);
  const int tile0 = (SPLIT == 1 ? block.y : plan.first()[q0]) / KT, n_tiles = min(q0 + BQ - 1, last) / KT + 1 - tile0;
  const bf16* kbase = qkv + h + (head / group) * DH;
  const Loads loads(ld, wave, lane);
  auto load_stage = [&](int stage, int t) __attribute__((always_inline)) {
    char* st = smem + stage * STAGE;
    loads.request(st, kbase, ld, (tile0 + t) * KT, total, wave);
    loads.request(st + TBYTES, kbase + hkv, ld, (tile0 + t) * KT, total, wave);
  };
  bf16x8 qf[KS];
  load_row<DH>(qf, qkv + (size_t)min(q, last) * ld + head * DH, half);  // (rows past the end: computed, not stored)
  const int first = plan.first()[q], first_hi = plan.first()[min(qw0 + 31, last)], first_lo = plan.first()[qw0];
  load_stage(0, 0);
  if (n_tiles > 1) load_stage(1, 1);
  wait_loads_visibly();
  const unsigned span = (unsigned)(q - first);
  const float c = scale * kLog2e;
  f32x16 acc[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d) acc[d] = zero16();
  float ref = -INFINITY, l_run = 0.f;
  const TileReads<DH, DH == 128 && SPLIT == 2 ? 4 : KS, DH == 128 ? 4 : KS> reads(lane, (int)lds_byte(smem) + slice * SUB * 32 * DH * 2);
  auto tile = [&](auto stage, int t) __attribute__((always_inline)) {
    if (t + 1 < n_tiles) wait_loads<2 * Loads::N>();
    else wait_loads<0>();
    __syncthreads();
#pragma unroll
    for (int sub = 0; sub < SUB; ++sub) {
      const int ktile = decltype(stage)::value * STAGE + sub * 32 * DH * 2, vtile = ktile + TBYTES;
      const int key0 = (tile0 + t) * KT + 32 * (slice * SUB + sub);
      if (key0 > qw0 + 31 || key0 + 31 < first_lo || qw0 > last) continue;
      // fragment f: rows of K for the scores, then columns of V
      auto fragment = [&](int f) __attribute__((always_inline)) {
        return f < KS ? reads.row_fragment(ktile, f) : reads.col_fragment(vtile, (f - KS) / DT, (f - KS) % DT);
      };
      bf16x8 ring[RING];
#pragma unroll
      for (int f = 0; f < RING; ++f) ring[f] = fragment(f);
      f32x16 p = zero16();
#pragma unroll
      for (int m = 0; m < KS; ++m) {
        p = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[m % RING], qf[m], p, 0, 0, 0);
        if (m + RING < KS + 2 * DT) ring[m % RING] = fragment(m + RING);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (key0 + 31 > qw0 || key0 < first_hi) {
        const int rel = key0 + 4 * half - first;
        asm volatile("");  // a branch: as selects every tile would pay for the mask
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if ((unsigned)(rel + 8 * (e >> 2) + (e & 3)) > span) p[e] = -INFINITY;
      }
      float mx = p[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) mx = fmaxf(mx, p[e]);
      mx = exponent_of(fmaxf(mx, __shfl_xor(mx, 32, 64)), c);
      const bool outgrown = __builtin_amdgcn_ballot_w64(mx - ref > 8.0f) != 0;
      if (outgrown) {
        const float now = fmaxf(ref, mx), alpha = fast_exp2(ref - (now == -INFINITY ? 0.f : now));
        ref = now;
        l_run *= alpha;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[d][e] *= alpha;
      }
      const float to = ref == -INFINITY ? 0.f : ref;
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        p[e] = fast_exp2(fmaf(p[e], c, -to));
        sum += p[e];
      }
      l_run += sum;
      const bf16x8 pf[2] = {pack_bf16x8(p, 0), pack_bf16x8(p, 8)};
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int m = 0; m < 2 * DT; ++m) {
        acc[m % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[(KS + m) % RING], pf[m / DT], acc[m % DT], 0, 0, 0);
        if (m + RING < 2 * DT) ring[(KS + m) % RING] = fragment(KS + m + RING);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if (t + 2 < n_tiles) {
      __syncthreads();
      load_stage(decltype(stage)::value, t + 2);
    }
  };
  for (int t = 0; t < n_tiles; t += 2)
    static_for<0, 2>([&](auto stage) __attribute__((always_inline)) {
      if (t + decltype(stage)::value < n_tiles) tile(stage, t + decltype(stage)::value);
    });
  float l = l_run + __shfl_xor(l_run, 32, 64);
  if constexpr (SPLIT == 2) {
    float* xch = reinterpret_cast<float*>(smem) + (wave & 1) * (64 * (DT * 16 + 2));
    __syncthreads();
    if (slice == 1) {
      put_partial<DT>(xch, acc, lane);
      xch[(DT * 16) * 64 + lane] = ref;
      xch[(DT * 16 + 1) * 64 + lane] = l;
    }
    __syncthreads();
    if (slice == 1) return;
    const float ref1 = xch[(DT * 16) * 64 + lane], l1 = xch[(DT * 16 + 1) * 64 + lane], to = fmaxf(ref, ref1);
    const float a0 = fast_exp2(ref - to), a1 = fast_exp2(ref1 - to);
    l = l * a0 + l1 * a1;
    ref = to;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[d][e] = acc[d][e] * a0 + xch[(d * 16 + e) * 64 + lane] * a1;
  }
  const uint32_t redo = rows_to_redo(not_finite<DT>(acc) && !is_nan(l), total - qw0);
  if (q <= last && !(redo >> (lane & 31) & 1)) {
    const float inv = 1.0f / l;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int b = 0; b < 4; b += 2) {
        f32x4 v[2];
#pragma unroll
        for (int r = 0; r < 8; ++r) v[r >> 2][r & 3] = acc[d][4 * b + r] * inv;
        store_pair(o + (size_t)q * h + head * DH + 32 * d + 8 * b, v[0], v[1], half);
      }
  }
  if (q <= last && half == 0) lse[(size_t)head * rows + q] = fmaf(ref, 0.6931471805599453f, __logf(l));
  if (redo) redo_packed_forward_rows<bf16, DH>(redo, qw0, plan, qkv, o, h, hkv, group, head, scale);
}

// ==================================================================================
// Backward.  dQ blocks own rows, dK/dV blocks keys, 32 a wave; both form S and dP again, so that nothing is added up in memory and
// results do not depend on an order.
// ==================================================================================

// 128 / SPLIT query rows of a head from q0 on, key_first the first key that they see.  SPLIT as in the forward, NST stages in LDS.
template <int DH, int SPLIT, int NST>
__device__ __forceinline__ void packed_dq_block(char* smem, int q0, int key_first, int head, PackedPlan plan, int total,
                                                const bf16* __restrict__ qkv, const bf16* __restrict__ d_o,
                                                const float* __restrict__ lse, const float* __restrict__ from_lse,
                                                const float* __restrict__ from_delta, bf16* __restrict__ dqkv, int h, int hkv, int group,
                                                float scale) {
  constexpr int DT = DH / 32, KS = DH / 16, KT = 32 * SPLIT, BQ = 128 / SPLIT, TBYTES = KT * DH * 2, STAGE = 2 * TBYTES;
  constexpr int RING = DH == 128 ? 8 : 4;
  using Loads = BlockLoads<DH, KT>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  const int last = total - 1, ld = h + 2 * hkv, slice = wave / (4 / SPLIT);
  const int qw0 = q0 + 32 * (wave % (4 / SPLIT)), q = qw0 + (lane & 31), qc = min(q, last);
  const int tile0 = key_first / KT, n_tiles = min(q0 + BQ - 1, last) / KT + 1 - tile0;
  const bf16* kbase = qkv + h + (head / group) * DH;
  const Loads loads(ld, wave, lane);
  auto load_stage = [&](int stage, int t) __attribute__((always_inline)) {
    char* st = smem + stage * STAGE;
    loads.request(st, kbase, ld, (tile0 + t) * KT, total, wave);
    loads.request(st + TBYTES, kbase + hkv, ld, (tile0 + t) * KT, total, wave);
  };
  bf16x8 qf[KS], dof[KS];
  load_row<DH>(qf, qkv + (size_t)qc * ld + head * DH, half);  // (rows past the end: computed, not stored)
  load_row<DH>(dof, d_o + (size_t)qc * h + head * DH, half);
  const float c = scale * kLog2e;
  const float lse_q = from_lse[(size_t)head * plan.rows + qc] * -c, delta_q = -from_delta[(size_t)head * plan.rows + qc];
  const int first = plan.first()[q], first_hi = plan.first()[min(qw0 + 31, last)], first_lo = plan.first()[min(qw0, last)];
  load_stage(0, 0);
  if (n_tiles > 1) load_stage(1, 1);
  wait_loads_visibly();
  const unsigned span = (unsigned)(q - first);
  f32x16 dq[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d) dq[d] = zero16();
  const TileReads<DH, KS, KS> reads(lane, (int)lds_byte(smem) + slice * 32 * DH * 2);
  auto tile = [&](auto stage, int t) __attribute__((always_inline)) {
    if (t + 1 < n_tiles) wait_loads<2 * Loads::N>();
    else wait_loads<0>();
    __syncthreads();
    if (NST == 3 && t + 2 < n_tiles) load_stage((decltype(stage)::value + 2) % 3, t + 2);
    const int ktile = decltype(stage)::value * STAGE, vtile = ktile + TBYTES, key0 = (tile0 + t) * KT + 32 * slice;
    if (key0 <= qw0 + 31 && key0 + 31 >= first_lo && qw0 <= last) {
      // fragment f: of K and of V in turn for the scores and dP, then columns of K
      auto fragment = [&](int f) __attribute__((always_inline)) {
        if (f < 2 * KS) return reads.row_fragment(f & 1 ? vtile : ktile, f >> 1);
        return reads.col_fragment(ktile, (f - 2 * KS) / DT, (f - 2 * KS) % DT);
      };
      bf16x8 ring[RING];
#pragma unroll
      for (int f = 0; f < RING; ++f) ring[f] = fragment(f);
      f32x16 p = zero16(), ds = zero16();
#pragma unroll
      for (int m = 0; m < 2 * KS; ++m) {
        if (m & 1) ds = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[m % RING], dof[m >> 1], ds, 0, 0, 0);
        else p = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[m % RING], qf[m >> 1], p, 0, 0, 0);
        if (m + RING < 2 * KS + 2 * DT) ring[m % RING] = fragment(m + RING);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        p[e] = fast_exp2(fmaf(p[e], c, -lse_q));
        ds[e] = p[e] * (ds[e] - delta_q);
      }
      if (key0 + 31 > qw0 || key0 < first_hi) {
        const int rel = key0 + 4 * half - first;
        asm volatile("");  // a branch: as selects every tile would pay for the mask
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if ((unsigned)(rel + 8 * (e >> 2) + (e & 3)) > span) ds[e] = 0.f;
      }
      const TwoTerms w(ds);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int m = 0; m < 2 * DT; ++m) {
        dq[m % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[(2 * KS + m) % RING], w.rest[m / DT], dq[m % DT], 0, 0, 0);
        dq[m % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[(2 * KS + m) % RING], w.first[m / DT], dq[m % DT], 0, 0, 0);
        if (m + RING < 2 * DT) ring[(2 * KS + m) % RING] = fragment(2 * KS + m + RING);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if (NST == 2 && t + 2 < n_tiles) {
      __syncthreads();
      load_stage(decltype(stage)::value, t + 2);
    }
  };
  for (int t = 0; t < n_tiles; t += NST)
    static_for<0, NST>([&](auto stage) __attribute__((always_inline)) {
      if (t + decltype(stage)::value < n_tiles) tile(stage, t + decltype(stage)::value);
    });
  if constexpr (SPLIT == 2) {
    float* xch = reinterpret_cast<float*>(smem) + (wave & 1) * (64 * DT * 16);
    __syncthreads();
    if (slice == 1) put_partial<DT>(xch, dq, lane);
    __syncthreads();
    if (slice == 1) return;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) dq[d][e] += xch[(d * 16 + e) * 64 + lane];
  }
  const uint32_t redo = rows_to_redo(not_finite<DT>(dq) && !is_nan(lse_q + delta_q), total - qw0);
  if (q <= last && !(redo >> (lane & 31) & 1)) {
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int b = 0; b < 4; b += 2) {
        f32x4 v[2];
#pragma unroll
        for (int r = 0; r < 8; ++r) v[r >> 2][r & 3] = dq[d][4 * b + r] * scale;
        store_pair(dqkv + (size_t)q * ld + head * DH + 32 * d + 8 * b, v[0], v[1], half);
      }
  }
  if (redo) redo_packed_dq_rows<bf16, DH>(redo, qw0, plan, qkv, d_o, lse, from_delta, dqkv, h, hkv, group, head, scale, -1.f);
}

// 128 / SPLIT keys of a key/value head from k0 on, query_end the row behind the last that sees one of them; walks the query tiles of
// every head of the group.  Heads of 128: the last V fragments stand in LDS, a place per lane, for want of registers (three where a
// fourth would leave one block a CU).
template <int DH, int SPLIT, int NST>
struct KeyBlock {
  static constexpr int KT = 32 * SPLIT, TBYTES = KT * DH * 2, STATS = 4 * 256, STAGE = 2 * TBYTES + STATS;
  static constexpr int V_IN_LDS = DH == 128 ? (SPLIT == 1 ? 4 : 3) : 0, V_AT = NST * STAGE, BYTES = V_AT + 4 * V_IN_LDS * 1024;
};
template <int DH, int SPLIT, int NST>
__device__ __forceinline__ void packed_dkv_block(char* smem, int k0, int query_end, int kv_head, PackedPlan plan, int total,
                                                 const bf16* __restrict__ qkv, const bf16* __restrict__ d_o,
                                                 const float* __restrict__ lse, const float* __restrict__ from_lse,
                                                 const float* __restrict__ from_delta, bf16* __restrict__ dqkv, int h, int hkv, int group,
                                                 float scale) {
  using B = KeyBlock<DH, SPLIT, NST>;
  constexpr int DT = DH / 32, KS = DH / 16, KT = B::KT, TBYTES = B::TBYTES, RING = 3, V_IN_REG = KS - B::V_IN_LDS;
  using Loads = BlockLoads<DH, KT>;
  int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int last = total - 1, ld = h + 2 * hkv, slice = wave / (4 / SPLIT), head0 = kv_head * group;
  const int kw0 = k0 + 32 * (wave % (4 / SPLIT));
  int key = kw0 + (lane & 31);
  const int tile0 = k0 / KT, n_q = (query_end - 1) / KT + 1 - tile0, n_it = group * n_q;
  const Loads q_loads(ld, wave, lane), do_loads(h, wave, lane);
  const float* stat_of = half ? from_delta : from_lse;
  int g_next = 0, t_next = 0;  // the next tile to ask for
  auto load_stage = [&](int stage) __attribute__((always_inline)) {
    char* st = smem + stage * B::STAGE;
    const int head = head0 + g_next, row0 = (tile0 + t_next) * KT;
    q_loads.request(st, qkv + head * DH, ld, row0, total, wave);
    do_loads.request(st + TBYTES, d_o + head * DH, h, row0, total, wave);
    // the statistics of the 32 rows that this wave takes, in a place of its own
    float_to_lds(__builtin_amdgcn_readfirstlane((int)lds_byte(st + 2 * TBYTES + wave * 256)),
                 stat_of + (size_t)head * plan.rows + min(row0 + 32 * slice + (lane & 31), last));
    if (++t_next == n_q) t_next = 0, ++g_next;
  };
  bf16x8 kf[KS], vf[V_IN_REG];
  char* vslot = smem + B::V_AT + (wave * B::V_IN_LDS * 64 + lane) * 16;
  {
    const bf16* krow = qkv + (size_t)min(key, last) * ld + h + kv_head * DH;  // (keys past the end: computed, not stored)
    load_row<DH>(kf, krow, half);
    bf16x8 v[KS];
    load_row<DH>(v, krow + hkv, half);
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) {
      if (kk < V_IN_REG) vf[kk] = v[kk];
      else *reinterpret_cast<bf16x8*>(vslot + (kk - V_IN_REG) * 1024) = v[kk];
    }
  }
  const int end = plan.end()[key], end_lo = plan.end()[min(kw0, last)], end_hi = plan.end()[min(kw0 + 31, last)];
  load_stage(0);
  if (n_it > 1) load_stage(1);
  wait_loads_visibly();
  const float c = scale * kLog2e;
  f32x16 dk[DT], dv[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d) dk[d] = dv[d] = zero16();
  int t_now = 0;
  auto tile = [&](auto stage, int it) __attribute__((always_inline)) {
    constexpr int kLoads = 2 * Loads::N + 1;
    if (it + 1 < n_it) wait_loads<kLoads>();
    else wait_loads<0>();
    __syncthreads();
    if (NST == 3 && it + 2 < n_it) load_stage((decltype(stage)::value + 2) % 3);
    const int q0 = (tile0 + t_now) * KT + 32 * slice;
    if (++t_now == n_q) t_now = 0;
    if (q0 + 31 >= kw0 && q0 < end_hi && kw0 <= last) {
      int lane_l = lane;
      asm volatile("" : "+v"(lane_l));  // addresses are formed again rather than kept across tiles, where every register is taken
      const TileReads<DH, 2, 2> reads(lane_l, (int)lds_byte(smem) + decltype(stage)::value * B::STAGE + slice * 32 * DH * 2);
      const char* vslot_l = smem + B::V_AT + (wave * B::V_IN_LDS * 64 + lane_l) * 16;
      const float* stat = reinterpret_cast<const float*>(smem + decltype(stage)::value * B::STAGE + 2 * TBYTES + wave * 256);
      const int half_l = lane_l >> 5;
      // fragment f: of Q and of dO in turn for the scores and dP, then columns of dO and of Q in turn
      auto fragment = [&](int f) __attribute__((always_inline)) {
        if (f < 2 * KS) return reads.row_fragment(f & 1 ? TBYTES : 0, f >> 1);
        f -= 2 * KS;
        return reads.col_fragment(f & 1 ? 0 : TBYTES, (f >> 1) / DT, (f >> 1) % DT);
      };
      bf16x8 ring[RING];
#pragma unroll
      for (int f = 0; f < RING; ++f) ring[f] = fragment(f);
      f32x16 p, ds;  // the row statistics are the initial value: S - lse / scale and dP - delta
#pragma unroll
      for (int b = 0; b < 4; ++b) {  // register 4 b + r is query row 8 b + 4 half + r
        const f32x4 vl = *reinterpret_cast<const f32x4*>(stat + 8 * b + 4 * half_l);
        const f32x4 vd = *reinterpret_cast<const f32x4*>(stat + 32 + 8 * b + 4 * half_l);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          p[4 * b + r] = vl[r];
          ds[4 * b + r] = vd[r];
        }
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int m = 0; m < 2 * KS; ++m) {
        if (m & 1) {
          bf16x8 v;
          if ((m >> 1) < V_IN_REG) v = vf[m >> 1];
          else v = *reinterpret_cast<const bf16x8*>(vslot_l + ((m >> 1) - V_IN_REG) * 1024);
          ds = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[m % RING], v, ds, 0, 0, 0);
        } else {
          p = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[m % RING], kf[m >> 1], p, 0, 0, 0);
        }
        ring[m % RING] = fragment(m + RING);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        p[e] = fast_exp2(p[e] * c);
        ds[e] *= p[e];
      }
      if (q0 < kw0 + 31 || q0 + 32 > end_lo) {  // the diagonal, or rows past the end of a sequence
        const int rel = q0 + 4 * half - key;
        const unsigned span = (unsigned)(end - key);
        asm volatile("");  // a branch: as selects every tile would pay for the mask
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if ((unsigned)(rel + 8 * (e >> 2) + (e & 3)) >= span) p[e] = ds[e] = 0.f;  // dS too: 0 times a dP that is not finite is no 0
      }
      const bf16x8 w[2][2] = {{pack_bf16x8(p, 0), pack_bf16x8(ds, 0)}, {pack_bf16x8(p, 8), pack_bf16x8(ds, 8)}};
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int m = 0; m < 4 * DT; ++m) {
        const int step = (m >> 1) / DT, d = (m >> 1) % DT;
        if (m & 1) dk[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[(2 * KS + m) % RING], w[step][1], dk[d], 0, 0, 0);
        else dv[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[(2 * KS + m) % RING], w[step][0], dv[d], 0, 0, 0);
        if (m + RING < 4 * DT) ring[(2 * KS + m) % RING] = fragment(2 * KS + m + RING);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if (NST == 2 && it + 2 < n_it) {
      __syncthreads();
      load_stage(decltype(stage)::value);
    }
  };
  for (int it = 0; it < n_it; it += NST)
    static_for<0, NST>([&](auto stage) __attribute__((always_inline)) {
      if (it + decltype(stage)::value < n_it) tile(stage, it + decltype(stage)::value);
    });
  // rebuilt rather than kept across the loop
  lane = (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
  half = lane >> 5;
  key = kw0 + (lane & 31);
  if constexpr (SPLIT == 2) {
    float* xch = reinterpret_cast<float*>(smem) + (wave & 1) * (2 * 64 * DT * 16);
    __syncthreads();
    if (slice == 1) {
      put_partial<DT>(xch, dk, lane);
      put_partial<DT>(xch + 64 * DT * 16, dv, lane);
    }
    __syncthreads();
    if (slice == 1) return;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        dk[d][e] += xch[(d * 16 + e) * 64 + lane];
        dv[d][e] += xch[((DT + d) * 16 + e) * 64 + lane];
      }
  }
  bf16* out = dqkv + h + kv_head * DH;
  const size_t stat_at = (size_t)head0 * plan.rows;
  const uint32_t bad_k = rows_to_redo(not_finite<DT>(dk), total - kw0), bad_v = rows_to_redo(not_finite<DT>(dv), total - kw0);
  const uint32_t redo = keys_to_redo(bad_k, bad_v, lse + stat_at, from_delta + stat_at, min(key, last), group, plan.rows);
  if (key <= last && !(redo >> (lane & 31) & 1)) {
    bf16* to = out + (size_t)key * ld;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int b = 0; b < 4; b += 2) {
        f32x4 vk[2], vv[2];
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          vk[r >> 2][r & 3] = dk[d][4 * b + r] * scale;
          vv[r >> 2][r & 3] = dv[d][4 * b + r];
        }
        store_pair(to + 32 * d + 8 * b, vk[0], vk[1], half);
        store_pair(to + hkv + 32 * d + 8 * b, vv[0], vv[1], half);
      }
  }
  if (redo)
    redo_packed_key_rows<bf16, DH>(redo, kw0, plan, qkv, d_o, lse, from_delta, out, out + hkv, ld, h, hkv, group, group, head0,
                                   scale, -1.f);
}

template <int DH, int SPLIT, int NST>
__global__ __launch_bounds__(256, DH == 128 ? 2 : 3) void packed_wide_bwd_kernel(
    const bf16* __restrict__ qkv, const int* words, const bf16* __restrict__ d_o, const float* __restrict__ lse,
    const float* __restrict__ from_lse, const float* __restrict__ from_delta, bf16* __restrict__ dqkv, int rows, int h, int hkv, int group,
    float scale, int dkv_blocks) {
  extern __shared__ __align__(16) char smem[];
  const PackedPlan plan{words, rows};
  const int total = plan.total();
  if (total == 0) return;
  // dK/dV blocks first, as one of them does up to a group's heads more: the dQ blocks start on the CUs that light ones leave early
  // (4096 rows in 21 sequences, 32 heads of 128 over 8: 105 us, the other way round 117)
  if ((int)blockIdx.x < dkv_blocks) {
    const int n_kv = hkv / DH, at = blockIdx.x / n_kv;
    const int2 block = plan.query_order()[at / SPLIT];
    const int k0 = block.x * kPlanBlock + at % SPLIT * (128 / SPLIT);
    if (k0 >= total) return;
    const int end = SPLIT == 1 ? block.y : plan.end()[min(k0 + 128 / SPLIT, total) - 1];
    packed_dkv_block<DH, SPLIT, NST>(smem, k0, end, blockIdx.x % n_kv, plan, total, qkv, d_o, lse, from_lse, from_delta, dqkv, h, hkv,
                                     group, scale);
  } else {
    const int x = blockIdx.x - dkv_blocks, n_heads = h / DH, at = x / n_heads;
    const int2 block = plan.key_order()[at / SPLIT];
    const int q0 = block.x * kPlanBlock + (SPLIT - 1 - at % SPLIT) * (128 / SPLIT);
    if (q0 >= total) return;
    packed_dq_block<DH, SPLIT, NST>(smem, q0, SPLIT == 1 ? block.y : plan.first()[q0], head_of_block(x, n_heads, group), plan, total, qkv,
                                    d_o, lse, from_lse, from_delta, dqkv, h, hkv, group, scale);
  }
}

// What the backward adds to scores and to dP, as the initial value of their accumulators: from_lse = -lse / scale and from_delta = -delta,
// delta = dO . O of a row and head.  Bound by memory.  A block takes 32 rows of a head, DH / 8 lanes a row with 16 bytes of both each, all
// asked for before the first is used, and writes their values next to each other: 8192 rows, 40 heads of 64, the whole backward 94 us with
// a row of all heads after the other, whose results go to as many places as there are heads, 87 so (two to eight heads a block the same).
constexpr int kStatRows = 32;
template <int DH>
__global__ __launch_bounds__(256) void packed_stats_kernel(const bf16* __restrict__ o, const bf16* __restrict__ d_o,
                                                           const float* __restrict__ lse, float* __restrict__ from_lse,
                                                           float* __restrict__ from_delta, int rows, int n_heads, float to_lse) {
  constexpr int LANES = DH / 8, STEP = 256 / LANES, N = kStatRows / STEP;
  __shared__ float sums[kStatRows];
  const int head = blockIdx.x % n_heads, row0 = blockIdx.x / n_heads * kStatRows;
  const int mine = threadIdx.x / LANES, e = threadIdx.x % LANES * 8;
  bf16x8 a[N], b[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const size_t at = ((size_t)min(row0 + mine + i * STEP, rows - 1) * n_heads + head) * DH + e;
    a[i] = *reinterpret_cast<const bf16x8*>(o + at);
    b[i] = *reinterpret_cast<const bf16x8*>(d_o + at);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float d = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) d = fmaf((float)a[i][j], (float)b[i][j], d);
#pragma unroll
    for (int m = 1; m < LANES; m <<= 1) d += __shfl_xor(d, m);
    if (e == 0) sums[mine + i * STEP] = d;
  }
  __syncthreads();
  const int row = row0 + threadIdx.x;
  if (threadIdx.x < kStatRows && row < rows) {
    const size_t at = (size_t)head * rows + row;
    from_lse[at] = lse[at] * to_lse;
    from_delta[at] = -sums[threadIdx.x];
  }
}

// ---- host side -------------------------------------------------------------------------------------------------
template <int DH>
static bool statistics(const bf16* o, const bf16* d_o, const float* lse, float* stats, int rows, int n_heads, hipStream_t stream) {
  packed_stats_kernel<DH><<<n_heads * ceil_div(rows, kStatRows), 256, 0, stream>>>(o, d_o, lse, stats, stats + (size_t)n_heads * rows,
                                                                                  rows, n_heads, -sqrtf((float)DH));
  return launch_ok("packed_stats_kernel");
}

template <int DH, int SPLIT, int NST>
static bool wide_backward(const bf16* qkv, const int* plan, const float* lse, const float* stats, const bf16* d_o, bf16* dqkv, int rows,
                           int h, int n_heads, int n_kv_heads, hipStream_t stream) {
  constexpr int dq = NST * 2 * 32 * SPLIT * DH * 2, dkv = KeyBlock<DH, SPLIT, NST>::BYTES;
  constexpr int merge = SPLIT == 2 ? 4 * 64 * (DH / 32) * 16 * 4 : 0;
  constexpr int smem = dkv > merge ? (dkv > dq ? dkv : dq) : (merge > dq ? merge : dq);
  static LdsLimit lds;
  if (!lds.allow(packed_wide_bwd_kernel<DH, SPLIT, NST>, smem)) return false;
  const int blocks = ceil_div(rows, kPlanBlock) * SPLIT;
  packed_wide_bwd_kernel<DH, SPLIT, NST><<<(n_kv_heads + n_heads) * blocks, 256, smem, stream>>>(
      qkv, plan, d_o, lse, stats, stats + (size_t)n_heads * rows, dqkv, rows, h, n_kv_heads * DH, n_heads / n_kv_heads,
      1.0f / sqrtf((float)DH), n_kv_heads * blocks);
  return launch_ok("packed_wide_bwd_kernel");
}

template <int DH, int SPLIT, int SUB>
static bool wide_forward(const bf16* qkv, const int* plan, bf16* o, float* lse, int rows, int h, int n_heads, int n_kv_heads,
                          hipStream_t stream) {
  constexpr int smem = 2 * 2 * 32 * SPLIT * SUB * DH * 2;
  static LdsLimit lds;
  if (!lds.allow(packed_wide_fwd_kernel<DH, SPLIT, SUB>, smem)) return false;
  packed_wide_fwd_kernel<DH, SPLIT, SUB><<<n_heads * ceil_div(rows, kPlanBlock) * SPLIT, 256, smem, stream>>>(
      qkv, plan, o, lse, rows, h, n_kv_heads * DH, n_heads / n_kv_heads, 1.0f / sqrtf((float)DH));
  return launch_ok("packed_wide_fwd_kernel");
}

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
static bool few_backward(const bf16* qkv, const int* plan, const float* lse, const float* stats, const bf16* d_o, bf16* dqkv, int rows,
                         int h, int n_heads, int n_kv_heads, hipStream_t stream) {
  using F = Few<DH>;
  constexpr int smem = F::AFTER + F::W * F::NS * 256 + 2 * F::W * 4;
  static LdsLimit lds;
  if (!lds.allow(packed_few_bwd_kernel<DH>, smem)) return false;
  const int tiles = ceil_div(rows, kPlanBlock) * 4;
  packed_few_bwd_kernel<DH><<<(n_kv_heads + n_heads) * tiles, 64 * F::W, smem, stream>>>(
      qkv, plan, d_o, lse, stats, stats + (size_t)n_heads * rows, dqkv, rows, h, n_kv_heads * DH, n_heads / n_kv_heads,
      1.0f / sqrtf((float)DH), n_kv_heads * tiles);
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
  if (o == qkv) {
    set_error("attention_packed_forward: o is another tensor than qkv");
    return false;
  }
  if (dtype == kF32)
    return attention_packed_forward_f32((const float*)qkv, plan, (float*)o, lse, rows, h, n_heads, n_kv_heads, stream);
  // Larger blocks share more of each tile, smaller ones fill more of the 256 CUs and leave shorter chains behind a long sequence; lengths
  // are not known here.  us, few / 64 rows / 128 rows, sequences of 40 rows, of 800 to 1024, one:
  //   heads of 64: 64 blocks of 128 rows (all heads) 6.0 6.3 7.8, 10.8 16.5 25.2;  128: 9.3 6.4 7.8, 12.6 13.9 19.6, 25 42 67;
  //     512: 32 10.7 10.1, 44 23 30, 84 54 70;  640: 42 14.5 12.4, 58 26 30;
  //   heads of 128: 64: 8.2 8.6 10.0, 14.9 22.4 34.9;  128: 12.9 8.6 10.4, 18.7 18.8 27.2, 40 57 94;  256: 24 11.4 11.3, 36 25 36;
  //     320: 31 16.1 13.5, 43 23 29;  512: 48 20.7 15.3, 67 33 41, 137 89 102;  640: 60 26 20, 87 45 43.
  const int64_t blocks = (int64_t)n_heads * ceil_div(rows, kPlanBlock);
  auto launch = h / n_heads == 128 ? (blocks <= 64 ? few_forward<128> : blocks <= 384 ? wide_forward<128, 2, 1> : wide_forward<128, 1, 1>)
                                   : (blocks <= 64 ? few_forward<64> : blocks <= 512 ? wide_forward<64, 2, 1> : wide_forward<64, 1, 2>);
  return launch((const bf16*)qkv, plan, (bf16*)o, lse, rows, h, n_heads, n_kv_heads, stream);
}

size_t attention_packed_backward_workspace(int dtype, int rows, int h, int n_heads, int n_kv_heads) {
  const size_t stats = (size_t)n_heads * rows;
  // delta, and in bf16 the scaled lse; in fp32 partial results of dK and dV behind it, 16-byte aligned
  return (dtype == kBF16 ? 2 * stats : (stats + 3) / 4 * 4 + attention_packed_f32_partials(rows, h, n_heads, n_kv_heads)) * sizeof(float);
}

bool attention_packed_backward(int dtype, const void* qkv, const int* plan, const void* o, const float* lse, const void* d_o,
                               void* dqkv, void* workspace, int rows, int h, int n_heads, int n_kv_heads, hipStream_t stream) {
  if (!check("attention_packed_backward", dtype, rows, h, n_heads, n_kv_heads, plan,
             (uintptr_t)qkv | (uintptr_t)o | (uintptr_t)d_o | (uintptr_t)dqkv | (uintptr_t)workspace,
             !qkv || !plan || !o || !lse || !d_o || !dqkv || !workspace, (uintptr_t)lse))
    return false;
  if (dqkv == qkv || dqkv == d_o) {
    set_error("attention_packed_backward: dqkv is another tensor than qkv and d_o");
    return false;
  }
  float* stats = (float*)workspace;
  if (dtype == kF32)
    return attention_delta_f32((const float*)o, (const float*)d_o, stats, rows, h, n_heads, stream) &&
           attention_packed_backward_f32((const float*)qkv, plan, lse, stats, (const float*)d_o, (float*)dqkv,
                                         stats + ((size_t)n_heads * rows + 3) / 4 * 4, rows, h, n_heads, n_kv_heads, stream);
  if (!(h / n_heads == 128 ? statistics<128> : statistics<64>)((const bf16*)o, (const bf16*)d_o, lse, stats, rows, n_heads, stream))
    return false;
  const int group = n_heads / n_kv_heads, row_blocks = ceil_div(rows, kPlanBlock);
  // As in the forward; blocks of keys are n_kv_heads x row_blocks, and each walks its whole group.  us, as there:
  //   few or not by n_heads x row_blocks: heads of 64, no groups: 32: 9.7 9.6 11.6, 13.7 20.2 32.3;  64: 14.4 10.0 13.2, 21.2 23.3 37.2;
  //     groups of 4: 128: 16.8 19.0 28.0, 27 60 108;  256: 31 22 36, 49 73 129 (200 rows each 36 36 56);
  //     heads of 128, no groups: 32: 12.6 13.0 15.2, 22.8 29.3 44.0;  64: 19.5 13.9 18.0, 33.9 34.2 51.3;
  //     groups of 4: 128: 26 28 38, 58 90 151;  256: 46 31 50, 85 111 181 (200 rows each 55 53 78);
  //   64 or 128 rows by n_kv_heads x row_blocks: heads of 64: 256: 42 18.4 16.6, 59 35 50;  groups of 4 106 41 44, 165 107 178, 378 299 463;
  //     512: 85 30 27, 113 52 61, 216 155 171;  640: 104 35 32, 146 69 67;
  //     heads of 128: 256: 63 30 26, 101 55 70;  groups of 4 157 74 66, 292 163 250, 782 521 696;  320: 75 37 33, 119 65 61;
  //     512: 121 56 47, 189 97 89, 429 269 264.
  const bool few = (int64_t)n_heads * row_blocks <= std::min(32 * group, 128), narrow = (int64_t)n_kv_heads * row_blocks <= 256;
  auto launch = h / n_heads == 64 ? (few ? few_backward<64> : narrow ? wide_backward<64, 2, 2> : wide_backward<64, 1, 2>)
                                  : (few ? few_backward<128> : narrow ? wide_backward<128, 2, 2> : wide_backward<128, 1, 3>);
  return launch((const bf16*)qkv, plan, lse, stats, (const bf16*)d_o, (bf16*)dqkv, rows, h, n_heads, n_kv_heads, stream);
}

}  // namespace po
