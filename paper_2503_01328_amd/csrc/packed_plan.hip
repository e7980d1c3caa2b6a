// The maps of a packed batch, built on the GPU from its sequence lengths, so that a program that learns the lengths there, or captures
// its step into a graph, need not wait for them: starts, each row's sequence and position, and the plan of the attention calls
// (packed_plan.h).
//
// One launch.  Every block scans all lengths for itself (16384 of them are 64 KiB from the L2; a scan in a launch of its own would cost
// more than repeating it) and keeps where each sequence ends in LDS; a thread then finds the sequence of the first of its four rows by
// bisection and walks on from there.  The orders come from counting, for each block of 128 rows, the blocks that come before
// it: the work of all of them stands in LDS too, a wave counts for one block at a time.
// Sums of lengths stop at `rows`: a length below zero counts as zero, sequences that reach past the rows are cut there.
#include "packed_plan.h"

namespace po {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64, kRowsPerThread = 4;
constexpr int kMaxSequences = 16384, kMaxRows = 1 << 21;  // 64 KiB of LDS each, for the ends and for the work of the blocks

__device__ __forceinline__ int capped_sum(int a, int b, int cap) { return min(a + b, cap); }  // both at most 2^21

// The sequence that holds `row`: the first that ends behind it.  row < ends[n - 1].
__device__ __forceinline__ int sequence_of(const int* ends, int n, int row) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (ends[mid] > row) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

}  // namespace

__global__ __launch_bounds__(kThreads) void packed_plan_kernel(const int* __restrict__ lengths, int n, int rows,
                                                               int* __restrict__ starts, int* __restrict__ positions,
                                                               int* __restrict__ sequence, int* __restrict__ plan) {
  extern __shared__ int lds[];
  int* ends = lds;              // [n]
  int* wave_sums = lds + n;     // [kWaves]
  unsigned* work = reinterpret_cast<unsigned*>(wave_sums + kWaves);  // [blocks]: tiles of keys << 16 | tiles of queries
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;

  // Each thread sums `per` lengths, the waves scan those sums, and every thread writes its ends.
  const int per = (n + kThreads - 1) / kThreads, from = min(tid * per, n), to = min(from + per, n);
  int sum = 0;
  for (int i = from; i < to; ++i) sum = capped_sum(sum, min(max(lengths[i], 0), rows), rows);
  int before = sum;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int v = __shfl_up(before, o, 64);
    if (lane >= o) before = capped_sum(before, v, rows);
  }
  if (lane == 63) wave_sums[wave] = before;
  before = __shfl_up(before, 1, 64);
  if (lane == 0) before = 0;
  __syncthreads();
  for (int w = 0; w < wave; ++w) before = capped_sum(before, wave_sums[w], rows);
  for (int i = from; i < to; ++i) ends[i] = before = capped_sum(before, min(max(lengths[i], 0), rows), rows);
  __syncthreads();

  const int total = ends[n - 1];
  if (starts)
    for (int i = blockIdx.x * kThreads + tid; i <= n; i += gridDim.x * kThreads) starts[i] = i ? ends[i - 1] : 0;

  const PackedPlan p{plan, rows};
  const int blocks = p.blocks(), padded = p.padded();
  const int row0 = (blockIdx.x * kThreads + tid) * kRowsPerThread;
  if (row0 < padded) {
    int j = row0 < total ? sequence_of(ends, n, row0) : 0, first[kRowsPerThread], end[kRowsPerThread];
#pragma unroll
    for (int u = 0; u < kRowsPerThread; ++u) {
      const int row = row0 + u;
      int seq = -1, pos = -1;
      first[u] = rows;
      end[u] = total;
      if (row < total) {
        while (ends[j] <= row) ++j;
        first[u] = j ? ends[j - 1] : 0;
        end[u] = ends[j];
        seq = j;
        pos = row - first[u];
      }
      if (row < rows) {
        if (sequence) sequence[row] = seq;
        if (positions) positions[row] = pos;
      }
    }
    if (plan) {
      *reinterpret_cast<int4*>(plan + kPlanHeader + row0) = make_int4(first[0], first[1], first[2], first[3]);
      *reinterpret_cast<int4*>(plan + kPlanHeader + padded + row0) = make_int4(end[0], end[1], end[2], end[3]);
    }
  }
  if (!plan) return;
  if (blockIdx.x == 0 && tid < kPlanHeader) plan[tid] = tid == 0 ? total : tid == 1 ? rows : 0;

  for (int b = tid; b < blocks; b += kThreads) {
    const int r0 = b * kPlanBlock, r1 = min(r0 + kPlanBlock, total);
    unsigned w = 0;
    if (r0 < total) {
      const int j = sequence_of(ends, n, r0), first = j ? ends[j - 1] : 0, end = ends[sequence_of(ends, n, r1 - 1)];
      w = (unsigned)((r1 - (first & ~63) + 63) >> 6) << 16 | (unsigned)((end - r0 + 63) >> 6);
    }
    work[b] = w;
  }
  __syncthreads();
  int* key_order = plan + kPlanHeader + 2 * padded;
  int* query_order = key_order + blocks;
  for (int b = blockIdx.x * kWaves + wave; b < blocks; b += gridDim.x * kWaves) {
    const unsigned mine = work[b], keys = mine >> 16, queries = mine & 0xffff;
    int k = 0, q = 0;
    for (int c = lane; c < blocks; c += 64) {
      const unsigned other = work[c];
      k += other >> 16 > keys || (other >> 16 == keys && c < b);
      q += (other & 0xffff) > queries || ((other & 0xffff) == queries && c < b);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      k += __shfl_xor(k, o, 64);
      q += __shfl_xor(q, o, 64);
    }
    if (lane == 0) {
      key_order[k] = b;
      query_order[q] = b;
    }
  }
}

size_t packed_plan_bytes(int rows) {
  if (rows <= 0 || rows > kMaxRows) return 0;
  const PackedPlan p{nullptr, rows};
  return ((size_t)kPlanHeader + 2 * (size_t)p.padded() + 2 * (size_t)p.blocks()) * sizeof(int);
}

bool packed_plan(const int* lengths, int n, int rows, int* starts, int* positions, int* sequence, int* plan,
                 hipStream_t stream) {
  if (!lengths || n <= 0 || n > kMaxSequences || rows <= 0 || rows > kMaxRows || (uintptr_t)plan % 16 != 0) {
    set_error("packed_plan: lengths=%p sequences=%d rows=%d plan=%p (1 to %d sequences, 1 to %d rows, the plan 16-byte aligned)",
              (const void*)lengths, n, rows, (void*)plan, kMaxSequences, kMaxRows);
    return false;
  }
  const PackedPlan p{plan, rows};
  const int smem = (n + kWaves + p.blocks()) * (int)sizeof(int);
  static LdsLimit lds;
  if (!lds.allow(packed_plan_kernel, (kMaxSequences + kWaves + kMaxRows / kPlanBlock) * (int)sizeof(int))) return false;
  packed_plan_kernel<<<ceil_div(p.padded(), kThreads * kRowsPerThread), kThreads, smem, stream>>>(lengths, n, rows, starts,
                                                                                                 positions, sequence, plan);
  return launch_ok("packed_plan_kernel");
}

}  // namespace po
