// The maps of a packed batch, built on the GPU from its sequence lengths, so that a program that learns the lengths there, or captures
// its step into a graph, need not wait for them: starts, each row's sequence and position, and the plan of the attention calls
// (packed_plan.h).
//
// One launch.  Every block scans all lengths for itself (16384 of them are 64 KiB from the L2; a scan in a launch of its own would cost
// more than repeating it) and keeps where each sequence ends in LDS; a thread then finds the sequence of its row by bisection.  The orders
// come from counting, for each block of 128 rows, the blocks that come before it: the work of all of them stands in LDS too, a wave counts
// for one block at a time.
// Bound by latency, of the launch, the scan and the bisections: 2048 rows in 8 sequences 4.8 us, 131072 rows in 4000 10.8.
// Sums of lengths stop at `rows`: a length below zero counts as zero, sequences that reach past the rows are cut there.
#include <algorithm>

#include "packed_plan.h"

namespace po {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
// One block a CU: beyond, rows are walked rather than everything scanned by ever more blocks.  2097152 rows in 16384 sequences 482 us
// without this bound, 165 with it, 209 with twice as many; 500000 rows 44, 36 and 44.
constexpr int kMaxGrid = 256;
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

__device__ __forceinline__ int scan(int v, int lane, int cap) {  // inclusive, over the wave
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(v, o, 64);
    if (lane >= o) v = capped_sum(v, u, cap);
  }
  return v;
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
  for (int i = tid; i < n; i += kThreads) ends[i] = min(max(lengths[i], 0), rows);
  __syncthreads();
  const int per = (n + kThreads - 1) / kThreads, from = min(tid * per, n), to = min(from + per, n);
  int sum = 0;
  for (int i = from; i < to; ++i) sum = capped_sum(sum, ends[i], rows);
  int before = scan(sum, lane, rows);
  if (lane == 63) wave_sums[wave] = before;
  before = __shfl_up(before, 1, 64);
  if (lane == 0) before = 0;
  __syncthreads();
  const int waves = scan(lane < kWaves ? wave_sums[lane] : 0, lane, rows);
  if (wave > 0) before = capped_sum(before, __shfl(waves, wave - 1, 64), rows);
  for (int i = from; i < to; ++i) ends[i] = before = capped_sum(before, ends[i], rows);
  __syncthreads();

  const int total = ends[n - 1];
  if (starts)
    for (int i = blockIdx.x * kThreads + tid; i <= n; i += gridDim.x * kThreads) starts[i] = i ? ends[i - 1] : 0;

  const PackedPlan p{plan, rows};
  const int blocks = p.blocks(), padded = p.padded();
  for (int row = blockIdx.x * kThreads + tid; row < padded; row += gridDim.x * kThreads) {
    const bool held = row < total;
    const int j = held ? sequence_of(ends, n, row) : -1, first = !held ? rows : j ? ends[j - 1] : 0;
    if (row < rows) {
      if (sequence) sequence[row] = j;
      if (positions) positions[row] = held ? row - first : -1;
    }
    if (plan) {
      plan[kPlanHeader + row] = first;
      plan[kPlanHeader + padded + row] = held ? ends[j] : total;
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
  int2* key_order = reinterpret_cast<int2*>(plan + kPlanHeader + 2 * padded);
  int2* query_order = key_order + blocks;
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
    if (lane < 2) {  // lane 0: the first row's sequence, lane 1: the last one's
      const int r0 = b * kPlanBlock, r1 = min(r0 + kPlanBlock, total);
      const int j = r0 < total ? sequence_of(ends, n, lane ? r1 - 1 : r0) : -1;
      (lane ? query_order[q] : key_order[k]) = make_int2(b, j < 0 ? 0 : lane ? ends[j] : j ? ends[j - 1] : 0);
    }
  }
}

size_t packed_plan_bytes(int rows) {
  if (rows <= 0 || rows > kMaxRows) return 0;
  const PackedPlan p{nullptr, rows};
  return ((size_t)kPlanHeader + 2 * (size_t)p.padded() + 4 * (size_t)p.blocks()) * sizeof(int);
}

bool packed_plan(const int* lengths, int n, int rows, int* starts, int* positions, int* sequence, int* plan,
                 hipStream_t stream) {
  if (!lengths || n <= 0 || n > kMaxSequences || rows <= 0 || rows > kMaxRows || (uintptr_t)plan % 16 != 0) {
    set_error("packed_plan: lengths=%p sequences=%d rows=%d plan=%p (1 to %d sequences, 1 to %d rows, the plan 16-byte aligned)",
              (const void*)lengths, n, rows, (void*)plan, kMaxSequences, kMaxRows);
    return false;
  }
  const PackedPlan p{plan, rows};
  // Blocks read the lengths while others write: a plan from lengths that change meanwhile would name blocks that are none.
  const struct {
    uintptr_t at;
    size_t bytes;
  } arrays[] = {{(uintptr_t)lengths, 4 * (size_t)n}, {(uintptr_t)starts, 4 * ((size_t)n + 1)}, {(uintptr_t)positions, 4 * (size_t)rows},
                {(uintptr_t)sequence, 4 * (size_t)rows}, {(uintptr_t)plan, packed_plan_bytes(rows)}};
  for (const auto& a : arrays)
    for (const auto& b : arrays)
      if (a.at % 4 != 0 || (&a != &b && a.at && b.at && a.at < b.at + b.bytes && b.at < a.at + a.bytes)) {
        set_error("packed_plan: lengths=%p starts=%p positions=%p sequence=%p plan=%p (4-byte aligned, and none overlaps another)",
                  (const void*)lengths, (void*)starts, (void*)positions, (void*)sequence, (void*)plan);
        return false;
      }
  const int smem = (n + kWaves + p.blocks()) * (int)sizeof(int);
  static LdsLimit lds;
  if (!lds.allow(packed_plan_kernel, (kMaxSequences + kWaves + kMaxRows / kPlanBlock) * (int)sizeof(int))) return false;
  packed_plan_kernel<<<std::min(ceil_div(p.padded(), kThreads), kMaxGrid), kThreads, smem, stream>>>(lengths, n, rows, starts, positions, sequence, plan);
  return launch_ok("packed_plan_kernel");
}

}  // namespace po
