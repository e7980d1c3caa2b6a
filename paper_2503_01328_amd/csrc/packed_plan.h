// The plan of a packed batch: what po_op_packed_plan leaves for the attention calls, in 32-bit words.
//
//   [0] rows that sequences hold (`total`), [1] the row count the plan was made for, [2..15] unused
//   first[padded]   first row of the row's sequence
//   end[padded]     the row behind the last of the row's sequence
//   key_order[blocks][2], query_order[blocks][2]   blocks of 128 rows, those that meet the most tiles of 64 keys (queries) first, lower
//                                                  ones first among equals, each with the first key that its rows see (the row behind
//                                                  the last that sees its keys); blocks without a row of a sequence come last
// padded: rows rounded up to whole blocks.  Rows behind the last sequence have first = rows (no key is visible to them) and
// end = total (they are visible to no query, and both arrays never decrease).
#pragma once

#include "kernels.h"

namespace po {

constexpr int kPlanHeader = 16, kPlanBlock = 128;

struct PackedPlan {
  const int* words;
  int rows;
  __host__ __device__ __forceinline__ int blocks() const { return (rows + kPlanBlock - 1) / kPlanBlock; }
  __host__ __device__ __forceinline__ int padded() const { return blocks() * kPlanBlock; }
  // 0 for a plan that was made for other rows: its blocks then do nothing
  __device__ __forceinline__ int total() const { return words[1] == rows ? words[0] : 0; }
  __host__ __device__ __forceinline__ const int* first() const { return words + kPlanHeader; }
  __host__ __device__ __forceinline__ const int* end() const { return first() + padded(); }
  __host__ __device__ __forceinline__ const int2* key_order() const { return reinterpret_cast<const int2*>(end() + padded()); }
  __host__ __device__ __forceinline__ const int2* query_order() const { return key_order() + blocks(); }
};

}  // namespace po
