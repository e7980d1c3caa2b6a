// Tensors into their 8-bit form (saved8.h) and back: up to eight of any shapes in a launch, a layer's saved set.
//
// Bound by memory: a value is read (2 or 4 bytes) and 33/32 bytes are written, and the other way round.  A lane takes eight columns,
// four lanes a block of 32: its exponent is two lane exchanges away, nothing goes through LDS.
// A bf16 saved set of 168 million values (4096 rows, h 4096, f 16384): 88 us to save, 87 to restore, 5.8 TB/s; five fp32 tensors of 128 rows 3.7 us.
#include "saved8.h"

namespace po {

namespace {

struct Tensor8 {
  void* x;
  uint8_t *codes, *scales;
  int64_t ld;              // of x, elements
  uint32_t chunks;         // eights of codes altogether
  uint32_t row_chunks;     // eights of codes in a row
  int cols;                // of x in a row
  int flat;                // x is one run of whole blocks: a row of any length
  uint32_t first_block;
};
struct Table8 {
  Tensor8 t[kMaxSaved8Tensors];
  int n;
};

// SAVE: x into codes and scales, else back.  A thread takes UNROLL chunks, a block's worth apart.
template <typename T, bool SAVE, int UNROLL>
__global__ __launch_bounds__(256) void saved8_kernel(Table8 tab) {
  Tensor8 t = tab.t[0];
#pragma unroll
  for (int i = 1; i < kMaxSaved8Tensors; ++i)
    if (i < tab.n && blockIdx.x >= tab.t[i].first_block) t = tab.t[i];
  const uint32_t base = (blockIdx.x - t.first_block) * (256u * UNROLL) + threadIdx.x;
  float v[UNROLL][8];
  uint2 codes[UNROLL];
  unsigned byte[UNROLL];
  T* at[UNROLL];
  int held[UNROLL];  // columns of x in the chunk (at most zero: padding)
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    const uint32_t i = base + 256u * u;
    held[u] = 0;
    if (i < t.chunks) {
      if (t.flat) {
        at[u] = (T*)t.x + (size_t)i * 8;
        held[u] = 8;
      } else {
        const uint32_t row = i / t.row_chunks, col = (i - row * t.row_chunks) * 8;
        at[u] = (T*)t.x + (size_t)row * t.ld + col;
        held[u] = t.cols - (int)col;
      }
      if (SAVE) {
        load_eight(v[u], at[u], held[u]);
      } else {
        codes[u] = *(const uint2*)(t.codes + (size_t)i * 8);
        byte[u] = t.scales[i / 4];
      }
    } else if (SAVE) {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[u][k] = 0.f;
    }
  }
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    const uint32_t i = base + 256u * u;
    if (SAVE) {
      codes[u] = saved8_encode(v[u], byte[u]);
      if (i < t.chunks) {
        store_past(t.codes + (size_t)i * 8, codes[u]);
        if (i % 4 == 0) t.scales[i / 4] = (uint8_t)byte[u];
      }
    } else if (i < t.chunks) {
      saved8_decode(codes[u], byte[u], v[u]);
      store_eight(at[u], v[u], held[u]);
    }
  }
}

// Rows of a tensor, and whether two share an element: columns of one wide tensor do not, though their rows interleave.
struct Rows {
  const void* p;
  int rows, cols, ld, size;
  uint64_t span() const { return ((uint64_t)(rows - 1) * ld + cols) * size; }
};
bool rows_overlap(const Rows& a, const Rows& b) {
  if (!overlap(a.p, a.span(), b.p, b.span())) return false;
  const int64_t apart = (int64_t)(intptr_t)b.p - (int64_t)(intptr_t)a.p, ld = (int64_t)a.ld * a.size;
  if (a.ld != b.ld || apart % a.size != 0) return true;
  const int64_t at = (apart % ld + ld) % ld;  // b's first column in a's rows, bytes
  return at < (int64_t)a.cols * a.size || at + (int64_t)b.cols * b.size > ld;
}

bool table_of(const char* what, bool save, int dtype, int n, const void* const* x, const int* rows, const int* cols, const int* ld,
              const void* const* saved, Table8& tab, int& unroll) {
  if (n < 1 || n > kMaxSaved8Tensors || !x || !rows || !cols || !ld || !saved) {
    set_error("%s: n=%d (1 to %d tensors) or a NULL array", what, n, kMaxSaved8Tensors);
    return false;
  }
  const int size = dtype == kF32 ? 4 : 2;
  uint64_t total = 0;
  for (int i = 0; i < n; ++i) {
    if (rows[i] < 1 || cols[i] < 1 || ld[i] < cols[i] || saved8_codes(rows[i], cols[i]) / 8 > kMaxSaved8Chunks) {
      set_error("%s: tensor %d: rows=%d cols=%d ld=%d (at least one row and column, ld at least cols, at most %lld values)", what, i, rows[i],
                cols[i], ld[i], (long long)kMaxSaved8Chunks * 8);
      return false;
    }
    if (!x[i] || !saved[i] || (uintptr_t)x[i] % size != 0 || (uintptr_t)saved[i] % 16 != 0) {
      set_error("%s: tensor %d: a NULL pointer, x=%p not aligned to its type or saved=%p not to 16 bytes", what, i, x[i], saved[i]);
      return false;
    }
    total += (uint64_t)saved8_codes(rows[i], cols[i]) / 8;
  }
  for (int i = 0; i < n; ++i)
    for (int j = 0; j < n; ++j) {
      const Rows xi{x[i], rows[i], cols[i], ld[i], size}, xj{x[j], rows[j], cols[j], ld[j], size};
      const uint64_t bi = saved8_bytes(rows[i], cols[i]), bj = saved8_bytes(rows[j], cols[j]);
      if (overlap(x[i], xi.span(), saved[j], bj) || (i < j && (save ? overlap(saved[i], bi, saved[j], bj) : rows_overlap(xi, xj)))) {
        set_error("%s: tensors %d and %d: what is written overlaps what is read or written", what, i, j);
        return false;
      }
    }
  // Two chunks a thread keep more loads under way (save 98 us, one 103, four 105, before stores went past the caches); a small set spreads over
  // more blocks instead.
  unroll = total >= 2u * 256 * 1024 ? 2 : 1;
  tab.n = n;
  uint64_t block = 0;
  for (int i = 0; i < n; ++i) {
    Tensor8& t = tab.t[i];
    const int64_t padded = saved8_cols(cols[i]);
    t.x = const_cast<void*>(x[i]);
    t.codes = (uint8_t*)const_cast<void*>(saved[i]);
    t.scales = t.codes + saved8_codes(rows[i], cols[i]);
    t.ld = ld[i];
    t.cols = cols[i];
    t.chunks = (uint32_t)(saved8_codes(rows[i], cols[i]) / 8);
    t.row_chunks = (uint32_t)(padded / 8);
    t.flat = padded == cols[i] && (rows[i] == 1 || ld[i] == cols[i]);
    t.first_block = (uint32_t)block;
    block += ceil_div64(t.chunks, 256 * unroll);
  }
  return true;
}

template <typename T, bool SAVE>
void launch(const Table8& tab, int unroll, hipStream_t stream) {
  const Tensor8& last = tab.t[tab.n - 1];
  const unsigned blocks = last.first_block + (unsigned)ceil_div64(last.chunks, 256 * unroll);
  if (unroll == 2)
    saved8_kernel<T, SAVE, 2><<<blocks, 256, 0, stream>>>(tab);
  else
    saved8_kernel<T, SAVE, 1><<<blocks, 256, 0, stream>>>(tab);
}

}  // namespace

bool save8(int dtype, int n, const void* const* x, const int* rows, const int* cols, const int* ld, void* const* saved, hipStream_t stream) {
  Table8 tab;
  int unroll;
  if (!table_of("save8", true, dtype, n, x, rows, cols, ld, (const void* const*)saved, tab, unroll)) return false;
  (dtype == kF32 ? launch<float, true> : launch<bf16, true>)(tab, unroll, stream);
  return launch_ok("saved8_kernel");
}

bool restore8(int dtype, int n, const void* const* saved, const int* rows, const int* cols, const int* ld, void* const* x, hipStream_t stream) {
  Table8 tab;
  int unroll;
  if (!table_of("restore8", false, dtype, n, (const void* const*)x, rows, cols, ld, saved, tab, unroll)) return false;
  (dtype == kF32 ? launch<float, false> : launch<bf16, false>)(tab, unroll, stream);
  return launch_ok("saved8_kernel");
}

}  // namespace po
