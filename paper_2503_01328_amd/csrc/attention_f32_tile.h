// What the fp32 attention kernels share: the product of fp32 matrix cores, a wave's copy of 32 rows in LDS and how it is read, partial
// results of waves.
#pragma once

#include "attention_rows.h"
#include "mfma_common.h"

namespace po {

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ f32x16 mfma(float a, float b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 zero16() {
  f32x16 z;
#pragma unroll
  for (int e = 0; e < 16; ++e) z[e] = 0.f;
  return z;
}
// exp(x scale).  Two multiplications: with scale log2(e) as one constant its rounding is the same in every term of a row.
__device__ __forceinline__ float exp_scaled(float x, float scale) { return __builtin_amdgcn_exp2f(x * scale * kLog2e); }
// Row `row` of a matrix: this half-wave's 16-byte pieces.
template <int DH>
__device__ __forceinline__ void load_pieces(f32x4 (&f)[DH / 8], const float* row, int half) {
#pragma unroll
  for (int kk = 0; kk < DH / 8; ++kk) f[kk] = *reinterpret_cast<const f32x4*>(row + 8 * kk + 4 * half);
}

// A wave's copy of 32 rows of a matrix in LDS: piece c (16 bytes) of row r at place c ^ place_of(r), so that the reads of one
// piece of eight rows and of 32 floats of two rows that are four apart both fall into different banks.
template <int DH>
constexpr int kTileBytes = 32 * DH * 4;
template <int DH>
__device__ __forceinline__ int place_of(int row) {
  return (row & 7) ^ (DH % 64 == 0 ? ((row >> 2) & 1) << 3 : 0);
}
// Requests rows row0 .. row0 + 31 of the matrix at m (rows past `last`: the last one) into the tile at LDS byte `tile`.
template <int DH>
__device__ __forceinline__ void request_tile(unsigned tile, const float* m, int ld, int row0, int last, int lane) {
  const i32x4 buf = buffer_of(m + (size_t)row0 * ld, 0xffffffe0u);
  const int max_row = last - row0;
#pragma unroll
  for (int u = 0; u < kTileBytes<DH> / 1024; ++u) {
    const int byte = u * 1024 + lane * 16, row = byte / (DH * 4), c = (byte % (DH * 4) >> 4) ^ place_of<DH>(row);
    buffer_to_lds(tile + 1024u * u, (unsigned)min(row, max_row) * (unsigned)ld * 4 + c * 16, buf);
  }
}
// Where a lane reads in the first of a wave's two tiles; everything else is a constant offset from there.  (Left to itself the
// compiler keeps an address register per read, and spills.)
template <int DH>
struct LaneReads {
  static constexpr int PB = DH % 64 == 0 ? 8 : 4, RB = DH % 64 == 0 ? 2 : 1;
  int piece[PB];   // pieces 2 kk + lane / 32, kk < PB, of row lane % 32
  int row[4][RB];  // element 32 d + lane % 32, d < RB, of rows 4 (lane / 32) + r
  __device__ __forceinline__ LaneReads(int at, int lane) {
    const int half = lane >> 5, i = lane & 31;
#pragma unroll
    for (int k = 0; k < PB; ++k) {
      piece[k] = at + i * (DH * 4) + (((2 * k + half) ^ place_of<DH>(i)) << 4);
      asm volatile("" : "+v"(piece[k]));
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int d = 0; d < RB; ++d) {
        row[r][d] = at + (4 * half + r) * (DH * 4) + (((8 * d + (i >> 2)) ^ place_of<DH>(4 * half + r)) << 4) + (i & 3) * 4;
        asm volatile("" : "+v"(row[r][d]));
      }
  }
};
// c += rows of tile TILE times b over the head dimension.
template <int DH, int TILE>
__device__ __forceinline__ f32x16 dot_tile(const char* lds, const LaneReads<DH>& l, const f32x4 (&b)[DH / 8]) {
  constexpr int PB = LaneReads<DH>::PB;
  f32x16 c = zero16();
  auto piece = [&](int kk) {
    return *reinterpret_cast<const f32x4*>(lds + l.piece[kk % PB] + TILE * kTileBytes<DH> + kk / PB * PB * 32);
  };
  f32x4 a[2] = {piece(0), piece(1)};  // read two pieces ahead of their four MFMAs
#pragma unroll
  for (int kk = 0; kk < DH / 8; ++kk) {
    const f32x4 v = a[kk & 1];
    if (kk + 2 < DH / 8) a[kk & 1] = piece(kk + 2);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int j = 0; j < 4; ++j) c = mfma(v[j], b[kk][j], c);
  }
  return c;
}
// acc[d] += M^T w over the 32 rows of tile TILE: first operand rows of M, second w.
template <int DH, int TILE>
__device__ __forceinline__ void accumulate_rows(f32x16 (&acc)[DH / 32], const char* lds, const LaneReads<DH>& l,
                                                const f32x16& w) {
  constexpr int RB = LaneReads<DH>::RB, DT = DH / 32;
  auto element = [&](int e, int d) {
    return *reinterpret_cast<const float*>(lds + l.row[e & 3][d % RB] + TILE * kTileBytes<DH> + d / RB * RB * 128 +
                                           (e >> 2) * 8 * DH * 4);
  };
  constexpr int AHEAD = DT < 4 ? 3 : 2;  // a row is read that many steps ahead
  float a[4][DT];
#pragma unroll
  for (int e = 0; e < AHEAD; ++e)
#pragma unroll
    for (int d = 0; d < DT; ++d) a[e][d] = element(e, d);
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    if (e + AHEAD < 16)
#pragma unroll
      for (int d = 0; d < DT; ++d) a[(e + AHEAD) & 3][d] = element(e + AHEAD, d);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[d] = mfma(a[e & 3][d], w[e], acc[d]);
  }
}
// A partial result of one wave in LDS: [register][lane].
template <int N>
__device__ __forceinline__ void put_partial(float* p, const f32x16 (&acc)[N], int lane) {
#pragma unroll
  for (int d = 0; d < N; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) p[(d * 16 + e) * 64 + lane] = acc[d][e];
}
// The four waves' rows to redo, left in LDS before the barrier: all of them, and this wave's share (every fourth).
__device__ __forceinline__ uint32_t all_redo(const uint32_t* masks) {
  return __builtin_amdgcn_readfirstlane(masks[0] | masks[1] | masks[2] | masks[3]);
}
__device__ __forceinline__ uint32_t share_of(uint32_t redo, int wave) { return redo & (0x11111111u << wave); }
// Blocks by falling weight, of which every one finds a place at once: the first 256 go to a CU each, the next 256 to the same
// CUs in the same order, so every other such row is turned round: the heaviest block shares its CU with the lightest.
__device__ __forceinline__ int snake(int block, int blocks) {
  const int first = block & ~255;
  return first & 256 ? first + min(255, blocks - 1 - first) - (block - first) : block;
}

}  // namespace po
