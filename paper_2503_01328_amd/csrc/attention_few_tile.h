// What the bf16 attention kernels whose blocks own 32 rows share: their stages in LDS, a wave's loads of a tile of 32 rows, products
// with such a tile, partial results of waves.
#pragma once

#include "attention_rows.h"
#include "attention_tile.h"

namespace po {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kRows = 32;  // of a tile and of a block

// Waves of a block, their stages, bytes of a tile and of a stage (two tiles), and where in LDS what follows the stages begins.  Heads
// of 128 need more than 256 registers in the backward: one wave per SIMD.  In the forward they have eight waves too, for which LDS has
// room for one stage each: the next K is requested once the scores are formed, the next V behind the product (four waves of two
// stages / this, us: 100 rows, 16 heads 6.1 / 5.6, 512 rows, 8 heads 9.0 / 8.6, 777 rows, 10 heads 15.2 / 12.0, 4096 rows, 2 heads 40.6 / 28.7).
template <int DH, bool FORWARD = false>
struct Few {
  static constexpr int W = DH == 64 || FORWARD ? 8 : 4, NS = DH == 64 || !FORWARD ? 2 : 1, TILE = kRows * DH * 2, STAGE = 2 * TILE, LOADS = TILE / 1024;
  static constexpr int AFTER = W * NS * STAGE;
};

__device__ __forceinline__ f32x16 zero16() {
  f32x16 z;
#pragma unroll
  for (int e = 0; e < 16; ++e) z[e] = 0.f;
  return z;
}

// A wave's loads of a tile of 32 rows that are ld elements apart: the byte offset of a lane's 16 bytes in each of them.
template <int DH>
struct TileLoads {
  unsigned off[Few<DH>::LOADS];
  __device__ __forceinline__ TileLoads(int ld, int lane) {
#pragma unroll
    for (int u = 0; u < Few<DH>::LOADS; ++u) {
      const int byte = u * 1024 + lane * 16, row = byte / (DH * 2), c = (byte % (DH * 2) >> 4) ^ swz<DH>(row);
      off[u] = (unsigned)row * (unsigned)ld * 2u + c * 16;
    }
  }
  // Rows row0 .. row0 + 31 of the matrix at m into the tile at LDS byte `tile`; rows from s on become zeros.
  __device__ __forceinline__ void request(unsigned tile, const bf16* m, int ld, int row0, int s) const {
    const int rows = min(s - row0, kRows);  // at least one
    const i32x4 buf = buffer_of(m + (size_t)row0 * ld, ((unsigned)(rows - 1) * (unsigned)ld + DH) * 2u);
#pragma unroll
    for (int u = 0; u < Few<DH>::LOADS; ++u) buffer_to_lds(tile + 1024u * u, off[u], buf);
  }
};
// Lane L's 4 bytes at p land in LDS at lds + 4 L.
__device__ __forceinline__ void float_to_lds(unsigned lds, const float* p) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds), "v"(p) : "memory");
}

// A maximum in units of the exponent, rounded once: what a sum is scaled by cancels exactly where it is scaled again, between tiles, in
// the merge and in lse, which a product fused into those differences would not (scores of deviation 6, 2048 rows: lse 6.7e-8 off,
// as the 128-row blocks' is 5.5e-8).
__device__ __forceinline__ float exponent_of(float m, float c) {
#pragma clang fp contract(off)
  return m * c;
}

// c += rows of the tile times b over the head dimension.
template <int DH>
__device__ __forceinline__ f32x16 dot_tile(const char* tile, const bf16x8 (&b)[DH / 16], f32x16 c, int lane) {
#pragma unroll
  for (int kk = 0; kk < DH / 16; ++kk)
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_row_fragment<DH>(tile, lane & 31, 2 * kk + (lane >> 5)), b[kk], c, 0, 0, 0);
  return c;
}
// acc[d] += tile^T w over the tile's 32 rows.
template <int DH, bool EDGE>
__device__ __forceinline__ void accumulate_tile(f32x16 (&acc)[DH / 32], const char* tile, const f32x16& w, int lane) {
#pragma unroll
  for (int st = 0; st < 2; ++st) {
    const Weights<EDGE> terms = weights_of<EDGE>(w, 8 * st);
#pragma unroll
    for (int d = 0; d < DH / 32; ++d)
      acc[d] = multiply<EDGE>(read_tr_fragment<DH>(tile, 16 * st, 32 * d, lane), terms, acc[d]);
  }
}
template <int DH>
__device__ __forceinline__ void load_row(bf16x8 (&f)[DH / 16], const bf16* row, int half) {
#pragma unroll
  for (int kk = 0; kk < DH / 16; ++kk) f[kk] = *reinterpret_cast<const bf16x8*>(row + 16 * kk + 8 * half);
}
// A partial result of one wave in LDS: [register][lane].
template <int N>
__device__ __forceinline__ void put_partial(float* p, const f32x16 (&acc)[N], int lane) {
#pragma unroll
  for (int d = 0; d < N; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) p[(d * 16 + e) * 64 + lane] = acc[d][e];
}
// The waves' rows to redo, left in LDS before the barrier: all of them, and this wave's share.
template <int W>
__device__ __forceinline__ uint32_t all_redo(const uint32_t* masks) {
  uint32_t m = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) m |= masks[w];
  return __builtin_amdgcn_readfirstlane(m);
}
template <int W>
__device__ __forceinline__ uint32_t share_of(uint32_t redo, int wave) {
  return redo & ((W == 8 ? 0x01010101u : 0x11111111u) << wave);
}
__device__ __forceinline__ void store4(bf16* p, const f32x4& v) {
  bf16x4 b;
#pragma unroll
  for (int r = 0; r < 4; ++r) b[r] = (bf16)v[r];
  *reinterpret_cast<bf16x4*>(p) = b;
}

}  // namespace po
