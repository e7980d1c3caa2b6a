// The 8-bit form of a saved activation [rows, cols], and how a lane makes and reads it.
//
// One buffer: codes uint8 [rows, C], then scale bytes uint8 [rows, C / 32], C = cols rounded up to 32 (codes behind the last column
// are zeros).  A block is 32 consecutive columns of a row.  Its exponent e is the least integer, at least -117, with amax <= 448 2^e
// (amax: its largest finite magnitude), its scale byte e + 127, a code the e4m3 number (four bits of exponent, three of fraction, largest
// 448) nearest to x / 2^e, ties to even.  What is not finite becomes NaN; magnitudes are cut at 1.875 2^127, so that no value is
// rounded to an infinity.
//
// A scale that is a power of two makes a restored value four significant bits and an exponent: exact in bf16 as in fp32, so every reader
// of a checkpoint, whatever it computes in, sees the same numbers.  e >= -117 keeps each of them zero or a normal number.
// The one rounding to fewer bits, at most 2^-4 of a value (2^-10 2^e for those under 2^-6 2^e), is the point of the form: 1.03 bytes a value.
#pragma once

#include "kernels.h"

namespace po {

constexpr int kSaved8Block = 32;
constexpr unsigned kSaved8LeastByte = 127 - 117;

inline int64_t saved8_cols(int64_t cols) { return (cols + kSaved8Block - 1) / kSaved8Block * kSaved8Block; }
inline int64_t saved8_codes(int rows, int cols) { return rows * saved8_cols(cols); }
inline uint64_t saved8_bytes(int rows, int cols) {
  const int64_t n = saved8_codes(rows, cols);
  return (uint64_t)(n + n / kSaved8Block + 15) / 16 * 16;
}

// Scale byte of a block whose largest finite magnitude is amax = m 2^E: E - 8, one more where m is over 1.75.
__device__ __forceinline__ unsigned saved8_scale_byte(float amax) {
  return max((__float_as_uint(amax) + 0x1fffffu) >> 23, kSaved8LeastByte + 8u) - 8u;
}
__device__ __forceinline__ float saved8_scale(unsigned byte) { return __uint_as_float(byte << 23); }
__device__ __forceinline__ float saved8_inverse(unsigned byte) { return __uint_as_float((254u - byte) << 23); }

// The largest of four neighbouring lanes, in all of them.
__device__ __forceinline__ float max_of_four(float v) {
  v = fmaxf(v, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0xb1, 0xf, 0xf, true)));  // lanes 1 0 3 2
  return fmaxf(v, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x4e, 0xf, 0xf, true)));  // lanes 2 3 0 1
}
__device__ __forceinline__ float amax_of(const float (&v)[8]) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float a = fabsf(v[i]);
    m = fmaxf(m, a < __builtin_inff() ? a : 0.f);
  }
  return m;
}
// Eight columns into their codes.  Four neighbouring lanes hold a block, all of them call it; `byte`: the block's scale byte.
__device__ __forceinline__ uint2 saved8_encode(const float (&v)[8], unsigned& byte) {
  byte = saved8_scale_byte(max_of_four(amax_of(v)));
  const float inverse = saved8_inverse(byte), most = 0x1.Ep127f;
  float w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i)
    w[i] = fabsf(v[i]) < __builtin_inff() ? fminf(fmaxf(v[i], -most), most) * inverse : __builtin_nanf("");
  int lo = 0, hi = 0;
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(w[0], w[1], lo, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(w[2], w[3], lo, true);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(w[4], w[5], hi, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(w[6], w[7], hi, true);
  return make_uint2((unsigned)lo, (unsigned)hi);
}
__device__ __forceinline__ void saved8_decode(uint2 codes, unsigned byte, float (&v)[8]) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const float scale = saved8_scale(byte);
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes.x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes.x, true);
  const f32x2 c = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes.y, false), d = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes.y, true);
  v[0] = a[0] * scale;
  v[1] = a[1] * scale;
  v[2] = b[0] * scale;
  v[3] = b[1] * scale;
  v[4] = c[0] * scale;
  v[5] = c[1] * scale;
  v[6] = d[0] * scale;
  v[7] = d[1] * scale;
}

// Eight columns of a row from `p` on, of which `n` are there (the others: zero): one vector from wherever it
// starts where all eight are there (4096 rows of 4097, bf16: saved in 11.6 us, with single values 26.5; of 4096 10.8).
template <typename T>
__device__ __forceinline__ void load_eight(float (&v)[8], const T* p, int n) {
  if (n >= 8) {
    T x[8];
    __builtin_memcpy(x, p, sizeof(x));
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = to_f32(x[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? to_f32(p[i]) : 0.f;
  }
}
// Results that no later part of the same kernel reads are stored past the caches (non-temporal): they are too large to be kept there, and lines
// that are only written cost reads of others (a saved set of 168 million values restored: 123 us, so 86).
__device__ __forceinline__ void store_past(void* p, uint4 v) {
  typedef unsigned u4 __attribute__((ext_vector_type(4)));
  __builtin_nontemporal_store(u4{v.x, v.y, v.z, v.w}, reinterpret_cast<u4*>(p));
}
__device__ __forceinline__ void store_past(void* p, uint2 v) {
  typedef unsigned u2 __attribute__((ext_vector_type(2)));
  __builtin_nontemporal_store(u2{v.x, v.y}, reinterpret_cast<u2*>(p));
}
template <typename T>
__device__ __forceinline__ void store_eight(T* p, const float (&v)[8], int n) {
  constexpr int V = Vec16<T>::N;
  if (n >= 8) {
    typedef unsigned anywhere __attribute__((ext_vector_type(4), aligned(2)));
#pragma unroll
    for (int k = 0; k < 8; k += V) {
      Vec16<T> x;
#pragma unroll
      for (int i = 0; i < V; ++i) x.v[i] = from_f32<T>(v[k + i]);
      __builtin_nontemporal_store(__builtin_bit_cast(anywhere, x), reinterpret_cast<anywhere*>(p + k));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = from_f32<T>(v[i]);
  }
}

// Whether two ranges of memory share a byte.
inline bool overlap(const void* a, uint64_t a_bytes, const void* b, uint64_t b_bytes) {
  const uint64_t p = (uint64_t)(uintptr_t)a, q = (uint64_t)(uintptr_t)b;
  return a && b && p < q + b_bytes && q < p + a_bytes;
}

}  // namespace po
