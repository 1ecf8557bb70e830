// Rows in 8 bits: e4m3 codes and one power of two for each row (token and KV
// head), kept as a byte (exponent + 127; 255: the row is NaN).
#pragma once

#include "device_common.hpp"

namespace padoc {
namespace e4m3 {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kMinByte = 63;    // 2^-64
constexpr uint32_t kNan = 255;  // a row that is NaN

// Byte of a row whose largest magnitude has the fp32 bits `a`: the smallest
// exponent e with |x| <= 448 * 2^e.  448 = 1.75 * 2^8, so e = exponent(a) - 8,
// and one more where a's fraction is above 1.75: adding 0x1fffff to the bits
// carries into the exponent exactly then.  Rows with an infinity, a NaN or a
// magnitude of 248 * 2^120 and more (which would round to 2^128) are NaN.
__device__ __forceinline__ uint32_t scale_byte(uint32_t a) {
  if (a >= 0x7f780000u) return kNan;
  const int b = (int)((a + 0x1fffffu) >> 23) - 8;
  return (uint32_t)(b < kMinByte ? kMinByte : b);
}
// 2^-e of a byte (the row's values times it are within +-448; kNan gives some
// number), and 2^e.
__device__ __forceinline__ float inverse_scale(uint32_t b) { return __uint_as_float((254u - (b == kNan ? 127u : b)) << 23); }
__device__ __forceinline__ float scale_value(uint32_t b) { return __uint_as_float(b << 23); }  // kNan: infinity

// Codes of four values times s, rounded to nearest-even; K rows that are NaN hold
// NaN codes (their scores are NaN then, and masked like others), V rows zeros
// (their scale alone says so: a NaN code would reach every column of a product).
constexpr uint32_t kNanCodes = 0x7f7f7f7fu;
__device__ __forceinline__ uint32_t codes4(float x0, float x1, float x2, float x3, float s) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(x0 * s, x1 * s, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x2 * s, x3 * s, r, true);
}

// The bf16 values of eight codes times 2^e (`scale`; exact: a code has four
// significant bits).  NaN codes give NaN.
__device__ __forceinline__ bf16x8_t values8(uint32_t lo, uint32_t hi, float scale) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return bf16x8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// The fp32 values of four codes.
__device__ __forceinline__ void values4(uint32_t w, float (&x)[4]) {
  const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
  const auto b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  x[0] = a[0];
  x[1] = a[1];
  x[2] = b[0];
  x[3] = b[1];
}

// Bytes of the caches of one (block, KV head): its codes of K (and of V), its scales.
template <int D>
__device__ __forceinline__ int64_t codes_at(int64_t blk, int32_t kvh, int32_t Hkv) {
  return (blk * Hkv + kvh) * (D * kBlock);
}
__device__ __forceinline__ int64_t scales_at(int64_t blk, int32_t kvh, int32_t Hkv) {
  return (blk * Hkv + kvh) * (2 * kBlock);
}
// Byte of dims [c, ..) of token t within a (block, head)'s K codes.
__device__ __forceinline__ int k_at(int t, int c) { return (c >> 4) * (kBlock * 16) + t * 16 + (c & 15); }

// Whether a byte of w is 255.
__device__ __forceinline__ bool has_nan(uint32_t w) { return ((~w - 0x01010101u) & w & 0x80808080u) != 0; }

}  // namespace e4m3
}  // namespace padoc
