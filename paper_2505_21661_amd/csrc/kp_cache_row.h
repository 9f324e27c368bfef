// A row of keys or values of the paged cache, as it is written.
//
// A row of D values becomes D e4m3 codes and one exponent byte: top = its largest finite magnitude, e the least integer
// with top <= 448 2^e, code = top-preserving round to nearest even of x 2^-e.  With top = 1.f 2^x, 448 = 1.75 2^8: e is
// x - 8 where 1.f <= 1.75, x - 7 otherwise, read off the bits of top.  The scaling is exact, so the code carries one
// rounding (at most 2^-4 of the value, 2^-10 2^e below 2^-6 2^e) and the row reads back exactly as the codes say.
#pragma once
#include "kp_attn.h"

namespace kp {
namespace attn {

// Codes of the 8 values that lane c of a row's D / 8 lanes has, and the row's exponent byte; all of them call it.
template <class T, int D>
__device__ __forceinline__ u32x2 quantise_row(const u32x4& raw, uint8_t* exponent) {
  float x[8], top = 0.f;
#pragma unroll
  for (int n = 0; n < 8; ++n) {
    x[n] = T::to_float((raw[n >> 1] >> (16 * (n & 1))) & 0xFFFFu);
    const bool finite = __builtin_fabsf(x[n]) < INFINITY;
    top = fmaxf(top, finite ? __builtin_fabsf(x[n]) : 0.f);
    x[n] = finite ? x[n] : __builtin_nanf("");
  }
#pragma unroll
  for (int d = 1; d < D / 8; d <<= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
  const uint32_t bits = __builtin_bit_cast(uint32_t, top);
  int e = (int)(bits >> 23) - ((bits & 0x7FFFFFu) <= 0x600000u ? 135 : 134);
  e = top == 0.f ? 0 : (e < -126 ? -126 : e);
  const float scale = __builtin_bit_cast(float, (uint32_t)(127 - e) << 23);
  u32x2 codes;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    int p = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * w] * scale, x[4 * w + 1] * scale, 0, false);
    p = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * w + 2] * scale, x[4 * w + 3] * scale, p, true);
    codes[w] = (uint32_t)p;
  }
  *exponent = (uint8_t)(e + 127);
  return codes;
}

// Number of the row of the cache that a slot holds of a head.
__device__ __forceinline__ uint32_t row_of_slot(uint64_t slot, uint32_t head, uint32_t hkv, uint32_t page_log2) {
  const uint32_t page = (uint32_t)(slot >> page_log2), in = (uint32_t)slot & ((1u << page_log2) - 1u);
  return ((page * hkv + head) << page_log2) + in;
}

// Lane c's part of a row to where it belongs: copied or quantised.
template <class T, int D, bool E4M3>
__device__ __forceinline__ void put_row(const u32x4& raw, uint8_t* cache, uint8_t* exps, uint32_t row, uint32_t c) {
  if constexpr (!E4M3) {
    *reinterpret_cast<u32x4*>(cache + (size_t)row * (2 * D) + 16u * c) = raw;
  } else {
    uint8_t exponent;
    const u32x2 codes = quantise_row<T, D>(raw, &exponent);
    *reinterpret_cast<u32x2*>(cache + (size_t)row * D + 8u * c) = codes;
    if (c == 0) exps[row] = exponent;
  }
}

}  // namespace attn
}  // namespace kp
