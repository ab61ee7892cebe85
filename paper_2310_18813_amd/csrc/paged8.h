// A paged cache of 8 bits: e4m3 codes (OCP: 448 the largest, 0x7f and 0xff NaN, no infinities) times a power of two for every
// position and key head.
//
// The scale is a power of two so that it rounds nothing: a code is a floating-point number, with the same three bits behind its leading one
// wherever the scale puts it, and code times scale is a bf16 or fp16 number, which the matrix cores take as it is.  gfx950 multiplies by
// it while it converts.
#pragma once
#include "paged.h"

namespace spec {

struct e4m3_t { uint8_t v; };

// What limits the scales of a cache for rows of type T.
//   least   the least exponent: fp16's smallest number is 2^-24, the smallest code 2^-9; for bf16 far above the edge of its range
//   most    the largest number of four bits that the type holds: larger magnitudes become it (off by less than 1 / 16 of themselves, as any code may be)
//   beyond  from here on a magnitude rounds to the type's infinity
template <class T> struct Codes;
template <> struct Codes<bf16_t> {
  static constexpr int least = -100;
  static constexpr float most = 0x1.ep127f, beyond = 0x1.ffp127f;
};
template <> struct Codes<f16_t> {
  static constexpr int least = -15;
  static constexpr float most = 61440.f, beyond = 65520.f;
};

// 64 bits to 32 so that what is rounded to a few bits afterwards is rounded as if at once: the low bits are cut off, and where they were not zero the
// last one kept is 1.
__device__ __forceinline__ float to_odd(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t hi = (uint32_t)(u >> 32) | min((uint32_t)u, 1u);
  return (float)__builtin_bit_cast(double, (uint64_t)hi << 32);
}

__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// Where the scale of a position and key head lies.
__device__ __forceinline__ size_t paged_scale(const PagedArgs &a, int page, int h, int pos) {
  return (((size_t)(uint32_t)page * a.n_kv_heads + h) << a.page_shift) + (pos & ((1 << a.page_shift) - 1));
}


// Two codes of a word (the upper ones: HI), times a power of two, as two values of type T.
template <class T, bool HI> __device__ __forceinline__ uint32_t decode2(uint32_t w, float scale) {
  if constexpr (std::is_same<T, bf16_t>::value) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HI));
  else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, HI));
}
// 16 codes
template <class T> __device__ __forceinline__ void decode16(const u32x4_v &c, float scale, u32x4_v &y0, u32x4_v &y1) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    y0[2 * i] = decode2<T, false>(c[i], scale); y0[2 * i + 1] = decode2<T, true>(c[i], scale);
    y1[2 * i] = decode2<T, false>(c[2 + i], scale); y1[2 * i + 1] = decode2<T, true>(c[2 + i], scale);
  }
}

}  // namespace spec
