// fp8.cuh -- e4m3 codes with a power of two beside them (caches in 8 bits).
#pragma once
#include "common.cuh"

namespace kvk {

// What stands at p, or `other` where `in` is not set, by one predicated load: a value
// chosen behind the load would be a look at it, which waits for it.
#define KVK_LOAD_IF(name, T, op)                                                                              \
  __device__ __forceinline__ int name(const T *p, bool in, int other) {                                      \
    int r;                                                                                                    \
    asm volatile("{\n .reg .pred q;\n setp.ne.u32 q, %2, 0;\n mov.b32 %0, %3;\n @q ld.global." op " %0, [%1];\n}\n" \
                 : "=&r"(r)                                                                                   \
                 : "l"(p), "r"(in ? 1u : 0u), "r"(other));                                                    \
    return r;                                                                                                 \
  }
KVK_LOAD_IF(load_if, int32_t, "s32")
KVK_LOAD_IF(load_if, uint16_t, "u16")
KVK_LOAD_IF(load_if, uint8_t, "u8")
KVK_LOAD_IF(load_if, int8_t, "s8")
#undef KVK_LOAD_IF

// 2^e, -126 <= e <= 127
__device__ __forceinline__ float pow2f(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// least e in [lo, hi] with top <= 448 2^e = 1.75 2^(e + 8)
__device__ __forceinline__ int code_exponent(float top, int lo, int hi) {
  const uint32_t b = __float_as_uint(top);
  return min(max((int)(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0), lo), hi);
}

// two codes, nearest even, at most 448 in magnitude; NaN to 0x7f
__device__ __forceinline__ uint32_t code2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t code2_of_f16(uint32_t h) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(r) : "r"(h));
  return r;
}
// two codes as f16 (exact)
__device__ __forceinline__ uint32_t code2_f16(uint32_t c) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)c));
  return r;
}
__device__ __forceinline__ float finite_or_nan(float x) { return fabsf(x) <= 3.4028234e38f ? x : __int_as_float(0x7fc00000); }

// the codes of two pairs of the dtype, times the power of two `up`; finite numbers, and
// any (those that are not finite to NaN)
// (f16: the product is exact, or below 2^-14 and so the code 0 however it is rounded)
template <bool BF16>
__device__ __forceinline__ uint32_t code4(uint32_t a, uint32_t b, float up) {
  if constexpr (BF16) {
    const float2 x = unpack2<BF16>(a), y = unpack2<BF16>(b);
    return code2(x.x * up, x.y * up) | code2(y.x * up, y.y * up) << 16;
  } else {
    const uint32_t f = pack_f16(up, up);
    return code2_of_f16(hmul2_u32(a, f)) | code2_of_f16(hmul2_u32(b, f)) << 16;
  }
}
template <bool BF16>
__device__ __forceinline__ uint32_t code4_any(uint32_t a, uint32_t b, float up) {
  const float2 x = unpack2<BF16>(a), y = unpack2<BF16>(b);
  return code2(finite_or_nan(x.x) * up, finite_or_nan(x.y) * up) | code2(finite_or_nan(y.x) * up, finite_or_nan(y.y) * up) << 16;
}
// the codes nearest to four codes times a power of two
__device__ __forceinline__ uint32_t codes_times(uint32_t c, float down) {
  const float2 x = unpack2<false>(code2_f16(c & 0xffffu)), y = unpack2<false>(code2_f16(c >> 16));
  return code2(x.x * down, x.y * down) | code2(y.x * down, y.y * down) << 16;
}

}  // namespace kvk
