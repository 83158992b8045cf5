// The 16-bit element types of the generation operators (fp16 and bf16), two
// values to a 32-bit register.
#pragma once

#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

namespace p4q {

template <bool kBf16>
__device__ __forceinline__ float2 unpack2(uint32_t u) {
  if (kBf16) return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&u));
  return __half22float2(*reinterpret_cast<const __half2*>(&u));
}

// Rounds to nearest even; x in the low half.
template <bool kBf16>
__device__ __forceinline__ uint32_t pack2(float x, float y) {
  if (kBf16) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  const __half2 h = __floats2half2_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&h);
}

template <bool kBf16>
__device__ __forceinline__ float from16(uint16_t b) {
  if (kBf16) return __uint_as_float(static_cast<uint32_t>(b) << 16);
  return __half2float(__ushort_as_half(b));
}

}  // namespace p4q
