// The 8-bit cache's format: e4m3 codes and a power-of-two scale per row.
//
//   a = max |v|;  k = least integer >= -96 with a <= 448 * 2^k (0 for a row of zeros);  code = e4m3(v 2^-k);  byte = k + 127
// A power of two costs a floating-point code nothing against a / 448: the relative step is the same in every binade, and a
// lands in (224, 448] 2^k, so at most one of the 18 binades below it is given away.  In return every code times its
// scale is exact in bf16, scales multiply exactly, and a byte holds them.
// Rows whose largest number is below 2^-96 448 lose what is smaller than 2^-106; the limit keeps 2^-k and what the
// attention kernels form with it (probabilities times 2^k) inside fp32.  No call writes a byte below 31.
#pragma once

#include <cuda_fp8.h>

#include "ta_common.cuh"

namespace ta {

// A code as the kernels' templates see it.
struct e4m3 {
  uint8_t v;
};

namespace q8 {

constexpr int kNan = 255, kMinByte = 127 - 96;

// Scale byte of a row from the bits of its largest |v| (compared as unsigned numbers, so that a NaN is the largest).
__host__ __device__ __forceinline__ int scale_byte(uint32_t amax_bits) {
  if (amax_bits == 0) return 127;
  if (amax_bits >= 0x7f800000u) return kNan;
  const int b = (int)(amax_bits >> 23) - 8 + ((amax_bits & 0x7fffffu) > 0x600000u ? 1 : 0);      // 448 = 1.75 * 2^8
  return b < kMinByte ? kMinByte : b;
}
// 2^-k of a byte that scale_byte returned
__host__ __device__ __forceinline__ uint32_t inverse_bits(int byte) { return byte == kNan ? 0x7fc00000u : (uint32_t)(254 - byte) << 23; }
// 2^k of any byte (0: a subnormal; 255: NaN)
__host__ __device__ __forceinline__ uint32_t scale_bits(int byte) {
  return byte == kNan ? 0x7fc00000u : (byte == 0 ? 0x00400000u : (uint32_t)byte << 23);
}

#if defined(__CUDACC__)
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }
__device__ __forceinline__ float scale(int byte) { return __uint_as_float(scale_bits(byte)); }
__device__ __forceinline__ float inverse(int byte) { return __uint_as_float(inverse_bits(byte)); }
// codes of a, b in the low and high byte (NaN: 0x7f)
__device__ __forceinline__ uint32_t codes2(float a, float b) { return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3); }
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) { return codes2(a, b) | codes2(c, d) << 16; }
__device__ __forceinline__ float2 values2(uint32_t codes) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(codes & 0xffffu), __NV_E4M3);
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}
__device__ __forceinline__ float value(uint8_t code) { return values2(code).x; }
// the eight values of eight codes
__device__ __forceinline__ void values8(uint2 c, float (&f)[8]) {
  const uint32_t w[4] = {c.x, c.x >> 16, c.y, c.y >> 16};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 v = values2(w[e]);
    f[2 * e] = v.x; f[2 * e + 1] = v.y;
  }
}
__device__ __forceinline__ uint2 codes8(const float (&f)[8], float inv) {
  return make_uint2(codes4(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv), codes4(f[4] * inv, f[5] * inv, f[6] * inv, f[7] * inv));
}
#endif

}  // namespace q8
}  // namespace ta
