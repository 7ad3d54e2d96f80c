// e4m3 codes with a scale for every block of 16 rows of a head: what the kernels that write such pages share.
#pragma once
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace rest_e4m3 {

constexpr int kBlockRows = 16;                          // rows that share a scale (the smallest page)
constexpr float kLeastScale = 0x1p-60f, kMostScale = 0x1p60f;

// The smallest power of two s with most <= 448 s, within the limits of scales.  448 = 1.75 * 2^8, so the exponent
// of `most` decides, and whether its fraction exceeds 1.75.
__device__ __forceinline__ float fitting_scale(float most) {
  const uint32_t bits = __float_as_uint(most);
  const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7FFFFFu) > 0x600000u);
  return __uint_as_float((uint32_t)(min(max(e, -60), 60) + 127) << 23);
}
__device__ __forceinline__ float within_limits(float s) { return fminf(fmaxf(s, kLeastScale), kMostScale); }   // NaN: the least

// two codes, the first in the low byte; NaN stays NaN, what is beyond 448 becomes 448
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  return __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ float2 unpack2(uint32_t two) {
  return __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3)));
}
// four codes as other multiples of their scale
__device__ __forceinline__ uint32_t rescale4(uint32_t x, float ratio) {
  const float2 a = unpack2(x & 0xFFFFu), b = unpack2(x >> 16);
  return pack2(a.x * ratio, a.y * ratio) | pack2(b.x * ratio, b.y * ratio) << 16;
}
__device__ __forceinline__ uint4 rescale16(uint4 x, float ratio) {
  return make_uint4(rescale4(x.x, ratio), rescale4(x.y, ratio), rescale4(x.z, ratio), rescale4(x.w, ratio));
}
// the largest magnitude among 16 codes, NaN passed over
__device__ __forceinline__ float largest16(uint4 x) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t code = w[i] >> (8 * j) & 0x7Fu;
      top = max(top, code == 0x7Fu ? 0u : code);        // (magnitudes are ordered like their codes)
    }
  return unpack2(top).x;
}
__device__ __forceinline__ float warp_max(float x) {
#pragma unroll
  for (int d = 16; d; d >>= 1) x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, d));
  return x;
}

}  // namespace rest_e4m3
