// e4m3 codes with block scales and the 16-bit element types: what the quantizer and the norms share.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace mixaq {

constexpr int FP8_BLOCK = 128;                 // columns that share a scale

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
template <class T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// Eight consecutive elements as they lie in memory
template <class T> struct Vec8 { T v[8]; };
// a load of memory that the kernel itself may write later (rows updated in place); p 16-byte aligned
template <class T> __device__ __forceinline__ void load_row8(const T* p, Vec8<T>& r) {
  uint4* d = reinterpret_cast<uint4*>(&r);
#pragma unroll
  for (int i = 0; i < (int)sizeof(Vec8<T>) / 16; ++i) d[i] = reinterpret_cast<const uint4*>(p)[i];
}
// max(|a|, |b|), no number if either is none (the sign of the result means nothing)
__device__ __forceinline__ float max_abs(float a, float b) {
  float r;
  asm("max.NaN.xorsign.abs.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// Scale of a block and its reciprocal.  A power of two is taken from the exponent field: 448 = 1.75 * 2^8, so amax <= 448 * 2^j holds
// for the exponent of amax less 8, or one more where its mantissa is above 1.75 (which the addition carries into the exponent).
__device__ __forceinline__ void block_scale(float amax, bool pow2, float& scale, float& inv) {
  const float a = fabsf(amax);
  if (pow2) {
    const int e = max((int)((__float_as_uint(a) + 0x1fffffu) >> 23) - 8, 1);
    scale = __uint_as_float((uint32_t)e << 23);
    inv = __uint_as_float((uint32_t)(254 - e) << 23);
  } else {
    // a / 448, correctly rounded (Markstein): the product with the rounded reciprocal, corrected by its exact remainder
    const float r = 2.23214296e-3f, t = __fmul_rn(a, r);
    scale = fmaxf(__fmaf_rn(__fmaf_rn(-448.0f, t, a), r, t), 1.17549435e-38f);
    inv = __frcp_rn(scale);
  }
  if (!(a <= 3.402823466e38f)) scale = inv = __uint_as_float(0x7fc00000u);
}

// four values to four codes
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
  return lo | (hi << 16);
}
__device__ __forceinline__ uint2 codes8(const float2 (&f)[4], float inv) {
  float2 t[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) t[i] = __fmul2_rn(f[i], make_float2(inv, inv));
  return make_uint2(codes4(t[0].x, t[0].y, t[1].x, t[1].y), codes4(t[2].x, t[2].y, t[3].x, t[3].y));
}
__device__ __forceinline__ uint2 codes8(const float (&f)[8], float inv) {
  return make_uint2(codes4(__fmul_rn(f[0], inv), __fmul_rn(f[1], inv), __fmul_rn(f[2], inv), __fmul_rn(f[3], inv)),
                    codes4(__fmul_rn(f[4], inv), __fmul_rn(f[5], inv), __fmul_rn(f[6], inv), __fmul_rn(f[7], inv)));
}
__device__ __forceinline__ void store_codes(uint8_t* p, uint2 w, int n) {                  // p 8-byte aligned; the first n codes
  if (n >= 8) { *reinterpret_cast<uint2*>(p) = w; return; }
#pragma unroll
  for (int i = 0; i < 8; ++i) if (i < n) p[i] = (uint8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
}

}  // namespace mixaq
