// Rows of K and V on their way into the paged cache: eight channels of a lane, their codes and the scales (cache.hip, cache_rope.hip).
#pragma once
#include "cache.h"

namespace dma {

// Eight channels of a lane, as they come, and as fp32.
template <typename T> struct Raw8;
template <> struct Raw8<__bf16> { uint4 x; };
template <> struct Raw8<float> { float4 a, b; };
__device__ __forceinline__ void load_raw(const __bf16* src, Raw8<__bf16>& r) { r.x = *reinterpret_cast<const uint4*>(src); }
__device__ __forceinline__ void load_raw(const float* src, Raw8<float>& r) {
  r.a = reinterpret_cast<const float4*>(src)[0];
  r.b = reinterpret_cast<const float4*>(src)[1];
}
__device__ __forceinline__ void to_f32(const Raw8<__bf16>& r, float* x) {
  const uint32_t u[4] = {r.x.x, r.x.y, r.x.z, r.x.w};
#pragma unroll
  for (int e = 0; e < 4; e++) {
    x[2 * e] = __uint_as_float(u[e] << 16);
    x[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
  }
}
__device__ __forceinline__ void to_f32(const Raw8<float>& r, float* x) {
  x[0] = r.a.x; x[1] = r.a.y; x[2] = r.a.z; x[3] = r.a.w;
  x[4] = r.b.x; x[5] = r.b.y; x[6] = r.b.z; x[7] = r.b.w;
}

// And out again: fp32 values rounded once, or as they came.
template <typename T> __device__ __forceinline__ void store8(T* dst, const float* x);
template <> __device__ __forceinline__ void store8(__bf16* dst, const float* x) {
  bf16x8 v;
#pragma unroll
  for (int e = 0; e < 8; e++) v[e] = (__bf16)x[e];
  *reinterpret_cast<bf16x8*>(dst) = v;
}
template <> __device__ __forceinline__ void store8(float* dst, const float* x) {
  reinterpret_cast<float4*>(dst)[0] = make_float4(x[0], x[1], x[2], x[3]);
  reinterpret_cast<float4*>(dst)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void store_raw(__bf16* dst, const Raw8<__bf16>& r) { *reinterpret_cast<uint4*>(dst) = r.x; }
__device__ __forceinline__ void store_raw(float* dst, const Raw8<float>& r) {
  reinterpret_cast<float4*>(dst)[0] = r.a;
  reinterpret_cast<float4*>(dst)[1] = r.b;
}

template <int CTRL> __device__ __forceinline__ uint32_t dpp_quad(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true);
}
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

// The scale byte that four neighbouring lanes (32 channels) share, from the bits of the largest magnitude of a lane's (as integers: the
// bits of NaN are above those of every number): the power of two at which it rounds to at most 6, 2^(exponent - 2) or, from a
// mantissa of 1.75 on, twice that.  A block that holds an infinity or NaN has the byte 255.  Bytes 2 to 252: what the cache holds is
// finite and normal in fp32 and bf16 alike.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
  top = max(top, dpp_quad<0xb1>(top));
  top = max(top, dpp_quad<0x4e>(top));
  return top >= 0x7f800000u ? 255u : (uint32_t)max(2, min(252, (int)((top + 0x200000u) >> 23) - 2));
}
// The codes of a lane's eight channels, and that byte.
__device__ __forceinline__ uint32_t quantise8(const Raw8<__bf16>& r, uint32_t& byte) {
  const uint32_t u[4] = {r.x.x, r.x.y, r.x.z, r.x.w};
  u16x2 top = __builtin_bit_cast(u16x2, u[0] & 0x7fff7fffu);
#pragma unroll
  for (int e = 1; e < 4; e++) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, u[e] & 0x7fff7fffu));
  byte = scale_byte((uint32_t)max(top[0], top[1]) << 16);
  const float scale = mx_scale(byte);
  uint32_t code = 0;
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, __builtin_bit_cast(bf16x2, u[0]), scale, 0);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, __builtin_bit_cast(bf16x2, u[1]), scale, 1);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, __builtin_bit_cast(bf16x2, u[2]), scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, __builtin_bit_cast(bf16x2, u[3]), scale, 3);
}
__device__ __forceinline__ uint32_t quantise8(const Raw8<float>& r, uint32_t& byte) {
  float x[8];
  to_f32(r, x);
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; e++) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
  byte = scale_byte(top);
  const float scale = mx_scale(byte);
  uint32_t code = 0;
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[0], x[1], scale, 0);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[2], x[3], scale, 1);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[4], x[5], scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[6], x[7], scale, 3);
}

}  // namespace dma
