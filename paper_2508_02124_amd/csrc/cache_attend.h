// Attention from the paged cache: what its kernels share (cache_decode.hip, cache_prefix.hip).
#pragma once
#include "cache.h"
#include "select.h"

namespace dma {

template <int N, typename F> __device__ __forceinline__ float over_groups(float x, F&& op) {  // over the lanes l % N
  if constexpr (N == 2) x = op(x, dpp_move<0x4e>(x));
  if constexpr (N <= 4) x = op(x, dpp_move<0x124>(x));
  x = op(x, dpp_move<0x128>(x));
  const unsigned u = __builtin_bit_cast(unsigned, x);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  x = op(__builtin_bit_cast(float, (unsigned)a[0]), __builtin_bit_cast(float, (unsigned)a[1]));
  const unsigned v = __builtin_bit_cast(unsigned, x);
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return op(__builtin_bit_cast(float, (unsigned)b[0]), __builtin_bit_cast(float, (unsigned)b[1]));
}
template <int N> __device__ __forceinline__ float lanes_sum(float x) {  // over N neighbouring lanes
  if constexpr (N == 8) return group_sum<8>(x);
  if constexpr (N == 4) x += dpp_move<0x4e>(x);
  return x + dpp_move<0xb1>(x);
}

// e^(s - ref).  Scores stay in natural units: times log2(e), those of masked keys (the type's lowest value) would be infinite.
__device__ __forceinline__ float weight(float s, float ref) { return fast_exp2((s - ref) * LOG2E); }

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// q . k over the 32 channels of a lane: bf16 queries multiply pairs of bf16 values (what the cache holds is exact in bf16), fp32
// ones fp32 values.
template <typename TQ> struct Query;
template <> struct Query<__bf16> {
  uint4 x[4];
  __device__ __forceinline__ void load(const __bf16* q) {
#pragma unroll
    for (int i = 0; i < 4; i++) x[i] = reinterpret_cast<const uint4*>(q)[i];
  }
  template <int I> __device__ __forceinline__ float dot8(uint32_t code, float sc, float s) const {
    const uint32_t q[4] = {x[I].x, x[I].y, x[I].z, x[I].w};
    static_for<4>([&](auto b) {
      constexpr int B = decltype(b)::value;
      s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, q[B]), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, sc, B), s, false);
    });
    return s;
  }
};
template <> struct Query<float> {
  float x[32];
  __device__ __forceinline__ void load(const float* q) {
#pragma unroll
    for (int i = 0; i < 32; i++) x[i] = q[i];
  }
  template <int I> __device__ __forceinline__ float dot8(uint32_t code, float sc, float s) const {
    static_for<4>([&](auto b) {
      constexpr int B = decltype(b)::value;
      const auto v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, sc, B);
      s = fmaf(x[8 * I + 2 * B], v[0], s);
      s = fmaf(x[8 * I + 2 * B + 1], v[1], s);
    });
    return s;
  }
};

}  // namespace dma
