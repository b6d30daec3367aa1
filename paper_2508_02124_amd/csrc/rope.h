// Rotary positions: what the kernels that turn pairs of channels share (rope.hip, cache_rope.hip).
#pragma once
#include "cache.h"

namespace dma {

// A head's first `rot` channels in pairs: (i, i + rot / 2), or the neighbours (2 i, 2 i + 1).  Pair i turns by position * freqs[i].
struct RopeArgs {
  const float* freqs;
  int rot;
};

#ifdef __HIPCC__
struct Turn {
  double c, s;
};

// Cosine and sine of position * f, to about 1e-16.  The product of 31 and 24 bits is held in two doubles, and its multiple of
// pi / 2 subtracted in two parts (pi / 2 = HI + LO), so that far positions lose nothing; what is left, at most pi / 4, goes through
// Taylor's series (the first term left out is below 1e-18).  In 32 bits an angle of 10^5 radians would be off by 0.004.
__device__ __forceinline__ Turn turn_of(int position, float f) {
  constexpr double HI = 1.57079632679489661923, LO = 6.12323399573676588613e-17, PER = 0.63661977236758134308;
  constexpr double ROUND = 6755399441055744.0;  // 1.5 * 2^52: what is added to it loses its fraction
  const double p = (double)position, g = (double)f, angle = p * g, rest = fma(p, g, -angle);
  const double t = fma(angle, PER, ROUND), n = t - ROUND;
  const int quarter = __double2loint(t);  // (the low bits of n)
  const double r = fma(-n, HI, angle) + fma(-n, LO, rest), r2 = r * r;
  double s = 1.0 / 355687428096000.0, c = 1.0 / 20922789888000.0;
  s = fma(s, r2, -1.0 / 1307674368000.0);
  s = fma(s, r2, 1.0 / 6227020800.0);
  s = fma(s, r2, -1.0 / 39916800.0);
  s = fma(s, r2, 1.0 / 362880.0);
  s = fma(s, r2, -1.0 / 5040.0);
  s = fma(s, r2, 1.0 / 120.0);
  s = fma(s, r2, -1.0 / 6.0);
  s = fma(s * r2, r, r);
  c = fma(c, r2, -1.0 / 87178291200.0);
  c = fma(c, r2, 1.0 / 479001600.0);
  c = fma(c, r2, -1.0 / 3628800.0);
  c = fma(c, r2, 1.0 / 40320.0);
  c = fma(c, r2, -1.0 / 720.0);
  c = fma(c, r2, 1.0 / 24.0);
  c = fma(c, r2, -0.5);
  c = fma(c, r2, 1.0);
  const double a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;
  return {(quarter + 1) & 2 ? -a : a, quarter & 2 ? -b : b};
}
#endif

int launch_rope(const dma_shape& s, const void* Q, long q_stride, const void* K, long k_stride, const int32_t* cu,
                const int32_t* positions, const RopeArgs& rope, bool next, bool inverse, void* Qo, long qo_stride, void* Ko,
                long ko_stride, hipStream_t st);
int launch_cache_append_rope(const dma_cache_shape& s, int n_rows, const void* Q, long q_stride, const void* K, long k_stride,
                             const void* V, long v_stride, const float* W, const float* A, const float* z, const int32_t* slots,
                             const int32_t* row_req, const int32_t* row_len, int n_prefixes, const int32_t* prefix_len,
                             const int32_t* req_prefix, const RopeArgs& rope, bool next, void* Qo, void* pages, hipStream_t st);

}  // namespace dma
