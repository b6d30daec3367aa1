// Rotary positions of packed Q and K, and the rotation back that carries gradients: y1 = x1 cos a - x2 sin a,
// y2 = x1 sin a + x2 cos a for every pair of channels, a = position * frequency.  The transpose is the rotation by -a.
#include "cache_rows.h"
#include "rope.h"

namespace dma {

struct RopeRows {
  const void *q, *k;
  void *qo, *ko;
  long q_stride, k_stride, qo_stride, ko_stride;
  const int32_t *cu, *positions;
  int T, n_docs, H_q, H;  // q-heads, and all heads (either kind may be left out)
  int first;              // token of this launch
};

// The last document that starts at or before t: 64 of the starts at a time, a lane each.
__device__ __forceinline__ int document_start(const int32_t* __restrict__ cu, int n_docs, int t, int l) {
  int lo = 0, n = n_docs;  // it is one of the n from lo on
  while (n > 1) {
    const int step = (n + 63) / 64;
    const int i = min(l * step, n - 1);
    const unsigned long long m = __ballot(cu[lo + i] <= t);  // (ascending: the lanes before one that is behind t)
    const int last = max(0, __popcll(m) - 1);
    const int at = min(last * step, n - 1);
    n = min(step, n - at);
    lo += at;
  }
  return cu[lo];
}

// A wave has a token: a lane 16 channels, eight whole pairs (or channels that stay), of every 64 / (D / 16)-th head, so that a load of the wave
// covers whole heads in a row.  The lanes of one place in the heads share their eight angles: each forms 8 / heads of them (or, with
// more than eight heads at a time, one that others form too), and takes the rest from the others.
// What bounds it is memory: every value is read and written once.  16384 tokens of 40 heads of 128 in bf16 64 us (5.3 TB/s; a copy of 4 GiB
// reaches 4.75, here a part of what was written is still in the last cache), 65536 of 32 heads of 64 99 (5.4), 5003 of 20 heads of 256
// in fp32 50 (4.1: a start of some microseconds), one token 3.0.  With eight tokens to a wave, each lane in its place of every head, loads
// were in pieces of 32 bytes, and each lane formed eight angles: 84, 118 and 58 us.  A loop over tokens took 168 registers instead of 92 (106
// instead of 99 us).
template <typename T, int D, bool NEXT>
__global__ __launch_bounds__(256) void rope_kernel(RopeRows p, RopeArgs rope, int heads, int inverse) {
  constexpr int TASKS = D / 16, HEADS = 64 / TASKS, OWN = HEADS < 8 ? 8 / HEADS : 1, U = 5;
  const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), task = l % TASKS, hs = l / TASKS;
  const int h0 = blockIdx.y * heads, h1 = min(p.H, h0 + heads);
  const bool turned = task < rope.rot / 16;
  const int a = NEXT ? 16 * task : turned ? 8 * task : rope.rot + 16 * (task - rope.rot / 16);
  const int b = !NEXT && turned ? a + rope.rot / 2 : a + 8;
  float f[OWN];
#pragma unroll
  for (int e = 0; e < OWN; e++) f[e] = turned ? rope.freqs[8 * task + (OWN * hs + e) % 8] : 0.f;
  const long t = (long)p.first + (long)blockIdx.x * 4 + w;
  if (t >= p.T) return;
  const int position = p.positions ? p.positions[t] : (int)t - document_start(p.cu, p.n_docs, (int)t, l);
  Raw8<T> x[U], y[U];
  auto load = [&](int hb) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int h = min(hb + u * HEADS + hs, h1 - 1);
      const T* src = h < p.H_q ? (const T*)p.q + t * p.q_stride + (long)h * D : (const T*)p.k + t * p.k_stride + (long)(h - p.H_q) * D;
      load_raw(src + a, x[u]);
      load_raw(src + b, y[u]);
    }
  };
  load(h0);  // (on their way under the angles)
  float c[8], s[8];
  {
    Turn turn[OWN];
#pragma unroll
    for (int e = 0; e < OWN; e++) turn[e] = turn_of(position, f[e]);
#pragma unroll
    for (int e = 0; e < 8; e++) {
      const int lane = ((e / OWN) * TASKS + task) * 4;
      c[e] = __int_as_float(__builtin_amdgcn_ds_bpermute(lane, __float_as_int((float)turn[e % OWN].c)));
      s[e] = __int_as_float(__builtin_amdgcn_ds_bpermute(lane, __float_as_int((float)turn[e % OWN].s)));
      s[e] = inverse ? -s[e] : s[e];
    }
  }
  for (int hb = h0; hb < h1; hb += U * HEADS) {
    if (hb != h0) load(hb);
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int h = hb + u * HEADS + hs;
      if (h >= h1) continue;
      T* dst = h < p.H_q ? (T*)p.qo + t * p.qo_stride + (long)h * D : (T*)p.ko + t * p.ko_stride + (long)(h - p.H_q) * D;
      if (turned) {
        float v[16], o[16];
        to_f32(x[u], v);
        to_f32(y[u], v + 8);
#pragma unroll
        for (int e = 0; e < 8; e++) {
          const int i = NEXT ? 2 * e : e, j = NEXT ? 2 * e + 1 : e + 8;
          o[i] = fmaf(v[i], c[e], -(v[j] * s[e]));
          o[j] = fmaf(v[i], s[e], v[j] * c[e]);
        }
        store8<T>(dst + a, o);
        store8<T>(dst + b, o + 8);
      } else {
        store_raw(dst + a, x[u]);
        store_raw(dst + b, y[u]);
      }
    }
  }
}

// (2^22 tokens to a launch: it has fewer than 2^32 threads)
template <typename T, int D>
static void rope_t(RopeRows p, const RopeArgs& rope, bool next, bool inverse, hipStream_t st) {
  constexpr int HEADS = 64 / (D / 16), MOST = 1 << 22;
  for (;;) {
    const int tokens = p.T - p.first < MOST ? p.T - p.first : MOST;
    const long tiles = (tokens + 3) / 4;
    int heads = (int)((tiles * p.H + 4 * CUS - 1) / (4 * CUS));  // of a workgroup: fewer where there are few tokens, whole rounds of a wave
    heads = (heads + HEADS - 1) / HEADS * HEADS;
    heads = heads > p.H ? p.H : heads;
    const dim3 grid((unsigned)tiles, (unsigned)((p.H + heads - 1) / heads));
    if (next) rope_kernel<T, D, true><<<grid, 256, 0, st>>>(p, rope, heads, inverse);
    else rope_kernel<T, D, false><<<grid, 256, 0, st>>>(p, rope, heads, inverse);
    if (p.T - p.first <= MOST) return;
    p.first += MOST;
  }
}

int launch_rope(const dma_shape& s, const void* Q, long q_stride, const void* K, long k_stride, const int32_t* cu,
                const int32_t* positions, const RopeArgs& rope, bool next, bool inverse, void* Qo, long qo_stride, void* Ko,
                long ko_stride, hipStream_t st) {
  const int H_q = Q ? s.H_q : 0;
  const RopeRows p = {Q, K, Qo, Ko, q_stride, k_stride, qo_stride, ko_stride, cu, positions, s.T, s.n_docs, H_q, H_q + (K ? s.H_kv : 0), 0};
  auto go = [&](auto t) {
    using T = std::remove_pointer_t<decltype(t)>;
    if (s.d == 256) rope_t<T, 256>(p, rope, next, inverse, st);
    else if (s.d == 128) rope_t<T, 128>(p, rope, next, inverse, st);
    else rope_t<T, 64>(p, rope, next, inverse, st);
  };
  if (s.dtype == DMA_BF16) go((__bf16*)nullptr); else go((float*)nullptr);
  return hipGetLastError() == hipSuccess ? DMA_OK : DMA_EHIP;
}

}  // namespace dma
