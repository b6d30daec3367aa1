// Rows into the paged cache with K and q turned to their positions on the way (rope.h): K is held in 4 bits, the codes of the turned
// value itself, without a rounding before them; q leaves in its type.
#include "cache_rows.h"
#include "rope.h"
#include "select.h"

namespace dma {

struct AppendRows {
  const void *q, *k, *v;
  void* qo;
  long q_stride, k_stride, v_stride;
  const float *W, *A, *z;
  const int32_t *slots, *row_req, *row_len, *prefix_len, *req_prefix;
  int n_rows, n_prefixes;
  int first;  // row of this launch
};

// A value of 64 bits in 32: the nearer of its two neighbours with an odd last bit, unless it is a value of 32 bits itself.  What is rounded
// from that to fewer bits is what would come of the value itself: no result of a rounding, nor a border between two, is odd in all of 24 bits.
__device__ __forceinline__ float to_odd(double x) {
  const float f = (float)x;
  const double back = (double)f;
  const uint32_t bits = __float_as_uint(f);
  const uint32_t step = fabs(back) > fabs(x) ? bits - 1u : bits + 1u;
  return __uint_as_float(back == x || x != x || (bits & 1u) ? bits : step);
}

// The codes of a lane's eight values of 64 bits, and their scale byte (scale_byte of cache_rows.h: the exponent is that of the leading word).
__device__ __forceinline__ uint32_t quantise8(const double* x, uint32_t& byte) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; e++) top = max(top, (uint32_t)__double2hiint(x[e]) & 0x7fffffffu);
  top = max(top, dpp_quad<0xb1>(top));
  top = max(top, dpp_quad<0x4e>(top));
  byte = top >= 0x7ff00000u ? 255u : (uint32_t)max(2, min(252, (int)((top + 0x40000u) >> 20) - 898));
  const float scale = mx_scale(byte);
  uint32_t code = 0;
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, to_odd(x[0]), to_odd(x[1]), scale, 0);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, to_odd(x[2]), to_odd(x[3]), scale, 1);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, to_odd(x[4]), to_odd(x[5]), scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, to_odd(x[6]), to_odd(x[7]), scale, 3);
}

// The same eight channels of another lane of the wave.
__device__ __forceinline__ uint32_t from_lane(uint32_t x, int lane) { return (uint32_t)__builtin_amdgcn_ds_bpermute(lane * 4, (int)x); }
__device__ __forceinline__ Raw8<__bf16> from_lane(const Raw8<__bf16>& r, int lane) {
  return {make_uint4(from_lane(r.x.x, lane), from_lane(r.x.y, lane), from_lane(r.x.z, lane), from_lane(r.x.w, lane))};
}
__device__ __forceinline__ float from_lane(float x, int lane) { return __uint_as_float(from_lane(__float_as_uint(x), lane)); }
__device__ __forceinline__ Raw8<float> from_lane(const Raw8<float>& r, int lane) {
  return {make_float4(from_lane(r.a.x, lane), from_lane(r.a.y, lane), from_lane(r.a.z, lane), from_lane(r.a.w, lane)),
          make_float4(from_lane(r.b.x, lane), from_lane(r.b.y, lane), from_lane(r.b.z, lane), from_lane(r.b.w, lane))};
}
__device__ __forceinline__ double from_lane(double x, int lane) {
  return __hiloint2double((int)from_lane((uint32_t)__double2hiint(x), lane), (int)from_lane((uint32_t)__double2loint(x), lane));
}

// A wave has a row: D / 8 lanes a head, eight channels each, 64 / (D / 8) heads at a time, so that a load of the wave covers whole heads in a
// row.  The angles are the same in every head: each lane forms one (two at 256 channels) and takes the others of its pairs from the lanes that
// have them.  Pairs half a rotation apart lie in two lanes, which exchange their values.  Nothing is shared between waves.
// What bounds it is memory: 65536 rows of 32 and 8 heads of 128 318 us (1.44 GB, 4.5 TB/s), one row 4.9 and 333 5.9 (the launch and a
// chain of three loads).  With 64 / (D / 8) rows to a wave, each lane in its place of every head and forming four angles, 350.
// A loop over rows in the kernel took 153 registers instead of 108 (35 us more).
template <typename T, int D, bool NEXT>
__global__ __launch_bounds__(256) void cache_append_rope_kernel(CacheRef c, AppendRows p, RopeArgs rope, int heads) {
  constexpr int LPR = D / 8, HEADS = 64 / LPR, GMAX = 4, PAIRS = NEXT ? 4 : 8, FORMERS = NEXT ? HEADS : 2 * HEADS;
  constexpr int OWN = PAIRS > FORMERS ? PAIRS / FORMERS : 1;
  const int tid = threadIdx.x, l = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), sub = l % LPR, hs = l / LPR;
  const int half = rope.rot / 16;  // lanes of half the turned channels of a head
  const int G = c.H_q / c.H_kv, g0 = blockIdx.y * heads, g1 = min(c.H_kv, g0 + heads);
  const bool turned = sub < 2 * half, first = sub < half;
  const int unit = first || NEXT ? sub : sub - half, other = !NEXT && turned ? (first ? l + half : l - half) : l;
  const long t = (long)p.first + (long)blockIdx.x * 4 + w;
  if (t >= p.n_rows) return;
  const int r = (int)t;
  // the row's place and position
  const uint32_t slot = (uint32_t)p.slots[r];
  char* page = slot < c.n_slots ? cache_page(c, slot) : nullptr;
  const uint32_t place = cache_place(c, slot);
  long position = (long)p.row_len[r] - 1;
  if (p.n_prefixes) {
    const int req = p.row_req ? p.row_req[r] : r;
    const int prefix = (uint32_t)req < (uint32_t)c.n_reqs ? p.req_prefix[req] : -1;
    if ((uint32_t)prefix < (uint32_t)p.n_prefixes) position = max(position, 0l) + max(0l, (long)p.prefix_len[prefix]);
  }
  position = max(0l, min(position, 0x7fffffffl));
  auto load = [&](const void* base, long stride, int h) __attribute__((always_inline)) {
    Raw8<T> x;
    load_raw((const T*)base + (long)r * stride + (long)h * D + 8 * sub, x);
    return x;
  };
  Raw8<T> k = load(p.k, p.k_stride, min(g0 + hs, g1 - 1)), v = load(p.v, p.v_stride, min(g0 + hs, g1 - 1));
  double cs[PAIRS], sn[PAIRS];
  {
    const int former = NEXT || first ? hs : HEADS + hs;
    Turn turn[OWN];
#pragma unroll
    for (int e = 0; e < OWN; e++) turn[e] = turn_of((int)position, turned ? rope.freqs[PAIRS * unit + (OWN * former + e) % PAIRS] : 0.f);
#pragma unroll
    for (int e = 0; e < PAIRS; e++) {
      constexpr int PER = OWN;
      const int from = e / PER, lane = !turned ? l : from < HEADS ? from * LPR + unit : (from - HEADS) * LPR + unit + half;
      cs[e] = from_lane(turn[e % PER].c, lane);
      sn[e] = from_lane(turn[e % PER].s, lane);
      if (!NEXT && !first) sn[e] = -sn[e];  // (the second of a pair: y2 = x2 cos a + x1 sin a)
    }
  }
  for (int gb = g0; gb < g1; gb += HEADS) {
    const int g = min(gb + hs, g1 - 1);
    const bool mine = page && gb + hs < g1;
    if (gb != g0) {
      k = load(p.k, p.k_stride, g);
      v = load(p.v, p.v_stride, g);
    }
    float x[8], y[8];
    double turned_k[8];
    to_f32(k, x);
    if constexpr (NEXT) {
#pragma unroll
      for (int e = 0; e < 4; e++) {
        turned_k[2 * e] = fma((double)x[2 * e], cs[e], -((double)x[2 * e + 1] * sn[e]));
        turned_k[2 * e + 1] = fma((double)x[2 * e], sn[e], (double)x[2 * e + 1] * cs[e]);
      }
    } else {
      to_f32(from_lane(k, other), y);
#pragma unroll
      for (int e = 0; e < 8; e++) turned_k[e] = fma((double)x[e], cs[e], -((double)y[e] * sn[e]));
    }
#pragma unroll
    for (int e = 0; e < 8; e++) turned_k[e] = turned ? turned_k[e] : (double)x[e];
    uint32_t kb, vb;
    const uint32_t kc = quantise8(turned_k, kb), vc = quantise8(v, vb);
    const uint32_t at = ((uint32_t)g << c.shift) + place;
    if (mine) {
      uint32_t* codes = reinterpret_cast<uint32_t*>(page + (at * D + 4 * sub));
      codes[0] = kc;
      codes[LPR] = vc;
      if (sub % 4 == 0) {
        uint8_t* bytes = reinterpret_cast<uint8_t*>(page + (c.off_scales + at * (D / 16) + sub / 4));
        bytes[0] = (uint8_t)kb;
        bytes[D / 32] = (uint8_t)vb;
      }
    }
    auto put_score = [&](int h, float zv) {
      reinterpret_cast<float*>(page + c.off_z)[((uint32_t)h << c.shift) + place] = zv;
    };
    if (!p.W) {
      for (int h = sub; h < G; h += LPR)
        if (mine) put_score(g * G + h, p.z[(size_t)(g * G + h) * p.n_rows + r]);
    } else {  // the scores of z_kernel, bit for bit: the same sums in the same order
      to_f32(v, x);
      for (int h0 = 0; h0 < G; h0 += GMAX) {
        float own = 0.f;
#pragma unroll
        for (int hh = 0; hh < GMAX; hh++) {
          Raw8<float> raw;
          load_raw(p.W + (size_t)(g * G + min(h0 + hh, G - 1)) * D + 8 * sub, raw);
          float wv[8], acc = 0.f;
          to_f32(raw, wv);
#pragma unroll
          for (int e = 0; e < 8; e++) acc = fmaf(wv[e], x[e], acc);
          acc = group_sum<LPR>(acc);
          own = sub == hh ? acc : own;
        }
        if (sub < min(GMAX, G - h0) && mine) {
          const int h = g * G + h0 + sub;
          const float sp = fmaxf(own, 0.f) + log1pf(expf(-fabsf(own)));
          put_score(h, expf(p.A[h] * sp));
        }
      }
    }
  }
  if (!p.q) return;
  float cf[PAIRS], sf[PAIRS];
#pragma unroll
  for (int e = 0; e < PAIRS; e++) {
    cf[e] = (float)cs[e];
    sf[e] = (float)sn[e];
  }
  constexpr int U = sizeof(T) == 4 ? 2 : 4;
  const int h1 = g1 * G;
  for (int hb = g0 * G; hb < h1; hb += U * HEADS) {
    Raw8<T> q[U];
#pragma unroll
    for (int u = 0; u < U; u++) q[u] = load(p.q, p.q_stride, min(hb + u * HEADS + hs, h1 - 1));
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int h = hb + u * HEADS + hs;
      T* dst = (T*)p.qo + ((long)r * c.H_q + h) * D + 8 * sub;
      float x[8], y[8], o[8];
      to_f32(q[u], x);
      if constexpr (NEXT) {
#pragma unroll
        for (int e = 0; e < 4; e++) {
          o[2 * e] = fmaf(x[2 * e], cf[e], -(x[2 * e + 1] * sf[e]));
          o[2 * e + 1] = fmaf(x[2 * e], sf[e], x[2 * e + 1] * cf[e]);
        }
      } else {
        to_f32(from_lane(q[u], other), y);
#pragma unroll
        for (int e = 0; e < 8; e++) o[e] = fmaf(x[e], cf[e], -(y[e] * sf[e]));
      }
      if (h >= h1) continue;
      if (turned) store8<T>(dst, o);
      else store_raw(dst, q[u]);
    }
  }
}

// (2^22 rows to a launch: it has fewer than 2^32 threads)
template <typename T, int D>
static void append_rope_t(const CacheRef& c, AppendRows p, const RopeArgs& rope, bool next, hipStream_t st) {
  constexpr int HEADS = 64 / (D / 8), MOST = 1 << 22;
  for (; p.first < p.n_rows; p.first += MOST) {
    const int rows = p.n_rows - p.first < MOST ? p.n_rows - p.first : MOST, tiles = (rows + 3) / 4;
    long heads = (long)tiles * c.H_kv / (4 * CUS);  // kv-heads of a workgroup: one round of a wave where there are few rows
    heads = (heads + HEADS - 1) / HEADS * HEADS;
    heads = heads < HEADS ? HEADS : heads > c.H_kv ? c.H_kv : heads;
    const dim3 grid((unsigned)tiles, (unsigned)((c.H_kv + heads - 1) / heads));
    if (next) cache_append_rope_kernel<T, D, true><<<grid, 256, 0, st>>>(c, p, rope, (int)heads);
    else cache_append_rope_kernel<T, D, false><<<grid, 256, 0, st>>>(c, p, rope, (int)heads);
  }
}

int launch_cache_append_rope(const dma_cache_shape& s, int n_rows, const void* Q, long q_stride, const void* K, long k_stride,
                             const void* V, long v_stride, const float* W, const float* A, const float* z, const int32_t* slots,
                             const int32_t* row_req, const int32_t* row_len, int n_prefixes, const int32_t* prefix_len,
                             const int32_t* req_prefix, const RopeArgs& rope, bool next, void* Qo, void* pages, hipStream_t st) {
  const CacheRef c = cache_ref(s, pages);
  const AppendRows p = {Q, K, V, Qo, q_stride, k_stride, v_stride, W, A, z, slots, row_req, row_len, prefix_len, req_prefix, n_rows, n_prefixes, 0};
  auto go = [&](auto t) {
    using T = std::remove_pointer_t<decltype(t)>;
    if (s.d == 256) append_rope_t<T, 256>(c, p, rope, next, st);
    else if (s.d == 128) append_rope_t<T, 128>(c, p, rope, next, st);
    else append_rope_t<T, 64>(c, p, rope, next, st);
  };
  if (s.dtype == DMA_BF16) go((__bf16*)nullptr); else go((float*)nullptr);
  return hipGetLastError() == hipSuccess ? DMA_OK : DMA_EHIP;
}

}  // namespace dma
