// Decode over the paged 4-bit cache (cache.h): for each new row the min(k, n) best of its request's first n tokens by (score
// descending, position ascending) (Eq. 4), and attention over them (Eq. 5-6).
#include "cache.h"
#include "select.h"

namespace dma {

struct CacheRows {
  const int32_t *table, *row_req, *row_len;
  int n_rows, k, kcap;
};

// What a row sees: its request and the number of keys (0: no row).
struct CacheRow {
  const int32_t* pages;
  int n;
};
__device__ __forceinline__ CacheRow cache_row(const CacheRef& c, const CacheRows& p, int r) {
  const int b = p.row_req ? p.row_req[r] : r;
  if (b < 0 || b >= c.n_reqs) return {p.table, 0};
  const long long cap = (long long)c.max_pages << c.shift;
  return {p.table + (size_t)b * c.max_pages, (int)max(0ll, min((long long)p.row_len[r], cap))};
}

// Slot and score of position j (a page number out of range: no slot, and a score behind all others).
__device__ __forceinline__ uint32_t cache_slot(const CacheRef& c, const CacheRow& row, int j) {
  const uint32_t page = (uint32_t)row.pages[j >> c.shift];
  return page < (uint32_t)c.n_pages ? page << c.shift | ((uint32_t)j & ((1u << c.shift) - 1u)) : 0xffffffffu;
}
__device__ __forceinline__ float cache_score(const CacheRef& c, uint32_t slot, int h) {
  if (slot >= c.n_slots) return -INFINITY;
  return reinterpret_cast<const float*>(cache_page(c, slot) + c.off_z)[((size_t)h << c.shift) + cache_place(c, slot)];
}

// ------------------------------------------------------------------ the kept set
// One workgroup per (row, head): the threshold digit by digit, then the list in order of position.
__global__ __launch_bounds__(1024) void cache_select_kernel(CacheRef c, CacheRows p, int32_t* kept) {
  const int rh = blockIdx.x, r = rh / c.H_q, h = rh - r * c.H_q;
  const int tid = threadIdx.x, w = tid >> 6, l = tid & 63;
  const CacheRow row = cache_row(c, p, r);
  const int n = row.n, kk = min(p.k, n);
  int32_t* list = kept + (size_t)rh * p.kcap;
  for (int i = kk + tid; i < p.kcap; i += 1024) list[i] = -1;
  if (kk == n) {
    for (int j = tid; j < n; j += 1024) list[j] = (int32_t)cache_slot(c, row, j);
    return;
  }
  __shared__ uint32_t hist[256], s_prefix, s_left, wsum[16][2];
  uint32_t prefix = 0, left = (uint32_t)kk;
  for (int pass = 3; pass >= 0; pass--) {
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
    for (int j = tid; j < n; j += 1024) {
      const uint32_t key = desc_key(cache_score(c, cache_slot(c, row, j), h));
      if (pass == 3 || key >> (8 * pass + 8) == prefix) atomicAdd(&hist[(key >> (8 * pass)) & 255u], 1u);
    }
    __syncthreads();
    if (tid == 0) {
      uint32_t digit = 0, run = 0;
      while (run + hist[digit] < left) run += hist[digit++];
      s_prefix = prefix << 8 | digit;
      s_left = left - run;
    }
    __syncthreads();
    prefix = s_prefix;
    left = s_left;
  }
  // keys before the threshold, and the first `left` of those equal to it
  const int per = (n + 16 * 64 - 1) / (16 * 64) * 64, j0 = w * per, j1 = min(n, j0 + per);
  uint32_t better = 0, equal = 0;
  for (int jb = j0; jb < j1; jb += 64) {
    const int j = jb + l;
    const uint32_t key = j < j1 ? desc_key(cache_score(c, cache_slot(c, row, j), h)) : 0xffffffffu;
    better += (uint32_t)__popcll(__ballot(j < j1 && key < prefix));
    equal += (uint32_t)__popcll(__ballot(j < j1 && key == prefix));
  }
  if (l == 0) {
    wsum[w][0] = better;
    wsum[w][1] = equal;
  }
  __syncthreads();
  better = equal = 0;
  for (int i = 0; i < w; i++) {
    better += wsum[i][0];
    equal += wsum[i][1];
  }
  const unsigned long long before = (1ull << l) - 1ull;
  for (int jb = j0; jb < j1; jb += 64) {
    const int j = jb + l;
    const uint32_t slot = j < j1 ? cache_slot(c, row, j) : 0xffffffffu;
    const uint32_t key = j < j1 ? desc_key(cache_score(c, slot, h)) : 0xffffffffu;
    const bool b = j < j1 && key < prefix, e = j < j1 && key == prefix;
    const unsigned long long bm = __ballot(b), em = __ballot(e);
    const uint32_t eq = equal + (uint32_t)__popcll(em & before);
    const uint32_t at = better + (uint32_t)__popcll(bm & before) + min(eq, left);
    if (b || (e && eq < left)) list[at] = (int32_t)slot;
    better += (uint32_t)__popcll(bm);
    equal += (uint32_t)__popcll(em);
  }
}

// ------------------------------------------------------------------ attention over a part of the list
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

// One workgroup per (CH kept keys, row, head).  A key's K (and V) row is held by D / 32 lanes, 32 channels with one scale each; a
// wave takes 64 keys at a time, all of them requested before the first is used, and has one running maximum.  The G heads
// of a kv-head have the same part of their lists on one XCD at the same time (decode_attend_kernel).
template <typename TQ, int D, int CH>
__global__ __launch_bounds__(256) void cache_attend_kernel(CacheRef c, CacheRows p, const TQ* __restrict__ q, long q_stride,
                                                           const int32_t* __restrict__ kept, float* __restrict__ part,
                                                           TQ* __restrict__ o, float* __restrict__ lse, int nsplit, float scale) {
  constexpr int LPG = D / 32, NG = 64 / LPG, U = 64 / NG;
  const unsigned wg = blockIdx.x;
  const int G = c.H_q / c.H_kv, idx = (int)(wg >> 3), unit = (idx / G) * 8 + (int)(wg & 7);
  const int rows_g = p.n_rows * c.H_kv, sp = unit / rows_g, rg = unit - sp * rows_g;
  if (sp >= nsplit) return;
  const int r = rg / c.H_kv, g = rg - r * c.H_kv, h = g * G + idx % G, rh = r * c.H_q + h;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), l = tid & 63, sub = l % LPG, grp = l / LPG;
  const int kk = min(p.k, cache_row(c, p, r).n), i0 = sp * CH, cnt = min(CH, kk - i0);
  if (cnt <= 0) {
    if (nsplit == 1) {
      if (tid < D) o[(size_t)rh * D + tid] = TQ(0.f);
      if (tid == 0) lse[(size_t)h * p.n_rows + r] = -INFINITY;
    }
    return;
  }
  __shared__ uint32_t ids[CH];
  __shared__ float zs[CH];  // scores; -inf: the key takes no part
  const int32_t* list = kept + (size_t)rh * p.kcap + i0;
#pragma unroll
  for (int i = tid; i < CH; i += 256) {
    const uint32_t slot = i < cnt ? (uint32_t)list[i] : 0xffffffffu;
    ids[i] = slot < c.n_slots ? slot : 0u;
    zs[i] = cache_score(c, slot, h);
  }
  Query<TQ> qv;
  qv.load(q + (size_t)r * q_stride + (size_t)h * D + 32 * sub);
  float m = -INFINITY, lsum = 0.f, acc[32];
#pragma unroll
  for (int e = 0; e < 32; e++) acc[e] = 0.f;
  __syncthreads();
#pragma unroll 1
  for (int base = w * 64; base < cnt; base += 256) {
    uint4 kr[U], vr[U];
    uint32_t kb[U], vb[U];
    float s2[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
      const uint32_t slot = ids[base + u * NG + grp];
      const char* page = cache_page(c, slot);
      const uint32_t at = ((uint32_t)g << c.shift) + cache_place(c, slot);
      const uint4* codes = reinterpret_cast<const uint4*>(page + (size_t)at * D);
      const uint8_t* scales = reinterpret_cast<const uint8_t*>(page) + c.off_scales + (size_t)at * (D / 16);
      kr[u] = codes[sub];
      vr[u] = codes[LPG + sub];
      kb[u] = scales[sub];
      vb[u] = scales[LPG + sub];
    }
    float top = m;
#pragma unroll
    for (int u = 0; u < U; u++) {
      const float sc = mx_scale(kb[u]), zb = zs[base + u * NG + grp];
      float s = qv.template dot8<0>(kr[u].x, sc, 0.f);
      s = qv.template dot8<1>(kr[u].y, sc, s);
      s = qv.template dot8<2>(kr[u].z, sc, s);
      s = lanes_sum<LPG>(qv.template dot8<3>(kr[u].w, sc, s));
      s2[u] = zb == -INFINITY ? -INFINITY : fmaf(s, scale, zb);  // (whatever such a key holds)
      top = fmaxf(top, s2[u]);
    }
    top = over_groups<LPG>(top, [](float a, float b) { return fmaxf(a, b); });
    const float ref = top == -INFINITY ? 0.f : top, alpha = weight(m, ref);
    m = top;
    lsum *= alpha;
#pragma unroll
    for (int e = 0; e < 32; e++) acc[e] *= alpha;
#pragma unroll
    for (int u = 0; u < U; u++) {
      const float pv = weight(s2[u], ref), sc = s2[u] == -INFINITY ? 0.f : mx_scale(vb[u]);
      lsum += pv;
      const uint32_t code[4] = {vr[u].x, vr[u].y, vr[u].z, vr[u].w};
#pragma unroll
      for (int i = 0; i < 4; i++) {
        static_for<4>([&](auto b) {
          constexpr int B = decltype(b)::value;
          const auto v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[i], sc, B);
          acc[8 * i + 2 * B] = fmaf(pv, v[0], acc[8 * i + 2 * B]);
          acc[8 * i + 2 * B + 1] = fmaf(pv, v[1], acc[8 * i + 2 * B + 1]);
        });
      }
    }
  }
  const auto add = [](float a, float b) { return a + b; };
  lsum = over_groups<LPG>(lsum, add);
#pragma unroll
  for (int e = 0; e < 32; e++) acc[e] = over_groups<LPG>(acc[e], add);
  __shared__ __align__(16) float mo[4][D];
  __shared__ float ml[4][2];
  if (grp == 0) {
#pragma unroll
    for (int e = 0; e < 32; e += 4)
      *reinterpret_cast<float4*>(&mo[w][32 * sub + e]) = make_float4(acc[e], acc[e + 1], acc[e + 2], acc[e + 3]);
  }
  if (l == 0) {
    ml[w][0] = m;
    ml[w][1] = lsum;
  }
  __syncthreads();
  if (tid < D) {
    const float M = fmaxf(fmaxf(ml[0][0], ml[1][0]), fmaxf(ml[2][0], ml[3][0])), ref = M == -INFINITY ? 0.f : M;
    float num = 0.f, den = 0.f;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const float w8 = weight(ml[i][0], ref);
      num = fmaf(mo[i][tid], w8, num);
      den = fmaf(ml[i][1], w8, den);
    }
    if (nsplit == 1) {
      o[(size_t)rh * D + tid] = TQ(den == 0.f ? 0.f : num / den);
      if (tid == 0) lse[(size_t)h * p.n_rows + r] = den == 0.f ? -INFINITY : fmaf(__builtin_amdgcn_logf(den), LN2, M);
    } else {
      float* out = part + ((size_t)rh * nsplit + sp) * (D + 2);
      out[tid] = num;
      if (tid == 0) {
        out[D] = M;
        out[D + 1] = den;
      }
    }
  }
}

// The parts of one (row, head) together: o = sum_s o_s e^(M_s - M) / sum_s l_s e^(M_s - M), eight parts requested at a time.
template <typename TQ, int D>
__global__ __launch_bounds__(D) void cache_merge_kernel(CacheRef c, CacheRows p, const float* __restrict__ part,
                                                        TQ* __restrict__ o, float* __restrict__ lse, int nsplit, int ch) {
  const int rh = blockIdx.x, r = rh / c.H_q, h = rh - r * c.H_q, t = threadIdx.x;
  const int kk = min(p.k, cache_row(c, p, r).n), ns = (kk + ch - 1) / ch;
  const float* ps = part + (size_t)rh * nsplit * (D + 2);
  float M = -INFINITY, num = 0.f, den = 0.f;
  for (int s0 = 0; s0 < ns; s0 += 8) {
    float Ms[8], ls[8], os[8];
#pragma unroll
    for (int u = 0; u < 8; u++) {
      const float* x = ps + (size_t)min(s0 + u, ns - 1) * (D + 2);
      Ms[u] = x[D];
      ls[u] = x[D + 1];
      os[u] = x[t];
    }
    float top = M;
#pragma unroll
    for (int u = 0; u < 8; u++) top = fmaxf(top, Ms[u]);
    const float ref = top == -INFINITY ? 0.f : top, alpha = weight(M, ref);
    M = top;
    num *= alpha;
    den *= alpha;
#pragma unroll
    for (int u = 0; u < 8; u++) {
      if (s0 + u >= ns) continue;  // (past the end the last part was read again)
      const float w8 = weight(Ms[u], ref);
      num = fmaf(os[u], w8, num);
      den = fmaf(ls[u], w8, den);
    }
  }
  o[(size_t)rh * D + t] = TQ(den == 0.f ? 0.f : num / den);  // (no key took part: zeros, -infinity)
  if (t == 0) lse[(size_t)h * p.n_rows + r] = den == 0.f ? -INFINITY : fmaf(__builtin_amdgcn_logf(den), LN2, M);
}

// Kept keys per workgroup of the attention.
static int attend_chunk(const dma_cache_shape& s, int n_rows, int kcap) {
  return (long)n_rows * s.H_q * ((kcap + 511) / 512) >= 4 * CUS ? 512 : 256;
}

static int list_length(const dma_cache_shape& s, int k) {
  const long cap = (long)s.max_pages * s.page_size;
  return (int)(k < cap ? k : cap);
}

size_t cache_decode_bytes(const dma_cache_shape& s, int n_rows, int k) {
  const int kcap = list_length(s, k), ch = attend_chunk(s, n_rows, kcap), nsplit = (kcap + ch - 1) / ch;
  return align_up((size_t)n_rows * s.H_q * nsplit * (s.d + 2) * 4, 256);
}

template <typename TQ, int D>
static void decode_t(const dma_cache_shape& s, const CacheRef& c, const CacheRows& p, float scale, const void* q, long q_stride,
                     void* o, float* lse, const int32_t* kept, float* part, hipStream_t st) {
  const int ch = attend_chunk(s, p.n_rows, p.kcap), nsplit = (p.kcap + ch - 1) / ch;
  const long units = ((long)p.n_rows * s.H_kv * nsplit + 7) / 8 * 8;
  const unsigned grid = (unsigned)(units * (s.H_q / s.H_kv));
  if (ch == 512)
    cache_attend_kernel<TQ, D, 512><<<grid, 256, 0, st>>>(c, p, (const TQ*)q, q_stride, kept, part, (TQ*)o, lse, nsplit, scale);
  else
    cache_attend_kernel<TQ, D, 256><<<grid, 256, 0, st>>>(c, p, (const TQ*)q, q_stride, kept, part, (TQ*)o, lse, nsplit, scale);
  if (nsplit > 1)
    cache_merge_kernel<TQ, D><<<(unsigned)(p.n_rows * s.H_q), D, 0, st>>>(c, p, part, (TQ*)o, lse, nsplit, ch);
}

int launch_cache_decode(const dma_cache_shape& s, int n_rows, int k, float scale, const void* q, long q_stride,
                        const void* pages, const int32_t* table, const int32_t* row_req, const int32_t* row_len, void* o,
                        float* lse, int32_t* kept, void* ws, hipStream_t st) {
  const CacheRef c = cache_ref(s, pages);
  const CacheRows p = {table, row_req, row_len, n_rows, k, list_length(s, k)};
  cache_select_kernel<<<(unsigned)(n_rows * s.H_q), 1024, 0, st>>>(c, p, kept);
  if (hipGetLastError() != hipSuccess) return DMA_EHIP;
  auto go = [&](auto t) {
    using T = std::remove_pointer_t<decltype(t)>;
    if (s.d == 256) decode_t<T, 256>(s, c, p, scale, q, q_stride, o, lse, kept, (float*)ws, st);
    else if (s.d == 128) decode_t<T, 128>(s, c, p, scale, q, q_stride, o, lse, kept, (float*)ws, st);
    else decode_t<T, 64>(s, c, p, scale, q, q_stride, o, lse, kept, (float*)ws, st);
  };
  if (s.dtype == DMA_BF16) go((__bf16*)nullptr); else go((float*)nullptr);
  return hipGetLastError() == hipSuccess ? DMA_OK : DMA_EHIP;
}

}  // namespace dma
