// Decode over the paged 4-bit cache (cache.h): for each new row the min(k, n) best of its request's first n tokens by (score
// descending, position ascending) (Eq. 4), and attention over them (Eq. 5-6).
#include "cache_attend.h"
#include "cache_select.h"

namespace dma {

// ------------------------------------------------------------------ the kept sets
template <int S, bool SLICED, int WAVES>
__global__ __launch_bounds__(512, WAVES) void cache_select_kernel(CacheRef c, CacheRows p, SliceWork sw, int32_t* kept) {
  select_block<S, SLICED, false>(c, p, sw, kept, nullptr, (int)blockIdx.x);
}

template <int S>
__global__ __launch_bounds__(512, 4) void cache_slice_kernel(CacheRef c, CacheRows p, SliceWork sw, int32_t* kept) {
  slice_block<S, false>(c, p, sw, kept, nullptr, (int)blockIdx.x);
}

static void launch_select(const dma_cache_shape& s, const CacheRef& c, const CacheRows& p, const SelectWork& wk, void* ws, int32_t* kept,
                          hipStream_t st) {
  const int pairs = p.n_rows * s.H_q;
  char* base = (char*)ws;
  SliceWork sw = {(uint2*)(base + wk.off_counts), (uint2*)(base + wk.off_listed), (uint4*)(base + wk.off_bounds), wk.room, wk.parts, 0, wk.pairs};
  auto select = [&](auto width) {
    constexpr int S = decltype(width)::value;
    if (wk.parts) {
      for (; sw.first < pairs; sw.first += wk.pairs) {
        sw.pairs = pairs - sw.first < wk.pairs ? pairs - sw.first : wk.pairs;
        cache_select_kernel<S, true, 6><<<(unsigned)(sw.pairs * wk.parts), 512, 0, st>>>(c, p, sw, kept);
        cache_slice_kernel<S><<<(unsigned)(sw.pairs * wk.parts), 512, 0, st>>>(c, p, sw, kept);
      }
    } else if (pairs > 3 * CUS) {
      cache_select_kernel<S, false, 8><<<(unsigned)pairs, 512, 0, st>>>(c, p, sw, kept);
    } else {
      cache_select_kernel<S, false, 6><<<(unsigned)pairs, 512, 0, st>>>(c, p, sw, kept);
    }
  };
  if (s.page_size >= 64) select(std::integral_constant<int, 1>{});
  else if (s.page_size == 32) select(std::integral_constant<int, 2>{});
  else select(std::integral_constant<int, 4>{});
}

// ------------------------------------------------------------------ attention over a part of the list
// One workgroup per (ch kept keys, row, head).  A key's K (and V) row is held by D / 32 lanes, 32 channels with one scale each; a
// wave takes 32 keys at a time, all of them requested before the first is used.  Weights are formed with the reference so far; only
// a score more than 5 above it leads to the wave's maximum and a rescaling (sums in 32 bits hold weights up to e^5 as well as
// up to 1).  The G heads of a kv-head have the same part of their lists on one XCD at the same time (decode_attend_kernel).
// Bound by HBM and the vector unit together: 24 rows of 32 heads, 2048 of 5461 keys each, 36 us: 138 MB from HBM, 3.8 TB/s (a third of
// the scale and score lines for keys that are not kept), and 12.3 M instructions of a wave, 20 us of the four SIMDs.  16 rows of
// 2 x 32 lists of 1024: 22 us; one row of 32 heads 6 us and 3 of the merge.  Further ahead than one step: + 1 and + 3 us (registers); 16 keys
// a step: rows of 256 channels + 1, 256 lists of 2048 + 3; a branch around the last, empty request + 0.8.
// ALL: the window keeps every key that a request can have, so nothing was selected, and the lists are written here.
template <typename TQ, int D, bool ALL>
__global__ __launch_bounds__(256) void cache_attend_kernel(CacheRef c, CacheRows p, const TQ* __restrict__ q, long q_stride,
                                                           int32_t* __restrict__ kept, float* __restrict__ part,
                                                           TQ* __restrict__ o, float* __restrict__ lse, int ch, int nsplit,
                                                           float scale) {
  constexpr int LPG = D / 32, NG = 64 / LPG, KEYS = 32, U = KEYS / NG;
  const unsigned wg = blockIdx.x;
  const int G = c.H_q / c.H_kv, idx = (int)(wg >> 3), unit = (idx / G) * 8 + (int)(wg & 7);
  const int rows_g = p.n_rows * c.H_kv, sp = unit / rows_g, rg = unit - sp * rows_g;
  if (sp >= nsplit) return;
  const int r = rg / c.H_kv, g = rg - r * c.H_kv, h = g * G + idx % G, rh = r * c.H_q + h;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), l = tid & 63, sub = l % LPG, grp = l / LPG;
  int32_t* list = kept + (size_t)rh * p.kcap;
  int i0 = sp * ch + w * KEYS;
  uint32_t id[U];
  if (!ALL) {  // (requested before the number of kept keys is known)
#pragma unroll
    for (int u = 0; u < U; u++) id[u] = (uint32_t)list[min(i0 + u * NG + grp, p.kcap - 1)];
  }
  Query<TQ> qv;
  qv.load(q + (size_t)r * q_stride + (size_t)h * D + 32 * sub);
  const CacheRow row = cache_row(c, p, r);
  const int kk = min(p.k, row.n), end = min(kk, (sp + 1) * ch);
  auto finish = [&](float num, float den, float M) {  // (all threads)
    if (tid >= D) return;
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
  };
  bool bad = false;
  if constexpr (ALL) {
#pragma unroll
    for (int u = 0; u < U; u++) id[u] = cache_slot(c, row, min(i0 + u * NG + grp, p.kcap - 1));
    for (int j = tid; j << c.shift < row.n; j += 256) bad |= (uint32_t)row.pages[j] >= (uint32_t)c.n_pages;
  }
  if (sp * ch >= kk) {
    if (ALL)
      for (int i = sp * ch + tid; i < min(p.kcap, (sp + 1) * ch); i += 256) list[i] = -1;
    if (nsplit == 1) finish(0.f, 0.f, -INFINITY);
    return;
  }
  // byte offsets in a page of this lane's part of the head's first token
  const uint32_t k_off = ((uint32_t)g << c.shift) * D + 16 * sub, z_off = c.off_z + ((uint32_t)h << c.shift) * 4;
  const uint32_t b_off = c.off_scales + ((uint32_t)g << c.shift) * (D / 16) + sub, page_bytes = (uint32_t)c.page_bytes;
  float m = -INFINITY, ref = 0.f, limit = -INFINITY, lsum = 0.f, acc[32];
#pragma unroll
  for (int e = 0; e < 32; e++) acc[e] = 0.f;
  struct Keys {  // of a step, on their way
    uint4 kr[U], vr[U];
    uint32_t kb[U], vb[U];
    float s[U];
    uint32_t there;
  };
  // the keys at i0 (in id), and the ids of those behind them
  auto fetch = [&](Keys& x) {
    x.there = 0;
#pragma unroll
    for (int u = 0; u < U; u++) {
      const bool there = i0 + u * NG + grp < end && id[u] < c.n_slots;
      const uint32_t slot = there ? id[u] : 0u, place = cache_place(c, slot);
      const char* page = c.pages + (unsigned long long)(slot >> c.shift) * page_bytes;
      const uint4* codes = reinterpret_cast<const uint4*>(page + (k_off + place * D));
      const uint8_t* scales = reinterpret_cast<const uint8_t*>(page + (b_off + place * (D / 16)));
      x.kr[u] = codes[0];
      x.vr[u] = codes[LPG];
      x.kb[u] = scales[0];
      x.vb[u] = scales[LPG];
      x.s[u] = *reinterpret_cast<const float*>(page + (z_off + place * 4));
      x.there |= there ? 1u << u : 0u;
    }
    i0 += 4 * KEYS;
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int next = min(i0 + u * NG + grp, p.kcap - 1);
      id[u] = ALL ? cache_slot(c, row, next) : (uint32_t)list[next];
    }
  };
  auto take = [&](Keys& x) {
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < U; u++) {
      const float sc = mx_scale(x.kb[u]), zb = x.there >> u & 1 ? x.s[u] : -INFINITY;
      float s = qv.template dot8<0>(x.kr[u].x, sc, 0.f);
      s = qv.template dot8<1>(x.kr[u].y, sc, s);
      s = qv.template dot8<2>(x.kr[u].z, sc, s);
      s = lanes_sum<LPG>(qv.template dot8<3>(x.kr[u].w, sc, s));
      x.s[u] = zb == -INFINITY ? -INFINITY : fmaf(s, scale, zb);  // (whatever such a key holds)
      top = fmaxf(top, x.s[u]);
    }
    if (__ballot(top > limit)) {
      top = fmaxf(m, over_groups<LPG>(top, [](float a, float b) { return fmaxf(a, b); }));
      const float alpha = weight(m, top);
      m = ref = top;
      limit = top + 5.f;
      lsum *= alpha;
#pragma unroll
      for (int e = 0; e < 32; e++) acc[e] *= alpha;
    }
#pragma unroll
    for (int u = 0; u < U; u++) {
      const float pv = weight(x.s[u], ref), sc = x.s[u] == -INFINITY ? 0.f : mx_scale(x.vb[u]);
      lsum += pv;
      const uint32_t code[4] = {x.vr[u].x, x.vr[u].y, x.vr[u].z, x.vr[u].w};
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
  };
  if (i0 < end) {
    Keys even, odd;  // (one that moves into the other costs a tenth of the instructions)
    fetch(even);
#pragma unroll 1
    for (;;) {
      const bool more = i0 < end;
      fetch(odd);
      take(even);
      if (!more) break;
      const bool again = i0 < end;
      fetch(even);
      take(odd);
      if (!again) break;
    }
  }
  const auto add = [](float a, float b) { return a + b; };
  lsum = over_groups<LPG>(lsum, add);
  const auto across = [](const auto& both) { return __builtin_bit_cast(float, (unsigned)both[0]) + __builtin_bit_cast(float, (unsigned)both[1]); };
  const auto bits = [](float x) { return __builtin_bit_cast(unsigned, x); };
#pragma unroll
  for (int e = 0; e < 16; e++) acc[e] = across(__builtin_amdgcn_permlane32_swap(bits(acc[e]), bits(acc[e + 16]), false, false));
#pragma unroll
  for (int e = 0; e < 8; e++) {  // (from here on each row of 16 lanes has sums of its own: a quarter of the channels)
    acc[e] = across(__builtin_amdgcn_permlane16_swap(bits(acc[e]), bits(acc[e + 8]), false, false));
    if constexpr (LPG == 2) acc[e] += dpp_move<0x4e>(acc[e]);
    if constexpr (LPG <= 4) acc[e] += dpp_move<0x124>(acc[e]);
    acc[e] += dpp_move<0x128>(acc[e]);
  }
  __shared__ __align__(16) float mo[4][D];
  __shared__ float ml[4][2];
  if ((l & 15) < LPG) {
    float4* to = reinterpret_cast<float4*>(&mo[w][32 * sub + 16 * (l >> 5) + 8 * (l >> 4 & 1)]);
    to[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
    to[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
  }
  if (l == 0) {
    ml[w][0] = m;
    ml[w][1] = lsum;
  }
  if (ALL ? __syncthreads_or(bad) : (__syncthreads(), 0)) {  // a page is out of range: the row sees nothing
    for (int i = sp * ch + tid; i < min(p.kcap, (sp + 1) * ch); i += 256) list[i] = -1;
    finish(0.f, 0.f, -INFINITY);
    return;
  }
  if (ALL)
    for (int i = sp * ch + tid; i < min(p.kcap, (sp + 1) * ch); i += 256) list[i] = i < kk ? (int32_t)cache_slot(c, row, i) : -1;
  const float M = fmaxf(fmaxf(ml[0][0], ml[1][0]), fmaxf(ml[2][0], ml[3][0])), mr = M == -INFINITY ? 0.f : M;
  float num = 0.f, den = 0.f;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const float w8 = weight(ml[i][0], mr);
    num = fmaf(mo[i][tid % D], w8, num);
    den = fmaf(ml[i][1], w8, den);
  }
  finish(num, den, M);
}

// The parts of one (row, head) together: o = sum_s o_s e^(M_s - M) / sum_s l_s e^(M_s - M), eight parts requested at a time: 2.8 us,
// a launch and two loads.
template <typename TQ, int D>
__global__ __launch_bounds__(D) void cache_merge_kernel(CacheRef c, CacheRows p, const float* __restrict__ part,
                                                        TQ* __restrict__ o, float* __restrict__ lse, int ch, int nsplit) {
  const int rh = blockIdx.x, r = rh / c.H_q, h = rh - r * c.H_q, t = threadIdx.x;
  const float* ps = part + (size_t)rh * nsplit * (D + 2);
  const int kk = min(p.k, cache_row(c, p, r).n), ns = (kk + ch - 1) / ch;
  float M = -INFINITY, num = 0.f, den = 0.f;
  for (int s0 = 0; s0 == 0 || s0 < ns; s0 += 8) {  // (the first parts are requested before their number is known)
    float Ms[8], ls[8], os[8];
#pragma unroll
    for (int u = 0; u < 8; u++) {
      const float* x = ps + (size_t)min(s0 + u, nsplit - 1) * (D + 2);
      Ms[u] = x[D];
      ls[u] = x[D + 1];
      os[u] = x[t];
    }
    float top = M;
#pragma unroll
    for (int u = 0; u < 8; u++) top = fmaxf(top, s0 + u < ns ? Ms[u] : -INFINITY);
    const float ref = top == -INFINITY ? 0.f : top, alpha = weight(M, ref);
    M = top;
    num *= alpha;
    den *= alpha;
#pragma unroll
    for (int u = 0; u < 8; u++) {
      if (s0 + u >= ns) continue;  // (not written)
      const float w8 = weight(Ms[u], ref);
      num = fmaf(os[u], w8, num);
      den = fmaf(ls[u], w8, den);
    }
  }
  o[(size_t)rh * D + t] = TQ(den == 0.f ? 0.f : num / den);  // (no key took part: zeros, -infinity)
  if (t == 0) lse[(size_t)h * p.n_rows + r] = den == 0.f ? -INFINITY : fmaf(__builtin_amdgcn_logf(den), LN2, M);
}

// Kept keys per workgroup of the attention, a multiple of 256 (two steps of each wave): shorter parts where there are few lists.
constexpr int ATTEND_WGS = CUS;
static int attend_part(const dma_cache_shape& s, int n_rows, int kcap) {
  const long lists = (long)n_rows * s.H_q, most = (kcap + 255) / 256;
  long parts = (ATTEND_WGS + lists - 1) / lists;
  if (parts > most) parts = most;
  return (int)(((kcap + parts - 1) / parts + 255) / 256 * 256);
}

// The workspace: partial outputs, then, where rows can be long, what the parts of a row tell each other.
struct DecodeWork {
  SelectWork select;
  size_t total;
};
static DecodeWork decode_work(const dma_cache_shape& s, int n_rows, int k) {
  const int kcap = list_length(s, k);
  const size_t pairs = (size_t)n_rows * s.H_q;
  DecodeWork wk;
  // (No size is less for more rows.  Partial outputs: fewer than ATTEND_WGS + lists of them, and where there are as many lists, none.)
  const size_t some = pairs < ATTEND_WGS ? pairs : ATTEND_WGS, each = (kcap + 255) / 256, outs = pairs * each < ATTEND_WGS + some ? pairs * each : ATTEND_WGS + some;
  wk.total = each > 1 && s.H_q < ATTEND_WGS ? align_up(outs * (s.d + 2) * 4, 256) : 0;
  wk.select = select_work(s, pairs, kcap, s.max_len, wk.total);
  return wk;
}

size_t cache_decode_bytes(const dma_cache_shape& s, int n_rows, int k) {
  return n_rows == 0 ? 0 : decode_work(s, n_rows, k).total;
}

template <typename TQ, int D>
static void decode_t(const dma_cache_shape& s, const CacheRef& c, const CacheRows& p, float scale, const void* q, long q_stride,
                     void* o, float* lse, int32_t* kept, float* part, bool all, hipStream_t st) {
  const int ch = attend_part(s, p.n_rows, p.kcap), nsplit = (p.kcap + ch - 1) / ch;
  const long units = ((long)p.n_rows * s.H_kv * nsplit + 7) / 8 * 8;
  const unsigned grid = (unsigned)(units * (s.H_q / s.H_kv));
  if (all)
    cache_attend_kernel<TQ, D, true><<<grid, 256, 0, st>>>(c, p, (const TQ*)q, q_stride, kept, part, (TQ*)o, lse, ch, nsplit, scale);
  else
    cache_attend_kernel<TQ, D, false><<<grid, 256, 0, st>>>(c, p, (const TQ*)q, q_stride, kept, part, (TQ*)o, lse, ch, nsplit, scale);
  if (nsplit > 1)
    cache_merge_kernel<TQ, D><<<(unsigned)(p.n_rows * s.H_q), D, 0, st>>>(c, p, part, (TQ*)o, lse, ch, nsplit);
}

int launch_cache_decode(const dma_cache_shape& s, int n_rows, int k, float scale, const void* q, long q_stride,
                        const void* pages, const int32_t* table, const int32_t* row_req, const int32_t* row_len, void* o,
                        float* lse, int32_t* kept, void* ws, hipStream_t st) {
  const CacheRef c = cache_ref(s, pages);
  const CacheRows p = {table, row_req, row_len, n_rows, k, list_length(s, k)};
  const bool all = k >= (long)s.max_pages * s.page_size;
  if (!all) {
    launch_select(s, c, p, decode_work(s, n_rows, k).select, ws, kept, st);
    if (hipGetLastError() != hipSuccess) return DMA_EHIP;
  }
  auto go = [&](auto t) {
    using T = std::remove_pointer_t<decltype(t)>;
    if (s.d == 256) decode_t<T, 256>(s, c, p, scale, q, q_stride, o, lse, kept, (float*)ws, all, st);
    else if (s.d == 128) decode_t<T, 128>(s, c, p, scale, q, q_stride, o, lse, kept, (float*)ws, all, st);
    else decode_t<T, 64>(s, c, p, scale, q, q_stride, o, lse, kept, (float*)ws, all, st);
  };
  if (s.dtype == DMA_BF16) go((__bf16*)nullptr); else go((float*)nullptr);
  return hipGetLastError() == hipSuccess ? DMA_OK : DMA_EHIP;
}

}  // namespace dma
