// Decode over the paged 4-bit cache for requests that share prefixes: a row's keys are those of its prefix, then its request's own, and it
// keeps the min(k, n) best of all of them by (score descending, position ascending).
//
// The min(k, P) best of a prefix are listed once for each of its heads, the min(k, m) best of a row's own keys for each row.  What a row
// keeps are the k best of the two lists together: a cut through each of them.
#include "cache_attend.h"
#include "cache_select.h"

namespace dma {

struct PrefixRows {
  CacheRows own, pre;  // the rows, and the prefixes as rows of their requests
  const int32_t* req_prefix;
  const int32_t *list_own, *list_pre;  // [rows or prefixes][H_q][kcap]
};

// What a row sees: its own keys (0: no row) and those of its prefix.
struct PrefixRow {
  int own, pre, prefix;
};
__device__ __forceinline__ PrefixRow prefix_row(const CacheRef& c, const PrefixRows& p, int r) {
  PrefixRow row = {cache_row(c, p.own, r).n, 0, 0};
  const int req = p.own.row_req ? p.own.row_req[r] : r;
  const int prefix = row.own > 0 && p.pre.n_rows ? p.req_prefix[req] : -1;  // (own > 0: the request is in range)
  if ((uint32_t)prefix < (uint32_t)p.pre.n_rows) {
    row.prefix = prefix;
    row.pre = cache_row(c, p.pre, prefix).n;
  }
  return row;
}

// The last key that a row keeps of either list: those before it in (key, place in the list) order, and itself.
struct Cut {
  uint32_t key;
  int pre, own;  // of the keys equal to it, those up to this place of the list (-1: none)
};

// One workgroup per (row, head): digit by digit, the key at which the lists' common count reaches k; among equal keys the prefix's are first.
__global__ __launch_bounds__(256) void prefix_cut_kernel(CacheRef c, PrefixRows p, Cut* __restrict__ cuts) {
  __shared__ uint32_t hist[256];
  __shared__ uint32_t st[2];
  __shared__ uint32_t wsum[4];
  const int rh = blockIdx.x, r = rh / c.H_q, h = rh - r * c.H_q, tid = threadIdx.x, l = tid & 63, w = tid >> 6;
  const PrefixRow row = prefix_row(c, p, r);
  const int k = p.own.k, n_pre = min(k, row.pre), n_own = min(k, row.own);
  const int32_t* own = p.list_own + (size_t)rh * p.own.kcap;
  const int32_t* pre = p.list_pre + ((size_t)row.prefix * c.H_q + h) * p.own.kcap;
  auto key = [&](const int32_t* list, int i) { return score_key(cache_score(c, (uint32_t)list[i], h)); };
  Cut cut = {NO_KEY, -1, -1};
  if ((long)n_pre + n_own > k) {
    uint32_t prefix = 0, need = (uint32_t)k;
    for (int shift = 24; shift >= 0; shift -= 8) {
      hist[tid] = 0;
      __syncthreads();
      const auto count = [&](uint32_t x) {
        if (shift == 24 || x >> (shift + 8) == prefix) atomicAdd(&hist[x >> shift & 255u], 1u);
      };
      for (int i = tid; i < n_pre; i += 256) count(key(pre, i));
      for (int i = tid; i < n_own; i += 256) count(key(own, i));
      __syncthreads();
      if (tid == 0) {
        uint32_t run = 0, d = 0;
        while (run + hist[d] < need) run += hist[d++];
        st[0] = d;
        st[1] = need - run;
      }
      __syncthreads();
      prefix = prefix << 8 | st[0];
      need = st[1];
      __syncthreads();
    }
    cut.key = prefix;
    // the place of the need-th key equal to it, through the prefix's list and then the row's own
    uint32_t seen = 0;
    auto walk = [&](const int32_t* list, int n) {
      int last = -1;
      for (int i0 = 0; i0 < n && seen < need; i0 += 256) {
        const bool eq = i0 + tid < n && key(list, i0 + tid) == cut.key;
        const unsigned long long m = __ballot(eq);
        if (l == 0) wsum[w] = (uint32_t)__popcll(m);
        __syncthreads();
        uint32_t at = seen;
        for (int i = 0; i < w; i++) at += wsum[i];
        at += lanes_before(m);
        if (eq && at + 1 <= need) last = i0 + tid;
        seen += wsum[0] + wsum[1] + wsum[2] + wsum[3];
        __syncthreads();
      }
      const int best = (int)last_lane(wave_scan((uint32_t)(last + 1), 0u, [](uint32_t a, uint32_t b) { return max(a, b); }));
      if (l == 0) wsum[w] = (uint32_t)best;
      __syncthreads();
      const int all = (int)max(max(wsum[0], wsum[1]), max(wsum[2], wsum[3])) - 1;
      __syncthreads();
      return all;
    };
    cut.pre = walk(pre, n_pre);
    cut.own = walk(own, n_own);
  }
  if (tid == 0) cuts[rh] = cut;
}

// One workgroup per (row, head), over both lists; the form of cache_attend_kernel.
template <typename TQ, int D>
__global__ __launch_bounds__(256) void prefix_attend_kernel(CacheRef c, PrefixRows p, const Cut* __restrict__ cuts,
                                                            const TQ* __restrict__ q, long q_stride, TQ* __restrict__ o,
                                                            float* __restrict__ lse, float scale) {
  constexpr int LPG = D / 32, NG = 64 / LPG;
  const int rh = blockIdx.x, r = rh / c.H_q, h = rh - r * c.H_q, g = h / (c.H_q / c.H_kv);
  const int tid = threadIdx.x, w = tid >> 6, l = tid & 63, sub = l % LPG, grp = l / LPG;
  const PrefixRow row = prefix_row(c, p, r);
  const int k = p.own.k, n_pre = min(k, row.pre), n_own = min(k, row.own);
  const int32_t* own = p.list_own + (size_t)rh * p.own.kcap;
  const int32_t* pre = p.list_pre + ((size_t)row.prefix * c.H_q + h) * p.own.kcap;
  const Cut cut = cuts[rh];
  const bool bad = (n_own > 0 && own[0] < 0) || (n_pre > 0 && pre[0] < 0);  // a page is out of range: the row sees nothing
  Query<TQ> qv;
  qv.load(q + (size_t)r * q_stride + (size_t)h * D + 32 * sub);
  float m = -INFINITY, lsum = 0.f, acc[32];
#pragma unroll
  for (int e = 0; e < 32; e++) acc[e] = 0.f;
  const long n = bad || !n_own ? 0 : (long)n_pre + n_own;
  for (long i0 = (long)w * NG; i0 < n; i0 += 4 * NG) {
    const long i = i0 + grp;
    const bool of_pre = i < n_pre;
    const int at = (int)(of_pre ? i : i - n_pre);
    const uint32_t id = i < n ? (uint32_t)(of_pre ? pre : own)[at] : 0xffffffffu;
    const uint32_t slot = id < c.n_slots ? id : 0u, place = cache_place(c, slot);
    const char* page = cache_page(c, slot);
    const size_t at_g = ((size_t)g << c.shift) + place;
    const uint4* codes = reinterpret_cast<const uint4*>(page + at_g * D + 16 * sub);
    const uint8_t* scales = reinterpret_cast<const uint8_t*>(page + c.off_scales + at_g * (D / 16) + sub);
    const uint4 kr = codes[0], vr = codes[LPG];
    const float z = reinterpret_cast<const float*>(page + c.off_z)[((size_t)h << c.shift) + place], ks = mx_scale(scales[0]);
    const uint32_t key = score_key(z);
    const bool there = id < c.n_slots && z != -INFINITY && (key < cut.key || (key == cut.key && at <= (of_pre ? cut.pre : cut.own)));
    float s = qv.template dot8<0>(kr.x, ks, 0.f);
    s = qv.template dot8<1>(kr.y, ks, s);
    s = qv.template dot8<2>(kr.z, ks, s);
    s = lanes_sum<LPG>(qv.template dot8<3>(kr.w, ks, s));
    s = there ? fmaf(s, scale, z) : -INFINITY;
    const float top = fmaxf(m, over_groups<LPG>(s, [](float a, float b) { return fmaxf(a, b); }));
    const float ref = top == -INFINITY ? 0.f : top, alpha = weight(m, ref), pv = weight(s, ref), vs = there ? mx_scale(scales[LPG]) : 0.f;
    m = top;
    lsum = fmaf(lsum, alpha, pv);
    const uint32_t code[4] = {vr.x, vr.y, vr.z, vr.w};
#pragma unroll
    for (int i4 = 0; i4 < 4; i4++) {
      static_for<4>([&](auto b) {
        constexpr int Bp = decltype(b)::value;
        const auto v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[i4], vs, Bp);
        acc[8 * i4 + 2 * Bp] = fmaf(acc[8 * i4 + 2 * Bp], alpha, pv * v[0]);
        acc[8 * i4 + 2 * Bp + 1] = fmaf(acc[8 * i4 + 2 * Bp + 1], alpha, pv * v[1]);
      });
    }
  }
  const auto add = [](float a, float b) { return a + b; };
  lsum = over_groups<LPG>(lsum, add);
  __shared__ float mo[4][D], ml[4][2];
#pragma unroll
  for (int e = 0; e < 32; e++) {
    acc[e] = over_groups<LPG>(acc[e], add);
    if (grp == 0) mo[w][32 * sub + e] = acc[e];
  }
  if (l == 0) {
    ml[w][0] = m;
    ml[w][1] = lsum;
  }
  __syncthreads();
  if (tid >= D) return;
  const float M = fmaxf(fmaxf(ml[0][0], ml[1][0]), fmaxf(ml[2][0], ml[3][0])), mr = M == -INFINITY ? 0.f : M;
  float num = 0.f, den = 0.f;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const float w8 = weight(ml[i][0], mr);
    num = fmaf(mo[i][tid], w8, num);
    den = fmaf(ml[i][1], w8, den);
  }
  o[(size_t)rh * D + tid] = TQ(den == 0.f ? 0.f : num / den);
  if (tid == 0) lse[(size_t)h * p.own.n_rows + r] = den == 0.f ? -INFINITY : fmaf(__builtin_amdgcn_logf(den), LN2, M);
}

struct PrefixWork {
  size_t off_pre, off_own, off_cuts, total;
  SelectWork pre, own;
};
static PrefixWork prefix_work(const dma_cache_shape& s, int n_rows, int k, int n_prefixes, int max_prefix) {
  const int kcap = list_length(s, k);
  const size_t pairs = (size_t)n_rows * s.H_q, pre_pairs = (size_t)n_prefixes * s.H_q;
  PrefixWork wk = {};
  auto take = [&](size_t bytes) { size_t at = wk.total; wk.total = align_up(at + bytes, 256); return at; };
  wk.off_pre = take(pre_pairs * kcap * 4);
  wk.off_own = take(pairs * kcap * 4);
  wk.off_cuts = take(pairs * sizeof(Cut));
  if (n_prefixes) wk.pre = select_work(s, pre_pairs, kcap, max_prefix, wk.total);
  wk.own = select_work(s, pairs, kcap, s.max_len, wk.total);
  return wk;
}

size_t cache_decode_prefix_bytes(const dma_cache_shape& s, int n_rows, int k, int n_prefixes, int max_prefix) {
  return n_rows == 0 ? 0 : prefix_work(s, n_rows, k, n_prefixes, max_prefix).total;
}

int launch_cache_decode_prefix(const dma_cache_shape& s, int n_rows, int k, float scale, const void* q, long q_stride,
                               const void* pages, const int32_t* table, const int32_t* row_req, const int32_t* row_len,
                               int n_prefixes, int max_prefix, const int32_t* prefix_req, const int32_t* prefix_len,
                               const int32_t* req_prefix, void* o, float* lse, void* ws, hipStream_t st) {
  const CacheRef c = cache_ref(s, pages);
  const PrefixWork wk = prefix_work(s, n_rows, k, n_prefixes, max_prefix);
  const int kcap = list_length(s, k);
  char* base = (char*)ws;
  int32_t *list_pre = (int32_t*)(base + wk.off_pre), *list_own = (int32_t*)(base + wk.off_own);
  Cut* cuts = (Cut*)(base + wk.off_cuts);
  const PrefixRows p = {{table, row_req, row_len, n_rows, k, kcap}, {table, prefix_req, prefix_len, n_prefixes, k, kcap}, req_prefix,
                        list_own, list_pre};
  if (n_prefixes) launch_select(s, c, p.pre, wk.pre, ws, list_pre, st);
  launch_select(s, c, p.own, wk.own, ws, list_own, st);
  const unsigned pairs = (unsigned)(n_rows * s.H_q);
  prefix_cut_kernel<<<pairs, 256, 0, st>>>(c, p, cuts);
  if (hipGetLastError() != hipSuccess) return DMA_EHIP;
  auto go = [&](auto t, auto width) {
    using T = std::remove_pointer_t<decltype(t)>;
    constexpr int D = decltype(width)::value;
    prefix_attend_kernel<T, D><<<pairs, 256, 0, st>>>(c, p, cuts, (const T*)q, q_stride, (T*)o, lse, scale);
  };
  auto types = [&](auto width) {
    if (s.dtype == DMA_BF16) go((__bf16*)nullptr, width); else go((float*)nullptr, width);
  };
  if (s.d == 256) types(std::integral_constant<int, 256>{});
  else if (s.d == 128) types(std::integral_constant<int, 128>{});
  else types(std::integral_constant<int, 64>{});
  return hipGetLastError() == hipSuccess ? DMA_OK : DMA_EHIP;
}

}  // namespace dma
