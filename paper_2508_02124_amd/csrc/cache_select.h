// The kept set of a row of the paged cache: the min(k, n) best of its request's first n tokens by (score descending, position
// ascending) (cache_decode.hip, cache_prefix.hip).  Every source that includes this has kernels of its own.
#pragma once
#include "cache.h"
#include "select.h"

namespace dma {
namespace {

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
  const int len = p.row_len[r], b = p.row_req ? p.row_req[r] : r;  // (requested together)
  const bool there = b >= 0 && b < c.n_reqs;
  const long long cap = (long long)c.max_pages << c.shift;
  return {p.table + (size_t)(there ? b : 0) * c.max_pages, there ? (int)max(0ll, min((long long)len, cap)) : 0};
}

// Slot of position j, and a slot's score (a page number out of range: no slot, and a score behind all others).
__device__ __forceinline__ uint32_t cache_slot(const CacheRef& c, const CacheRow& row, int j) {
  const uint32_t page = (uint32_t)row.pages[j >> c.shift];
  return page < (uint32_t)c.n_pages ? page << c.shift | ((uint32_t)j & ((1u << c.shift) - 1u)) : 0xffffffffu;
}
__device__ __forceinline__ float cache_score(const CacheRef& c, uint32_t slot, int h) {
  if (slot >= c.n_slots) return -INFINITY;
  return reinterpret_cast<const float*>(cache_page(c, slot) + c.off_z)[((size_t)h << c.shift) + cache_place(c, slot)];
}

// ------------------------------------------------------------------ scores of chunks of positions
// A wave reads 64 consecutive positions at a time (a chunk), every NW-th chunk.  The page numbers of its 64 next chunks are one
// load (S = 1: pages of 64 tokens or more, one page a chunk), two (S = 2) or four (S = 4: lane l has the pages of the quarters of the
// l-th); a chunk's page then comes out of a lane into a scalar register, and so does the address.
template <int S> struct PageRun {
  uint32_t pg[S];
  // The pages of the chunks first, first + step, ... of a row (the last entries of the table for those behind its end).
  __device__ __forceinline__ void load(const CacheRef& c, const CacheRow& row, int first, int step, int l) {
#pragma unroll
    for (int q = 0; q < S; q++) pg[q] = (uint32_t)row.pages[min((64 * (first + step * l) + 64 / S * q) >> c.shift, c.max_pages - 1)];
  }
  // Whether one of them, of the row's n positions, is out of range (it is page 0 from here on).
  __device__ __forceinline__ bool check(const CacheRef& c, int n, int first, int step, int l) {
    bool bad = false;
#pragma unroll
    for (int q = 0; q < S; q++) {
      const bool out = pg[q] >= (uint32_t)c.n_pages;
      bad |= out && 64 * (first + step * l) + 64 / S * q < n;
      pg[q] = out ? 0u : pg[q];
    }
    return __ballot(bad) != 0;
  }
  // page of this lane's position in the u-th chunk
  __device__ __forceinline__ uint32_t page(int u, int l) const {
    uint32_t x = (uint32_t)__builtin_amdgcn_readlane((int)pg[0], u);
#pragma unroll
    for (int q = 1; q < S; q++) {
      const uint32_t y = (uint32_t)__builtin_amdgcn_readlane((int)pg[q], u);
      x = l >= 64 / S * q ? y : x;
    }
    return x;
  }
  // The score of this lane's position in it (read also where the row has ended: a place of some page); j: the chunk's first
  // position, scores: those of page 0.
  __device__ __forceinline__ float score(const CacheRef& c, const char* scores, int j, int u, int l) const {
    const uint32_t mask = (1u << c.shift) - 1u;
    const float* z = reinterpret_cast<const float*>(scores + (size_t)page(u, l) * c.page_bytes);
    return S == 1 ? (z + ((uint32_t)j & mask))[l] : z[(uint32_t)l & mask];
  }
  __device__ __forceinline__ int32_t slot(const CacheRef& c, int j, int u, int l) const {
    const uint32_t mask = (1u << c.shift) - 1u, first = page(u, l) << c.shift;
    return (int32_t)(S == 1 ? (first | ((uint32_t)j & mask)) | (uint32_t)l : first | ((uint32_t)l & mask));
  }
};

// Keys ascend from the best score to the worst, -0 and +0 the same, NaN beside one of the infinities; NO_KEY is behind every score's.
constexpr uint32_t BEST_KEY = 0x007fffffu, NO_KEY = 0xffffffffu;
__device__ __forceinline__ uint32_t score_key(float z) { return max(BEST_KEY, min(desc_key(z), NO_KEY - 1)); }
__device__ __forceinline__ uint32_t lanes_before(unsigned long long m) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0u));
}

// ------------------------------------------------------------------ the kept set by one workgroup
// The chunks of a row go round the waves, R to each; a lane holds its keys in registers (longer rows: in rounds of as many, read
// again in every pass).  A histogram of equal bins between the row's smallest and largest key finds the bin of the kk-th best.
// Keys before the bin are counted chunk by chunk; those of the bin move to LDS, each wave's to places of its own, where each
// counts those before it, by key and position, and adds itself to its chunk's count if it is kept.  A scan of the counts says where the
// chunks' slots go.  (A bin of many keys, ties above all, is narrowed down digit by digit, and the chunks are counted afterwards.)
// What bounds it is the chain: the row, its pages, the scores, and six barriers with a few LDS accesses between.  So the
// chunks do not depend on the length (the page numbers are on their way before it is known), and nothing goes through an atomic
// that returns.  48 lists of 5461 keys 10.7 us, 768 of them 17.4 (17 MB of scores, 1 TB/s; its vector instructions alone are 7 us), 1024
// of 4096 18.6.  24 keys to a lane are as many as the registers of three workgroups hold: 20 took the same for such rows,
// but cut those of more than 10240 keys into slices, two launches.
template <int NT> struct SelectShared {
  static constexpr int HIST = 4096, NW = NT / 64, NEAR = NT / NW;  // counters; keys of a bin that a wave can list
  __align__(16) uint32_t hist[HIST];
  __align__(16) uint32_t near[NT];  // entry e of wave w at e * NW + w
  uint32_t near_pos[NT];
  __align__(16) uint32_t kept[256], equal[256];  // per chunk of a round
  uint32_t wsum[NW][2];
  uint32_t st[4];
};

// A histogram has 1024 bins of four counters each, one for every fourth lane (scores share their leading bits: many lanes of a wave
// count in one bin), or, for rows of more than 4096 keys, 2048 of two: half the keys in a bin then (whole calls, us, 1024 / 2048 bins:
// lists x keys: 768 x 5461 55.1 / 53.4, 256 x 8192 29.2 / 26.7, 1024 x 4096 49.9 / 50.6, 768 x 1000 18.9 / 19.7).
struct KeyBins {
  int bits, shift;  // 2^bits bins of 2^shift counters
  __device__ __forceinline__ explicit KeyBins(bool fine) : bits(fine ? 11 : 10), shift(fine ? 1 : 2) {}
  __device__ __forceinline__ uint32_t word(uint32_t bin, int l) const { return (bin << shift) + (l & ((1 << shift) - 1)); }
};

// The bin at which the running count of the histogram reaches `remaining`, the rank inside it and its count (st[0..2]); CLEAR: leaves
// the histogram cleared.
template <int NT, bool CLEAR = true> __device__ __forceinline__ void pick_digit(SelectShared<NT>& m, const KeyBins& bins, uint32_t remaining) {
  static_assert(SelectShared<NT>::HIST == 8 * NT, "");
  const int tid = threadIdx.x, w = tid >> 6, l = tid & 63;
  uint4* hist4 = reinterpret_cast<uint4*>(m.hist);
  __syncthreads();
  const uint4 x = hist4[2 * tid], y = hist4[2 * tid + 1];
  if (CLEAR) hist4[2 * tid] = hist4[2 * tid + 1] = make_uint4(0, 0, 0, 0);
  uint32_t cn[4] = {x.x + x.y, x.z + x.w, y.x + y.y, y.z + y.w};  // this thread's bins: four, or two
  if (bins.shift == 2) {
    cn[0] += cn[1];
    cn[2] += cn[3];
    cn[1] = cn[3] = 0;
  }
  const uint32_t sum = cn[0] + cn[1] + cn[2] + cn[3];
  const uint32_t inc = wave_scan(sum, 0u, [](uint32_t a, uint32_t b) { return a + b; });
  if (l == 63) m.wsum[w][0] = inc;
  __syncthreads();
  uint32_t run = inc - sum;
#pragma unroll
  for (int i = 0; i < NT / 64; i++) run += i < w ? m.wsum[i][0] : 0u;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    if (run < remaining && remaining <= run + cn[i]) {  // exactly one bin of one thread
      m.st[0] = (uint32_t)(4 * tid + i) >> (bins.shift - 1);
      m.st[1] = remaining - run;
      m.st[2] = cn[i];
    }
    run += cn[i];
  }
  __syncthreads();
}

// Exclusive sums of a table of 256 counts at the entries u * 8 + w of this wave: entry u comes out of lane 2 u + w / 4.
__device__ __forceinline__ uint32_t chunk_offsets(const uint32_t* counts, int w, int l, uint32_t& total) {
  const uint4 x = reinterpret_cast<const uint4*>(counts)[l];
  const uint32_t sum = x.x + x.y + x.z + x.w, inc = wave_scan(sum, 0u, [](uint32_t a, uint32_t b) { return a + b; });
  total = last_lane(inc);
  const int i = w & 3;
  return inc - sum + (i > 0 ? x.x : 0u) + (i > 1 ? x.y : 0u) + (i > 2 ? x.z : 0u);
}

// KEYS: the listed keys go to `keys`, at the same places.
template <int NT, int R, int S, bool LONG, bool KEYS>
__device__ __forceinline__ void select_row(const CacheRef& c, const CacheRow& row, int h, int kk, int32_t* list, uint32_t* keys, SelectShared<NT>& m) {
  using M = SelectShared<NT>;
  constexpr int NW = M::NW, NEAR = M::NEAR, STEP = 4;
  static_assert(NW == 8 && R <= 32 && R % STEP == 0, "");
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), l = tid & 63, n = row.n;
  const char* scores = c.pages + c.off_z + ((size_t)h << c.shift) * 4;
  const KeyBins bins(n > 4096);
  const int rounds = LONG ? (n + NW * R * 64 - 1) / (NW * R * 64) : 1;
  PageRun<S> run;
  uint32_t key[R];
  bool bad = false;
  auto chunk = [&](int round, int u) { return ((round * R + u) * NW + w) * 64; };  // its first position
  auto fetch = [&](int round) {
    if (LONG) run.load(c, row, round * R * NW + w, NW, l);
    bad |= run.check(c, n, round * R * NW + w, NW, l);
#pragma unroll
    for (int u = 0; u < R; u++) key[u] = NO_KEY;
#pragma unroll
    for (int u0 = 0; u0 < R; u0 += STEP)
      if ((round * R + u0) * NW * 64 < n) {
#pragma unroll
        for (int u = u0; u < u0 + STEP; u++) key[u] = __float_as_uint(run.score(c, scores, chunk(round, u), u, l));
        __builtin_amdgcn_sched_barrier(0);  // (addresses of all chunks at once would spill)
      }
  };
  auto to_keys = [&](int round) {
#pragma unroll
    for (int u = 0; u < R; u++)
      if ((round * R + u / STEP * STEP) * NW * 64 < n) key[u] = l < n - chunk(round, u) ? score_key(__uint_as_float(key[u])) : NO_KEY;
  };
  // f(key, u) for the keys of a round; positions behind the row's end have NO_KEY
  auto each = [&](int round, auto f) {
    int left = n - round * R * NW * 64;
    asm volatile("" : "+s"(left));  // (comparisons kept from one pass to the next would spill)
#pragma unroll
    for (int u0 = 0; u0 < R; u0 += STEP)
      if (u0 * NW * 64 < left) {
#pragma unroll
        for (int u = u0; u < u0 + STEP; u++) f(key[u], u);
      }
  };
  auto every = [&](auto f) {
    if constexpr (!LONG) {
      each(0, f);
    } else {
      for (int round = 0; round < rounds; round++) {
        fetch(round);
        to_keys(round);
        each(round, f);
      }
    }
  };
  uint4* hist4 = reinterpret_cast<uint4*>(m.hist);
  uint32_t kmin = NO_KEY, kmax = 0;
  if (!LONG) run.load(c, row, w, NW, l);
  for (int i = tid; i < M::HIST / 4; i += NT) hist4[i] = make_uint4(0, 0, 0, 0);
  m.near[tid] = NO_KEY;
  if (tid < 256) m.kept[tid] = 0;
  if (tid == 0) m.st[3] = NO_KEY;
  if (!LONG) {
    fetch(0);
    to_keys(0);
  }
  every([&](uint32_t k32, int) {
    kmin = min(kmin, k32);
    kmax = max(kmax, k32 == NO_KEY ? 0u : k32);
  });
  kmin = last_lane(wave_scan(kmin, NO_KEY, [](uint32_t x, uint32_t y) { return min(x, y); }));
  kmax = last_lane(wave_scan(kmax, 0u, [](uint32_t x, uint32_t y) { return max(x, y); }));
  if (l == 0) {
    m.wsum[w][0] = kmin;
    m.wsum[w][1] = bad ? NO_KEY : kmax;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NW; i++) {
    kmin = min(kmin, m.wsum[i][0]);
    kmax = max(kmax, m.wsum[i][1]);
  }
  if (kmax == NO_KEY) {  // a page is out of range: the row sees nothing
    for (int i = tid; i < kk; i += NT) list[i] = -1;
    return;
  }
  kmin = (uint32_t)__builtin_amdgcn_readfirstlane((int)kmin);
  const uint32_t range = (uint32_t)__builtin_amdgcn_readfirstlane((int)(kmax - kmin));
  const int sh0 = max(0, 32 - (range ? __clz((int)range) : 32) - bins.bits);  // (key - kmin) >> sh0 < 2^bits
  // (positions without a key count in the last bin, behind every key of it)
  every([&](uint32_t k32, int) {
    atomicAdd(&m.hist[bins.word(min((k32 - kmin) >> sh0, (1u << bins.bits) - 1u), l)], 1u);
  });
  pick_digit<NT>(m, bins, (uint32_t)kk);
  const uint32_t base = kmin + (m.st[0] << sh0);  // first key of the bin
  const uint32_t width = min(1u << sh0, NO_KEY - base);
  uint32_t need_eq = m.st[1], n_eq = m.st[2], sub = 0;
  auto put = [&](int round, uint32_t at, auto keeps) {  // keeps(key, chunk)
#pragma unroll
    for (int q = 0; q < S; q++) asm volatile("" : "+v"(run.pg[q]));  // (the pages out of their lanes again, not kept since the scores)
    int left = n - round * R * NW * 64;
    asm volatile("" : "+s"(left));
#pragma unroll
    for (int u0 = 0; u0 < R; u0 += STEP)
      if (u0 * NW * 64 < left) {
#pragma unroll
        for (int u = u0; u < u0 + STEP; u++) {
          const unsigned long long k = __ballot(keeps(key[u], u));
          const int32_t x = run.slot(c, chunk(round, u), u, l);
          if (keeps(key[u], u)) {
            const uint32_t to = (uint32_t)__builtin_amdgcn_readlane((int)at, 2 * u + (w >> 2)) + lanes_before(k);
            list[to] = x;
            if constexpr (KEYS) keys[to] = key[u];
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
  };
  if constexpr (!LONG) {
    uint32_t count = 0;  // the wave's keys of the bin
    int left = n;
    asm volatile("" : "+s"(left));
#pragma unroll
    for (int u0 = 0; u0 < R; u0 += STEP)
      if (u0 * NW * 64 < left) {  // (four chunks are compared before the first result is used)
        unsigned long long in[STEP];
        uint32_t before[STEP];
#pragma unroll
        for (int e = 0; e < STEP; e++) {
          before[e] = (uint32_t)__popcll(__ballot(key[u0 + e] < base));
          in[e] = __ballot(key[u0 + e] - base < width);
        }
        if (l == 0) {
#pragma unroll
          for (int e = 0; e < STEP; e++) m.kept[(u0 + e) * NW + w] = before[e];
        }
        if (in[0] | in[1] | in[2] | in[3]) {
#pragma unroll
          for (int e = 0; e < STEP; e++) {
            const uint32_t i = count + lanes_before(in[e]);
            if (key[u0 + e] - base < width && i < NEAR) {
              m.near[i * NW + w] = key[u0 + e] - base;
              m.near_pos[i * NW + w] = (uint32_t)(chunk(0, u0 + e) + l);
            }
            count += (uint32_t)__popcll(in[e]);
          }
        }
      }
    if (l == 0) m.wsum[w][1] = count;
    __syncthreads();
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < NW; i++) most = max(most, m.wsum[i][1]);
    if (most <= NEAR) {
      const uint32_t x = m.near[tid];
      if (x != NO_KEY) {
        uint32_t less = 0, equal = 0;
        for (uint32_t i = 0; i < most * NW; i += 8) {
          const uint4 q = *reinterpret_cast<const uint4*>(&m.near[i]), r = *reinterpret_cast<const uint4*>(&m.near[i + 4]);
          const uint32_t cs[8] = {q.x, q.y, q.z, q.w, r.x, r.y, r.z, r.w};
#pragma unroll
          for (int e = 0; e < 8; e++) {
            less += cs[e] < x;
            equal += cs[e] == x;
          }
        }
        const uint32_t pos = m.near_pos[tid];
        if (equal > 1)
          for (uint32_t i = 0; i < most * NW; i++) less += m.near[i] == x && m.near_pos[i] < pos;
        if (less < need_eq) atomicAdd(&m.kept[pos >> 6], 1u);
        if (less + 1 == need_eq) {  // the last one that is kept, and the first that is not
          m.st[0] = x;
          m.st[1] = pos;
        }
        if (less == need_eq) m.st[3] = x;
      }
      __syncthreads();
      const uint32_t thr = (uint32_t)__builtin_amdgcn_readfirstlane((int)(base + m.st[0]));
      const int last = __builtin_amdgcn_readfirstlane((int)m.st[1]);
      uint32_t total;
      const uint32_t at = chunk_offsets(m.kept, w, l, total);
      if (m.st[3] != m.st[0]) put(0, at, [&](uint32_t k32, int) { return k32 <= thr; });
      else put(0, at, [&](uint32_t k32, int u) { return k32 < thr || (k32 == thr && l <= last - chunk(0, u)); });
      return;
    }
  }
  for (int sh = sh0; sh > 0;) {  // (at most 22 bits are left: three rounds)
    const int bits = min(bins.bits, sh), s2 = sh - bits;
    uint32_t from = base;
    asm volatile("" : "+v"(from));  // (the differences of all keys, kept from round to round, would spill)
    every([&](uint32_t k32, int) {
      const uint32_t x = k32 - from;  // (of keys before the bin it wraps round to the far end: never equal to `sub`)
      if (k32 != NO_KEY && (x >> sh) == sub) atomicAdd(&m.hist[bins.word((x >> s2) & ((1u << bits) - 1u), l)], 1u);
    });
    pick_digit<NT>(m, bins, need_eq);
    sub = (sub << bits) | m.st[0];
    need_eq = m.st[1];
    n_eq = m.st[2];
    sh = s2;
  }
  const uint32_t thr = (uint32_t)__builtin_amdgcn_readfirstlane((int)(base + sub));
  const bool ties = n_eq != need_eq;  // some keys equal to the threshold are left out: those of the highest positions
  uint32_t done = 0, done_eq = 0;
  for (int round = 0; round < rounds; round++) {
    if (LONG) {
      fetch(round);
      to_keys(round);
    }
    uint32_t kept = 0, equal = 0;  // lane u: of this wave's chunk u
    each(round, [&](uint32_t k32, int u) {
      const uint32_t b = (uint32_t)__popcll(__ballot(ties ? k32 < thr : k32 <= thr)), e = (uint32_t)__popcll(__ballot(k32 == thr));
      kept = l == u ? b : kept;
      equal = l == u ? e : equal;
    });
    if (l < 32) {
      m.kept[l * NW + w] = kept;
      m.equal[l * NW + w] = equal;
    }
    __syncthreads();
    uint32_t total, total_eq = 0;
    const uint32_t at = done + chunk_offsets(m.kept, w, l, total);
    if (!ties) {
      put(round, at, [&](uint32_t k32, int) { return k32 <= thr; });
    } else {
      const uint32_t at_eq = done_eq + chunk_offsets(m.equal, w, l, total_eq);
      each(round, [&](uint32_t k32, int u) {
        const unsigned long long bm = __ballot(k32 < thr), em = __ballot(k32 == thr);
        if (bm | em) {
          const uint32_t first = (uint32_t)__builtin_amdgcn_readlane((int)at, 2 * u + (w >> 2));
          const uint32_t eq = (uint32_t)__builtin_amdgcn_readlane((int)at_eq, 2 * u + (w >> 2)) + lanes_before(em);  // equal ones before
          const int32_t x = run.slot(c, chunk(round, u), u, l);
          if (k32 < thr || (k32 == thr && eq < need_eq)) {
            const uint32_t to = first + lanes_before(bm) + min(eq, need_eq);
            list[to] = x;
            if constexpr (KEYS) keys[to] = k32;
          }
        }
      });
    }
    done += total;
    done_eq += total_eq;
    if (round + 1 < rounds) __syncthreads();
  }
}

// ------------------------------------------------------------------ the kept set of a long row, by slices
// Rows of more than SELECT_SHORT keys are cut into slices of SLICE keys.  The first launch takes from a sample of the whole row two
// keys that the kk-th best very likely lies between (3.5 standard deviations of its rank in the sample to either side, or as much as
// the lists hold; of 4096 keys instead of 2048, 5 us more, if that is less than 3.5 of 2048); it counts a
// slice's keys that are better and lists those between, with their positions.  The second ranks the listed keys of all slices, a few
// per cent of the row, for the exact threshold (by key and position: no ties are left), and writes a slice's kept slots behind those
// of the slices before it.  Where the threshold lies outside after all, or a list is too short for its keys (ties, above all), or
// the row has more than SLICES_MAX slices, one workgroup selects alone.
// A row's slices go round its `parts` workgroups.  How many rows are long the host does not know, so there are only as many parts
// as keep the chip busy: workgroups that find nothing to do cost 1 ns each.
// Both launches are chains of loads and barriers again: 32 lists of 65536 keys 11.9 and 10.4 us (8.4 MB each: 0.8 TB/s); whole
// calls, with one workgroup to a list, 105 us, so 28.6, 256 such lists 116.  One workgroup alone takes 0.2 ms for 131072 keys, 0.7 for 524288.
constexpr int SELECT_REGS = 24, SELECT_SHORT = 512 * SELECT_REGS;
constexpr int SLICE_CHUNKS = 16, SLICE = 512 * SLICE_CHUNKS, SLICES_MAX = 64;
constexpr int SAMPLE = 2048, LISTED = 8192;  // keys that the lists of a row hold together at most, an equal share for each slice

struct SliceWork {
  uint2* counts;  // [pairs of a launch][SLICES_MAX]: better keys, listed keys (more than the share: not all are)
  uint2* listed;  // [pairs of a launch][room]: key, position
  uint4* bounds;  // [pairs of a launch]: first and last key of the lists; the same, or those of the sample where the lists have no end
  int room, parts;
  int first, pairs;  // the pairs (row * H_q + head) of this launch
};

// The keys of a slice, its chunks in turn to the waves (NO_KEY behind the row's end), once slice_pages has asked for its pages.
// False: a page is out of range.
template <int S>
__device__ __forceinline__ void slice_pages(const CacheRef& c, const CacheRow& row, int slice, PageRun<S>& run) {
  run.load(c, row, slice * (SLICE / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), 8, threadIdx.x & 63);
}
template <int S>
__device__ __forceinline__ bool slice_keys(const CacheRef& c, const CacheRow& row, int h, int slice, PageRun<S>& run, uint32_t* key) {
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, n = row.n;
  const char* scores = c.pages + c.off_z + ((size_t)h << c.shift) * 4;
  const bool bad = run.check(c, n, slice * (SLICE / 64) + w, 8, l);
#pragma unroll
  for (int u0 = 0; u0 < SLICE_CHUNKS; u0 += 4) {
#pragma unroll
    for (int u = u0; u < u0 + 4; u++) key[u] = __float_as_uint(run.score(c, scores, slice * SLICE + (u * 8 + w) * 64, u, l));
    __builtin_amdgcn_sched_barrier(0);
  }
#pragma unroll
  for (int u = 0; u < SLICE_CHUNKS; u++) key[u] = l < n - (slice * SLICE + (u * 8 + w) * 64) ? score_key(__uint_as_float(key[u])) : NO_KEY;
  return !bad;
}

// How far from its expected rank in a sample the key at that share of the row may lie: 3.5 standard deviations.
__device__ __forceinline__ float bracket(float share, float size) { return 3.5f * sqrtf(size * share * (1.f - share)) + 3.f; }

// Counts and lists of one workgroup's slices of a long row.
template <int S>
__device__ __forceinline__ void list_slices(const CacheRef& c, const CacheRow& row, int h, int kk, int pair, int part, const SliceWork& sw,
                                            SelectShared<512>& m) {
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), l = tid & 63, n = row.n;
  const int slices = (n - 1) / SLICE + 1, share = sw.room / slices;
  const KeyBins bins(false);
  if (slices > SLICES_MAX || part >= slices) return;
  PageRun<S> run;
  slice_pages<S>(c, row, part, run);
  uint4* hist4 = reinterpret_cast<uint4*>(m.hist);
  for (int i = tid; i < m.HIST / 4; i += 512) hist4[i] = make_uint4(0, 0, 0, 0);
  // The sample: one key of each of 2048 equal parts of the row, or of 4096 where the lists would be too long for their share, at a
  // place in it that follows no period.
  const float kept_share = (float)kk / (float)n, room = ((float)share - 5.f * sqrtf((float)share)) / SLICE;  // (slices differ)
  const bool wide = 2.f * bracket(kept_share, SAMPLE) > room * SAMPLE;
  const int log_n = wide ? 12 : 11;
  static_assert(SAMPLE == 2048, "");
  uint32_t sample[SAMPLE / 256], key[SLICE_CHUNKS];
#pragma unroll
  for (int e = 0; e < SAMPLE / 256; e++) {
    if (e >= SAMPLE / 512 && !wide) continue;
    const uint32_t i = (uint32_t)(e * 512 + tid), width = (uint32_t)n >> log_n;
    const int j = (int)((unsigned long long)i * (uint32_t)n >> log_n) + (int)((i * 2654435761u >> 16) * width >> 16);
    sample[e] = score_key(cache_score(c, cache_slot(c, row, j), h));
  }
  bool good = slice_keys<S>(c, row, h, part, run, key);
  uint32_t kmin = NO_KEY, kmax = 0;
  auto each = [&](auto f) {
#pragma unroll
    for (int e = 0; e < SAMPLE / 256; e++)
      if (e < SAMPLE / 512 || wide) f(sample[e]);
  };
  each([&](uint32_t k) {
    kmin = min(kmin, k);
    kmax = max(kmax, k);
  });
  kmin = last_lane(wave_scan(kmin, NO_KEY, [](uint32_t x, uint32_t y) { return min(x, y); }));
  kmax = last_lane(wave_scan(kmax, 0u, [](uint32_t x, uint32_t y) { return max(x, y); }));
  if (l == 0) {
    m.wsum[w][0] = kmin;
    m.wsum[w][1] = kmax;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; i++) {
    kmin = min(kmin, m.wsum[i][0]);
    kmax = max(kmax, m.wsum[i][1]);
  }
  const uint32_t range = kmax - kmin;
  const int sh = max(0, 32 - (range ? __clz((int)range) : 32) - bins.bits);
  each([&](uint32_t k) { atomicAdd(&m.hist[bins.word((k - kmin) >> sh, l)], 1u); });
  const float size = (float)(1 << log_n), middle = kept_share * size, off = fminf(bracket(kept_share, size), 0.5f * room * size);
  // The first (end = 0) or last key of the sample's keys that cannot be told from the one of that rank: those of a bin, or, if these
  // are so many that the lists would grow by an eighth (wide: a 32nd) of their share, of a 1024th of it.
  auto key_of_rank = [&](uint32_t rank, uint32_t end) {
    pick_digit<512, false>(m, bins, rank);
    const uint32_t digit = m.st[0], left = m.st[1], first = kmin + (digit << sh), crowd = m.st[2];
    if (sh == 0 || crowd * SLICE <= (uint32_t)share << (wide ? log_n - 5 : log_n - 3)) return __builtin_elementwise_add_sat(first, (end << sh) - end);
    const int s2 = max(0, sh - bins.bits);
    __syncthreads();
    for (int i = tid; i < m.HIST / 4; i += 512) hist4[i] = make_uint4(0, 0, 0, 0);
    __syncthreads();
    each([&](uint32_t k) {
      if ((k - kmin) >> sh == digit) atomicAdd(&m.hist[bins.word((k - first) >> s2, l)], 1u);
    });
    pick_digit<512>(m, bins, left);
    const uint32_t found = __builtin_elementwise_add_sat(first + (m.st[0] << s2), (end << s2) - end);
    each([&](uint32_t k) { atomicAdd(&m.hist[bins.word((k - kmin) >> sh, l)], 1u); });
    return found;
  };
  uint32_t lo = 0, hi = NO_KEY - 1;
  if (middle - off >= 1.f) lo = key_of_rank((uint32_t)(middle - off), 0u);
  if (middle + off < size) hi = min(key_of_rank((uint32_t)(middle + off) + 1u, 1u), hi);
  lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)lo);
  hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)hi);
  if (tid == 0 && part == 0) sw.bounds[pair] = make_uint4(lo, hi, lo ? lo : kmin, hi == NO_KEY - 1 ? kmax : hi);
  for (int slice = part; slice < slices; slice += sw.parts) {
    if (slice != part) {
      slice_pages<S>(c, row, slice, run);
      good = slice_keys<S>(c, row, h, slice, run, key);
    }
    uint32_t better = 0, mine = 0;  // keys of this wave
#pragma unroll
    for (int u = 0; u < SLICE_CHUNKS; u++) {
      better += (uint32_t)__popcll(__ballot(key[u] < lo));
      mine += (uint32_t)__popcll(__ballot(key[u] - lo <= hi - lo));
    }
    __syncthreads();  // (wsum: the last digit's, or the slice's before)
    if (l == 0) {
      m.wsum[w][0] = better;
      m.wsum[w][1] = good ? mine : NO_KEY >> 4;  // (a page is out of range: the second launch sees an impossible count)
    }
    __syncthreads();
    uint32_t all_better = 0, all = 0, at = 0;
#pragma unroll
    for (int i = 0; i < 8; i++) {
      at += i < w ? m.wsum[i][1] : 0u;
      all_better += m.wsum[i][0];
      all += m.wsum[i][1];
    }
    uint2* listed = sw.listed + (size_t)pair * sw.room + slice * share;
#pragma unroll
    for (int u = 0; u < SLICE_CHUNKS; u++) {
      const bool in = key[u] - lo <= hi - lo;
      const unsigned long long b = __ballot(in);
      const uint32_t i = at + lanes_before(b);
      if (in && i < (uint32_t)share) listed[i] = make_uint2(key[u], (uint32_t)(slice * SLICE + (u * 8 + w) * 64 + l));
      at += (uint32_t)__popcll(b);
    }
    if (tid == 0) sw.counts[(size_t)pair * SLICES_MAX + slice] = make_uint2(all_better, all);
  }
}

// Workgroups per (row, head): one that selects for a short row, or, SLICED, parts of a long one (a second launch follows).  Not SLICED:
// the caller's bound says that no row is long; one that is all the same is selected by one workgroup.
// WAVES: four workgroups share a compute unit where 64 registers hold what they need (8), at the price of some in scratch, three where
// they do not (6).  Four are worth it from more lists on than three of each compute unit are (whole calls, us, 6 / 8: 256 lists of
// 8192 keys 26.7 / 27.1, 768 of 5461 53.4 / 54.2, 1024 of 4096 50.6 / 48.9, 2048 of 4096 79.0 / 78.1; SLICED, 2048 parts of 8192: 115.3 / 115.2).
// Not `whole`: rows that keep all their keys get no list.  EITHER: the launch is for rows in slices, but these may be none (no parts: there is no room for what slices tell each other).
template <int S, bool SLICED, bool KEYS, bool EITHER = false>
__device__ __forceinline__ void select_block(const CacheRef& c, const CacheRows& p, const SliceWork& sw, int32_t* kept, uint32_t* keys, int block,
                                             bool whole = true) {
  const int part = SLICED ? block / sw.pairs : 0, pair = block - part * sw.pairs, rh = sw.first + pair;
  const int r = rh / c.H_q, h = rh - r * c.H_q;
  const int tid = threadIdx.x;
  const CacheRow row = cache_row(c, p, r);
  const bool slices = SLICED && (!EITHER || sw.parts);
  const int n = row.n, kk = min(p.k, n), parts = slices && n > SELECT_SHORT ? sw.parts : 1;
  if (part && n <= SELECT_SHORT) return;
  int32_t* list = kept + (size_t)rh * p.kcap;
  if (kk == n && !whole) return;
  if (kk == n) {  // (a page out of range anywhere: none is kept)
    bool bad = false;
    for (long long j = tid; j << c.shift < n; j += 512) bad |= (uint32_t)row.pages[j] >= (uint32_t)c.n_pages;
    const int there = __syncthreads_or(bad) ? 0 : n;
    for (long long j = part * 512 + tid; j < (KEYS ? n : p.kcap); j += parts * 512) {
      const int32_t slot = j < there ? (int32_t)cache_slot(c, row, (int)j) : -1;
      list[j] = slot;
      if constexpr (KEYS) keys[(size_t)rh * p.kcap + j] = score_key(cache_score(c, (uint32_t)slot, h));
    }
    return;
  }
  __shared__ SelectShared<512> m;
  keys += KEYS ? (size_t)rh * p.kcap : 0;
  if (n <= SELECT_SHORT) select_row<512, SELECT_REGS, S, false, KEYS>(c, row, h, kk, list, keys, m);
  else if (slices) {
    if constexpr (SLICED) list_slices<S>(c, row, h, kk, pair, part, sw, m);
  } else if constexpr (!SLICED || EITHER) {
    select_row<512, SELECT_REGS, S, true, KEYS>(c, row, h, kk, list, keys, m);
  }
}

template <int S, bool KEYS>
__device__ __forceinline__ void slice_block(const CacheRef& c, const CacheRows& p, const SliceWork& sw, int32_t* kept, uint32_t* keys, int block) {
  const int part = block / sw.pairs, pair = block - part * sw.pairs, rh = sw.first + pair, r = rh / c.H_q, h = rh - r * c.H_q;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), l = tid & 63;
  uint2 cnt = sw.counts[(size_t)pair * SLICES_MAX + l];  // lane s: of slice s
  const uint4 bounds = sw.bounds[pair];
  const CacheRow row = cache_row(c, p, r);
  PageRun<S> run;
  slice_pages<S>(c, row, part, run);
  const int n = row.n, kk = min(p.k, n);
  if (n <= SELECT_SHORT || part * SLICE >= n || kk == n) return;
  int32_t* list = kept + (size_t)rh * p.kcap;
  keys += KEYS ? (size_t)rh * p.kcap : 0;
  __shared__ SelectShared<512> m;
  __shared__ __align__(16) uint32_t cand[LISTED];
  const int slices = (n - 1) / SLICE + 1, share = sw.room / slices;
  const KeyBins bins(false);
  const auto add = [](uint32_t x, uint32_t y) { return x + y; };
  if (l >= slices) cnt = make_uint2(0, 0);
  const unsigned long long over = __ballot(cnt.y > (uint32_t)share);
  const uint32_t upto = wave_scan(min(cnt.y, (uint32_t)share), 0u, add);
  const uint32_t better = last_lane(wave_scan(cnt.x, 0u, add)), all = last_lane(upto);
  const bool found = slices <= SLICES_MAX && !over && better < (uint32_t)kk && (uint32_t)kk - better <= all;
  // f(first listed key of slice s in LDS, their number, s) for the slices of this wave, every eighth
  auto lists = [&](auto f) {
    for (int s = w; s < slices; s += 8) {
      const uint32_t have = (uint32_t)__builtin_amdgcn_readlane((int)cnt.y, s), end = (uint32_t)__builtin_amdgcn_readlane((int)upto, s);
      f(end - have, have, s);
    }
  };
  const uint2* listed = sw.listed + (size_t)pair * sw.room;
  uint32_t* near_all = &m.st[3];
  uint32_t key[SLICE_CHUNKS], base = 0, rank = 0, n_near = NO_KEY, digit = 0;
  int sh = 0;
  // (keys beyond the sample's are in the first or the last bin: bins over all that a list may hold would be too wide for its keys)
  const uint32_t from = (uint32_t)__builtin_amdgcn_readfirstlane((int)bounds.z);
  auto bin = [&](uint32_t k) { return min(__builtin_elementwise_sub_sat(k, from) >> sh, (1u << bins.bits) - 1u); };
  if (found) {
    uint4* hist4 = reinterpret_cast<uint4*>(m.hist);
    for (int i = tid; i < m.HIST / 4; i += 512) hist4[i] = make_uint4(0, 0, 0, 0);
    if (tid == 0) *near_all = 0;
    const uint32_t range = (uint32_t)__builtin_amdgcn_readfirstlane((int)bounds.w) - from;
    sh = max(0, 32 - (range ? __clz((int)range) : 32) - bins.bits);
    lists([&](uint32_t to, uint32_t have, int s) {
      for (uint32_t i0 = 0; i0 < have; i0 += 256) {
        uint32_t k[4];
#pragma unroll
        for (int e = 0; e < 4; e++) k[e] = listed[s * share + min(i0 + e * 64 + l, have - 1)].x;
#pragma unroll
        for (int e = 0; e < 4; e++)
          if (i0 + e * 64 + l < have) cand[to + i0 + e * 64 + l] = k[e];
      }
    });
    (void)slice_keys<S>(c, row, h, part, run, key);  // (on its way under the search for the threshold)
    __syncthreads();
    for (uint32_t i = tid; i < all; i += 512) atomicAdd(&m.hist[bins.word(bin(cand[i]), l)], 1u);
    pick_digit<512>(m, bins, (uint32_t)kk - better);
    digit = (uint32_t)__builtin_amdgcn_readfirstlane((int)m.st[0]);
    base = digit ? from + (digit << sh) : 0u;
    rank = m.st[1];
    n_near = m.st[2];
  }
  if (n_near > 512) {  // (ties, or nothing found at all)
    __syncthreads();
    if (part == 0) select_row<512, SELECT_REGS, S, true, KEYS>(c, row, h, kk, list, keys, m);
    return;
  }
  // The bin's keys with their positions (again from the lists); kept keys of every slice that are before the bin (m.equal).
  lists([&](uint32_t to, uint32_t have, int s) {
    uint32_t ahead = (uint32_t)__builtin_amdgcn_readlane((int)cnt.x, s);
    for (uint32_t i0 = 0; i0 < have; i0 += 64) {
      const bool there = i0 + l < have;
      const uint32_t k = there ? cand[to + i0 + l] : NO_KEY;
      ahead += (uint32_t)__popcll(__ballot(k < base));
      if (there && bin(k) == digit) {
        const uint32_t e = atomicAdd(near_all, 1u);
        m.near[e] = k;
        m.near_pos[e] = listed[s * share + i0 + l].y;
      }
    }
    if (l == 0) m.equal[s] = ahead;
  });
  if (tid < 256 - 16 * 8) m.kept[16 * 8 + tid] = 0;  // (chunks that a slice does not have)
  uint32_t* first_out = &m.wsum[0][0];
  if (tid == 0) *first_out = NO_KEY;
  __syncthreads();
  if (tid < (int)n_near) {
    const uint32_t k = m.near[tid], pos = m.near_pos[tid];
    uint32_t less = 0;
    for (uint32_t i = 0; i < n_near; i++) less += m.near[i] < k || (m.near[i] == k && m.near_pos[i] < pos);
    if (less < rank) atomicAdd(&m.equal[pos / SLICE], 1u);
    if (less + 1 == rank) {  // the last one that is kept, and the first that is not
      m.st[0] = k;
      m.st[1] = pos;
    }
    if (less == rank) *first_out = k;
  }
  __syncthreads();
  const uint32_t thr = (uint32_t)__builtin_amdgcn_readfirstlane((int)m.st[0]);
  const int last = __builtin_amdgcn_readfirstlane((int)m.st[1]);
  const uint32_t of_slice = l < slices ? m.equal[l] : 0u, before = wave_scan(of_slice, 0u, add) - of_slice;  // lane s: kept before slice s
  for (int slice = part; slice < slices; slice += sw.parts) {
    if (slice != part) {
      slice_pages<S>(c, row, slice, run);
      (void)slice_keys<S>(c, row, h, slice, run, key);
    }
    // keeps(u): whether this lane's key of chunk u is kept
    auto put = [&](auto keeps) {
      if (slice != part) __syncthreads();
      uint32_t count[SLICE_CHUNKS];
#pragma unroll
      for (int u = 0; u < SLICE_CHUNKS; u++) count[u] = (uint32_t)__popcll(__ballot(keeps(u)));
      if (l == 0) {
#pragma unroll
        for (int u = 0; u < SLICE_CHUNKS; u++) m.kept[u * 8 + w] = count[u];
      }
      __syncthreads();
      uint32_t total;
      const uint32_t at = (uint32_t)__builtin_amdgcn_readlane((int)before, slice) + chunk_offsets(m.kept, w, l, total);
#pragma unroll
      for (int q = 0; q < S; q++) asm volatile("" : "+v"(run.pg[q]));
#pragma unroll
      for (int u = 0; u < SLICE_CHUNKS; u++) {
        const unsigned long long b = __ballot(keeps(u));
        const int32_t slot = run.slot(c, slice * SLICE + (u * 8 + w) * 64, u, l);
        if (keeps(u)) {
          const uint32_t to = (uint32_t)__builtin_amdgcn_readlane((int)at, 2 * u + (w >> 2)) + lanes_before(b);
          list[to] = slot;
          if constexpr (KEYS) keys[to] = key[u];
        }
        if (u % 4 == 3) __builtin_amdgcn_sched_barrier(0);  // (addresses of all chunks at once would spill)
      }
    };
    if (*first_out != thr) put([&](int u) { return key[u] <= thr; });
    else put([&](int u) { return key[u] < thr || (key[u] == thr && l <= last - (slice * SLICE + (u * 8 + w) * 64)); });
  }
}

inline int list_length(const dma_cache_shape& s, int k) {
  const long cap = (long)s.max_pages * s.page_size;
  return (int)(k < cap ? k : cap);
}

// What the parts of the rows tell each other, where rows can be long.
struct SelectWork {
  size_t off_counts, off_listed, off_bounds;
  int parts;  // of a long row; 0: no row is long
  int room;   // keys of a row's lists
  int pairs;  // (row, head) pairs of a launch
};
constexpr int SELECT_WGS = 8 * CUS;  // workgroups that the parts are chosen for

// The lists of a pair take 64 KiB, and half as much from more than LISTED_PAIRS pairs on; there is room for twice as many of those, and
// more go through the same room, 256 MiB, in several launches (room for every pair: 0.5 GiB for 256 rows of 32 heads, 2 for
// 1024).  Whole calls of 32 heads, us, room for every pair / this: 160 rows of 20000 to 60000 keys 1044 / 1043, of 60000 to 130000 1871 /
// 1999 (half lists take the larger sample there), 256 of 14000 to 30000 1143 / 1145, 256 of which every eighth has 60000 keys and the others
// 3000 608 / 609 (whole lists, launches of 4096 / 2048 pairs: 666 / 799), 1024 of 500 to 3000 983 / 995.  (6 bytes a key, its place in
// the slice for its position: 196 MiB, but one row of 65536 keys 28.6 / 29.2.)
constexpr int LISTED_PAIRS = 4096;
// Its place behind the first `total` bytes of a workspace (pairs > 0; no size is less for more of them).  bound: on a row's keys, 0: none known.
inline SelectWork select_work(const dma_cache_shape& s, size_t pairs, int kcap, int bound, size_t& total) {
  SelectWork wk;
  auto take = [&](size_t bytes) { size_t at = total; total = align_up(total + bytes, 256); return at; };
  const long cap = (long)s.max_pages * s.page_size, longest = bound > 0 && bound < cap ? bound : cap;
  const size_t launches = (pairs + 2 * LISTED_PAIRS - 1) / (2 * LISTED_PAIRS);
  wk.pairs = (int)((pairs + launches - 1) / launches);
  const long slices = longest <= SELECT_SHORT || kcap == cap ? 0 : (longest + SLICE - 1) / SLICE, most = SELECT_WGS / (long)wk.pairs;
  wk.parts = (int)(slices < most ? slices : most < 1 && slices ? 1 : most);
  wk.room = pairs > LISTED_PAIRS ? LISTED / 2 : LISTED;
  const size_t whole = pairs < LISTED_PAIRS ? pairs : LISTED_PAIRS, most_pairs = pairs < 2 * LISTED_PAIRS ? pairs : 2 * LISTED_PAIRS;
  wk.off_counts = take(wk.parts ? most_pairs * SLICES_MAX * 8 : 0);
  wk.off_listed = take(wk.parts ? whole * LISTED * 8 : 0);  // (wk.pairs * wk.room are never more)
  wk.off_bounds = take(wk.parts ? most_pairs * 16 : 0);
  return wk;
}

}  // namespace
}  // namespace dma
