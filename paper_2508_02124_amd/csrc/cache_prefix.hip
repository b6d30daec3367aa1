// Decode over the paged 4-bit cache for requests that share prefixes: a row's keys are those of its prefix, then its request's own, and it
// keeps the min(k, n) best of all of them by (score descending, position ascending).
//
// The min(k, P) best of a prefix are listed once for each of its heads; what a row keeps are the k best of that list and its own keys
// together, a cut through both.  So a prefix is selected from once, and its listed K and V are gathered and decoded once for 32 rows: they are
// the columns of two matrix products whose weights each row masks by its own cut.  Four launches (five behind long prefixes; where lists
// of more than 8192 pairs are made in slices, the first two in turns):
//   prefix_select_kernel (prefix_slice_kernel)   the lists, and the rows in order of their prefixes
//   prefix_cut_kernel                            a row's cut, and which of its own keys it keeps
//   prefix_tile_kernel                           attention to the prefixes, in parts
//   prefix_own_kernel                            attention to a row's own keys, joined with the parts
#include "cache_attend.h"
#include "cache_select.h"

namespace dma {

constexpr int TILE_ROWS = 32;

// What a row sees: its own keys (0: no row) and the prefix (-1: none) with its keys, and its request.
struct PrefixRow {
  int own, pre, prefix, req;
};
// Rows of one prefix (count 0: behind the last tile; only that many of the rows are there).
struct PrefixTile {
  int prefix, count, pre, unused;
  int rows[TILE_ROWS];
};
// What a row keeps: of the prefix's list the keys before `key`, and those equal to it up to place `last`; of its own the `count` that
// are listed (-1: a page is out of range, the row sees nothing).
struct Cut {
  uint32_t key;
  int last, count, unused;
};

struct PrefixArgs {
  CacheRows own, pre;  // the rows, and the prefixes as rows of the requests that hold them
  const int32_t* req_prefix;
  PrefixRow* rows;
  PrefixTile* tiles;
  int32_t *list_pre, *list_own;    // [prefixes or rows][H_q][kcap]
  uint32_t *keys_pre, *keys_own;   // the listed keys
  Cut* cuts;                       // [rows][H_q]
  float* part;                     // [rows][H_q][nsplit]: D sums over a part of the prefix's list, their reference, their weight, and two more
  int max_tiles, nsplit;
  bool listed;                     // rows of more than k keys of their own have lists of them
};

// ------------------------------------------------------------------ the rows by prefix
// One workgroup: what each row sees, and the rows of each prefix together, in tiles.  (A row's result does not depend on its place in a
// tile, so the order inside a prefix may be any.)  It runs beside the workgroups that select, which take longer.
__device__ __forceinline__ void group_rows(const CacheRef& c, const PrefixArgs& p) {
  __shared__ uint32_t cursor[CACHE_REQS_MAX];  // rows of a prefix, then the place of the next one: tile * 32 + row in it
  __shared__ uint32_t wsum[8];
  const int tid = threadIdx.x, l = tid & 63, w = tid >> 6, n_prefixes = p.pre.n_rows;
  constexpr int PER = CACHE_REQS_MAX / 512;
  for (int i = tid; i < n_prefixes; i += 512) cursor[i] = 0;
  __syncthreads();
  for (int r = tid; r < p.own.n_rows; r += 512) {
    const int req = p.own.row_req ? p.own.row_req[r] : r;
    PrefixRow row = {cache_row(c, p.own, r).n, 0, -1, req};
    if (n_prefixes && row.own > 0) {  // (the request is in range)
      const int prefix = p.req_prefix[req];
      if ((uint32_t)prefix < (uint32_t)n_prefixes) row.pre = cache_row(c, p.pre, prefix).n;
      if (row.pre > 0) {
        row.prefix = prefix;
        atomicAdd(&cursor[prefix], 1u);
      }
    }
    p.rows[r] = row;
  }
  __syncthreads();
  if (!n_prefixes) return;
  uint32_t count[PER], tiles = 0;
#pragma unroll
  for (int e = 0; e < PER; e++) {
    const int i = tid * PER + e;
    count[e] = i < n_prefixes ? cursor[i] : 0u;
    tiles += (count[e] + TILE_ROWS - 1) / TILE_ROWS;
  }
  uint32_t tile0 = wave_scan(tiles, 0u, [](uint32_t a, uint32_t b) { return a + b; });
  if (l == 63) wsum[w] = tile0;
  __syncthreads();
  tile0 -= tiles;
  uint32_t all_tiles = 0;
#pragma unroll
  for (int i = 0; i < 8; i++) {
    tile0 += i < w ? wsum[i] : 0u;
    all_tiles += wsum[i];
  }
#pragma unroll
  for (int e = 0; e < PER; e++) {
    const int i = tid * PER + e;
    if (i >= n_prefixes) break;
    const int pre = count[e] ? cache_row(c, p.pre, i).n : 0;
    cursor[i] = tile0 * TILE_ROWS;
    for (uint32_t a = 0; a < count[e]; a += TILE_ROWS, tile0++) {
      PrefixTile& t = p.tiles[tile0];
      t.prefix = i;
      t.count = (int)min(count[e] - a, (uint32_t)TILE_ROWS);
      t.pre = pre;
    }
  }
  for (int i = (int)all_tiles + tid; i < p.max_tiles; i += 512) p.tiles[i].count = 0;
  __syncthreads();
  for (int r = tid; r < p.own.n_rows; r += 512) {
    const int prefix = p.rows[r].prefix;  // (this thread wrote it)
    if (prefix >= 0) {
      const uint32_t at = atomicAdd(&cursor[prefix], 1u);
      p.tiles[at / TILE_ROWS].rows[at % TILE_ROWS] = r;
    }
  }
}

// ------------------------------------------------------------------ the lists
struct SelectSet {
  CacheRows rows;
  SliceWork sw;
  int32_t* list;
  uint32_t* keys;
  int wgs;
};

// The prefixes' lists, and those of rows with more than k keys of their own.  GROUP: the first workgroup orders the rows.  Chains of
// loads and barriers, as in cache_decode.hip: 32 lists of 16384 keys 11.4 us and 10.3 for the slices (one workgroup to a list: 32), 32 of 4096 9.4.
template <int S, bool SLICED, bool GROUP>
__global__ __launch_bounds__(512, 6) void prefix_select_kernel(CacheRef c, PrefixArgs p, SelectSet a, SelectSet b) {
  int block = (int)blockIdx.x - (GROUP ? 1 : 0);
  if (GROUP && block < 0) {
    group_rows(c, p);
    return;
  }
  const bool first = block < a.wgs;
  if (!first) block -= a.wgs;
  const CacheRows rows = first ? a.rows : b.rows;
  const SliceWork sw = first ? a.sw : b.sw;
  select_block<S, SLICED, true, true>(c, rows, sw, first ? a.list : b.list, first ? a.keys : b.keys, block, first);
}
template <int S>
__global__ __launch_bounds__(512, 4) void prefix_slice_kernel(CacheRef c, SelectSet a, SelectSet b) {
  int block = (int)blockIdx.x;
  const bool first = block < a.wgs;
  if (!first) block -= a.wgs;
  const CacheRows rows = first ? a.rows : b.rows;
  const SliceWork sw = first ? a.sw : b.sw;
  slice_block<S, true>(c, rows, sw, first ? a.list : b.list, first ? a.keys : b.keys, block);
}

// ------------------------------------------------------------------ a row's cut
// NW waves per (row, head).  All keys wait in registers, 64 of the prefix's list or of the row's own to each (what these do not hold is read again
// in every pass).  The cut is looked for between the smallest and the largest key: a pass counts the keys before two probes, to either side of where a
// straight line through the counts at both ends has it (every third pass at thirds), until 64 keys are left, which are ranked; or a
// probe has exactly k before it; or only equal keys are left, whose places are then halved.  About three passes, six at most on scores of the usual kinds.
// (Halving alone took 13, one probe 7 and up to 17 -- the slowest row is what a launch takes.)  Counts are kept in the lanes and summed once a pass:
// one ballot a register needed three scalar instructions, which four SIMDs share (64 rows of 32 heads, 2048 + 400 keys: 83 us instead of 26).
// A row with more than k keys of its own has a list of the best of them, unless the caller's bound says that there are none; else they are
// read where they are.
constexpr int CUT_LIST = 1024, CUT_OWN = 512;  // keys that a wave holds, of the list and of the row's own
template <int NW>
__global__ __launch_bounds__(64 * NW) void prefix_cut_kernel(CacheRef c, PrefixArgs p) {
  constexpr int RC = CUT_LIST / 64, RO = CUT_OWN / 64;
  constexpr uint32_t NEAR = 64;  // keys that a wave ranks, a lane each
  __shared__ uint32_t sums[4][NW], n_near[NW];
  __shared__ unsigned long long near[NW][NEAR];  // key and place
  const int G = c.H_q / c.H_kv, idx = (int)(blockIdx.x >> 3), unit = (idx / G) * 8 + (int)(blockIdx.x & 7);
  if (unit >= p.own.n_rows * c.H_kv) return;
  const int r = unit / c.H_kv, g = unit - r * c.H_kv, h = g * G + idx % G, rh = r * c.H_q + h;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), l = tid & 63;
  const PrefixRow info = p.rows[r];
  const int k = p.own.k, n_pre = min(k, info.pre);
  const bool listed = p.listed && info.own > k;
  const int n_own = listed ? k : info.own;
  if (n_own <= 0) {
    if (tid == 0) p.cuts[rh] = {0u, -1, 0, 0};
    return;
  }
  const int32_t* pages = p.own.table + (size_t)info.req * c.max_pages;
  int32_t* list = p.list_own + (size_t)rh * p.own.kcap;
  const uint32_t* keys_own = p.keys_own + (size_t)rh * p.own.kcap;
  const size_t at_pre = ((size_t)max(info.prefix, 0) * c.H_q + h) * p.pre.kcap;
  const uint32_t* keys_pre = p.keys_pre + at_pre;
  const int first_pre = n_pre > 0 ? p.list_pre[at_pre] : 0;
  uint32_t kc[RC], ko[RO], id[RO];
  bool bad = first_pre < 0 || (listed && list[0] < 0);  // (a page is out of range: the list says so)
  auto place_of = [&](int u) { return (u * NW + w) * 64 + l; };
  // (all loads of four registers are on their way before the first is used: places behind the end read the last one)
  auto fetch_c = [&]() __attribute__((always_inline)) {
    static_for<RC / 4>([&](auto quad) __attribute__((always_inline)) {
      constexpr int U0 = 4 * decltype(quad)::value;
      static_for<4>([&](auto e) __attribute__((always_inline)) { kc[U0 + decltype(e)::value] = NO_KEY; });
      if (U0 * NW * 64 < n_pre)
        static_for<4>([&](auto e) __attribute__((always_inline)) {
          constexpr int X = U0 + decltype(e)::value;
          kc[X] = keys_pre[min(place_of(X), n_pre - 1)];
        });
    });
  };
  // slot of the own key at place j, of that page, and where its score is
  auto slot_of = [&](uint32_t page, int j) __attribute__((always_inline)) {
    const bool out = page >= (uint32_t)c.n_pages;
    bad |= out;
    return (out ? 0u : page << c.shift) | ((uint32_t)j & ((1u << c.shift) - 1u));
  };
  auto score_at = [&](uint32_t slot) __attribute__((always_inline)) {
    return reinterpret_cast<const float*>(cache_page(c, slot) + c.off_z) + ((size_t)h << c.shift) + cache_place(c, slot);
  };
  auto fetch_o = [&](int round) __attribute__((always_inline)) {
    auto each = [&](auto f) __attribute__((always_inline)) {  // f(index, place) of the registers that hold something, four at a time
      static_for<RO / 4>([&](auto quad) __attribute__((always_inline)) {
        constexpr int U0 = 4 * decltype(quad)::value;
        if ((round * RO + U0) * NW * 64 < n_own)
          static_for<4>([&](auto e) __attribute__((always_inline)) {
            constexpr int X = U0 + decltype(e)::value;
            f(std::integral_constant<int, X>{}, min(place_of(round * RO + X), n_own - 1));
          });
      });
    };
    static_for<RO>([&](auto u) __attribute__((always_inline)) {
      ko[decltype(u)::value] = NO_KEY;
      id[decltype(u)::value] = 0;
    });
    if (listed) {
      each([&](auto u, int j) __attribute__((always_inline)) {
        id[decltype(u)::value] = (uint32_t)list[j];
        ko[decltype(u)::value] = keys_own[j];
      });
    } else {
      each([&](auto u, int j) __attribute__((always_inline)) { id[decltype(u)::value] = (uint32_t)pages[j >> c.shift]; });
      each([&](auto u, int j) __attribute__((always_inline)) {
        constexpr int X = decltype(u)::value;
        id[X] = slot_of(id[X], j);
        ko[X] = __float_as_uint(*score_at(id[X]));
      });
      static_for<RO>([&](auto u) __attribute__((always_inline)) { ko[decltype(u)::value] = score_key(__uint_as_float(ko[decltype(u)::value])); });
    }
    static_for<RO>([&](auto u) __attribute__((always_inline)) {
      constexpr int X = decltype(u)::value;
      ko[X] = place_of(round * RO + X) < n_own ? ko[X] : NO_KEY;
    });
  };
  const bool selects = (long)n_pre + n_own > k;
  if (selects) fetch_c();  // (on their way while the pages of the row's own keys lead to their scores)
  fetch_o(0);
  if (selects)
    static_for<RC>([&](auto u) __attribute__((always_inline)) {
      constexpr int X = decltype(u)::value;
      kc[X] = place_of(X) < n_pre ? kc[X] : NO_KEY;
    });
  const int rounds = (n_own + 64 * NW * RO - 1) / (64 * NW * RO);
  if (!listed && rounds > 1)
    for (int j = tid; (long)j << c.shift < n_own; j += 64 * NW) bad |= (uint32_t)pages[j] >= (uint32_t)c.n_pages;
  // f(key, place in its list, whether that is the prefix's) for all of this wave's keys; what the registers do not hold is read again
  auto every = [&](auto f) __attribute__((always_inline)) {
    static_for<RC / 8>([&](auto eight) __attribute__((always_inline)) {
      constexpr int U0 = 8 * decltype(eight)::value;
      if (U0 * NW * 64 < n_pre)
        static_for<8>([&](auto e) __attribute__((always_inline)) { f(kc[U0 + decltype(e)::value], place_of(U0 + decltype(e)::value), true); });
    });
    static_for<RO / 8>([&](auto eight) __attribute__((always_inline)) {
      constexpr int U0 = 8 * decltype(eight)::value;
      if (U0 * NW * 64 < n_own)
        static_for<8>([&](auto e) __attribute__((always_inline)) { f(ko[U0 + decltype(e)::value], place_of(U0 + decltype(e)::value), false); });
    });
#pragma unroll 1
    for (int i0 = place_of(RC) - l; i0 < n_pre; i0 += NW * 64) {  // (all lanes stay: f may count over them)
      const uint32_t key = keys_pre[min(i0 + l, n_pre - 1)];
      f(i0 + l < n_pre ? key : NO_KEY, i0 + l, true);
    }
#pragma unroll 1
    for (int i0 = place_of(RO) - l; i0 < n_own; i0 += NW * 64) {
      const int i = min(i0 + l, n_own - 1);
      const uint32_t key = listed ? keys_own[i] : score_key(*score_at(slot_of((uint32_t)pages[i >> c.shift], i)));
      f(i0 + l < n_own ? key : NO_KEY, i0 + l, false);
    }
  };
  int turn = 0;
  auto over_waves = [&](uint32_t x, auto op) __attribute__((always_inline)) {
    if constexpr (NW > 1) {
      turn ^= 1;
      if (l == 0) sums[turn][w] = x;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < NW; i++) x = i == 0 ? sums[turn][0] : op(x, sums[turn][i]);
    }
    return (uint32_t)__builtin_amdgcn_readfirstlane((int)x);
  };
  const auto add = [](uint32_t a, uint32_t b) { return a + b; };
  uint32_t cut_key = NO_KEY;
  int cut_pre = -1, cut_own = -1;  // of the keys equal to cut_key, those up to these places are kept
  if (selects) {
    uint32_t least = NO_KEY, most = 0;
    every([&](uint32_t key, int, bool pre) __attribute__((always_inline)) {
      least = min(least, key);
      if (pre || n_pre < k) most = max(most, key + 1u);  // (k of the prefix: the worst of them bounds the cut; NO_KEY + 1 is 0)
    });
    least = last_lane(wave_scan(least, NO_KEY, [](uint32_t a, uint32_t b) { return min(a, b); }));
    most = last_lane(wave_scan(most, 0u, [](uint32_t a, uint32_t b) { return max(a, b); }));
    // fewer than k keys are before lo, at least k before hi
    uint32_t lo = over_waves(least, [](uint32_t a, uint32_t b) { return min(a, b); });
    uint32_t hi = over_waves(most, [](uint32_t a, uint32_t b) { return max(a, b); });
    uint32_t before_lo = 0, before_hi = NO_KEY, first = hi - min((hi - lo) / 16, hi - lo - 1u), second = hi;
    bool found = false;
    for (int step = 1;; step++) {
      uint32_t n = 0, m = 0;
      every([&](uint32_t key, int, bool) __attribute__((always_inline)) {
        n += key < first;
        m += key < second;
      });
      n = last_lane(wave_scan(n, 0u, add));
      m = last_lane(wave_scan(m, 0u, add));
      turn ^= 1;
      if (l == 0) {
        sums[turn][w] = n;
        sums[2 + turn][w] = m;
      }
      __syncthreads();
      n = m = 0;
#pragma unroll
      for (int i = 0; i < NW; i++) {
        n += sums[turn][i];
        m += sums[2 + turn][i];
      }
      n = (uint32_t)__builtin_amdgcn_readfirstlane((int)n);
      m = (uint32_t)__builtin_amdgcn_readfirstlane((int)m);
      found = n == (uint32_t)k || m == (uint32_t)k;
      if (found) {  // exactly the keys before it
        cut_key = n == (uint32_t)k ? first : second;
        break;
      }
      if (n > (uint32_t)k) {
        hi = first;
        before_hi = n;
      } else {
        const bool beyond = m < (uint32_t)k;
        lo = beyond ? second : first;
        before_lo = beyond ? m : n;
        hi = beyond ? hi : second;
        before_hi = beyond ? before_hi : m;
      }
      const uint32_t width = hi - lo, left = before_hi - before_lo;
      if (width <= 1u || left <= NEAR) break;
      const float each = __builtin_amdgcn_rcpf((float)left), share = (float)((uint32_t)k - before_lo) * each;
      const float off = step % 3 ? (__builtin_amdgcn_sqrtf((float)left) + 1.f) * each : 1.f / 6.f, at = step % 3 ? share : 0.5f;
      auto probe = [&](float x) {
        const uint32_t ahead = (uint32_t)((float)width * fmaxf(x, 0.f));
        return (uint32_t)__builtin_amdgcn_readfirstlane((int)(lo + min(max(ahead, 1u), width - 1u)));
      };
      first = probe(at - off);
      second = probe(at + off);
    }
    const uint32_t need = (uint32_t)k - before_lo, left = before_hi - before_lo;  // the need-th of the left ones is the last that is kept
    if (!found && left <= NEAR) {
      // each wave lists its own of them; a lane then takes one, and counts those before it
      uint32_t mine = 0;
      every([&](uint32_t key, int place, bool pre) __attribute__((always_inline)) {
        const unsigned long long in = __ballot(key - lo < hi - lo);
        if (in) {
          if (key - lo < hi - lo) near[w][mine + lanes_before(in)] = (unsigned long long)key << 32 | ((uint32_t)place + (pre ? 0u : (uint32_t)n_pre));
          mine += (uint32_t)__popcll(in);
        }
      });
      if (l == 0) n_near[w] = mine;
      __syncthreads();
      unsigned long long one = ~0ull;
      uint32_t at = (uint32_t)l, rank = 0;
#pragma unroll
      for (int i = 0; i < NW; i++) {
        const uint32_t have = n_near[i];
        if (at < have) one = near[i][at];
        at = at < have ? 1u << 30 : at - have;  // (taken, or further on)
      }
#pragma unroll
      for (int i = 0; i < NW; i++) {
        const uint32_t have = n_near[i];
        for (uint32_t j = 0; j < have; j += 4) {
          unsigned long long other[4];
#pragma unroll
          for (int e = 0; e < 4; e++) other[e] = near[i][min(j + e, NEAR - 1u)];
#pragma unroll
          for (int e = 0; e < 4; e++) rank += j + e < have && other[e] < one;
        }
      }
      const int last = (int)__builtin_ctzll(__ballot(rank == need - 1u && one != ~0ull));
      cut_key = (uint32_t)__builtin_amdgcn_readlane((int)(one >> 32), last);
      const int place = __builtin_amdgcn_readlane((int)(uint32_t)one, last);
      cut_pre = min(place, n_pre - 1);
      cut_own = place - n_pre;
    } else if (!found) {  // keys equal to lo are on both sides: the prefix's are first
      cut_key = lo;
      long from = 0, upto = (long)n_pre + n_own;  // fewer than `need` of them are before place `from`, at least as many before `upto`
      while (upto - from > 1) {
        const long middle = (from + upto) / 2;
        const int before_pre = (int)min(middle, (long)n_pre), before_own = (int)(middle - before_pre);
        uint32_t n = 0;
        every([&](uint32_t key, int place, bool pre) __attribute__((always_inline)) { n += (key == lo) & (place < (pre ? before_pre : before_own)); });
        if (over_waves(last_lane(wave_scan(n, 0u, add)), add) < need) from = middle; else upto = middle;
      }
      cut_pre = (int)min(upto, (long)n_pre) - 1;
      cut_own = (int)(upto - n_pre) - 1;
    }
  }
  const bool gone = over_waves(__ballot(bad) ? 1u : 0u, [](uint32_t a, uint32_t b) { return a | b; }) != 0;
  // the slots of its own keys that are kept, wave by wave behind one another (all are in registers before one is written)
  uint32_t total = 0;
#pragma unroll 1
  for (int round = 0; round < rounds && !gone; round++) {
    if (round) fetch_o(round);
    uint32_t mine = 0;
    unsigned long long kept[RO];
    static_for<RO>([&](auto u) __attribute__((always_inline)) {
      constexpr int X = decltype(u)::value;
      kept[X] = __ballot(ko[X] < cut_key || (ko[X] == cut_key && ko[X] != NO_KEY && place_of(round * RO + X) <= cut_own));
      mine += (uint32_t)__popcll(kept[X]);
    });
    uint32_t at = total, all = mine;
    if constexpr (NW > 1) {
      turn ^= 1;
      if (l == 0) sums[turn][w] = mine;
      __syncthreads();
      all = 0;
#pragma unroll
      for (int i = 0; i < NW; i++) {
        at += i < w ? sums[turn][i] : 0u;
        all += sums[turn][i];
      }
    }
    static_for<RO>([&](auto u) __attribute__((always_inline)) {
      constexpr int X = decltype(u)::value;
      const uint32_t to = at + lanes_before(kept[X]);
      if (kept[X] >> l & 1 && to < (uint32_t)p.own.kcap) list[to] = (int32_t)id[X];  // (there are never more than k)
      at += (uint32_t)__popcll(kept[X]);
    });
    total += all;
  }
  if (tid == 0) p.cuts[rh] = {cut_key, cut_pre, gone ? -1 : (int)total, 0};
}

// ------------------------------------------------------------------ the prefix, for 32 rows at a time
// Two values, x and y, as sums of bf16 ones: each term is what is left, rounded.
template <int N> struct Terms {
  bf16x8 t[N];
  __device__ __forceinline__ void split(int i, float x, float y) {  // (i even)
#pragma unroll
    for (int n = 0; n < N; n++) {
      typedef float f32x2 __attribute__((ext_vector_type(2)));
      const bf16x2 both = __builtin_convertvector((f32x2){x, y}, bf16x2);
      t[n][i] = both[0];
      t[n][i + 1] = both[1];
      if (n + 1 < N) {
        const uint32_t bits = __builtin_bit_cast(uint32_t, both);
        x -= __uint_as_float(bits << 16);
        y -= __uint_as_float(bits & 0xffff0000u);
      }
    }
  }
};

// Joins the weighted sums of parts with references of their own.
struct Joined {
  float M, num, den;
  __device__ __forceinline__ void add(float m, float n, float d) {
    const float top = fmaxf(M, m), ref = top == -INFINITY ? 0.f : top, a = weight(M, ref), b = weight(m, ref);
    M = top;
    num = num * a + n * b;
    den = den * a + d * b;
  }
};

// One workgroup per (tile of 32 rows, head, part of the list); a wave takes 32 listed keys at a time.  Their K rows go from memory to the A operand
// of S^T = K Q^T (a lane has half a row; which channel is which product's does not matter, as long as Q has them in the same places), the
// rows' queries are the B operand.  A row is then a column of S^T, in two lanes, which mask it by the row's cut and form the weights with a
// reference of the row's own.  Its weights are the B operand of O^T += V^T P^T as they lie; V goes through LDS to be transposed.  What the cache
// holds is exact in bf16; the weights, and fp32 queries, are sums of bf16 terms (two terms of a weight: off by 2^-16 of it; one term, 2^-8,
// would show beside the rounding of the output; three for fp32, 2^-24).
// What bounds it is the chain of the list, the rows of the keys and the products of a step or two per wave, and the join at the end: 64 rows of 32
// heads, window 2048 of 16384, 14 us (2.1 GFLOP, a row's 2048 keys gathered twice instead of 64 times).
template <typename TQ, int D, int NW>
__global__ __launch_bounds__(64 * NW) void prefix_tile_kernel(CacheRef c, PrefixArgs p, const TQ* __restrict__ q, long q_stride, float scale) {
  constexpr bool F32 = sizeof(TQ) == 4;
  constexpr int KS = D / 16, CB = D / 32, NQ = D / 64, NTQ = F32 ? 3 : 1, NTP = F32 ? 3 : 2, PITCH = D + 4;
  constexpr int TILE_BYTES = 32 * D * 2, OUT_BYTES = 32 * PITCH * 4;
  constexpr int WAVE_BYTES = TILE_BYTES > OUT_BYTES ? TILE_BYTES : OUT_BYTES;
  __shared__ __align__(16) char mem[NW * WAVE_BYTES];  // a V tile of each wave; in the end its sums
  __shared__ __align__(16) uint32_t s_key[NW][32];
  __shared__ __align__(16) float s_z[NW][32];
  __shared__ __align__(16) float ml[NW][2][32];
  __shared__ __align__(16) uint32_t s_nan[NW][32];  // blocks of a key's V that are no numbers; in the end, of a row's sums
  __shared__ int tile_row[32];
  const int G = c.H_q / c.H_kv, idx = (int)(blockIdx.x >> 3), unit = (idx / G) * 8 + (int)(blockIdx.x & 7);
  const int per = p.max_tiles * c.H_kv, sp = unit / per, tg = unit - sp * per;
  if (sp >= p.nsplit) return;
  const int t = tg / c.H_kv, g = tg - t * c.H_kv, h = g * G + idx % G;
  const PrefixTile* tp = p.tiles + t;
  const int listed_row = tp->rows[threadIdx.x & 31];  // (with the tile's head, not behind it)
  const struct { int prefix, count, pre; } tile = {tp->prefix, tp->count, tp->pre};
  if (tile.count == 0) return;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), l = tid & 63, n = l & 31, hh = l >> 5;
  const int n_keys = min(p.pre.k, tile.pre), step = p.nsplit * NW * 32;
  const size_t at_pre = ((size_t)tile.prefix * c.H_q + h) * p.pre.kcap;
  const int32_t* list = p.list_pre + at_pre;
  const uint32_t* keys = p.keys_pre + at_pre;
  uint16_t* vt = reinterpret_cast<uint16_t*>(mem + w * WAVE_BYTES);
  int j0 = (sp * NW + w) * 32;
  uint32_t id = (uint32_t)list[min(j0 + n, n_keys - 1)], key = keys[min(j0 + n, n_keys - 1)];
  const int first_row = __builtin_amdgcn_readfirstlane(listed_row);  // (with all lanes there: in a branch it would be the first of that branch)
  const int row = n < tile.count ? listed_row : first_row;
  if (tid < 32) tile_row[tid] = row;
  struct Raw {
    uint4 k[NQ], v[NQ];
    uint32_t kb, vb, key;
  };
  const uint32_t page_bytes = (uint32_t)c.page_bytes;
  auto load_bytes = [&](const char* src) -> uint32_t {
    if constexpr (D == 256) return *reinterpret_cast<const uint32_t*>(src);
    if constexpr (D == 128) return *reinterpret_cast<const uint16_t*>(src);
    return *reinterpret_cast<const uint8_t*>(src);
  };
  // the keys at j0, and the ids of those behind them
  auto fetch = [&](Raw& x) {
    const bool there = j0 + n < n_keys && id < c.n_slots;
    const uint32_t slot = there ? id : 0u, place = cache_place(c, slot), at = ((uint32_t)g << c.shift) + place;
    const char* page = c.pages + (unsigned long long)(slot >> c.shift) * page_bytes;
    const uint4* codes = reinterpret_cast<const uint4*>(page + at * D) + NQ * hh;
    const char* bytes = page + (c.off_scales + at * (D / 16) + hh * (D / 64));
#pragma unroll
    for (int i = 0; i < NQ; i++) {
      x.k[i] = codes[i];
      x.v[i] = codes[i + 2 * NQ];
    }
    x.kb = load_bytes(bytes);
    x.vb = load_bytes(bytes + D / 32);
    x.key = there ? key : NO_KEY;
    j0 += step;
    id = (uint32_t)list[min(j0 + n, n_keys - 1)];
    key = keys[min(j0 + n, n_keys - 1)];
  };
  Raw cur;
  const bool any = j0 < n_keys;
  int at0 = j0;
  if (any) fetch(cur);
  const Cut cut = n < tile.count ? p.cuts[(size_t)row * c.H_q + h] : Cut{0u, -1, 0, 0};
  // channel 8 s + e of this half of the row: the lane's part of product s
  // (fp32 queries are split where they are used: kept, their three terms took 192 registers at 256 channels, and 87 spilled -- 17 rows of 16
  // heads, window 1024: the call 46.8 -> 37.9; 64 rows 76.0 -> 66.3, of 128 channels 64.5 -> 63.9, of 64 47.0 -> 46.3)
  const TQ* src = q + (size_t)row * q_stride + (size_t)h * D + hh * (D / 2);
  auto query = [&](int s) __attribute__((always_inline)) {
    Terms<NTQ> x;
    if constexpr (F32) {
      const float4 a = reinterpret_cast<const float4*>(src + 8 * s)[0], b = reinterpret_cast<const float4*>(src + 8 * s)[1];
      x.split(0, a.x, a.y);
      x.split(2, a.z, a.w);
      x.split(4, b.x, b.y);
      x.split(6, b.z, b.w);
    } else {
      x.t[0] = *reinterpret_cast<const bf16x8*>(src + 8 * s);
    }
    return x;
  };
  Terms<NTQ> qf[F32 ? 1 : KS];
  if constexpr (!F32) {
#pragma unroll
    for (int s = 0; s < KS; s++) qf[s] = query(s);
  }
  FragOffsets<D> fo;
  fo.init(l);
  float m = -INFINITY, ref = 0.f, limit = -INFINITY, lsum = 0.f;
  uint32_t nan = 0;
  f32x16 acc[CB];
#pragma unroll
  for (int b = 0; b < CB; b++)
#pragma unroll
    for (int v = 0; v < 16; v++) acc[b][v] = 0.f;
  while (at0 < n_keys) {
    Raw next;
    if (j0 < n_keys) fetch(next); else j0 += step;
    const float z = key_value(cur.key);
    const bool counts = cur.key != NO_KEY && z != -INFINITY;
    // V to LDS, a half row of a lane; blocks that are no numbers, and keys that count for nothing, as zeros
    uint32_t nans = 0;
#pragma unroll
    for (int b = 0; b < NQ; b++) {
      const uint32_t byte = cur.vb >> (8 * b) & 255u;
      nans |= byte == 255u && counts ? 1u << (NQ * hh + b) : 0u;
      const float sc = counts && byte != 255u ? mx_scale(byte) : 0.f;
      const uint32_t code[4] = {cur.v[b].x, cur.v[b].y, cur.v[b].z, cur.v[b].w};
#pragma unroll
      for (int i = 0; i < 4; i++) {
        uint4 out;
        out.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[i], sc, 0));
        out.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[i], sc, 1));
        out.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[i], sc, 2));
        out.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[i], sc, 3));
        *reinterpret_cast<uint4*>(vt + TileLayout<D>::off(n, (D / 16) * hh + 4 * b + i)) = out;
      }
    }
    if (hh == 0) {
      s_key[w][n] = counts ? cur.key : NO_KEY;  // (one that counts for nothing is behind every cut)
      s_z[w][n] = z;
    }
    const bool some_nan = __ballot(nans != 0) != 0;
    if (some_nan) {
      const uint32_t other = __builtin_amdgcn_permlane32_swap(nans, nans, false, false)[0] | __builtin_amdgcn_permlane32_swap(nans, nans, false, false)[1];
      if (hh == 0) s_nan[w][n] = other;
    }
    asm volatile("" ::: "memory");  // (a wave's LDS accesses are in order: it reads what it wrote)
    f32x16 s;
#pragma unroll
    for (int v = 0; v < 16; v++) s[v] = 0.f;
#pragma unroll
    for (int b = 0; b < NQ; b++) {
      const float sc = mx_scale(cur.kb >> (8 * b) & 255u);
      const uint32_t code[4] = {cur.k[b].x, cur.k[b].y, cur.k[b].z, cur.k[b].w};
#pragma unroll
      for (int i = 0; i < 4; i++) {
        uint4 a;
        a.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[i], sc, 0));
        a.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[i], sc, 1));
        a.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[i], sc, 2));
        a.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[i], sc, 3));
        const Terms<NTQ> qn = F32 ? query(4 * b + i) : qf[F32 ? 0 : 4 * b + i];
#pragma unroll
        for (int x = NTQ - 1; x >= 0; x--) s = mfma32(__builtin_bit_cast(bf16x8, a), qn.t[x], s);
      }
    }
    // this lane's keys: 8 (v / 4) + 4 hh + v % 4; the row keeps those before its cut, and where it falls among equal ones in this tile, those
    // up to its place
    const uint32_t bound = cut.last >= at0 + 31 ? cut.key + 1u : cut.key;
    const bool among = __ballot(cut.last >= at0 && cut.last < at0 + 31) != 0;
    float top = -INFINITY;
#pragma unroll
    for (int b = 0; b < 4; b++) {
      const uint4 kk = *reinterpret_cast<const uint4*>(&s_key[w][8 * b + 4 * hh]);
      const float4 zz = *reinterpret_cast<const float4*>(&s_z[w][8 * b + 4 * hh]);
      const uint32_t ks[4] = {kk.x, kk.y, kk.z, kk.w};
      const float zs[4] = {zz.x, zz.y, zz.z, zz.w};
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const float x = fmaf(s[4 * b + e], scale, zs[e]);
        bool keep = ks[e] < bound;
        if (among) keep = keep | ((ks[e] == cut.key) & (at0 + 8 * b + 4 * hh + e <= cut.last) & (ks[e] != NO_KEY));
        s[4 * b + e] = keep ? x : -INFINITY;
        top = fmaxf(top, s[4 * b + e]);
      }
    }
    if (some_nan) {
#pragma unroll
      for (int b = 0; b < 4; b++) {
        const uint4 nn = *reinterpret_cast<const uint4*>(&s_nan[w][8 * b + 4 * hh]);
        nan |= (s[4 * b] == -INFINITY ? 0u : nn.x) | (s[4 * b + 1] == -INFINITY ? 0u : nn.y) | (s[4 * b + 2] == -INFINITY ? 0u : nn.z) |
               (s[4 * b + 3] == -INFINITY ? 0u : nn.w);
      }
    }
    top = half_swap_max(top);
    if (__ballot(top > limit)) {
      const float now = top > limit ? top : m, alpha = top > limit ? weight(m, now) : 1.f;
      ref = top > limit ? now : ref;
      limit = top > limit ? now + 5.f : limit;
      m = now;
      lsum *= alpha;
#pragma unroll
      for (int b = 0; b < CB; b++)
#pragma unroll
        for (int v = 0; v < 16; v++) acc[b][v] *= alpha;
    }
    Terms<NTP> pf[2];
#pragma unroll
    for (int v = 0; v < 16; v += 2) {
      const float pv = weight(s[v], ref), pw = weight(s[v + 1], ref);
      lsum += pv + pw;
      pf[v / 8].split(v % 8, pv, pw);
    }
#pragma unroll
    for (int x = 0; x < 2; x++)
#pragma unroll
      for (int b = 0; b < CB; b++) {
        const bf16x8 vf = fo.tr_frag(vt, 16 * x, b);
#pragma unroll
        for (int y = NTP - 1; y >= 0; y--) acc[b] = mfma32(vf, pf[x].t[y], acc[b]);
      }
    asm volatile("" ::: "memory");
    cur = next;
    at0 += step;
  }
  lsum = half_swap_sum(lsum);
  {
    const auto both = __builtin_amdgcn_permlane32_swap(nan, nan, false, false);
    nan = both[0] | both[1];
  }
  if (hh == 0) {
    ml[w][0][n] = m;
    ml[w][1][n] = lsum;
    s_nan[w][n] = nan;
  }
  asm volatile("" ::: "memory");
  float* out = reinterpret_cast<float*>(vt) + n * PITCH;  // (over the wave's own tile, which it has read)
#pragma unroll
  for (int b = 0; b < CB; b++)
#pragma unroll
    for (int v = 0; v < 16; v += 4)
      *reinterpret_cast<float4*>(out + 32 * b + 2 * v + 4 * hh) = make_float4(acc[b][v], acc[b][v + 1], acc[b][v + 2], acc[b][v + 3]);
  __syncthreads();
  // four channels of a row to a thread
  constexpr int QUADS = D / 4, PER_PASS = 64 * NW / QUADS;
  const int ch = tid % QUADS * 4;
  for (int rr = tid / QUADS; rr < tile.count; rr += PER_PASS) {
    const size_t rh = (size_t)tile_row[rr] * c.H_q + h;
    float M = -INFINITY, den = 0.f, num[4] = {0.f, 0.f, 0.f, 0.f};
    uint32_t nans = 0;
#pragma unroll
    for (int x = 0; x < NW; x++) M = fmaxf(M, ml[x][0][rr]);
    const float mr = M == -INFINITY ? 0.f : M;
#pragma unroll
    for (int x = 0; x < NW; x++) {
      const float4 v = *reinterpret_cast<const float4*>(mem + x * WAVE_BYTES + (rr * PITCH + ch) * 4);
      const float w8 = weight(ml[x][0][rr], mr);
      den = fmaf(ml[x][1][rr], w8, den);
      num[0] = fmaf(v.x, w8, num[0]);
      num[1] = fmaf(v.y, w8, num[1]);
      num[2] = fmaf(v.z, w8, num[2]);
      num[3] = fmaf(v.w, w8, num[3]);
      nans |= s_nan[x][rr];
    }
    if (nans >> (ch / 32) & 1) num[0] = num[1] = num[2] = num[3] = NAN;
    float* to = p.part + (rh * p.nsplit + sp) * (D + 4);
    *reinterpret_cast<float4*>(to + ch) = make_float4(num[0], num[1], num[2], num[3]);
    if (ch == 0) *reinterpret_cast<float2*>(to + D) = make_float2(M, den);
  }
}

// ------------------------------------------------------------------ a row's own keys, and all of it together
// NW waves per (row, head), 32 of the listed keys to a wave at a time, in the form of cache_attend_kernel.  The parts of the prefix are
// requested first and joined last.  A chain of loads too: 2048 (row, head)s of about 50 kept keys each 9.2 us, 128 of 38 4.4.
template <typename TQ, int D, int NW>
__global__ __launch_bounds__(64 * NW) void prefix_own_kernel(CacheRef c, PrefixArgs p, const TQ* __restrict__ q, long q_stride,
                                                             TQ* __restrict__ o, float* __restrict__ lse, float scale) {
  constexpr int LPG = D / 32, NG = 64 / LPG, KEYS = 32, U = KEYS / NG, PER = (D + 64 * NW - 1) / (64 * NW), PARTS = 4;
  __shared__ __align__(16) float mo[NW][D];
  __shared__ float ml[NW][2];
  const int G = c.H_q / c.H_kv, idx = (int)(blockIdx.x >> 3), unit = (idx / G) * 8 + (int)(blockIdx.x & 7);
  if (unit >= p.own.n_rows * c.H_kv) return;
  const int r = unit / c.H_kv, g = unit - r * c.H_kv, h = g * G + idx % G, rh = r * c.H_q + h;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), l = tid & 63, sub = l % LPG, grp = l / LPG;
  const int32_t* list = p.list_own + (size_t)rh * p.own.kcap;
  uint32_t id[U];
  int i0 = w * KEYS;
#pragma unroll
  for (int u = 0; u < U; u++) id[u] = (uint32_t)list[min(i0 + u * NG + grp, p.own.kcap - 1)];  // (before their number is known)
  const float* parts = p.part + (size_t)rh * p.nsplit * (D + 4);
  float part_m[PARTS], part_den[PARTS], part_num[PARTS][PER];
  const int n_parts = p.pre.n_rows ? p.nsplit : 0;
  auto request = [&](int first) __attribute__((always_inline)) {
    if (n_parts)
#pragma unroll
      for (int i = 0; i < PARTS; i++) {
        const float* x = parts + (size_t)min(first + i, n_parts - 1) * (D + 4);
        part_m[i] = x[D];
        part_den[i] = x[D + 1];
#pragma unroll
        for (int e = 0; e < PER; e++) part_num[i][e] = x[min(tid + e * 64 * NW, D - 1)];
      }
  };
  request(0);
  Query<TQ> qv;
  qv.load(q + (size_t)r * q_stride + (size_t)h * D + 32 * sub);
  const int count = p.cuts[rh].count, prefix = p.rows[r].prefix;
  // Attention to the kept ones, each wave to its own; the form of cache_attend_kernel.
  const uint32_t k_off = ((uint32_t)g << c.shift) * D + 16 * sub, z_off = c.off_z + ((uint32_t)h << c.shift) * 4;
  const uint32_t b_off = c.off_scales + ((uint32_t)g << c.shift) * (D / 16) + sub, page_bytes = (uint32_t)c.page_bytes;
  float m = -INFINITY, ref = 0.f, limit = -INFINITY, lsum = 0.f, acc[32];
#pragma unroll
  for (int e = 0; e < 32; e++) acc[e] = 0.f;
  struct Keys {
    uint4 kr[U], vr[U];
    uint32_t kb[U], vb[U];
    float s[U];
    uint32_t there;
  };
  auto take = [&](Keys& x) __attribute__((always_inline)) {
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
  auto fetch = [&](Keys& x) __attribute__((always_inline)) {  // the keys at i0 (in id), and the ids of those behind them
    x.there = 0;
#pragma unroll
    for (int u = 0; u < U; u++) {
      const bool there = i0 + u * NG + grp < count && id[u] < c.n_slots;
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
    i0 += NW * KEYS;
#pragma unroll
    for (int u = 0; u < U; u++) id[u] = (uint32_t)list[min(i0 + u * NG + grp, p.own.kcap - 1)];
  };
  if (i0 < count) {
    Keys even, odd;
    fetch(even);
#pragma unroll 1
    for (;;) {
      const bool more = i0 < count;
      if (more) fetch(odd);
      take(even);
      if (!more) break;
      const bool again = i0 < count;
      if (again) fetch(even);
      take(odd);
      if (!again) break;
    }
  }
  lsum = over_groups<LPG>(lsum, [](float a, float b) { return a + b; });
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
  if ((l & 15) < LPG) {
    float4* to = reinterpret_cast<float4*>(&mo[w][32 * sub + 16 * (l >> 5) + 8 * (l >> 4 & 1)]);
    to[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
    to[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
  }
  if (l == 0) {
    ml[w][0] = m;
    ml[w][1] = lsum;
  }
  __syncthreads();
  float M = -INFINITY, den = 0.f;
#pragma unroll
  for (int i = 0; i < NW; i++) M = fmaxf(M, ml[i][0]);
  const float mr = M == -INFINITY ? 0.f : M;
#pragma unroll
  for (int i = 0; i < NW; i++) den = fmaf(ml[i][1], weight(ml[i][0], mr), den);
  Joined j[PER];
#pragma unroll
  for (int e = 0; e < PER; e++) {
    float num = 0.f;
#pragma unroll
    for (int i = 0; i < NW; i++) num = fmaf(mo[i][min(tid + e * 64 * NW, D - 1)], weight(ml[i][0], mr), num);
    j[e] = {M, num, den};
  }
  if (prefix >= 0)
    for (int first = 0; first < n_parts; first += PARTS) {
      if (first) request(first);
#pragma unroll
      for (int i = 0; i < PARTS; i++)
        if (first + i < n_parts) {
#pragma unroll
          for (int e = 0; e < PER; e++) j[e].add(part_m[i], part_num[i][e], part_den[i]);
        }
    }
#pragma unroll
  for (int e = 0; e < PER; e++) {
    const int t = tid + e * 64 * NW;
    if (t >= D) break;
    const bool none = count < 0 || j[e].den == 0.f;  // (a page is out of range, or no key took part)
    o[(size_t)rh * D + t] = TQ(none ? 0.f : j[e].num / j[e].den);
    if (t == 0) lse[(size_t)h * p.own.n_rows + r] = none ? -INFINITY : fmaf(__builtin_amdgcn_logf(j[e].den), LN2, j[e].M);
  }
}

// ------------------------------------------------------------------ host side
struct PrefixWork {
  size_t off_rows, off_tiles, off_list_pre, off_keys_pre, off_list_own, off_keys_own, off_cuts, off_part, total;
  SelectWork pre, own;
  bool listed;
  int max_tiles, nsplit;
  long own_bound;  // on a row's own keys
};
// A row of at most so many keys of its own needs no list of the best of them for its cut (40 requests x 5 rows of 500 keys, window 512, 16
// heads: the lists' launch 13 -> 21 us with them).
constexpr int OWN_DIRECT = 2048;
constexpr int tile_waves(int d) { return d == 256 ? 4 : 8; }
static PrefixWork prefix_work(const dma_cache_shape& s, int n_rows, int k, int n_prefixes, int max_prefix) {
  const int kcap = list_length(s, k);
  const long cap = (long)s.max_pages * s.page_size;
  const size_t pairs = (size_t)n_rows * s.H_q, pre_pairs = (size_t)n_prefixes * s.H_q;
  PrefixWork wk = {};
  auto take = [&](size_t bytes) { size_t at = wk.total; wk.total = align_up(at + bytes, 256); return at; };
  wk.own_bound = s.max_len > 0 && s.max_len < cap ? s.max_len : cap;
  wk.listed = wk.own_bound > (k > OWN_DIRECT ? k : OWN_DIRECT);
  const long groups = n_prefixes < n_rows ? n_prefixes : n_rows;
  wk.max_tiles = n_prefixes ? (int)((n_rows + (TILE_ROWS - 1) * groups) / TILE_ROWS) : 0;
  // parts of the lists: so many that every compute unit has one, as long as a wave has a step to take (one part: 64 rows x 32 heads, window 2048,
  // 55.9 -> 67.9 us, 17 x 16 of 256 channels in fp32 46.5 -> 87.9)
  const long per = 32 * tile_waves(s.d), most = (kcap + per - 1) / per, want = wk.max_tiles ? CUS / ((long)wk.max_tiles * s.H_q) : 1;
  wk.nsplit = (int)(want < 1 ? 1 : want > most ? most : want);
  wk.off_rows = take((size_t)n_rows * sizeof(PrefixRow));
  wk.off_tiles = take((size_t)wk.max_tiles * sizeof(PrefixTile));
  wk.off_cuts = take(pairs * sizeof(Cut));
  // (there are at least n_rows / 32 tiles, so several parts of each pair are at most 32 * CUS: room that never is less for more rows)
  const size_t parts = pairs * most < TILE_ROWS * CUS ? pairs * most : pairs > TILE_ROWS * CUS ? pairs : TILE_ROWS * CUS;
  wk.off_part = take(n_prefixes ? parts * (s.d + 4) * 4 : 0);
  wk.off_list_pre = take(pre_pairs * kcap * 4);
  wk.off_keys_pre = take(pre_pairs * kcap * 4);
  wk.off_list_own = take(pairs * kcap * 4);
  wk.off_keys_own = take(wk.listed ? pairs * kcap * 4 : 0);
  if (n_prefixes) wk.pre = select_work(s, pre_pairs, kcap, max_prefix, wk.total);
  if (wk.listed) wk.own = select_work(s, pairs, kcap, s.max_len, wk.total);
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
  const PrefixArgs p = {{table, row_req, row_len, n_rows, k, kcap}, {table, prefix_req, prefix_len, n_prefixes, k, kcap}, req_prefix,
                        (PrefixRow*)(base + wk.off_rows), (PrefixTile*)(base + wk.off_tiles),
                        (int32_t*)(base + wk.off_list_pre), (int32_t*)(base + wk.off_list_own), (uint32_t*)(base + wk.off_keys_pre),
                        (uint32_t*)(base + wk.off_keys_own), (Cut*)(base + wk.off_cuts), (float*)(base + wk.off_part), wk.max_tiles, wk.nsplit, wk.listed};
  const int pairs = n_rows * s.H_q;
  // the lists: prefixes first, rows behind them.  A set without slices has no share of what slices tell each other: all of its pairs
  // are in the first launch.  One with slices goes through that room in as many launches as it takes.
  auto set_of = [&](const CacheRows& rows, const SelectWork& w, int32_t* list, uint32_t* keys) {
    return SelectSet{rows, {(uint2*)(base + w.off_counts), (uint2*)(base + w.off_listed), (uint4*)(base + w.off_bounds), w.room, w.parts, 0, 0},
                     list, keys, 0};
  };
  SelectSet a = set_of(p.pre, wk.pre, p.list_pre, p.keys_pre), b = set_of(p.own, wk.own, p.list_own, p.keys_own);
  const int pre_pairs = n_prefixes * s.H_q, own_pairs = wk.listed ? pairs : 0;
  const bool sliced = wk.pre.parts > 0 || wk.own.parts > 0;
  auto select = [&](auto width) {
    constexpr int S = decltype(width)::value;
    auto share = [](SelectSet& x, int all, int per) {  // pairs of this launch
      const int left = all - x.sw.first;
      x.sw.pairs = x.sw.parts && left > per ? per : left;
      x.wgs = x.sw.pairs * (x.sw.parts ? x.sw.parts : 1);
    };
    for (bool group = true;; group = false) {
      share(a, pre_pairs, wk.pre.pairs);
      share(b, own_pairs, wk.own.pairs);
      const unsigned wgs = (unsigned)(a.wgs + b.wgs);
      if (!sliced) prefix_select_kernel<S, false, true><<<wgs + 1, 512, 0, st>>>(c, p, a, b);
      else if (group) prefix_select_kernel<S, true, true><<<wgs + 1, 512, 0, st>>>(c, p, a, b);
      else prefix_select_kernel<S, true, false><<<wgs, 512, 0, st>>>(c, p, a, b);
      SelectSet a2 = a, b2 = b;
      if (!a.sw.parts) a2.wgs = 0;
      if (!b.sw.parts) b2.wgs = 0;
      if (a2.wgs + b2.wgs) prefix_slice_kernel<S><<<(unsigned)(a2.wgs + b2.wgs), 512, 0, st>>>(c, a2, b2);
      a.sw.first += a.sw.pairs;
      b.sw.first += b.sw.pairs;
      if (a.sw.first >= pre_pairs && b.sw.first >= own_pairs) break;
    }
  };
  if (s.page_size >= 64) select(std::integral_constant<int, 1>{});
  else if (s.page_size == 32) select(std::integral_constant<int, 2>{});
  else select(std::integral_constant<int, 4>{});
  if (hipGetLastError() != hipSuccess) return DMA_EHIP;
  const int G = s.H_q / s.H_kv;
  const unsigned grid = (unsigned)(((long)n_rows * s.H_kv + 7) / 8 * 8 * G);
  // Waves of a (row, head) pair: two where there are many pairs, more where there are few.  Whole calls, us, two / four: 2048 pairs (64 rows,
  // window 2048 of 16384 + 400 keys) 55.9 / 64.0, 3200 60.2 / 69.7, 272 (window 1024 of 4096 + 123) 46.5 / 46.6, 256 (window 4096, 1000 +
  // 2000) 57.6 / 39.2, 32 (window 4096, 9000 + 9000) 99.8 / 59.2.  Eight for the attention of few pairs: 256 39.9 -> 37.0, 32 59.3 -> 57.5, the
  // shortest the same; for the cut only where four do not hold a row's keys: 57.5 -> 48.9, but 43.2 -> 44.6 where they do.
  const bool many = pairs >= 4 * CUS, few = pairs <= CUS;
  if (many) prefix_cut_kernel<2><<<grid, 128, 0, st>>>(c, p);
  else if (few && (kcap > CUT_LIST * 4 || wk.own_bound > CUT_OWN * 4)) prefix_cut_kernel<8><<<grid, 512, 0, st>>>(c, p);
  else prefix_cut_kernel<4><<<grid, 256, 0, st>>>(c, p);
  auto go = [&](auto t, auto width) {
    using T = std::remove_pointer_t<decltype(t)>;
    constexpr int D = decltype(width)::value, NW = tile_waves(D);
    if (n_prefixes) {
      const unsigned tiles = (unsigned)(((long)wk.max_tiles * s.H_kv * wk.nsplit + 7) / 8 * 8 * G);
      prefix_tile_kernel<T, D, NW><<<tiles, 64 * NW, 0, st>>>(c, p, (const T*)q, q_stride, scale);
    }
    if (many) prefix_own_kernel<T, D, 2><<<grid, 128, 0, st>>>(c, p, (const T*)q, q_stride, (T*)o, lse, scale);
    else if (few) prefix_own_kernel<T, D, 8><<<grid, 512, 0, st>>>(c, p, (const T*)q, q_stride, (T*)o, lse, scale);
    else prefix_own_kernel<T, D, 4><<<grid, 256, 0, st>>>(c, p, (const T*)q, q_stride, (T*)o, lse, scale);
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
