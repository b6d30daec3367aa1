// The paged cache: pages and slots for a step's new tokens (assign), rows into it (append) and out of it (read).
//
// K and V are held in 4 bits: an OCP e2m1 code (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign) per channel and one power of two per
// 32 channels of a token's head, 17 / 32 bytes a channel against bf16's 2.  The content scores (Eq. 3) are formed from V as it comes, not
// as it is stored, and held in fp32: they decide which keys a row keeps.
#include "cache.h"
#include "cache_rows.h"
#include "select.h"

namespace dma {

// ------------------------------------------------------------------ pages and slots
// A request with n tokens owns ceil(n / ps) pages.  Requests that shrink push the pages they no longer need on the stack of
// free pages, in order of request and page; those that grow pop theirs, in the same order.  The places on the stack are
// exclusive prefix sums over the requests, so no step depends on another request's outcome but through the sum: a request
// that asks for pages is served if all pages asked for up to and with it are there.
struct AssignArgs {
  const int32_t* change;
  int32_t *lens, *table, *free_list, *cu_rows, *row_req, *row_len, *slots, *status;
  int n_reqs, n_pages, max_pages, shift, n_rows;
};

// Sums that stay at 2^32 - 1 once they reach it, above every number of rows or pages.
__device__ __forceinline__ uint32_t add_sat(uint32_t x, uint32_t y) { return __builtin_elementwise_add_sat(x, y); }

// Exclusive sums over the workgroup's threads of two numbers each, and the totals; s_part: 2 x 16 words, for this call alone.
__device__ __forceinline__ void scan_block(uint32_t& x, uint32_t& y, uint32_t* s_part, uint32_t& all_x, uint32_t& all_y) {
  const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), nw = blockDim.x >> 6;
  x = wave_scan(x, 0u, add_sat);
  y = wave_scan(y, 0u, add_sat);
  if (l == 63) {
    s_part[w] = x;
    s_part[16 + w] = y;
  }
  x = dpp<0x138, 0xf>(0u, x);  // wave_shr:1
  y = dpp<0x138, 0xf>(0u, y);
  __syncthreads();
  const uint32_t ix = wave_scan(l < nw ? s_part[l & 15] : 0u, 0u, add_sat);  // (lane i: up to wave i)
  const uint32_t iy = wave_scan(l < nw ? s_part[16 + (l & 15)] : 0u, 0u, add_sat);
  all_x = last_lane(ix);
  all_y = last_lane(iy);
  if (w) {
    x = add_sat(x, (uint32_t)__builtin_amdgcn_readlane((int)ix, w - 1));
    y = add_sat(y, (uint32_t)__builtin_amdgcn_readlane((int)iy, w - 1));
  }
}

// The last b with first[b] <= i, of n > 0 ascending entries.
__device__ __forceinline__ int find_request(const int32_t* first, int n, int i) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= i) lo = mid; else hi = mid;
  }
  return lo;
}

// Rows that the one workgroup writes itself: a launch of their own costs more than these (see cache_rows_kernel).
constexpr int ASSIGN_ROWS = 4096;

// One workgroup, four requests to a thread.  All that it waits for is one after another -- the lengths, two scans, the pages -- so the
// sums are formed in registers (data-parallel moves, saturating 32 bits), and the rows take the pages of their tokens from the
// same place of the stack as the table does, not from the table.
// Bound by that chain, not by its bytes: 256 requests that grow by a token each 4.4 us alone, of which 2 to 3 are the launch; 777 of which
// 529 grow (25540 tokens, 1594 pages) and others give 9881 pages back, and the same taken back, 14 us on average (2 MB a call, half a
// microsecond at a copy's rate): all pages move through this one workgroup.  The first form, with sums in LDS and the pages read
// back from the table, took 9.3 and 28 us a call.
template <int NT>
__global__ __launch_bounds__(NT) void cache_assign_kernel(AssignArgs p) {
  constexpr int PER = 4, REQS = NT * PER;
  __shared__ int32_t first[REQS + 1];               // first row of every request
  __shared__ int32_t back[REQS + 1], taken[REQS];   // pages given back, and taken, by the requests before it
  __shared__ int32_t length[REQS];                  // its tokens so far; -1 if it is not served
  __shared__ uint32_t s_part[2][32];
  __shared__ uint32_t s_used;
  const int tid = threadIdx.x;
  const long long cap = (long long)p.max_pages << p.shift;
  int32_t* stack = p.free_list + FREE_HEADER;
  auto pages = [&](long long n) { return (int)((n + (1 << p.shift) - 1) >> p.shift); };
  int old[PER], change[PER];
#pragma unroll
  for (int e = 0; e < PER; e++) {
    const int b = tid * PER + e;
    old[e] = b < p.n_reqs ? p.lens[b] : 0;
    change[e] = b < p.n_reqs ? p.change[b] : 0;
  }
  const int have0 = max(0, min(p.free_list[0], p.n_pages));
  if (tid == 0) s_used = 0;
  uint32_t freed[PER], ends[PER], sum_f = 0, sum_g = 0;
#pragma unroll
  for (int e = 0; e < PER; e++) {
    old[e] = (int)max(0ll, min((long long)old[e], cap));
    freed[e] = change[e] < 0 ? (uint32_t)(pages(old[e]) - pages(max(0ll, (long long)old[e] + change[e]))) : 0u;
    sum_f = add_sat(sum_f, freed[e]);
    sum_g = add_sat(sum_g, (uint32_t)max(change[e], 0));
  }
  uint32_t run_f = sum_f, run_g = sum_g, all_f, all_g;
  scan_block(run_f, run_g, s_part[0], all_f, all_g);
  const uint32_t freed_all = min(all_f, (uint32_t)(p.n_pages - have0));  // (never more, unless the caller's tables are damaged)
  const uint32_t have = (uint32_t)have0 + freed_all;
  uint32_t need[PER], sum_n = 0;
  int state[PER];
#pragma unroll
  for (int e = 0; e < PER; e++) {
    const int b = tid * PER + e;
    const uint32_t grow = (uint32_t)max(change[e], 0);
    if (b < p.n_reqs) {
      back[b] = (int)min(run_f, (uint32_t)p.n_pages);
      first[b] = (int)min(run_g, (uint32_t)p.n_rows);
      p.cu_rows[b] = first[b];
    }
    run_f = add_sat(run_f, freed[e]);
    run_g = add_sat(run_g, grow);
    ends[e] = run_g;
    const long long after = (long long)old[e] + change[e];
    state[e] = !grow ? DMA_CACHE_SERVED : after > cap ? DMA_CACHE_TOO_LONG : ends[e] > (uint32_t)p.n_rows ? DMA_CACHE_NO_ROWS : DMA_CACHE_SERVED;
    need[e] = grow && !state[e] ? (uint32_t)(pages(after) - pages(old[e])) : 0u;
    sum_n = add_sat(sum_n, need[e]);
  }
  uint32_t run_n = sum_n, none = 0, all_n, all_0, used = 0;
  scan_block(run_n, none, s_part[1], all_n, all_0);
#pragma unroll
  for (int e = 0; e < PER; e++) {
    const int b = tid * PER + e;
    const uint32_t before = run_n;
    run_n = add_sat(run_n, need[e]);
    if (need[e] && run_n > have) state[e] = DMA_CACHE_NO_PAGES;
    if (need[e] && !state[e]) used = run_n;  // (those that are served are the first ones of all that need any)
    if (b < p.n_reqs) {
      taken[b] = (int)min(before, have);
      length[b] = state[e] ? -1 : old[e];
      p.status[b] = state[e];
      p.lens[b] = state[e] ? old[e] : (int)max(0ll, (long long)old[e] + change[e]);
    }
  }
  used = last_lane(wave_scan(used, 0u, [](uint32_t x, uint32_t y) { return max(x, y); }));
  if ((tid & 63) == 0 && used) atomicMax(&s_used, used);
  if (tid == 0) {
    first[p.n_reqs] = (int)min(all_g, (uint32_t)p.n_rows);
    p.cu_rows[p.n_reqs] = first[p.n_reqs];
    back[p.n_reqs] = (int)freed_all;
  }
  __syncthreads();
  if (freed_all) {
    for (int i0 = tid; i0 < (int)freed_all; i0 += 4 * NT) {
      int32_t* entry[4];
      int32_t page[4];
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const int i = i0 + e * NT;
        entry[e] = nullptr;
        if (i < (int)freed_all) {
          const int b = find_request(back, p.n_reqs, i);  // (it shrank: its pages are the last ones of its old length)
          const int place = pages(length[b]) - (back[b + 1] - back[b]) + i - back[b];
          entry[e] = p.table + (size_t)b * p.max_pages + min(max(place, 0), p.max_pages - 1);
          page[e] = *entry[e];
        }
      }
#pragma unroll
      for (int e = 0; e < 4; e++)
        if (entry[e]) {
          stack[have0 + i0 + e * NT] = page[e];
          *entry[e] = -1;
        }
    }
    __syncthreads();  // (the stack's new top is read below)
  }
  const int n_used = (int)s_used;
  if (tid == 0) p.free_list[0] = (int)have - n_used;
  for (int i0 = tid; i0 < n_used; i0 += 4 * NT) {
    int at[4], to[4];
    int32_t page[4];
#pragma unroll
    for (int e = 0; e < 4; e++) {
      const int i = i0 + e * NT;
      if (i < n_used) {
        at[e] = find_request(taken, p.n_reqs, i);
        to[e] = pages(length[at[e]]) + i - taken[at[e]];
        page[e] = stack[(int)have - 1 - i];
      }
    }
#pragma unroll
    for (int e = 0; e < 4; e++)
      if (i0 + e * NT < n_used) p.table[(size_t)at[e] * p.max_pages + to[e]] = page[e];
  }
  if (p.n_rows > ASSIGN_ROWS) return;
  for (int r = tid; r < p.n_rows; r += NT) {
    int req = -1, len = 0, slot = -1;
    if (r < first[p.n_reqs]) {
      const int b = find_request(first, p.n_reqs, r), n = length[b];
      if (n >= 0) {
        const int pos = n + (r - first[b]), place = pos >> p.shift, more = place - pages(n);
        const int page = more >= 0 ? stack[(int)have - 1 - (taken[b] + more)] : p.table[(size_t)b * p.max_pages + place];
        if ((uint32_t)page < (uint32_t)p.n_pages) {  // (else the lists are damaged, and the row is not there)
          req = b;
          len = pos + 1;
          slot = (page << p.shift) | (pos & ((1 << p.shift) - 1));
        }
      }
    }
    p.row_req[r] = req;
    p.row_len[r] = len;
    p.slots[r] = slot;
  }
}

// The rows of a step with many of them, from what cache_assign_kernel wrote: one a thread, 4.7 us where 777 requests
// grow by hundreds of tokens (several a thread: 44 instead of 37 us for such a call and the one that takes it back).
__global__ __launch_bounds__(256) void cache_rows_kernel(AssignArgs p) {
  __shared__ int32_t first[CACHE_REQS_MAX + 1];
  for (int b = threadIdx.x; b <= p.n_reqs; b += 256) first[b] = p.cu_rows[b];
  __syncthreads();
  const int r = blockIdx.x * 256 + threadIdx.x;
  if (r >= p.n_rows) return;
  int req = -1, len = 0, slot = -1;
  if (r < first[p.n_reqs]) {
    const int b = find_request(first, p.n_reqs, r);
    const int state = p.status[b], pos = p.lens[b] - (first[b + 1] - first[b]) + (r - first[b]);  // (the length has the new tokens)
    if (state == DMA_CACHE_SERVED) {
      const int page = p.table[(size_t)b * p.max_pages + (pos >> p.shift)];
      if ((uint32_t)page < (uint32_t)p.n_pages) {
        req = b;
        len = pos + 1;
        slot = (page << p.shift) | (pos & ((1 << p.shift) - 1));
      }
    }
  }
  p.row_req[r] = req;
  p.row_len[r] = len;
  p.slots[r] = slot;
}

__global__ __launch_bounds__(256) void cache_reset_kernel(int32_t* lens, int32_t* table, int32_t* free_list, int n_reqs,
                                                          int n_pages, size_t entries) {
  const size_t step = gridDim.x * (size_t)256, i0 = blockIdx.x * (size_t)256 + threadIdx.x;
  for (size_t i = i0; i < entries; i += step) table[i] = -1;
  for (size_t i = i0; i < (size_t)n_reqs; i += step) lens[i] = 0;
  for (size_t i = i0; i < (size_t)n_pages; i += step) free_list[FREE_HEADER + i] = n_pages - 1 - (int)i;  // (the lowest are taken first)
  if (i0 < FREE_HEADER) free_list[i0] = i0 == 0 ? n_pages : 0;
}

int launch_cache_reset(const dma_cache_shape& s, int32_t* lens, int32_t* table, int32_t* free_list, hipStream_t st) {
  const size_t entries = (size_t)s.n_reqs * s.max_pages;
  const size_t most = entries > (size_t)s.n_pages ? entries : (size_t)s.n_pages, blocks = (most + 255) / 256;
  cache_reset_kernel<<<(unsigned)(blocks < 64 * CUS ? blocks : 64 * CUS), 256, 0, st>>>(lens, table, free_list, s.n_reqs, s.n_pages, entries);
  return hipGetLastError() == hipSuccess ? DMA_OK : DMA_EHIP;
}

int launch_cache_assign(const dma_cache_shape& s, int n_rows, const int32_t* change, int32_t* lens, int32_t* table,
                        int32_t* free_list, int32_t* cu_rows, int32_t* row_req, int32_t* row_len, int32_t* slots,
                        int32_t* status, hipStream_t st) {
  const AssignArgs p = {change, lens, table, free_list, cu_rows, row_req, row_len, slots, status,
                        s.n_reqs, s.n_pages, s.max_pages, cache_layout(s).shift, n_rows};
  if (s.n_reqs <= 1024 && n_rows <= 1024) cache_assign_kernel<256><<<1, 256, 0, st>>>(p);
  else cache_assign_kernel<1024><<<1, 1024, 0, st>>>(p);
  if (hipGetLastError() != hipSuccess) return DMA_EHIP;
  if (n_rows > ASSIGN_ROWS) cache_rows_kernel<<<(unsigned)((n_rows + 255) / 256), 256, 0, st>>>(p);
  return hipGetLastError() == hipSuccess ? DMA_OK : DMA_EHIP;
}

// ------------------------------------------------------------------ rows into the cache
// Rows whose K and V are more than this (and bf16) are read past the caches: with the pages they do not fit the last one, of 256 MB, and
// would only drive each other out.  Rows of 8 heads of 128 channels, us through / past: 65536 from memory 103 / 82, 65536 just made by
// other kernels, these included, 192 / 183, 49152 (192 MiB) 135 / 130, 40960 (160 MiB) 102 / 111, 16384 48 / 54.  (fp32 ones come in half
// lines, which then are fetched twice: 5003 rows of 4 heads of 256, in and out, 24.7 / 27.2.  Codes stored past the caches: + 1 us.)
constexpr size_t APPEND_PAST = (size_t)176 << 20;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <bool PAST, typename T> __device__ __forceinline__ void load_row(const T* src, Raw8<T>& r) {
  if constexpr (PAST) r.x = __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src)));
  else load_raw(src, r);
}

// Rows of a tile, for rows of that many bytes: more workgroups of fewer registers where a row is long.  In and out, 64 / 32 rows, us:
// 5003 x 4 heads of 256 fp32 channels 27.0 / 24.4, 9001 x 4 of 256 in bf16 24.9 / 22.8, 9001 x 4 of 128 in fp32 22.0 / 20.8, 65536 x 8 of
// 128 in bf16 163.2 / 162.0, 20001 x 16 of 64 in bf16 50.7 / 51.8.
constexpr int tile_size(int bytes) { return bytes >= 256 ? 32 : 64; }

// Where the rows of a tile go: the page (none: null) and the place in it, worked out once for all of a row's lanes (a 64-bit
// product each).
struct TileRows {
  char* page[64];
  uint32_t place[64];
};
__device__ __forceinline__ void tile_rows(const CacheRef& c, const int32_t* __restrict__ slots, int tile, int t0, int n_rows,
                                          TileRows& rows) {
  if ((int)threadIdx.x < tile) {
    const int t = t0 + threadIdx.x;
    const uint32_t slot = t < n_rows ? (uint32_t)slots[t] : 0xffffffffu;
    rows.page[threadIdx.x] = slot < c.n_slots ? cache_page(c, slot) : nullptr;
    rows.place[threadIdx.x] = cache_place(c, slot);
  }
}

// One workgroup per (tile of rows, kv-head).  A row is held by D / 8 lanes; K and V of all rows of the tile are requested before the
// first is used.  The scores are those of z_kernel, bit for bit: the same sums in the same order.
// Bound by HBM: 65536 rows of 8 heads of 128 channels, 32 scores each, out of a projection of 48 heads, 82 us for 350 MB (4.3 TB/s;
// a copy reaches 4.75).  One row: 4.1 us, the latency of slots, rows, sums and two barriers behind a launch.  (A row's pages worked out by each of its lanes, and fp32 values where
// bf16 ones do, 960 vector instructions instead of 730, took as long; so do heads before rows in the order of the workgroups.  Passes
// without a row left out: + 3 us, a call of one row as before.)
template <typename T, int D, int GMAX, bool PAST>
__global__ __launch_bounds__(256) void cache_append_kernel(CacheRef c, const T* __restrict__ K, long k_stride,
                                                           const T* __restrict__ V, long v_stride,
                                                           const float* __restrict__ W, const float* __restrict__ A,
                                                           const float* __restrict__ z, const int32_t* __restrict__ slots,
                                                           int n_rows) {
  constexpr int TILE = tile_size(D * sizeof(T));
  __shared__ float zs[GMAX * TILE];
  __shared__ TileRows rows;
  constexpr int LPR = D / 8, RPP = 256 / LPR, NP = TILE / RPP;
  __shared__ __align__(16) uint8_t bytes[TILE][D / 16];  // the rows' scales, K's and V's, which leave together
  const int g = blockIdx.y, G = c.H_q / c.H_kv, t0 = blockIdx.x * TILE;
  const int tid = threadIdx.x, sub = tid % LPR, rl = tid / LPR;
  tile_rows(c, slots, TILE, t0, n_rows, rows);
  Raw8<T> k[NP], v[NP];
#pragma unroll
  for (int pass = 0; pass < NP; pass++) {
    const long t = min(t0 + pass * RPP + rl, n_rows - 1);
    load_row<PAST>(K + t * k_stride + (long)g * D + 8 * sub, k[pass]);
    load_row<PAST>(V + t * v_stride + (long)g * D + 8 * sub, v[pass]);
  }
  __syncthreads();
#pragma unroll
  for (int pass = 0; pass < NP; pass++) {
    const int r = pass * RPP + rl;
    char* page = rows.page[r];
    const uint32_t at = ((uint32_t)g << c.shift) + rows.place[r];
    uint32_t kb, vb;
    const uint32_t kc = quantise8(k[pass], kb), vc = quantise8(v[pass], vb);
    if (page) {
      uint32_t* codes = reinterpret_cast<uint32_t*>(page + (at * D + 4 * sub));
      codes[0] = kc;
      codes[LPR] = vc;
    }
    if (sub % 4 == 0) {
      bytes[r][sub / 4] = (uint8_t)kb;
      bytes[r][D / 32 + sub / 4] = (uint8_t)vb;
    }
  }
  auto put_score = [&](int h, int r, float zv) {
    if (char* page = rows.page[r])
      reinterpret_cast<float*>(page + c.off_z)[((uint32_t)h << c.shift) + rows.place[r]] = zv;
  };
  auto put_bytes = [&]() {  // (behind a barrier)
    if (tid < TILE && rows.page[tid]) {
      using Bytes = std::conditional_t<D == 64, uint32_t, std::conditional_t<D == 128, uint2, uint4>>;
      char* to = rows.page[tid] + (c.off_scales + (((uint32_t)g << c.shift) + rows.place[tid]) * (D / 16));
      *reinterpret_cast<Bytes*>(to) = *reinterpret_cast<const Bytes*>(bytes[tid]);
    }
  };
  if (!W) {
    __syncthreads();
    put_bytes();
    for (int i = tid; i < G * TILE; i += 256) {
      const int h = g * G + i / TILE, r = i % TILE;
      if (t0 + r < n_rows) put_score(h, r, z[(size_t)h * n_rows + t0 + r]);
    }
    return;
  }
  for (int h0 = 0; h0 < G; h0 += GMAX) {
    float wreg[GMAX][8];
#pragma unroll
    for (int hh = 0; hh < GMAX; hh++) {
      Raw8<float> raw;
      load_raw(W + (size_t)(g * G + min(h0 + hh, G - 1)) * D + 8 * sub, raw);
      to_f32(raw, wreg[hh]);
    }
    if (h0) __syncthreads();  // (the scores of the heads before are on their way)
#pragma unroll
    for (int pass = 0; pass < NP; pass++) {
      float x[8];
      to_f32(v[pass], x);
#pragma unroll
      for (int hh = 0; hh < GMAX; hh++) {
        float acc = 0.f;
#pragma unroll
        for (int e = 0; e < 8; e++) acc = fmaf(wreg[hh][e], x[e], acc);
        acc = group_sum<LPR>(acc);
        if (sub == hh % LPR) zs[hh * TILE + pass * RPP + rl] = acc;
      }
    }
    __syncthreads();
    if (!h0) put_bytes();
    for (int i = tid; i < min(GMAX, G - h0) * TILE; i += 256) {
      const int h = g * G + h0 + i / TILE;
      const float x = zs[i], sp = fmaxf(x, 0.f) + log1pf(expf(-fabsf(x)));
      put_score(h, i % TILE, expf(A[h] * sp));
    }
  }
}

// ------------------------------------------------------------------ rows out of it
// The same tiles; rows without a slot come back as zeros with a score of -infinity.  Bound by HBM, writes above all: 65536 rows as
// above 66 us for 355 MB; that this is more than a copy's 4.75 TB/s is because some of its output is still in the last cache when
// it ends.  (Stores past the caches: 53 instead of 73 us in a row, but the kernel that uses the rows
// loses more, 141 -> 153 together.  Codes read past them: 65536 rows - 4 us, 20001 of 16 heads of 64 channels + 6.)
template <typename T, int D>
__global__ __launch_bounds__(256) void cache_read_kernel(CacheRef c, const int32_t* __restrict__ slots, T* __restrict__ K,
                                                         T* __restrict__ V, float* __restrict__ z, int n_rows) {
  constexpr int TILE = tile_size(D * sizeof(T)), LPR = D / 8, RPP = 256 / LPR, NP = TILE / RPP;
  __shared__ TileRows rows;
  const int g = blockIdx.y, G = c.H_q / c.H_kv, t0 = blockIdx.x * TILE;
  const int tid = threadIdx.x, sub = tid % LPR, rl = tid / LPR;
  tile_rows(c, slots, TILE, t0, n_rows, rows);
  __syncthreads();
  uint32_t kc[NP], vc[NP], kb[NP], vb[NP];
#pragma unroll
  for (int pass = 0; pass < NP; pass++) {
    const int r = pass * RPP + rl;
    const char* page = rows.page[r];
    const uint32_t at = ((uint32_t)g << c.shift) + rows.place[r];
    kc[pass] = vc[pass] = kb[pass] = vb[pass] = 0;
    if (page) {
      const uint32_t* codes = reinterpret_cast<const uint32_t*>(page + (at * D + 4 * sub));
      const uint8_t* scales = reinterpret_cast<const uint8_t*>(page + (c.off_scales + at * (D / 16) + sub / 4));
      kc[pass] = codes[0];
      vc[pass] = codes[LPR];
      kb[pass] = scales[0];
      vb[pass] = scales[D / 32];
    }
  }
  auto put = [&](T* dst, uint32_t code, uint32_t byte) {
    const float sc = mx_scale(byte);
    if constexpr (sizeof(T) == 2) {
      const uint4 out = make_uint4(
          __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, sc, 0)),
          __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, sc, 1)),
          __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, sc, 2)),
          __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, sc, 3)));
      *reinterpret_cast<uint4*>(dst) = out;
    } else {
      const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, sc, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, sc, 1);
      const auto e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, sc, 2), f = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, sc, 3);
      reinterpret_cast<float4*>(dst)[0] = make_float4(a[0], a[1], b[0], b[1]);
      reinterpret_cast<float4*>(dst)[1] = make_float4(e[0], e[1], f[0], f[1]);
    }
  };
#pragma unroll
  for (int pass = 0; pass < NP; pass++) {
    const int t = t0 + pass * RPP + rl;
    if (t < n_rows) {
      put(K + ((size_t)t * c.H_kv + g) * D + 8 * sub, kc[pass], kb[pass]);
      put(V + ((size_t)t * c.H_kv + g) * D + 8 * sub, vc[pass], vb[pass]);
    }
  }
  for (int i = tid; i < G * TILE; i += 256) {
    const int h = g * G + i / TILE, r = i % TILE;
    if (t0 + r >= n_rows) continue;
    const char* page = rows.page[r];
    z[(size_t)h * n_rows + t0 + r] = page ? reinterpret_cast<const float*>(page + c.off_z)[((uint32_t)h << c.shift) + rows.place[r]] : -INFINITY;
  }
}

template <typename T, int D>
static void append_t(const dma_cache_shape& s, int n_rows, const void* K, long k_stride, const void* V, long v_stride,
                     const float* W, const float* A, const float* z, const int32_t* slots, void* pages, hipStream_t st) {
  const CacheRef c = cache_ref(s, pages);
  const int tile = tile_size(s.d * (s.dtype == DMA_F32 ? 4 : 2));
  const dim3 grid((unsigned)((n_rows + tile - 1) / tile), (unsigned)s.H_kv);
  const int G = s.H_q / s.H_kv;
  const bool past = sizeof(T) == 2 && (size_t)n_rows * s.H_kv * D * 4 > APPEND_PAST;
#define DMA_APPEND(GM) \
  if (past) cache_append_kernel<T, D, GM, sizeof(T) == 2><<<grid, 256, 0, st>>>(c, (const T*)K, k_stride, (const T*)V, v_stride, W, A, z, slots, n_rows); \
  else cache_append_kernel<T, D, GM, false><<<grid, 256, 0, st>>>(c, (const T*)K, k_stride, (const T*)V, v_stride, W, A, z, slots, n_rows)
  if (G == 1) { DMA_APPEND(1); }
  else if (G == 2) { DMA_APPEND(2); }
  else { DMA_APPEND(4); }
#undef DMA_APPEND
}

int launch_cache_append(const dma_cache_shape& s, int n_rows, const void* K, long k_stride, const void* V, long v_stride,
                        const float* W, const float* A, const float* z, const int32_t* slots, void* pages, hipStream_t st) {
  auto go = [&](auto t) {
    using T = std::remove_pointer_t<decltype(t)>;
    if (s.d == 256) append_t<T, 256>(s, n_rows, K, k_stride, V, v_stride, W, A, z, slots, pages, st);
    else if (s.d == 128) append_t<T, 128>(s, n_rows, K, k_stride, V, v_stride, W, A, z, slots, pages, st);
    else append_t<T, 64>(s, n_rows, K, k_stride, V, v_stride, W, A, z, slots, pages, st);
  };
  if (s.dtype == DMA_BF16) go((__bf16*)nullptr); else go((float*)nullptr);
  return hipGetLastError() == hipSuccess ? DMA_OK : DMA_EHIP;
}

int launch_cache_read(const dma_cache_shape& s, int n_rows, const int32_t* slots, const void* pages, void* K, void* V,
                      float* z, hipStream_t st) {
  const CacheRef c = cache_ref(s, pages);
  const int tile = tile_size(s.d * (s.dtype == DMA_F32 ? 4 : 2));
  const dim3 grid((unsigned)((n_rows + tile - 1) / tile), (unsigned)s.H_kv);
  auto go = [&](auto t) {
    using T = std::remove_pointer_t<decltype(t)>;
    if (s.d == 256) cache_read_kernel<T, 256><<<grid, 256, 0, st>>>(c, slots, (T*)K, (T*)V, z, n_rows);
    else if (s.d == 128) cache_read_kernel<T, 128><<<grid, 256, 0, st>>>(c, slots, (T*)K, (T*)V, z, n_rows);
    else cache_read_kernel<T, 64><<<grid, 256, 0, st>>>(c, slots, (T*)K, (T*)V, z, n_rows);
  };
  if (s.dtype == DMA_BF16) go((__bf16*)nullptr); else go((float*)nullptr);
  return hipGetLastError() == hipSuccess ? DMA_OK : DMA_EHIP;
}

}  // namespace dma
