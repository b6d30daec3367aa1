// The paged cache in 4 bits: where things lie in a page, and what its kernels share (cache.hip, cache_decode.hip).
#pragma once
#include "common.h"

namespace dma {

constexpr int CACHE_REQS_MAX = 4096;  // places for requests: their row offsets and page counts wait in LDS (cache_assign_kernel)
constexpr int CACHE_TOKENS_MAX = 1 << 30;  // of the pool, of a request (so that a position and a step beyond fit an int)
constexpr int CACHE_ROWS_MAX = 1 << 28;    // of a step (a launch has fewer than 2^32 threads: 256 for 32 rows)
constexpr int FREE_HEADER = 4;        // int32 before the stack of the free list: [0] = number of free pages

struct CacheLayout {
  size_t page_bytes;
  uint32_t off_scales, off_z;  // byte offsets in a page
  int shift;                   // log2 of the page size
};
static inline CacheLayout cache_layout(const dma_cache_shape& s) {
  CacheLayout c;
  const size_t codes = (size_t)s.H_kv * s.page_size * s.d, scales = codes / 16;
  c.off_scales = (uint32_t)codes;
  c.off_z = (uint32_t)(codes + scales);
  c.page_bytes = align_up(codes + scales + (size_t)s.H_q * s.page_size * 4, 256);
  c.shift = ceil_log2(s.page_size);
  return c;
}

// What a kernel needs of the cache.  Slots (page << shift | place in it) and page numbers come from the caller's device memory:
// every one is compared with n_slots or n_pages before it is an address.
struct CacheRef {
  char* pages;
  size_t page_bytes;
  uint32_t off_scales, off_z, n_slots;
  int shift, n_pages, max_pages, n_reqs, H_q, H_kv;
};
static inline CacheRef cache_ref(const dma_cache_shape& s, const void* pages) {
  const CacheLayout l = cache_layout(s);
  return {const_cast<char*>(static_cast<const char*>(pages)), l.page_bytes, l.off_scales, l.off_z,
          (uint32_t)s.n_pages << l.shift, l.shift, s.n_pages, s.max_pages, s.n_reqs, s.H_q, s.H_kv};
}

#ifdef __HIPCC__
__device__ __forceinline__ char* cache_page(const CacheRef& c, uint32_t slot) {
  return c.pages + (size_t)(slot >> c.shift) * c.page_bytes;
}
__device__ __forceinline__ uint32_t cache_place(const CacheRef& c, uint32_t slot) { return slot & ((1u << c.shift) - 1u); }
// The scale of 32 codes as a float: byte b is 2^(b - 127), b = 255 an infinity, which the conversions take as "not a number".
__device__ __forceinline__ float mx_scale(uint32_t byte) { return __uint_as_float(byte << 23); }
#endif

int launch_cache_reset(const dma_cache_shape& s, int32_t* lens, int32_t* table, int32_t* free_list, hipStream_t st);
int launch_cache_assign(const dma_cache_shape& s, int n_rows, const int32_t* change, int32_t* lens, int32_t* table,
                        int32_t* free_list, int32_t* cu_rows, int32_t* row_req, int32_t* row_len, int32_t* slots,
                        int32_t* status, hipStream_t st);
int launch_cache_append(const dma_cache_shape& s, int n_rows, const void* K, long k_stride, const void* V, long v_stride,
                        const float* W, const float* A, const float* z, const int32_t* slots, void* pages, hipStream_t st);
int launch_cache_read(const dma_cache_shape& s, int n_rows, const int32_t* slots, const void* pages, void* K, void* V,
                      float* z, hipStream_t st);
size_t cache_decode_bytes(const dma_cache_shape& s, int n_rows, int k);
int launch_cache_decode(const dma_cache_shape& s, int n_rows, int k, float scale, const void* q, long q_stride,
                        const void* pages, const int32_t* table, const int32_t* row_req, const int32_t* row_len, void* o,
                        float* lse, int32_t* kept, void* ws, hipStream_t st);
size_t cache_decode_prefix_bytes(const dma_cache_shape& s, int n_rows, int k, int n_prefixes, int max_prefix);
int launch_cache_decode_prefix(const dma_cache_shape& s, int n_rows, int k, float scale, const void* q, long q_stride,
                               const void* pages, const int32_t* table, const int32_t* row_req, const int32_t* row_len,
                               int n_prefixes, int max_prefix, const int32_t* prefix_req, const int32_t* prefix_len,
                               const int32_t* req_prefix, void* o, float* lse, void* ws, hipStream_t st);

}  // namespace dma
