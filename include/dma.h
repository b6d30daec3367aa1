/*
 * dma.h -- C ABI of the MI355X (gfx950) Dynamic Mask Attention hot path.
 *
 * The operations are those of arxiv 2508.02124, Section 4 ("Method"):
 *   dma_mask_gen : content scores  z = exp(A * softplus(v . w))            (Eq. 3)
 *                  and the per-row top-k + causal kept sets                (Eq. 4, Listing 1)
 *   dma_fwd      : O = softmax(Q K^T * scale + z, over the kept set) V     (Eq. 5-6, Alg. 1)
 *   dma_bwd      : dQ, dK, dV and the gradient into z                      (Eq. 7-10, Alg. 2)
 *
 * Conventions for every entry point
 *   - All tensor arguments are DEVICE pointers, 16-byte aligned, densely packed,
 *     token-major, last dimension contiguous:
 *         Q, O, dO, dQ : [T, H_q , d]      K, V, dK, dV : [T, H_kv, d]
 *         z, dz, LSE   : [H_q, T] float    expiry       : [H_q, T] int32
 *         W : [H_q, d] float               A            : [H_q] float
 *         cu_seqlens   : [n_docs + 1] int32, cu[0] = 0, cu[n_docs] = T
 *     Q/K/V/O/dO/dQ/dK/dV are bf16 (dtype DMA_BF16) or float (DMA_F32, a slow
 *     debug path).  A fixed batch of B sequences of length L is T = B*L with
 *     cu_seqlens = {0, L, 2L, ...}.
 *   - q-head h reads kv-head h / (H_q / H_kv) (contiguous grouping).
 *   - The `dma_shape` argument is a HOST pointer, read during the call.
 *   - The caller owns every buffer.  The compute entry points allocate nothing,
 *     free nothing and keep no pointer after the call returns.  The library's only
 *     state between calls: the host array of event handles that dma_profile_events
 *     was given (per host thread, until it is called with NULL), and the address of
 *     dma_decode_static's own device scratch array (per GPU).
 *   - Work is enqueued on `stream` (a hipStream_t passed as void*; NULL = the
 *     default stream) and the call returns without synchronising.
 *   - Return value: DMA_OK (0) or a negative dma_status.  All argument checks
 *     happen before the first launch, so a failing call enqueues nothing.
 *   - Outputs are fully overwritten; the caller need not clear them.
 */
#ifndef DMA_H_
#define DMA_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  DMA_OK = 0,
  DMA_EINVAL = -1,       /* null pointer, misaligned pointer, T<=0, k<=0, n_docs<=0, H_q % H_kv != 0;
                            of the paged cache: n_rows<0, a stride below the row or not a multiple of 8 */
  DMA_EUNSUPPORTED = -2, /* d not in {64,128,256} (cross-head scores: {64,128}),
                            unknown dtype, more than 256 q-heads per kv-head,
                            more than 32 heads for the cross-head scores,
                            bf16 dma_fwd / dma_bwd with T >= 2^24 or Q (or K, V) larger than 4 GiB;
                            rotary channels that are not a multiple of 16;
                            of the paged cache: page sizes and numbers other than stated there             */
  DMA_EWORKSPACE = -3,   /* ws_bytes smaller than dma_workspace_bytes() / dma_cache_decode_bytes() /
                            dma_cache_decode_prefix_bytes() */
  DMA_EHIP = -4          /* a launch failed (hipGetLastError) */
} dma_status;

typedef enum { DMA_BF16 = 0, DMA_F32 = 1 } dma_dtype;

typedef struct {
  int32_t T;            /* total packed tokens                                        */
  int32_t n_docs;       /* number of documents (sequences) packed into T              */
  int32_t max_seqlen;   /* upper bound on the longest document (0 => T).  It chooses between
                           equal ways of working; a bound that is too small costs time
                           but changes no result.  (dma_mask_gen_bias: also the length
                           of a bias row that the documents share, which must hold)    */
  int32_t H_q;          /* query heads                                                */
  int32_t H_kv;         /* key/value heads, divides H_q                               */
  int32_t d;            /* head dimension: 64, 128 or 256 (256: not for the cross-head
                           scores)                                                    */
  int32_t k;            /* keep-window (the paper's w): kept keys per query row;
                           k larger than a document keeps all of its causal keys      */
  int32_t causal;       /* 1: candidates of row i are the keys j <= i of its document;
                           0: all keys of its document (every row keeps the same keys)  */
  int32_t dtype;        /* dma_dtype of Q/K/V/O and their gradients                   */
  float softmax_scale;  /* 0 => d^-1/2                                                */
} dma_shape;

/* Size in bytes of the opaque mask plan written by dma_mask_gen (slot table,
 * per-block key lists and scratch of the selection), and of the scratch
 * workspace dma_fwd / dma_bwd need.  0 if the shape is invalid.
 * The plan is not linear in T: its slot table holds one int32 per (q-head, block of
 * 256 query rows, slot), slots = min(k, T) rounded up to 128, i.e. about
 * H_q * T * min(k, T) / 64 bytes, on top of about 40 bytes per (q-head, token)
 * (scores, expiry, key lists, scratch of the selection).  Examples with H_q = 32: 36 MiB
 * at T = 16384, k = 2048; 111 MiB at T = 65536, k = 1024; 0.58 GiB at k = 16384; 2.1 GiB
 * at T = k = 65536 (every key kept: the quadratic corner).  There is no cap: a caller
 * that sweeps k towards T pays this. */
size_t dma_mask_bytes(const dma_shape* shape);
size_t dma_workspace_bytes(const dma_shape* shape);

/*
 * Where the parts of the mask plan lie, for tools and tests that inspect what dma_mask_gen wrote
 * (the occupancy structure of Section 4.2: per block of query rows, the keys resident for the whole
 * block -- one slot column each -- and the keys that enter or expire inside it).  The attention
 * entry points need none of this.  `out` is a HOST pointer; offsets are bytes from the start of the
 * mask buffer.  Returns DMA_OK or the error of an invalid shape.
 *   blocks         int32[nblk_cap][4]: {document, first row, end row, document start}; document -1 past the end
 *   slot_table     int32[H_q][nblk_cap][kpad]: resident key of each slot column; below 0 = none for the whole
 *                  block (-2 - key: that key enters inside the block and stays to its end; -1 otherwise.
 *                  dma_version() < 141 does not say whether a plan has such entries)
 *   partial_count  int32[H_q][nblk_cap];  partial_list int32[H_q][nblk_cap][max_partial]
 *   header         int32[16], [0] = number of blocks;  zq float[H_q][T] = z / softmax_scale
 */
typedef struct {
  int32_t block_rows;   /* query rows per block                          */
  int32_t group_cols;   /* slot columns per key-stationary workgroup     */
  int32_t max_partial;  /* capacity of a block's partial list            */
  int32_t nblk_cap;     /* rows of the block table: T / block_rows + n_docs */
  int32_t kpad;         /* slot-table row length                         */
  int32_t reserved;
  uint64_t off_header, off_zq, off_blocks, off_slot_table, off_partial_count, off_partial_list, total;
} dma_mask_layout;
int dma_mask_describe(const dma_shape* shape, dma_mask_layout* out);

/*
 * Mask generation (Eq. 3, Eq. 4, Listing 1's mask block).
 *   V          in   [T, H_kv, d]
 *   W, A       in   per-q-head projection vector and gate.  W == NULL means the
 *                   caller supplies z (A is then ignored); z must be finite.
 *   z          out if W != NULL, else in.  z[h, j] = exp(A_h * softplus(w_h . v_{g(h), j}))
 *   expiry     out  e[h, j] (global row index) = first row >= j of j's document
 *                   that does NOT keep key j; e == j: never kept; e == end of the
 *                   document: kept to the end.  Row i keeps key j  <=>  j <= i < e[h, j].
 *                   The kept set of a row is its min(k, i - doc_start + 1) best causal
 *                   keys by (z descending, index ascending).  With causal == 0 every row of a
 *                   document keeps the document's min(k, n) best keys: e[h, j] = end of the
 *                   document for those keys (kept by all rows) and e[h, j] = j for the others.
 *   topk_idx   out, nullable: [H_q, T, k] int32, the kept keys of each row as global
 *                   indices in ascending order, padded with -1 (debug; O(T k) memory).
 *   mask       out  dma_mask_bytes(shape) bytes; consumed by dma_fwd / dma_bwd.  It also holds
 *                   z / softmax_scale (the attention kernels start their score accumulators
 *                   at it) and that softmax_scale itself.  The plan is the authority on both:
 *                   dma_fwd / dma_bwd read the scores and the scale from it, not from their
 *                   own z and shape->softmax_scale arguments (which therefore cannot disagree
 *                   with the stored scores); a changed z or scale needs a new dma_mask_gen.
 *                   The other fields of the shape must be the ones the plan was made with.
 */
int dma_mask_gen(const dma_shape* shape, const void* V, const float* W, const float* A,
                 const int32_t* cu_seqlens, float* z, int32_t* expiry, int32_t* topk_idx,
                 void* mask, void* stream);

/*
 * Mask generation with a further, caller-supplied attention bias (Section 1, "Kernel Design": the
 * kernel takes masks and biases with batch, head and query broadcasting).  The bias holds one value
 * per key, broadcast over the query rows; it is added to the scores of the kept pairs next to z,
 *     S_ij = scale q_i . k_j + z[h, j] + bias[h, j],
 * while the kept sets are selected on z alone (Eq. 4 ranks the content scores).  Everything else is
 * dma_mask_gen; dma_fwd / dma_bwd are called as usual with the mask written here.
 *   bias            in  float, finite (a large negative value acts as a key mask)
 *   bias_heads      H_q: one row per q-head; 1: one row shared by all heads (head broadcast)
 *   bias_per_token  != 0: bias is [bias_heads, T], packed like z;
 *                   == 0: bias is [bias_heads, shape->max_seqlen], indexed by the key's position in
 *                   its document and shared by all documents (batch broadcast); max_seqlen must be
 *                   set and no document may be longer
 * z and the bias enter the score as a sum, so the dz of dma_bwd is also the gradient with respect
 * to the bias as applied; dma_bias_bwd reduces it over the heads and documents that share an entry:
 *   dbias out [bias_heads, T] or [bias_heads, max_seqlen] float, fully overwritten (no atomics).
 * A bias per (query, key) pair has no per-key structure and is not supported.
 */
int dma_mask_gen_bias(const dma_shape* shape, const void* V, const float* W, const float* A,
                      const int32_t* cu_seqlens, const float* bias, int32_t bias_heads, int32_t bias_per_token,
                      float* z, int32_t* expiry, int32_t* topk_idx, void* mask, void* stream);
int dma_bias_bwd(const dma_shape* shape, const float* dz, const int32_t* cu_seqlens, int32_t bias_heads,
                 int32_t bias_per_token, float* dbias, void* stream);

/*
 * Forward (Eq. 5-6; online softmax as in Alg. 1, query-stationary).
 *   O   out [T, H_q, d]     LSE out [H_q, T], natural-log sum-exp of the kept scores.
 *   ws  not used (may be NULL, ws_bytes 0).
 */
int dma_fwd(const dma_shape* shape, const void* Q, const void* K, const void* V, const float* z,
            const int32_t* expiry, const void* mask, const int32_t* cu_seqlens,
            void* O, float* LSE, void* ws, size_t ws_bytes, void* stream);

/*
 * Backward (Eq. 7-10; Alg. 2 with D_i = rowsum(dO o O)).
 *   dQ out [T, H_q, d]; dK, dV out [T, H_kv, d], summed over the q-heads of a group;
 *   dz out [H_q, T] = sum over query rows of dS (exactly 0 for keys never kept).
 *   dV is the attention-path gradient only (not the path through z).
 *   dK, dV and dz are accumulated with floating-point atomics: results can differ
 *   in the last bits between runs.
 */
int dma_bwd(const dma_shape* shape, const void* Q, const void* K, const void* V, const void* O,
            const void* dO, const float* LSE, const float* z, const int32_t* expiry,
            const void* mask, const int32_t* cu_seqlens,
            void* dQ, void* dK, void* dV, float* dz, void* ws, size_t ws_bytes, void* stream);

/*
 * Gradient of the content scores (the chain rule of Eq. 3; Section 6: the bias is the path by
 * which gradients reach the score parameters).  With x = w_h . v_{g(h), j}, z = exp(A_h softplus(x)):
 *   dz  in  [H_q, T]        the gradient that dma_bwd returned for the bias
 *   dW  out [H_q, d] f32    dW_h = sum_j dx_{h,j} v_{g(h),j},  dx = dz z A_h sigmoid(x)
 *   dA  out [H_q]    f32    dA_h = sum_j dz z softplus(x)
 *   dV  [T, H_kv, d], dtype of V: the part of dV that flows through z,
 *       sum over the q-heads h of kv-head g of dx_{h,j} w_h; written if accumulate == 0, added
 *       to the existing contents (e.g. the dV of dma_bwd; one rounding of the sum) otherwise.
 * z is recomputed from V, W, A.  dW and dA are accumulated with floating-point atomics.  No
 * workspace; shape->k, n_docs and softmax_scale are not used.  Errors as for the other entry points.
 * Shapes whose group (H_q / H_kv q-heads per kv-head) does not fit the kernel's 64 KiB of LDS --
 * (tile * d + 2 G d + 2 G tile + G) floats with tile = 64 tokens (32 at d = 256), i.e. more than 47 / 21 / 14 q-heads per kv-head at d = 64 / 128 / 256 --
 * are refused with DMA_EUNSUPPORTED before any launch.
 */
int dma_mask_bwd(const dma_shape* shape, const void* V, const float* W, const float* A, const float* dz,
                 float* dW, float* dA, void* dV, int accumulate, void* stream);

/*
 * dma_bwd and then dma_mask_bwd with accumulate: the backward of a whole step.  The arguments are theirs; the same
 * results, but the two parts of dV are added before they are rounded.  Groups of 1, 2, 4 or 8 q-heads in bf16 save a pass
 * over dV and two launches, other shapes take the two calls' launches.
 */
int dma_bwd_scores(const dma_shape* shape, const void* Q, const void* K, const void* V, const void* O,
                   const void* dO, const float* LSE, const float* z, const int32_t* expiry,
                   const void* mask, const int32_t* cu_seqlens, const float* W, const float* A,
                   void* dQ, void* dK, void* dV, float* dz, float* dW, float* dA, void* ws, size_t ws_bytes,
                   void* stream);

/*
 * Rotary positions (Listing 1 turns q and k before the attention): pair i of a head's first `rot` channels is turned by the angle
 * a = position * freqs[i],
 *     y1 = x1 cos a - x2 sin a,   y2 = x1 sin a + x2 cos a,
 * the pairs being the channels (i, i + rot / 2), or the neighbours (2 i, 2 i + 1) if interleaved != 0; channels from rot on stay.
 *   Q, K       in   T rows of [H_q, d] and [H_kv, d], q_stride and k_stride elements apart (multiples of 8 of at least the row: both may be
 *                   parts of one projection's output); either may be NULL and is then left out
 *   positions  in   nullable: [T] int32, of any sign; NULL: a token's position is its place in its document (cu_seqlens, else not read;
 *                   tokens behind the last document count on in it)
 *   freqs      in   [rot / 2] float, e.g. base^(-2 i / rot); |position * freqs[i]| is below 2^50 (a pair beyond that, or with a frequency
 *                   that is no number, gets values without meaning, and no other pair does)
 *   rot        a multiple of 16, at most d
 *   inverse    != 0: turned by -a.  That is the transpose, so the gradients of Q and K are those of Qo and Ko turned with inverse = 1
 *   Qo, Ko     out  rows qo_stride and ko_stride elements apart (what lies between rows is left as it is); Qo may be Q, and Ko K, with the
 *                   same stride, else no output overlaps an input
 * Angles are reduced in 64 bits, so that far positions are as exact as near ones; products are in fp32, rounded once to the type.
 * shape->k, max_seqlen, causal and softmax_scale are not used, n_docs only with cu_seqlens.
 */
int dma_rope(const dma_shape* shape, const void* Q, int64_t q_stride, const void* K, int64_t k_stride,
             const int32_t* cu_seqlens, const int32_t* positions, const float* freqs, int32_t rot, int interleaved,
             int inverse, void* Qo, int64_t qo_stride, void* Ko, int64_t ko_stride, void* stream);

/*
 * Content scores with the paper's full sampling tensor (Eq. 3 states Delta in R^{n_h x d_h x n_h};
 * Listing 1 flattens the values of all heads of a token before the projection): the score of q-head
 * h contracts the token's value vectors of ALL kv-heads,
 *     z[h, j] = exp(A_h * softplus(sum_{g, c} V[j, g, c] * Delta[h, g, c])).
 *   Delta in  [H_q, H_kv * d] float, row h = the [H_kv, d] weights of head h (the layout of a linear
 *             layer's weight from the flattened values to the heads)
 *   z     out [H_q, T]; pass it to dma_mask_gen with W == NULL (caller-supplied scores).
 * dma_scores_xhead_bwd is its chain rule, the counterpart of dma_mask_bwd:
 *   dz in [H_q, T];  dDelta out [H_q, H_kv * d] f32 = sum_j dx[h, j] V[j, g, c];  dA out [H_q] f32;
 *   dV [T, H_kv, d], dtype of V: sum_h dx[h, j] Delta[h, g, c], written (accumulate == 0) or added.
 * dDelta and dA are accumulated with floating-point atomics.  H_q <= 32 (DMA_EUNSUPPORTED beyond);
 * shape->k, n_docs and softmax_scale are not used.  No workspace.
 */
int dma_scores_xhead(const dma_shape* shape, const void* V, const float* Delta, const float* A, float* z,
                     void* stream);
int dma_scores_xhead_bwd(const dma_shape* shape, const void* V, const float* Delta, const float* A, const float* dz,
                         float* dDelta, float* dA, void* dV, int accumulate, void* stream);

/*
 * Decode: the newest row of every sequence against its KV cache (Eq. 4-6 for one query row; the
 * regime of the paper's largest speed-ups, Section 5).  Sequence b occupies rows
 * [cu_seqlens[b], cu_seqlens[b+1]) of K, V and z, its last row being the new token; that row's
 * candidates are all n keys of the sequence, of which it keeps the min(k, n) best by
 * (z descending, index ascending).
 *   q     in  [n_docs, H_q, d]   the query of the last row of each sequence
 *   K, V  in  [T, H_kv, d];  z in [H_q, T] (the caller appends the new token's score, e.g. with
 *             dma_mask_gen on the new row or its own Eq. 3)
 *   o     out [n_docs, H_q, d];  lse out [H_q, n_docs] (natural log; -inf and o = 0 for an empty sequence)
 *   kept  out [n_docs, H_q, min(k, T)] int32: the kept keys of each (sequence, head) as global row
 *             indices, ascending, the first min(k, n) entries valid.  The buffer also carries
 *             the kernels' scratch behind that array (per-chunk partial outputs), so it is
 *             required and must hold dma_decode_kept_bytes(shape) bytes (DMA_EWORKSPACE otherwise).
 * Stateless: the selection is redone from z on every call (z is n floats per head, the gathered
 * K/V rows are min(k, n) d-vectors; both are read once or a few times).  No mask plan is needed.
 */
size_t dma_decode_kept_bytes(const dma_shape* shape);
int dma_decode(const dma_shape* shape, const void* q, const void* K, const void* V, const float* z,
               const int32_t* cu_seqlens, void* o, float* lse, int32_t* kept, size_t kept_bytes, void* stream);

/*
 * dma_decode for callers that cannot allocate device memory or pass a scratch region: code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same operation, same
 * kernels and same results as dma_decode, but the kernels' scratch (per-chunk partial outputs, the
 * selection's histograms and counts) lies in a device array owned by the library, of
 * DMA_DECODE_STATIC_SCRATCH_BYTES on every GPU the library is used on (held until the process ends;
 * its address is looked up on the first call on each device).  The call allocates and frees nothing.
 *   kept  out [n_docs, H_q, min(k, T)] int32 only (no scratch behind it)
 *   Shapes whose scratch, dma_decode_static_scratch_bytes(shape), exceeds the array are refused with
 *   DMA_EWORKSPACE before anything is enqueued (e.g. 1 sequence x 32 heads x k = 2048 x d = 128
 *   needs 0.32 MiB; about 12 such sequences fit).
 *   Every call on a GPU uses that GPU's one array: calls that overlap in time on one GPU (two
 *   streams, two threads) race; calls on one stream are ordered and safe.  Nothing in the array
 *   needs clearing by the caller (each call clears what it accumulates into with a fill kernel).
 */
#define DMA_DECODE_STATIC_SCRATCH_BYTES (4u << 20)
size_t dma_decode_static_scratch_bytes(const dma_shape* shape);
int dma_decode_static(const dma_shape* shape, const void* q, const void* K, const void* V, const float* z,
                      const int32_t* cu_seqlens, void* o, float* lse, int32_t* kept, void* stream);

/*
 * Decode in a loop, with the kept sets carried from step to step (Eq. 4 as a one-in / one-out update:
 * the newest key joins the kept set, or replaces its worst member if it beats it).  For callers
 * that keep every sequence in a region of fixed capacity: sequence b owns rows
 * [cu_seqlens[b], cu_seqlens[b+1]) of K, V and z and currently fills the first seq_lens[b] of them
 * (clamped to the capacity), the last of these being the new token.
 *   seq_lens in  [n_docs] int32 (device)
 *   refresh  != 0: select the kept sets from all scores, as dma_decode does (the first step, or after
 *            anything but "every non-empty sequence grew by exactly one token" happened);
 *            == 0: `kept` still holds what the previous call left for lengths seq_lens[b] - 1; it is
 *            updated in place in O(k) per (sequence, head) instead of O(n).
 *   q, o, lse, kept, kept_bytes: as for dma_decode; the entries of `kept` are global row indices.
 * The scores of earlier tokens must not change between calls (they depend on each token's own value
 * vector only).  Every other argument and error as for dma_decode.
 */
int dma_decode_step(const dma_shape* shape, const void* q, const void* K, const void* V, const float* z,
                    const int32_t* cu_seqlens, const int32_t* seq_lens, int refresh, void* o, float* lse,
                    int32_t* kept, size_t kept_bytes, void* stream);

/*
 * A paged key/value cache in 4 bits, and decode over it: the cache of a server that holds many requests of different
 * and growing lengths.  Four calls make a step: dma_cache_assign gives the step's new tokens their places, dma_cache_append
 * writes their K, V and content scores there, dma_cache_decode attends from them, and, where a request ends or drafts of it
 * are rejected, the next dma_cache_assign takes their places back.  None of them looks at a length on the host, allocates
 * or synchronises, so a step can be captured in a graph.
 *
 *   pages        dma_cache_bytes(shape) bytes: the pool of n_pages pages of page_size tokens (dma_cache_describe)
 *   block_table  [n_reqs, max_pages] int32: the pages of each request, in order; -1 behind its last one
 *   seq_lens     [n_reqs] int32: cached tokens of each request
 *   free_list    dma_cache_free_bytes(shape) bytes, int32: [0] number of free pages, [4 ...] a stack of them
 *   slots        [n_rows] int32: place of a token, page * page_size + place in the page; below 0: none
 *   row_req      [n_rows] int32: request of a row; below 0: none
 *   row_len      [n_rows] int32: keys that a row sees, the first row_len of its request; 0: none
 * n_rows is the capacity of a step's row arrays, not its number of rows, at most 2^28, and may be 0 (nothing is done, or
 * enqueued, but by dma_cache_assign).  dtype is the type of K, V, q and o; what the cache holds does not depend on it.
 *
 * A token's K (and V) of one kv-head is held as d codes of 4 bits and d / 32 scale bytes (OCP microscaling, e2m1 with e8m0): channel c
 * stands for  code[c] * 2^(byte[c / 32] - 127),  code in {0, 0.5, 1, 1.5, 2, 3, 4, 6} with a sign.  The power of two is the one
 * at which the largest of the 32 rounds to at most 6 (byte 2 to 252), values go to the nearest code, ties to the even one: an
 * error of at most a fifth of the largest value of the 32.  Where the byte is at its limits: at most 2^-127 if the largest value is
 * below 5 * 2^-127 (values up to 2^-127 become 0), and at most a quarter of it from 1.75 * 2^127 on (values end at 6 * 2^125).
 * A block with an infinity or NaN has byte 255 and reads as NaN.
 *
 * Numbers of pages, slots and requests in device memory are checked where they are used: one out of range is a row that is not
 * there, never an address.  Calls that write the same arrays must be ordered by the caller (one stream).
 */
typedef struct {
  int32_t n_reqs;      /* places for requests, 1 to 4096                                        */
  int32_t n_pages;     /* pages of the pool; n_pages * page_size <= 2^30                        */
  int32_t max_pages;   /* pages of one request at most; max_pages * page_size <= 2^30           */
  int32_t page_size;   /* tokens of a page: 16, 32, 64, 128 or 256                              */
  int32_t H_q;         /* query heads                                                           */
  int32_t H_kv;        /* key/value heads, divides H_q                                          */
  int32_t d;           /* head dimension: 64, 128 or 256                                        */
  int32_t dtype;       /* dma_dtype of K, V, q, o                                               */
  int32_t max_len;     /* upper bound on the keys that a row of dma_cache_decode sees (0 => max_pages * page_size).  It chooses
                          between equal ways of working; a bound that is too small costs time but changes no result          */
} dma_cache_shape;

/* Bytes of the pool, of the free list, and of the scratch of one dma_cache_decode; 0 if an argument is invalid. */
size_t dma_cache_bytes(const dma_cache_shape* shape);
size_t dma_cache_free_bytes(const dma_cache_shape* shape);
size_t dma_cache_decode_bytes(const dma_cache_shape* shape, int32_t n_rows, int32_t k);

/* Where things lie in a page, bytes from its start: for kv-head g and place t of the page
 *   K codes  off_codes + ((g * page_size + t) * 2    ) * d / 2,  V codes  ... * 2 + 1 ...   d / 2 bytes each, low nibble first
 *   K scales off_scales + ((g * page_size + t) * 2   ) * d / 32, V scales ... * 2 + 1 ...   d / 32 bytes each
 *   score of q-head h: float at off_scores + (h * page_size + t) * 4
 * Pages are page_bytes apart (a multiple of 256) and hold nothing of each other: one can be copied or moved as a whole. */
typedef struct {
  uint64_t page_bytes, off_codes, off_scales, off_scores;
} dma_cache_layout;
int dma_cache_describe(const dma_cache_shape* shape, dma_cache_layout* out);

/* An empty cache: seq_lens 0, block_table -1, all pages free (the lowest are taken first).  The pool needs no clearing. */
int dma_cache_reset(const dma_cache_shape* shape, int32_t* seq_lens, int32_t* block_table, int32_t* free_list, void* stream);

/*
 * Places for a step.  Request b grows by change[b] tokens, or, below 0, gives back its last -change[b] (at most all it has:
 * INT32_MIN ends it).  The pages given back go on the free list first, then those that grow take theirs.
 *   change     in      [n_reqs]
 *   seq_lens, block_table, free_list   in and out
 *   cu_rows    out     [n_reqs + 1]: the new tokens of request b are the rows cu_rows[b] .. cu_rows[b + 1]
 *   row_req, row_len, slots   out   [n_rows], fully written: -1, 0, -1 for rows behind the last, of requests not served and, should the
 *                      lists be damaged, of tokens whose page is out of range.
 *                      A row sees the keys up to and with its own token: row_len = its position + 1
 *   status     out     [n_reqs]: 0 served, or why not.  A request that is not served keeps its length and pages; its rows keep
 *                      their places among the rows.  Pages are promised in order of the requests: once one does not find enough,
 *                      those behind it that need any are not served either.
 */
typedef enum {
  DMA_CACHE_SERVED = 0,
  DMA_CACHE_NO_PAGES = 1,  /* the free list is too short                     */
  DMA_CACHE_TOO_LONG = 2,  /* more than max_pages pages                      */
  DMA_CACHE_NO_ROWS = 3    /* its rows end behind n_rows                     */
} dma_cache_status;
int dma_cache_assign(const dma_cache_shape* shape, int32_t n_rows, const int32_t* change, int32_t* seq_lens,
                     int32_t* block_table, int32_t* free_list, int32_t* cu_rows, int32_t* row_req, int32_t* row_len,
                     int32_t* slots, int32_t* status, void* stream);

/*
 * Rows into the cache.
 *   K, V   in  n_rows rows of [H_kv, d], k_stride and v_stride elements apart (multiples of 8 of at least H_kv * d: K and V may be parts of
 *              one projection's output)
 *   W, A   in  the score parameters as for dma_mask_gen: the cache gets z = exp(A softplus(w . v)), of V as given, the
 *              scores that dma_mask_gen forms, bit for bit
 *   z      in  if W == NULL: the scores, [H_q, n_rows] (A is then ignored); else ignored.  A score of -infinity takes its key
 *              out of the attention; NaN and +infinity make the rows that keep the key NaN.
 *   slots  in  where each row goes; rows without a slot are left out.  No two rows may have the same slot.
 */
int dma_cache_append(const dma_cache_shape* shape, int32_t n_rows, const void* K, int64_t k_stride, const void* V,
                     int64_t v_stride, const float* W, const float* A, const float* z, const int32_t* slots, void* pages,
                     void* stream);

/*
 * dma_cache_append with rotary positions (dma_rope) on the way: K goes into the cache turned, and the rows' queries are turned in the
 * same call.  The token of row r has the position row_len[r] - 1 (0 if that is below 0) behind the prefix of its request:
 *   row_req     in  nullable (row r is then request r, n_rows <= n_reqs); row_len in, as dma_cache_assign gives them
 *   n_prefixes, prefix_len [n_prefixes], req_prefix [n_reqs]   as for dma_cache_decode_prefix; with n_prefixes == 0 neither is read, nor row_req
 *               A prefix counts with its prefix_len as given (below 0: 0), also beyond max_pages * page_size and whatever request holds it
 *               (prefix_req is not given: for a holder out of range, whose prefix has no tokens there, prefix_len has to be 0); positions
 *               end at 2^31 - 1
 *   Q           in  nullable: n_rows rows of [H_q, d], q_stride elements apart, every row turned, also one without a slot
 *   Qo          out [n_rows, H_q, d]; may be Q if that is packed, else it overlaps no input
 *   freqs, rot, interleaved   as for dma_rope
 * The codes are those of the turned value as 64 bits give it: nothing is rounded before them (rows that dma_rope wrote have been, to their
 * type).  V and the scores, which come from V, are dma_cache_append's bit for bit, and so is everything else.
 */
int dma_cache_append_rope(const dma_cache_shape* shape, int32_t n_rows, const void* Q, int64_t q_stride, const void* K,
                          int64_t k_stride, const void* V, int64_t v_stride, const float* W, const float* A, const float* z,
                          const int32_t* slots, const int32_t* row_req, const int32_t* row_len, int32_t n_prefixes,
                          const int32_t* prefix_len, const int32_t* req_prefix, const float* freqs, int32_t rot,
                          int interleaved, void* Qo, void* pages, void* stream);

/*
 * Rows out of the cache, for the entry points over plain K, V and z (dma_mask_gen with W == NULL, dma_fwd, dma_decode).
 *   K, V   out [n_rows, H_kv, d]: the values that the codes stand for, exact in either dtype
 *   z      out [H_q, n_rows].  Rows without a slot: K = V = 0, z = -infinity.
 */
int dma_cache_read(const dma_cache_shape* shape, int32_t n_rows, const int32_t* slots, const void* pages, void* K, void* V,
                   float* z, void* stream);

/*
 * Decode over the cache: row r keeps the min(k, n) best of the first n = row_len[r] keys of its request by (z descending,
 * position ascending) and attends to them (Eq. 4-6), with the arithmetic of the values that dma_cache_read returns.  Several
 * rows of a request, each with its own length, are independent (drafts, the end of a prompt).
 *   q        in  n_rows rows of [H_q, d], q_stride elements apart (a multiple of 8 of at least H_q * d)
 *   row_req  in  nullable: row r is then request r (n_rows <= n_reqs), and seq_lens may serve as row_len
 *   softmax_scale  0 => d^-1/2
 *   o        out [n_rows, H_q, d];  lse out [H_q, n_rows], natural log.  A row that sees nothing (no request, no keys, or a page out
 *                of range among its own), or nothing but scores of -infinity: o = 0, lse = -infinity
 *   kept     out [n_rows, H_q, min(k, max_pages * page_size)] int32: the slots of the kept keys in order of position, -1 behind
 *                them
 *   ws       dma_cache_decode_bytes(shape, n_rows, k) bytes of scratch (NULL if that is 0); calls that overlap need one each.  At most
 *                261 MiB, reached at 8192 heads of rows where max_len allows rows of more than 12288 keys, else below 1 MiB; more
 *                rows never need less, so the scratch of the largest step serves all
 * DMA_EUNSUPPORTED where (n_rows + 8) * H_q * ceil(min(k, max_pages * page_size) / 256) reaches 2^22: a whole prompt goes through
 * dma_mask_gen and dma_fwd.
 */
int dma_cache_decode(const dma_cache_shape* shape, int32_t n_rows, int32_t k, float softmax_scale, const void* q,
                     int64_t q_stride, const void* pages, const int32_t* block_table, const int32_t* row_req,
                     const int32_t* row_len, void* o, float* lse, int32_t* kept, void* ws, size_t ws_bytes, void* stream);

/*
 * Decode for requests that share prefixes.  A prefix (a system prompt, a document that many ask about) lies in the cache once, as the
 * tokens of a request of its own; a request behind it holds only what comes after.  Row r sees the tokens of its request's prefix and then the
 * first row_len[r] of its own, and keeps the min(k, n) best of all n of them by (z descending, position ascending, the prefix's first): what
 * dma_cache_decode would make of one request with all the tokens.
 *   n_prefixes   number of prefixes, at most 4096
 *   max_prefix   upper bound on their lengths (0 => max_pages * page_size).  Like shape->max_len, the bound on a row's own keys, it chooses
 *                between equal ways of working; one that is too small costs time but changes no result
 *   prefix_req   in [n_prefixes] int32: the request that holds each; one out of range is a prefix without tokens
 *   prefix_len   in [n_prefixes] int32: its tokens (their number may be less than that request has; beyond max_pages * page_size a row sees
 *                the first max_pages * page_size)
 *   req_prefix   in [n_reqs] int32: the prefix of each request, 0 to n_prefixes - 1; any other value: none.  (A prefix of a prefix is not
 *                looked at.)  The last three are not read if n_prefixes is 0
 *   q, q_stride, pages, block_table, row_req, row_len, softmax_scale, o, lse   as for dma_cache_decode; a row that has no request or no
 *                keys of its own, or a page out of range among its own or its prefix's, sees nothing
 *   ws           dma_cache_decode_prefix_bytes(shape, n_rows, k, n_prefixes, max_prefix) bytes of scratch; calls that overlap need one
 *                each.  Of every row and head it holds the list of its own kept keys, 4 bytes for each of min(k, max_pages * page_size), 8
 *                where max_len allows rows of more than max(k, 2048) keys; of every prefix and head 8 for each; and the parts of the
 *                prefixes' attention, (d + 4) * 4 bytes for each row and head, of at least 8192
 * A prefix is selected from, gathered and decoded once for all of its rows.  The limit on rows is dma_cache_decode's, with n_rows + n_prefixes
 * in the place of n_rows.
 */
size_t dma_cache_decode_prefix_bytes(const dma_cache_shape* shape, int32_t n_rows, int32_t k, int32_t n_prefixes,
                                     int32_t max_prefix);
int dma_cache_decode_prefix(const dma_cache_shape* shape, int32_t n_rows, int32_t k, float softmax_scale, const void* q,
                            int64_t q_stride, const void* pages, const int32_t* block_table, const int32_t* row_req,
                            const int32_t* row_len, int32_t n_prefixes, int32_t max_prefix, const int32_t* prefix_req,
                            const int32_t* prefix_len, const int32_t* req_prefix, void* o, float* lse, void* ws,
                            size_t ws_bytes, void* stream);

/*
 * Per-stage timing aid.  dma_mask_gen, dma_fwd and dma_bwd each launch several kernels, so a
 * caller cannot bracket one of them with events from outside.  `events` is a HOST array of
 * 2 * DMA_N_STAGES hipEvent_t handles (as void*) owned by the caller, or NULL to switch the aid
 * off (the default).  While set -- per host thread -- every entry point records events[2*s] on its
 * stream immediately before stage s and events[2*s + 1] immediately after it.  Nothing is
 * synchronised; the caller reads the events after synchronising the stream itself.  The library
 * keeps the `events` pointer (not a copy of the array) until the next call of this function on the
 * same host thread: the array must stay valid that long.  A measurement aid: the step's results do
 * not depend on it.
 */
typedef enum {
  DMA_STAGE_Z = 0,          /* mask_gen: block table + content scores (Eq. 3)            */
  DMA_STAGE_SORT = 1,       /* mask_gen: selection (Eq. 4): evictions by blocks; or a sort  */
  DMA_STAGE_EXPIRY = 2,     /* mask_gen: expiry of every key, after a sort (else empty)   */
  DMA_STAGE_PLAN = 3,       /* mask_gen: expiries, slots, slot table, partial lists, topk_idx       */
  DMA_STAGE_FWD = 4,        /* fwd: the attention kernel                                  */
  DMA_STAGE_BWD_ZERO = 5,   /* bwd: (empty: the dQ stage clears the fp32 accumulators)   */
  DMA_STAGE_BWD_DQ = 6,     /* bwd: D and dQ (query-stationary)                           */
  DMA_STAGE_BWD_DKV = 7,    /* bwd: dK, dV, dz (key-stationary)                           */
  DMA_STAGE_BWD_PART = 8,   /* bwd: (empty: the DKV stage has the partial lists too)      */
  DMA_STAGE_BWD_CVT = 9,    /* bwd: fp32 accumulators -> output dtype                     */
  DMA_N_STAGES = 10
} dma_stage;
void dma_profile_events(void** events);

const char* dma_strerror(int status);
int dma_version(void);

#ifdef __cplusplus
}
#endif
#endif /* DMA_H_ */
