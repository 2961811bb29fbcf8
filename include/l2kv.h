/*
 * l2kv -- L2-norm KV-cache compression and decode attention for AMD MI355X
 * (CDNA4, gfx950).  C ABI of libl2kv.so.
 *
 * Method: arXiv 2406.11430, "A Simple and Effective L2 Norm-Based Strategy for
 * KV Cache Compression".  Its rule (Sec. 1, Sec. 3): per layer and head, keep
 * the cached keys with the lowest L2 norm together with their values and drop
 * the rest; decoding then runs ordinary scaled dot-product attention (Eq. 2,
 * in the decode form of Eq. 4) over the smaller cache.
 *
 * Conventions shared by every call
 * --------------------------------
 *  - All tensor pointers are DEVICE pointers unless a parameter name starts
 *    with h_.  The caller owns every buffer; the library never allocates,
 *    frees, synchronises or copies to the host.
 *  - Every call only enqueues work on `stream` (a hipStream_t passed as
 *    void*; NULL = the default stream) and returns.
 *  - Arguments are validated on the host BEFORE anything is enqueued; a
 *    negative status means nothing was launched and no device memory was
 *    touched.  L2KV_ERR_LAUNCH wraps a failed kernel launch.
 *  - "Head" means one (layer, sequence, KV head) triple.  The rule is
 *    independent per layer and head (Eq. 5: the dropped set D_{l,h}), so any
 *    number of layers / sequences can be flattened into n_heads.
 *  - A K or V row is D contiguous elements; head i starts `head_stride`
 *    ELEMENTS after head i-1 (head_stride >= T*D).  Supported:
 *    D in {64, 128} for fp32 and bf16, D = 256 for bf16 only (rows of at most
 *    512 bytes).  Base pointers of K, V, Kc, Vc, Q
 *    must be 16-byte aligned and head_stride*sizeof(elem) a multiple of 16;
 *    norms / index / O / workspace pointers 4-byte aligned (workspace 16).
 *  - Outputs must not alias inputs.
 *  - Placement (performance only, no entry point allocates): on MI355X the
 *    288 GiB of device memory behave as three regions of 96 GiB, and a launch
 *    that streams its K rows from one region and its V rows from another
 *    runs about 9 % slower than one whose two streams share a region.  Keep
 *    the K and the V cache of a layer in one allocation, made early.
 *  - Global state of the library: a per-device cache of the compute-unit
 *    count and, for l2kv_decode_attn_static only, the per-device address of
 *    its scratch array.  No call changes a kernel attribute or a device
 *    setting.  Calls are thread-safe as long as they do not share a workspace.
 */
#ifndef L2KV_H
#define L2KV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { L2KV_F32 = 0, L2KV_BF16 = 1 } l2kv_dtype;

typedef enum {
    L2KV_OK = 0,
    L2KV_ERR_NULL = -1,      /* a required pointer is NULL                     */
    L2KV_ERR_SHAPE = -2,     /* a size is <= 0, too large, or D unsupported    */
    L2KV_ERR_DTYPE = -3,     /* dtype is not L2KV_F32 / L2KV_BF16              */
    L2KV_ERR_RATIO = -4,     /* keep_ratio outside (0, 1] or not finite        */
    L2KV_ERR_WORKSPACE = -5, /* workspace NULL or smaller than *_workspace_bytes */
    L2KV_ERR_ALIGN = -6,     /* pointer or stride alignment violated           */
    L2KV_ERR_LAUNCH = -7     /* the HIP runtime refused a launch               */
} l2kv_status;

/* Eviction strategy.  LOWEST is the paper's method; HIGHEST is the control of
 * Sec. 4 (the highest-norm tokens are the ones kept). */
typedef enum { L2KV_KEEP_LOWEST = 0, L2KV_KEEP_HIGHEST = 1 } l2kv_mode;

/*
 * Number of rows kept out of T at keep_ratio r: k = ceil(r*T), clamped to
 * [1, T]; a product r*T within 1e-9 relative of an integer counts as that
 * integer (so 0.55*100 -> 55).  The paper fixes only that the count is exact
 * (|D_{l,h}| = m, Eq. 5) and quotes "compression ratios" X (Sec. 4), which
 * are r = 1 - X.  Host function; returns 0 for T <= 0 or r outside (0,1].
 */
int64_t l2kv_keep_count(int64_t T, double keep_ratio);

/*
 * Squared L2 norm of every cached key (the quantity the rule of Sec. 1 /
 * Sec. 3 ranks by; the square keeps the order and needs no sqrt):
 *     norms[i][t] = sum_d K[i][t][d]^2          fp32
 * summed in a fixed order so the result is reproducible bit for bit: the row
 * is cut into 16 chunks of D/16 consecutive elements, each chunk is summed
 * left to right, and the 16 partial sums are added as a balanced binary tree
 * over neighbours; every product and sum is rounded to fp32 separately.
 *   K      in : n_heads slabs of T rows (layout above), read once
 *   norms  out: [n_heads][T] fp32, dense
 * Errors: NULL, SHAPE (n_heads, T <= 0; T > 2^31-1; D; head_stride < T*D),
 * DTYPE, ALIGN, LAUNCH.
 */
l2kv_status l2kv_norms(const void* K, l2kv_dtype dt, int64_t n_heads, int64_t T,
                       int32_t D, int64_t head_stride, float* norms, void* stream);

/*
 * Selection (the eviction rule of Sec. 1: the lowest-norm keys stay in the
 * cache; Eq. 5: exactly m pairs dropped per layer and head).  For every head, the
 * k = l2kv_keep_count(T, keep_ratio) positions that come first in the total
 * order (uint32 bit pattern of the fp32 squared norm, token index) -- ties go
 * to the lower token index -- written in ascending token order.
 *   norms      in : [n_heads][T] fp32 (>= +0; +Inf / NaN patterns sort last)
 *   kept_idx   out: [n_heads][k] int32, strictly ascending per head
 *   kept_count out: [n_heads] int32, every entry = k; may be NULL
 *   workspace     : l2kv_select_workspace_bytes(n_heads, T) bytes, 16-aligned;
 *                   contents need not be initialised and are undefined after.
 *                   For a few long heads (at most 64, beyond 32768 tokens)
 *                   several workgroups share a head through it; two calls
 *                   whose queried size is above 256 must therefore not use one
 *                   workspace at the same time, on other streams either.  Any
 *                   size from 256 bytes on is accepted: below the queried size
 *                   every head is selected by one workgroup, which does not
 *                   touch the buffer.
 * Errors: NULL, SHAPE, RATIO, WORKSPACE, ALIGN, LAUNCH.
 */
l2kv_status l2kv_select(const float* norms, int64_t n_heads, int64_t T,
                        double keep_ratio, int32_t* kept_idx, int32_t* kept_count,
                        void* workspace, size_t workspace_bytes, void* stream);

/* Same with an explicit kept count k (1 <= k <= T) and strategy.  HIGHEST
 * orders by descending norm, ties again to the lower token index. */
l2kv_status l2kv_select_k(const float* norms, int64_t n_heads, int64_t T,
                          int64_t k, l2kv_mode mode, int32_t* kept_idx,
                          int32_t* kept_count, void* workspace,
                          size_t workspace_bytes, void* stream);

size_t l2kv_select_workspace_bytes(int64_t n_heads, int64_t T);

/*
 * Keys for the keep-random control of Sec. 4 (a random subset of the tokens
 * is kept):
 * keys[i][t] receives, as a 32-bit pattern stored in an fp32 array, the hash
 *     x = t*0x9E3779B1 + i*0x85EBCA77 + seed   (mod 2^32)
 *     x ^= x>>16; x *= 0x85EBCA6B; x ^= x>>13; x *= 0xC2B2AE35; x ^= x>>16
 * (the 32-bit finalizer of MurmurHash3).  l2kv_select_k orders by bit pattern,
 * so running it on these keys instead of norms keeps k pseudo-random tokens per
 * head, reproducibly.  keys out: [n_heads][T].  Errors: NULL, SHAPE, ALIGN, LAUNCH.
 */
l2kv_status l2kv_random_keys(int64_t n_heads, int64_t T, uint32_t seed, float* keys, void* stream);

/*
 * Compaction (Sec. 1: the values of the kept keys stay with them): the kept rows of K
 * and of V copied, byte for byte and in the order of kept_idx, into dense
 * caches:
 *     Kc[i][j][:] = K[i][kept_idx[i][j]][:],   Vc likewise.
 *   K, V     in : n_heads slabs of T rows (layout above); dropped rows are
 *                 never read.  V may be NULL together with Vc (K only).
 *   kept_idx in : [n_heads][k] int32, every entry in [0, T) (an entry outside
 *                 that range is forced into it on the device: a wrong row is
 *                 copied, nothing is read outside the head)
 *   Kc, Vc   out: [n_heads][k][D], dense
 * Errors: NULL, SHAPE (k <= 0, k > T, ...), DTYPE, ALIGN, LAUNCH.
 */
l2kv_status l2kv_compact(const void* K, const void* V, l2kv_dtype dt,
                         const int32_t* kept_idx, int64_t n_heads, int64_t T,
                         int64_t k, int32_t D, int64_t head_stride,
                         void* Kc, void* Vc, void* stream);

/*
 * The whole compression step (the rule of Sec. 1 as one operation: keep the
 * lowest-norm keys and their values) in one call: l2kv_norms, l2kv_select and
 * l2kv_compact enqueued back to back on `stream`, with the same results as the
 * three separate calls.
 *   slab_heads : 0 = all heads at once (three launches; one or two for short
 *                heads, five for a few long ones).  > 0 = the three
 *                steps are enqueued slab by slab of that many consecutive
 *                heads, so that the compaction's second read of
 *                the kept K rows of a slab can be served by the caches while
 *                the slab still fits them.  On an MI355X this is SLOWER than
 *                slab_heads = 0 at the shapes measured (a slab of a few heads
 *                leaves most of the chip idle during its selection, and every
 *                launch costs); the mode exists so that the trade can be
 *                measured.
 *   norms      out: [n_heads][T] fp32 (needed as scratch; left filled)
 *   kept_idx   out: [n_heads][k], k = l2kv_keep_count(T, keep_ratio)
 *   Kc, Vc     out: [n_heads][k][D] (scratch memory of the selection before
 *                they are filled)
 *   workspace     : at least 256 bytes, 16-aligned, as for l2kv_select of the
 *                same heads; not touched, so calls may share it
 * Errors: NULL, SHAPE, DTYPE, RATIO, WORKSPACE, ALIGN, LAUNCH (a launch failure
 * part-way leaves the earlier slabs done).
 */
l2kv_status l2kv_compress(const void* K, const void* V, l2kv_dtype dt, int64_t n_heads,
                          int64_t T, int32_t D, int64_t head_stride, double keep_ratio,
                          int64_t slab_heads, float* norms, int32_t* kept_idx, void* Kc,
                          void* Vc, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Decode attention (Eq. 2 for a single query row; Eq. 4: the query attends to
 * every row of the cache it is handed, the current token's row included by
 * the caller).  For each sequence b and query head hq, with KV head
 * hkv = hq / (Hq/Hkv) (consecutive query heads share a KV head):
 *     O[b][hq][:] = softmax_j( scale * Q[b][hq] . Kc[b][hkv][j] ) . Vc[b][hkv]
 * over j in [0, kv_len).  No mask.  Scores are never written to memory: the
 * cache is streamed once per KV head for all Hq/Hkv query heads, split over
 * row ranges with an online softmax, and the partial results are merged.
 *   Q   in : [B][Hq][D], dtype dt
 *   Kc,Vc in: (b,hkv) slab starts (b*Hkv+hkv)*kv_head_stride elements in;
 *             kv_len rows of D
 *   scale  : softmax scale; <= 0 selects 1/sqrt(D) (Eq. 2)
 *   O   out: [B][Hq][D] fp32
 *   workspace: l2kv_decode_workspace_bytes(B, Hq, kv_len, D) bytes,
 *              16-aligned.  It starts with one arrival counter per
 *              (sequence, KV head) followed by the split partials.  The
 *              counters must be ZERO before the first call that uses this
 *              buffer (zero-fill the whole buffer once); every call leaves
 *              them zero again, so the buffer can be reused call after call
 *              for any shape it is large enough for.  Two calls that share a
 *              workspace must not overlap in time.
 * The rows need not have been compacted: an uncompressed layer is attended to
 * in place by passing the original cache and kv_len = T.
 * Arithmetic: fp32 accumulation throughout; for bf16 caches q.k is formed with
 * the packed bf16 dot instruction (exact bf16 products, fp32 sum), for fp32
 * caches with fp32 FMAs; softmax and the value sum are fp32.  (Where several
 * workgroups share a head, a partial value sum below 2^-141 counts as zero.)
 * Errors: NULL, SHAPE (Hq % Hkv != 0, Hq/Hkv > 8 -- > 4 for D = 256 --,
 * kv_len <= 0, ...), DTYPE, WORKSPACE, ALIGN, LAUNCH.
 */
l2kv_status l2kv_decode_attn(const void* Q, const void* Kc, const void* Vc,
                             l2kv_dtype dt, int32_t B, int32_t Hq, int32_t Hkv,
                             int64_t kv_len, int32_t D, int64_t kv_head_stride,
                             float scale, float* O, void* workspace,
                             size_t workspace_bytes, void* stream);

/* Same with the element type of O chosen by the caller: L2KV_F32 (O is float*,
 * identical to l2kv_decode_attn) or L2KV_BF16 (O is [B][Hq][D] bf16, 2-byte
 * aligned: the fp32 result rounded to nearest even once, at the very end).
 * Errors: as l2kv_decode_attn; DTYPE also for an unknown out_dt. */
l2kv_status l2kv_decode_attn_out(const void* Q, const void* Kc, const void* Vc,
                                 l2kv_dtype dt, int32_t B, int32_t Hq, int32_t Hkv,
                                 int64_t kv_len, int32_t D, int64_t kv_head_stride,
                                 float scale, l2kv_dtype out_dt, void* O, void* workspace,
                                 size_t workspace_bytes, void* stream);

/* Same with the number of row ranges per KV head chosen by the caller
 * (1 <= n_splits <= l2kv_decode_max_splits(kv_len); 0 = library default).
 * The result does not depend on n_splits beyond fp32 rounding. */
l2kv_status l2kv_decode_attn_splits(const void* Q, const void* Kc, const void* Vc,
                                    l2kv_dtype dt, int32_t B, int32_t Hq, int32_t Hkv,
                                    int64_t kv_len, int32_t D, int64_t kv_head_stride,
                                    float scale, int32_t n_splits, float* O,
                                    void* workspace, size_t workspace_bytes,
                                    void* stream);

int32_t l2kv_decode_max_splits(int64_t kv_len);

/* Zero-fills a decode workspace with a small kernel on `stream` (the "zero
 * before first use" of l2kv_decode_attn; safe under graph capture, where a
 * memset node is not).  workspace_bytes: the size from
 * l2kv_decode_workspace_bytes (always a multiple of 16).
 * Errors: NULL, WORKSPACE (size 0 or not a multiple of 16), ALIGN, LAUNCH. */
l2kv_status l2kv_decode_workspace_init(void* workspace, size_t workspace_bytes, void* stream);
size_t  l2kv_decode_workspace_bytes(int32_t B, int32_t Hq, int64_t kv_len, int32_t D);

/*
 * l2kv_decode_attn for callers that cannot allocate device memory or pass a
 * workspace: code under HIP graph capture, tight serving loops, harnesses that
 * forbid hipMalloc.  Same arguments, same kernels, same result as
 * l2kv_decode_attn, but the arrival counters and split partials live in a
 * scratch array inside the library (L2KV_STATIC_SCRATCH_BYTES of device memory
 * per GPU, held until the process ends).  The call itself allocates and frees
 * nothing and records no memset.
 *   Limit: counters (4 bytes per (sequence, KV head), padded to 256) plus
 *   B*Hq*(workgroups per KV head)*(D+4)*4 bytes of partials must fit the
 *   scratch array; larger shapes return L2KV_ERR_WORKSPACE and launch nothing.
 *   (32k-context batch of 4 x 32 query heads: 0.4 MB.)
 *   All calls on one GPU share that GPU's array: two calls that may overlap in
 *   time (different streams without an ordering between them, or two host
 *   threads) race and give wrong results; calls ordered on one stream are fine.
 *   The first call on a device looks the array up and enqueues one small fill
 *   kernel on `stream`; make that first call outside graph capture.
 * Errors: as l2kv_decode_attn, L2KV_ERR_WORKSPACE for a shape beyond the limit,
 * L2KV_ERR_LAUNCH if the array cannot be located on the current device.
 */
#define L2KV_STATIC_SCRATCH_BYTES (4u << 20)
l2kv_status l2kv_decode_attn_static(const void* Q, const void* Kc, const void* Vc,
                                    l2kv_dtype dt, int32_t B, int32_t Hq, int32_t Hkv,
                                    int64_t kv_len, int32_t D, int64_t kv_head_stride,
                                    float scale, float* O, void* stream);

/* ------------------------------------------------------------------------
 * Ragged batches and streaming eviction.
 *
 * Sec. 4 ("Language Modelling Tasks"): the cache is allowed to grow to a
 * pre-defined length, after which the tokens with the highest key norm are
 * discarded.  A batch of sequences of different lengths is held ragged:
 *
 *   prompt tensors   K, V [n_planes][total_tokens][D], norms [n_planes][total_tokens];
 *                    sequence s = rows in_offsets[s] .. in_offsets[s+1]-1 of every plane
 *   slot cache       Kc, Vc [n_planes][total_slots][D], norms_c [n_planes][total_slots] fp32,
 *                    pos_c [n_planes][total_slots] int32 (original token id of each slot);
 *                    sequence s owns slots slot_offsets[s] .. slot_offsets[s+1]-1 of every
 *                    plane, of which the first lens[s] are occupied (same count in all planes)
 *
 * n_planes = layers x KV heads (plane = layer*Hkv + head).  All offset arrays
 * are DEVICE int64 [n_seq+1], ascending, first entry 0; lens / budgets /
 * token_ids are DEVICE int32 [n_seq].  Their contents cannot be checked on the
 * host: the kernels clamp what they read so that nothing is accessed outside
 * the buffers described by total_tokens / total_slots, but inconsistent
 * arrays give meaningless results.  Slot order inside a sequence carries no
 * meaning (attention is order-free); after l2kv_compact_ragged it is ascending
 * token order, evictions then move the last slot into the hole.
 * ------------------------------------------------------------------------ */

/*
 * Selection on a ragged batch: for every plane and sequence, the
 * k_s = out_offsets[s+1]-out_offsets[s] positions with the lowest (norm bits,
 * position) among its T_s = in_offsets[s+1]-in_offsets[s] tokens (k_s is capped
 * at T_s; the caller normally sets it with l2kv_keep_count(T_s, keep_ratio)).
 * Positions are relative to the sequence start, ascending.
 *   kept_idx out: [n_planes][total_kept] int32, sequence s at out_offsets[s]
 *   max_len     : an upper bound of all T_s (chooses the kernel variant; tokens
 *                 of a sequence beyond it would be ignored)
 * Errors: NULL, SHAPE, ALIGN, LAUNCH.
 */
l2kv_status l2kv_select_ragged(const float* norms, int32_t n_planes, int32_t n_seq,
                               int64_t total_tokens, const int64_t* in_offsets,
                               const int64_t* out_offsets, int64_t total_kept, int64_t max_len,
                               l2kv_mode mode, int32_t* kept_idx, void* stream);

/*
 * Compaction of a ragged batch into the slot cache: slot j of sequence s gets
 * row kept_idx[..][j] of that sequence (K, V, its norm, and the position as
 * token id).  Sets up the cache that l2kv_stream_* and l2kv_decode_attn_ragged
 * work on; lens[s] = k_s is the caller's to fill.  k_s is capped at the
 * sequence's slot capacity.  max_kept: an upper bound of all k_s (checked against
 * total_kept; the launch itself is sized by total_kept).
 * Errors: NULL, SHAPE, DTYPE, ALIGN, LAUNCH.
 */
l2kv_status l2kv_compact_ragged(const void* K, const void* V, const float* norms, l2kv_dtype dt,
                                const int32_t* kept_idx, int32_t n_planes, int32_t n_seq,
                                int64_t total_tokens, const int64_t* in_offsets,
                                const int64_t* out_offsets, int64_t total_kept, int64_t max_kept,
                                const int64_t* slot_offsets, int64_t total_slots, int32_t D,
                                void* Kc, void* Vc, float* norms_c, int32_t* pos_c, void* stream);

/*
 * Append the current token of every sequence (Eq. 4: its K_t, V_t join the
 * cache before the query attends): Knew, Vnew [n_layers][n_seq][Hkv][D] go to
 * slot lens_in[s] of sequence s in plane layer*Hkv+head, with the squared key
 * norm (same fixed summation order as l2kv_norms) and token_ids[s].
 * lens_out[s] = lens_in[s] + 1; a sequence whose slots are all occupied is left
 * unchanged (lens_out[s] = lens_in[s]).  lens_out must not be lens_in.
 * Errors: NULL, SHAPE, DTYPE, ALIGN, LAUNCH.
 */
l2kv_status l2kv_stream_append(const void* Knew, const void* Vnew, l2kv_dtype dt, int32_t n_layers,
                               int32_t n_seq, int32_t Hkv, int32_t D, const int32_t* token_ids,
                               const int64_t* slot_offsets, int64_t total_slots,
                               const int32_t* lens_in, int32_t* lens_out, void* Kc, void* Vc,
                               float* norms_c, int32_t* pos_c, void* stream);

/*
 * Evict down to the budget: in every plane, while sequence s holds more than
 * budgets[s] slots, the slot with the largest (norm bits, token id) is dropped
 * (among equal norms the later token goes first -- the reverse of the keep
 * order of l2kv_select) and the last slot is moved into its place.
 * lens_out[s] = min(lens_in[s], budgets[s]).  lens_out must not be lens_in.
 * With a fixed budget the kept token set equals l2kv_select over all tokens
 * seen; with budgets[s] = l2kv_keep_count(tokens seen, keep_ratio) it is the
 * keep_ratio "enforced incrementally".
 * Errors: NULL, SHAPE, DTYPE, ALIGN, LAUNCH.
 */
l2kv_status l2kv_stream_evict(l2kv_dtype dt, int32_t n_planes, int32_t n_seq, int32_t D,
                              const int64_t* slot_offsets, int64_t total_slots,
                              const int32_t* lens_in, const int32_t* budgets, int32_t* lens_out,
                              void* Kc, void* Vc, float* norms_c, int32_t* pos_c, void* stream);

/*
 * Decode attention over ONE layer of the slot cache: Q [n_seq][Hq][D]; Kc, Vc
 * point at that layer's Hkv planes ([Hkv][total_slots][D]); sequence s attends
 * to its lens[s] occupied slots (0 slots give a zero output row).
 *   seq_order: a DEVICE int32 [n_seq] permutation of 0..n_seq-1 giving
 *             the order in which the sequences are launched; with the longest
 *             sequence first (l2kv_length_order) the library hands
 *             (sequence, KV head) pairs, longest first and in pieces where the
 *             first is much longer than a workgroup's share, to one workgroup per
 *             compute unit, whichever is free next (a work list in the
 *             workspace), which is faster on batches of mixed lengths (bf16
 *             caches with heads of 128 elements; other row sizes are launched
 *             as a grid in the given order).  It only steers scheduling:
 *             outputs land at the sequence's own rows of O in any case.  An
 *             array that is not a permutation computes some sequences twice
 *             and others not at all (entries are forced into 0..n_seq-1); the
 *             workspace is left ready for the next call all the same.
 *             The order may be stale (lengths change from step to step).
 *             NULL: batches of 2..512 sequences whose longest has 2048 rows or
 *             more (bf16, D = 128) get a longest-first order worked out inside the call (one
 *             small extra kernel, about 7 us per call on an MI355X); all other
 *             batches are launched in batch order.  Either way the call is
 *             made of plain kernel launches and may be captured into a graph.
 *   max_len : an upper bound of all lens[s] (sizes the workspace and, but for
 *             batches with an order, the decomposition; rows beyond it are still
 *             attended to)
 * A layer that is left uncompressed (Sec. 4 skips the first layers by default)
 * needs no copy at all: pass its prompt tensors as Kc, Vc with slot_offsets =
 * the prompt offsets, total_slots = total_tokens and lens[s] = T_s.  Per-head
 * keep counts (the outlook of Sec. 8) are the same call with every (sequence,
 * KV head) laid out as one "sequence" of a single plane (Hkv = 1, Hq = the
 * query group), as produced by l2kv_select_ragged / l2kv_compact_ragged with one
 * k per head.
 *   n_splits: 0 = library default
 *   workspace: l2kv_decode_ragged_workspace_bytes(n_seq, Hq, max_len, D) bytes
 *              (the uniform workspace plus room for that order), same
 *              zero-before-first-use contract as l2kv_decode_attn
 * Errors: as l2kv_decode_attn.
 */
l2kv_status l2kv_decode_attn_ragged(const void* Q, const void* Kc, const void* Vc, l2kv_dtype dt,
                                    int32_t n_seq, int32_t Hq, int32_t Hkv, int32_t D,
                                    const int32_t* lens, const int64_t* slot_offsets,
                                    const int32_t* seq_order, int64_t total_slots, int64_t max_len,
                                    float scale, int32_t n_splits, float* O, void* workspace,
                                    size_t workspace_bytes, void* stream);

/*
 * Longest-first order of a batch: order[r] = the sequence with the r-th largest
 * lens (equal lengths: lower index first).  lens, order: DEVICE int32 [n_seq],
 * distinct arrays; n_seq <= 65535.  A set-up call (one workgroup, quadratic in
 * n_seq); its result can serve many decode steps.
 * Errors: NULL, SHAPE, ALIGN, LAUNCH.
 */
l2kv_status l2kv_length_order(const int32_t* lens, int32_t n_seq, int32_t* order, void* stream);

size_t l2kv_decode_ragged_workspace_bytes(int32_t n_seq, int32_t Hq, int64_t max_len, int32_t D);

/* ---------------------------------------------------------------------------
 * Before and beside the compressed cache: rotary positions, attention of whole
 * prompts, drafted trees.
 *
 * Tokens of several sequences are packed: sequence s = tokens
 * offsets[s] .. offsets[s+1]-1 of every tensor (DEVICE int64 [n_seq+1],
 * ascending, first entry 0; sequences may be empty; tokens behind the last one have
 * no effect and nothing is written for them).  As above, contents of device arrays cannot be
 * checked on the host: the kernels force what they read into the buffers.
 * Q, K and V of a token are heads of D contiguous elements, a token's heads side by
 * side; the *_stride arguments are the ELEMENTS between two tokens (>= heads*D,
 * a multiple of 16 bytes), so the three may be parts of one projection's output.
 * What a call writes must not overlap what it reads.
 * ------------------------------------------------------------------------ */

/* Which two elements of a head are turned together, of the first rot_dim = R:
 * HALF (i, i + R/2), INTERLEAVED (2i, 2i + 1), i = 0 .. R/2-1. */
typedef enum { L2KV_ROTARY_HALF = 0, L2KV_ROTARY_INTERLEAVED = 1 } l2kv_rotary_layout;

/* Frequencies for contexts `factor` times longer than the original:
 * PLAIN    f_i = base^(-2i/R)
 * LINEAR   f_i / factor (positions are interpolated)
 * BASE     base raised to base * factor^(R/(R-2)): the last pair slows down by
 *          the factor, the first not at all
 * BANDS    pairs that turn at least `high` times over original_len keep f_i, those
 *          that turn at most `low` times take f_i / factor, between them a
 *          linear ramp in the number of turns */
typedef enum { L2KV_ROTARY_PLAIN = 0, L2KV_ROTARY_LINEAR = 1, L2KV_ROTARY_BASE = 2, L2KV_ROTARY_BANDS = 3 } l2kv_rotary_scaling;

/*
 * The angles per position of the R/2 pairs, in radians (host function, to be
 * copied to the device once).  rot_dim: a multiple of 16, 16..256; base > 0;
 * factor > 0 is not read for PLAIN, original_len > 0 and 0 <= low < high for BANDS only.
 * Errors: NULL, SHAPE.
 */
l2kv_status l2kv_rotary_freqs(int32_t rot_dim, double base, l2kv_rotary_scaling scaling, double factor,
                              int64_t original_len, double low, double high, double* h_freqs);

/*
 * Rotary positions on the way into the cache: l2kv_stream_append for any number
 * of tokens per sequence and one layer, with the rotation in it.  Token t at
 * position p = positions[t] has the pairs (x1, x2) of every query and key head
 * turned by theta = p * freqs[i]:
 *     x1' = amplitude * (x1 cos theta - x2 sin theta)
 *     x2' = amplitude * (x2 cos theta + x1 sin theta)
 * in fp64, rounded to fp32 and for bf16 from there (as a conversion by way of float
 * does); elements from rot_dim on, and V, are copied.
 *   Q, K, V    in : [total_tokens] x Hq, Hkv, Hkv heads; Q may be NULL together
 *                   with Qr (keys and values only; Hq and q_stride are not read)
 *   positions  in : DEVICE int32 [total_tokens], of either sign
 *   freqs      in : DEVICE double [rot_dim/2]
 *   Qr        out : [total_tokens][Hq][D], dense
 *   Kc, Vc    out : [Hkv][total_slots][D]; norms_c, pos_c [Hkv][total_slots]:
 *                   squared norm of the key AS STORED, summed as in
 *                   l2kv_norms, and positions[t]
 *   token_offsets, slot_offsets, lens_in: the j-th token of sequence s goes to
 *                   slot lens_in[s] + j of the sequence; a token that finds its
 *                   sequence's slots occupied is not stored (its queries are turned
 *                   all the same).  lens_out[s] = lens_in[s] + tokens stored; may be
 *                   NULL (calls for further layers), must not be lens_in.
 *                   All four NULL, n_seq not read: token t goes to row t of every
 *                   plane (prompts, packed as they are; nodes of drafted trees).
 * Errors: NULL (also for one of the three arrays without the others), SHAPE
 * (rot_dim not a multiple of 16 or above D, layout, total_slots < total_tokens
 * without offsets, amplitude not finite, more than 2^24-1 workgroups of four tokens or more, ...), DTYPE, ALIGN, LAUNCH.
 */
l2kv_status l2kv_rotary_append(const void* Q, const void* K, const void* V, l2kv_dtype dt, int64_t total_tokens,
                               int32_t Hq, int32_t Hkv, int32_t D, int64_t q_stride, int64_t k_stride,
                               int64_t v_stride, const int32_t* positions, const double* freqs, int32_t rot_dim,
                               l2kv_rotary_layout layout, double amplitude, int32_t n_seq,
                               const int64_t* token_offsets, const int64_t* slot_offsets,
                               const int32_t* lens_in, int32_t* lens_out, int64_t total_slots, void* Qr,
                               void* Kc, void* Vc, float* norms_c, int32_t* pos_c, void* stream);

/*
 * Causal attention of packed prompts (Eq. 2 with the mask of a decoder): query i of
 * the n_q tokens of sequence s attends to its rows j <= i + n_kv - n_q, that is,
 * the last query sees all n_kv rows and the first ones of a prompt, or all that
 * was in the cache before, are seen by every query.  n_kv may be larger than n_q (a further chunk of
 * a prompt, over a cache that may have been compressed) or smaller (the
 * first queries then see nothing).  A query that sees no row, or whose scores are all
 * minus infinity, gets zeros.  Rows that a query does not see have no effect on
 * it, whatever they hold.
 *   Q    in : [total_q] x Hq heads
 *   K, V in : KV head h starts h * kv_head_stride elements in; sequence s has rows
 *             kv_offsets[s] on, n_kv = kv_lens[s] of them, or up to
 *             kv_offsets[s+1] where kv_lens is NULL (always at most up to there).
 *             total_rows: rows that can be read from the start of every head.
 *             Planes [Hkv][total_rows][D]: kv_head_stride = total_rows * D.
 *             Caches [B][Hkv][T][D]: kv_head_stride = T*D, kv_offsets[b] = b*Hkv*T,
 *             kv_lens[b] <= T or NULL (all T), total_rows = ((B-1)*Hkv + 1) * T.
 *             With several KV heads a sequence has at most kv_head_stride / D rows,
 *             whatever offsets and lengths say: its rows of the next head follow.
 *   max_kv  : an upper bound of all n_kv, at least 1 (sizes the workspace and the
 *             decomposition; rows beyond it are still attended to)
 *   scale   : softmax scale; <= 0 selects 1/sqrt(D)
 *   O   out : [total_q][Hq][D], dense, of type dt
 *   workspace: l2kv_prompt_attn_workspace_bytes(...) bytes, 16-aligned; contents
 *             irrelevant before and after, one per call that may run at the same
 *             time.  May be NULL where that is 0.
 *             The size does NOT grow with the arguments: few tokens over many rows need
 *             room for parts, many of them none.  A buffer for calls of several sizes
 *             has the largest of theirs, or, for any sizes of one D,
 *             compute units (l2kv_device_info) * (2048 * (D + 4) + 24) bytes.
 * Arithmetic: fp32 scores, softmax and sums; for bf16, products on the matrix unit
 * with the softmax weights rounded to bf16 (their sum is that of the rounded ones; O is
 * off by about a tenth more than by its own rounding, and differs by that much from
 * l2kv_decode_attn*, which hold weights in fp32) and O rounded once.  Weights are at
 * most 1: sums leave the range of fp32 only where those of a plain softmax do
 * (bf16 values below 2^-110 in size may count as zero).
 * NaN and infinities reach the results of the queries that see them.
 * Errors: NULL, SHAPE (Hq % Hkv != 0, Hq/Hkv > 8 -- > 4 for D = 256 --, ...), DTYPE, WORKSPACE, ALIGN, LAUNCH.
 */
l2kv_status l2kv_prompt_attn(const void* Q, const void* K, const void* V, l2kv_dtype dt, int32_t n_seq, int32_t Hq,
                             int32_t Hkv, int32_t D, int64_t total_q, int64_t q_stride, const int64_t* q_offsets,
                             int64_t total_rows, int64_t kv_head_stride, const int64_t* kv_offsets,
                             const int32_t* kv_lens, int64_t max_kv, float scale, void* O, void* workspace,
                             size_t workspace_bytes, void* stream);

size_t l2kv_prompt_attn_workspace_bytes(int32_t n_seq, int32_t Hq, int32_t Hkv, int64_t total_q, int64_t max_kv,
                                        int32_t D, l2kv_dtype dt);

/*
 * Attention of drafted tokens over a slot cache: decode attention with several
 * queries per sequence that also see one another as a mask allows (a tree of
 * drafts: a node sees its ancestors and itself).  Node i of sequence s attends to the
 * lens[s] occupied slots and to those nodes j of its sequence whose bit is set:
 *     mask[node][j / 32] >> (j % 32) & 1
 * with i's own bit the caller's to set.  The nodes' keys and values are not in the
 * cache but in Kt, Vt (l2kv_rotary_append without offsets puts them there, with
 * positions by their depth); l2kv_stream_append_path moves those that are
 * accepted.  A node that sees no row gets zeros; what a node does not see has no effect on it.
 *   Q      in : [total_nodes] x Hq heads, node_offsets DEVICE int64 [n_seq+1]
 *   Kc, Vc in : one layer's planes, kv_head_stride, total_slots, slot_offsets as
 *               kv_head_stride, total_rows, kv_offsets of l2kv_prompt_attn
 *   lens   in : DEVICE int32 [n_seq], at most as many as the sequence has slots (forced to that); 0 allowed
 *   max_len   : an upper bound of all lens (as max_kv of l2kv_prompt_attn; 0 allowed)
 *   Kt, Vt in : [Hkv][total_nodes][D]
 *   mask   in : DEVICE uint32 [total_nodes][mask_words], mask_words >= 1; nodes of a
 *               sequence beyond 32 * mask_words are not seen
 *   O     out : [total_nodes][Hq][D], dense, of type dt
 *   workspace : l2kv_tree_attn_workspace_bytes(...), as for l2kv_prompt_attn
 * Arithmetic and errors: as l2kv_prompt_attn.
 */
l2kv_status l2kv_tree_attn(const void* Q, const void* Kc, const void* Vc, const void* Kt, const void* Vt, l2kv_dtype dt,
                           int32_t n_seq, int32_t Hq, int32_t Hkv, int32_t D, int64_t total_nodes, int64_t q_stride,
                           const int64_t* node_offsets, const uint32_t* mask, int32_t mask_words,
                           int64_t total_slots, int64_t kv_head_stride, const int64_t* slot_offsets,
                           const int32_t* lens, int64_t max_len, float scale, void* O, void* workspace,
                           size_t workspace_bytes, void* stream);

size_t l2kv_tree_attn_workspace_bytes(int32_t n_seq, int32_t Hq, int32_t Hkv, int64_t total_nodes, int64_t max_len,
                                      int32_t D, l2kv_dtype dt);

/*
 * The accepted tokens of a drafted tree join the cache, all layers in one call:
 * rows path[s][0 .. path_lens[s]-1] of sequence s's nodes, in that order, go to slots
 * lens_in[s], lens_in[s]+1, ... of every plane, K, V, norm and token id, and
 * lens_out[s] = lens_in[s] + the number stored (at most as many as there is room
 * for, and none for a sequence without nodes).  An entry outside the sequence's nodes
 * is forced into them.
 *   Kt, Vt in : [n_planes][total_nodes][D]; norms_t, pos_t [n_planes][total_nodes]
 *   path   in : DEVICE int32 [n_seq][max_path]; path_lens DEVICE int32 [n_seq], 0..max_path
 * lens_out must not be lens_in.  Errors: NULL, SHAPE, DTYPE, ALIGN, LAUNCH.
 */
l2kv_status l2kv_stream_append_path(const void* Kt, const void* Vt, const float* norms_t, const int32_t* pos_t,
                                    l2kv_dtype dt, int32_t n_planes, int32_t n_seq, int32_t D, int64_t total_nodes,
                                    const int64_t* node_offsets, const int32_t* path, int32_t max_path,
                                    const int32_t* path_lens, const int64_t* slot_offsets, int64_t total_slots,
                                    const int32_t* lens_in, int32_t* lens_out, void* Kc, void* Vc,
                                    float* norms_c, int32_t* pos_c, void* stream);

/* ---------------------------------------------------------------------------
 * The cache in pages.
 *
 * A slot cache [planes][total_slots][D] with norms_c, pos_c [planes][total_slots] whose slots are handed out in pages
 * of page_size (16, 32, 64, 128 or 256): page p = slots p*page_size .. of every plane, total_slots = n_pages *
 * page_size.  Row r of sequence s lies at slot
 *     page_table[s][r / page_size] * page_size + r % page_size
 * page_table: DEVICE int32 [n_seq][max_pages], the same for all planes (layers and KV heads); -1 where there is no page.
 * A sequence has at most max_pages * page_size rows (at most 2^31-1).  An entry that is no page's number is forced into
 * them where rows are read, and takes no row where they are written.  Several sequences may hold the same page: who
 * writes rows first asks l2kv_pages_reserve for them, and writes those only that it was given: a sequence whose request is refused
 * still names the pages that it shares, and what is written there reaches all who hold them.  l2kv_paged_append_reserved takes what was given.
 * ------------------------------------------------------------------------ */

/*
 * l2kv_rotary_append with norms of the heads before the rotation.  Every query head (where q_weight is given) and every
 * key head (k_weight) is divided by the root of its mean square and multiplied by the weights, one for each element:
 *     y[d] = x[d] / sqrt( sum_e x[e]^2 / D + eps ) * weight[d]
 * and then turned as in l2kv_rotary_append; elements from rot_dim on are normed alike.  All of it in fp64, rounded to
 * fp32 and for bf16 from there.  norms_c are those of the keys as stored.
 *   q_weight, k_weight in: DEVICE fp32 [D], NULL: heads of that kind are not normed
 *   eps   : >= 0, finite (0 and a head of zeros give NaN)
 * Everything else as l2kv_rotary_append, which both NULL makes it.
 * Errors: as l2kv_rotary_append; SHAPE for eps.
 */
l2kv_status l2kv_norm_rotary_append(const void* Q, const void* K, const void* V, l2kv_dtype dt, int64_t total_tokens,
                                    int32_t Hq, int32_t Hkv, int32_t D, int64_t q_stride, int64_t k_stride,
                                    int64_t v_stride, const float* q_weight, const float* k_weight, double eps,
                                    const int32_t* positions, const double* freqs, int32_t rot_dim,
                                    l2kv_rotary_layout layout, double amplitude, int32_t n_seq,
                                    const int64_t* token_offsets, const int64_t* slot_offsets,
                                    const int32_t* lens_in, int32_t* lens_out, int64_t total_slots, void* Qr,
                                    void* Kc, void* Vc, float* norms_c, int32_t* pos_c, void* stream);

/*
 * The same into pages: the j-th token of sequence s becomes row lens_in[s] + j of it.  A token whose row has no page is
 * not stored (its queries are turned all the same).  lens_out[s] = lens_in[s] + the tokens stored before the first such
 * one; may be NULL (calls for further layers), must not be lens_in.
 *   Kc, Vc out: one layer's planes [Hkv][n_pages*page_size][D]; norms_c, pos_c likewise
 * Errors: as l2kv_norm_rotary_append; SHAPE for page_size, max_pages, n_pages.
 */
l2kv_status l2kv_paged_append(const void* Q, const void* K, const void* V, l2kv_dtype dt, int64_t total_tokens,
                              int32_t Hq, int32_t Hkv, int32_t D, int64_t q_stride, int64_t k_stride,
                              int64_t v_stride, const float* q_weight, const float* k_weight, double eps,
                              const int32_t* positions, const double* freqs, int32_t rot_dim,
                              l2kv_rotary_layout layout, double amplitude, int32_t n_seq,
                              const int64_t* token_offsets, const int32_t* page_table, int32_t max_pages,
                              int32_t page_size, int32_t n_pages, const int32_t* lens_in, int32_t* lens_out,
                              void* Qr, void* Kc, void* Vc, float* norms_c, int32_t* pos_c, void* stream);

/*
 * The same within what l2kv_pages_reserve gave: rows from ends[s] on are not stored either, whatever their entries say, and
 * lens_out[s] ends before them.  So where free pages do not suffice, sequences without room keep their length, and nobody
 * writes a page that others hold, without a word from the device in between.
 *   ends : DEVICE int32 [n_seq], NULL: no such ends (l2kv_paged_append); must not be lens_out, may be lens_in (nothing is stored)
 * Errors: as l2kv_paged_append.
 */
l2kv_status l2kv_paged_append_reserved(const void* Q, const void* K, const void* V, l2kv_dtype dt, int64_t total_tokens,
                                       int32_t Hq, int32_t Hkv, int32_t D, int64_t q_stride, int64_t k_stride,
                                       int64_t v_stride, const float* q_weight, const float* k_weight, double eps,
                                       const int32_t* positions, const double* freqs, int32_t rot_dim,
                                       l2kv_rotary_layout layout, double amplitude, int32_t n_seq,
                                       const int64_t* token_offsets, const int32_t* page_table, int32_t max_pages,
                                       int32_t page_size, int32_t n_pages, const int32_t* lens_in, const int32_t* ends,
                                       int32_t* lens_out, void* Qr, void* Kc, void* Vc, float* norms_c, int32_t* pos_c,
                                       void* stream);

/*
 * Attention of the last tokens of every sequence, one or many, over all its rows in pages: l2kv_prompt_attn with the
 * rows found by the page table.  Query i of the n_q of sequence s attends to its rows j <= i + n_kv - n_q; a single
 * token (a decode step) sees all n_kv.  The rows of the new tokens themselves are in the cache already
 * (l2kv_paged_append).  Rows of a page behind the last are not seen, whatever they hold.
 *   Q      in : [total_q] x Hq heads, q_offsets DEVICE int64 [n_seq+1]
 *   Kc, Vc in : one layer's planes [Hkv][n_pages*page_size][D]
 *   kv_lens in: DEVICE int32 [n_seq], rows of every sequence (0 allowed)
 *   max_kv    : an upper bound of all of them, 1 .. max_pages*page_size (sizes the workspace and the decomposition;
 *               rows beyond it are still attended to)
 *   O     out : [total_q][Hq][D], dense, of type dt
 *   workspace : l2kv_paged_attn_workspace_bytes(...), as for l2kv_prompt_attn, with the same bound for all sizes
 * How a batch is worked on goes by its sizes, which are all that the host knows of it:
 *   total_q <= n_seq: as a decode step, every token by itself.  Softmax weights are held in fp32 for both types (as in
 *             l2kv_decode_attn*), so O is off by its own rounding alone.  A sequence with several tokens has its rows read for each of them:
 *             a chunk among places without tokens belongs into a call without those places.
 *   total_q > n_seq : as chunks, the rows of a sequence once for a block of tokens.  Arithmetic as l2kv_prompt_attn, bf16 weights rounded for the
 *             matrix unit, for the single tokens of such a batch as well: the same token may differ in its last bits between the two.
 *   more than 1024 sequences: an item for each (block of tokens, KV head) and none is cut, so one that is far longer than the others runs long.
 * Otherwise arithmetic and errors: as l2kv_prompt_attn; SHAPE for page_size, max_pages, n_pages and where n_seq * max_pages exceeds 2^31-1.
 */
l2kv_status l2kv_paged_attn(const void* Q, const void* Kc, const void* Vc, l2kv_dtype dt, int32_t n_seq, int32_t Hq,
                            int32_t Hkv, int32_t D, int64_t total_q, int64_t q_stride, const int64_t* q_offsets,
                            const int32_t* page_table, int32_t max_pages, int32_t page_size, int32_t n_pages,
                            const int32_t* kv_lens, int64_t max_kv, float scale, void* O, void* workspace,
                            size_t workspace_bytes, void* stream);

size_t l2kv_paged_attn_workspace_bytes(int32_t n_seq, int32_t Hq, int32_t Hkv, int64_t total_q, int64_t max_kv, int32_t D,
                                       l2kv_dtype dt);

/*
 * The pages' bookkeeping, in device memory, so that a serving loop needs no word from the device:
 *   refs       DEVICE int32 [n_pages]: holders of every page (entries of page tables that name it)
 *   free_pages DEVICE int32 [n_pages]: the first free_count[0] are the pages without holders, the last of them the next
 *              to be handed out; free_count DEVICE int32 [1]
 * l2kv_pages_init makes all pages free and every entry of a table -1 (several tables: -1 in the others is the caller's
 * to write).  Which page goes where depends on nothing but the order of the entries: sequence after sequence, page
 * after page.  Calls that share refs, free_pages or a workspace must not overlap in time.  n_seq <= 65535.
 * Errors of the four calls: NULL, SHAPE (also n_seq * max_pages beyond 2^30 or n_pages * page_size beyond 2^31-1), ALIGN, LAUNCH;
 * of those with a workspace, l2kv_pages_workspace_bytes(n_pages) bytes, 16-aligned, contents irrelevant before
 * and after, WORKSPACE.
 */
l2kv_status l2kv_pages_init(int32_t* page_table, int32_t n_seq, int32_t max_pages, int32_t* refs, int32_t* free_pages,
                            int32_t* free_count, int32_t n_pages, void* stream);

/*
 * Sequences that go on from others: sequence i of table_out has the pages and the length of sequence parents[i] of
 * table_in (a number outside 0..n_in-1: none), each page held once more.  A parent may have any number of children.
 * What table_out named before is written over, not released (l2kv_pages_release).
 *   table_in  in : [n_in][max_pages], lens_in [n_in]; pages up to lens_in are taken over
 *   parents   in : DEVICE int32 [n_out]
 *   table_out out: [n_out][max_pages], lens_out [n_out]; neither may be an input
 */
l2kv_status l2kv_pages_fork(const int32_t* table_in, const int32_t* lens_in, int32_t n_in, const int32_t* parents,
                            int32_t n_out, int32_t max_pages, int32_t page_size, int32_t n_pages, int32_t* table_out,
                            int32_t* lens_out, int32_t* refs, void* stream);

/*
 * Room for rows from[s] .. to[s]-1 of every sequence, to be written by it alone: entries of these rows that are -1 get a
 * free page; a page that others hold as well is copied, all planes with norms and ids, and the copy takes its
 * place (where all holders of a page ask for it in the same call the last keeps it).
 *   from, to in : DEVICE int32 [n_seq]; from >= to, from < 0 or to > max_pages * page_size asks for nothing
 *   ends    out : [n_seq], to[s] where the sequence has its room, else from[s]: nothing was asked for, or the free pages do not
 *                 suffice and nothing of it was changed.  Sequences are served in order: behind one that does not fit
 *                 only those that need no page get theirs.  Must not be an input.
 *   Kc, Vc, norms_c, pos_c: all planes of the cache, [n_planes][n_pages*page_size]
 * Errors: also DTYPE.
 */
l2kv_status l2kv_pages_reserve(int32_t* page_table, int32_t n_seq, int32_t max_pages, int32_t page_size,
                               const int32_t* from, const int32_t* to, int32_t* ends, int32_t* refs, int32_t* free_pages,
                               int32_t* free_count, int32_t n_pages, l2kv_dtype dt, int32_t n_planes, int32_t D, void* Kc,
                               void* Vc, float* norms_c, int32_t* pos_c, void* workspace, size_t workspace_bytes,
                               void* stream);

/*
 * Sequences give up their pages behind the first keep_lens[s] rows (0: all): the entries become -1, each page has a holder
 * less, and those without any are free again (released and reserved once more in the same order, the same ones come
 * back).  keep_lens DEVICE int32 [n_seq].
 */
l2kv_status l2kv_pages_release(int32_t* page_table, int32_t n_seq, int32_t max_pages, int32_t page_size,
                               const int32_t* keep_lens, int32_t* refs, int32_t* free_pages, int32_t* free_count,
                               int32_t n_pages, void* workspace, size_t workspace_bytes, void* stream);

size_t l2kv_pages_workspace_bytes(int64_t n_pages);

/*
 * Compaction in pages (the rule of Sec. 1 on a paged cache): of every plane and sequence the min(keep[s], lens_in[s]) rows
 * with the lowest (norm bits, row), in the order of the rows, become rows 0, 1, ... of the sequence in table_out;
 * K, V, norm and token id.  As many in every plane, other ones in each.  Rows are appended behind one another, so the
 * lower row is the earlier token and ties go to it, as in l2kv_select.
 *   Kc, Vc, norms_c, pos_c: [n_planes][n_pages*page_size], read and written; the pages of table_out must not be those of
 *             table_in (l2kv_pages_reserve before, l2kv_pages_release behind); pages that several sequences hold are only read
 *   table_in [n_seq][max_in], lens_in, keep [n_seq]; table_out [n_seq][max_out], lens_out [n_seq] = rows kept, at most
 *             max_out * page_size.  A row whose entry of table_out is no page is counted and not written, so where room may have been
 *             refused, keep is what the reservation of it (from 0 to the rows to be kept) left in its ends: a sequence
 *             without room then keeps no row in table_out, and its rows stay in table_in.  lens_out must not be an input.
 *   total_rows, total_kept: upper bounds of the sums of lens_in and of the rows kept (size the workspace and the launches;
 *             what goes beyond them is left out); total_kept < 2^28
 *   max_len : an upper bound of lens_in, at most total_rows (chooses the kernel variant; rows beyond it are left out)
 *   workspace: l2kv_paged_compress_workspace_bytes(...) bytes, 16-aligned; contents irrelevant before and after, one per call
 *             that may run at the same time.  One that was sized for no fewer planes, sequences, rows and kept rows is always enough.
 * Errors: NULL, DTYPE, SHAPE, WORKSPACE, ALIGN, LAUNCH.
 */
l2kv_status l2kv_paged_compress(void* Kc, void* Vc, float* norms_c, int32_t* pos_c, l2kv_dtype dt, int32_t n_planes,
                                int32_t n_seq, int32_t D, int32_t page_size, int32_t n_pages, const int32_t* table_in,
                                int32_t max_in, const int32_t* lens_in, const int32_t* keep, const int32_t* table_out,
                                int32_t max_out, int32_t* lens_out, int64_t total_rows, int64_t total_kept,
                                int64_t max_len, void* workspace, size_t workspace_bytes, void* stream);

size_t l2kv_paged_compress_workspace_bytes(int64_t n_planes, int64_t n_seq, int64_t total_rows, int64_t total_kept);

/* ---------------------------------------------------------------------------
 * Attention-loss analysis (Sec. 3, Eq. 5-7)
 *
 * When m of the T cached pairs of a head are dropped, the attention loss L^m is
 * the sum of the attention scores a_p (softmax of Eq. 2 over the FULL cache) of
 * the dropped pairs (Eq. 5).  The norm rule drops the highest key norms; the
 * ideal rule, which would need the next query in advance, drops the lowest
 * scores and gives the reference loss L^{m,ref}.  Y^m = L^m - L^{m,ref} >= 0
 * (Eq. 6) and Y = sum over m = 1..T of Y^m (Eq. 7) measure how far the norm
 * order is from the ideal order for that head and query.
 * ------------------------------------------------------------------------ */

/*
 * Discard order of the norm rule.  drop_rank[h][t] = number of positions of
 * head h that are discarded before position t when pairs go highest norm
 * first and, among equal norms, later position first -- the exact reverse of
 * the keep order of l2kv_select, so l2kv_select(k) keeps the positions with
 * drop_rank >= T-k and the m dropped pairs of Eq. 5 are those with
 * drop_rank < m.  Each row of drop_rank is a permutation of 0..T-1.
 *   norms     in : [n_heads][T] fp32, dense (as written by l2kv_norms)
 *   drop_rank out: [n_heads][T] int32
 *   workspace    : l2kv_norm_ranks_workspace_bytes(n_heads, T) bytes of device
 *                  memory, 16-byte aligned; contents irrelevant before and after
 * n_heads <= 2^31-1, T <= 2^31-1.  Errors: NULL, SHAPE, WORKSPACE, ALIGN, LAUNCH.
 */
l2kv_status l2kv_norm_ranks(const float* norms, int64_t n_heads, int64_t T, int32_t* drop_rank,
                            void* workspace, size_t workspace_bytes, void* stream);

size_t l2kv_norm_ranks_workspace_bytes(int64_t n_heads, int64_t T);

/*
 * Attention loss of one query per head over the uncompressed cache:
 *   a[b][hq][p]      = softmax_p( scale * Q[b][hq] . K[b][hq / (Hq/Hkv)][p] )       (Eq. 2)
 *   loss[b][hq]      = L^m      = sum of a_p over drop_rank[b][hkv][p] < m          (Eq. 5)
 *   loss_ref[b][hq]  = L^{m,ref} = sum of the m smallest a_p                        (Eq. 6)
 *   alr[b][hq]       = Y = sum_{m'=1..T} ( L^{m'} - L^{m',ref} )                    (Eq. 7)
 *   Q         in : [B][Hq][D], dense, dtype dt
 *   K         in : [B][Hkv] slabs of [T][D], k_head_stride elements apart, dtype dt
 *   drop_rank in : [B][Hkv][T] int32 from l2kv_norm_ranks (values outside 0..T-1
 *                  are not detected and give meaningless sums)
 *   m            : number of dropped pairs for loss / loss_ref, 0..T
 *                  (T - k for a cache compressed to k rows)
 *   scale        : softmax scale; <= 0 selects 1/sqrt(D)
 *   alr, loss, loss_ref out: [B][Hq] double each; loss and loss_ref may be NULL
 *   workspace    : l2kv_alr_workspace_bytes(B, Hq, T) bytes, 16-byte aligned;
 *                  contents irrelevant before and after
 * Scores are computed in fp32 and summed in fp64; Hq/Hkv <= 8, B*Hkv <= 65535.
 * All device pointers; enqueues on `stream` and returns.
 * Errors: NULL, DTYPE, SHAPE, WORKSPACE, ALIGN, LAUNCH.
 */
l2kv_status l2kv_alr(const void* Q, const void* K, l2kv_dtype dt, const int32_t* drop_rank, int32_t B,
                     int32_t Hq, int32_t Hkv, int64_t T, int32_t D, int64_t k_head_stride, float scale,
                     int64_t m, double* alr, double* loss, double* loss_ref, void* workspace,
                     size_t workspace_bytes, void* stream);

size_t l2kv_alr_workspace_bytes(int32_t B, int32_t Hq, int64_t T);

/*
 * Measurement aid: streams `bytes` bytes from `data` (rounded down to a
 * multiple of 8192) through the compute units with the loads of the norm
 * pass, computes nothing and stores nothing -- the rate this launch reaches is
 * the read-stream ceiling of the device for that buffer, against which the
 * kernels above can be judged (it depends on where the buffer lies in device
 * memory).  `sink`: 4 writable device bytes; written only if a block of the
 * data XORs to one particular 32-bit value, which keeps the loads alive.
 * Errors: NULL, ALIGN (data 16, sink 4), SHAPE (fewer than 8192 bytes, or
 * more than 2^31 - 1 blocks of 8192), LAUNCH.
 */
l2kv_status l2kv_read_probe(const void* data, size_t bytes, uint32_t* sink, void* stream);

/*
 * What the current HIP device reports about itself (host function, no kernel):
 * compute units, peak memory clock in kHz and memory bus width in bits, so
 * that a benchmark can print them next to the bandwidth peak it assumes.  Any
 * of the three pointers may be NULL.  Errors: LAUNCH if the runtime refuses
 * the query.
 */
l2kv_status l2kv_device_info(int32_t* h_compute_units, int32_t* h_memory_clock_khz,
                             int32_t* h_memory_bus_bits);

/* Static, NUL-terminated description of a status code. */
const char* l2kv_status_string(l2kv_status s);

/* Library version as major*10000 + minor*100 + patch. */
int32_t l2kv_version(void);

#ifdef __cplusplus
}
#endif
#endif /* L2KV_H */
