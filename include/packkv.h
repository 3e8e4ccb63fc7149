/*
 * packkv.h -- C ABI of the PackKV decode hot path for AMD MI355X (gfx950).
 *
 * A KV cache that is token-wise quantized and bit-packed in independent
 * 64-token blocks (PackKV, arXiv 2512.24449, Sec. III), an append-side
 * compressor, and fused kernels that stream the packed cache from HBM,
 * decode it on chip and compute q.K^T and p.V without ever writing
 * decompressed data back (Sec. III-C).
 *
 * Conventions for every entry point
 *   - "device" pointers are HIP device memory of the current device, owned by
 *     the caller; the library allocates no device memory and keeps only host
 *     bookkeeping inside kv_cache_t.
 *   - `hip_stream` is a hipStream_t passed as void* (NULL = default stream).
 *     Work is enqueued on it and the call returns without synchronizing
 *     unless stated otherwise.
 *   - Return value: KV_OK (0) or a negative KV_ERR_* code.  No exceptions, no
 *     aborts.  kv_strerror() gives a short text.
 *   - A kv_cache_t is not thread-safe; distinct handles are independent.
 *   - Inputs must be finite fp16 values; NaN/Inf never cause out-of-bounds
 *     accesses but produce unspecified codes.
 *
 * Cache layout (Sec. II-A): tokens arrive as fp16 [batch][n][n_kv_heads][128].
 * Packed format (Sec. III-B.3, III-B.4, III-C): one chunk per
 * (block of 64 tokens, batch, kv-head), chunk index c = (block*B + b)*H + h,
 * chunks stored back to back in c order in one arena per tensor.  A pack is the
 * 16 codes of one channel d in one token group g (tokens 16g..16g+15) with their
 * minimum subtracted: `width` = ceil(log2(range + 1)) bits per code, 0..4.  The
 * default layout (packs of 16 tokens) stores exactly 16*width bits per pack as
 * bit planes, which the decode kernels feed to the matrix cores as they are:
 *     pack list       V chunks: pack p = g*128 + d (group-major)
 *                     K chunks: pack p = d*4 + g   (channel-major)
 *     bytes [0,512)   header, byte p = (width << 4) | min of pack p
 *     region E        for p = 0..511 in turn: if width >= 2 a 32-bit word L with
 *                     the low two bits of the 16 codes, and if width == 4 a
 *                     second word H with their high two bits; in both, token i
 *                     of the group sits at bits [4i, 4i+2) for i < 8 and at
 *                     [4(i-8)+2, 4(i-8)+4) for i >= 8
 *     region O        for p = 0..511 in turn: if width is odd a 16-bit word T
 *                     with the top bit (bit width-1) of the 16 codes, token i
 *                     at bit 4*(i%4) + i/4
 *     then            zero padding to a multiple of 16 bytes
 * (all words little-endian; see kv_config_t for packs of 8 tokens and for the
 * wide layout that fine quantization scales use, which keep contiguous packs).
 * index[c] (uint32) is the chunk start in 16-byte units, index[n_chunks] the
 * arena end.  token_meta[b*max_tokens + t] (uint32) = scale_fp16 | min_fp16<<16
 * (Sec. III-B.2: one scale and minimum per token over all kv-heads).
 */
#ifndef PACKKV_H
#define PACKKV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define KV_OK 0
#define KV_ERR_ARG (-1)          /* null pointer, bad size, misaligned buffer        */
#define KV_ERR_UNSUPPORTED (-2)  /* head_dim != 128, block != 64, pack size, rel...  */
#define KV_ERR_CAPACITY (-3)     /* append beyond max_tokens / arena too small       */
#define KV_ERR_HIP (-4)          /* a HIP runtime call failed                        */

#define KV_HEAD_DIM 128
#define KV_BLOCK_TOKENS 64
#define KV_PACK_SIZE 16                      /* default pack size                      */
#define KV_CHUNK_HEADER 512                  /* header bytes of a chunk, packs of 16   */
#define KV_CHUNK_MAX_BYTES (512 + 512 * 8)   /* largest chunk, packs of 16             */
#define KV_CHUNK_HEADER_PACK8 1024           /* the same with packs of 8 tokens        */
#define KV_CHUNK_MAX_BYTES_PACK8 (1024 + 1024 * 4)
#define KV_CHUNK_HEADER_WIDE 2048            /* wide chunks: codes above 15            */
#define KV_CHUNK_MAX_BYTES_WIDE (2048 + 1024 * 8)
#define KV_PAGE_BYTES 65536                  /* page of a paged arena (kv_page_pool_t) */

typedef struct kv_cache kv_cache_t; /* opaque, host memory owned by the library */
typedef struct kv_page_pool kv_page_pool_t; /* the same: pages shared by paged caches */

#define KV_REPACK_NONE 0
#define KV_REPACK_V_MEDIAN 1

/* Parameters of Sec. IV-A: relative quantization scales (K 0.1, V 0.2 are the
 * paper's defaults), pack size 16, repacking none, block 64.  Pack size 8 (the
 * other good point of the pack-size study, Sec. IV-B): a chunk then has 1024
 * header bytes, indexed [token_group * 128 + channel] with token groups of 8,
 * and packs of `width` bytes.  A relative scale below 1/15 gives codes above 15
 * ("wide" chunks for that tensor: packs of 8 tokens with widths up to 8 bits,
 * 1024 width bytes followed by 1024 minimum bytes, then the packs); it needs
 * pack_size 8, and its lower bound is 1/255.
 * KV_REPACK_V_MEDIAN
 * (Sec. III-B.3, "Faster Repacking with V Median"): inside every block of 64
 * tokens, K and V are packed with their tokens sorted by the lower median of the
 * token's quantized V vector over all kv-heads (ascending, ties in arrival
 * order); scores then come out in that storage order (see token_order). */
typedef struct {
    int32_t batch;         /* B >= 1                                              */
    int32_t n_kv_heads;    /* H_kv >= 1                                           */
    int32_t n_q_heads;     /* H_q, a multiple of H_kv; H_q / H_kv from 1 to 4 (packs of 16;
                              1 to 8 with packs of 8), or a product s * g with s <= 16 and g
                              in that range (8, 12, 16, 64 ...): such a group runs as s groups
                              of g heads over the same kv-head; B * H_kv * s at most 65535 */
    int32_t head_dim;      /* must be 128                                         */
    int32_t block_tokens;  /* must be 64                                          */
    int32_t pack_size;     /* 16 or 8                                             */
    int32_t repack;        /* KV_REPACK_NONE or KV_REPACK_V_MEDIAN                */
    int32_t tail_capacity; /* raw fp16 tail buffer in tokens, must be 64          */
    float k_rel_scale;     /* in [1/15, 1]; down to 1/255 with pack_size 8        */
    float v_rel_scale;     /* the same                                            */
    int64_t max_tokens;    /* per batch element, rounded up to a block internally */
} kv_config_t;

/* Bytes of each caller-provided device buffer. */
typedef struct {
    size_t k_arena, v_arena;           /* packed chunks                           */
    size_t k_index, v_index;           /* uint32 [max_chunks + 1]                 */
    size_t k_token_meta, v_token_meta; /* uint32 [B][max_tokens]                  */
    size_t k_tail, v_tail;             /* fp16 [B][tail_capacity][H_kv][128]      */
    size_t workspace;                  /* status words, chunk sizes, V partials, and the
                                          compressor's staging area: at most 75 MB (packs of
                                          8: 84 MB), and at most what the cache's chunks can
                                          take; with half of that area a cache works too, its
                                          large appends in twice as many parts (packs of 8:
                                          with any part of it, or none and slower appends) */
    size_t token_order;                /* uint8 [B][max_tokens]; 0 without repacking */
    size_t k_pages, v_pages;           /* paged caches only: uint32 page lists; else 0 */
} kv_sizes_t;

/* Device buffers, each at least as large as kv_query_sizes said and 256-byte
 * aligned.  They must stay valid until kv_cache_destroy. */
typedef struct {
    void *k_arena, *v_arena;
    void *k_index, *v_index;
    void *k_token_meta, *v_token_meta;
    void *k_tail, *v_tail;
    void *workspace;
    /* With repacking: token_order[b][blk*64 + s] = position inside block blk (0..63,
     * arrival order) of the token stored at slot s; scores[b][hq][blk*64 + s] belongs
     * to token blk*64 + token_order[b][blk*64 + s].  Unused (may be null) without. */
    void *token_order;
    /* Paged caches only (kv_cache_create_paged; k_arena and v_arena are then unused and may be
     * null): [0] = pages held by the tensor, [1] = 16-byte units used in the newest of them,
     * [2 + i] = number of the i-th page taken.  Written by the library. */
    void *k_pages, *v_pages;
} kv_buffers_t;

/* Filled by kv_cache_stats. */
typedef struct {
    int64_t tokens;        /* cached tokens per batch element (packed + tail)     */
    int64_t packed_tokens; /* tokens living in chunks                             */
    int64_t tail_tokens;   /* tokens in the raw fp16 tail                         */
    int64_t n_chunks;      /* chunks per tensor                                   */
    int64_t k_bytes;       /* K arena bytes in use (header + payload + padding)   */
    int64_t v_bytes;
    int64_t index_bytes;   /* per tensor                                          */
    int64_t token_meta_bytes; /* per tensor                                       */
    int32_t overflow;      /* sticky: an append did not fit into an arena         */
    /* what the chunk bytes of each tensor consist of (chunks dropped by an overflow
     * count nothing): pack metadata (the header bytes), payload (exactly
     * pack_size * width bits per pack) and the zero padding up to 16 bytes       */
    int64_t k_header_bytes, k_payload_bytes, k_padding_bytes;
    int64_t v_header_bytes, v_payload_bytes, v_padding_bytes;
} kv_stats_t;

/*
 * Buffer sizes for a configuration.  `bits_per_element_budget` sizes the two
 * arenas: 0 means worst case (every pack at its largest width: 4.5 bits per
 * element with headers for packs of 16, 5 for packs of 8, 10 for wide chunks);
 * a positive value reserves that many bits per cached element
 * (it is clamped to the worst case).  Host only.
 */
int kv_query_sizes(const kv_config_t *cfg, double bits_per_element_budget, kv_sizes_t *out);

/*
 * Create an empty cache over caller-owned device buffers.  Enqueues a small
 * kernel on the default stream that clears the status words and index[0] and
 * synchronizes with it.  `sizes` are the real sizes of the buffers (arenas may
 * be larger or smaller than kv_query_sizes proposed; smaller arenas can
 * overflow, see kv_cache_stats).
 */
int kv_cache_create(const kv_config_t *cfg, const kv_buffers_t *buffers, const kv_sizes_t *sizes,
                    kv_cache_t **out);
int kv_cache_destroy(kv_cache_t *cache);

/*
 * Buffering, quantization, bit-packing and appending (Sec. III-B.1-4).
 * k_new, v_new: device fp16 [B][n_new][H_kv][128].  Tokens go to the raw
 * tail; whenever the tail holds 64 tokens they are quantized token-wise
 * (scale = rel*(max-min) over the token's H_kv*128 values, fp16 scale and
 * minimum), bit-packed in packs of 16 (or 8) tokens per channel, and appended to the
 * arenas as one chunk per (batch, kv-head); the tail then empties.  Several
 * full blocks in one call are compressed straight from k_new/v_new.
 * Errors: KV_ERR_CAPACITY if tokens + n_new > max_tokens (nothing is done).
 * An arena that is too small is detected on the device: the block is dropped
 * from that tensor and a sticky overflow flag is set.  Rule for dropped blocks:
 * kv_k_matvec scores the tokens of a block missing from K as -infinity, so
 * kv_softmax gives them weight 0 (a row of nothing else comes out as zeros);
 * kv_v_matvec adds nothing for a block missing from V; kv_decode_attention
 * leaves a block out when either tensor dropped it.  The three-step path and
 * the fused path therefore agree whenever no block is missing from V alone.
 * An arena larger than 2^32 * 16 bytes is used up to that size only.
 */
int kv_compress_append(kv_cache_t *cache, const void *k_new, const void *v_new, int32_t n_new,
                       void *hip_stream);
/*
 * The same for bf16 inputs (device bf16 [B][n_new][H_kv][128]): every value enters as
 * its fp16 rounding (to nearest even) -- exact for values in fp16's normal range,
 * since fp16 has the longer significand; smaller magnitudes round in fp16's
 * subnormal grid, magnitudes above 65504 become infinities (see "Inputs must be
 * finite").  From there on the path is the fp16 one: the tail stores fp16, and the
 * packed bytes are those kv_compress_append gives for the rounded values.
 */
int kv_compress_append_bf16(kv_cache_t *cache, const void *k_new, const void *v_new, int32_t n_new,
                            void *hip_stream);

/*
 * Fused K path (Sec. III-C.1): scores[b][hq][t] = sm_scale * sum_d
 * q[b][hq][d] * Khat[b][t][hq / G][d] for every cached token t, where Khat is
 * scale_t*code + min_t for packed tokens and the raw fp16 value for tail
 * tokens.  q: device fp16 [B][H_q][128]; scores: device fp32 [B][H_q][ld_scores],
 * ld_scores >= tokens (q 16-byte aligned).  fp32 accumulation.  One launch covers
 * all chunks.  With packs of 16 the products run on the matrix cores: the codes
 * enter exactly, q as three 4-bit pieces per value (a head's values below 2^-12
 * of its largest magnitude lose their low bits), sums in fp32.
 */
int kv_k_matvec(kv_cache_t *cache, const void *q, float sm_scale, float *scores, int64_t ld_scores,
                void *hip_stream);

/*
 * Fused V path (Sec. III-C.2): out[b][hq][d] = sum_t p[b][hq][t] *
 * Vhat[b][t][hq / G][d].  p: device fp32 [B][H_q][ld_p], ld_p >= tokens;
 * out: device fp32 [B][H_q][128].  fp32 accumulation in a fixed order (no
 * floating-point atomics): the result is bitwise reproducible.  Uses the
 * workspace for per-split partial sums; calls on one cache must not overlap.
 * With packs of 16 the products run on the matrix cores: the codes enter
 * exactly, the weights p_t * scale_t of a block rounded to 20 bits (16 with four
 * query heads per kv-head) below the block's largest weight of that head, and
 * the same rounded weights multiply the codes, the pack minimums and the token
 * minimums.  p must be non-negative.
 */
int kv_v_matvec(kv_cache_t *cache, const float *p, int64_t ld_p, float *out, void *hip_stream);

/*
 * kv_v_matvec for callers that cannot allocate device memory or hand over a
 * workspace for the call: code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc.  Same arguments, same kernels, same result
 * (bitwise, as long as the split count is not lowered, see below); the per-split
 * partial sums go to a fixed array inside the library (KV_NOALLOC_MAX_SPLIT_ROWS
 * rows of 132 floats, about 4.3 MB, held by every GPU the library runs on until
 * the process ends) instead of the cache's workspace, of which only counters of
 * this entry point's own are used (short contexts).  The call allocates and
 * frees nothing.  The context axis is split over at most
 * KV_NOALLOC_MAX_SPLIT_ROWS / (batch * n_q_heads) workgroups per stream;
 * KV_ERR_CAPACITY if batch * n_q_heads exceeds KV_NOALLOC_MAX_SPLIT_ROWS.
 * All calls on one GPU share the array: calls that overlap on one GPU (other
 * streams, other caches, other threads) race and give wrong results; calls on
 * one stream are ordered and safe.
 */
#define KV_NOALLOC_MAX_SPLIT_ROWS 8192
int kv_v_matvec_noalloc(kv_cache_t *cache, const float *p, int64_t ld_p, float *out, void *hip_stream);

/*
 * Row softmax between the two matvecs (smx in the attention definition of
 * Sec. III-B.3), in place: scores[b][hq][0..tokens) <- softmax over the cached
 * tokens, for every (b, hq); entries [tokens, ld_scores) are left alone.
 * scores: device fp32 [B][H_q][ld_scores] as written by kv_k_matvec.  fp32,
 * reductions in a fixed order (bitwise reproducible).  Long rows are cut into
 * segments whose statistics pass through the workspace; calls on one cache
 * must not overlap.  KV_ERR_ARG on an empty cache or ld_scores < tokens.
 */
int kv_softmax(kv_cache_t *cache, float *scores, int64_t ld_scores, void *hip_stream);

/*
 * Fused decode attention (the attention of one new query as defined in
 * Sec. III-B.3, Att(q, K, V) = softmax(sm_scale * K q)^T V, computed with the
 * fused decompression of Sec. III-C):
 *   out[b][hq][:] = sum_t softmax_t(sm_scale * q[b][hq] . Khat[b][t][hq / G]) * Vhat[b][t][hq / G][:]
 * over all cached tokens (packed blocks and raw tail) in one pass: scores and
 * probabilities stay on chip.  q: device fp16 [B][H_q][128]; out: device fp32
 * [B][H_q][128].  Equivalent to kv_k_matvec -> softmax -> kv_v_matvec up to
 * fp32 rounding.  Fixed-order fp32 accumulation, bitwise reproducible.  Uses the
 * workspace for per-split partial results; calls on one cache must not overlap.
 * KV_ERR_ARG on an empty cache or if q is not 16-byte aligned.  Blocks dropped by
 * an arena overflow (in either tensor) are left out of the softmax.
 */
int kv_decode_attention(kv_cache_t *cache, const void *q, float sm_scale, float *out, void *hip_stream);

/*
 * ---- paged arena ------------------------------------------------------------
 * The packed format stores chunks wherever the index says (Sec. III-B.4 needs an
 * appendable layout, not a contiguous one).  A paged cache keeps no arena of its
 * own: its chunks live in fixed pages of KV_PAGE_BYTES that it takes, as it grows,
 * from a pool shared with other caches, and gives back with kv_cache_release -- so
 * the memory a cache holds follows its compressed size, not its worst case.
 *   - a chunk never crosses a page boundary: a chunk that does not fit behind the
 *     previous one of its tensor starts a fresh page (K and V fill their own pages);
 *   - the index of a paged cache has two words per chunk, index[2c] = start and
 *     index[2c + 1] = end, in 16-byte units from the start of the pool's pages
 *     (a pool is therefore limited to 64 GiB); a dropped chunk has start = end;
 *   - pages are taken and returned on the device, inside the stream of the call
 *     (no host synchronization).  If the pool cannot cover an append, all chunks of
 *     that tensor in that call are dropped and the sticky overflow flag is set,
 *     exactly as with a full contiguous arena.
 *   - calls that take or return pages of one pool (kv_compress_append,
 *     kv_cache_release, kv_cache_destroy of its caches) must be ordered by the
 *     caller: one stream, or events between streams.  Reads never touch the pool state.
 * Everything else (token metadata, tails, token order, every read entry point)
 * works as with a contiguous cache and gives bitwise the same results.
 */
/* Device bytes of the pool's bookkeeping (`state`) for n_pages pages. */
size_t kv_page_pool_state_bytes(int64_t n_pages);
/*
 * pages: device, n_pages * KV_PAGE_BYTES bytes, 256-byte aligned; state: device,
 * kv_page_pool_state_bytes(n_pages), 256-byte aligned; both caller-owned and valid
 * until kv_page_pool_destroy.  1 <= n_pages < 2^20.  Marks every page free (a
 * small kernel on `hip_stream`, synchronized before returning); page 0 is handed
 * out first.
 */
int kv_page_pool_create(void *pages, int64_t n_pages, void *state, void *hip_stream, kv_page_pool_t **out);
/* Host bookkeeping only; destroy the caches that use the pool first. */
int kv_page_pool_destroy(kv_page_pool_t *pool);
/* Number of free pages.  Reads device state: synchronizes `hip_stream`. */
int kv_page_pool_free_pages(kv_page_pool_t *pool, int64_t *free_pages, void *hip_stream);
/*
 * Buffer sizes of a paged cache: arenas 0, indices of 2 * max_chunks words, page
 * lists sized for the worst case, the rest as kv_query_sizes.  Host only.
 */
int kv_query_sizes_paged(const kv_config_t *cfg, kv_sizes_t *out);
/*
 * As kv_cache_create, over the pages of `pool` (buffers->k_arena / v_arena are ignored).
 */
int kv_cache_create_paged(const kv_config_t *cfg, kv_page_pool_t *pool, const kv_buffers_t *buffers,
                          const kv_sizes_t *sizes, kv_cache_t **out);
/*
 * Empties the cache: 0 tokens, overflow flag cleared; a paged cache gives all its
 * pages back to its pool (a kernel on `hip_stream`, no synchronization).  The
 * cache can be filled again.  kv_cache_destroy of a paged cache that still holds
 * tokens does the same on the default stream and synchronizes.
 */
int kv_cache_release(kv_cache_t *cache, void *hip_stream);

/* Counters and byte accounting.  Reads device state: synchronizes `hip_stream`.
 * For a paged cache k_bytes / v_bytes are the bytes of the pages held and
 * index_bytes counts two words per chunk. */
int kv_cache_stats(kv_cache_t *cache, kv_stats_t *out, void *hip_stream);

/*
 * Adopt externally written buffer contents (a cache restored from a copy of
 * its arenas, indices, token metadata, tails and, with repacking, token
 * order): afterwards the cache holds
 * `tokens` tokens per batch element, floor(tokens/64)*64 of them packed.
 * Host bookkeeping only; the caller is responsible for the buffer contents.
 */
int kv_cache_restore(kv_cache_t *cache, int64_t tokens);

/* Cached tokens per batch element (host bookkeeping, no synchronization). */
int64_t kv_cache_tokens(const kv_cache_t *cache);

const char *kv_strerror(int code);

/* ---- 4-bit paged cache ------------------------------------------------------
 * A second cache beside the packed one, for batches whose sequences differ: every
 * sequence has its own length and its own number of new tokens, attention takes
 * one or many query rows of each, with an optional window.  Rows are held at a
 * fixed rate in pages of KV_FP4_PAGE_TOKENS tokens that the caller hands out.
 *
 * Values (the block format of OCP Microscaling, MXFP4, with blocks along the head
 * dimension): for every KV_FP4_GROUP consecutive channels x of a token and kv-head
 * one scale 2^e, e the least integer with max|x| <= 7 * 2^e, kept within -23 .. 13;
 * for every channel the sign and the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 to
 * |x| / 2^e (ties to the even code, above 6: 6).  The value read is code * 2^e: it
 * is exact in fp16, bf16 and fp32.  |x - value| <= 2^e where |x| <= 7 * 2^13 (half a
 * step of the largest codes), magnitudes above 49152 and infinities are held as 49152
 * with their sign, a NaN as 0: a cache holds finite values only.
 *
 * Layout of a page: n_kv_heads blocks of kv_fp4_head_bytes = 64 * (D + D / 16) bytes
 * (D = head_dim):
 *     K codes   byte [token][D / 2]: channel 2i in the low half of byte i, 2i + 1 in the high half
 *     K scales  byte [token][D / 32]: e + 127
 *     V codes   uint32 [token / 8][D]: bits 4i .. 4i + 3 hold token 8 * (token / 8) + i
 *     V scales  byte [D / 32][token]: e + 127
 * A code is sign << 3 | index into the magnitudes above.
 *
 * Which tokens a call is about is said by a kv_fp4_batch_t.  Its arrays are read on
 * the device when the call's kernels run, so a captured call follows what they then
 * hold.  Nothing they hold makes a kernel touch memory outside the page table, the pages
 * and the rows: a page number outside 0 .. n_pages - 1 marks a page that is missing
 * (its tokens are skipped by an append, read as zeros and seen by no row), and so are
 * positions from 64 * table_pages on.
 */
#define KV_FP4_PAGE_TOKENS 64
#define KV_FP4_GROUP 32

typedef struct kv_fp4_cache kv_fp4_cache_t; /* opaque, host memory owned by the library */

/* Types of rows that go in and come out. */
#define KV_TYPE_FP16 0
#define KV_TYPE_BF16 1
#define KV_TYPE_FP32 2 /* outputs only */

typedef struct {
    int32_t n_kv_heads; /* H_kv >= 1                                              */
    int32_t n_q_heads;  /* H_q, any multiple of H_kv                              */
    int32_t head_dim;   /* 128 or 64                                              */
    int64_t n_pages;    /* 1 .. 2^31 - 1                                          */
} kv_fp4_config_t;

/* Bytes of the two device buffers of a cache. */
typedef struct {
    size_t pages;     /* n_pages * n_kv_heads * 64 * (head_dim + head_dim / 16)   */
    size_t workspace; /* partial results of attention, weights and selection      */
} kv_fp4_sizes_t;

/* A ragged batch: sequence b holds lens[b] tokens, the last new_rows[b] of which
 * are the call's; row i of them lies at row first_row[b] + i of the call's tensors
 * and at position lens[b] - new_rows[b] + i of the sequence.  All arrays are device
 * memory.  Rows outside the tensors are left out. */
typedef struct {
    int32_t batch;             /* sequences, 1 .. 65535                           */
    int32_t max_new;           /* most new rows of a sequence; new_rows above it count as it.  append and read take
                                  max_new * n_kv_heads * head_dim below 2^37, attention max_new * n_q_heads / n_kv_heads up to 2^22 */
    int32_t table_pages;       /* pages of a sequence at most: 1 .. 2^24          */
    const int32_t *lens;       /* [batch], negative: 0                            */
    const int32_t *new_rows;   /* [batch]; null: max_new of every sequence        */
    const int32_t *first_row;  /* [batch]; null: b * max_new                      */
    const int32_t *page_table; /* [batch][table_pages]; null: page i of sequence b is b * table_pages + i */
} kv_fp4_batch_t;

/* Host only. */
int kv_fp4_query_sizes(const kv_fp4_config_t *cfg, kv_fp4_sizes_t *out);
/*
 * A cache over caller-owned device buffers, both 256-byte aligned and at least as
 * large as kv_fp4_query_sizes said; valid until kv_fp4_cache_destroy.  Enqueues a
 * small kernel on the default stream that clears counters in the workspace and
 * synchronizes with it.  The pages' contents are taken as they are (pages that another
 * cache of the same configuration has filled can be used).
 */
int kv_fp4_cache_create(const kv_fp4_config_t *cfg, void *pages, void *workspace, const kv_fp4_sizes_t *sizes,
                        kv_fp4_cache_t **out);
int kv_fp4_cache_destroy(kv_fp4_cache_t *cache);

/*
 * Quantizes the batch's new rows and writes them into their pages.  k, v: device
 * [n_rows][H_kv][D] of `type` (KV_TYPE_FP16 or KV_TYPE_BF16), consecutive rows k_stride
 * and v_stride elements apart (at least H_kv * D; multiples of 8, pointers 16-byte
 * aligned: k and v may be parts of one projection's output).  Other tokens of the pages
 * keep their values.  A page that is written must belong to one sequence of
 * the call only; full pages may be shared by sequences.
 */
int kv_fp4_append(kv_fp4_cache_t *cache, const kv_fp4_batch_t *batch, const void *k, int64_t k_stride, const void *v,
                  int64_t v_stride, int32_t type, int64_t n_rows, void *hip_stream);
/*
 * The values of the batch's new rows as the cache holds them (new_rows = lens: of
 * whole sequences).  k, v: device [n_rows][H_kv][D], contiguous, 16-byte aligned, of
 * `type` (any of the three: the values are exact in each); one of them may be null.
 * Rows of no sequence are left as they were; a row whose position the sequence does not
 * have (new_rows above lens) or whose page is missing is zeros.
 */
int kv_fp4_read(kv_fp4_cache_t *cache, const kv_fp4_batch_t *batch, void *k, void *v, int32_t type, int64_t n_rows,
                void *hip_stream);
/*
 * Attention of the batch's new rows over their sequences (append them first):
 *   out[row][hq][:] = sum_t softmax_t(sm_scale * q[row][hq] . Khat[t][hq / G]) * Vhat[t][hq / G][:]
 * over the tokens t that the row at position p sees: t <= p, and with window > 0 also
 * t > p - window or t < sinks (the first tokens stay visible).  window = 0: no
 * window.  Tokens that no row sees are not read: their pages may be missing.  A row that
 * sees nothing becomes zeros (lse: -infinity).  sm_scale: below 2.3e38 in size
 * (sm_scale * log2(e) is finite in fp32); with 0 all tokens that a row sees weigh the same.
 * q: device [n_rows][H_q][D] of `type` (fp16 or bf16), rows q_stride elements apart (a
 * multiple of 8, at least H_q * D), 16-byte aligned; out: device [n_rows][H_q][D]
 * contiguous of `out_type` (any), 16-byte aligned, not overlapping q; lse: null, or device fp32
 * [n_rows][H_q], the natural logarithm of the softmax's sum (with the scores' maximum
 * in it), for joining this result with one over other tokens.  Rows of no sequence are
 * left as they were.
 * q.Khat: exact products on the matrix cores, fp32 sums; softmax in fp32, of differences to the row's
 * largest score (which may be as large as fp32 holds); its weights
 * enter the product with Vhat as fp16 (scaled by a power of two: a relative error of
 * at most 2^-11 down to 2^-26 of the row's largest weight), sums in fp32.  A NaN or
 * infinity in q makes its row and head NaN where it sees a token, and no other.  Sums have a fixed order: the result
 * is bitwise reproducible.  Uses the workspace: attention calls on one cache must not overlap.
 */
int kv_fp4_attention(kv_fp4_cache_t *cache, const kv_fp4_batch_t *batch, const void *q, int64_t q_stride, int32_t type,
                     int64_t n_rows, float sm_scale, int32_t window, int32_t sinks, void *out, int32_t out_type,
                     float *lse, void *hip_stream);

/*
 * The attention weight that every cached token gets from the batch's new rows:
 *   mass[b][h][t] = past[b][h][t] + sum over the rows that see t and the heads hq of h of
 *                                   exp(sm_scale * q[row][hq] . Khat[t][h] - lse[row][hq])
 * with q, sm_scale, window, sinks (and so which rows see t) and lse as the call of kv_fp4_attention on the same batch had or
 * gave them.  mass: device fp32 [batch][H_kv][mass_tokens]; written are the places of the tokens that the sequence holds
 * (and the page table and mass have room for), others are left as they were.  past: null (0), or of mass's
 * size, mass itself or not overlapping it (mass overlaps nothing else that the call reads: KV_ERR_ARG); it is not read for the call's own
 * tokens, positions from lens - new_rows on, which no earlier row has seen.  A token that no row sees, and one of a missing page, keeps past's.  max_new may be 0: mass is then past.
 * fp32 throughout, q.Khat as in attention; what lse is off by (a few 2^-24 of its size) is a factor of a row's weights.  A row whose lse is
 * -infinity gives nothing, whatever its q is; another whose q (unless sm_scale is 0) or lse is NaN makes the tokens that it sees NaN.  Sums
 * have a fixed order: the result is bitwise reproducible.  Uses the workspace: calls of kv_fp4_attention, kv_fp4_weights and kv_fp4_select on one cache must not overlap.
 */
int kv_fp4_weights(kv_fp4_cache_t *cache, const kv_fp4_batch_t *batch, const void *q, int64_t q_stride, int32_t type,
                   int64_t n_rows, float sm_scale, int32_t window, int32_t sinks, const float *lse, const float *past,
                   float *mass, int64_t mass_tokens, void *hip_stream);
/*
 * Which tokens a sequence keeps, for every kv-head by itself: all if it holds no more than its budget, else as many as the budget,
 * namely the first `sinks`, then the last `recent` (as many of both as the budget has room for), then of the others those of the
 * largest mass, of equal ones the first (0 and -0 are equal, a NaN is above all).  mass as of kv_fp4_weights; tokens from mass_tokens on have
 * 0.  budgets: device int32 [batch], or null: keep of each; a budget above keep (1 or more) is keep, below 0 it is 0.
 * kept: device int32 [batch][H_kv][keep], the positions in ascending order, -1 behind them; n_kept: device int32 [batch],
 * how many: the least of lens, the table's room and the budget.  Of the batch lens and table_pages are used; pages are not read.
 * kept and n_kept overlap neither each other nor lens, mass or budgets (KV_ERR_ARG): sequences whose lens are an n_kept are cut into another one.
 * Uses the workspace, as kv_fp4_weights does.
 */
int kv_fp4_select(kv_fp4_cache_t *cache, const kv_fp4_batch_t *batch, const float *mass, int64_t mass_tokens, int32_t keep,
                  const int32_t *budgets, int32_t sinks, int32_t recent, int32_t *kept, int32_t *n_kept, void *hip_stream);
/*
 * Moves kept tokens together: token i of (sequence b, kv-head h) of `to` becomes token kept[b][h][i] of `from`, for i below
 * n_kept[b] (device int32 [batch]; at most keep), bit by bit.  kept: device int32 [batch][H_kv][keep], in any order, a position as
 * often as one likes; one that the sequence does not hold (lens, room of the table) or whose page is missing becomes a token of zeros.
 * `to`: as many sequences, and the pages that they go to, which belong to one sequence of the call only and are none that the call reads;
 * what would go to a page that is missing is left out.  Its lens are not read (they may be n_kept itself: the batch of the sequences
 * from then on).  In the group of eight tokens that the last one is in, those behind it become zeros.
 * mass, mass_out: both null, or device fp32 [batch][H_kv][mass_tokens] and, not overlapping, [batch][H_kv][mass_out_tokens]: weights that go with
 * the tokens (0 of a token that mass has no room for); places from n_kept on are left as they were.  mass_out overlaps nothing that the call
 * reads (KV_ERR_ARG).
 * From then on a token's position in the cache is no longer its position in the text: rotary positions of later rows count on
 * from the text's.
 */
int kv_fp4_compact(kv_fp4_cache_t *cache, const kv_fp4_batch_t *from, const kv_fp4_batch_t *to, const int32_t *kept, int32_t keep,
                   const int32_t *n_kept, const float *mass, int64_t mass_tokens, float *mass_out, int64_t mass_out_tokens,
                   void *hip_stream);

/* ---- rotary positions -------------------------------------------------------
 * Of query and key rows, before keys are appended to a cache (of either kind) and queries attend.  For pair i of the first
 * `dims` channels of a head, channels (x, y) at (i, i + dims / 2), or (2i, 2i + 1) where interleaved, and a row's position p:
 *     a = 2 pi * p * turns[i] / 2^64
 *     x' = magnitude * (x cos a - y sin a),  y' = magnitude * (y cos a + x sin a)
 * Channels from dims on are copied.  p * turns is exact modulo a turn and cut to 2^-32 of one, at any position; what it is more than a number of
 * quarter turns then becomes an fp32 number of radians (off by 1.4e-7 at most).  Sums are fp32, rounded once.
 */
typedef struct {
    int32_t head_dim;      /* even, 2 .. 512                                      */
    int32_t dims;          /* even, 2 .. head_dim                                 */
    int32_t interleaved;   /* 0: pairs (i, i + dims / 2)                          */
    float magnitude;       /* finite                                              */
    const uint64_t *turns; /* device [dims / 2]: turns that a position makes, in 2^-64 (modulo a turn) */
} kv_rotary_t;
/*
 * positions: device int32 [n_rows], any values, read when the kernel runs.  q: device [n_rows][n_q_heads][head_dim] of `type` (any of the
 * three), rows q_stride values apart (at least n_q_heads * head_dim), aligned to its type; k likewise, with n_k_heads; either number of heads may be
 * 0 and its pointers null then.  q_out, k_out: of the same type and shape, the input itself (same stride) or not overlapping anything that the call
 * reads, nor each other (KV_ERR_ARG); values between rows' ends and the next rows are left as they were.  inverse != 0: the angle's sign is
 * turned (the transpose of the operation: it takes gradients back, and rows too, with a magnitude of 1).  Rows of 16-byte aligned heads are fastest.
 */
int kv_rotary(const kv_rotary_t *rotary, const int32_t *positions, int64_t n_rows, int32_t type, int32_t inverse, const void *q,
              int64_t q_stride, int32_t n_q_heads, void *q_out, int64_t q_out_stride, const void *k, int64_t k_stride,
              int32_t n_k_heads, void *k_out, int64_t k_out_stride, void *hip_stream);

/* ---- measurement companions (same shapes, uncompressed fp16 cache) ---------
 * The comparison kernels of Sec. IV-E, hand-written for the same shapes:
 * plain fp16 matrix-vector products over an uncompressed cache stored as
 * fp16 [B][H_kv][tokens][128] (head-major, each (b, h) matrix contiguous).
 * n_q_heads / n_kv_heads from 1 to 8 (KV_ERR_UNSUPPORTED otherwise).
 */
int kv_fp16_k_matvec(const void *k_cache, const void *q, float sm_scale, float *scores,
                     int64_t ld_scores, int32_t batch, int32_t n_kv_heads, int32_t n_q_heads,
                     int64_t tokens, void *hip_stream);
/* workspace: device, at least kv_fp16_v_workspace_bytes(...) bytes. */
int kv_fp16_v_matvec(const void *v_cache, const float *p, int64_t ld_p, float *out, int32_t batch,
                     int32_t n_kv_heads, int32_t n_q_heads, int64_t tokens, void *workspace,
                     void *hip_stream);
size_t kv_fp16_v_workspace_bytes(int32_t batch, int32_t n_q_heads);
/* Streaming-read ceiling: reads `bytes` (multiple of 16) of device memory with
 * sixteen independent 16-byte loads per thread and xors every word into
 * checksum[0] (device uint32; accumulated, the caller clears it): one kernel
 * launch and nothing else.  Used to measure achievable HBM read bandwidth next
 * to the 8 TB/s peak. */
int kv_stream_read(const void *src, size_t bytes, uint32_t *checksum, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* PACKKV_H */
