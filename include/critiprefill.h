/*
 * critiprefill.h - C ABI of the MI355X (gfx950) prefill-attention library.
 *
 * The library runs the CritiPrefill prefill-attention path on one GPU:
 *
 *   critiprefill_estimate          Algorithm 1 "Estimation of Query Criticality in One Layer"
 *   critiprefill_select            Algorithm 2 "Pruned Attention", the argtop_k(S[j], B/block size) step
 *   critiprefill_sparse_attn       Algorithm 2, the per-segment attention loop
 *   critiprefill_select_shared / critiprefill_sparse_attn_shared   the same two steps with one list per KV head
 *   critiprefill_dense_causal_attn Eq. 2 (O = softmax(Q K^T / sqrt(d)) V) with the prefill causal mask
 *
 * and what a program does around a prefill and after it, on a cache of pages (second half of this file):
 *
 *   critiprefill_norm_rope         norms of queries and keys for each head and the position rotation, in one pass
 *   critiprefill_norm_rope_write   the same, with keys and values going straight into the cache
 *   critiprefill_cache_write / critiprefill_cache_read   keys and values into the cache and back, as they are, in 8 or in 4 bits
 *   critiprefill_paged_attn        attention of each sequence's new tokens, one or many, over its pages
 *
 * Conventions common to all entry points
 * --------------------------------------
 * Pointers: every data pointer is DEVICE memory owned by the caller, 16-byte aligned.  Inputs are
 *   only read; outputs are fully overwritten.  The library allocates and frees nothing.
 * Stream:   `hip_stream` is a hipStream_t passed as void* (NULL = the default stream).  Calls only
 *   enqueue work on that stream and never synchronise; results are ready when the stream reaches
 *   that point.
 * Layouts:  Q and O are [batch, n_q_heads, seq_len, head_dim], K and V are
 *   [batch, n_kv_heads, seq_len, head_dim]; the strides of the first three axes are given in
 *   ELEMENTS in the parameter block, the channel stride is 1.  Query head h reads K/V head
 *   h / (n_q_heads / n_kv_heads) (the single-head description of the paper extended head by head).
 *   n1 = ceil(seq_len / segment_size) query segments, n2 = ceil(seq_len / block_size) KV blocks,
 *   r = segment_size / block_size blocks under one segment.
 * Errors:   the return value is 0 on success or a negative CP_ERR_* code.  All checks happen before
 *   any kernel is launched; on error no output is touched.  Nothing is printed and nothing throws.
 */
#ifndef CRITIPREFILL_H
#define CRITIPREFILL_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
    CP_OK = 0,
    CP_ERR_NULL = -1,        /* a required pointer is NULL */
    CP_ERR_SHAPE = -2,       /* non-positive size, n_q_heads % n_kv_heads != 0, block_size does not divide segment_size */
    CP_ERR_UNSUPPORTED = -3, /* head_dim != 128, unknown dtype, softmax_domain or cache_format, n2 > 8192, list longer than the API allows,
                                bf16 estimate with batch * n_q_heads > 65535, sizes of the cache beyond the limits named there */
    CP_ERR_ALIGN = -4,       /* a pointer is not 16-byte aligned or a stride is not a multiple of 8 elements */
    CP_ERR_WORKSPACE = -5,   /* workspace smaller than critiprefill_workspace_bytes(), critiprefill_paged_workspace_bytes() */
    CP_ERR_LAUNCH = -6       /* the HIP runtime refused a launch */
};

enum { CP_DTYPE_FP32 = 0, CP_DTYPE_BF16 = 1 };

typedef struct critiprefill_params {
    int32_t batch, n_q_heads, n_kv_heads, head_dim; /* head_dim must be 128 */
    int32_t seq_len;                                /* n: queries and keys share positions 0..n-1 (prefill) */
    int32_t segment_size, block_size;               /* s, b; b divides s */
    int32_t budget_blocks;                          /* k = budget tokens / block size (Algorithm 2) */
    int32_t local_blocks;                           /* L blocks just before the segment that are always kept */
    int32_t dtype;                                  /* CP_DTYPE_*: element type of Q, K, V, O */
    float attn_scale;                               /* logit scale of attention; 0 -> 1/sqrt(head_dim) (Eq. 2) */
    float score_scale;                              /* logit scale inside the estimation softmax; 0 -> 1/sqrt(head_dim) */
    float alpha;                                    /* layer fusion S = alpha*S + (1-alpha)*S' (Algorithm 1); used only with prev_scores */
    int32_t softmax_domain;                         /* 0: softmax over all n2 blocks, mask afterwards (listing order); 1: over visible blocks */
    int64_t q_stride[3], kv_stride[3], o_stride[3]; /* elements: batch, head, token */
} critiprefill_params;

/* Length of one block list: budget_blocks + local_blocks + r. */
int32_t critiprefill_list_len(const critiprefill_params *p);

/* Bytes of scratch critiprefill_estimate needs (the max/min representatives of Algorithm 1 and, for bf16,
 * the per-chunk softmax statistics of the score step). */
size_t critiprefill_workspace_bytes(const critiprefill_params *p);

/*
 * Algorithm 1.  Writes scores[batch, n_q_heads, n1, n2] (fp32, contiguous): for every query head the
 * element-wise max/min representatives of each segment and block, the four representative products
 * scaled by score_scale with a row softmax over blocks, S = max((S1+S3)/2, (S2+S4)/2), blocks that
 * lie wholly after the segment set to 0, and, when prev_scores is not NULL, the layer fusion
 * alpha*S + (1-alpha)*prev_scores (prev_scores has the shape of scores; it may alias scores).
 * Values below the smallest normal fp32 are written as 0.
 * q, k: device, dtype per params.  workspace: device, >= critiprefill_workspace_bytes().
 */
int critiprefill_estimate(const critiprefill_params *p, const void *q, const void *k,
                          const float *prev_scores, float *scores,
                          void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * critiprefill_estimate for callers that cannot allocate device memory and have no workspace to hand in
 * (code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc): the same kernels and
 * the same result, bit for bit, with the scratch in a fixed array inside the library's device image
 * instead of a caller workspace.  Calls no allocating routine.
 * Limit: critiprefill_workspace_bytes(p) must not exceed CRITIPREFILL_STATIC_SCRATCH_BYTES (32 MiB; the five
 * benchmark configurations need 0.1 to 28 MiB), otherwise CP_ERR_WORKSPACE and nothing is launched.
 * Every GPU the library runs on holds its own copy of the array until the process ends; the device that is
 * current at the call is used (it must be the device of hip_stream).  All calls on one GPU share the array:
 * two calls whose kernels may overlap (different streams, or threads) race; calls on one stream are ordered.
 * Nothing in the array has to start at zero (every value read by a call was written by that call).
 * CP_ERR_LAUNCH if the array's device address cannot be resolved.
 */
#define CRITIPREFILL_STATIC_SCRATCH_BYTES (32u << 20)
int critiprefill_estimate_static(const critiprefill_params *p, const void *q, const void *k,
                                 const float *prev_scores, float *scores, void *hip_stream);

/*
 * Algorithm 2, the top-k line.  For every row (batch, head, segment j) of scores: the candidates are
 * blocks 0 .. j*r - L_j - 1 with L_j = min(local_blocks, j*r); the min(budget_blocks, #candidates)
 * largest scores are kept (ties to the smaller index); the list written to
 * block_idx[batch, n_q_heads, n1, list_len] (int32) is those indices ascending, then the L_j local
 * blocks, then the segment's own blocks; the unused tail is -1 and block_cnt[batch, n_q_heads, n1]
 * (int32) holds the list length.
 */
int critiprefill_select(const critiprefill_params *p, const float *scores,
                        int32_t *block_idx, int32_t *block_cnt, void *hip_stream);

/*
 * Algorithm 2, the attention loop, all segments in one launch.  Query t of segment j attends to the
 * tokens u <= t of the blocks listed in block_idx[batch, head, j, 0..block_cnt-1] (any strictly
 * ascending list of block indices < n2 is accepted; row pitch critiprefill_list_len()).
 * out has the dtype and strides (o_stride) of the parameter block.  lse (nullable) receives
 * log(sum exp(scaled logits)) per query, fp32 [batch, n_q_heads, seq_len]; a query with no visible
 * key gets output 0 and lse -inf.
 */
int critiprefill_sparse_attn(const critiprefill_params *p, const void *q, const void *k, const void *v,
                             const int32_t *block_idx, const int32_t *block_cnt,
                             void *out, float *lse, void *hip_stream);

/*
 * Extension of the paper's single-head description (it gives no rule for sharing a list between heads):
 * ONE list per (batch, KV head, segment) for all query heads of that KV head, taken from the element-wise
 * maximum of their scores.  critiprefill_select_shared reads scores[batch, n_q_heads, n1, n2] and writes
 * block_idx[batch, n_kv_heads, n1, list_len] / block_cnt[batch, n_kv_heads, n1] by the same rule as
 * critiprefill_select applied to max over the group's heads; critiprefill_sparse_attn_shared is
 * critiprefill_sparse_attn reading those lists (query head h uses the list of KV head
 * h / (n_q_heads / n_kv_heads)).  Same argument checks and errors as the per-head entry points.
 */
int critiprefill_select_shared(const critiprefill_params *p, const float *scores,
                               int32_t *block_idx, int32_t *block_cnt, void *hip_stream);
int critiprefill_sparse_attn_shared(const critiprefill_params *p, const void *q, const void *k, const void *v,
                                    const int32_t *block_idx, const int32_t *block_cnt,
                                    void *out, float *lse, void *hip_stream);

/* Eq. 2 with the causal mask u <= t: the dense baseline.  Same tensors as sparse_attn, no lists. */
int critiprefill_dense_causal_attn(const critiprefill_params *p, const void *q, const void *k, const void *v,
                                   void *out, float *lse, void *hip_stream);

/*
 * The cache
 * ---------
 * K and V of all sequences lie in pages of page_size tokens: k_cache and v_cache are [n_pages, n_kv_heads, page_size, row],
 * contiguous, so that a head's tokens of a page are one piece.  A row is 128 elements of `dtype` (CP_CACHE_PLAIN), or (CP_CACHE_MXFP8) 128
 * OCP e4m3 elements with one power of two for each 32 channels: the bytes e of k_scale and v_scale, [n_pages,
 * n_kv_heads, page_size, 4], stand for 2^(e - 127); 2^e is the smallest with max |x| <= 448 * 2^e, e in 1 .. 254.  Values that are not
 * finite have no part in the maximum and are held as NaN.  With CP_CACHE_PLAIN the scales are not read and may be NULL.
 * CP_CACHE_MXFP4: a row is 128 OCP e2m1 elements (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign), 64 bytes, the even channel of two in the lower half of their byte, and
 * scales as above: 2^e is the smallest with max |x| <= 7 * 2^e, e in 2 .. 252.  An element is rounded to the nearest, ties to the even code; what lies above 6 is off by a unit at
 * most, no more than rounding costs between 4 and 6, where the next scale's steps would be two units.  (e == 252 alone holds larger maxima, as 6 * 2^125.)  32 channels that
 * are not all finite have e = 255 and are NaN together; that is what e = 255 stands for under any elements.  253 and 254 no write gives: what a row that sees a token with them gets has no meaning.
 * A token's place is its slot, page * page_size + offset; a token whose slot is not in 0 .. n_pages * page_size - 1 has no place: it is
 * not written, and read as zeros.  Two tokens of one written call must not have the same slot: what it then holds is made of both.
 *
 * Tensors are [tokens, heads, 128]: `tokens` rows, those of all sequences one after another, with strides of token and head in the
 * parameter block (elements, multiples of 8; channels lie together), so that the parts of a joint projection are read where they are.
 * Written tensors: strides of at least 128 that leave every row its own place.  tokens == 0 (and n_seqs == 0) is no error: nothing is launched or looked at.
 */
enum { CP_CACHE_PLAIN = 0, CP_CACHE_MXFP8 = 1, CP_CACHE_MXFP4 = 4 };     /* 2 and 3 are not formats */

typedef struct critiprefill_cache_params {
    int32_t n_q_heads, n_kv_heads, head_dim;  /* head_dim must be 128; n_q_heads is not read by cache_write and cache_read */
    int32_t dtype;                            /* CP_DTYPE_*: of Q, K, V, the outputs, the weights and plain pages */
    int32_t tokens;                           /* rows of the tensors */
    int32_t cache_format;                     /* CP_CACHE_* */
    int32_t page_size, n_pages;               /* page_size: a power of two, 16 or more; n_pages * page_size < 2^31 */
    int32_t n_seqs, max_pages;                /* paged_attn: sequences, and the pitch of the page table; max_pages * page_size < 2^30, and all tiles of new tokens
                                                 (16 rows or more each) by the steps over max_pages * page_size keys (64 or more each) by n_kv_heads < 2^31 */
    int32_t max_q_len, max_kv_len;            /* paged_attn: new tokens, and tokens in all, that a sequence has at most, 0: not known (tokens, and
                                                 max_pages * page_size).  They choose the kernel and the way the work is cut; more are right too.  A table much
                                                 wider than the sequences are long hides that these are short: 32 single tokens of 760 keys 26 us, with max_kv_len 20;
                                                 over pages of 4 bits 3 single tokens and a chunk of 300 of 2300 keys in a table of 131072 49 us, with max_kv_len 39 */
    int32_t rotary_dim, rotary_interleaved;   /* norm_rope: channels that turn (0 .. 128, a multiple of 16), and how they pair */
    float norm_eps, attn_scale;               /* attn_scale: 0 -> 1/sqrt(head_dim) */
    int64_t q_stride[2], k_stride[2], v_stride[2]; /* token, head.  cache_read: k_stride, v_stride are the outputs' */
    int64_t o_stride[2], ko_stride[2];        /* q_out or out; k_out */
} critiprefill_cache_params;

/*
 * For every token and head, in fp32 and rounded once: y = x / sqrt(mean(x^2) + norm_eps) * weight over the head's 128 channels (q_weight,
 * k_weight: 128 elements of dtype; NULL: y = x), then for c < rotary_dim / 2 the channels (c, c + rotary_dim / 2), or (2c, 2c + 1) with
 * rotary_interleaved, turned by the angle positions[token] * inv_freq[c]: (y1 cos - y2 sin, y2 cos + y1 sin).  inv_freq: rotary_dim / 2
 * doubles, radians for each position; the angle is worked out in fp64.  positions: int32[tokens], of any sign.  Both may be NULL with rotary_dim == 0.
 * q_out may be q and k_out may be k, with the same strides; other overlaps are not allowed.
 */
int critiprefill_norm_rope(const critiprefill_cache_params *p, const void *q, const void *k, const void *q_weight, const void *k_weight,
                           const double *inv_freq, const int32_t *positions, void *q_out, void *k_out, void *hip_stream);

/* The same for q; k goes, and v as it is, to slots[token] of the cache (int32[tokens]).  With CP_CACHE_MXFP8 and CP_CACHE_MXFP4 k is quantised from fp32. */
int critiprefill_norm_rope_write(const critiprefill_cache_params *p, const void *q, const void *k, const void *v, const void *q_weight, const void *k_weight,
                                 const double *inv_freq, const int32_t *positions, const int32_t *slots, void *q_out, void *k_cache, void *v_cache,
                                 uint8_t *k_scale, uint8_t *v_scale, void *hip_stream);

/* k, v of `tokens` tokens into the cache, and the values that the cache holds for `tokens` slots, in any order, back as tensors of dtype. */
int critiprefill_cache_write(const critiprefill_cache_params *p, const void *k, const void *v, const int32_t *slots, void *k_cache, void *v_cache,
                             uint8_t *k_scale, uint8_t *v_scale, void *hip_stream);
int critiprefill_cache_read(const critiprefill_cache_params *p, const int32_t *slots, const void *k_cache, const void *v_cache, const uint8_t *k_scale,
                            const uint8_t *v_scale, void *k, void *v, void *hip_stream);

/* Bytes of scratch critiprefill_paged_attn needs: parts of results that several workgroups work on.  It depends on heads, dtype, cache_format and max_q_len
 * (tokens where that is 0) alone, not on lengths.  Contents do not matter before a call; calls that may overlap need one each.  0 for a block that paged_attn refuses. */
size_t critiprefill_paged_workspace_bytes(const critiprefill_cache_params *p);

/*
 * Attention of new tokens over the cache, which holds their own K and V already.  Sequence i has the rows q_start[i] .. q_start[i + 1] - 1 of q
 * (q_start: int32[n_seqs + 1], ascending from 0 to tokens), kv_len[i] tokens in all, the new ones last, and token u of it lies in page
 * page_table[i, u / page_size] (int32[n_seqs, max_pages]) at u % page_size.  The t-th of its n new tokens sees the tokens u <= kv_len[i] - n + t.
 * out[tokens, n_q_heads, 128] has dtype and o_stride; lse (nullable, fp32 [tokens, n_q_heads]) receives log(sum exp(scaled logits)).  A
 * row that sees nothing gets output 0 and lse -inf.  All four arrays are read on the device and the lengths never by the host: a captured call follows them.
 * Whatever they hold, nothing outside the tensors is touched: rows and lengths are cut to the tensors' sizes, tokens of a page outside the pool are seen
 * by no row, and with a q_start that does not ascend nothing is done.  Rows of no sequence are not written.  out must not overlap q or the cache.  At most 64
 * query heads for a KV head.
 * Logits, maxima and sums are fp32.  Over pages of 4 bits fp32 queries and weights go into their products as bf16 numbers that add up to them: of one below 2^-110 what lies below
 * 2^-133 is lost.  With dtype bf16 a weight is rounded to bf16 for its product with V (not for the sum of weights), and out once at the end.
 * The same call on the same contents gives the same bits.  Where a row's sum over keys is cut depends on the other sequences of the call, max_q_len and max_kv_len, and so do its last bits.
 */
int critiprefill_paged_attn(const critiprefill_cache_params *p, const void *q, const void *k_cache, const void *v_cache, const uint8_t *k_scale,
                            const uint8_t *v_scale, const int32_t *page_table, const int32_t *q_start, const int32_t *kv_len, void *out, float *lse,
                            void *workspace, size_t workspace_bytes, void *hip_stream);

const char *critiprefill_strerror(int status);
int critiprefill_version(void);

#ifdef __cplusplus
}
#endif
#endif /* CRITIPREFILL_H */
