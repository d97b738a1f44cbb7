/*
 * lynx/attention.h -- the attention half of a decode step, beside the MoE half that lynx.h declares: cache pages and slots of
 * a step's tokens, norms and rotation of queries and keys with the write into the paged cache, attention over that cache, and
 * attention of a batch that shares a long prefix.
 *
 * Conventions are those of lynx.h: DEVICE pointers owned by the caller unless a parameter says "host", kernels only enqueued
 * on `stream`, no allocation, no synchronisation, nothing read back on the host (a sequence of calls can be captured into a
 * hipGraph), LYNX_OK or a negative error with lynx_last_error(), nothing enqueued on error.  Inputs are assumed finite, except
 * that cache slots which no token occupies may hold anything.  No index array can cause an access out of bounds: tokens
 * whose page number lies outside [0, num_pages) are not written and not seen by any query, row ranges are clamped to [0, T], and
 * lengths to what a row of the block table can hold; what rows of out hold that lie in several requests' ranges, or in the range
 * of a request whose q_start lies in front of an earlier one's, is not specified.
 *
 * A step: B requests, request b brings new_len[b] >= 0 new tokens behind the ctx_len[b] it has in the cache.  The T rows of q,
 * k, v, out, positions and slots hold the new tokens of request 0, then of request 1, and so on: request b's are rows
 * q_start[b] .. q_start[b+1]-1.  Rows behind the last request's are padding (a captured graph has a fixed T), and so are rows in
 * front of the first one's where q_start[0] > 0 (part of a larger step); the attention calls take padding rows that hold anything.
 *
 * Paged cache of one layer, page_size tokens a page (a multiple of 16), KVH key heads of D channels, elements bf16 or FP8 E4M3:
 *   k_cache [num_pages][KVH][page_size][D]    v_cache [num_pages][KVH][D][page_size]
 * (values transposed inside the page: what the second product of attention multiplies is then contiguous).  Token j of request b
 * sits in page block_table[b][j / page_size] at place j % page_size; its slot is page * page_size + place.  Both arrays start
 * on 16 bytes.  FP8: value = code * k_scale or v_scale (host floats, > 0 and finite); bf16 caches take 1 for both.
 *
 * Limits: 1 <= B <= LYNX_MAX_REQUESTS, 0 <= T <= LYNX_MAX_STEP_TOKENS, D = 64 or 128, KVH divides QH, QH <= 1024,
 * QH / KVH <= 256, page_size <= LYNX_MAX_PAGE_SIZE, num_pages <= LYNX_MAX_PAGES, max_pages * page_size <= 2^29, and for the
 * attention calls (B + T * QH / KVH / 16) * max_pages * page_size < 2^37.
 */
#ifndef LYNX_ATTENTION_H
#define LYNX_ATTENTION_H

#include "../lynx.h"

#ifdef __cplusplus
extern "C" {
#endif

#define LYNX_MAX_REQUESTS 1024
#define LYNX_MAX_STEP_TOKENS 65536
#define LYNX_MAX_PAGES 1048576
#define LYNX_MAX_PAGE_SIZE 1024
#define LYNX_CACHE_BF16 0
#define LYNX_CACHE_FP8 1

/*
 * Pages and slots of a step's tokens, from request lengths alone.
 *   ctx_len [B] int32 = tokens a request has in the cache; new_len [B] int32 = tokens it brings now, 0 = none, negative = the
 *   request has ended: its pages go back to the free ones and its seq_len becomes 0.
 *   block_table [B][max_pages] int32, in and out: entries of pages that a request holds already are kept, those of new pages
 *   are filled in, no other entry is written.  The first shared_pages entries of every row are pages the batch shares: never
 *   taken from the free ones and never given back (a request that starts on a shared prefix has ctx_len = its length).
 *   free_ring [num_pages] int32, in and out, and ring_state [2] int32 = {head, count}: the free pages are the count entries from
 *   place head on, round the ring.  New pages are taken at the head, in request order and token order; pages of ended requests
 *   are put behind the last free one, in the same orders, and are not given out again by the same call.  A head or count outside
 *   the ring is brought into it: the head modulo num_pages, the count to 0 .. num_pages.
 *   q_start [B+1] int32 out; seq_len [B] int32 out = ctx_len + new_len (0 for an ended request); positions [T] int32 out =
 *   place of the token in its sequence, 0 in padding rows; slots [T] int32 out, -1 in padding rows and for pages outside the
 *   cache; ring_state_out [2] int32 out.  seq_len may be ctx_len and ring_state_out may be ring_state, so that a captured
 *   step goes on from where its last replay ended; all other arrays are distinct.
 *   status [1] int32 out: 0, or a sum of
 *     LYNX_KV_NO_PAGES   the free pages did not suffice: the first request that they do not cover, and all behind it that bring
 *                        tokens, get none (they keep ctx_len, bring no rows and can be tried again);
 *     LYNX_KV_NO_ROWS    the same for the T rows;
 *     LYNX_KV_TOO_LONG   a request does not fit its row of the block table, or has a negative length: it alone is passed over;
 *     LYNX_KV_LOST_PAGES the ring has no place for all pages of the ended requests, which no pool of num_pages pages comes to whose
 *                        pages are each in one place (a count that is wrong, a page in two rows, shared_pages smaller than when
 *                        the rows were filled): as many as there is place for were put back, in order, the others are lost.
 */
#define LYNX_KV_NO_PAGES 1
#define LYNX_KV_NO_ROWS 2
#define LYNX_KV_TOO_LONG 4
#define LYNX_KV_LOST_PAGES 8
int lynx_kv_assign(const int32_t *ctx_len, const int32_t *new_len, int B, int T, int page_size, int num_pages, int max_pages,
                   int shared_pages, int32_t *block_table, int32_t *free_ring, const int32_t *ring_state, int32_t *q_start,
                   int32_t *seq_len, int32_t *positions, int32_t *slots, int32_t *ring_state_out, int32_t *status, void *stream);

/*
 * Norms of queries and keys for each head, their rotation by position, and the write of keys and values into the cache.
 *   For a head row x of q or k, all in fp32:  y = x * rsqrt(mean(x^2) + eps) * w  (no norm where its weight is NULL), then for
 *   the first `rot` channels, pairs (a, b) = (y[i], y[i + rot/2]) or, interleaved, (y[2i], y[2i+1]):
 *     a' = a cos(phi) - b sin(phi),  b' = b cos(phi) + a sin(phi),  phi = positions[t] * freqs[i],
 *   channels from rot on pass.  The product is taken and reduced to one turn in fp64, so far positions lose nothing.  One rounding
 *   to bf16 (or to E4M3 after the division by its scale, magnitudes beyond 448 to 448) at the end.  A NaN in k or v stays one in
 *   either cache.
 *   q [T][QH][D], k, v [T][KVH][D] bf16; q_stride, k_stride, v_stride = elements from one token to the next (heads of a token are
 *   contiguous), so that q, k, v can be parts of one row of a fused projection.  q_weight, k_weight [D] bf16 or NULL.
 *   freqs [rot/2] fp64, radians per position; rot = 0 (freqs may be NULL) rotates nothing.
 *   q_out [T][QH][D] bf16 out, rows q_out_stride apart; may be q itself.  All T rows are computed.
 *   slots [T]: where k and v go; tokens with a slot outside [0, num_pages * page_size) write nothing into the cache.
 *   No slot may appear twice (lynx_kv_assign's do not).  T == 0 is a no-op.
 * rot % 16 == 0 and rot <= D; pointers of 16-byte aligned rows: strides multiples of 8 elements, pointers on 16 bytes, else
 * LYNX_ERR_INVALID_ARG.
 */
int lynx_qk_norm_rope(const uint16_t *q, int64_t q_stride, const uint16_t *k, int64_t k_stride, const uint16_t *v,
                      int64_t v_stride, const uint16_t *q_weight, const uint16_t *k_weight, float eps, const int32_t *positions,
                      const int32_t *slots, const double *freqs, int rot, int interleaved, int T, int QH, int KVH, int D,
                      uint16_t *q_out, int64_t q_out_stride, void *k_cache, void *v_cache, int cache_format, float k_scale,
                      float v_scale, int num_pages, int page_size, void *stream);

/* Bytes of device workspace that lynx_attention and lynx_attention_prefix need for these sizes (contents need not be
 * preserved; calls that share a workspace must not overlap in time), 0 for sizes that they refuse.  prefix_len = 0 for
 * lynx_attention.  The workspace starts on 256 bytes.  The size does not fall when B, T or prefix_len grows: a workspace for the
 * largest step serves all smaller ones.  lynx_attention: about 288 * max(512, KVH) * (D + 2) * 4 bytes, 77 MB for D = 128 and up to 512 key
 * heads.  A prefix adds about 2 * R * KVH * (D + 2) * 4 bytes, R = min(T * QH / KVH, 128 * B, B * prefix_len / 4); where R * KVH is less than 65536,
 * the half of it for the prefix's own parts may be up to what 65536 takes (34 MB for D = 128). */
size_t lynx_attention_workspace_bytes(int B, int T, int QH, int KVH, int D, int prefix_len);

/*
 * Attention over the paged cache.  Row t of request b is at position pos = seq_len[b] - (q_start[b+1] - q_start[b]) + (t -
 * q_start[b]) and sees its tokens j <= pos with j > pos - window or j < sinks; window = 0: all j <= pos.
 *   out[t][h] = sum_j softmax_j(scale * q[t][h] . k_j) v_j over the tokens it sees, k and v of key head h / (QH / KVH).
 *   lse [T][QH] fp32 out or NULL = log(sum_j exp(scale * q . k_j)), natural.  A row that sees nothing: out 0, lse -inf.
 *   Rows outside every request are left as they were.
 * bf16 operands on the matrix cores, running maximum and sums in fp32; the softmax weights are rounded to bf16 for the second
 * product (their sum is taken before the rounding).  The new tokens' keys and values are in the cache already.
 *   max_new (host): the largest number of new tokens of a request, as far as the caller knows it (1 for a pure decode batch);
 *   which kernels are launched goes by it, the result does not depend on it being right.
 *   scale > 0, scale * k_scale a normal float; scores, q . k and times scale * k_scale * log2 e, within a float's range; window, sinks >= 0.  q_stride, out_stride as in lynx_qk_norm_rope (lse is dense); out does
 *   not overlap q (a row is read by several workgroups).
 */
int lynx_attention(const uint16_t *q, int64_t q_stride, const void *k_cache, const void *v_cache, int cache_format,
                   float k_scale, float v_scale, int num_pages, int page_size, const int32_t *block_table, int max_pages,
                   const int32_t *q_start, const int32_t *seq_len, int B, int T, int max_new, int QH, int KVH, int D, float scale,
                   int window, int sinks, uint16_t *out, int64_t out_stride, float *lse, void *workspace, void *stream);

/*
 * lynx_attention (without a window) for a batch whose sequences all begin with the same prefix_len tokens: their keys and values
 * are read once for the rows of the whole batch instead of once per request, and the two parts of each row's softmax are joined.
 *   prefix_table [ceil(prefix_len / page_size)] int32 = the pages of the prefix.  The rows of block_table hold whole sequences, the
 *   prefix included: the tokens from the last multiple of 64 in the prefix on are read through them (a prefix that ends inside a
 *   page is copied into each request's own page there).
 *   prefix_len (host) >= 0, <= max_pages * page_size; it need not be a multiple of anything.  Rows at positions inside the
 *   prefix see what is up to them, as in lynx_attention.
 *   Where that would not pay, T * QH / KVH >= 128 * B or > B * prefix_len / 4 (prompt chunks, whose rows fill the matrix products by
 *   themselves; a prefix that is short against them), the prefix is read through block_table, too, as lynx_attention does.
 */
int lynx_attention_prefix(const uint16_t *q, int64_t q_stride, const void *k_cache, const void *v_cache, int cache_format,
                          float k_scale, float v_scale, int num_pages, int page_size, const int32_t *block_table, int max_pages,
                          const int32_t *q_start, const int32_t *seq_len, const int32_t *prefix_table, int prefix_len, int B, int T,
                          int max_new, int QH, int KVH, int D, float scale, uint16_t *out, int64_t out_stride, float *lse,
                          void *workspace, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* LYNX_ATTENTION_H */
