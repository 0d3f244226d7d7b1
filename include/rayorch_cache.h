/*
 * rayorch_cache.h — C ABI of the model-step operators beside the lineage path.
 *
 * A Call's model step takes the Grains of a ready batch and keeps, for every
 * sequence it works on (a parent: a document, a video, a stream of frames), a
 * paged key/value cache.  The bookkeeping of such a cache is lineage:
 *
 *   - the pages of a sequence are the children of the expansion
 *     sequences -> pages, in ordinal order: d_page_base is that expansion's
 *     d_offsets, and d_pages names the pool page of each child;
 *   - the new tokens of a step are the children of the expansion
 *     sequences -> tokens: d_tok_base is its d_offsets, d_tok_seq its
 *     d_child_parent; ro_expand (or ro_expand_noalloc) writes both.
 *
 *   ro_rotary        rotary positions with several axes, and their gradient
 *   ro_cache_append  rotary on q and k; k and v into the cache's pages
 *   ro_cache_attend  attention of the new tokens over the cache
 *   ro_cache_weigh   the attention weight every cached token gathered
 *   ro_cache_evict   keeps each head's heaviest tokens, in fresh pages
 *
 * The conventions of rayorch_gpu.h hold: d_ pointers are device memory of the
 * context's GPU and are not kept; work is issued on the context's stream, in
 * call order, after the Calls' pending admissions; nothing waits on the host
 * and nothing throws.  Argument errors that the host can see are RO_E_INVAL
 * with no side effects (RO_E_OVERFLOW beyond a stated limit).  What only the
 * GPU can see is recorded in the context and returned by the next call that
 * synchronises: RO_E_CAPACITY where a length exceeds the sequence's pages or
 * an output, RO_E_INVAL where a page, a sequence, a token range or a range of a
 * page list (beyond the list's last offset) is out of bounds.  Nothing outside
 * the described arrays is read or written even then: the tokens concerned are
 * left out, and the call's results are void.
 * Workspaces belong to the context and grow on demand, so a call that will be
 * captured into a CUDA graph runs once uncaptured first.  Graphs stay good when
 * a later call needs larger ones: those that captured calls use live as long as
 * the context.
 *
 * Types: RO_BF16 and RO_F16 (ro_rotary also RO_F32).  Sums, softmax
 * statistics, rotations and scores are computed in 32 bits and rounded once,
 * to the output's type; attention rounds the softmax weights of a tile to the
 * cache's type for the matrix product with the values (f16 weights are held
 * higher by a power of two for it: none above 2^-36 of its row's largest is
 * lost).
 * Tensors are [tokens][heads][head_dim] with an element stride of 1 in the
 * last dimension and token and head strides in elements.  Where not said
 * otherwise the cache operators want 16-byte aligned pointers and strides that
 * are multiples of 8 elements.  Limits: head_dim a multiple of 8 up to 128
 * (ro_rotary: even, up to 256), fewer than 2^31 tokens per call and per
 * sequence, at most 65,535 heads.
 */
#ifndef RAYORCH_CACHE_H
#define RAYORCH_CACHE_H

#include "rayorch_gpu.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { RO_BF16 = 0, RO_F16 = 1, RO_F32 = 2 };

/* A paged cache: pools k and v of n_pages pages of page_size tokens, each
 * [page][head][slot][head_dim] with the given strides in elements (the same
 * for k and v), and the page lists of n_seqs sequences. */
typedef struct {
  void* d_k;
  void* d_v;
  int32_t dtype;                /* RO_BF16 or RO_F16 */
  uint32_t n_pages, page_size, n_heads, head_dim;
  uint32_t n_seqs;
  uint64_t page_stride, head_stride, slot_stride;
  const uint64_t* d_page_base;  /* uint64[n_seqs+1]: first page of each sequence, ascending */
  const uint32_t* d_pages;      /* uint32[d_page_base[n_seqs]]: pool pages, in order */
} ro_cache;

/* Rotary positions with n_axes axes (1 to 4).  The first 2R dimensions of a
 * head turn, R = pairs[0] + .. + pairs[n_axes-1]; the rest pass through.  Pair
 * p of R (counted over all axes, axis 0's first) turns by
 * pos[token][axis of p] * base^(-p/R) radians; it is dimensions (p, p + R), or
 * (2p, 2p + 1) if interleaved.  base >= 1. */
typedef struct {
  uint32_t n_axes;
  uint32_t pairs[4];
  uint32_t interleaved;
  double base;
} ro_rope;

/* ------------------------------------------------------------------------
 * ro_rotary — turn a tensor by its positions.
 *   d_x, d_out  [n_tokens][n_heads][head_dim] of `dtype`, strides in elements
 *               (tok, head), any alignment to the element; d_out may be d_x
 *               with the same strides.
 *   d_pos       int32[n_tokens][n_axes], any value; the angle is reduced to a
 *               turn in integers, so large positions lose no accuracy.
 *   inverse     non-zero: turn back.  The gradient of the turned tensor is the
 *               inverse turn of the incoming gradient, so this is the
 *               operator's backward pass.
 */
ro_status ro_rotary(ro_ctx* ctx, int32_t dtype, const void* d_x, uint64_t x_tok, uint64_t x_head,
                    void* d_out, uint64_t out_tok, uint64_t out_head, uint64_t n_tokens,
                    uint32_t n_heads, uint32_t head_dim, const int32_t* d_pos, const ro_rope* rope,
                    int32_t inverse);

/* ------------------------------------------------------------------------
 * ro_cache_append — put a step's new tokens into the cache.
 *   d_tok_base  uint64[n_seqs+1] and d_tok_seq uint32[n_tokens]: the expansion
 *               sequences -> new tokens (see above); n_tokens its children.
 *   d_len       uint32[n_seqs]: tokens each sequence holds with the new ones.
 *               Token t of sequence s goes to slot
 *               d_len[s] - (new tokens of s) + (t - d_tok_base[s]); a slot
 *               before 0 is left out (a chunk longer than its cache).
 *   d_pos, rope positions int32[n_tokens][n_axes] and their rotary; rope NULL
 *               (d_pos then unused): k and q are copied as they are.
 *   d_q, d_q_out  [n_tokens][n_q_heads][head_dim]: turned (d_q_out may be d_q
 *               with the same strides); n_q_heads 0 leaves q out.
 *   d_k, d_v    [n_tokens][n_heads][head_dim] of the cache's type; k is turned.
 */
ro_status ro_cache_append(ro_ctx* ctx, const ro_cache* cache, const uint64_t* d_tok_base,
                          const uint32_t* d_tok_seq, uint64_t n_tokens, const uint32_t* d_len,
                          const int32_t* d_pos, const ro_rope* rope, const void* d_q, uint64_t q_tok,
                          uint64_t q_head, uint32_t n_q_heads, void* d_q_out, uint64_t qo_tok,
                          uint64_t qo_head, const void* d_k, uint64_t k_tok, uint64_t k_head,
                          const void* d_v, uint64_t v_tok, uint64_t v_head);

/* ------------------------------------------------------------------------
 * ro_cache_attend — attention of new tokens over the cache that holds them.
 * n_q_heads is a multiple of the cache's heads; query head g reads cache head
 * g / (n_q_heads / n_heads).  A new token at slot a sees the slots j <= a with
 * window == 0, j > a - window, or j < sinks (a sliding window that counts the
 * token itself, and first tokens that stay visible).
 *   d_out = sum_j p_j v_j, p = softmax over the seen j of scale * q.k_j;
 *   d_lse = ln sum_j exp(scale * q.k_j), float[n_tokens][n_q_heads] or NULL.
 * A token that sees nothing (its slot lies before 0) gets out 0, lse -inf.
 * Slots that no token of a sequence's chunk sees are never used, whatever
 * they hold.  (Tokens of one chunk share tiles: a NaN or infinity in a value
 * that one of them sees may reach others of the same sequence.)
 *   max_new     bound on the new tokens of any sequence (0: n_tokens); a
 *               sequence with more is left out and recorded (RO_E_INVAL).
 *   max_len     expected largest d_len (0: unknown); it only guides how the
 *               keys are split over the GPU.
 *   d_out       [n_tokens][n_q_heads][head_dim] of the cache's type; not d_q.
 * Results do not depend on scheduling: equal calls give equal bits.
 */
ro_status ro_cache_attend(ro_ctx* ctx, const ro_cache* cache, const uint64_t* d_tok_base,
                          uint64_t n_tokens, uint32_t max_new, const uint32_t* d_len,
                          uint32_t max_len, const void* d_q, uint64_t q_tok, uint64_t q_head,
                          uint32_t n_q_heads, float scale, uint32_t window, uint32_t sinks,
                          void* d_out, uint64_t out_tok, uint64_t out_head, float* d_lse);

/* ------------------------------------------------------------------------
 * ro_cache_weigh — the attention weight that cached tokens gathered.
 * For every sequence s, cache head h and slot j < d_len[s]:
 *   d_score[s][h][j] = decay * d_past[s][h][j]  (0 for the step's new slots)
 *     + sum over s's new tokens and h's query heads of
 *       exp(scale * q.k_j - lse), where the token sees slot j.
 * Arguments as in ro_cache_attend; d_lse is its d_lse output.  d_past and
 * d_score are float[n_seqs][n_heads][score_cap]; they may be the same array
 * (but may not overlap otherwise).
 * Slots from d_len[s] on are not touched.  A length above score_cap is
 * recorded (RO_E_CAPACITY).  Equal calls give equal bits.
 */
ro_status ro_cache_weigh(ro_ctx* ctx, const ro_cache* cache, const uint64_t* d_tok_base,
                         uint64_t n_tokens, uint32_t max_new, const uint32_t* d_len,
                         const void* d_q, uint64_t q_tok, uint64_t q_head, uint32_t n_q_heads,
                         float scale, uint32_t window, uint32_t sinks, const float* d_lse,
                         float decay, const float* d_past, float* d_score, uint64_t score_cap);

/* ------------------------------------------------------------------------
 * ro_cache_evict — cut every sequence back to at most `budget` tokens.
 * A sequence of at most budget tokens keeps them all.  Of a longer one every
 * cache head keeps the first `sinks`, the last `recent` and, of the rest, the
 * budget - sinks - recent tokens with the largest score (equal scores, and
 * -0 with 0: the lowest slot; a NaN counts below every number), in slot order.
 * Kept keys, values and scores move to the sequence's new pages.
 *   d_score     float[n_seqs][n_heads][score_cap] (see ro_cache_weigh).
 *   d_dst_base, d_dst_pages  the new page lists, as d_page_base and d_pages:
 *               ceil(min(length, budget) / page_size) pages per sequence.  No
 *               new page may be one of the old ones (the old ones are free
 *               once the call is done).  Too few pages: RO_E_CAPACITY is
 *               recorded and the tokens past them are not moved.
 *   d_keep      uint32[n_seqs][n_heads][budget] out: kept slots, ascending
 *               (entries past the kept ones are not written).
 *   d_len_out   uint32[n_seqs] out: min(length, budget); may be d_len (but may
 *               not overlap it otherwise: RO_E_INVAL).
 *   d_score_out float[n_seqs][n_heads][score_cap] out or NULL: kept scores;
 *               no part of d_score.
 * sinks + recent <= budget, budget >= 1.
 */
ro_status ro_cache_evict(ro_ctx* ctx, const ro_cache* cache, const uint32_t* d_len,
                         const float* d_score, uint64_t score_cap, uint32_t budget, uint32_t sinks,
                         uint32_t recent, const uint64_t* d_dst_base, const uint32_t* d_dst_pages,
                         uint32_t* d_keep, uint32_t* d_len_out, float* d_score_out);

#ifdef __cplusplus
}
#endif
#endif /* RAYORCH_CACHE_H */
