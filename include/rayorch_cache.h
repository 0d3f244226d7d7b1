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
 * and for steps that branch and answer:
 *
 *   ro_cache_attend_biased  attention with capped scores, a distance bias,
 *                           document and prefix masks
 *   ro_sample               tokens from logits and given random numbers
 *   ro_cache_fork           sequences go on in any number of continuations
 *   ro_cache_compact        the pages in use move to the low end of the pool
 *   ro_cache_copy           the same copies of pages in another layer's pool
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
 * lost); products scale * q.k without a cap stay below 2^22 in size over f16
 * caches, 2^28 over bf16 ones.
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
 * scale is finite, times log2 e too.
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

/* ------------------------------------------------------------------------
 * ro_cache_attend_biased — attention whose scores are capped, fall with
 * distance, or are masked by documents and prefixes.  With a = the slot of a
 * new token t and x_j = scale * q.k_j:
 *   cap > 0:   x_j becomes cap * tanh(x_j / cap);
 *   d_slope:   then slope[query head] * |a - j| is taken off (finite slopes of
 *              either sign; distances count slots; what passes 32 bits' range
 *              counts as infinite);
 *   d_first:   t sees no slot before d_first[t], the first one of its
 *              document; sinks are the `sinks` slots from there on.  A token
 *              whose d_first lies behind its own slot sees nothing (tokens
 *              that only pad a chunk);
 *   d_until:   t also sees the slots behind its own that lie before d_until[t]
 *              (a prefix's or a frame's end; clipped to the sequence's length).
 * So t sees slot j when first <= a, first <= j < max(a + 1, until) and
 * window == 0, j > a - window, or j < first + sinks.  Everything else is
 * ro_cache_attend's: arguments, outputs, empty rows (out 0, lse -inf), unseen
 * slots never used, equal bits for equal calls.
 * cap must be 0 or from 1e-6 to 1e30, with |scale / cap| 0 or from 1e-37 to 1e30.
 */
typedef struct {
  float cap;                    /* 0: none */
  const float* d_slope;         /* float[n_q_heads] or NULL (0) */
  const uint32_t* d_first;      /* uint32[n_tokens] or NULL (0) */
  const uint32_t* d_until;      /* uint32[n_tokens] or NULL (0) */
} ro_bias;

ro_status ro_cache_attend_biased(ro_ctx* ctx, const ro_cache* cache, const uint64_t* d_tok_base,
                                 uint64_t n_tokens, uint32_t max_new, const uint32_t* d_len,
                                 uint32_t max_len, const void* d_q, uint64_t q_tok, uint64_t q_head,
                                 uint32_t n_q_heads, float scale, uint32_t window, uint32_t sinks,
                                 const ro_bias* bias, void* d_out, uint64_t out_tok,
                                 uint64_t out_head, float* d_lse);

/* ------------------------------------------------------------------------
 * Pages of a cache that several sequences share.  d_refs counts for every pool
 * page how many entries of page lists name it (and whatever else holds it); a
 * page with 0 is free.  Shared pages are full ones: a page that a sequence still
 * writes is its own.  Outputs share no memory with inputs or one another but
 * where it is said (RO_E_INVAL; recorded where they lie behind the first entry of
 * a page list whose length only the GPU knows).
 */
/* Copies of pages: d_n[0] of them (at most cap), copy i the first d_slots[i]
 * slots of pool page d_from[i] to page d_to[i]. */
typedef struct {
  uint32_t* d_from;             /* uint32[cap] */
  uint32_t* d_to;               /* uint32[cap] */
  uint32_t* d_slots;            /* uint32[cap] */
  uint32_t* d_n;                /* uint32 (one) */
  uint64_t cap;
} ro_moves;

/* A page list's entry for which the pool had no page. */
#define RO_NO_PAGE 0xFFFFFFFFu

/* ------------------------------------------------------------------------
 * ro_cache_fork — sequences go on in their continuations: an expansion
 * sequences -> continuations.  A sequence without any ends (its pages are
 * released), one with one goes on, one with several is forked; continuations
 * and their pages are the children of another expansion, continuations -> pages,
 * and any of them may have more pages than its tokens fill (room to grow).
 *   d_len        uint32[n_seqs]: tokens each sequence holds.
 *   d_child_base uint64[n_seqs+1], d_child_parent uint32[n_children]: the
 *                expansion sequences -> continuations (see ro_expand).
 *   d_dst_base   uint64[n_children+1], d_dst_seq uint32[n_dst]: the expansion
 *                continuations -> pages; n_dst its children.
 *   d_refs       uint32[cache->n_pages] (see above).
 *   d_refs_out   uint32[n_pages] out: with the old lists' entries taken off and
 *                the new ones' added; may be d_refs.
 *   d_dst_pages  uint32[n_dst] out: the continuations' page lists.  Pages full
 *                of tokens are the parent's; so are the further ones for its
 *                first continuation, where d_refs is 1; every other entry, in
 *                order, gets the next page that is free in d_refs, lowest first.
 *   d_len_out    uint32[n_children] out: tokens of each continuation, its
 *                parent's (not d_len).
 *   moves        out: the copies of open pages, parent to continuation, in
 *                order; cap >= n_children.  The cache's pools are copied by this
 *                call, those of other layers with ro_cache_copy.
 * Recorded: RO_E_CAPACITY when the pool has too few free pages (those entries
 * are RO_NO_PAGE, and not copied to) or a continuation's pages do not hold its
 * parent's tokens; RO_E_INVAL for parents, pages and ranges out of bounds, and
 * for a page whose d_refs is below its entries.
 */
ro_status ro_cache_fork(ro_ctx* ctx, const ro_cache* cache, const uint32_t* d_len,
                        const uint64_t* d_child_base, const uint32_t* d_child_parent,
                        uint64_t n_children, const uint64_t* d_dst_base, const uint32_t* d_dst_seq,
                        uint64_t n_dst, uint32_t* d_dst_pages, uint32_t* d_len_out,
                        const uint32_t* d_refs, uint32_t* d_refs_out, const ro_moves* moves);

/* ------------------------------------------------------------------------
 * ro_cache_compact — the U pages in use (d_refs > 0) move to the U lowest
 * places: the k-th used page at or above U goes to the k-th free one below U.
 *   d_pages_out  uint32[n_list] out: cache->d_pages with moved pages renamed;
 *                may be d_pages.  n_list >= d_page_base[n_seqs], else
 *                RO_E_CAPACITY is recorded and the rest is not written.
 *   d_refs       uint32[n_pages]; d_refs_out uint32[n_pages] out, moved along
 *                (0 from U on); may be d_refs.
 *   d_n_used     uint32 out: U.
 *   moves        out: the moves, ascending, of page_size slots each; cap at
 *                least n_pages / 2.  The cache's pools are copied by this call,
 *                those of other layers with ro_cache_copy.
 * Recorded: RO_E_INVAL for a list's page that is out of bounds or free (it
 * keeps its name).
 */
ro_status ro_cache_compact(ro_ctx* ctx, const ro_cache* cache, uint32_t* d_pages_out,
                           uint64_t n_list, const uint32_t* d_refs, uint32_t* d_refs_out,
                           uint32_t* d_n_used, const ro_moves* moves);

/* ------------------------------------------------------------------------
 * ro_cache_copy — copy pages within the cache's pools (k and v), for instance
 * those of another layer after ro_cache_fork or ro_cache_compact.  No page that
 * a copy writes may be read or written by another one.  Recorded: RO_E_INVAL for
 * a page or a number of slots out of bounds (that copy is left out),
 * RO_E_CAPACITY when d_n is above cap (cap copies are made).
 * cache->d_page_base and d_pages are not read.
 */
ro_status ro_cache_copy(ro_ctx* ctx, const ro_cache* cache, const ro_moves* moves);

/* ------------------------------------------------------------------------
 * ro_sample — draw each row's token from its logits and a given random number.
 * With w_i = exp((x_i - max x) / temperature) and the tokens in order, larger
 * logit first and equal ones (0 and -0 among them) by index, a token stays when
 *   top_k:  it is among the first top_k (0: all);
 *   top_p:  the sum of w over the tokens ahead of it is less than top_p times
 *           the sum over those that top_k leaves (1: all stay; 0: the first);
 *   min_p:  w_i >= min_p (0: all).
 * The token drawn is the first of those that stay, by index, whose running sum
 * of w passes u times the sum over all of them.  temperature 0 draws the
 * largest logit, the first of equal ones.  A logit that is -inf or NaN is never
 * drawn and does not count; differences of logits past 32 bits' range are
 * infinite.
 *   d_logits   [n_rows][vocab] of `dtype` (bf16, f16 or f32), row_stride
 *              elements from row to row, any alignment to the element.
 *   how        settings of each row, NULL (also in it): the neutral ones.
 *   d_u        float[n_rows], 0 <= u < 1.
 *   d_token    uint32[n_rows] out; RO_NO_TOKEN where nothing can be drawn.
 *   d_logp     float[n_rows] out or NULL: ln of the drawn token's share of the
 *              sum over those that stay (-inf where none).
 *   d_kept     uint32[n_rows] out or NULL: how many stay (drawing the largest: 1).
 * Weights are about 2^-40 exact and their sums are exact: tokens do not depend
 * on how the work is split.  vocab is at most 393,216.  Outputs share no memory
 * with inputs or one another (RO_E_INVAL).  Recorded: RO_E_INVAL for
 * a row whose settings or u are out of range or NaN (RO_NO_TOKEN there).
 */
#define RO_NO_TOKEN 0xFFFFFFFFu
typedef struct {
  const float* d_temperature;   /* float[n_rows] or NULL (1); finite, at least 0 */
  const uint32_t* d_top_k;      /* uint32[n_rows] or NULL (0) */
  const float* d_top_p;         /* float[n_rows] or NULL (1); 0 to 1 */
  const float* d_min_p;         /* float[n_rows] or NULL (0); 0 to 1 */
} ro_sampling;

ro_status ro_sample(ro_ctx* ctx, int32_t dtype, const void* d_logits, uint64_t row_stride,
                    uint64_t n_rows, uint32_t vocab, const ro_sampling* how, const float* d_u,
                    uint32_t* d_token, float* d_logp, uint32_t* d_kept);

#ifdef __cplusplus
}
#endif
#endif /* RAYORCH_CACHE_H */
