// ro_step_api.cu — host side of include/rayorch_cache.h: argument checks, the
// choice of kernel by sizes, types and alignment, workspaces and launches.
#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "ro_step.h"

using namespace ro;

namespace {

constexpr uint32_t MAX_HEADS = 65535;
constexpr float LOG2_E = 1.44269504088896340736f;
constexpr uint64_t MAX_GRID = 0x7FFFFFFFull;
// Runs whose partial results a call keeps: 1,024 of attend_tiles' 133 KB,
// 16,384 of attend_few's 8 KB (about 136 MB either way, and the workspace's
// headroom of an eighth).
constexpr uint64_t MAX_RUNS = 1024, MAX_FEW_RUNS = 16384;

#define RO_TRY(x)               \
  do {                          \
    ro_status _s = (x);         \
    if (_s != RO_OK) return _s; \
  } while (0)

bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) % n) == 0; }
// two arrays of the same number of bytes
bool overlap(const void* p, const void* q, uint64_t bytes) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
  return (a < b ? b - a : a - b) < bytes;
}
// rows that are turned in place lie where they were
bool in_place_elsewhere(const void* x, uint64_t x_tok, uint64_t x_head, const void* y, uint64_t y_tok, uint64_t y_head,
                        uint64_t n_tokens, uint32_t n_heads) {
  return x == y && ((n_tokens > 1 && x_tok != y_tok) || (n_heads > 1 && x_head != y_head));
}

ro_status check_rope(StepCall& c, const char* fn, const ro_rope* r, uint32_t head_dim) {
  if (r->n_axes < 1 || r->n_axes > 4) return c.refuse(RO_E_INVAL, "%s: 1 to 4 axes", fn);
  uint64_t R = 0;
  for (uint32_t i = 0; i < r->n_axes; ++i) R += r->pairs[i];
  if (R == 0 || 2 * R > head_dim) return c.refuse(RO_E_INVAL, "%s: the pairs do not fit the head", fn);
  if (!(r->base >= 1.0) || !std::isfinite(r->base)) return c.refuse(RO_E_INVAL, "%s: base must be finite, at least 1", fn);
  return RO_OK;
}

// Frequencies of the pairs in 2^-64 turns, from doubles: a relative error of
// about 2^-52, which the largest position (2^31) makes 1e-6 radians of angle.
void fill_rope(const ro_rope* r, RopeTable* t) {
  // the last table of this thread: a program's calls share one description
  thread_local ro_rope last = {};
  thread_local RopeTable table = {};
  const bool same = last.n_axes == r->n_axes && std::equal(r->pairs, r->pairs + r->n_axes, last.pairs) &&
                    last.interleaved == r->interleaved && last.base == r->base;
  if (!same) {
    uint32_t p = 0, R = 0;
    for (uint32_t i = 0; i < r->n_axes; ++i) R += r->pairs[i];
    for (uint32_t i = 0; i < r->n_axes; ++i)
      for (uint32_t k = 0; k < r->pairs[i]; ++k, ++p) {
        const double turns = std::pow(r->base, -(double)p / (double)R) / 6.283185307179586476925;
        table.axis[p] = (uint8_t)i;
        table.freq[p] = (uint64_t)std::ldexp(turns, 64);
      }
    table.n_axes = r->n_axes;
    table.pairs = R;
    table.interleaved = r->interleaved != 0;
    last = *r;
  }
  *t = table;
}

// The widest access, in elements, that pairs, strides and pointers allow.
int turn_vec(const TurnArgs& a, size_t elem) {
  for (int v = 16 / (int)elem; v > 1; v /= 2) {
    bool ok = a.rope.pairs % v == 0 && (a.head_dim / 2) % v == 0;
    for (uint32_t k = 0; ok && k < a.n_parts; ++k) {
      const TurnPart& p = a.part[k];
      ok = aligned(p.src, v * elem) && aligned(p.dst, v * elem) && p.src_tok % v == 0 && p.src_head % v == 0 &&
           p.dst_head % v == 0 && (p.paged ? a.page_stride % v == 0 && a.slot_stride % v == 0 : p.dst_tok % v == 0);
    }
    if (ok) return v;
  }
  return 1;
}

ro_status check_cache(StepCall& c, const char* fn, const ro_cache* k) {
  if (!k) return c.refuse(RO_E_INVAL, "%s: NULL cache", fn);
  if (!k->d_k || !k->d_v || !k->d_page_base || !k->d_pages) return c.refuse(RO_E_INVAL, "%s: NULL in the cache", fn);
  if (k->dtype != RO_BF16 && k->dtype != RO_F16) return c.refuse(RO_E_INVAL, "%s: the cache is bf16 or f16", fn);
  if (!k->n_pages || !k->page_size || !k->n_heads || !k->n_seqs)
    return c.refuse(RO_E_INVAL, "%s: a cache without pages, slots, heads or sequences", fn);
  if (k->head_dim == 0 || k->head_dim % 8 || k->head_dim > 128)
    return c.refuse(RO_E_INVAL, "%s: head_dim must be a multiple of 8, at most 128", fn);
  if (k->n_heads > MAX_HEADS || k->n_seqs >= 0x80000000u || k->page_size >= 0x80000000u)
    return c.refuse(RO_E_OVERFLOW, "%s: too many heads, sequences or slots", fn);
  if (!aligned(k->d_k, 16) || !aligned(k->d_v, 16) || k->page_stride % 8 || k->head_stride % 8 || k->slot_stride % 8)
    return c.refuse(RO_E_INVAL, "%s: pools want 16-byte pointers and strides of 8 elements", fn);
  return RO_OK;
}

ro_status check_rows(StepCall& c, const char* fn, const ro_cache* k, const uint64_t* tok_base, uint64_t n_tokens,
                     const uint32_t* len, const void* q, uint64_t q_tok, uint64_t q_head, uint32_t n_q_heads,
                     float scale) {
  if (!tok_base || !len || (n_tokens && !q)) return c.refuse(RO_E_INVAL, "%s: NULL argument", fn);
  if (n_tokens >= 0x80000000ull) return c.refuse(RO_E_OVERFLOW, "%s: 2^31 tokens or more", fn);
  if (!n_q_heads || n_q_heads > MAX_HEADS || n_q_heads % k->n_heads)
    return c.refuse(RO_E_INVAL, "%s: query heads must be a multiple of the cache's", fn);
  if (!aligned(q, 16) || q_tok % 8 || q_head % 8)
    return c.refuse(RO_E_INVAL, "%s: q wants a 16-byte pointer and strides of 8 elements", fn);
  if (!std::isfinite(scale * LOG2_E)) return c.refuse(RO_E_INVAL, "%s: scale must be finite, times log2 e too", fn);
  return RO_OK;
}

PagedArgs paged(const ro_cache* k) {
  PagedArgs p;
  p.k = k->d_k;
  p.v = k->d_v;
  p.page_stride = k->page_stride;
  p.head_stride = k->head_stride;
  p.slot_stride = k->slot_stride;
  p.page_base = k->d_page_base;
  p.pages = k->d_pages;
  p.n_pages = k->n_pages;
  p.page_size = k->page_size;
  p.n_heads = k->n_heads;
  p.head_dim = k->head_dim;
  p.n_seqs = k->n_seqs;
  p.page_shift = -1;
  if ((k->page_size & (k->page_size - 1)) == 0)
    for (p.page_shift = 0; (1u << p.page_shift) < k->page_size;) ++p.page_shift;
  return p;
}

RowsArgs rows_of(const uint64_t* tok_base, const uint32_t* len, uint64_t n_tokens, uint32_t max_new, uint32_t group,
                 const void* q, uint64_t q_tok, uint64_t q_head, uint32_t window, uint32_t sinks, float scale) {
  RowsArgs r;
  r.tok_base = tok_base;
  r.len = len;
  r.n_tokens = n_tokens;
  r.max_new = max_new ? max_new : (uint32_t)n_tokens;
  r.group = group;
  r.q = q;
  r.q_tok = q_tok;
  r.q_head = q_head;
  // slots are below 2^31: a wider window sees everything
  r.window = window < 0x80000000u ? window : 0u;
  r.sinks = std::min(sinks, 0x7FFFFFFFu);
  r.scale_log2 = scale * LOG2_E;
  return r;
}

ro_status check_moves(StepCall& c, const char* fn, const ro_moves* m, uint64_t least, MoveArgs* out) {
  if (!m || !m->d_n || (m->cap && (!m->d_from || !m->d_to || !m->d_slots))) return c.refuse(RO_E_INVAL, "%s: NULL in the moves", fn);
  if (m->cap < least) return c.refuse(RO_E_INVAL, "%s: room for %llu moves, %llu can be needed", fn, (unsigned long long)m->cap,
                                      (unsigned long long)least);
  if (m->cap >= 0x80000000ull) return c.refuse(RO_E_OVERFLOW, "%s: 2^31 moves or more", fn);
  *out = {m->d_from, m->d_to, m->d_slots, m->d_n, m->cap};
  return RO_OK;
}
// ranges of bytes that share one
bool touch(const void* p, uint64_t p_bytes, const void* q, uint64_t q_bytes) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
  return p_bytes && q_bytes && a < b + q_bytes && b < a + p_bytes;
}
// Whether an output shares bytes with an input or with another output.  (An input
// that changes in place is its output.)
struct Bytes {
  const void* p;
  uint64_t n;
};
bool clash(std::initializer_list<Bytes> outs, std::initializer_list<Bytes> ins) {
  for (const Bytes* o = outs.begin(); o != outs.end(); ++o) {
    for (const Bytes& i : ins)
      if (touch(o->p, o->n, i.p, i.n)) return true;
    for (const Bytes* q = outs.begin(); q != o; ++q)
      if (touch(o->p, o->n, q->p, q->n)) return true;
  }
  return false;
}
// Flags, ranks and counts of a plan over the pool's pages.
ro_status plan_scratch(StepCall& c, uint64_t items, PagesArgs* a, uint32_t* ctas) {
  *ctas = pages_ctas(items, c.sms());
  const uint64_t counts = (uint64_t)*ctas * PG_WARPS, pages = a->c.n_pages;
  void* p = nullptr;
  RO_TRY(c.scratch(SS_PAGES, counts * sizeof(PageCounts) + (pages + ceil_div(pages, 32)) * sizeof(uint32_t), &p));
  a->counts = (PageCounts*)p;
  a->list = (uint32_t*)(a->counts + counts);
  return RO_OK;
}

// ro_cache_attend and, with a bias, ro_cache_attend_biased
ro_status attend(const char* fn, StepCall& c, const ro_cache* cache, const uint64_t* d_tok_base, uint64_t n_tokens,
                 uint32_t max_new, const uint32_t* d_len, uint32_t max_len, const void* d_q, uint64_t q_tok,
                 uint64_t q_head, uint32_t n_q_heads, float scale, uint32_t window, uint32_t sinks,
                 const ro_bias* bias, void* d_out, uint64_t out_tok, uint64_t out_head, float* d_lse) {
  RO_TRY(check_cache(c, fn, cache));
  RO_TRY(check_rows(c, fn, cache, d_tok_base, n_tokens, d_len, d_q, q_tok, q_head, n_q_heads, scale));
  if (n_tokens && !d_out) return c.refuse(RO_E_INVAL, "%s: NULL output", fn);
  if (!aligned(d_out, 16) || out_tok % 8 || out_head % 8)
    return c.refuse(RO_E_INVAL, "%s: the output wants a 16-byte pointer and strides of 8 elements", fn);
  if (bias) {
    // (the cap in log2 and scale / cap are normal numbers then, or 0)
    const float ratio = std::fabs(scale / bias->cap);
    if (!(bias->cap == 0.f ||
          (bias->cap >= 1e-6f && bias->cap <= 1e30f && (scale == 0.f || (ratio >= 1e-37f && ratio <= 1e30f)))))
      return c.refuse(RO_E_INVAL, "%s: cap must be 0 or from 1e-6 to 1e30, and scale / cap 0 or from 1e-37 to 1e30", fn);
    if (!aligned(bias->d_slope, 4) || !aligned(bias->d_first, 4) || !aligned(bias->d_until, 4))
      return c.refuse(RO_E_INVAL, "%s: a pointer off its type's alignment", fn);
  }
  if (n_tokens == 0) return RO_OK;
  if (d_out == d_q) return c.refuse(RO_E_INVAL, "%s: the output cannot be q", fn);
  RO_TRY(c.begin());
  AttendArgs a = {};
  a.c = paged(cache);
  const uint32_t group = n_q_heads / cache->n_heads;
  a.r = rows_of(d_tok_base, d_len, n_tokens, max_new, group, d_q, q_tok, q_head, window, sinks, scale);
  a.out = d_out;
  a.out_tok = out_tok;
  a.out_head = out_head;
  a.lse = d_lse;
  a.n_q_heads = n_q_heads;
  a.err = c.err();
  if (bias) {
    a.biased = 1;
    a.b.cap_log2 = bias->cap * LOG2_E;
    a.b.to_z = bias->cap != 0.f ? scale / bias->cap : 0.f;
    a.b.slope = bias->d_slope;
    a.b.first = bias->d_first;
    a.b.until = bias->d_until;
  }
  uint64_t keys = max_len ? max_len : 0x7FFFFFFFu;
  keys = std::min<uint64_t>(keys, (uint64_t)cache->n_pages * cache->page_size);
  if (a.r.window) keys = std::min<uint64_t>(keys, (uint64_t)a.r.window + a.r.sinks + a.r.max_new);
  keys = std::max<uint64_t>(keys, 1);
  const uint64_t max_rows = (uint64_t)a.r.max_new * group;
  void* p = nullptr;
  // At most 16 rows a sequence: bound by the cache's bytes.
  if (max_rows <= 16) {
    const uint64_t work = (uint64_t)cache->n_seqs * cache->n_heads, stage = attend_few_keys(cache->head_dim);
    if (work > MAX_GRID) return c.refuse(RO_E_OVERFLOW, "%s: too many sequences and heads", fn);
    a.tiles = cache->n_seqs;
    // Runs that fill two CTAs an SM in whole rounds, of at most 96 stages of
    // 16 KB (longer ones leave SMs idle at the end where lengths differ) and
    // at least 3, one for each warp (shorter ones cost more than they
    // save).  One sequence of 777 slots, 4 heads of 64: 7.2 us at 3 stages, 9.1
    // at 8, 7.8 at 2; of 100,000 slots, 8 heads of 128: 70 us in one round, 84 in
    // two; 64 ragged sequences of up to 32,000 slots: 432 us at 96 stages, 476 at
    // 32, 565 at 16.
    const uint64_t stages = ceil_div(keys, stage), places = (uint64_t)c.sms() * 2;
    const uint64_t each = ceil_div(stages * work, places);
    a.chunk = (uint32_t)std::max<uint64_t>(3, ceil_div(each, ceil_div(each, 96)));
    a.max_chunks = (uint32_t)std::min<uint64_t>(ceil_div(stages, a.chunk),
                                                std::min<uint64_t>(1024, std::max<uint64_t>(1, MAX_FEW_RUNS / work)));
    // Up to eight runs that the GPU holds at once are a cluster and join in
    // shared memory; more go through L2 and a ticket.
    const bool cluster = a.max_chunks > 1 && a.max_chunks <= 8 && work * a.max_chunks <= places;
    if (a.max_chunks > 1 && !cluster) {
      RO_TRY(c.scratch(SS_PARTIAL, attend_few_partial(a), &p));
      a.partial = (float*)p;
      RO_TRY(c.scratch(SS_COUNTER, (size_t)work * 4, &p));
      a.counter = (uint32_t*)p;
    }
    // Many short sequences: a warp alone for each (sequence, head), where its
    // stages one after another, about 1 us for 8 KB, take less than the rounds
    // of larger CTAs, about 6 us each.  2,048 of 40 slots of 128: 13 us against
    // 41, of 300: 55 against 79; 5,600 of up to 150: 42 against 110.  On either
    // side of the rule: 1,024 of up to 300 slots 23.4 against 24.4, of up to 600
    // 44 against 32.
    const bool alone = a.max_chunks == 1 && work > places && ceil_div(keys, attend_short_keys(cache->head_dim)) * places <= 5 * work;
    launch_attend_few(c.launch(), a, cache->dtype, cluster, alone);
    return c.launched(fn);
  }
  // More: the tensor-core kernel, if the pages and the group fit its tiles.
  if (attend_tiles_fits(a)) {
    const uint32_t toks = attend_tile_tokens(group);
    const uint64_t tiles = a.r.max_new <= toks ? (uint64_t)cache->n_seqs : n_tokens / toks + cache->n_seqs + 1;
    const uint64_t work = tiles * cache->n_heads, slots = ceil_div(keys, 128);
    if (work > MAX_GRID / 256) return c.refuse(RO_E_OVERFLOW, "%s: too many row tiles", fn);
    a.tiles = (uint32_t)tiles;
    // One CTA an SM takes pairs of row tiles in turn.  Where that is few rounds,
    // split the slots into the number of runs that takes the least time: rounds
    // of runs, each its tiles of slots plus about 6 tiles' time of its own.
    // (512 new tokens over 64,000 slots: 327 us in 2 runs, 311 in 7, 611 unsplit;
    // 64 over 32,000: 38 us in 16 runs, 53 in 8, 319 unsplit.)
    const uint64_t sms = (uint64_t)c.sms();
    const uint64_t pairs = std::min<uint64_t>(work, (uint64_t)cache->n_seqs * ceil_div(a.r.max_new, toks) * cache->n_heads);
    uint64_t runs = 1, least = ~0ull;
    for (uint64_t k = 1; k == 1 || (k <= 32 && pairs < 4 * sms && pairs * k <= MAX_RUNS); ++k) {
      const uint64_t each = ceil_div(slots, k), time = ceil_div(pairs * ceil_div(slots, each), sms) * (each + 6);
      if (time < least) {
        least = time;
        runs = k;
      }
    }
    a.pairs = (uint32_t)pairs;   // whose numbers have no gaps: partial results for these alone
    a.chunk = runs == 1 ? 0x40000000u : (uint32_t)ceil_div(slots, runs);
    a.max_chunks = runs == 1 ? 1u : (uint32_t)ceil_div(slots, a.chunk);
    RO_TRY(c.scratch(SS_COUNTER, 2 * sizeof(uint32_t), &p));
    a.counter = (uint32_t*)p;
    if (a.max_chunks > 1) {
      RO_TRY(c.scratch(SS_JOIN, attend_tiles_join(a), &a.join));
      RO_TRY(c.scratch(SS_PARTIAL, attend_tiles_partial(a), &p));
      a.partial = (float*)p;
    }
    if (launch_attend_tiles(c.launch(), a, cache->dtype, c.sms())) return c.launched(fn);
  }
  const uint32_t rows = 64;
  const uint32_t toks = std::max<uint32_t>(1, rows / group), row_tiles = (uint32_t)ceil_div(group, rows);
  const uint64_t tiles =
      (a.r.max_new <= toks ? (uint64_t)cache->n_seqs : n_tokens / toks + cache->n_seqs + 1) * row_tiles;
  const uint64_t work = tiles * cache->n_heads;
  if (work > MAX_GRID) return c.refuse(RO_E_OVERFLOW, "%s: too many row tiles", fn);
  a.tiles = (uint32_t)tiles;
  // Keys of one CTA: about four CTAs' worth of work per place of the GPU, in
  // steps of 64 keys and at least 128 (a shorter run costs more in its join
  // than it saves).
  const uint64_t split = std::max<uint64_t>(1, (uint64_t)c.sms() * 2 * 4 / work);
  a.chunk = (uint32_t)std::min<uint64_t>(0x40000000u, std::max<uint64_t>(128, ceil_div(ceil_div(keys, split), 64) * 64));
  a.max_chunks = (uint32_t)std::min<uint64_t>(ceil_div(keys, a.chunk), 1024);
  if (a.max_chunks > 1) {
    RO_TRY(c.scratch(SS_PARTIAL, (size_t)work * a.max_chunks * rows * ((cache->head_dim <= 64 ? 64 : 128) + 2) * 4, &p));
    a.partial = (float*)p;
    RO_TRY(c.scratch(SS_COUNTER, (size_t)work * 4, &p));
    a.counter = (uint32_t*)p;
  }
  launch_attend_rows(c.launch(), a, cache->dtype);
  return c.launched(fn);
}

}  // namespace

extern "C" {

ro_status ro_rotary(ro_ctx* ctx, int32_t dtype, const void* d_x, uint64_t x_tok, uint64_t x_head, void* d_out,
                    uint64_t out_tok, uint64_t out_head, uint64_t n_tokens, uint32_t n_heads, uint32_t head_dim,
                    const int32_t* d_pos, const ro_rope* rope, int32_t inverse) {
  const char* fn = "ro_rotary";
  StepCall c(ctx);
  RO_TRY(c.status);
  if (dtype != RO_BF16 && dtype != RO_F16 && dtype != RO_F32) return c.refuse(RO_E_INVAL, "%s: unknown type", fn);
  if (!rope || (n_tokens && n_heads && (!d_x || !d_out || !d_pos))) return c.refuse(RO_E_INVAL, "%s: NULL argument", fn);
  if (head_dim == 0 || head_dim % 2 || head_dim > 2 * ROPE_MAX_PAIRS)
    return c.refuse(RO_E_INVAL, "%s: head_dim must be even, at most 256", fn);
  if (n_tokens >= 0x80000000ull || n_heads > MAX_HEADS) return c.refuse(RO_E_OVERFLOW, "%s: too many tokens or heads", fn);
  RO_TRY(check_rope(c, fn, rope, head_dim));
  const size_t elem = dtype == RO_F32 ? 4 : 2;
  if (!aligned(d_x, elem) || !aligned(d_out, elem)) return c.refuse(RO_E_INVAL, "%s: a pointer off its type's alignment", fn);
  if (in_place_elsewhere(d_x, x_tok, x_head, d_out, out_tok, out_head, n_tokens, n_heads))
    return c.refuse(RO_E_INVAL, "%s: in place with other strides", fn);
  if (n_tokens == 0 || n_heads == 0) return RO_OK;
  RO_TRY(c.begin());
  TurnArgs a = {};
  a.n_tokens = n_tokens;
  a.head_dim = head_dim;
  a.n_parts = 1;
  a.inverse = inverse != 0;
  a.pos = d_pos;
  a.part[0] = {d_x, d_out, x_tok, x_head, out_tok, out_head, n_heads, 1u, 0u};
  a.err = c.err();
  fill_rope(rope, &a.rope);
  launch_turn(c.launch(), a, dtype, turn_vec(a, elem), c.sms());
  return c.launched(fn);
}

ro_status ro_cache_append(ro_ctx* ctx, const ro_cache* cache, const uint64_t* d_tok_base, const uint32_t* d_tok_seq,
                          uint64_t n_tokens, const uint32_t* d_len, const int32_t* d_pos, const ro_rope* rope,
                          const void* d_q, uint64_t q_tok, uint64_t q_head, uint32_t n_q_heads, void* d_q_out,
                          uint64_t qo_tok, uint64_t qo_head, const void* d_k, uint64_t k_tok, uint64_t k_head,
                          const void* d_v, uint64_t v_tok, uint64_t v_head) {
  const char* fn = "ro_cache_append";
  StepCall c(ctx);
  RO_TRY(c.status);
  RO_TRY(check_cache(c, fn, cache));
  if (!d_tok_base || !d_len || (n_tokens && (!d_tok_seq || !d_k || !d_v || (rope && !d_pos) ||
                                             (n_q_heads && (!d_q || !d_q_out)))))
    return c.refuse(RO_E_INVAL, "%s: NULL argument", fn);
  if (n_tokens >= 0x80000000ull || n_q_heads > MAX_HEADS)
    return c.refuse(RO_E_OVERFLOW, "%s: too many tokens or heads", fn);
  if (rope) RO_TRY(check_rope(c, fn, rope, cache->head_dim));
  for (const void* p : {d_q, (const void*)d_q_out, d_k, d_v})
    if (!aligned(p, 16)) return c.refuse(RO_E_INVAL, "%s: pointers must be 16-byte aligned", fn);
  for (uint64_t s : {q_tok, q_head, qo_tok, qo_head, k_tok, k_head, v_tok, v_head})
    if (s % 8) return c.refuse(RO_E_INVAL, "%s: strides must be multiples of 8 elements", fn);
  if (n_q_heads && in_place_elsewhere(d_q, q_tok, q_head, d_q_out, qo_tok, qo_head, n_tokens, n_q_heads))
    return c.refuse(RO_E_INVAL, "%s: q in place with other strides", fn);
  if (n_tokens == 0) return RO_OK;
  RO_TRY(c.begin());
  TurnArgs a = {};
  a.n_tokens = n_tokens;
  a.head_dim = cache->head_dim;
  a.pos = d_pos;
  const uint32_t turn = rope != nullptr;
  if (n_q_heads) a.part[a.n_parts++] = {d_q, d_q_out, q_tok, q_head, qo_tok, qo_head, n_q_heads, turn, 0u};
  a.part[a.n_parts++] = {d_k, cache->d_k, k_tok, k_head, 0, cache->head_stride, cache->n_heads, turn, 1u};
  a.part[a.n_parts++] = {d_v, cache->d_v, v_tok, v_head, 0, cache->head_stride, cache->n_heads, 0u, 1u};
  a.tok_base = d_tok_base;
  a.tok_seq = d_tok_seq;
  a.len = d_len;
  a.page_base = cache->d_page_base;
  a.pages = cache->d_pages;
  a.n_seqs = cache->n_seqs;
  a.n_pages = cache->n_pages;
  a.page_size = cache->page_size;
  a.page_stride = cache->page_stride;
  a.slot_stride = cache->slot_stride;
  a.err = c.err();
  if (rope) fill_rope(rope, &a.rope);
  launch_turn(c.launch(), a, cache->dtype, turn_vec(a, 2), c.sms());
  return c.launched(fn);
}

ro_status ro_cache_attend(ro_ctx* ctx, const ro_cache* cache, const uint64_t* d_tok_base, uint64_t n_tokens,
                          uint32_t max_new, const uint32_t* d_len, uint32_t max_len, const void* d_q, uint64_t q_tok,
                          uint64_t q_head, uint32_t n_q_heads, float scale, uint32_t window, uint32_t sinks,
                          void* d_out, uint64_t out_tok, uint64_t out_head, float* d_lse) {
  StepCall c(ctx);
  RO_TRY(c.status);
  return attend("ro_cache_attend", c, cache, d_tok_base, n_tokens, max_new, d_len, max_len, d_q, q_tok, q_head,
                n_q_heads, scale, window, sinks, nullptr, d_out, out_tok, out_head, d_lse);
}

ro_status ro_cache_attend_biased(ro_ctx* ctx, const ro_cache* cache, const uint64_t* d_tok_base, uint64_t n_tokens,
                                 uint32_t max_new, const uint32_t* d_len, uint32_t max_len, const void* d_q,
                                 uint64_t q_tok, uint64_t q_head, uint32_t n_q_heads, float scale, uint32_t window,
                                 uint32_t sinks, const ro_bias* bias, void* d_out, uint64_t out_tok, uint64_t out_head,
                                 float* d_lse) {
  StepCall c(ctx);
  RO_TRY(c.status);
  if (!bias) return c.refuse(RO_E_INVAL, "ro_cache_attend_biased: NULL bias");
  return attend("ro_cache_attend_biased", c, cache, d_tok_base, n_tokens, max_new, d_len, max_len, d_q, q_tok, q_head,
                n_q_heads, scale, window, sinks, bias, d_out, out_tok, out_head, d_lse);
}

ro_status ro_cache_weigh(ro_ctx* ctx, const ro_cache* cache, const uint64_t* d_tok_base, uint64_t n_tokens,
                         uint32_t max_new, const uint32_t* d_len, const void* d_q, uint64_t q_tok, uint64_t q_head,
                         uint32_t n_q_heads, float scale, uint32_t window, uint32_t sinks, const float* d_lse,
                         float decay, const float* d_past, float* d_score, uint64_t score_cap) {
  const char* fn = "ro_cache_weigh";
  StepCall c(ctx);
  RO_TRY(c.status);
  RO_TRY(check_cache(c, fn, cache));
  RO_TRY(check_rows(c, fn, cache, d_tok_base, n_tokens, d_len, d_q, q_tok, q_head, n_q_heads, scale));
  if ((n_tokens && !d_lse) || (score_cap && !d_score)) return c.refuse(RO_E_INVAL, "%s: NULL argument", fn);
  if (!std::isfinite(decay)) return c.refuse(RO_E_INVAL, "%s: decay must be finite", fn);
  if (score_cap >= 0x80000000ull) return c.refuse(RO_E_OVERFLOW, "%s: 2^31 scores a head or more", fn);
  const uint64_t units = (uint64_t)cache->n_seqs * cache->n_heads;
  if (units > MAX_GRID || ceil_div(score_cap, WG_KEYS) > MAX_GRID / units)
    return c.refuse(RO_E_OVERFLOW, "%s: too many scores", fn);
  if (score_cap == 0) return RO_OK;
  if (d_past && d_past != d_score && overlap(d_past, d_score, units * score_cap * sizeof(float)))
    return c.refuse(RO_E_INVAL, "%s: past scores are d_score or another array", fn);
  RO_TRY(c.begin());
  WeighArgs a = {};
  a.c = paged(cache);
  a.r = rows_of(d_tok_base, d_len, n_tokens, max_new, n_q_heads / cache->n_heads, d_q, q_tok, q_head, window, sinks,
                scale);
  a.lse = d_lse;
  a.n_q_heads = n_q_heads;
  a.decay = decay;
  a.past = d_past;
  a.score = d_score;
  a.score_cap = score_cap;
  a.err = c.err();
  if ((uint64_t)a.r.max_new * a.r.group <= 16) {
    // bound by the keys' bytes: runs of stages as in the attention of few rows;
    // nothing is joined, so short runs cost less
    const uint64_t stages = ceil_div(score_cap, weigh_few_keys(cache->head_dim));
    const uint64_t each = ceil_div(stages * units, (uint64_t)c.sms() * 2);
    a.chunk = (uint32_t)std::max<uint64_t>(3, ceil_div(each, ceil_div(each, 48)));
    a.chunk = (uint32_t)std::min<uint64_t>(a.chunk, stages);
    a.tiles = (uint32_t)std::min<uint64_t>(ceil_div(stages, a.chunk), 65535);
    launch_weigh_few(c.launch(), a, cache->dtype);
    return c.launched(fn);
  }
  // Behind a window most tiles of slots only have their past scores decayed: a
  // second kernel's, which leaves the tiles of the sinks and of the window.
  const uint64_t all = ceil_div(score_cap, WT_KEYS);
  const uint64_t seen = ceil_div(a.r.sinks, WT_KEYS) + ceil_div((uint64_t)a.r.window + a.r.max_new, WT_KEYS) + 1;
  a.unseen = a.r.window != 0 && seen < all;
  a.tiles = (uint32_t)(a.unseen ? seen : all);
  if (n_tokens && weigh_tiles_fits(a)) {
    void* p = nullptr;
    RO_TRY(c.scratch(SS_COUNTER, 2 * sizeof(uint32_t), &p));
    a.counter = (uint32_t*)p;
    if (launch_weigh_tiles(c.launch(), a, cache->dtype, c.sms())) return c.launched(fn);
  }
  a.unseen = 0;
  a.tiles = (uint32_t)ceil_div(score_cap, WG_KEYS);
  launch_weigh(c.launch(), a, cache->dtype);
  return c.launched(fn);
}

ro_status ro_cache_evict(ro_ctx* ctx, const ro_cache* cache, const uint32_t* d_len, const float* d_score,
                         uint64_t score_cap, uint32_t budget, uint32_t sinks, uint32_t recent,
                         const uint64_t* d_dst_base, const uint32_t* d_dst_pages, uint32_t* d_keep,
                         uint32_t* d_len_out, float* d_score_out) {
  const char* fn = "ro_cache_evict";
  StepCall c(ctx);
  RO_TRY(c.status);
  RO_TRY(check_cache(c, fn, cache));
  if (!d_len || !d_dst_base || !d_dst_pages || !d_keep || !d_len_out || (score_cap && !d_score))
    return c.refuse(RO_E_INVAL, "%s: NULL argument", fn);
  if (budget == 0 || (uint64_t)sinks + recent > budget)
    return c.refuse(RO_E_INVAL, "%s: sinks and recent tokens must fit the budget", fn);
  if (d_len_out != d_len && overlap(d_len, d_len_out, (uint64_t)cache->n_seqs * sizeof(uint32_t)))
    return c.refuse(RO_E_INVAL, "%s: lengths are cut in place or into another array", fn);
  if (score_cap >= 0x80000000ull || budget >= 0x80000000u)
    return c.refuse(RO_E_OVERFLOW, "%s: 2^31 scores or a budget of 2^31 or more", fn);
  if ((uint64_t)cache->n_seqs * cache->n_heads > MAX_GRID / 4096)
    return c.refuse(RO_E_OVERFLOW, "%s: too many sequences and heads", fn);
  if (d_score_out && overlap(d_score, d_score_out, (uint64_t)cache->n_seqs * cache->n_heads * score_cap * sizeof(float)))
    return c.refuse(RO_E_INVAL, "%s: scores cannot be cut in place", fn);
  RO_TRY(c.begin());
  EvictArgs a = {};
  a.c = paged(cache);
  a.len = d_len;
  a.score = d_score;
  a.score_cap = score_cap;
  a.budget = budget;
  a.sinks = sinks;
  a.recent = recent;
  a.dst_base = d_dst_base;
  a.dst_pages = d_dst_pages;
  a.keep = d_keep;
  a.len_out = d_len_out;
  a.score_out = d_score_out;
  a.err = c.err();
  launch_evict(c.launch(), a, c.sms());
  return c.launched(fn);
}

ro_status ro_cache_fork(ro_ctx* ctx, const ro_cache* cache, const uint32_t* d_len, const uint64_t* d_child_base,
                        const uint32_t* d_child_parent, uint64_t n_children, const uint64_t* d_dst_base,
                        const uint32_t* d_dst_seq, uint64_t n_dst, uint32_t* d_dst_pages, uint32_t* d_len_out,
                        const uint32_t* d_refs, uint32_t* d_refs_out, const ro_moves* moves) {
  const char* fn = "ro_cache_fork";
  StepCall c(ctx);
  RO_TRY(c.status);
  RO_TRY(check_cache(c, fn, cache));
  if (!d_len || !d_child_base || !d_refs || !d_refs_out || (n_children && (!d_child_parent || !d_dst_base || !d_len_out)) ||
      (n_dst && (!d_dst_seq || !d_dst_pages)))
    return c.refuse(RO_E_INVAL, "%s: NULL argument", fn);
  if (n_children >= 0x80000000ull || n_dst >= 0x80000000ull || cache->n_pages >= 0xFFFFFFFEu)
    return c.refuse(RO_E_OVERFLOW, "%s: too many continuations or pages", fn);
  if (n_dst && !n_children) return c.refuse(RO_E_INVAL, "%s: pages without continuations", fn);
  PagesArgs a = {};
  RO_TRY(check_moves(c, fn, moves, n_children, &a.m));
  const uint64_t pool = (uint64_t)cache->n_pages * sizeof(uint32_t);
  if (d_refs_out != d_refs && touch(d_refs, pool, d_refs_out, pool))
    return c.refuse(RO_E_INVAL, "%s: counts change in place or in another array", fn);
  if (touch(d_len, (uint64_t)cache->n_seqs * 4, d_len_out, n_children * 4) || touch(cache->d_pages, 4, d_dst_pages, n_dst * 4))
    return c.refuse(RO_E_INVAL, "%s: the continuations' lengths and pages go to arrays of their own", fn);
  const uint64_t room = moves->cap * 4, starts = ((uint64_t)cache->n_seqs + 1) * 8;
  // (of the page list only the GPU knows the length: the kernel looks at the rest)
  if (clash({{d_dst_pages, n_dst * 4}, {d_len_out, n_children * 4}, {d_refs_out, pool},
             {moves->d_from, room}, {moves->d_to, room}, {moves->d_slots, room}, {moves->d_n, 4}},
            {{d_len, (uint64_t)cache->n_seqs * 4}, {d_child_base, starts}, {d_child_parent, n_children * 4},
             {d_dst_base, n_children ? (n_children + 1) * 8 : 0}, {d_dst_seq, n_dst * 4},
             {d_refs, d_refs == d_refs_out ? 0 : pool}, {cache->d_page_base, starts}, {cache->d_pages, 4}}))
    return c.refuse(RO_E_INVAL, "%s: outputs share memory with inputs or one another", fn);
  RO_TRY(c.begin());
  a.c = paged(cache);
  a.refs = d_refs;
  a.refs_out = d_refs_out;
  a.len = d_len;
  a.child_base = d_child_base;
  a.child_parent = d_child_parent;
  a.dst_base = d_dst_base;
  a.dst_seq = d_dst_seq;
  a.dst_pages = d_dst_pages;
  a.len_out = d_len_out;
  a.n_children = n_children;
  a.n_dst = n_dst;
  a.err = c.err();
  uint32_t ctas = 0;
  RO_TRY(plan_scratch(c, std::max<uint64_t>(n_dst, cache->n_pages), &a, &ctas));
  launch_fork(c.launch(), a, ctas);
  MoveArgs copies = a.m;
  copies.cap = n_children;   // one a continuation at most
  launch_page_copy(c.launch(), a.c, copies, a.err, c.sms());
  return c.launched(fn);
}

ro_status ro_cache_compact(ro_ctx* ctx, const ro_cache* cache, uint32_t* d_pages_out, uint64_t n_list,
                           const uint32_t* d_refs, uint32_t* d_refs_out, uint32_t* d_n_used, const ro_moves* moves) {
  const char* fn = "ro_cache_compact";
  StepCall c(ctx);
  RO_TRY(c.status);
  RO_TRY(check_cache(c, fn, cache));
  if ((n_list && !d_pages_out) || !d_refs || !d_refs_out || !d_n_used) return c.refuse(RO_E_INVAL, "%s: NULL argument", fn);
  if (n_list >= 0x80000000ull || cache->n_pages >= 0xFFFFFFFEu)
    return c.refuse(RO_E_OVERFLOW, "%s: too many pages or entries", fn);
  PagesArgs a = {};
  RO_TRY(check_moves(c, fn, moves, cache->n_pages / 2, &a.m));
  const uint64_t pool = (uint64_t)cache->n_pages * sizeof(uint32_t);
  if (d_refs_out != d_refs && touch(d_refs, pool, d_refs_out, pool))
    return c.refuse(RO_E_INVAL, "%s: counts change in place or in another array", fn);
  // (of a list that does not change in place only the GPU knows the length: the kernel looks at the rest)
  const bool in_place = n_list && d_pages_out == cache->d_pages;
  const uint64_t room = moves->cap * 4;
  if (clash({{d_pages_out, n_list * 4}, {d_refs_out, pool},
             {d_n_used, 4}, {moves->d_from, room}, {moves->d_to, room}, {moves->d_slots, room}, {moves->d_n, 4}},
            {{d_refs, d_refs == d_refs_out ? 0 : pool}, {cache->d_page_base, ((uint64_t)cache->n_seqs + 1) * 8},
             {cache->d_pages, in_place ? 0ull : 4ull}}))
    return c.refuse(RO_E_INVAL, "%s: outputs share memory with inputs or one another", fn);
  RO_TRY(c.begin());
  a.c = paged(cache);
  a.refs = d_refs;
  a.refs_out = d_refs_out;
  a.pages_out = d_pages_out;
  a.n_list = n_list;
  a.n_used = d_n_used;
  a.err = c.err();
  uint32_t ctas = 0;
  RO_TRY(plan_scratch(c, std::max<uint64_t>(n_list, cache->n_pages), &a, &ctas));
  launch_compact(c.launch(), a, ctas);
  MoveArgs copies = a.m;
  copies.cap = cache->n_pages / 2;
  launch_page_copy(c.launch(), a.c, copies, a.err, c.sms());
  return c.launched(fn);
}

ro_status ro_cache_copy(ro_ctx* ctx, const ro_cache* cache, const ro_moves* moves) {
  const char* fn = "ro_cache_copy";
  StepCall c(ctx);
  RO_TRY(c.status);
  RO_TRY(check_cache(c, fn, cache));
  MoveArgs m = {};
  RO_TRY(check_moves(c, fn, moves, 0, &m));
  if (m.cap == 0) return RO_OK;
  RO_TRY(c.begin());
  launch_page_copy(c.launch(), paged(cache), m, c.err(), c.sms());
  return c.launched(fn);
}

ro_status ro_sample(ro_ctx* ctx, int32_t dtype, const void* d_logits, uint64_t row_stride, uint64_t n_rows,
                    uint32_t vocab, const ro_sampling* how, const float* d_u, uint32_t* d_token, float* d_logp,
                    uint32_t* d_kept) {
  const char* fn = "ro_sample";
  StepCall c(ctx);
  RO_TRY(c.status);
  if (dtype != RO_BF16 && dtype != RO_F16 && dtype != RO_F32) return c.refuse(RO_E_INVAL, "%s: unknown type", fn);
  if (n_rows && (!d_logits || !d_u || !d_token)) return c.refuse(RO_E_INVAL, "%s: NULL argument", fn);
  if (vocab == 0) return c.refuse(RO_E_INVAL, "%s: no tokens to draw from", fn);
  if (vocab > MAX_VOCAB || n_rows > MAX_GRID / 8)
    return c.refuse(RO_E_OVERFLOW, "%s: more than %u tokens or too many rows", fn, MAX_VOCAB);
  if (!aligned(d_logits, dtype == RO_F32 ? 4 : 2)) return c.refuse(RO_E_INVAL, "%s: a pointer off its type's alignment", fn);
  for (const void* p : {(const void*)d_u, (const void*)d_token, (const void*)d_logp, (const void*)d_kept,
                        how ? (const void*)how->d_temperature : nullptr, how ? (const void*)how->d_top_k : nullptr,
                        how ? (const void*)how->d_top_p : nullptr, how ? (const void*)how->d_min_p : nullptr})
    if (!aligned(p, 4)) return c.refuse(RO_E_INVAL, "%s: a pointer off its type's alignment", fn);
  if (n_rows == 0) return RO_OK;
  const uint64_t each = n_rows * 4, elem = dtype == RO_F32 ? 4 : 2;
  const ro_sampling neutral = {}, &set = how ? *how : neutral;
  if (clash({{d_token, each}, {d_logp, d_logp ? each : 0}, {d_kept, d_kept ? each : 0}},
            {{d_logits, ((n_rows - 1) * row_stride + vocab) * elem}, {d_u, each}, {set.d_temperature, set.d_temperature ? each : 0},
             {set.d_top_k, set.d_top_k ? each : 0}, {set.d_top_p, set.d_top_p ? each : 0}, {set.d_min_p, set.d_min_p ? each : 0}}))
    return c.refuse(RO_E_INVAL, "%s: outputs share memory with inputs or one another", fn);
  RO_TRY(c.begin());
  SampleArgs a = {};
  a.x = d_logits;
  a.stride = row_stride;
  a.rows = (uint32_t)n_rows;
  a.vocab = vocab;
  if (how) {
    a.temperature = how->d_temperature;
    a.top_k = how->d_top_k;
    a.top_p = how->d_top_p;
    a.min_p = how->d_min_p;
  }
  a.u = d_u;
  a.token = d_token;
  a.logp = d_logp;
  a.kept = d_kept;
  a.err = c.err();
  if (sample_queues(vocab, dtype, n_rows, c.sms())) {
    void* p = nullptr;
    RO_TRY(c.scratch(SS_ROWS, n_rows * sizeof(uint32_t), &p));
    a.queue = (uint32_t*)p;
    RO_TRY(c.scratch(SS_COUNTER, 3 * sizeof(uint32_t), &p));
    a.counter = (uint32_t*)p;
  }
  launch_sample(c.launch(), a, dtype, c.sms());
  return c.launched(fn);
}

}  // extern "C"
