// ro_step.h — host side of the model-step operators (include/rayorch_cache.h):
// what an entry point needs of a context, and the kernels' arguments.
#pragma once

#include "../../include/rayorch_cache.h"
#include "ro_internal.h"

namespace ro {

// One call on a context: entered (sticky errors returned, the context's
// device current until the call ends, the Calls' pending admissions waited
// for), its launches on the context's stream.
class StepCall {
 public:
  explicit StepCall(ro_ctx* c);
  ~StepCall();
  StepCall(const StepCall&) = delete;
  StepCall& operator=(const StepCall&) = delete;

  ro_status status;          // of entering; nothing may be launched unless RO_OK
  ro_status begin();         // after the argument checks, before the first launch
  ro_status refuse(ro_status st, const char* fmt, ...) __attribute__((format(printf, 3, 4)));
  ro_status launched(const char* what);
  // grow-only workspace of the context, zeroed when it grows
  ro_status scratch(int which, size_t bytes, void** p);
  const LaunchCfg& launch() const;
  uint32_t* err() const;
  int sms() const;

 private:
  ro_ctx* c_;
  int prev_ = -1;
};
// (SS_COUNTER is zero between calls, whichever kernel used it last)
enum StepScratch { SS_PARTIAL = 0, SS_COUNTER = 1, SS_JOIN = 2, SS_PAGES = 3, SS_ROWS = 4, SS_COUNT };

// ---- rotary, append -----------------------------------------------------------------
constexpr uint32_t ROPE_MAX_PAIRS = 128;
// Per pair its frequency in turns per position, in 1/2^64 turns: the product
// with an integer position wraps modulo a turn by itself.
struct RopeTable {
  uint32_t n_axes, pairs, interleaved, pad;
  uint8_t axis[ROPE_MAX_PAIRS];
  uint64_t freq[ROPE_MAX_PAIRS];
};
// A run of heads that a token's items cover in turn.
struct TurnPart {
  const void* src;
  void* dst;                 // flat: [token][head]; paged: the pool
  uint64_t src_tok, src_head, dst_tok, dst_head;
  uint32_t heads;
  uint32_t turn;             // 0: copied as it is
  uint32_t paged;
};
constexpr int TURN_THREADS = 256;
struct TurnArgs {
  uint64_t n_tokens;
  uint32_t head_dim, n_parts, tokens_per_cta, inverse;
  const int32_t* pos;
  TurnPart part[3];
  // paged parts
  const uint64_t* tok_base;
  const uint32_t* tok_seq;
  const uint32_t* len;
  const uint64_t* page_base;
  const uint32_t* pages;
  uint32_t n_seqs, n_pages, page_size;
  uint64_t page_stride, slot_stride;
  uint32_t* err;
  RopeTable rope;
};
// vec: elements of a thread's access (8, 4, 2, 1); dtype RO_BF16 / RO_F16 / RO_F32
void launch_turn(const LaunchCfg& L, const TurnArgs& a, int dtype, int vec, int sms);

// ---- attend, weigh --------------------------------------------------------------------
struct PagedArgs {
  const void* k;
  const void* v;
  uint64_t page_stride, head_stride, slot_stride;
  const uint64_t* page_base;
  const uint32_t* pages;
  uint32_t n_pages, page_size, n_heads, head_dim, n_seqs;
  int page_shift;            // log2 of page_size, -1: not a power of two
};
struct RowsArgs {             // the step's query rows
  const uint64_t* tok_base;
  const uint32_t* len;
  uint64_t n_tokens;
  uint32_t max_new;
  uint32_t group;            // query heads per cache head
  const void* q;
  uint64_t q_tok, q_head;
  uint32_t window, sinks;
  float scale_log2;          // scale * log2(e)
};
// ro_cache_attend_biased: x = cap tanh(scale q.k / cap) - slope |a - j|, in log2.
struct BiasArgs {
  float cap_log2;            // cap * log2(e); 0: none
  float to_z;                // scale / cap
  const float* slope;        // optional
  const uint32_t* first;     // optional
  const uint32_t* until;     // optional
};
struct AttendArgs {
  PagedArgs c;
  RowsArgs r;
  BiasArgs b;                // of use where biased
  uint32_t biased;
  uint32_t tiles;            // row tiles per cache head, at most
  uint32_t pairs;            // attend_tiles: (pair of row tiles, head) that there can be
  uint32_t chunk;            // of one CTA, more where max_chunks would not reach: keys
                             // (attend_rows), stages (attend_few), tiles (attend_tiles)
  uint32_t max_chunks;
  void* out;
  uint64_t out_tok, out_head;
  float* lse;                // optional
  uint32_t n_q_heads;
  float* partial;            // [tile][chunk][rows][head_dim + 2]
  uint32_t* counter;         // zero between calls
  void* join;                // attend_tiles: what its join kernel needs of each pair of row tiles
  uint32_t* err;
};
// at most 16 rows a sequence (alone: many short ones, a warp each, where the
// tensors can be mapped); slots of a stage, bytes of its runs' partial results
void launch_attend_few(const LaunchCfg& L, const AttendArgs& a, int dtype, bool cluster, bool alone);
uint32_t attend_few_keys(uint32_t head_dim);
uint32_t attend_short_keys(uint32_t head_dim);
size_t attend_few_partial(const AttendArgs& a);
cudaError_t prepare_attend_few_kernels();
// tiles of 64 rows, any page size
void launch_attend_rows(const LaunchCfg& L, const AttendArgs& a, int dtype);
cudaError_t prepare_attend_kernels();
// the tensor-core kernel: whether it takes these sizes, tokens of its CTA,
// bytes of what its join needs and of its runs' partial results; false: the
// tensors cannot be mapped
bool attend_tiles_fits(const AttendArgs& a);
uint32_t attend_tile_tokens(uint32_t group);
size_t attend_tiles_join(const AttendArgs& a);
size_t attend_tiles_partial(const AttendArgs& a);
bool launch_attend_tiles(const LaunchCfg& L, const AttendArgs& a, int dtype, int sms);
cudaError_t prepare_attend_tiles_kernels();

struct WeighArgs {
  PagedArgs c;
  RowsArgs r;
  const float* lse;
  uint32_t n_q_heads;
  float decay;
  const float* past;         // optional
  float* score;
  uint64_t score_cap;
  uint32_t tiles;            // along score_cap for each sequence and head, at most
  uint32_t chunk;            // weigh_few: stages of a CTA
  uint32_t unseen;           // weigh_tiles: the tiles before the windows are another kernel's
  uint32_t* counter;         // weigh_tiles: zero between calls
  uint32_t* err;
};
// at most 16 rows a sequence; slots of a stage
void launch_weigh_few(const LaunchCfg& L, const WeighArgs& a, int dtype);
uint32_t weigh_few_keys(uint32_t head_dim);
cudaError_t prepare_weigh_few_kernels();
// the tensor-core kernel: whether it takes these sizes, slots of its CTA;
// false: the tensors cannot be mapped
constexpr uint32_t WT_KEYS = 128;
bool weigh_tiles_fits(const WeighArgs& a);
bool launch_weigh_tiles(const LaunchCfg& L, const WeighArgs& a, int dtype, int sms);
cudaError_t prepare_weigh_tiles_kernels();
// any page size and group
constexpr int WG_THREADS = 128;
constexpr uint32_t WG_KEYS = 64, WG_ROWS = 64;
void launch_weigh(const LaunchCfg& L, const WeighArgs& a, int dtype);

// ---- evict ------------------------------------------------------------------------------
constexpr int ES_THREADS = 1024;
constexpr uint32_t ES_CACHED = 18432;   // keys a CTA of evict_select holds: 72 KB, two CTAs an SM
struct EvictArgs {
  PagedArgs c;
  const uint32_t* len;
  const float* score;
  uint64_t score_cap;
  uint32_t budget, sinks, recent;
  const uint64_t* dst_base;
  const uint32_t* dst_pages;
  uint32_t* keep;
  uint32_t* len_out;
  float* score_out;          // optional
  uint32_t cluster, cached;  // evict_select: CTAs and keys in shared memory
  uint32_t parts;            // evict_move: CTAs for each (sequence, head)
  uint32_t* err;
};
void launch_evict(const LaunchCfg& L, const EvictArgs& a, int sms);
cudaError_t prepare_evict_kernels();

// ---- fork, compact, copy --------------------------------------------------------------
constexpr int PG_THREADS = 1024;
constexpr uint32_t PG_WARPS = PG_THREADS / 32;
// A warp counts what its run of the lists and of the pool holds.
struct __align__(16) PageCounts {
  uint32_t fresh, moves, free, pad;
};
struct MoveArgs {
  uint32_t* from;
  uint32_t* to;
  uint32_t* slots;
  uint32_t* n;
  uint64_t cap;
};
struct PagesArgs {
  PagedArgs c;
  MoveArgs m;
  const uint32_t* refs;
  uint32_t* refs_out;
  PageCounts* counts;        // [gridDim][PG_WARPS]
  uint32_t* list;            // [n_pages]: fork: free pages by rank; compact: a late page's rank;
                             // then the pool's flags, 32 pages a word
  // fork
  const uint32_t* len;
  const uint64_t* child_base;
  const uint32_t* child_parent;
  const uint64_t* dst_base;
  const uint32_t* dst_seq;
  uint32_t* dst_pages;
  uint32_t* len_out;
  uint64_t n_children, n_dst;
  // compact
  uint32_t* pages_out;
  uint64_t n_list;
  uint32_t* n_used;
  uint32_t* err;
};
uint32_t pages_ctas(uint64_t items, int sms);
void launch_fork(const LaunchCfg& L, const PagesArgs& a, uint32_t ctas);
void launch_compact(const LaunchCfg& L, const PagesArgs& a, uint32_t ctas);
struct PageCopyArgs {
  PagedArgs c;
  MoveArgs m;
  uint32_t pieces;           // 4 KB pieces of a page's head
  uint32_t dense;            // a head's slots follow one another
  uint32_t* err;
};
void launch_page_copy(const LaunchCfg& L, const PagedArgs& c, const MoveArgs& m, uint32_t* err, int sms);

// ---- sample -----------------------------------------------------------------------------
constexpr uint32_t MAX_VOCAB = 393216;   // a thread's share of it bounds the error of its 32-bit sums
struct SampleArgs {
  const void* x;
  uint64_t stride;
  uint32_t rows, vocab;
  const float* temperature;  // these four optional
  const uint32_t* top_k;
  const float* top_p;
  const float* min_p;
  const float* u;
  uint32_t* token;
  float* logp;               // optional
  uint32_t* kept;            // optional
  uint32_t cluster, blocks;  // CTAs of a row, 16-byte blocks of a slice
  uint32_t staged;           // slices are held in shared memory
  uint32_t* queue;           // [rows], where wide ones are queued
  uint32_t* counter;         // of the queue's rows, a ticket, rows taken: zero between calls
  uint32_t* err;
};
// whether wide rows are queued for a second kernel (a.queue and a.counter are then given)
bool sample_queues(uint32_t vocab, int dtype, uint64_t rows, int sms);
void launch_sample(const LaunchCfg& L, const SampleArgs& a, int dtype, int sms);
cudaError_t prepare_sample_kernels();

}  // namespace ro
