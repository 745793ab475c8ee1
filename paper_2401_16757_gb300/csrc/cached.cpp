// Entry points of the cached-attention operators: argument checks, the choice
// of kernels and the workspace.  Nothing is allocated and nothing waits for
// the device.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstring>
#include <initializer_list>

#include "cached.h"
#include "internal.h"
#include "kernels.h"

namespace swapnet {

// Microseconds of the tensor-core kernel: a unit's start and end, a tile of
// keys, the join of shared units.
constexpr double kUnitUs = 5.0, kTileUs = 1.0, kJoinUs = 8.0;

// How many CTAs share the keys of a (sequence, key head), for the whole cache
// (how much of it is filled only the device knows): the count that takes the
// least time where every SM gets its share of all work, but for half a CTA at
// the end (lengths and causal limits differ).  In microseconds: a tile of a CTA
// by itself, a tile of an SM's time when all are busy, a CTA's start and end,
// and the join where there is one.
static int choose_splits(int64_t ctas, int tiles, double alone, double busy, double fixed, double join) {
  int best = 1;
  double least = 1e30;
  for (int s = 1; s <= tiles && s <= 128; ++s) {
    const double one = (tiles + s - 1) / s * alone + fixed;
    const double t = std::max(one, ctas * (tiles * busy + s * fixed) / kSms + 0.5 * one) + (s > 1 && join > 0.0 ? join + 0.02 * s : 0.0);
    if (t < least * 0.995) {
      least = t;
      best = s;
    }
  }
  return best;
}

CachedPlan cached_plan(const CachedArgs& a) {
  CachedPlan p;
  std::memset(&p, 0, sizeof(p));
  const int64_t rows = (int64_t)a.tokens * a.group, pairs = (int64_t)a.n_seq * a.kv_heads;
  // Warp products of 16 rows or tensor cores with 128 (us, 8 key heads of 128
  // unless said otherwise): 16 rows on 8000 keys x 32 sequences 118 / 122, 500 x
  // 1 10.6 / 15.4, 32000 x 1 36 / 34.5, 32 key heads 500 x 32 61 / 103; 20 rows,
  // which would take two products, 233 / 123, 13.2 / 15.4, 60 / 34.6.
  p.tc = rows > kFewAttnRows;
  p.spill = a.weights && !p.tc;
  if (p.tc) {
    const int row_tile = rows <= 64 ? 64 : 128, queries = std::min(row_tile / a.group, a.tokens);
    const int64_t units = pairs * ((a.tokens + queries - 1) / queries);
    const double tiles = (a.max_seq + 127) / 128 + (a.k_new ? 1 : 0);
    // A CTA per unit, or equal runs of all tiles and a join.  From two units
    // per SM on the block scheduler evens out what the runs would (512 units
    // of up to 33 tiles: 275 against 283 us); below that the join's 8 us decide:
    // 32 units of 5 tiles 14.9 against 18.4 us (13.2 now), 4 units of 1025 tiles
    // about 1000 against 41.
    const int ctas = run_ctas(a.kv_heads);
    const double alone = std::ceil((double)units / kSms) * (kUnitUs + tiles * kTileUs);
    const double shared = kUnitUs + std::max(2.0, units * tiles / ctas) * kTileUs + (double)units / ctas + kJoinUs;
    p.splits = units >= 2 * kSms || alone <= shared ? 1 : 0;
    if (units > 0x7fffffff) p.splits = 0;
    if (p.splits == 0) {
      p.part_bytes = align_up((uint64_t)2 * ctas * row_tile * a.dim * 4);
      p.ml_bytes = align_up((uint64_t)2 * ctas * row_tile * 8);
      p.unit_bytes = align_up((uint64_t)ctas * 16);
    }
    return p;
  }
  p.splits = choose_splits(pairs, (a.max_seq + 63) / 64, 0.5, 0.7, 1.5, 2.5);
  p.score_ld = (a.max_seq + 15) / 16 * 16;
  const uint64_t all = (uint64_t)pairs * rows;
  if (p.splits > 1) p.part_bytes = align_up(all * p.splits * a.dim * 4);
  if (p.splits > 1 || p.spill) p.ml_bytes = align_up(all * p.splits * 8);
  if (p.spill) p.score_bytes = align_up(all * p.score_ld * 4);
  return p;
}

int weights_splits(const CachedArgs& a) {
  const int tiles = (int)(((int64_t)a.tokens * a.group + 127) / 128);
  return choose_splits((int64_t)a.n_seq * a.kv_heads, (a.max_seq + 127) / 128, 0.3 + 0.35 * tiles, 0.3 + 0.35 * tiles, 1.0, 0.0);
}

int run_cached_attention(CachedArgs a, const CachedPlan& p, void* workspace, bool early, cudaStream_t s) {
  char* w = static_cast<char*>(workspace);
  a.splits = p.splits;
  a.part = reinterpret_cast<float*>(w);
  a.ml = reinterpret_cast<float*>(w + p.part_bytes);
  a.scores = p.spill ? reinterpret_cast<float*>(w + p.part_bytes + p.ml_bytes) : nullptr;
  a.score_ld = p.score_ld;
  a.units = reinterpret_cast<int4*>(w + p.part_bytes + p.ml_bytes + p.score_bytes);
  if (int rc = p.tc ? launch_attention_rows(a, early, s) : launch_attention_few(a, early, s)) return rc;
  if (!p.tc)
    if (int rc = launch_attention_join(a, s)) return rc;
  return a.weights && !p.spill ? launch_weights(a, weights_splits(a), true, s) : SWAPNET_OK;
}

void state_attention(const Model& m, char* state, int index, CachedArgs* out) {
  const StateLayout& s = m.st;
  CachedArgs a;
  std::memset(&a, 0, sizeof(a));
  a.dtype = m.dtype;
  a.n_seq = 1;
  a.tokens = s.tokens;
  a.heads = a.kv_heads = s.heads;
  a.group = 1;
  a.dim = s.width / s.heads;
  a.max_seq = s.max_seq;
  a.scale_log2 = 1.4426950408889634f / sqrtf((float)a.dim);
  a.q_stride = a.kv_stride = a.new_stride = a.out_stride = s.width;
  a.seq_stride = (int64_t)(2 * s.cache_bytes) / m.es;  // (layers taken as sequences)
  a.rows_step = 0;
  auto at = [&](uint64_t off) { return reinterpret_cast<char*>(reinterpret_cast<uintptr_t>(state) + off); };
  const uint64_t qkv = (uint64_t)s.tokens * s.width * m.es, stats = (uint64_t)s.heads * s.tokens;
  a.lens = reinterpret_cast<const int*>(at(0));
  a.k = at(s.caches + 2 * (uint64_t)index * s.cache_bytes);
  a.v = at(s.caches + (2 * (uint64_t)index + 1) * s.cache_bytes);
  a.lse = reinterpret_cast<float*>(at(s.lse));
  if (s.flags & SWAPNET_ATTENTION_TREE) {
    a.counts = reinterpret_cast<const int*>(at(s.count));
    a.parents = reinterpret_cast<const int*>(at(s.parents));
    a.k_new = at(s.drafts + 2 * (uint64_t)index * s.draft_bytes);
    a.v_new = at(s.drafts + (2 * (uint64_t)index + 1) * s.draft_bytes);
    a.q = at(s.queries + index * qkv);
    a.lse += index * stats;
  } else {
    a.len_add = s.tokens;  // the layer's own rows are in the cache, the position is not yet advanced
    if (s.flags & SWAPNET_ATTENTION_WEIGHTS)
      a.weights = reinterpret_cast<float*>(at(s.weights)) + (uint64_t)index * s.heads * s.max_seq;
    a.weights_in = a.weights;
  }
  *out = a;
}

int error_word(int** out) {
  static std::atomic<int*> cached[64];
  const int dev = device_index();
  if (dev >= 0)
    if (int* p = cached[dev].load(std::memory_order_acquire)) {
      *out = p;
      return SWAPNET_OK;
    }
  if (int rc = tc_error_word(out)) return rc;
  if (dev >= 0) cached[dev].store(*out, std::memory_order_release);
  return SWAPNET_OK;
}

int cached_launches(const CachedArgs& a, const CachedPlan& p) {
  return 1 + (p.splits != 1 || p.spill ? 1 : 0) + (a.weights && !p.spill ? 1 : 0);
}

namespace {

// What both attention entry points require of their arguments.
int fill_args(const swapnet_cached_attention* c, CachedArgs* a) {
  if (!c) SN_FAIL(SWAPNET_ERR_INVALID_ARG, "null arguments");
  std::memset(a, 0, sizeof(*a));
  if (c->dtype != SWAPNET_F16 && c->dtype != SWAPNET_BF16) SN_FAIL(SWAPNET_ERR_UNSUPPORTED, "cached attention: fp16 or bf16 only");
  if (c->n_seq < 1 || c->tokens < 1 || c->heads < 1 || c->kv_heads < 1 || c->max_seq < 1)
    SN_FAIL(SWAPNET_ERR_INVALID_ARG, "cached attention: empty shape");
  if (c->heads % c->kv_heads) SN_FAIL(SWAPNET_ERR_INVALID_ARG, "cached attention: heads must be a multiple of kv_heads");
  if (c->head_dim != 64 && c->head_dim != 128) SN_FAIL(SWAPNET_ERR_UNSUPPORTED, "cached attention: head width must be 64 or 128");
  const int64_t group = c->heads / c->kv_heads;
  if (c->n_seq > 65535 || c->kv_heads > 65535 || group > 128 || (int64_t)c->tokens * group > (1 << 20) || c->max_seq > (1 << 30) ||
      (int64_t)c->n_seq * c->tokens > (1 << 30))
    SN_FAIL(SWAPNET_ERR_UNSUPPORTED, "cached attention: shape beyond the kernels' limits");
  if (!c->q || !c->k || !c->lens) SN_FAIL(SWAPNET_ERR_INVALID_ARG, "cached attention: null pointer");
  const int64_t kv_width = (int64_t)c->kv_heads * c->head_dim, width = (int64_t)c->heads * c->head_dim;
  a->dtype = c->dtype;
  a->n_seq = c->n_seq;
  a->tokens = c->tokens;
  a->heads = c->heads;
  a->kv_heads = c->kv_heads;
  a->group = (int)group;
  a->dim = c->head_dim;
  a->max_seq = c->max_seq;
  if (!(c->scale >= 0.f) || std::isinf(c->scale)) SN_FAIL(SWAPNET_ERR_INVALID_ARG, "cached attention: bad scale");
  a->scale_log2 = 1.4426950408889634f * (c->scale > 0.f ? c->scale : 1.0f / sqrtf((float)c->head_dim));
  if (std::isinf(a->scale_log2)) SN_FAIL(SWAPNET_ERR_INVALID_ARG, "cached attention: bad scale");
  a->q = c->q;
  a->k = c->k;
  a->v = c->v;
  a->k_new = c->k_new;
  a->v_new = c->v_new;
  a->q_stride = c->q_stride ? c->q_stride : width;
  a->kv_stride = c->kv_stride ? c->kv_stride : kv_width;
  a->seq_stride = c->seq_stride ? c->seq_stride : a->kv_stride * c->max_seq;
  a->new_stride = c->new_stride ? c->new_stride : kv_width;
  a->out_stride = c->out_stride ? c->out_stride : width;
  if (a->q_stride < width || a->kv_stride < kv_width || a->new_stride < kv_width || a->out_stride < width ||
      (c->n_seq > 1 && a->seq_stride < 1))
    SN_FAIL(SWAPNET_ERR_INVALID_ARG, "cached attention: a stride is smaller than a row");
  if ((a->q_stride | a->kv_stride | a->seq_stride | a->new_stride | a->out_stride) % 8)
    SN_FAIL(SWAPNET_ERR_MISALIGNED, "cached attention: strides must be multiples of 8 elements");
  if (!aligned16(c->q) || !aligned16(c->k) || !aligned16(c->v) || !aligned16(c->k_new) || !aligned16(c->v_new) || !aligned16(c->out))
    SN_FAIL(SWAPNET_ERR_MISALIGNED, "cached attention: pointers must be 16-byte aligned");
  if (!aligned4(c->lens, c->counts, c->parents, c->rows, c->lse, c->weights_in, c->weights))
    SN_FAIL(SWAPNET_ERR_MISALIGNED, "cached attention: int32 and float arrays must be 4-byte aligned");
  a->lens = c->lens;
  a->counts = c->counts;
  a->parents = c->parents;
  a->rows = c->rows;
  a->lens_step = a->counts_step = 1;
  a->rows_step = c->tokens;
  a->out = c->out;
  a->lse = c->lse;
  a->weights_in = c->weights_in;
  a->weights = c->weights;
  return SWAPNET_OK;
}

// The attention call's own rules, on top of fill_args.
int check_attention(const swapnet_cached_attention* c, CachedArgs* a) {
  if (int rc = fill_args(c, a)) return rc;
  if (!c->v || !c->out) SN_FAIL(SWAPNET_ERR_INVALID_ARG, "attention: null pointer");
  if (c->rows) SN_FAIL(SWAPNET_ERR_INVALID_ARG, "attention: a row list is for swapnet_attention_weights");
  if (!c->k_new != !c->v_new) SN_FAIL(SWAPNET_ERR_INVALID_ARG, "attention: drafted keys and values come together");
  if (c->parents && !c->k_new) SN_FAIL(SWAPNET_ERR_INVALID_ARG, "attention: a tree's nodes are given as k_new and v_new");
  if (c->k_new && c->tokens > kTreeMax) SN_FAIL(SWAPNET_ERR_UNSUPPORTED, "attention: at most 128 drafted nodes a sequence");
  if (c->weights && c->k_new)
    SN_FAIL(SWAPNET_ERR_INVALID_ARG, "attention: weights with a draft come from swapnet_attention_weights, once it is accepted");
  if (c->weights_in && !c->weights) SN_FAIL(SWAPNET_ERR_INVALID_ARG, "attention: weights_in without weights");
  if (c->weights && cached_plan(*a).spill == 0 && !c->lse)
    SN_FAIL(SWAPNET_ERR_INVALID_ARG, "attention: weights of more than 16 rows (tokens x heads / kv_heads) need lse");
  return SWAPNET_OK;
}

}  // namespace
}  // namespace swapnet

extern "C" {

int swapnet_attention_tree_workspace(const swapnet_cached_attention* c, uint64_t* bytes) {
  return swapnet::guard_abi([&]() -> int {
    using namespace swapnet;
    if (!bytes) SN_FAIL(SWAPNET_ERR_INVALID_ARG, "null output");
    CachedArgs a;
    if (int rc = check_attention(c, &a)) return rc;
    *bytes = plan_bytes(cached_plan(a));
    return SWAPNET_OK;
  });
}

int swapnet_attention_tree(const swapnet_cached_attention* c, void* workspace, uint64_t workspace_bytes, swapnet_stream stream) {
  return swapnet::guard_abi([&]() -> int {
    using namespace swapnet;
    CachedArgs a;
    if (int rc = check_attention(c, &a)) return rc;
    const CachedPlan p = cached_plan(a);
    const uint64_t need = plan_bytes(p);
    if (need && !workspace) SN_FAIL(SWAPNET_ERR_INVALID_ARG, "attention: null workspace");
    if (workspace_bytes < need) SN_FAIL(SWAPNET_ERR_INVALID_ARG, "attention: workspace too small");
    if (need && ((uintptr_t)workspace & (kAlign - 1))) SN_FAIL(SWAPNET_ERR_MISALIGNED, "attention: workspace must be 256-byte aligned");
    // (weights may be weights_in)
    if (shares({c->out, c->lse, c->weights, need ? workspace : nullptr},
               {c->q, c->k, c->v, c->k_new, c->v_new, c->lens, c->counts, c->parents}) ||
        shares({c->out, c->lse, need ? workspace : nullptr}, {c->weights_in}))
      SN_FAIL(SWAPNET_ERR_INVALID_ARG, "attention: a result must not be an input or another result");
    if (int rc = error_word(&a.err)) return rc;
    return run_cached_attention(a, p, workspace, false, reinterpret_cast<cudaStream_t>(stream));
  });
}

int swapnet_attention_weights(const swapnet_cached_attention* c, swapnet_stream stream) {
  return swapnet::guard_abi([&]() -> int {
    using namespace swapnet;
    CachedArgs a;
    if (int rc = fill_args(c, &a)) return rc;
    if (!c->lse || !c->weights) SN_FAIL(SWAPNET_ERR_INVALID_ARG, "cache weights: null pointer");
    if (c->k_new || c->v_new || c->parents) SN_FAIL(SWAPNET_ERR_INVALID_ARG, "cache weights: the queries are rows of the cache");
    if (shares({c->weights}, {c->q, c->k, c->lens, c->counts, c->rows, c->lse}))
      SN_FAIL(SWAPNET_ERR_INVALID_ARG, "cache weights: the result must not be an input");
    if (int rc = error_word(&a.err)) return rc;
    return launch_weights(a, weights_splits(a), false, reinterpret_cast<cudaStream_t>(stream));
  });
}

int swapnet_cache_evict(const swapnet_cache_eviction* c, swapnet_stream stream) {
  return swapnet::guard_abi([&]() -> int {
    using namespace swapnet;
    if (!c) SN_FAIL(SWAPNET_ERR_INVALID_ARG, "null arguments");
    EvictArgs a;
    std::memset(&a, 0, sizeof(a));
    if (c->dtype != SWAPNET_F16 && c->dtype != SWAPNET_BF16) SN_FAIL(SWAPNET_ERR_UNSUPPORTED, "eviction: fp16 or bf16 only");
    if (c->n_seq < 1 || c->kv_heads < 1 || c->head_dim < 1 || c->max_seq < 1 || c->keep < 1)
      SN_FAIL(SWAPNET_ERR_INVALID_ARG, "eviction: empty shape");
    if (c->head_dim % 8 || c->head_dim > 512) SN_FAIL(SWAPNET_ERR_UNSUPPORTED, "eviction: head width must be a multiple of 8, at most 512");
    if (c->n_seq > 65535 || c->kv_heads > 65535 || c->max_seq > (1 << 30) || (int64_t)c->keep * (c->head_dim / 8) > (1 << 30))
      SN_FAIL(SWAPNET_ERR_UNSUPPORTED, "eviction: shape beyond the kernels' limits");
    if (c->recent < 0 || c->sink < 0 || (int64_t)c->recent + c->sink > c->keep)
      SN_FAIL(SWAPNET_ERR_INVALID_ARG, "eviction: sink + recent must be within keep");
    if (!c->k || !c->v || !c->weights || !c->lens || !c->k_out || !c->v_out || !c->weights_out || !c->kept || !c->lens_out)
      SN_FAIL(SWAPNET_ERR_INVALID_ARG, "eviction: null pointer");
    const int64_t width = (int64_t)c->kv_heads * c->head_dim;
    a.n_seq = c->n_seq;
    a.kv_heads = c->kv_heads;
    a.dim = c->head_dim;
    a.max_seq = c->max_seq;
    a.keep = c->keep;
    a.recent = c->recent;
    a.sink = c->sink;
    a.out_seq = c->out_capacity ? c->out_capacity : c->max_seq;
    a.kv_stride = c->kv_stride ? c->kv_stride : width;
    a.seq_stride = c->seq_stride ? c->seq_stride : a.kv_stride * c->max_seq;
    a.out_stride = c->out_stride ? c->out_stride : width;
    a.out_seq_stride = c->out_seq_stride ? c->out_seq_stride : a.out_stride * a.out_seq;
    a.k = c->k;
    a.v = c->v;
    a.k_out = c->k_out;
    a.v_out = c->v_out;
    a.weights = c->weights;
    a.weights_out = c->weights_out;
    a.lens = c->lens;
    a.lens_step = 1;
    a.kept = c->kept;
    a.lens_out = c->lens_out;
    if (a.out_seq < a.keep) SN_FAIL(SWAPNET_ERR_INVALID_ARG, "eviction: out_capacity smaller than keep");
    if (a.kv_stride < width || a.out_stride < width || (c->n_seq > 1 && (a.seq_stride < 1 || a.out_seq_stride < 1)))
      SN_FAIL(SWAPNET_ERR_INVALID_ARG, "eviction: a stride is smaller than a row");
    if ((a.kv_stride | a.seq_stride | a.out_stride | a.out_seq_stride) % 8 || !aligned16(a.k) || !aligned16(a.v) ||
        !aligned16(a.k_out) || !aligned16(a.v_out))
      SN_FAIL(SWAPNET_ERR_MISALIGNED, "eviction: caches and strides must be 16-byte aligned");
    if (!aligned4(a.weights, a.weights_out, a.lens, a.kept, a.lens_out))
      SN_FAIL(SWAPNET_ERR_MISALIGNED, "eviction: int32 and float arrays must be 4-byte aligned");
    // in place means the same rows: another layout over the same memory would be read after it was written
    const bool same[3] = {a.k == a.k_out, a.v == a.v_out, a.weights == a.weights_out};
    if (same[0] != same[1] || same[0] != same[2])
      SN_FAIL(SWAPNET_ERR_INVALID_ARG, "eviction: keys, values and weights are all moved in place or all to other buffers");
    if (same[0] && (a.kv_stride != a.out_stride || a.seq_stride != a.out_seq_stride || a.out_seq != a.max_seq))
      SN_FAIL(SWAPNET_ERR_INVALID_ARG, "eviction: in place the output has the input's layout");
    if (a.lens == a.lens_out) SN_FAIL(SWAPNET_ERR_INVALID_ARG, "eviction: lens_out must not be lens (every head reads lens)");
    if (shares({a.k_out, a.v_out, a.weights_out, a.kept, a.lens_out}, {a.lens}) || shares({a.k_out}, {a.v, a.weights}) ||
        shares({a.v_out}, {a.k, a.weights}) || shares({a.weights_out}, {a.k, a.v}) || shares({a.kept, a.lens_out}, {a.k, a.v, a.weights}))
      SN_FAIL(SWAPNET_ERR_INVALID_ARG, "eviction: a result must not be another input or result");
    if (int rc = error_word(&a.err)) return rc;
    return launch_cache_evict(a, reinterpret_cast<cudaStream_t>(stream));
  });
}

int swapnet_tree_accept(const swapnet_tree_acceptance* c, swapnet_stream stream) {
  return swapnet::guard_abi([&]() -> int {
    using namespace swapnet;
    if (!c) SN_FAIL(SWAPNET_ERR_INVALID_ARG, "null arguments");
    AcceptArgs a;
    std::memset(&a, 0, sizeof(a));
    if (c->dtype != SWAPNET_F16 && c->dtype != SWAPNET_BF16) SN_FAIL(SWAPNET_ERR_UNSUPPORTED, "tree acceptance: fp16 or bf16 only");
    if (c->n_seq < 1 || c->tokens < 1 || c->width < 1 || c->max_seq < 1 || c->n_caches < 0)
      SN_FAIL(SWAPNET_ERR_INVALID_ARG, "tree acceptance: empty shape");
    if (c->tokens > kTreeMax || c->n_caches > kAcceptMaxCaches || c->n_seq > 65535 || c->max_seq > (1 << 30))
      SN_FAIL(SWAPNET_ERR_UNSUPPORTED, "tree acceptance: at most 128 nodes a sequence and 256 caches");
    if (c->width > (1 << 24)) SN_FAIL(SWAPNET_ERR_UNSUPPORTED, "tree acceptance: rows of at most 2^24 elements");
    if (c->width % 8) SN_FAIL(SWAPNET_ERR_UNSUPPORTED, "tree acceptance: width must be a multiple of 8");
    if (!c->ids || !c->targets || !c->lens || !c->path || !c->accepted || !c->next || !c->lens_out || (c->n_caches && (!c->caches || !c->drafts)))
      SN_FAIL(SWAPNET_ERR_INVALID_ARG, "tree acceptance: null pointer");
    a.n_seq = c->n_seq;
    a.tokens = c->tokens;
    a.width = c->width;
    a.max_seq = c->max_seq;
    a.n_caches = c->n_caches;
    a.cache_stride = c->cache_stride ? c->cache_stride : c->width;
    a.seq_stride = c->seq_stride ? c->seq_stride : a.cache_stride * c->max_seq;
    a.new_stride = c->new_stride ? c->new_stride : c->width;
    if (a.cache_stride < c->width || a.new_stride < c->width || (c->n_seq > 1 && a.seq_stride < 1))
      SN_FAIL(SWAPNET_ERR_INVALID_ARG, "tree acceptance: a stride is smaller than a row");
    if ((a.cache_stride | a.seq_stride | a.new_stride) % 8) SN_FAIL(SWAPNET_ERR_MISALIGNED, "tree acceptance: strides must be multiples of 8 elements");
    for (int i = 0; i < c->n_caches; ++i) {
      if (!c->caches[i] || !c->drafts[i]) SN_FAIL(SWAPNET_ERR_INVALID_ARG, "tree acceptance: null cache");
      if (!aligned16(c->caches[i]) || !aligned16(c->drafts[i]))
        SN_FAIL(SWAPNET_ERR_MISALIGNED, "tree acceptance: caches must be 16-byte aligned");
      a.caches[i] = c->caches[i];
      a.drafts[i] = c->drafts[i];
    }
    a.ids = c->ids;
    a.targets = c->targets;
    a.parents = c->parents;
    a.counts = c->counts;
    a.lens = c->lens;
    a.path = c->path;
    a.accepted = c->accepted;
    a.next = c->next;
    a.lens_out = c->lens_out;
    if (!aligned4(a.ids, a.targets, a.parents, a.counts, a.lens, a.path, a.accepted, a.next, a.lens_out))
      SN_FAIL(SWAPNET_ERR_MISALIGNED, "tree acceptance: int32 arrays must be 4-byte aligned");
    // every cache's CTA reads the inputs while the first one writes the results
    if (shares({a.path, a.accepted, a.next, a.lens_out}, {a.ids, a.targets, a.parents, a.counts, a.lens}))
      SN_FAIL(SWAPNET_ERR_INVALID_ARG, "tree acceptance: a result must not be an input or another result");
    if (int rc = error_word(&a.err)) return rc;
    return launch_tree_accept(a, reinterpret_cast<cudaStream_t>(stream));
  });
}

}  // extern "C"
