// Internal interface of the cached-attention operators (swapnet_attention_tree,
// swapnet_attention_weights, swapnet_cache_evict, swapnet_tree_accept): what
// their kernels get, filled in by the entry points once the arguments have
// been checked (cached.cpp).
#pragma once
#include <cuda_runtime.h>
#include <algorithm>
#include <cstdint>

namespace swapnet {

constexpr int kFewAttnRows = 16;   // of a (sequence, key head) that the few-row kernel takes
constexpr int kTreeMax = 128;  // drafted nodes of a sequence: one tile of keys, 128 ancestor bits

// Row r of a (sequence, key head) is query r / group of the sequence for head
// r % group of the group.
struct CachedArgs {
  int dtype, n_seq, tokens, heads, kv_heads, group, dim, max_seq;
  float scale_log2;  // log2(e) * scale
  const void *q, *k, *v, *k_new, *v_new;
  int64_t q_stride, kv_stride, seq_stride, new_stride, out_stride;  // elements
  // per sequence: lens[b * lens_step] + len_add cached rows, counts[b *
  // counts_step] queries, a list of queries at rows + b * rows_step (a step of
  // 0: one value for all)
  const int *lens, *counts, *parents, *rows;
  int lens_step, counts_step, rows_step, len_add;
  void* out;
  float* lse;
  const float* weights_in;
  float* weights;
  int* err;
  // workspace (attention): per (sequence, key head, split, row) the outputs
  // relative to that split's maximum, the maximum and the sum; with weights
  // on the few-row kernel the scaled scores [sequence][key head][row][score_ld]
  int splits;
  float *part, *ml, *scores;
  int64_t score_ld;
  int4* units;  // tensor-core kernel, runs: per CTA the unit that it begins and others go on with
                // (sequence, row tile, key head, how many share it; 0: none)
};
// CTAs that share the tiles of all units: as many runs for every key head as
// find an SM each.
constexpr int kSms = 152;
inline int run_ctas(int kv_heads) { return std::max(1, kSms / kv_heads) * kv_heads; }


// How a call runs, from its sizes alone.
struct CachedPlan {
  int tc;       // tensor-core kernel (rows in tiles of 128)
  int splits;   // few rows: CTAs that share the keys of a (sequence, key head);
                // tensor cores: 1: a CTA per unit, 0: equal runs of all tiles
  int spill;    // weights from stored scores; 0: from a second pass over the keys
  int64_t score_ld;
  uint64_t part_bytes, ml_bytes, score_bytes, unit_bytes;
};
CachedPlan cached_plan(const CachedArgs& a);
// Attention as that plan says, its workspace at `workspace`; weights too where
// asked for.  early: the launch may start while the one before it ends.
int run_cached_attention(CachedArgs a, const CachedPlan& p, void* workspace, bool early, cudaStream_t s);
inline uint64_t plan_bytes(const CachedPlan& p) { return p.part_bytes + p.ml_bytes + p.score_bytes + p.unit_bytes; }
int cached_launches(const CachedArgs& a, const CachedPlan& p);

int launch_attention_rows(const CachedArgs& a, bool early, cudaStream_t s);  // tcgen05
int launch_attention_few(const CachedArgs& a, bool early, cudaStream_t s);
int launch_attention_join(const CachedArgs& a, cudaStream_t s);   // splits -> out, lse (and weights from scores)
int launch_weights(const CachedArgs& a, int splits, bool early, cudaStream_t s);  // tcgen05
int weights_splits(const CachedArgs& a);

struct EvictArgs {
  int n_seq, kv_heads, dim, max_seq, keep, recent, sink, out_seq;
  int64_t kv_stride, seq_stride, out_stride, out_seq_stride;
  const void *k, *v;
  void *k_out, *v_out;
  const float* weights;
  float* weights_out;
  const int* lens;
  int lens_step;        // 0: one length for all sequences
  int *kept, *lens_out; // (lens_out: nullable)
  int* err;
};
int launch_cache_evict(const EvictArgs& a, cudaStream_t s);

constexpr int kAcceptMaxCaches = 256;
struct AcceptArgs {
  int n_seq, tokens, width, max_seq, n_caches;
  int64_t cache_stride, seq_stride, new_stride;  // elements
  const int *ids, *targets, *parents, *counts, *lens;
  int *path, *accepted, *next, *lens_out;
  int* err;
  void* caches[kAcceptMaxCaches];
  const void* drafts[kAcceptMaxCaches];
};
int launch_tree_accept(const AcceptArgs& a, cudaStream_t s);

}  // namespace swapnet
