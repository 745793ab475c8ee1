// Internal interface of the quantised-cache operators (swapnet_cache_append,
// swapnet_attention_quantized): what their kernels get, filled in by the entry
// points once the arguments have been checked (quant.cpp).
#pragma once
#include "cached.h"

namespace swapnet {

// Code formats of a cache; kCode16: rows of the storage type.
enum { kCodeI8 = 0, kCodeE4M3 = 1, kCode16 = 2 };
constexpr float kLeastScale = 7.888609052210118e-31f;  // 2^-100
constexpr int kMaxPosition = 1 << 24;  // an fp32 holds every whole number below

struct AppendArgs {
  int dtype, code, n_seq, tokens, heads, kv_heads, dim, max_seq, block, blocks;  // blocks: scales of a (sequence, head)
  int rope_dim, halves, axis1, axis2;  // (rope_dim 0: no rotation) the first pairs of axes 1 and 2
  float eps;
  const void *q, *k_new, *v_new, *q_gain, *k_gain;
  const int *lens, *counts, *positions;
  void *q_out, *k, *v;
  float *k_scale, *v_scale;
  const void *k_open, *v_open;
  void *k_open_out, *v_open_out;
  int* lens_out;
  int64_t q_stride, new_stride, out_stride, kv_stride, seq_stride;  // elements
  int* err;
  int q_ctas, kv_ctas, row_ctas, block_ctas;  // of a sequence: for queries, for 16-bit keys (and as many for values), all these; for blocks
  float2 turns[64];          // a pair's turns per position, as the sum of two numbers
};
int launch_cache_append(AppendArgs a, cudaStream_t s);

// The attention's arguments; of those of the 16-bit caches there are no draft
// and no weights, k and v are codes and kv_stride and seq_stride count them.
struct QuantArgs : CachedArgs {
  int code, block, block_log2, blocks;
  const float *k_scale, *v_scale;
};
// How a call runs, from its sizes alone; tc: 0 warp products, on the tensor cores
// 1 rows as rows, 2 keys as rows; ctas: of its attention launch, row_tile: rows
// of a unit.
CachedPlan quant_plan(const QuantArgs& a, int* ctas, int* row_tile);
int run_quant_attention(QuantArgs a, const CachedPlan& p, int ctas, int row_tile, void* workspace, cudaStream_t s);
constexpr int kQuantFewRows = 32;  // of a unit, at most, on warp products
// Their CTAs that an SM holds, by registers and shared memory.
constexpr int quant_few_resident(int rows, int dim) { return rows <= 8 ? (dim == 64 ? 4 : 3) : rows <= 16 && dim == 64 ? 3 : 2; }
int launch_quant_join(const QuantArgs& a, int queries, int row_tile, int nrt, cudaStream_t s);  // the units that runs shared
int launch_quant_few(const QuantArgs& a, int ctas, int row_tile, cudaStream_t s);  // warp products, with the join
int launch_quant_keys(const QuantArgs& a, int ctas, cudaStream_t s);  // tcgen05, keys as rows: units of 32 rows 128 wide, with the join
int launch_quant_rows(const QuantArgs& a, int ctas, cudaStream_t s);  // tcgen05, with the join

}  // namespace swapnet
