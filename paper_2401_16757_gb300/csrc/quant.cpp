// Entry points of the quantised-cache operators: argument checks, the choice
// of kernels and the workspace.  Nothing is allocated and nothing waits for
// the device.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "internal.h"
#include "kernels.h"
#include "quant.h"

namespace swapnet {

// Microseconds: a unit's start and end, a tile of 128 keys by itself and its
// share of a busy SM's time, the join of shared units, rounds of more units than
// fit at once, at least; warp products of up to 16 and 32 rows, the tensor cores
// with keys as rows (32), with rows of 64 and 128.
struct Costs {
  double unit, tile, busy, join, rounds;
};
constexpr Costs kFewCosts = {3.0, 0.9, 0.8, 5.0, 1.0}, kMoreCosts = {6.0, 1.3, 1.05, 6.0, 1.0}, kKeyCosts = {7.0, 0.8, 0.8, 8.0, 2.0},
                kTc64Costs = {8.0, 1.8, 1.8, 10.0, 1.0}, kTc128Costs = {8.0, 2.3, 2.3, 10.0, 1.0};
// CTAs that share the tiles of all units: as many as are resident, or for up to
// 16 rows, which the memory bounds, up to six times that where their runs are
// long: the memory does not serve all SMs alike, and CTAs that start later even
// that out (one token of 64 sequences, up to 16384 rows: 273 us with 456 runs,
// whose times lie between 174 and 279, 268 with three times, 259 with six times
// as many; 32 rows pay more for a run's end: 127 us with 304 runs, 141 with
// twice as many).
constexpr int kRunLeast = 24;  // tiles of such a run

// A way to run a call: rows of a unit, how its tiles are shared, its cost.
struct Way {
  int row_tile, splits, ctas;
  int64_t units;
  double us;
};
static Way way(const QuantArgs& a, const Costs& c, int row_tile, int resident) {
  Way w;
  const int queries = std::min(row_tile / a.group, a.tokens);
  w.row_tile = row_tile;
  w.units = (int64_t)a.n_seq * a.kv_heads * ((a.tokens + queries - 1) / queries);
  // A CTA per unit, or equal runs of all tiles and a join.  Where units queue for
  // the SMs, part of one waits for the last at the end (lengths and causal
  // limits differ).
  const double tiles = (a.max_seq + 127) / 128, slots = (double)kSms * resident;
  int runs = std::max(1, kSms * resident / a.kv_heads) * a.kv_heads;
  auto per_tile = [&](double on_sm) { return std::max(c.tile, c.busy * std::min((double)resident, std::ceil(on_sm))); };
  const double alone = (c.unit + per_tile((double)w.units / kSms) * tiles) * (w.units <= slots ? 1.0 : std::max(c.rounds, w.units / slots + 0.1));
  const double mine = std::max(2.0, w.units * tiles / runs);  // tiles of a run
  const double shared = c.unit * (1.0 + (double)w.units / runs) + per_tile(w.units * tiles / mine / kSms) * mine + c.join;
  if (row_tile <= 16) runs *= (int)std::min(6.0, std::max(1.0, mine / kRunLeast));
  // (tensor cores with two units per SM: 512 units of up to 33 tiles 178 us, in runs 219)
  w.splits = alone <= shared || w.units > 65535 || (resident == 1 && w.units >= 2 * kSms) ? 1 : 0;
  w.ctas = w.splits ? (int)w.units : runs;
  w.us = w.splits ? alone : shared;
  return w;
}

CachedPlan quant_plan(const QuantArgs& a, int* ctas, int* row_tile) {
  CachedPlan p;
  std::memset(&p, 0, sizeof(p));
  const int64_t rows = (int64_t)a.tokens * a.group;
  const int tile = rows <= 8 ? 8 : rows <= 16 ? 16 : 32;
  Way w;
  w.us = 1e30;
  if (a.group <= tile) w = way(a, rows <= 16 ? kFewCosts : kMoreCosts, tile, quant_few_resident(tile, a.dim));
  if (rows > 16 && a.group <= kQuantFewRows && a.dim == 128) {
    // 32 sequences, 8 key heads of 32 rows, up to 8000 keys 112 us, on warp
    // products 131 (16 rows 107 and 97, 8 x 8 of them on 2000 keys 24.5 and 22.6); 4
    // of up to 500 keys 12.5 and 18.3.  More rows are units that
    // convert the same keys, which pays while every unit has an SM: 8 x 8 of 64
    // rows, 2000 keys 26.6 us, with rows as the products' rows 42.1; 32 x 8 of
    // them, up to 8000 keys 208 and 161.
    const Way t = way(a, kKeyCosts, kQuantFewRows, 1);
    if (t.us <= w.us && (rows <= kQuantFewRows || (t.splits == 1 && t.units <= kSms))) {
      w = t;
      p.tc = 2;
    }
  }
  if (rows > kQuantFewRows) {
    // (two or more tiles of warp products for a small call: they start and end
    // sooner; 78 rows of 10 sequences on 2052 rows: 33 us on the tensor cores)
    const Way t = rows <= 64 ? way(a, kTc64Costs, 64, 1) : way(a, kTc128Costs, 128, 1);
    if (t.us <= w.us) {
      w = t;
      p.tc = 1;
    }
  }
  p.splits = w.splits;
  if (p.splits == 0) {
    p.part_bytes = align_up((uint64_t)2 * w.ctas * w.row_tile * a.dim * 4);
    p.ml_bytes = align_up((uint64_t)2 * w.ctas * w.row_tile * 8);
    p.unit_bytes = align_up((uint64_t)w.units * 8);
  }
  *ctas = w.ctas;
  *row_tile = w.row_tile;
  return p;
}

int run_quant_attention(QuantArgs a, const CachedPlan& p, int ctas, int row_tile, void* workspace, cudaStream_t s) {
  char* w = static_cast<char*>(workspace);
  a.splits = p.splits;
  a.part = reinterpret_cast<float*>(w);
  a.ml = reinterpret_cast<float*>(w + p.part_bytes);
  a.units = reinterpret_cast<int4*>(w + p.part_bytes + p.ml_bytes);
  if (p.tc == 2) return launch_quant_keys(a, ctas, s);
  return p.tc ? launch_quant_rows(a, ctas, s) : launch_quant_few(a, ctas, row_tile, s);
}

namespace {

constexpr double kTurn = 6.283185307179586476925;

int code_of(int dtype, int cache_dtype) {
  return cache_dtype == SWAPNET_I8 ? kCodeI8 : cache_dtype == SWAPNET_E4M3 ? kCodeE4M3 : cache_dtype == dtype ? kCode16 : -1;
}
bool valid_block(int block) { return block == 16 || block == 32 || block == 64 || block == 128; }

int check_append(const swapnet_cache_rows* c, AppendArgs* a) {
  if (!c) SN_FAIL(SWAPNET_ERR_INVALID_ARG, "null arguments");
  std::memset(a, 0, sizeof(*a));
  if (c->dtype != SWAPNET_F16 && c->dtype != SWAPNET_BF16) SN_FAIL(SWAPNET_ERR_UNSUPPORTED, "cache append: fp16 or bf16 only");
  a->code = code_of(c->dtype, c->cache_dtype);
  if (a->code < 0) SN_FAIL(SWAPNET_ERR_UNSUPPORTED, "cache append: the cache has the rows' type, I8 or E4M3");
  const bool coded = a->code != kCode16;
  if (c->n_seq < 1 || c->tokens < 1 || c->heads < 0 || c->kv_heads < 1 || c->max_seq < 1)
    SN_FAIL(SWAPNET_ERR_INVALID_ARG, "cache append: empty shape");
  if (c->head_dim != 64 && c->head_dim != 128) SN_FAIL(SWAPNET_ERR_UNSUPPORTED, "cache append: head width must be 64 or 128");
  if (coded ? !valid_block(c->block) : c->block != 0)
    SN_FAIL(SWAPNET_ERR_UNSUPPORTED, "cache append: block must be 16, 32, 64 or 128 rows (0 for a 16-bit cache)");
  if (c->n_seq > 65535 || c->heads > 65535 || c->kv_heads > 65535 || c->max_seq > kMaxPosition || (int64_t)c->n_seq * c->tokens > (1 << 30))
    SN_FAIL(SWAPNET_ERR_UNSUPPORTED, "cache append: shape beyond the kernels' limits");
  if (!c->k_new || !c->v_new || !c->lens || !c->k || !c->v) SN_FAIL(SWAPNET_ERR_INVALID_ARG, "cache append: null pointer");
  if (!c->q != !c->heads || !c->q_out != !c->heads)
    SN_FAIL(SWAPNET_ERR_INVALID_ARG, "cache append: heads, queries and their result come together");
  if (!c->heads && c->q_gain) SN_FAIL(SWAPNET_ERR_INVALID_ARG, "cache append: a gain without queries");
  if (coded && (!c->k_scale || !c->v_scale || !c->k_open || !c->v_open)) SN_FAIL(SWAPNET_ERR_INVALID_ARG, "cache append: null pointer");
  if (!coded && (c->k_scale || c->v_scale || c->k_open || c->v_open || c->k_open_out || c->v_open_out))
    SN_FAIL(SWAPNET_ERR_INVALID_ARG, "cache append: a 16-bit cache has no scales and no open rows");
  if (!c->k_open_out != !c->v_open_out) SN_FAIL(SWAPNET_ERR_INVALID_ARG, "cache append: k_open_out and v_open_out come together");
  if (!(c->theta >= 0.f) || std::isinf(c->theta) || !(c->eps >= 0.f) || std::isinf(c->eps))
    SN_FAIL(SWAPNET_ERR_INVALID_ARG, "cache append: bad theta or eps");
  const int rope = c->rope_dim ? c->rope_dim : c->head_dim;
  if (rope < 16 || rope > c->head_dim || rope % 16) SN_FAIL(SWAPNET_ERR_UNSUPPORTED, "cache append: rope_dim must be a multiple of 16 up to head_dim");
  a->axis1 = a->axis2 = rope / 2;
  bool axes = false;
  if (c->theta > 0.f) {
    a->rope_dim = rope;
    const int64_t n0 = c->sections[0], n1 = c->sections[1], n2 = c->sections[2];
    if (n0 < 0 || n1 < 0 || n2 < 0 || (n0 + n1 + n2 != 0 && n0 + n1 + n2 != rope / 2))
      SN_FAIL(SWAPNET_ERR_INVALID_ARG, "cache append: the sections' pairs must add up to rope_dim / 2");
    axes = n1 || n2;
    if (axes) {
      a->axis1 = (int)n0;
      a->axis2 = (int)(n0 + n1);
    }
    // theta^(-2 i / rope), i = 8 j + k: from 8 powers each (64 of them took 0.6 us of a call)
    double fine[8], coarse = 1.0;
    for (int k = 0; k < 8; ++k) fine[k] = std::pow((double)c->theta, -2.0 * k / rope) / kTurn;
    for (int i = 0; i < rope / 2; ++i) {
      if (i % 8 == 0) coarse = std::pow((double)c->theta, -2.0 * i / rope);
      double turns = coarse * fine[i % 8];
      if (!(turns <= 1e6)) SN_FAIL(SWAPNET_ERR_INVALID_ARG, "cache append: bad theta or eps");
      if (turns > 0.5) turns -= std::rint(turns);  // (exact; positions are whole numbers, only theta below 1 has such)
      a->turns[i].x = (float)turns;
      a->turns[i].y = (float)(turns - (double)a->turns[i].x);
    }
  } else if (c->positions) {
    SN_FAIL(SWAPNET_ERR_INVALID_ARG, "cache append: positions without a rotation");
  }
  a->dtype = c->dtype;
  a->n_seq = c->n_seq;
  a->tokens = c->tokens;
  a->heads = c->heads;
  a->kv_heads = c->kv_heads;
  a->dim = c->head_dim;
  a->max_seq = c->max_seq;
  a->block = c->block;
  a->blocks = coded ? (c->max_seq + c->block - 1) / c->block : 0;
  a->halves = c->halves != 0;
  a->eps = c->eps;
  a->q = c->q;
  a->k_new = c->k_new;
  a->v_new = c->v_new;
  a->q_gain = c->q_gain;
  a->k_gain = c->k_gain;
  a->lens = c->lens;
  a->counts = c->counts;
  a->positions = c->positions;
  a->q_out = c->q_out;
  a->k = c->k;
  a->v = c->v;
  a->k_scale = c->k_scale;
  a->v_scale = c->v_scale;
  a->k_open = c->k_open;
  a->v_open = c->v_open;
  a->k_open_out = c->k_open_out ? c->k_open_out : const_cast<void*>(c->k_open);
  a->v_open_out = c->v_open_out ? c->v_open_out : const_cast<void*>(c->v_open);
  a->lens_out = c->lens_out;
  const int64_t width = (int64_t)c->heads * c->head_dim, kv_width = (int64_t)c->kv_heads * c->head_dim;
  a->q_stride = c->q_stride ? c->q_stride : width;
  a->out_stride = c->out_stride ? c->out_stride : width;
  a->new_stride = c->new_stride ? c->new_stride : kv_width;
  a->kv_stride = c->kv_stride ? c->kv_stride : kv_width;
  a->seq_stride = c->seq_stride ? c->seq_stride : a->kv_stride * c->max_seq;
  if (a->q_stride < width || a->out_stride < width || a->new_stride < kv_width || a->kv_stride < kv_width ||
      (c->n_seq > 1 && a->seq_stride < 1))
    SN_FAIL(SWAPNET_ERR_INVALID_ARG, "cache append: a stride is smaller than a row");
  if ((a->q_stride | a->out_stride | a->new_stride) % 8 || (a->kv_stride | a->seq_stride) % (coded ? 16 : 8))
    SN_FAIL(SWAPNET_ERR_MISALIGNED, "cache append: strides must be multiples of 16 bytes");
  for (const void* p : {c->q, c->k_new, c->v_new, c->q_gain, c->k_gain, (const void*)c->q_out, (const void*)c->k, (const void*)c->v,
                        c->k_open, c->v_open, (const void*)c->k_open_out, (const void*)c->v_open_out})
    if (!aligned16(p)) SN_FAIL(SWAPNET_ERR_MISALIGNED, "cache append: pointers must be 16-byte aligned");
  if (!aligned4(c->lens, c->counts, c->positions, c->k_scale, c->v_scale, c->lens_out))
    SN_FAIL(SWAPNET_ERR_MISALIGNED, "cache append: int32 and float arrays must be 4-byte aligned");
  // (q_out may be q, the open rows' results the open rows)
  if (shares({c->q_out, c->k, c->v, c->k_scale, c->v_scale, c->lens_out},
             {c->k_new, c->v_new, c->q_gain, c->k_gain, c->lens, c->counts, c->positions, c->k_open, c->v_open}) ||
      shares({c->k, c->v, c->k_scale, c->v_scale, c->lens_out, a->k_open_out, a->v_open_out},
             {c->q, c->q_out, c->k_new, c->v_new, c->q_gain, c->k_gain, c->lens, c->counts, c->positions}))
    SN_FAIL(SWAPNET_ERR_INVALID_ARG, "cache append: a result must not be another input or result");
  if (coded && (a->k_open_out == c->v_open || a->v_open_out == c->k_open || (a->k_open_out == c->k_open) != (a->v_open_out == c->v_open)))
    SN_FAIL(SWAPNET_ERR_INVALID_ARG, "cache append: open rows of keys and values stay in place or both go elsewhere");
  if (c->q_out && c->q_out == c->q && a->q_stride != a->out_stride)
    SN_FAIL(SWAPNET_ERR_INVALID_ARG, "cache append: queries in place keep their stride");
  return SWAPNET_OK;
}

int check_quant(const swapnet_quantized_attention* c, QuantArgs* a) {
  if (!c) SN_FAIL(SWAPNET_ERR_INVALID_ARG, "null arguments");
  std::memset(static_cast<void*>(a), 0, sizeof(*a));
  if (c->dtype != SWAPNET_F16 && c->dtype != SWAPNET_BF16) SN_FAIL(SWAPNET_ERR_UNSUPPORTED, "quantised attention: fp16 or bf16 only");
  a->code = c->cache_dtype == SWAPNET_I8 ? kCodeI8 : c->cache_dtype == SWAPNET_E4M3 ? kCodeE4M3 : -1;
  if (a->code < 0) SN_FAIL(SWAPNET_ERR_UNSUPPORTED, "quantised attention: a cache of I8 or E4M3");
  if (c->n_seq < 1 || c->tokens < 1 || c->heads < 1 || c->kv_heads < 1 || c->max_seq < 1)
    SN_FAIL(SWAPNET_ERR_INVALID_ARG, "quantised attention: empty shape");
  if (c->heads % c->kv_heads) SN_FAIL(SWAPNET_ERR_INVALID_ARG, "quantised attention: heads must be a multiple of kv_heads");
  if (c->head_dim != 64 && c->head_dim != 128) SN_FAIL(SWAPNET_ERR_UNSUPPORTED, "quantised attention: head width must be 64 or 128");
  if (!valid_block(c->block)) SN_FAIL(SWAPNET_ERR_UNSUPPORTED, "quantised attention: block must be 16, 32, 64 or 128 rows");
  const int64_t group = c->heads / c->kv_heads;
  if (c->n_seq > 65535 || c->kv_heads > 65535 || group > 128 || (int64_t)c->tokens * group > (1 << 20) || c->max_seq > (1 << 30) ||
      (int64_t)c->n_seq * c->tokens > (1 << 30) || (int64_t)c->n_seq * c->tokens * c->kv_heads > 0x7fffffff)
    SN_FAIL(SWAPNET_ERR_UNSUPPORTED, "quantised attention: shape beyond the kernels' limits");
  if (!c->q || !c->k || !c->v || !c->k_scale || !c->v_scale || !c->lens || !c->out)
    SN_FAIL(SWAPNET_ERR_INVALID_ARG, "quantised attention: null pointer");
  if (!(c->scale >= 0.f) || std::isinf(c->scale)) SN_FAIL(SWAPNET_ERR_INVALID_ARG, "quantised attention: bad scale");
  a->scale_log2 = 1.4426950408889634f * (c->scale > 0.f ? c->scale : 1.0f / sqrtf((float)c->head_dim));
  if (std::isinf(a->scale_log2)) SN_FAIL(SWAPNET_ERR_INVALID_ARG, "quantised attention: bad scale");
  const int64_t kv_width = (int64_t)c->kv_heads * c->head_dim, width = (int64_t)c->heads * c->head_dim;
  a->dtype = c->dtype;
  a->n_seq = c->n_seq;
  a->tokens = c->tokens;
  a->heads = c->heads;
  a->kv_heads = c->kv_heads;
  a->group = (int)group;
  a->dim = c->head_dim;
  a->max_seq = c->max_seq;
  a->block = c->block;
  a->block_log2 = c->block == 16 ? 4 : c->block == 32 ? 5 : c->block == 64 ? 6 : 7;
  a->blocks = (c->max_seq + c->block - 1) / c->block;
  a->q = c->q;
  a->k = c->k;
  a->v = c->v;
  a->k_scale = c->k_scale;
  a->v_scale = c->v_scale;
  a->lens = c->lens;
  a->counts = c->counts;
  a->lens_step = a->counts_step = 1;
  a->out = c->out;
  a->lse = c->lse;
  a->q_stride = c->q_stride ? c->q_stride : width;
  a->kv_stride = c->kv_stride ? c->kv_stride : kv_width;
  a->seq_stride = c->seq_stride ? c->seq_stride : a->kv_stride * c->max_seq;
  a->out_stride = c->out_stride ? c->out_stride : width;
  if (a->q_stride < width || a->kv_stride < kv_width || a->out_stride < width || (c->n_seq > 1 && a->seq_stride < 1))
    SN_FAIL(SWAPNET_ERR_INVALID_ARG, "quantised attention: a stride is smaller than a row");
  if ((a->q_stride | a->out_stride) % 8 || (a->kv_stride | a->seq_stride) % 16)
    SN_FAIL(SWAPNET_ERR_MISALIGNED, "quantised attention: strides must be multiples of 16 bytes");
  if (!aligned16(c->q) || !aligned16(c->k) || !aligned16(c->v) || !aligned16(c->out))
    SN_FAIL(SWAPNET_ERR_MISALIGNED, "quantised attention: pointers must be 16-byte aligned");
  if (!aligned4(c->k_scale, c->v_scale, c->lens, c->counts, c->lse))
    SN_FAIL(SWAPNET_ERR_MISALIGNED, "quantised attention: int32 and float arrays must be 4-byte aligned");
  return SWAPNET_OK;
}

}  // namespace
}  // namespace swapnet

extern "C" {

int swapnet_cache_append(const swapnet_cache_rows* c, swapnet_stream stream) {
  return swapnet::guard_abi([&]() -> int {
    using namespace swapnet;
    AppendArgs a;
    if (int rc = check_append(c, &a)) return rc;
    if (int rc = error_word(&a.err)) return rc;
    return launch_cache_append(a, reinterpret_cast<cudaStream_t>(stream));
  });
}

int swapnet_attention_quantized_workspace(const swapnet_quantized_attention* c, uint64_t* bytes) {
  return swapnet::guard_abi([&]() -> int {
    using namespace swapnet;
    if (!bytes) SN_FAIL(SWAPNET_ERR_INVALID_ARG, "null output");
    QuantArgs a;
    if (int rc = check_quant(c, &a)) return rc;
    int ctas, row_tile;
    *bytes = plan_bytes(quant_plan(a, &ctas, &row_tile));
    return SWAPNET_OK;
  });
}

int swapnet_attention_quantized_tiling(const swapnet_quantized_attention* c, swapnet_quantized_tiling* t) {
  return swapnet::guard_abi([&]() -> int {
    using namespace swapnet;
    if (!t) SN_FAIL(SWAPNET_ERR_INVALID_ARG, "null output");
    QuantArgs a;
    if (int rc = check_quant(c, &a)) return rc;
    int ctas, row_tile;
    const CachedPlan p = quant_plan(a, &ctas, &row_tile);
    *t = swapnet_quantized_tiling{p.tc, row_tile, p.splits != 1, ctas};
    return SWAPNET_OK;
  });
}

int swapnet_attention_quantized(const swapnet_quantized_attention* c, void* workspace, uint64_t workspace_bytes, swapnet_stream stream) {
  return swapnet::guard_abi([&]() -> int {
    using namespace swapnet;
    QuantArgs a;
    if (int rc = check_quant(c, &a)) return rc;
    int ctas, row_tile;
    const CachedPlan p = quant_plan(a, &ctas, &row_tile);
    const uint64_t need = plan_bytes(p);
    if (need && !workspace) SN_FAIL(SWAPNET_ERR_INVALID_ARG, "quantised attention: null workspace");
    if (workspace_bytes < need) SN_FAIL(SWAPNET_ERR_INVALID_ARG, "quantised attention: workspace too small");
    if (need && ((uintptr_t)workspace & (kAlign - 1))) SN_FAIL(SWAPNET_ERR_MISALIGNED, "quantised attention: workspace must be 256-byte aligned");
    if (shares({c->out, c->lse, need ? workspace : nullptr}, {c->q, c->k, c->v, c->k_scale, c->v_scale, c->lens, c->counts}))
      SN_FAIL(SWAPNET_ERR_INVALID_ARG, "quantised attention: a result must not be an input or another result");
    if (int rc = error_word(&a.err)) return rc;
    return run_quant_attention(a, p, ctas, row_tile, workspace, reinterpret_cast<cudaStream_t>(stream));
  });
}

}  // extern "C"
