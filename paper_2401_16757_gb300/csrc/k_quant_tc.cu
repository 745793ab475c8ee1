// Attention of many query rows (chunks of a prompt, drafted runs) over a cache
// held in 8 bits, on the tcgen05 tensor cores; fp32 arithmetic, fixed orders of
// summation.
//
// Rows and units, runs of tiles and their join, the two softmaxes per tile (a
// half of the keys each) and the outputs in tensor memory are those of the
// 16-bit caches' attention (k_cached_tc.cu).  What differs:
//   codes    arrive by TMA as bytes in a ring of their own; four warps turn each
//            tile into the fp16 tile (128-byte swizzle) that the products read,
//            where the codes are exact.  tcgen05 has 8-bit operands, but then
//            queries and probabilities have to be 8-bit as well: two to four
//            parts of 4 bits each, for the same tensor time and less exactness
//   queries  as fp16, BF16 ones scaled by a power of two per row (the same warps)
//   scales   of keys: on the scores; of values 2^e f: e on the scores, f on the
//            probabilities (the sum takes p 2^-e), per part of 16 keys, which
//            lies in one block.  A lane of a softmax warp fetches one scale of
//            the next tile while this tile is computed
//            Scales as logarithms alone (one multiplication less a pair) came
//            out no faster
//   hidden   rows are masked in the scores; their codes are numbers (E4M3's two
//            that are none are cleared where rows of a tile are hidden), so that
//            a probability of 0 is all that hides a value
// Keys of a tile and values of the tile before are converted, and their products
// issued, as a pair: half of the waits of a tile at a time.
// Measured: 1000 queries on 4096 rows, 2 sequences x 32 heads, f16, I8: 181 us,
// 0.49 PFLOP/s (the second product of P not counted; the 16-bit caches' 124); 64
// rows of 32 x 8 units on up to 8000 rows, bf16, E4M3: 161.  No pipe is full: a tile of
// 128 x 128 takes about 4300 cycles, of which the tensor pipe is busy for 1540,
// the softmax warps for 2500 (64 rows: 1700), the conversion for 1550 (E4M3
// 1000); shared memory moves by count 260 KB of the 450 that it could, half of it
// codes and their fp16 form; instructions wait for their cache.  Slower: the
// reference from the overflow of packed probabilities instead of a maximum
// first (231 us), a single part of P (no faster), scores of half a tile at a time
// (no faster).
#include <algorithm>
#include <cstring>
#include <string>
#include <type_traits>

#include "internal.h"
#include "kernels.h"
#include "quant.cuh"

namespace swapnet {

namespace {

// warpgroups: TMA (warp 0) and MMA (warp 1); conversion; the softmax's two
constexpr int kSoftThreads = 256, kConvThreads = 128;
constexpr int kQtThreads = 128 + kConvThreads + kSoftThreads;
constexpr int kRegsIssue = 56, kRegsConv = 88, kRegsSoft = 184;
static_assert(128 * kRegsIssue + kConvThreads * kRegsConv + kSoftThreads * kRegsSoft <= kQtThreads * 128, "registers of a CTA");
// Where p lies, in log2 (see the 16-bit caches' PRange, and split_scale).
constexpr float kMost = kTop, kWide = kTop - 7.0f, kTight = kTop - 2.0f;
constexpr int kTightAt = 16;
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kTmO = 256;  // columns of O_0, O_1 behind it; S and P as there

template <int D> struct QtCfg {
  static constexpr int kHalves = D / 64;
  static constexpr int kBox = 128 * 128;              // bytes of a 128-row x 64-element fp16 box
  static constexpr int kTile = kHalves * kBox;
  static constexpr int kRaw = 128 * D;                // bytes of a tile's codes
  static constexpr int kSlots = 4;  // two pairs
  static constexpr int kRawSlots = D == 128 ? 3 : 6;
  static constexpr int kOffQ = 0;
  static constexpr int kOffRing = kTile;
  static constexpr int kOffRaw = kOffRing + kSlots * kTile;
  static constexpr int kOffX = kOffRaw + kRawSlots * kRaw;  // (m, l) of every softmax thread
  static constexpr int kOffBar = kOffX + kSoftThreads * 8;
  static constexpr int kOffStage = kOffBar + 384;           // REP 2: 16 columns of each half's 64 rows
  static constexpr int kOffNear = kOffStage + 2 * 64 * 20 * 4;
  static constexpr int kSmem = kOffNear + kNear * 8 + 1024;  // + alignment slack
  static_assert(kSmem <= 232448, "shared memory of a CTA");
};

// What a row's queries have been divided by.
template <typename T, int D> __device__ __forceinline__ float query_scale(const T* q) {
  if (std::is_same<T, __half>::value) return 1.0f;  // (as they are)
  uint32_t most = 0u;
#pragma unroll
  for (int c = 0; c < D / 8; ++c) most = max(most, largest_bits(reinterpret_cast<const uint4*>(q)[c]));
  return __uint_as_float((uint32_t)(query_exponent(most) - 14) << 23);
}

template <typename T, int D, int CODE, int REP>
__global__ void __launch_bounds__(kQtThreads, 1)
    attention_quant_rows_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                                const __grid_constant__ QuantArgs a, int queries, int nrt) {
  using F = QtCfg<D>;
  constexpr int kRowsMax = 128 / REP;
  constexpr int NK = 64 / REP;  // keys of a thread and tile
  constexpr int NG = NK / 16;   // parts of them
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  float2* ml = reinterpret_cast<float2*>(smem + F::kOffX);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + F::kOffBar);
  auto full = [&](int j) { return smem_u32(bars + (j & 1)); };      // a pair of fp16 tiles
  auto empty = [&](int j) { return smem_u32(bars + 4 + (j & 1)); };
  auto raw_full = [&](int s) { return smem_u32(bars + 8 + s); };    // a tile's codes
  auto raw_empty = [&](int s) { return smem_u32(bars + 14 + s); };
  // (P: one per half and buffer, a half may be two tiles ahead of the products)
  auto s_full = [&](int i) { return smem_u32(bars + 20 + (i & 1)); };
  auto p_full = [&](int h, int i) { return smem_u32(bars + 24 + 2 * h + (i & 1)); };
  auto o_full = [&](int h) { return smem_u32(bars + 28 + h); };
  const uint32_t q_full = smem_u32(bars + 30), q_free = smem_u32(bars + 31);  // a piece's queries
  const uint32_t o_done = smem_u32(bars + 32), o_free = smem_u32(bars + 33);  // a piece's outputs
  const uint32_t done_bar = smem_u32(bars + 34);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 35);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int2* near = reinterpret_cast<int2*>(smem + F::kOffNear);
  int64_t* sched = reinterpret_cast<int64_t*>(ml);  // (before the first results)

  const int warp = warp_index(), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < 2; ++s) {
      mbar_init(full(s), kConvThreads / 32);
      mbar_init(empty(s), 1);
    }
    for (int s = 0; s < F::kRawSlots; ++s) {
      mbar_init(raw_full(s), 1);
      mbar_init(raw_empty(s), kConvThreads / 32);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(o_full(i), 1);
      mbar_init(s_full(i), 1);
      for (int h = 0; h < 2; ++h) mbar_init(p_full(h, i), 4);
    }
    mbar_init(q_full, kConvThreads / 32);
    mbar_init(q_free, 1);
    mbar_init(o_done, 1);
    mbar_init(o_free, kSoftThreads / 32);
    mbar_init(done_bar, 1);
    *abort_flag = 0;
    fence_barrier_init();
    prefetch_tmap(&tmK);
    prefetch_tmap(&tmV);
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(tmem_slot), kTmemCols);
    tmem_relinquish();
  }
  pdl_wait();
  Cursor cur;
  tc_fence_before();
  const Run r_ = start_run(a, cur, near, sched, queries, nrt);
  const int kvh = r_.kvh;
  __syncthreads();  // (and sched is written again, as ml)
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  // (not before this CTA has its TMEM: a kernel that starts early may hold some
  // while it waits for this one's end)
  pdl_launch_dependents();
  // The run's tiles are taken in pairs: the keys of tile j with the values of tile
  // j - 1, across pieces; the last pair has values alone.  Tiles(j) yields them,
  // for every role in one loop (one place in the code for what it does: the CTA's
  // warps run five programs, whose instructions share the caches).
  struct Pair {
    bool keys, values, first, last;    // what there is; the keys' tile is its piece's first, last
    bool v_first, v_last;              // the same of the values' tile
    int b, tile, v_b, v_tile, piece, v_piece;
  };
  Pair pr;
  pr.keys = false;
  pr.piece = -1;
  int at = 0, of = 0;  // tile of the piece, its tiles
  auto next_pair = [&](int j) -> bool {  // j = 0, 1, 2, ...
    pr.values = j > 0;
    pr.v_first = pr.first;
    pr.v_last = pr.last;
    pr.v_b = pr.b;
    pr.v_tile = pr.tile;
    pr.v_piece = pr.piece;
    if (j > 0 && !pr.keys) return false;  // (the last pair has been)
    if (at == of) {
      pr.keys = cur.step(a, nrt, queries);
      at = 0;
      of = pr.keys ? cur.n : 0;
      if (pr.keys) ++pr.piece;
    }
    if (!pr.keys) return j > 0;
    pr.first = at == 0;
    pr.last = at == of - 1;
    pr.b = cur.b;
    pr.tile = cur.i0 + at;
    ++at;
    return true;
  };

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsIssue));
    if (warp == 0 && elect_one()) {
      // ---------------- TMA producer: the tiles' codes
      int pos = 0;
      bool ok = true;
      for (int j = 0; ok && next_pair(j); ++j) {
#pragma unroll 1
        for (int part = 0; part < 2; ++part) {
          if (!(part ? pr.values : pr.keys)) continue;
          const int s = pos % F::kRawSlots;
          if (pos >= F::kRawSlots && !(ok = mbar_wait_bounded(raw_empty(s), ((pos / F::kRawSlots) - 1) & 1, abort_flag, a.err))) break;
          mbar_arrive_expect_tx(raw_full(s), F::kRaw);
          tma_load_3d(smem_u32(smem + F::kOffRaw + s * F::kRaw), part ? &tmV : &tmK, raw_full(s), kvh * D,
                      (part ? pr.v_tile : pr.tile) * kKeys, part ? pr.v_b : pr.b);
          ++pos;
        }
      }
      // let every load issued land before the CTA can exit
      volatile int no_abort = 0;
      for (int p = max(0, pos - F::kRawSlots); p < pos; ++p)
        mbar_wait_bounded(raw_full(p % F::kRawSlots), (p / F::kRawSlots) & 1, &no_abort, nullptr);
    }
    if (warp == 1 && elect_one()) {
      // ---------------- MMA issuer
      constexpr uint32_t idesc_s = idesc_f16(0, 128, kKeys);
      constexpr uint32_t idesc_pv = idesc_f16(0, 128, D) | (1u << 16);  // B (values) MN-major
      const uint64_t qd = smem_desc_sw128(smem_u32(smem + F::kOffQ));
      const uint64_t kd = smem_desc_sw128(smem_u32(smem + F::kOffRing)), vd = desc_mn(smem_u32(smem + F::kOffRing + F::kTile));
      bool ok = true;
      auto wait = [&](uint32_t bar, uint32_t parity) { return ok = ok && mbar_wait_bounded(bar, parity, abort_flag, a.err); };
      for (int j = 0; ok && next_pair(j); ++j) {
        wait(full(j), (j >> 1) & 1);
        const uint64_t kt = kd + (uint64_t)((j & 1) * (2 * F::kTile >> 4)), vt = vd + (uint64_t)((j & 1) * (2 * F::kTile >> 4));  // the descriptors' address field counts 16 bytes
        // The next scores ahead of this tile's products, but for a new piece's,
        // whose queries may not be there yet.
#pragma unroll 1
        for (int turn = 0; ok && turn < 2; ++turn) {
          if ((turn == 1) == pr.first) {
            if (!pr.keys || (pr.first && !wait(q_full, pr.piece & 1))) continue;
            // (over the P of two tiles ago: the tensor core runs the MMAs of one
            // thread in the order of their issue, so its product, issued before,
            // has read it)
            tc_fence_after();
#pragma unroll
            for (int c = 0; c < F::kHalves; ++c)
#pragma unroll
              for (int k = 0; k < 4; ++k)
                tc_mma_f16(tmem + (uint32_t)(j & 1) * 128u, qd + (uint64_t)(c * (F::kBox >> 4) + 2 * k),
                           kt + (uint64_t)(c * (F::kBox >> 4) + 2 * k), idesc_s, (c | k) != 0);
            tc_commit(s_full(j));
            if (pr.last) tc_commit(q_free);
            continue;
          }
          if (!pr.values) continue;
          const int g = j - 1;
          if (pr.v_first && pr.v_piece > 0) wait(o_free, (pr.v_piece - 1) & 1);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (!wait(p_full(h, g), (g >> 1) & 1)) break;
            tc_fence_after();
            const uint32_t pt = tmem + (uint32_t)(g & 1) * 128u + (uint32_t)h * 64u;
#pragma unroll
            for (int part = 0; part < 2; ++part)  // of the probabilities
#pragma unroll
              for (int ks = 0; ks < 4; ++ks)  // 16 keys a step
                tc_mma_f16_ta(tmem + kTmO + (uint32_t)h * 128u, pt + (uint32_t)(part * 32 + ks * 8),
                              vt + (uint64_t)((h * 4 + ks) * (2048 >> 4)), idesc_pv, (uint32_t)(!pr.v_first || (part | ks) != 0));
            tc_commit(o_full(h));
          }
        }
        if (!ok) break;
        tc_commit(empty(j));
        if (pr.values && pr.v_last) tc_commit(o_done);
      }
      // every MMA issued must have finished before TMEM is freed
      tc_commit(done_bar);
      volatile int no_abort = 0;
      mbar_wait_bounded(done_bar, 0, &no_abort, nullptr);
    }
  } else if (warp < 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsConv));
    // ---------------- codes and queries to fp16
    const int ct = threadIdx.x - 128;
    // 16 codes a time: four lanes read 64 bytes of a row, their neighbours the
    // other 64 of the next, so that neither the reads nor the swizzled stores
    // meet in a bank
    const int r0 = ct >> 2;
    uint32_t from[F::kHalves], to[F::kHalves][2];  // of this thread's first chunks: in the codes, in the fp16 tile
#pragma unroll
    for (int u = 0; u < F::kHalves; ++u) {
      const int c = (ct & 3) + (F::kHalves == 2 ? 4 * ((r0 & 1) ^ u) : 0);
      from[u] = r0 * D + c * 16;
#pragma unroll
      for (int e = 0; e < 2; ++e) to[u][e] = (c >> 2) * F::kBox + r0 * 128 + ((((c & 3) * 2 + e) ^ (r0 & 7)) << 4);
    }
    int pos = 0, lim_min = 0, v_lim_min = 0;
    bool ok = true;
    for (int j = 0; ok && next_pair(j); ++j) {
      v_lim_min = lim_min;
      if (pr.keys && pr.first) lim_min = visible_limit(a, cur.z.len, cur.z.count, cur.rt * queries);
      ok = j < 2 || mbar_wait_bounded(empty(j), ((j >> 1) - 1) & 1, abort_flag, a.err);
#pragma unroll 1
      for (int part = 0; part < 2; ++part) {
        if (!(part ? pr.values : pr.keys)) continue;
        const int rs = pos % F::kRawSlots;
        ok = ok && mbar_wait_bounded(raw_full(rs), (pos / F::kRawSlots) & 1, abort_flag, a.err);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        const uint8_t* raw = smem + F::kOffRaw + rs * F::kRaw;
        uint8_t* tile = smem + F::kOffRing + ((j & 1) * 2 + part) * F::kTile;
        uint4 v[4][F::kHalves];  // (all read before the first store, which might be to the same memory for what the compiler knows)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int u = 0; u < F::kHalves; ++u) v[r][u] = *reinterpret_cast<const uint4*>(raw + r * 32 * D + from[u]);
        if (CODE == kCodeE4M3 && part && (pr.v_tile + 1) * kKeys > v_lim_min) {  // some rows are hidden from some queries
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int u = 0; u < F::kHalves; ++u)
              v[r][u] = make_uint4(numbers_only(v[r][u].x), numbers_only(v[r][u].y), numbers_only(v[r][u].z), numbers_only(v[r][u].w));
        }
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int u = 0; u < F::kHalves; ++u) {
            const uint2 x = pairs_near<CODE>(v[r][u].x), y = pairs_near<CODE>(v[r][u].y), z = pairs_near<CODE>(v[r][u].z),
                        w = pairs_near<CODE>(v[r][u].w);
            *reinterpret_cast<uint4*>(tile + r * 32 * 128 + to[u][0]) = make_uint4(x.x, x.y, y.x, y.y);
            *reinterpret_cast<uint4*>(tile + r * 32 * 128 + to[u][1]) = make_uint4(z.x, z.y, w.x, w.y);
          }
        __syncwarp();
        if (lane == 0) mbar_arrive(raw_empty(rs));
        ++pos;
      }
      if (!ok) break;
      fence_proxy_async_smem();  // the tiles are read by the tensor cores (async proxy)
      __syncwarp();
      if (lane == 0) mbar_arrive(full(j));
      if (!(pr.keys && pr.first)) continue;
      // a piece's queries: D / 8 lanes a row (REP 2: every row twice)
      ok = pr.piece == 0 || mbar_wait_bounded(q_free, (pr.piece - 1) & 1, abort_flag, a.err);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      constexpr int L = D / 8, kPass = kConvThreads / L, kBatch = 8;  // rows of a pass, passes whose loads are on the way together
      const int t0 = cur.rt * queries, rows = min(queries, cur.z.count - t0) * a.group, c = ct % L;
#pragma unroll 1
      for (int p0 = 0; p0 < rows; p0 += kBatch * kPass) {
        uint4 v[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          const int row = p0 + u * kPass + ct / L;
          v[u] = make_uint4(0u, 0u, 0u, 0u);
          if (row < rows)
            v[u] = reinterpret_cast<const uint4*>(static_cast<const T*>(a.q) + ((int64_t)cur.b * a.tokens + t0 + row / a.group) * a.q_stride +
                                                  (int64_t)(kvh * a.group + row % a.group) * D)[c];
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          const int row = p0 + u * kPass + ct / L;
          if (p0 + u * kPass >= kRowsMax) break;
          if (!std::is_same<T, __half>::value) {
            uint32_t most = largest_bits(v[u]);
#pragma unroll
            for (int off = L / 2; off > 0; off >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, off));
            const float by = __uint_as_float((uint32_t)(127 + 14 - (query_exponent(most) - 127)) << 23);
            v[u] = make_uint4(query_pair(v[u].x, by), query_pair(v[u].y, by), query_pair(v[u].z, by), query_pair(v[u].w, by));
          }
#pragma unroll
          for (int e = 0; e < REP; ++e) {
            const int r = row + e * kRowsMax;
            *reinterpret_cast<uint4*>(smem + F::kOffQ + (c >> 3) * F::kBox + r * 128 + (((c & 7) ^ (r & 7)) << 4)) = v[u];
          }
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(q_full);
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoft));
    // ---------------- softmax and output
    // two threads per row: `half` of a tile's keys, an output and a reference of
    // its own
    const int q4 = warp & 3, half = (warp - 8) >> 2;
    const int slot = q4 * 32 + lane, rep = slot / kRowsMax, row = slot % kRowsMax;
    const int aid = (warp - 8) * 32 + lane;
    const int kofs = half * 64 + rep * NK;  // this thread's first key of a tile
    const uint32_t lane_off = (uint32_t)(q4 * 32) << 16;
    const uint32_t tO = tmem + kTmO + (uint32_t)half * 128u + lane_off;
    auto row_sync = [&]() { asm volatile("bar.sync %0, 64;" ::"r"(1 + q4) : "memory"); };  // the two warps of the same rows
    auto all_sync = [&]() { asm volatile("bar.sync 5, %0;" ::"n"(kSoftThreads) : "memory"); };
    auto copy_sync = [&]() { asm volatile("bar.sync %0, 64;" ::"r"(8 + 2 * (q4 & 1) + half) : "memory"); };  // REP 2: a row's two lanes
    bool ok = true;
    int g0 = 0;
    int64_t at_tile = r_.first;
    for (int piece = 0; cur.step(a, nrt, queries); ++piece) {
      const int b = cur.b, n = cur.n, len = cur.z.len, count = cur.z.count;
      const int t0 = cur.rt * queries, rows = min(queries, count - t0) * a.group;
      const int lim_min = visible_limit(a, len, count, t0);
      const bool last = cur.i0 + n == cur.z.tiles, whole = cur.i0 == 0 && last;  // a piece up to the unit's end; all of it
      const bool works = q4 * 32 % kRowsMax < rows;  // the warp's lanes hold rows
      const int mine = min(row, rows - 1), t = t0 + mine / a.group;
      const int lim = visible_limit(a, len, count, t);
      // lane e < 4: the key scale of this warp's part e of 16 keys, lane 4 + e: the value scale
      const float* scale_from = (lane & 4 ? a.v_scale : a.k_scale) + ((int64_t)b * a.kv_heads + kvh) * a.blocks;
      const int scale_key = half * 64 + (q4 * 32 / kRowsMax) * NK + (lane & 3) * 16;
      auto fetch = [&](int i) {
        const int j = (cur.i0 + i) * kKeys + scale_key;
        return i < n && lane < 8 && (lane & 3) < NG && j < len ? scale_from[j >> a.block_log2] : 1.0f;
      };
      float scales = fetch(0);
      const T* q = static_cast<const T*>(a.q) + ((int64_t)b * a.tokens + t) * a.q_stride + (int64_t)(kvh * a.group + mine % a.group) * D;
      const float row_scale = a.scale_log2 * query_scale<T, D>(q);
      const bool one_scale = a.block >= NK;  // for all of a thread's keys of a tile
      float m = -INFINITY, l = 0.f;  // m: the reference, in log2 units
      float top = -INFINITY;         // the largest y so far
      const bool tighten = n >= 2 * kTightAt;
      for (int i = 0; i < n; ++i) {
        const int g = g0 + i;
        const int k0 = (cur.i0 + i) * kKeys;
        const bool masked = k0 + kKeys > lim_min;  // some of these keys are hidden from some rows
        const uint32_t tS = tmem + (uint32_t)(g & 1) * 128u + lane_off;
        const float now = scales;
        scales = fetch(i + 1);
        float fk[NG], ve[NG], vf[NG], vi[NG];
#pragma unroll
        for (int e = 0; e < NG; ++e) {
          if (e > 0 && one_scale) {
            fk[e] = fk[0], ve[e] = ve[0], vf[e] = vf[0], vi[e] = vi[0];
            continue;
          }
          fk[e] = __shfl_sync(0xffffffffu, now, e) * row_scale;
          split_scale(__shfl_sync(0xffffffffu, now, 4 + e), &ve[e], &vf[e], &vi[e]);
        }
        ok = ok && mbar_wait_bounded(s_full(g), (g >> 1) & 1, abort_flag, a.err);
        ok = __all_sync(0xffffffffu, ok);
        tc_fence_after();
        uint32_t hi[NK / 2], lo[NK / 2];
        if (works) {
          float2 y[NK / 2];
          float mx = -INFINITY;
          if (ok) {
            uint32_t s[NK];
#pragma unroll
            for (int c = 0; c < NK; c += 32)
              tmem_ld_32x32b_x32(tS + (uint32_t)(kofs + c), *reinterpret_cast<uint32_t(*)[32]>(s + c));
            tmem_ld_wait();
#pragma unroll
            for (int k = 0; k < NK / 2; ++k)
              y[k] = fma2(make_float2(__uint_as_float(s[2 * k]), __uint_as_float(s[2 * k + 1])), make_float2(fk[k / 8], fk[k / 8]),
                          make_float2(ve[k / 8], ve[k / 8]));
            if (masked) {
              const int seen = lim - k0 - kofs;
              const uint64_t see = seen >= 64 ? ~0ull : seen > 0 ? (1ull << seen) - 1ull : 0ull;
#pragma unroll
              for (int k = 0; k < NK / 2; ++k) {
                if (!(see >> (2 * k) & 1u)) y[k].x = -INFINITY;
                if (!(see >> (2 * k + 1) & 1u)) y[k].y = -INFINITY;
              }
#pragma unroll
              for (int e = 0; e < NG; ++e)
                if (seen <= 16 * e) vf[e] = 0.f;  // (whatever the scale of hidden rows is)
            }
            float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int k = 0; k < NK / 2; ++k) {
              mx4[(2 * k) & 3] = fmaxf(mx4[(2 * k) & 3], y[k].x);
              mx4[(2 * k + 1) & 3] = fmaxf(mx4[(2 * k + 1) & 3], y[k].y);
            }
            mx = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3]));
          }
          top = fmaxf(top, mx);
          const bool grow = mx - m > kMost || (tighten && i == kTightAt && top != -INFINITY);  // (also the first key seen)
          if (__any_sync(0xffffffffu, grow)) {
            float alpha = 1.f;
            if (grow) {
              const float ref = top - (tighten && i >= kTightAt ? kTight : kWide);
              alpha = ex2(m - ref);
              m = ref;
              l *= alpha;
            }
            if (i > 0) {  // O is at rest once the product of the tile before is done (the one before that is: these scores came after it)
              ok = ok && mbar_wait_bounded(o_full(half), (g - 1) & 1, abort_flag, a.err);
              ok = __all_sync(0xffffffffu, ok);
              tc_fence_after();
              if (ok) {
#pragma unroll 1  // (seldom run: short code, which the instruction cache has room beside the rest for)
                for (int c = 0; c < D; c += 16) {
                  uint32_t r[16];
                  tmem_ld_32x32b_x16(tO + (uint32_t)c, r);
                  tmem_ld_wait();
#pragma unroll
                  for (int e = 0; e < 16; ++e) r[e] = __float_as_uint(__uint_as_float(r[e]) * alpha);
                  tmem_st_x16(tO + (uint32_t)c, r);
                }
              }
            }
          }
          if (ok) {
            const float base = m == -INFINITY ? 0.f : m;
            const float2 base2 = make_float2(-base, -base), minus = make_float2(-1.f, -1.f);
            float2 sum2[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
            for (int k0 = 0; k0 < NK / 2; k0 += 8) {  // (step by step over eight pairs, a part of 16 keys: their latencies overlap)
              const float2 inv = make_float2(vi[k0 / 8], vi[k0 / 8]), frac = make_float2(vf[k0 / 8], vf[k0 / 8]);
              float2 p[8];
#pragma unroll
              for (int k = 0; k < 8; ++k) p[k] = add2(y[k0 + k], base2);
#pragma unroll
              for (int k = 0; k < 8; ++k) p[k] = make_float2(ex2(p[k].x), ex2(p[k].y));
#pragma unroll
              for (int k = 0; k < 8; ++k) sum2[k & 1] = fma2(p[k], inv, sum2[k & 1]);
#pragma unroll
              for (int k = 0; k < 8; ++k) p[k] = mul2(p[k], frac);
#pragma unroll
              for (int k = 0; k < 8; ++k) hi[k0 + k] = pack_pair<__half>(p[k].x, p[k].y);
#pragma unroll
              for (int k = 0; k < 8; ++k) p[k] = fma2(unpack_pair<__half>(hi[k0 + k]), minus, p[k]);
#pragma unroll
              for (int k = 0; k < 8; ++k) lo[k0 + k] = pack_pair<__half>(p[k].x, p[k].y);
            }
            l += (sum2[0].x + sum2[0].y) + (sum2[1].x + sum2[1].y);
          }
        }
        if (ok) {
          if (works) {
            // over the half's scores: hi parts of its keys, then the lo parts
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              const uint32_t* x = u ? lo : hi;
#pragma unroll
              for (int c = 0; c < 32; c += 16) {
                uint32_t w[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) w[e] = REP == 1 || (c + e) / (NK / 2) == rep ? x[(c + e) % (NK / 2)] : 0u;
                tmem_st_x16(tS + (uint32_t)(half * 64 + u * 32 + c), w);
              }
            }
            tmem_st_wait();
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(p_full(half, g));
        }
      }
      // ---- the piece's results: a thread joins the two halves of its row in
      // its share of the columns, and with REP 2 the row's two lanes meet in
      // shared memory
      ok = ok && mbar_wait_bounded(o_done, piece & 1, abort_flag, a.err);
      ok = __all_sync(0xffffffffu, ok);
      tc_fence_after();
      ml[half * 128 + slot] = make_float2(m, l);
      tc_fence_before();
      if (REP == 1) row_sync(); else all_sync();
      tc_fence_after();
      float M = -INFINITY, L = 0.f, f[2];
#pragma unroll
      for (int u = 0; u < 2 * REP; ++u) M = fmaxf(M, ml[u * kRowsMax + row].x);  // (half-major, then the copies of the rows)
      const float base = M == -INFINITY ? 0.f : M;
#pragma unroll
      for (int u = 0; u < 2 * REP; ++u) {
        const float2 x = ml[u * kRowsMax + row];
        L = fmaf(x.y, ex2(x.x - base), L);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) f[h] = ex2(ml[h * 128 + slot].x - base);  // 0 where no key was seen
      const float inv = L > 0.f ? 1.0f / L : (L == 0.f ? 0.f : L);  // (a NaN stays one)
      const bool writes = ok && row < rows && (REP == 1 || rep == 0);
      const int tq = t0 + row / a.group, hd = kvh * a.group + row % a.group;
      T* out = static_cast<T*>(a.out) + ((int64_t)b * a.tokens + tq) * a.out_stride + (int64_t)hd * D;
      const int64_t at = ((int64_t)2 * blockIdx.x + (cur.i0 == 0 ? 1 : 0)) * kRowsMax + row;
#pragma unroll 1
      for (int c = 0; c < D / 2; c += 32) {
        const int col = half * (D / 2) + c;
        float o[32];
        if (works) {
          uint32_t r[32];
          tmem_ld_32x32b_x32(tmem + kTmO + lane_off + (uint32_t)col, r);
          tmem_ld_wait();
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = __uint_as_float(r[e]) * f[0];
          tmem_ld_32x32b_x32(tmem + kTmO + 128u + lane_off + (uint32_t)col, r);
          tmem_ld_wait();
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = fmaf(__uint_as_float(r[e]), f[1], o[e]);
        }
        if (REP == 2) {
          float* stage = reinterpret_cast<float*>(smem + F::kOffStage) + (half * 64 + row) * 20;
#pragma unroll
          for (int c16 = 0; c16 < 32; c16 += 16) {
            if (rep == 1) {
#pragma unroll
              for (int e = 0; e < 16; e += 4)
                *reinterpret_cast<float4*>(stage + e) = make_float4(o[c16 + e], o[c16 + e + 1], o[c16 + e + 2], o[c16 + e + 3]);
            }
            copy_sync();
            if (rep == 0) {
#pragma unroll
              for (int e = 0; e < 16; e += 4) {
                const float4 x = *reinterpret_cast<const float4*>(stage + e);
                o[c16 + e] += x.x;
                o[c16 + e + 1] += x.y;
                o[c16 + e + 2] += x.z;
                o[c16 + e + 3] += x.w;
              }
            }
            copy_sync();
          }
        }
        if (!works || (REP == 2 && rep == 1)) continue;  // (the same for all lanes of a warp)
        if (whole) {
          uint4 v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e)
            v[e] = make_uint4(pack_pair<T>(o[8 * e] * inv, o[8 * e + 1] * inv), pack_pair<T>(o[8 * e + 2] * inv, o[8 * e + 3] * inv),
                              pack_pair<T>(o[8 * e + 4] * inv, o[8 * e + 5] * inv), pack_pair<T>(o[8 * e + 6] * inv, o[8 * e + 7] * inv));
          store_rows(v, reinterpret_cast<char*>(out + col), writes);
        } else {
          uint4 v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e)
            v[e] = make_uint4(__float_as_uint(o[4 * e]), __float_as_uint(o[4 * e + 1]), __float_as_uint(o[4 * e + 2]), __float_as_uint(o[4 * e + 3]));
          store_rows(v, reinterpret_cast<char*>(a.part + at * D + col), writes);
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0 && ok) mbar_arrive(o_free);
      if (writes && half == 0) {
        if (!whole)
          reinterpret_cast<float2*>(a.ml)[at] = make_float2(M, L);
        else if (a.lse)
          a.lse[((int64_t)b * a.heads + hd) * a.tokens + tq] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
      }
      if (a.splits != 1 && cur.i0 == 0 && aid == 0) record_unit(a, r_, cur, nrt, at_tile);
      at_tile += n;
      if (REP == 1) row_sync(); else all_sync();  // ml is written again
      g0 += n;
    }
    tc_fence_before();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, kTmemCols);
  }
}

int fail(cudaError_t e, const char* what) {
  if (e == cudaSuccess) e = cudaGetLastError();
  if (e != cudaSuccess) SN_FAIL(SWAPNET_ERR_CUDA, std::string(what) + ": " + cudaGetErrorString(e));
  return SWAPNET_OK;
}

template <typename T, int D, int CODE, int REP> int rows_t(const QuantArgs& a, int ctas, cudaStream_t s) {
  static std::atomic<uint64_t> known{0};
  const auto kern = attention_quant_rows_kernel<T, D, CODE, REP>;
  if (attr_needed(known)) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, QtCfg<D>::kSmem);
    if (e != cudaSuccess) return fail(e, "quantised attention: shared memory");
    attr_set(known);
  }
  const int queries = std::min(128 / REP / a.group, a.tokens), nrt = (a.tokens + queries - 1) / queries;
  CUtensorMap k, v;
  int rc = quant_maps(a, &k, &v, false);
  if (rc) return rc;
  kern<<<ctas, kQtThreads, QtCfg<D>::kSmem, s>>>(k, v, a, queries, nrt);
  rc = fail(cudaSuccess, "quantised attention launch");
  if (rc || a.splits == 1) return rc;
  return launch_quant_join(a, queries, 128 / REP, nrt, s);
}
template <typename T, int D, int CODE> int rows_r(const QuantArgs& a, int ctas, cudaStream_t s) {
  return a.tokens * a.group <= 64 ? rows_t<T, D, CODE, 2>(a, ctas, s) : rows_t<T, D, CODE, 1>(a, ctas, s);
}
template <typename T, int D> int rows_c(const QuantArgs& a, int ctas, cudaStream_t s) {
  return a.code == kCodeI8 ? rows_r<T, D, kCodeI8>(a, ctas, s) : rows_r<T, D, kCodeE4M3>(a, ctas, s);
}

}  // namespace

int launch_quant_rows(const QuantArgs& a, int ctas, cudaStream_t s) {
  if (a.dtype == SWAPNET_BF16) return a.dim == 128 ? rows_c<__nv_bfloat16, 128>(a, ctas, s) : rows_c<__nv_bfloat16, 64>(a, ctas, s);
  return a.dim == 128 ? rows_c<__half, 128>(a, ctas, s) : rows_c<__half, 64>(a, ctas, s);
}

}  // namespace swapnet
