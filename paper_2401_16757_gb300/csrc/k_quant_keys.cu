// Attention of units of up to 32 query rows per key head (short drafted runs,
// decode steps of wide groups, small calls) over a cache held in 8 bits, on the tcgen05 tensor cores
// with the keys as the rows of their products; fp32 arithmetic, fixed orders of
// summation.
//
// A tile of 128 keys has little to compute for 32 rows: 16 KB of keys and as
// many of values have to become fp16, whatever the rows.  With the rows as the
// products' rows (k_quant_tc.cu) three quarters of the products and of the softmax
// would be padding; on warp products (k_quant.cu) eight warps' registers are full.
//   S^T      [128 keys][32 rows] = K Q^T.  A thread turns the codes of one key
//            into fp16 and puts them straight into tensor memory, as the operand's
//            rows: keys pass through shared memory as bytes alone
//   p        two sets of four warps take a tile each in turn, with a reference m, a
//            sum l and an output O of their own.  A thread has one key: its scales
//            are its own and a mask is one number (which rows see the key).  m is
//            the set's, so a vote per tile tells whether some score is more than
//            2^14 above its row's m, which is set 2^7 below the largest then; only
//            then are m, l and O brought up to date (one tile in nine, beside a piece's
//            first two)
//   P        [128 keys][32 rows' high parts, 32 low parts] fp16, in shared memory:
//            both parts of a probability are columns of one product
//   O^T      [128 dims][64] += V^T P, V as it lies ([keys][dims], fp16, 128-byte
//            swizzle); the columns' halves are added at the end
// Scores are two tiles ahead of the products with the values.  Scales, queries,
// units, runs of tiles and their join as in the other kernels.
// Measured: 32 rows of 32 x 8 (sequence, key head)s on up to 8000 rows, E4M3 (0.34
// GB): 112 us, on warp products 131; 4 x 8 on up to 500 rows 12.5 and 18.3.  A tile
// takes about 2300 cycles; each of the programs of a CTA alone would take 1000 to
// 1300, but their instructions (4800 a tile) are issued at 0.4 a cycle and
// scheduler and wait for one another and for their caches.  Slower: all warps on
// one tile, 8 rows a thread (119), scores one tile ahead (117), twice the warps for
// the values (126), the conversion of keys unrolled (122; of values: 113 for 117),
// m at 2^5 below what the vote allows (119), the softmax eight rows at a time (113).
#include <algorithm>
#include <cstring>
#include <string>
#include <type_traits>

#include "internal.h"
#include "kernels.h"
#include "quant.cuh"

namespace swapnet {

namespace {

constexpr int kD = 128, kRows = 32;
// warpgroups: TMA (warp 0), MMA (warp 1), the units' records (warp 2); queries and
// keys to fp16; values; the softmax's two sets
constexpr int kQkThreads = 640, kSoftAt = 12;
constexpr int kRegsIssue = 56, kRegsConv = 80, kRegsSoft = 128;
static_assert(128 * kRegsIssue + 256 * kRegsConv + 256 * kRegsSoft <= kQkThreads * 96, "registers of a CTA");
constexpr float kMost = kTop, kWide = 7.0f;  // log2 of p: at most; of the largest where m is set
constexpr int kRaw = 128 * kD;               // bytes of a tile's codes
constexpr int kKeySlots = 4, kValueSlots = 3;
constexpr int kOffKeys = 0, kOffValues = kOffKeys + kKeySlots * kRaw;
constexpr int kOffV = kOffValues + kValueSlots * kRaw;  // two fp16 tiles
constexpr int kOffP = kOffV + 2 * 2 * kRaw;             // two
constexpr int kOffQ = kOffP + 2 * kRaw;
constexpr int kOffQs = kOffQ + kRows * kD * 2;          // scales of four pieces' queries
constexpr int kOffTop = kOffQs + 4 * kRows * 4;         // largest scores, [set][4 warps][row]
constexpr int kOffUp = kOffTop + 2 * 4 * kRows * 4;     // what -m grows by, [set][row]
constexpr int kOffM = kOffUp + 2 * kRows * 4;           // -m, [piece & 1][set][row]
constexpr int kOffSum = kOffM + 4 * kRows * 4;          // [piece & 1][set][4 warps][row]
constexpr int kOffBar = kOffSum + 4 * 4 * kRows * 4;
constexpr int kOffNear = kOffBar + 320;
constexpr int kQkSmem = kOffNear + kNear * 8 + 1024;  // + alignment slack
static_assert(kQkSmem <= 232448, "shared memory of a CTA");
// Tensor memory: two tiles of keys, four of scores, O of each set
constexpr uint32_t kTmemK = 0, kTmemS = 128, kTmemO = 256, kTmemCols = 512;

template <typename T> __device__ __forceinline__ T narrow(float x) {
  if constexpr (std::is_same<T, __half>::value) return __float2half_rn(x);
  else return __float2bfloat16_rn(x);
}
// Of 32 numbers per lane, over all lanes: lane r gets that of number r.
template <typename Op> __device__ __forceinline__ float reduce32(float (&v)[32], Op op) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int n = 16; n > 0; n >>= 1) {
    const bool up = lane & n;
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const float mine = up ? v[i + n] : v[i], other = up ? v[i] : v[i + n];
      v[i] = op(mine, __shfl_xor_sync(0xffffffffu, other, n));
    }
  }
  return v[0];
}
__device__ __forceinline__ void tmem_ld_x8(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr)
               : "memory");
}

template <typename T, int CODE>
__global__ void __launch_bounds__(kQkThreads, 1)
    attention_quant_keys_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                                const __grid_constant__ QuantArgs a, int queries, int nrt) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + kOffBar);
  auto key_full = [&](int s) { return smem_u32(bars + s); };  // a tile's codes
  auto key_empty = [&](int s) { return smem_u32(bars + 4 + s); };
  auto value_full = [&](int s) { return smem_u32(bars + 8 + s); };
  auto value_empty = [&](int s) { return smem_u32(bars + 12 + s); };
  auto k_full = [&](int g) { return smem_u32(bars + 16 + (g & 1)); };  // and their fp16
  auto k_free = [&](int g) { return smem_u32(bars + 18 + (g & 1)); };
  auto v_full = [&](int g) { return smem_u32(bars + 20 + (g & 1)); };
  auto s_full = [&](int g) { return smem_u32(bars + 32 + (g & 3)); };
  auto p_full = [&](int g) { return smem_u32(bars + 24 + (g & 1)); };
  auto pv_done = [&](int g) { return smem_u32(bars + 26 + (g & 1)); };  // its V and P are free, O at rest
  const uint32_t q_full = smem_u32(bars + 28), q_free = smem_u32(bars + 29);  // a piece's queries
  const uint32_t o_free = smem_u32(bars + 30), done_bar = smem_u32(bars + 31);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 36);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int2* near = reinterpret_cast<int2*>(smem + kOffNear);
  int64_t* sched = reinterpret_cast<int64_t*>(smem + kOffTop);  // (before the first results)
  float* q_scales = reinterpret_cast<float*>(smem + kOffQs);

  const int warp = warp_index(), lane = threadIdx.x & 31, q4 = warp & 3;
  if (threadIdx.x == 0) {
    for (int s = 0; s < kKeySlots; ++s) {
      mbar_init(key_full(s), 1);
      mbar_init(key_empty(s), 4);
    }
    for (int s = 0; s < kValueSlots; ++s) {
      mbar_init(value_full(s), 1);
      mbar_init(value_empty(s), 4);
    }
    for (int g = 0; g < 2; ++g) {
      mbar_init(k_full(g), 4);
      mbar_init(k_free(g), 1);
      mbar_init(v_full(g), 4);
      mbar_init(p_full(g), 4);
      mbar_init(pv_done(g), 1);
    }
    for (int g = 0; g < 4; ++g) mbar_init(s_full(g), 1);
    mbar_init(q_full, 4);
    mbar_init(q_free, 1);
    mbar_init(o_free, 8);
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
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_launch_dependents();  // (not before this CTA has its TMEM)
  const uint32_t lane_off = (uint32_t)(q4 * 32) << 16;

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsIssue));
    if (warp == 0 && elect_one()) {
      // ---------------- TMA producer: the tiles' codes
      int g = 0;
      bool ok = true;
      while (ok && cur.step(a, nrt, queries))
#pragma unroll 1
        for (int i = 0; ok && i < cur.n; ++i, ++g) {
          const int ks = g % kKeySlots, vs = g % kValueSlots, y = (cur.i0 + i) * kKeys;
          if (g >= kKeySlots && !(ok = mbar_wait_bounded(key_empty(ks), ((g / kKeySlots) - 1) & 1, abort_flag, a.err))) break;
          mbar_arrive_expect_tx(key_full(ks), kRaw);
          tma_load_3d(smem_u32(smem + kOffKeys + ks * kRaw), &tmK, key_full(ks), kvh * kD, y, cur.b);
          if (g >= kValueSlots && !(ok = mbar_wait_bounded(value_empty(vs), ((g / kValueSlots) - 1) & 1, abort_flag, a.err))) {
            // (the keys' load lands before the CTA can exit)
            volatile int no_abort = 0;
            mbar_wait_bounded(key_full(ks), (g / kKeySlots) & 1, &no_abort, nullptr);
            break;
          }
          mbar_arrive_expect_tx(value_full(vs), kRaw);
          tma_load_3d(smem_u32(smem + kOffValues + vs * kRaw), &tmV, value_full(vs), kvh * kD, y, cur.b);
        }
      // let every load issued land before the CTA can exit
      volatile int no_abort = 0;
      for (int j = max(0, g - kKeySlots); j < g; ++j) mbar_wait_bounded(key_full(j % kKeySlots), (j / kKeySlots) & 1, &no_abort, nullptr);
      for (int j = max(0, g - kValueSlots); j < g; ++j) mbar_wait_bounded(value_full(j % kValueSlots), (j / kValueSlots) & 1, &no_abort, nullptr);
    }
    if (warp == 2 && a.splits != 1 && elect_one()) {
      // ---------------- the units' records
      int64_t at_tile = r_.first;
      while (cur.step(a, nrt, queries)) {
        if (cur.i0 == 0) record_unit(a, r_, cur, nrt, at_tile);
        at_tile += cur.n;
      }
    }
    if (warp == 1 && elect_one()) {
      // ---------------- MMA issuer: the scores of a tile before the product of the one two before
      constexpr uint32_t idesc_s = idesc_f16(0, 128, kRows);
      constexpr uint32_t idesc_pv = idesc_f16(0, kD, 2 * kRows) | (1u << 15) | (1u << 16);  // A (values) and B (P) MN-major
      const uint64_t qd = smem_desc_sw128(smem_u32(smem + kOffQ));
      const uint64_t vd = desc_mn(smem_u32(smem + kOffV)), pd = desc_mn(smem_u32(smem + kOffP));
      bool ok = true;
      auto wait = [&](uint32_t bar, uint32_t parity) { return ok = ok && mbar_wait_bounded(bar, parity, abort_flag, a.err); };
      int i = 0, n = 0, piece = -1;
      bool keys = true;
      int at[2] = {-1, -1}, of[2] = {0, 0};  // the last two tiles: place in its piece (-1: none), piece
#pragma unroll 1
      for (int g = 0; ok; ++g, ++i) {
        if (i == n) {
          keys = keys && cur.step(a, nrt, queries);
          i = 0;
          n = keys ? cur.n : 0;
          ++piece;
        }
        if (keys) {
          if (i == 0 && !wait(q_full, piece & 1)) break;
          if (!wait(k_full(g), (g >> 1) & 1)) break;
          // (over the scores of four tiles ago: their P, which a product issued
          // before this has waited for, was made from them)
          tc_fence_after();
#pragma unroll
          for (int k = 0; k < 8; ++k)  // 16 dims a step
            tc_mma_f16_ta(tmem + kTmemS + (uint32_t)(g & 3) * kRows, tmem + kTmemK + (uint32_t)(g & 1) * 64u + (uint32_t)k * 8u,
                          qd + (uint64_t)((k >> 2) * (kRows * 128 >> 4) + 2 * (k & 3)), idesc_s, k != 0);
          tc_commit(s_full(g));
          tc_commit(k_free(g));
          if (i == n - 1) tc_commit(q_free);
        }
        if (at[0] >= 0) {
          const int j = g - 2;
          if (at[0] == 0 && of[0] > 0 && !wait(o_free, (of[0] - 1) & 1)) break;
          if (!wait(v_full(j), (j >> 1) & 1) || !wait(p_full(j), (j >> 1) & 1)) break;
          tc_fence_after();
#pragma unroll
          for (int k = 0; k < 8; ++k)  // 16 keys a step
            tc_mma_f16(tmem + kTmemO + (uint32_t)(j & 1) * (2 * kRows), vd + (uint64_t)((j & 1) * (2 * kRaw >> 4) + k * (2048 >> 4)),
                       pd + (uint64_t)((j & 1) * (kRaw >> 4) + k * (2048 >> 4)), idesc_pv, at[0] > 1 || k != 0);
          tc_commit(pv_done(j));
        }
        if (!keys && at[1] < 0) break;
        at[0] = at[1];
        of[0] = of[1];
        at[1] = keys ? i : -1;
        of[1] = piece;
        if (!keys) i = n - 1;  // (no more tiles)
      }
      // every MMA issued must have finished before TMEM is freed
      tc_commit(done_bar);
      volatile int no_abort = 0;
      mbar_wait_bounded(done_bar, 0, &no_abort, nullptr);
    }
  } else if (warp < 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsConv));
    // ---------------- queries and keys to fp16
    const int ct = threadIdx.x - 128;  // its key of a tile
    bool ok = true;
    int g = 0;
    for (int piece = 0; ok && cur.step(a, nrt, queries); ++piece) {
      ok = piece == 0 || mbar_wait_bounded(q_free, (piece - 1) & 1, abort_flag, a.err);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      {  // 16 lanes a row
        const int t0 = cur.rt * queries, rows = min(queries, cur.z.count - t0) * a.group, c = ct & 15;
        uint4 v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int row = u * 8 + (ct >> 4);
          v[u] = make_uint4(0u, 0u, 0u, 0u);
          if (row < rows)
            v[u] = reinterpret_cast<const uint4*>(static_cast<const T*>(a.q) + ((int64_t)cur.b * a.tokens + t0 + row / a.group) * a.q_stride +
                                                  (int64_t)(kvh * a.group + row % a.group) * kD)[c];
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int row = u * 8 + (ct >> 4);
          float scale = 1.0f;
          if (!std::is_same<T, __half>::value) {
            uint32_t most = largest_bits(v[u]);
#pragma unroll
            for (int off = 8; off > 0; off >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, off));
            const int x = query_exponent(most);
            const float by = __uint_as_float((uint32_t)(127 + 14 - (x - 127)) << 23);
            scale = __uint_as_float((uint32_t)(x - 14) << 23);
            v[u] = make_uint4(query_pair(v[u].x, by), query_pair(v[u].y, by), query_pair(v[u].z, by), query_pair(v[u].w, by));
          }
          if (c == 0) q_scales[(piece & 3) * kRows + row] = scale * a.scale_log2;
          *reinterpret_cast<uint4*>(smem + kOffQ + (c >> 3) * (kRows * 128) + row * 128 + (((c & 7) ^ (row & 7)) << 4)) = v[u];
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(q_full);
      }
#pragma unroll 1
      for (int i = 0; i < cur.n; ++i, ++g) {
        const int s = g % kKeySlots;
        ok = ok && mbar_wait_bounded(key_full(s), (g / kKeySlots) & 1, abort_flag, a.err);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        const uint8_t* raw = smem + kOffKeys + s * kRaw + ct * 128;
        ok = g < 2 || mbar_wait_bounded(k_free(g), ((g >> 1) - 1) & 1, abort_flag, a.err);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        tc_fence_after();
#pragma unroll 1  // (short code)
        for (int c = 0; c < 8; c += 2) {
          uint32_t w[16];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint4 x = *reinterpret_cast<const uint4*>(raw + (((c + e) ^ (ct & 7)) << 4));
            const uint2 w0 = pairs_near<CODE>(x.x), w1 = pairs_near<CODE>(x.y), w2 = pairs_near<CODE>(x.z), w3 = pairs_near<CODE>(x.w);
            w[8 * e] = w0.x, w[8 * e + 1] = w0.y, w[8 * e + 2] = w1.x, w[8 * e + 3] = w1.y;
            w[8 * e + 4] = w2.x, w[8 * e + 5] = w2.y, w[8 * e + 6] = w3.x, w[8 * e + 7] = w3.y;
          }
          tmem_st_x16(tmem + kTmemK + lane_off + (uint32_t)(g & 1) * 64u + (uint32_t)c * 8u, w);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(key_empty(s));
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(k_full(g));
      }
    }
  } else if (warp < kSoftAt) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsConv));
    // ---------------- values to fp16
    // 16 codes a time: four lanes read 64 bytes of a row, their neighbours the
    // other 64 of the next, so that neither the reads nor the swizzled stores
    // meet in a bank
    const int ct = threadIdx.x - 256, r0 = ct >> 2;
    uint32_t from[2], to[2][2];  // of this thread's first chunks: in the codes, in the fp16 tile
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int c = (ct & 3) + 4 * ((r0 & 1) ^ u);
      from[u] = r0 * kD + c * 16;
#pragma unroll
      for (int e = 0; e < 2; ++e) to[u][e] = (c >> 2) * kRaw + r0 * 128 + ((((c & 3) * 2 + e) ^ (r0 & 7)) << 4);
    }
    bool ok = true;
    int g = 0;
    while (ok && cur.step(a, nrt, queries)) {
      const int lim0 = visible_limit(a, cur.z.len, cur.z.count, cur.rt * queries);
#pragma unroll 1
      for (int i = 0; i < cur.n; ++i, ++g) {
        const int s = g % kValueSlots;
        ok = ok && mbar_wait_bounded(value_full(s), (g / kValueSlots) & 1, abort_flag, a.err);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        const uint8_t* raw = smem + kOffValues + s * kRaw;
        uint8_t* tile = smem + kOffV + (g & 1) * 2 * kRaw;
        const bool clean = CODE == kCodeE4M3 && (cur.i0 + i + 1) * kKeys > lim0;  // some rows are hidden from some queries
        ok = g < 2 || mbar_wait_bounded(pv_done(g), ((g >> 1) - 1) & 1, abort_flag, a.err);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
#pragma unroll
        for (int r = 0; r < 4; r += 2) {
          uint4 v[2][2];  // (read before the first store, which might be to the same memory for what the compiler knows)
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int u = 0; u < 2; ++u) v[e][u] = *reinterpret_cast<const uint4*>(raw + (r + e) * 32 * kD + from[u]);
          if (clean) {
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
              for (int u = 0; u < 2; ++u)
                v[e][u] = make_uint4(numbers_only(v[e][u].x), numbers_only(v[e][u].y), numbers_only(v[e][u].z), numbers_only(v[e][u].w));
          }
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              const uint2 x = pairs_near<CODE>(v[e][u].x), y = pairs_near<CODE>(v[e][u].y), z = pairs_near<CODE>(v[e][u].z),
                          w = pairs_near<CODE>(v[e][u].w);
              *reinterpret_cast<uint4*>(tile + (r + e) * 32 * 128 + to[u][0]) = make_uint4(x.x, x.y, y.x, y.y);
              *reinterpret_cast<uint4*>(tile + (r + e) * 32 * 128 + to[u][1]) = make_uint4(z.x, z.y, w.x, w.y);
            }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(value_empty(s));
        fence_proxy_async_smem();  // the tiles are read by the tensor cores (async proxy)
        __syncwarp();
        if (lane == 0) mbar_arrive(v_full(g));
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoft));
    // ---------------- softmax and output: a thread has a key of its set's tiles
    const int set = (warp - kSoftAt) >> 2, mine = q4 * 32 + lane;
    float* tops = reinterpret_cast<float*>(smem + kOffTop) + set * 4 * kRows;
    float* ups = reinterpret_cast<float*>(smem + kOffUp) + set * kRows;
    const uint32_t tO = tmem + kTmemO + lane_off;
    uint8_t* to = smem + kOffP + set * kRaw + mine * 128;
    auto set_sync = [&]() { asm volatile("bar.sync %0, 128;" ::"r"(1 + set) : "memory"); };
    auto set_any = [&](bool x) -> bool {
      uint32_t r;
      asm volatile(
          "{\n\t.reg .pred p, q;\n\t"
          "setp.ne.u32 p, %2, 0;\n\t"
          "bar.red.or.pred q, %1, 128, p;\n\t"
          "selp.u32 %0, 1, 0, q;\n\t}"
          : "=r"(r)
          : "r"(1 + set), "r"((uint32_t)x)
          : "memory");
      return r != 0;
    };
    bool ok = true;
    int g0 = 0;
    for (int piece = 0; cur.step(a, nrt, queries); ++piece) {
      const int b = cur.b, n = cur.n, count = cur.z.count, len = cur.z.len;
      const int t0 = cur.rt * queries, rows = min(queries, count - t0) * a.group;
      const bool whole = cur.i0 == 0 && n == cur.z.tiles;
      const int lim0 = len - count + t0 + 1;  // keys the first query sees (none: may be below 0)
      const int64_t scale_at = ((int64_t)b * a.kv_heads + kvh) * a.blocks;
      const float *key_scales = a.k_scale + scale_at, *value_scales = a.v_scale + scale_at;
      const int first = (g0 ^ set) & 1;  // the set's first tile
      auto block_of = [&](int i) {
        const int j = (cur.i0 + i) * kKeys + mine;
        return i < n && j < len ? j >> a.block_log2 : -1;
      };
      int block = block_of(first);
      float ks = block >= 0 ? key_scales[block] : 1.0f, vs = block >= 0 ? value_scales[block] : 1.0f;
      float* minus_ms = reinterpret_cast<float*>(smem + kOffM) + ((piece & 1) * 2 + set) * kRows;
      const float4* qs = reinterpret_cast<const float4*>(q_scales + (piece & 3) * kRows);
      float2 l2[16];
#pragma unroll
      for (int k = 0; k < 16; ++k) l2[k] = make_float2(0.f, 0.f);
#pragma unroll 1
      for (int i = first; i < n; i += 2) {
        const int g = g0 + i, k0 = (cur.i0 + i) * kKeys;
        const bool masked = k0 + kKeys > lim0;  // some of the tile's keys are hidden from some rows
        const int hidden = a.group * (k0 + mine - lim0 + 1);  // the rows before this one do not see the key
        const float k_scale = ks;
        float ve, vf, vi;
        split_scale(vs, &ve, &vf, &vi);
        block = block_of(i + 2);
        if (block >= 0) ks = key_scales[block], vs = value_scales[block];
        ok = ok && mbar_wait_bounded(s_full(g), (g >> 2) & 1, abort_flag, a.err);
        ok = __all_sync(0xffffffffu, ok);
        tc_fence_after();
        float2 y[16];
        {
          uint32_t s[32];
          tmem_ld_32x32b_x32(tmem + kTmemS + lane_off + (uint32_t)(g & 3) * kRows, s);
          tmem_ld_wait();
          const float2 by = make_float2(k_scale, k_scale), e = make_float2(ve, ve);
#pragma unroll
          for (int k = 0; k < 16; k += 2) {  // (the queries' scales have been there before the scores)
            const float4 q = qs[k / 2];
            y[k] = fma2(make_float2(__uint_as_float(s[2 * k]), __uint_as_float(s[2 * k + 1])), mul2(make_float2(q.x, q.y), by), e);
            y[k + 1] = fma2(make_float2(__uint_as_float(s[2 * k + 2]), __uint_as_float(s[2 * k + 3])), mul2(make_float2(q.z, q.w), by), e);
          }
        }
        if (masked) {
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            if (2 * k < hidden) y[k].x = -INFINITY;
            if (2 * k + 1 < hidden) y[k].y = -INFINITY;
          }
        }
        bool grow = i == first;
        if (!grow) {  // y - m from here on
          float most = -INFINITY;
#pragma unroll
          for (int k = 0; k < 16; k += 2) {
            const float4 x = reinterpret_cast<const float4*>(minus_ms)[k / 2];
            y[k] = add2(y[k], make_float2(x.x, x.y));
            y[k + 1] = add2(y[k + 1], make_float2(x.z, x.w));
            most = fmaxf(most, fmaxf(fmaxf(y[k].x, y[k].y), fmaxf(y[k + 1].x, y[k + 1].y)));
          }
          grow = set_any(ok && most > kMost);
        }
        if (i != first) {  // the set's product before: O is at rest, P's place free
          ok = ok && mbar_wait_bounded(pv_done(g), ((g >> 1) - 1) & 1, abort_flag, a.err);
          ok = __all_sync(0xffffffffu, ok);
          tc_fence_after();
        }
        if (grow) {  // lane r for row r
          float top[32];
#pragma unroll
          for (int k = 0; k < 16; ++k) top[2 * k] = y[k].x, top[2 * k + 1] = y[k].y;
          tops[q4 * kRows + lane] = reduce32(top, [](float u, float v) { return fmaxf(u, v); });
          set_sync();
          if (q4 == 0) {
            float most = tops[lane];
#pragma unroll
            for (int w = 1; w < 4; ++w) most = fmaxf(most, tops[w * kRows + lane]);
            const float up = (i == first ? most > -INFINITY : most > kMost) ? kWide - most : 0.f;
            minus_ms[lane] = i == first ? up : minus_ms[lane] + up;
            ups[lane] = up;
          }
          set_sync();
#pragma unroll
          for (int k = 0; k < 16; k += 2) {
            const float4 x = reinterpret_cast<const float4*>(ups)[k / 2];
            y[k] = add2(y[k], make_float2(x.x, x.y));
            y[k + 1] = add2(y[k + 1], make_float2(x.z, x.w));
            if (i == first) continue;  // (no sums yet, and 2^up may be infinite)
            l2[k] = mul2(l2[k], make_float2(ex2(x.x), ex2(x.y)));
            l2[k + 1] = mul2(l2[k + 1], make_float2(ex2(x.z), ex2(x.w)));
          }
          if (i != first && ok) {
#pragma unroll 1
            for (int c = 0; c < 2 * kRows; c += 16) {
              uint32_t o[16];
              tmem_ld_32x32b_x16(tO + (uint32_t)(set * 2 * kRows + c), o);
              tmem_ld_wait();
#pragma unroll
              for (int r = 0; r < 16; ++r) o[r] = __float_as_uint(__uint_as_float(o[r]) * ex2(ups[(c & 16) + r]));
              tmem_st_x16(tO + (uint32_t)(set * 2 * kRows + c), o);
            }
            tmem_st_wait();
          }
          set_sync();  // (before what has been read here is written again)
        }
        if (ok) {
          const float2 inv = make_float2(vi, vi), frac = make_float2(vf, vf), minus = make_float2(-1.f, -1.f);
#pragma unroll
          for (int c = 0; c < 2; ++c) {  // sixteen rows
            float2 z[8];
            uint32_t hi[8], lo[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) z[k] = make_float2(ex2(y[8 * c + k].x), ex2(y[8 * c + k].y));
#pragma unroll
            for (int k = 0; k < 8; ++k) l2[8 * c + k] = fma2(z[k], inv, l2[8 * c + k]);
#pragma unroll
            for (int k = 0; k < 8; ++k) z[k] = mul2(z[k], frac);
            if (masked) {  // (whatever the scale of hidden rows is)
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                if (16 * c + 2 * k < hidden) z[k].x = 0.f;
                if (16 * c + 2 * k + 1 < hidden) z[k].y = 0.f;
              }
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) hi[k] = pack_pair<__half>(z[k].x, z[k].y);
#pragma unroll
            for (int k = 0; k < 8; ++k) z[k] = fma2(unpack_pair<__half>(hi[k]), minus, z[k]);
#pragma unroll
            for (int k = 0; k < 8; ++k) lo[k] = pack_pair<__half>(z[k].x, z[k].y);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              *reinterpret_cast<uint4*>(to + (((2 * c + u) ^ (mine & 7)) << 4)) = make_uint4(hi[4 * u], hi[4 * u + 1], hi[4 * u + 2], hi[4 * u + 3]);
              *reinterpret_cast<uint4*>(to + (((4 + 2 * c + u) ^ (mine & 7)) << 4)) = make_uint4(lo[4 * u], lo[4 * u + 1], lo[4 * u + 2], lo[4 * u + 3]);
            }
          }
          fence_proxy_async_smem();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(p_full(g));
        }
      }
      // ---- the piece's results: the sets meet; lane r has the sums of row r, a
      // thread the outputs of a dim, 16 rows of both sets
      float* sums = reinterpret_cast<float*>(smem + kOffSum) + (piece & 1) * 8 * kRows;
      {
        float x[32];
#pragma unroll
        for (int k = 0; k < 16; ++k) x[2 * k] = l2[k].x, x[2 * k + 1] = l2[k].y;
        sums[(set * 4 + q4) * kRows + lane] = reduce32(x, [](float u, float v) { return u + v; });
      }
      // a set waits for its own products alone (a wait for a phase of the other
      // set's barrier would return at once while the phase before is open) and
      // learns of the other's at the barrier, with a fence on either side
      const int done = g0 + n - 1 - ((n - 1 - first) & 1);  // the set's last tile, if it has one
      if (done >= g0 + first) ok = ok && mbar_wait_bounded(pv_done(done), (done >> 1) & 1, abort_flag, a.err);
      ok = __all_sync(0xffffffffu, ok);
      tc_fence_after();
      tc_fence_before();
      asm volatile("bar.sync 3, 256;" ::: "memory");
      tc_fence_after();
      float f[2], own[2], M = -INFINITY, L = 0.f;
      const float* minus_m = reinterpret_cast<const float*>(smem + kOffM) + (piece & 1) * 2 * kRows + lane;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const float* x = sums + u * 4 * kRows + lane;
        own[u] = (x[0] + x[kRows]) + (x[2 * kRows] + x[3 * kRows]);
        f[u] = own[u] == 0.f ? -INFINITY : -minus_m[u * kRows];  // (0: nothing seen, maybe no tile and no m)
        M = fmaxf(M, f[u]);
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        f[u] = f[u] == -INFINITY ? 0.f : ex2(f[u] - M);
        L = fmaf(own[u], f[u], L);
      }
      const float inv = L > 0.f ? 1.0f / L : (L == 0.f ? 0.f : L);  // (a NaN stays one)
      const int64_t part = ((int64_t)2 * blockIdx.x + (cur.i0 == 0 ? 1 : 0)) * kRows;
      if (ok && set == 0 && q4 == 0 && lane < rows) {
        if (!whole)
          reinterpret_cast<float2*>(a.ml)[part + lane] = make_float2(M, L);
        else if (a.lse)
          a.lse[((int64_t)b * a.heads + kvh * a.group + lane % a.group) * a.tokens + t0 + lane / a.group] =
              L == 0.f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
      }
      int t = t0 + set * 16 / a.group, h = set * 16 % a.group;
#pragma unroll 1
      for (int c = set * 16; c < set * 16 + 16; c += 8) {
        float o[8];
        {
          uint32_t u[8], v[8];
          tmem_ld_x8(tO + (uint32_t)c, u);
          tmem_ld_x8(tO + (uint32_t)(c + kRows), v);
          tmem_ld_wait();
#pragma unroll
          for (int r = 0; r < 8; ++r) {
            const float by = __shfl_sync(0xffffffffu, f[0], c + r);
            o[r] = by == 0.f ? 0.f : (__uint_as_float(u[r]) + __uint_as_float(v[r])) * by;  // (a set without a tile has no O)
          }
          tmem_ld_x8(tO + (uint32_t)(c + 2 * kRows), u);
          tmem_ld_x8(tO + (uint32_t)(c + 3 * kRows), v);
          tmem_ld_wait();
#pragma unroll
          for (int r = 0; r < 8; ++r) {
            const float by = __shfl_sync(0xffffffffu, f[1], c + r);
            if (by != 0.f) o[r] = fmaf(__uint_as_float(u[r]) + __uint_as_float(v[r]), by, o[r]);
          }
        }
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          const float by = __shfl_sync(0xffffffffu, inv, c + r);
          if (ok && c + r < rows) {
            if (whole)
              static_cast<T*>(a.out)[((int64_t)b * a.tokens + t) * a.out_stride + (int64_t)(kvh * a.group + h) * kD + mine] = narrow<T>(o[r] * by);
            else
              a.part[(part + c + r) * kD + mine] = o[r];
          }
          if (++h == a.group) h = 0, ++t;
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0 && ok) mbar_arrive(o_free);
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

template <typename T, int CODE> int keys_t(const QuantArgs& a, int ctas, cudaStream_t s) {
  static std::atomic<uint64_t> known{0};
  const auto kern = attention_quant_keys_kernel<T, CODE>;
  if (attr_needed(known)) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kQkSmem);
    if (e != cudaSuccess) SN_FAIL(SWAPNET_ERR_CUDA, std::string("quantised attention: ") + cudaGetErrorString(e));
    attr_set(known);
  }
  const int queries = std::min(kRows / a.group, a.tokens), nrt = (a.tokens + queries - 1) / queries;
  CUtensorMap k, v;
  if (int rc = quant_maps(a, &k, &v, true)) return rc;
  kern<<<ctas, kQkThreads, kQkSmem, s>>>(k, v, a, queries, nrt);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) SN_FAIL(SWAPNET_ERR_CUDA, std::string("quantised attention launch: ") + cudaGetErrorString(e));
  return a.splits == 1 ? SWAPNET_OK : launch_quant_join(a, queries, kRows, nrt, s);
}

}  // namespace

int launch_quant_keys(const QuantArgs& a, int ctas, cudaStream_t s) {
  if (a.dtype == SWAPNET_BF16)
    return a.code == kCodeI8 ? keys_t<__nv_bfloat16, kCodeI8>(a, ctas, s) : keys_t<__nv_bfloat16, kCodeE4M3>(a, ctas, s);
  return a.code == kCodeI8 ? keys_t<__half, kCodeI8>(a, ctas, s) : keys_t<__half, kCodeE4M3>(a, ctas, s);
}

}  // namespace swapnet
