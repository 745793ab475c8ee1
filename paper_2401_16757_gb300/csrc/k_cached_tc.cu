// Attention of many query rows (wide drafted trees, runs of a prompt) over a
// key-value cache on the tcgen05 tensor cores; fp16 / bf16 storage, fp32
// arithmetic.
//
// Rows of a (sequence, key head) are its queries times the heads that share
// the key head, query-major: row t * group + h.  A unit is up to 128 of them;
// one CTA per SM takes units, or an equal run of all units' key tiles (128 keys
// each; the drafted nodes are one more tile, the last), whatever the
// sequences' lengths.  Per tile:
//   S = Q K^T     tcgen05.mma, M 128 (rows) x N 64 (keys), twice; Q, K and V by
//                 TMA (128-byte swizzle); S in two TMEM buffers, so that the
//                 next tile's S is computed during this tile's softmax
//   P             warps 4..11, two threads per row: the first 64 keys of every
//                 tile and the last 64 have a softmax of their own (reference m,
//                 sum l, output O_h), so that no thread asks another for
//                 anything.  Scores from TMEM, masks only in tiles that a limit
//                 crosses, p = 2^(s - m) back over the scores as two parts of
//                 the storage type, p_hi + p_lo: one part would leave 8 (bf16)
//                 or 11 (fp16) bits of p, less than the fp32 that the sums keep;
//                 two leave 17 (bf16) or 22 (fp16, down to its least step, see
//                 PRange), for a second product with V, whose tensor time is
//                 hidden behind the exponentials.  A third part has no room:
//                 TMEM is full with two tiles' scores and both outputs
//   O_h += P_h V  tcgen05.mma with A = P from TMEM, B = V as loaded (MN-major)
// O_0 and O_1 stay in TMEM.  m, the running maximum less a constant, is taken
// again only where p would pass 2^8 (bf16) or 2^15 (fp16): until then O is
// neither read nor rescaled, and fp32 holds the sums without loss (PRange: what
// the parts of p hold).
// With at most 64 rows (REP 2) the rows appear twice in the MMA's 128, and
// lanes 0..63 and 64..127 share a thread's keys, so that all warps work (the
// other 16 keys are zeros in a lane's P).
// K and V tiles pass through one ring in the order they are used, across
// units.  Every wait is bounded: on timeout the kernel records kDevErrTimeout,
// drains the loads and MMAs it started, frees TMEM and returns.
//
// Measured, caches larger than L2: 32 sequences x 8 key heads (group 4) of 128
// wide bf16 heads on up to 8000 rows (0.72 GB): 16 nodes 122 us, 5.9 TB/s; 24
// nodes 129, 5.6; 64 nodes 228 and 128 nodes 390, 0.62 and 0.75 PFLOP/s (the
// second product of P not counted).  1000 queries on 4096 rows, 2 sequences x 32
// heads, f16: 124 us, 0.72 PFLOP/s.  One sequence of 131001 rows, 4 key heads of
// 64 wide f16, 52 rows: 42 us, of which the join and a unit's start and end are
// 15.  32 heads x 64 nodes on 511 rows: 13.0 us.
// Up to about 100 rows per unit DRAM bounds it, beyond that the softmax warps: a
// tile of 128 x 128 takes them about 2500 cycles (1265 for exponentials and the
// two parts of P, 350 for the maximum, 320 to store P, 170 to load S, the rest
// waits), two warps per scheduler, which issue in 0.43 of the cycles.  Four
// threads per row (16 warps of 104 registers) were slower: 32 keys per thread
// leave few independent exponentials, and the two threads of a half have to
// agree on the maximum.  One softmax for all 128 keys of a row, its two threads
// exchanging maxima, took 182 us where a softmax per half took 163 (24 nodes, as
// above, in an earlier form).
#include <algorithm>
#include <cstring>
#include <string>
#include <type_traits>

#include "cached.cuh"
#include "internal.h"
#include "kernels.h"

namespace swapnet {

namespace {

constexpr int kSoftThreads = 256;
constexpr int kTcThreads = 64 + kSoftThreads;  // weights: TMA, MMA, sums
// attention: warps 0 (TMA) and 1 (MMA), two idle ones that complete their
// warpgroup, the softmax's 8; 384 x 168 registers at launch, of which
// setmaxnreg leaves 128 x 72 and gives 256 x 216
constexpr int kAtThreads = 128 + kSoftThreads;
constexpr int kRegsLow = 72, kRegsHigh = 216;
static_assert(128 * kRegsLow + kSoftThreads * kRegsHigh <= kAtThreads * 168, "registers of a CTA");
constexpr int kKeys = 128;       // keys of a tile
// Where p lies, in log2: at most kMost (then m is taken again), at first kWide
// for the largest score so far, from a long piece's tile kTightAt on kTight.
// bf16 has fp32's exponents.  fp16 has no step below 2^-24, so its p ends at
// 2^15, and a key is off by at most 2^-32 of the largest p in the wide range,
// 2^-37 in the tight one: 2^-20 of the values for 4000 keys, the most that stay
// in the wide range, as for 131072 in the tight one.  The wide range is for the
// first tiles, whose maxima grow by a few powers of two (us, caches larger
// than L2, fp16 without shift / 7, 12 from tile 16 on / 13 always: 24 nodes on
// 32 x 8000 rows 133.9 / 132.7 / 144.2; 1000 queries on 4096 rows, with weights,
// 212 / 210 / 244; 13 nodes on 131001 rows, 64 wide, 41.1 / 42.7 / 42.8; 200
// queries on 16 x 9000 rows, 64 wide, 193 / 201 / 224).
template <typename T> struct PRange {
  static constexpr float kMost = 8.0f, kWide = 0.0f, kTight = 0.0f;
  static constexpr int kTightAt = 0;  // (never)
};
template <> struct PRange<__half> {
  static constexpr float kMost = 15.0f, kWide = 7.0f, kTight = 12.0f;
  static constexpr int kTightAt = 16;
};
constexpr uint32_t kTmemCols = 512;
// TMEM columns: S [0, 128) and [128, 256), each half's P over its scores (hi
// then lo); O_0 [256, 256 + D), O_1 [384, 384 + D)
constexpr uint32_t kTmO = 256;

constexpr int kNear = 64;        // sequences whose sizes a CTA keeps

template <int D> struct TcCfg {
  static constexpr int kHalves = D / 64;             // 64-dim boxes of a tile
  static constexpr int kBox = 128 * 128;             // bytes of a 128-row x 64-element box
  static constexpr int kTile = kHalves * kBox;
  static constexpr int kSlots = D == 128 ? 5 : 8;    // what shared memory holds, up to eight
  static constexpr int kOffQ = 0;
  static constexpr int kOffRing = kTile;
  static constexpr int kOffX = kOffRing + kSlots * kTile;   // (m, l) of every thread
  static constexpr int kOffPar = kOffX + kSoftThreads * 8;  // parents, a copy per softmax warp
  static constexpr int kOffOdd = kOffPar + 8 * kTreeMax * 4;  // odd value rows, a bit each, of two tiles
  static constexpr int kOffBar = kOffOdd + 32;
  static constexpr int kOffStage = kOffBar + 256;           // REP 2: 32 columns of each half's 64 rows
  static constexpr int kOffNear = kOffStage + 2 * 64 * 36 * 4;
  static constexpr int kSmem = kOffNear + kNear * 8 + 1024;  // + alignment slack
  static_assert(kSmem <= 232448, "shared memory of a CTA");
};

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const void* tmap, uint32_t bar, int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
      "l"(tmap), "r"(bar), "r"(x), "r"(y), "r"(z)
      : "memory");
}
// D[tmem] (+)= A[tmem] * B[smem]
__device__ __forceinline__ void tc_mma_f16_ta(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(tmem_d),
      "r"(tmem_a), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_st_x16(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Descriptor of a B operand stored MN-major with the 128-byte swizzle: 8-row
// groups 1024 bytes apart, 64-column blocks one box apart.
__device__ __forceinline__ uint64_t desc_mn(uint32_t addr) {
  uint64_t d = 0;
  d |= (uint64_t)((addr & 0x3FFFFu) >> 4);
  d |= (uint64_t)(128 * 128 >> 4) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}

// ------------------------------------------------------------- who does what
// A unit is the rows [rt * queries, ...) of a (sequence, key head); pair =
// b * nrt + rt.  CTA c works for key head c % kv_heads, so that the CTAs of all
// heads, which share the cache's rows (a head's part of a row is 128 or 256
// bytes), pass the same rows at the same time: DRAM pages are opened once.
// With a.splits == 1 CTA c owns pair c / kv_heads.  Otherwise the tiles of all
// pairs, in order, are cut into equal runs, one per kv_heads CTAs, whatever the
// sequences' lengths: a unit may be spread over runs that follow one another,
// whose results meet in the join.  Every valid unit has at least one tile.
constexpr int kRunTiles = 2;  // of a run, where there are too few tiles for all CTAs
struct PairSize {
  int len, count, np, tiles;  // np: tiles of the cache, then one of the draft
};
__device__ __forceinline__ int2 seq_size(const CachedArgs& a, int b) {
  return make_int2(a.lens[b * a.lens_step] + a.len_add, a.counts ? a.counts[b * a.counts_step] : a.tokens);
}
__device__ __forceinline__ PairSize pair_size(const CachedArgs& a, int2 size, int rt, int queries) {
  PairSize p;
  p.len = size.x;
  p.count = size.y;
  p.np = p.tiles = 0;
  if (p.len < 0 || p.len > a.max_seq || p.count < 0 || p.count > a.tokens || rt * queries >= p.count) return p;
  const int last = min((rt + 1) * queries, p.count) - 1;
  p.np = (visible_limit(a, p.len, p.count, last) + kKeys - 1) / kKeys;
  if (!a.k_new && p.np == 0) p.np = 1;  // (nothing to see: zeros are written)
  p.tiles = p.np + (a.k_new ? 1 : 0);
  return p;
}

// A CTA's run of tiles, piece by piece (a piece: its part of one unit).
struct Cursor {
  int64_t left;       // tiles of the run from the next piece on
  int pair, next;     // pair and first tile of the next piece
  // the current piece
  int b, rt, i0, n;   // tiles [i0, i0 + n) of the unit
  // sizes of the sequences from b0 on, in shared memory: a step is on the way
  // of every warp
  const int2* near;
  int b0;
  PairSize z;
  __device__ __forceinline__ bool step(const CachedArgs& a, int nrt, int queries) {
    while (left > 0 && pair < a.n_seq * nrt) {
      b = pair / nrt;
      rt = pair % nrt;
      z = pair_size(a, b - b0 < kNear ? near[b - b0] : seq_size(a, b), rt, queries);
      if (z.tiles > next) {
        i0 = next;
        n = (int)min((int64_t)(z.tiles - next), left);
        left -= n;
        next += n;
        if (next == z.tiles) {
          next = 0;
          ++pair;
        }
        return true;
      }
      next = 0;
      ++pair;
    }
    return false;
  }
};

__device__ __forceinline__ float2 fma2(float2 x, float2 y, float2 z) {
  float2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(reinterpret_cast<unsigned long long&>(r))
      : "l"(reinterpret_cast<unsigned long long&>(x)), "l"(reinterpret_cast<unsigned long long&>(y)),
        "l"(reinterpret_cast<unsigned long long&>(z)));
  return r;
}
__device__ __forceinline__ float2 add2(float2 x, float2 y) {
  float2 r;
  asm("add.rn.f32x2 %0, %1, %2;"
      : "=l"(reinterpret_cast<unsigned long long&>(r))
      : "l"(reinterpret_cast<unsigned long long&>(x)), "l"(reinterpret_cast<unsigned long long&>(y)));
  return r;
}

// Every lane's 16 P bytes v, contiguous at `to`, for the lanes with `ok` (a row
// each): P lanes exchange their pieces (butterflies), so that a store writes
// 16 P bytes of a row side by side.  Rows written piece by piece, 32 rows a
// store, took 1850 cycles per 32 rows x 16 columns of eight warps.
template <int P> __device__ __forceinline__ void store_rows(uint4 (&v)[P], char* to, bool ok) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int st = 1; st < P; st <<= 1)
#pragma unroll
    for (int i = 0; i < P; ++i)
      if (!(i & st)) {
        const bool up = lane & st;
        uint4 x = up ? v[i] : v[i | st];
        x.x = __shfl_xor_sync(0xffffffffu, x.x, st);
        x.y = __shfl_xor_sync(0xffffffffu, x.y, st);
        x.z = __shfl_xor_sync(0xffffffffu, x.z, st);
        x.w = __shfl_xor_sync(0xffffffffu, x.w, st);
        if (up)
          v[i] = x;
        else
          v[i | st] = x;
      }
#pragma unroll
  for (int i = 0; i < P; ++i) {  // v[i]: piece lane % P of row i of the P lanes' rows
    const int from = (lane & ~(P - 1)) + i;
    char* row = reinterpret_cast<char*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(to), from));
    if (__shfl_sync(0xffffffffu, (int)ok, from)) *reinterpret_cast<uint4*>(row + (lane & (P - 1)) * 16) = v[i];
  }
}

template <typename T, int D, int REP>
__global__ void __launch_bounds__(kAtThreads, 1)
    attention_rows_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                          const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmKn,
                          const __grid_constant__ CUtensorMap tmVn, const __grid_constant__ CachedArgs a, int queries, int nrt) {
  using F = TcCfg<D>;
  constexpr int kRowsMax = 128 / REP;
  constexpr int NK = 64 / REP;  // keys of a thread and tile
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  float2* ml = reinterpret_cast<float2*>(smem + F::kOffX);
  uint32_t* odd_rows = reinterpret_cast<uint32_t*>(smem + F::kOffOdd);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + F::kOffBar);
  auto full = [&](int s) { return smem_u32(bars + s); };
  auto empty = [&](int s) { return smem_u32(bars + 8 + s); };
  // one per half and buffer: a half may be two tiles ahead of the products
  auto s_full = [&](int h, int i) { return smem_u32(bars + 16 + 2 * h + (i & 1)); };
  auto p_full = [&](int h, int i) { return smem_u32(bars + 20 + 2 * h + (i & 1)); };
  auto o_full = [&](int h) { return smem_u32(bars + 24 + h); };
  const uint32_t q_full = smem_u32(bars + 26), q_free = smem_u32(bars + 27);  // a piece's queries
  const uint32_t o_done = smem_u32(bars + 28), o_free = smem_u32(bars + 29);  // a piece's outputs
  const uint32_t done_bar = smem_u32(bars + 30);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 31);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int2* near = reinterpret_cast<int2*>(smem + F::kOffNear);
  int64_t* sched = reinterpret_cast<int64_t*>(ml);  // (before the first results)

  const int warp = warp_index(), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < F::kSlots; ++s) {
      mbar_init(full(s), 1);
      mbar_init(empty(s), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(o_full(i), 1);
      for (int h = 0; h < 2; ++h) {
        mbar_init(s_full(h, i), 1);
        mbar_init(p_full(h, i), 4);
      }
    }
    mbar_init(q_full, 1);
    mbar_init(q_free, 1);
    mbar_init(o_done, 1);
    mbar_init(o_free, kSoftThreads / 32);
    mbar_init(done_bar, 1);
    *abort_flag = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) odd_rows[w] = 0;
    fence_barrier_init();
    prefetch_tmap(&tmQ);
    prefetch_tmap(&tmK);
    prefetch_tmap(&tmV);
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(tmem_slot), kTmemCols);
    tmem_relinquish();
  }
  pdl_wait();
  Cursor cur;
  cur.next = 0;
  const int kvh = blockIdx.x % a.kv_heads, run = blockIdx.x / a.kv_heads;
  // sizes of the sequences from b0 on (with runs and more sequences than that, from the run's first)
  cur.b0 = a.splits == 1 ? run / nrt : 0;
  cur.near = near;
  auto fetch_near = [&]() {
    if (threadIdx.x < kNear && cur.b0 + (int)threadIdx.x < a.n_seq) near[threadIdx.x] = seq_size(a, cur.b0 + threadIdx.x);
  };
  if (a.splits == 1 || a.n_seq <= kNear) fetch_near();
  int64_t first_tile = 0, total = 0;  // the run's first tile in the order of all; their number
  int runs = 1;
  if (a.splits == 1) {
    cur.pair = run;
    const PairSize z = pair_size(a, seq_size(a, cur.pair / nrt), cur.pair % nrt, queries);
    cur.left = z.tiles;
    if (z.tiles == 0 && threadIdx.x == 0 && kvh == 0) {
      int len, count;
      seq_sizes(a, cur.pair / nrt, &len, &count);  // (reports what is out of range)
    }
    tc_fence_before();
  } else {
    // every thread adds up a run of pairs, then the threads' sums
    const int pairs = a.n_seq * nrt, per = (pairs + kAtThreads - 1) / kAtThreads;
    const int p0 = min((int)threadIdx.x * per, pairs), p1 = min(p0 + per, pairs);
    int64_t sum = 0;
    for (int p = p0; p < p1; ++p) {
      sum += pair_size(a, seq_size(a, p / nrt), p % nrt, queries).tiles;
      if (blockIdx.x == 0) {
        const int b = p / nrt, n = a.lens[b * a.lens_step] + a.len_add, c = a.counts ? a.counts[b * a.counts_step] : a.tokens;
        if (n < 0 || n > a.max_seq || c < 0 || c > a.tokens) atomicExch(a.err, kDevErrBounds);
      }
    }
    int64_t before = sum;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int64_t o = __shfl_up_sync(0xffffffffu, before, off);
      if (lane >= off) before += o;
    }
    if (lane == 31) sched[warp] = before;
    before -= sum;
    tc_fence_before();
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kAtThreads / 32; ++w) {
      if (w < warp) before += sched[w];
      total += sched[w];
    }
    runs = (int)min((int64_t)(gridDim.x / a.kv_heads), (total + kRunTiles - 1) / kRunTiles);
    first_tile = run < runs ? total * run / runs : total;
    cur.left = run < runs ? total * (run + 1) / runs - first_tile : 0;
    cur.pair = 0;
    if (cur.left > 0 && before <= first_tile && first_tile < before + sum) {
      int64_t at = before;
      for (int p = p0; p < p1; ++p) {
        const int tiles = pair_size(a, seq_size(a, p / nrt), p % nrt, queries).tiles;
        if (first_tile < at + tiles) {
          sched[16] = p;
          sched[17] = first_tile - at;
          break;
        }
        at += tiles;
      }
    }
    __syncthreads();
    if (cur.left > 0) {
      cur.pair = (int)sched[16];
      cur.next = (int)sched[17];
    }
    if (a.n_seq > kNear) {
      cur.b0 = cur.pair / nrt;
      fetch_near();
    }
  }
  __syncthreads();  // (and sched is written again, as ml)
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  // (not before this CTA has its TMEM: a kernel that starts early may hold some
  // while it waits for this one's end)
  pdl_launch_dependents();
  // a piece's tiles in the order of use: K0, K1, V0, K2, V1, ..., V(n-1)
  auto k_pos = [&](int i) { return i == 0 ? 0 : 2 * i - 1; };
  auto v_pos = [&](int i, int n) { return i == n - 1 ? 2 * n - 1 : 2 * i + 2; };

  // the softmax warps take registers that the others leave
  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsLow));
    if (warp == 0 && elect_one()) {
      // ---------------- TMA producer
      const int q_bytes = REP * F::kHalves * queries * a.group * 128;
      int pos = 0, piece = 0;
      bool ok = true;
      for (; ok && cur.step(a, nrt, queries); ++piece) {
        auto load = [&](int i, bool keys) -> bool {
          const int s = pos % F::kSlots;
          if (pos >= F::kSlots && !mbar_wait_bounded(empty(s), ((pos / F::kSlots) - 1) & 1, abort_flag, a.err)) return false;
          mbar_arrive_expect_tx(full(s), F::kTile);
          const bool nw = cur.i0 + i >= cur.z.np;
          const CUtensorMap* tm = keys ? (nw ? &tmKn : &tmK) : (nw ? &tmVn : &tmV);
#pragma unroll
          for (int h = 0; h < F::kHalves; ++h)
            tma_load_3d(smem_u32(smem + F::kOffRing + s * F::kTile + h * F::kBox), tm, full(s), kvh * D + h * 64,
                        nw ? 0 : (cur.i0 + i) * kKeys, cur.b);
          ++pos;
          return true;
        };
        ok = load(0, true) && (cur.n < 2 || load(1, true));
        if (!ok) break;
        if (piece > 0 && !mbar_wait_bounded(q_free, (piece - 1) & 1, abort_flag, a.err)) break;
        mbar_arrive_expect_tx(q_full, q_bytes);
#pragma unroll
        for (int c = 0; c < REP; ++c)
#pragma unroll
          for (int h = 0; h < F::kHalves; ++h)
            tma_load_3d(smem_u32(smem + F::kOffQ + h * F::kBox + c * (kRowsMax * 128)), &tmQ, q_full, h * 64, kvh * a.group,
                        cur.b * a.tokens + cur.rt * queries);
        for (int i = 0; ok && i < cur.n; ++i) ok = load(i, false) && (i + 2 >= cur.n || load(i + 2, true));
        if (!ok) {
          ++piece;  // its queries are on their way
          break;
        }
      }
      // let every load issued land before the CTA can exit
      volatile int no_abort = 0;
      if (piece > 0) mbar_wait_bounded(q_full, (piece - 1) & 1, &no_abort, nullptr);
      for (int j = max(0, pos - F::kSlots); j < pos; ++j)
        mbar_wait_bounded(full(j % F::kSlots), (j / F::kSlots) & 1, &no_abort, nullptr);
    }
    if (warp == 1 && elect_one()) {
      // ---------------- MMA issuer
      constexpr int bf = std::is_same<T, __nv_bfloat16>::value ? 1 : 0;
      constexpr uint32_t idesc_s = idesc_f16(bf, 128, kKeys / 2);
      constexpr uint32_t idesc_pv = idesc_f16(bf, 128, D) | (1u << 16);  // B (values) MN-major
      const uint64_t qd = smem_desc_sw128(smem_u32(smem + F::kOffQ));
      const uint64_t kd = smem_desc_sw128(smem_u32(smem + F::kOffRing)), vd = desc_mn(smem_u32(smem + F::kOffRing));
      int pos0 = 0, g0 = 0;  // of the piece: ring position, tiles before
      bool ok = true;
      auto wait = [&](uint32_t bar, uint32_t parity) { return mbar_wait_bounded(bar, parity, abort_flag, a.err); };
      for (int piece = 0; ok && cur.step(a, nrt, queries); ++piece) {
        const int n = cur.n;
        // The halves' scores and products take turns, so that one half's warps
        // (one of the two on each scheduler) take exponentials while the
        // other's wait, load and store.
        auto scores = [&](int i, int h) -> bool {
          const int pos = pos0 + k_pos(i), s = pos % F::kSlots, g = g0 + i;
          if (h == 0 && !wait(full(s), (pos / F::kSlots) & 1)) return false;
          // (over the P of two tiles ago: the tensor core runs the MMAs of one
          // thread in the order of their issue, so its product, issued before,
          // has read it)
          tc_fence_after();
          const uint64_t kt = kd + (uint64_t)(s * (F::kTile >> 4) + h * (64 * 128 >> 4));  // the descriptors' address field counts 16 bytes
#pragma unroll
          for (int c = 0; c < F::kHalves; ++c)
#pragma unroll
            for (int k = 0; k < 4; ++k)
              tc_mma_f16(tmem + (uint32_t)(g & 1) * 128u + (uint32_t)h * 64u, qd + (uint64_t)(c * (F::kBox >> 4) + 2 * k),
                         kt + (uint64_t)(c * (F::kBox >> 4) + 2 * k), idesc_s, (c | k) != 0);
          tc_commit(s_full(h, g));
          if (h == 1) {
            tc_commit(empty(s));
            if (i == n - 1) tc_commit(q_free);
          }
          return true;
        };
        ok = wait(q_full, piece & 1) && scores(0, 0) && scores(0, 1);
        for (int i = 0; ok && i < n; ++i) {
          const int pos = pos0 + v_pos(i, n), s = pos % F::kSlots, g = g0 + i;
          const uint64_t vt = vd + (uint64_t)(s * (F::kTile >> 4));
          for (int h = 0; ok && h < 2; ++h) {
            if (i + 1 < n && !(ok = scores(i + 1, h))) break;
            ok = (h == 1 || (wait(full(s), (pos / F::kSlots) & 1) && (i > 0 || piece == 0 || wait(o_free, (piece - 1) & 1)))) &&
                 wait(p_full(h, g), (g >> 1) & 1);
            if (!ok) break;
            tc_fence_after();
            const uint32_t pt = tmem + (uint32_t)(g & 1) * 128u + (uint32_t)h * 64u;
#pragma unroll
            for (int part = 0; part < 2; ++part)
#pragma unroll
              for (int ks = 0; ks < 4; ++ks)  // 16 keys a step
                tc_mma_f16_ta(tmem + kTmO + (uint32_t)h * 128u,
                              pt + (uint32_t)(part * 32 + ks * 8),
                              vt + (uint64_t)((h * 4 + ks) * (2048 >> 4)), idesc_pv, (uint32_t)(i | part | ks) != 0);
            tc_commit(o_full(h));
          }
          if (ok) tc_commit(empty(s));
        }
        if (ok) tc_commit(o_done);
        pos0 += 2 * n;
        g0 += n;
      }
      // every MMA issued must have finished before TMEM is freed
      tc_commit(done_bar);
      volatile int no_abort = 0;
      mbar_wait_bounded(done_bar, 0, &no_abort, nullptr);
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsHigh));
    // ---------------- softmax and output
    // two threads per row: `half` of a tile's keys, an output and a reference of
    // its own
    const int q4 = warp & 3, half = (warp - 4) >> 2;
    const int slot = q4 * 32 + lane, rep = slot / kRowsMax, row = slot % kRowsMax;
    const int aid = (warp - 4) * 32 + lane;
    const int kofs = half * 64 + rep * NK;  // this thread's first key of a tile
    const uint32_t lane_off = (uint32_t)(q4 * 32) << 16;
    const uint32_t tO = tmem + kTmO + (uint32_t)half * 128u + lane_off;
    auto row_sync = [&]() { asm volatile("bar.sync %0, 64;" ::"r"(1 + q4) : "memory"); };  // the two warps of the same rows
    auto all_sync = [&]() { asm volatile("bar.sync 5, %0;" ::"n"(kSoftThreads) : "memory"); };
    auto half_sync = [&]() { asm volatile("bar.sync %0, 128;" ::"r"(6 + half) : "memory"); };
    auto copy_sync = [&]() { asm volatile("bar.sync %0, 64;" ::"r"(8 + 2 * (q4 & 1) + half) : "memory"); };  // REP 2: a row's two lanes
    int* par = reinterpret_cast<int*>(smem + F::kOffPar) + (warp - 4) * kTreeMax;
    bool ok = true;
    int pos0 = 0, g0 = 0;
    int rest = 0, rest_rows = 0;  // the unit that this CTA begins and others go on with
    for (int piece = 0; cur.step(a, nrt, queries); ++piece) {
      const int b = cur.b, n = cur.n, np = cur.z.np, len = cur.z.len, count = cur.z.count;
      const int t0 = cur.rt * queries, rows = min(queries, count - t0) * a.group;
      const int lim_min = visible_limit(a, len, count, t0);
      const bool last = cur.i0 + n == cur.z.tiles, whole = cur.i0 == 0 && last;  // a piece up to the unit's end; all of it
      const bool works = q4 * 32 % kRowsMax < rows;  // the warp's lanes hold rows
      const int t = t0 + min(row, rows - 1) / a.group;
      const int lim = visible_limit(a, len, count, t);
      bool bad = false;  // a parent that is none
      if (a.parents && (last || cur.i0 == 0)) {  // (the first piece's CTA speaks for the join)
        __syncwarp();  // the piece before has read its parents
        for (int i = lane; i < count; i += 32) {
          par[i] = a.parents[(int64_t)b * a.tokens + i];
          bad = bad || par[i] < -1 || par[i] >= i;
        }
        __syncwarp();
        bad = __any_sync(0xffffffffu, bad);
        if (bad && aid == 0) atomicExch(a.err, kDevErrBounds);
      }
      using R = PRange<T>;
      float m = -INFINITY, l = 0.f;  // m: the reference, in log2 units
      float top = -INFINITY;         // the largest scaled score so far
      const bool tighten = R::kTightAt > 0 && n >= 2 * R::kTightAt;
      for (int i = 0; i < n; ++i) {
        const int g = g0 + i;
        const bool nw = cur.i0 + i >= np;
        const int k0 = nw ? 0 : (cur.i0 + i) * kKeys;
        const bool masked = nw || k0 + kKeys > lim_min;  // some of these keys are hidden from some rows
        const uint32_t tS = tmem + (uint32_t)(g & 1) * 128u + lane_off;
        ok = ok && mbar_wait_bounded(s_full(half, g), (g >> 1) & 1, abort_flag, a.err);
        ok = __all_sync(0xffffffffu, ok);
        tc_fence_after();
        uint32_t hi[NK / 2], lo[NK / 2];
        if (works) {
          uint32_t s[NK];
          float mx = -INFINITY;
          if (ok) {
#pragma unroll
            for (int c = 0; c < NK; c += 32)
              tmem_ld_32x32b_x32(tS + (uint32_t)(kofs + c), *reinterpret_cast<uint32_t(*)[32]>(s + c));
            tmem_ld_wait();
            if (masked) {
              uint64_t see = 0;
              if (nw && a.parents) {
                for (int j = bad ? -1 : t; j >= 0; j = par[j])
                  if ((uint32_t)(j - kofs) < (uint32_t)NK) see |= 1ull << (j - kofs);
              } else {
                const int seen = (nw ? t + 1 : lim - k0) - kofs;
                see = seen >= 64 ? ~0ull : seen > 0 ? (1ull << seen) - 1ull : 0ull;
              }
#pragma unroll
              for (int k = 0; k < NK; ++k)
                if (!(see >> k & 1u)) s[k] = 0xff800000u;  // -inf
            }
            float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int k = 0; k < NK; ++k) mx4[k & 3] = fmaxf(mx4[k & 3], __uint_as_float(s[k]));
            mx = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3])) * a.scale_log2;
          }
          top = fmaxf(top, mx);
          const bool grow = mx - m > R::kMost || (tighten && i == R::kTightAt && top != -INFINITY);  // (also the first key seen)
          if (__any_sync(0xffffffffu, grow)) {
            float alpha = 1.f;
            if (grow) {
              const float ref = (R::kTightAt ? top : mx) - (tighten && i >= R::kTightAt ? R::kTight : R::kWide);
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
            const float2 scale2 = make_float2(a.scale_log2, a.scale_log2), base2 = make_float2(-base, -base), minus = make_float2(-1.f, -1.f);
            float2 sum2[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
            for (int k0 = 0; k0 < NK / 2; k0 += 8) {  // (step by step over eight pairs: their latencies overlap)
              float2 p[8];
#pragma unroll
              for (int k = 0; k < 8; ++k)
                p[k] = fma2(make_float2(__uint_as_float(s[2 * (k0 + k)]), __uint_as_float(s[2 * (k0 + k) + 1])), scale2, base2);
#pragma unroll
              for (int k = 0; k < 8; ++k) p[k] = make_float2(ex2(p[k].x), ex2(p[k].y));
#pragma unroll
              for (int k = 0; k < 8; ++k) hi[k0 + k] = pack_pair<T>(p[k].x, p[k].y);
#pragma unroll
              for (int k = 0; k < 8; ++k) sum2[k & 1] = add2(sum2[k & 1], p[k]);
#pragma unroll
              for (int k = 0; k < 8; ++k) p[k] = fma2(unpack_pair<T>(hi[k0 + k]), minus, p[k]);
#pragma unroll
              for (int k = 0; k < 8; ++k) lo[k0 + k] = pack_pair<T>(p[k].x, p[k].y);
            }
            l += (sum2[0].x + sum2[0].y) + (sum2[1].x + sum2[1].y);
          }
        }
        uint32_t odd = 0;
        if (masked) {
          // A value row that some of the rows do not see must not reach them
          // even if it is infinite or not a number (0 x inf): rows behind the
          // last key are cleared, others that hold such a value as well, and
          // added by hand below where they are seen.  Each half looks after
          // the rows of its own product, so the halves go on taking turns.
          const int pos = pos0 + v_pos(i, n);
          uint8_t* vs = smem + F::kOffRing + (pos % F::kSlots) * F::kTile;
          ok = ok && mbar_wait_bounded(full(pos % F::kSlots), (pos / F::kSlots) & 1, abort_flag, a.err);
          ok = __all_sync(0xffffffffu, ok);
          const int have = min(kKeys, nw ? count : len - k0), hidden = nw ? 0 : min(have, max(0, lim_min - k0));  // from there on, from some rows
          // this thread's 16-byte chunks: one column of them, kStep rows apart (a
          // multiple of the swizzle's eight, so that they lie a constant apart)
          constexpr int kMine = 64 * (D / 8) / 128, kStep = 128 / (D / 8);
          const int c0 = aid & 127, r0 = half * 64 + c0 / (D / 8), x0 = c0 % (D / 8);
          uint8_t* mine = vs + (x0 >> 3) * F::kBox + r0 * 128 + (((x0 & 7) ^ (r0 & 7)) << 4);
          const uint4 none = make_uint4(0u, 0u, 0u, 0u);
          // (two buffers: a warp may look through the next tile's rows while
          // another still reads what was found in this one's; the tile after
          // that starts once every warp has handed over this one's P)
          uint32_t* odd_now = odd_rows + 4 * (g & 1);
          if (ok) {
            if (hidden < have) {
              uint4 v[kMine];
              uint32_t found = 0;
#pragma unroll
              for (int u = 0; u < kMine; ++u) v[u] = *reinterpret_cast<const uint4*>(mine + u * kStep * 128);
#pragma unroll
              for (int u = 0; u < kMine; ++u) found |= odd_chunk<T>(v[u]) ? 1u << u : 0u;
              if (found) {
#pragma unroll 1
                for (int u = 0; u < kMine; ++u) {
                  const int r = r0 + u * kStep;
                  if (found >> u & 1u && r >= hidden && r < have) atomicOr(&odd_now[r >> 5], 1u << (r & 31));
                }
              }
            }
#pragma unroll
            for (int u = 0; u < kMine; ++u)
              if (r0 + u * kStep >= have) *reinterpret_cast<uint4*>(mine + u * kStep * 128) = none;
          }
          if (hidden < have) {
            half_sync();
            odd = odd_now[2 * half] | odd_now[2 * half + 1];
            if (odd) {
#pragma unroll 1
              for (int u = 0; u < kMine; ++u) {
                const int r = r0 + u * kStep;
                if (odd_now[r >> 5] >> (r & 31) & 1u) *reinterpret_cast<uint4*>(mine + u * kStep * 128) = none;
              }
            }
          }
          fence_proxy_async_smem();  // V is read by the tensor cores (async proxy)
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
        if (odd) {
          uint32_t* odd_now = odd_rows + 4 * (g & 1);
          // O is at rest once this tile's product is done.  A parity cannot tell
          // phase g from phase g - 2, so phase g - 1 has to be known complete
          // before phase g is waited for: a piece's first tile has it from the
          // o_done of the piece before; for the others these scores only prove
          // phase g - 2 (they were issued before the product of g - 1, behind
          // that of g - 2), which is what makes the wait for g - 1 safe in turn.
          ok = ok && (i == 0 || mbar_wait_bounded(o_full(half), (g - 1) & 1, abort_flag, a.err)) &&
               mbar_wait_bounded(o_full(half), g & 1, abort_flag, a.err);
          ok = __all_sync(0xffffffffu, ok);
          tc_fence_after();
#pragma unroll 1
          for (int j = half * 64; j < half * 64 + 64; ++j) {
            if (!(odd_now[j >> 5] >> (j & 31) & 1u)) continue;
            const int rel = j - kofs;
            if (rel >= 0 && rel < NK && ok && works) {  // (the same for all lanes of a warp)
              float pj = 0.f;
#pragma unroll
              for (int k = 0; k < NK / 2; ++k) {
                const float2 h2 = unpack_pair<T>(hi[k]), l2 = unpack_pair<T>(lo[k]);
                if (rel == 2 * k) pj = h2.x + l2.x;
                if (rel == 2 * k + 1) pj = h2.y + l2.y;
              }
              const T* v = nw ? static_cast<const T*>(a.v_new) + ((int64_t)b * a.tokens + j) * a.new_stride
                              : static_cast<const T*>(a.v) + (int64_t)b * a.seq_stride + (int64_t)(k0 + j) * a.kv_stride;
              v += kvh * D;
#pragma unroll 1
              for (int c = 0; c < D; c += 16) {
                uint32_t r[16];
                tmem_ld_32x32b_x16(tO + (uint32_t)c, r);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 16; ++e)
                  if (pj != 0.f) r[e] = __float_as_uint(fmaf(pj, to_f<T>(v[c + e]), __uint_as_float(r[e])));
                tmem_st_x16(tO + (uint32_t)c, r);
                tmem_st_wait();
              }
              tc_fence_before();
            }
            tc_fence_after();
          }
          half_sync();  // everyone has read the odd rows
          if ((aid & 127) < 2) odd_now[2 * half + (aid & 127)] = 0;
          half_sync();
        }
      }
      // ---- the piece's results: a thread joins the two halves of its row in
      // its share of the columns, and with REP 2 the row's two lanes meet in
      // shared memory
      ok = ok && mbar_wait_bounded(o_done, piece & 1, abort_flag, a.err);
      ok = __all_sync(0xffffffffu, ok);
      tc_fence_after();
      ml[half * 128 + slot] = make_float2(m, l);
      tc_fence_before();  // (values that this half's warps added to its O by hand, which the other half's read below)
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
      const bool writes = ok && !bad && row < rows && (REP == 1 || rep == 0);
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
          float* stage = reinterpret_cast<float*>(smem + F::kOffStage) + (half * 64 + row) * 36;
          if (rep == 1) {
#pragma unroll
            for (int e = 0; e < 32; e += 4) *reinterpret_cast<float4*>(stage + e) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
          }
          copy_sync();
          if (rep == 0) {
#pragma unroll
            for (int e = 0; e < 32; e += 4) {
              const float4 x = *reinterpret_cast<const float4*>(stage + e);
              o[e] += x.x;
              o[e + 1] += x.y;
              o[e + 2] += x.z;
              o[e + 3] += x.w;
            }
          }
          copy_sync();
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
      rest = cur.i0 == 0 && !whole && !bad ? cur.z.tiles : 0;  // the run ends inside this unit
      rest_rows = rows;
      if (REP == 1) row_sync(); else all_sync();  // ml is written again
      pos0 += 2 * n;
      g0 += n;
    }
    if (a.splits != 1 && aid == 0) {
      int4 record = make_int4(0, 0, 0, 0);
      if (rest) {  // how many runs it reaches into
        const int64_t end = first_tile + (g0 - cur.n) + rest - 1;  // its last tile
        int c = (int)(end * runs / total);  // whose run that is, up to the rounding
        while (total * (c + 1) / runs <= end) ++c;
        while (total * c / runs > end) --c;
        record = make_int4(cur.b, cur.rt, kvh | rest_rows << 16, c - run + 1);
      }
      a.units[blockIdx.x] = record;
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

// ------------------------------------------------------------------- weights
// weights_j = weights_in_j + sum over rows of 2^(s_rj - lse_r): the scores with
// the keys as the MMA's rows, S^T = K Q^T (M 128 keys x N up to 128 rows), so
// that a key's sum over the rows stays in one thread.  A CTA takes every
// splits-th tile of 128 keys of a (sequence, key head) and passes all tiles of
// rows that see it; K and Q tiles by TMA, S in two TMEM buffers, two threads
// per key (their sums meet in shared memory).  Two CTAs share an SM: one's
// start and waits are the other's time.  Rows of a list are fetched one query
// at a time.
// Measured: 32 sequences of 8 key heads (group 4), 1 to 8 listed queries on
// up to 8000 rows (0.37 GB): 68.5 us, 5.3 TB/s; 1000 queries on 4096 rows, 2 x 32
// heads, f16: 87 us, 0.51 PFLOP/s; 512 queries x 32 heads on themselves: 8.2 us.
// Few rows are bound by reading the keys, many by the sum warps: about 1450
// cycles for 128 x 128 scores on an SM, of which the exponentials' unit is busy
// for 1024 (16 a cycle).  Warp products (16 rows each) in its place took 119 us
// for 4 listed rows where this took 64, so it serves every count of rows.
// LIST: rows of a list, in an instance of its own, since looking for entries out
// of range in the loop of the others took 4 % of theirs (211 us with the
// attention, 220 so) and 2.5 % of the list's.
template <int D> struct WtCfg {
  static constexpr int kHalves = D / 64;
  static constexpr int kBox = 128 * 128;
  static constexpr int kTile = kHalves * kBox;
  static constexpr int kSlots = 3;                         // of keys and queries
  static constexpr int kOffLse = kSlots * kTile;           // [2][128] of the rows
  static constexpr int kOffX = kOffLse + 2 * 128 * 4;
  static constexpr int kOffBar = kOffX + 2 * 128 * 4;
  static constexpr int kSmem = kOffBar + 256 + 1024;
  static_assert(2 * (kSmem + 1024) <= 233472, "two CTAs per SM");
};
constexpr int kSBufs = 2;
constexpr uint32_t kWtTmemCols = 256;  // two CTAs share the SM's 512

template <typename T, int D, bool LIST>
__global__ void __launch_bounds__(kTcThreads, 2)
    weights_rows_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                        const __grid_constant__ CachedArgs a, int queries) {
  using F = WtCfg<D>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  float* lse = reinterpret_cast<float*>(smem + F::kOffLse);
  float* xch = reinterpret_cast<float*>(smem + F::kOffX);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + F::kOffBar);
  auto k_full = [&](int s) { return smem_u32(bars + s); };
  auto k_empty = [&](int s) { return smem_u32(bars + 3 + s); };
  auto q_full = [&](int s) { return smem_u32(bars + 6 + s); };
  auto q_empty = [&](int s) { return smem_u32(bars + 9 + s); };
  auto s_full = [&](int s) { return smem_u32(bars + 12 + s); };
  auto s_empty = [&](int s) { return smem_u32(bars + 16 + s); };
  const uint32_t done_bar = smem_u32(bars + 20);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 21);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(bars + 22);
  // [2][4]: of a tile of listed rows, a bit per row that is none: the scores
  // there are another query's, which may be unused and hold anything
  uint32_t* none_rows = reinterpret_cast<uint32_t*>(bars + 24);

  const int warp = warp_index(), lane = threadIdx.x & 31;
  // (the tiles that most rows see start first)
  const int kvh = blockIdx.x, b = blockIdx.y, split = blockIdx.z;
  pdl_wait();
  int len, count;
  if (!seq_sizes(a, b, &len, &count)) return;
  const int ktiles = (len + kKeys - 1) / kKeys, nrt = (count + queries - 1) / queries;
  if (split >= ktiles) return;
  // the first tile of rows that sees key k0 (row i sees the keys below len - count + i + 1)
  auto first_tile = [&](int kt) { return max(0, kt * kKeys - (len - count)) / queries; };
  // one tile of rows: its queries stay, and two slots take keys in turn; more:
  // the queries pass through two slots for every tile of keys
  const bool one = nrt <= 1;
  const int ks = one ? 2 : 1, qs = one ? 1 : 2;
  uint8_t* smem_q = smem + ks * F::kTile;

  if (threadIdx.x == 0) {
    for (int s = 0; s < 2; ++s) {
      mbar_init(k_full(s), 1);
      mbar_init(k_empty(s), 1);
      mbar_init(q_full(s), 1);
      mbar_init(q_empty(s), 1);
    }
    for (int s = 0; s < kSBufs; ++s) {
      mbar_init(s_full(s), 1);
      mbar_init(s_empty(s), kSoftThreads / 32);
    }
    mbar_init(done_bar, 1);
    *abort_flag = 0;
    fence_barrier_init();
    prefetch_tmap(&tmQ);
    prefetch_tmap(&tmK);
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(tmem_slot), kWtTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_launch_dependents();  // (this CTA has its TMEM, see above)

  if (warp == 0) {
    if (nrt > 0 && elect_one()) {
      // ---------------- TMA producer
      auto load_q = [&](int rt, int slot) {
        const int t0 = rt * queries;
        const uint32_t dst = smem_u32(smem_q + slot * F::kTile);
        if (!LIST) {
          mbar_arrive_expect_tx(q_full(slot), F::kHalves * queries * a.group * 128);
#pragma unroll
          for (int h = 0; h < F::kHalves; ++h)
            tma_load_3d(dst + h * F::kBox, &tmQ, q_full(slot), h * 64, kvh * a.group, b * a.tokens + t0);
          return;
        }
        const int nq = min(queries, count - t0);
        mbar_arrive_expect_tx(q_full(slot), F::kHalves * nq * a.group * 128);
        for (int i = 0; i < nq; ++i) {
          const int q = min(max(a.rows[(int64_t)b * a.rows_step + t0 + i], 0), a.tokens - 1);
#pragma unroll
          for (int h = 0; h < F::kHalves; ++h)
            tma_load_3d(dst + h * F::kBox + i * a.group * 128, &tmQ, q_full(slot), h * 64, kvh * a.group, b * a.tokens + q);
        }
      };
      int it = 0, kp = 0;
      bool ok = true;
      for (int kt = split; ok && kt < ktiles; kt += (int)gridDim.z, ++kp) {
        const int s = kp % ks;
        if (kp >= ks && !mbar_wait_bounded(k_empty(s), ((kp / ks) - 1) & 1, abort_flag, a.err)) break;
        mbar_arrive_expect_tx(k_full(s), F::kTile);
#pragma unroll
        for (int h = 0; h < F::kHalves; ++h)
          tma_load_3d(smem_u32(smem + s * F::kTile + h * F::kBox), &tmK, k_full(s), kvh * D + h * 64, kt * kKeys, b);
        if (one) {
          if (kp == 0) load_q(0, 0);
          continue;
        }
        for (int rt = first_tile(kt); rt < nrt; ++rt, ++it) {
          const int slot = it % qs;
          if (it >= qs && !mbar_wait_bounded(q_empty(slot), ((it / qs) - 1) & 1, abort_flag, a.err)) {
            ok = false;
            ++kp;  // its keys are on their way
            break;
          }
          load_q(rt, slot);
        }
        if (!ok) break;
      }
      // let every load issued land before the CTA can exit
      volatile int no_abort = 0;
      for (int j = max(0, kp - ks); j < kp; ++j) mbar_wait_bounded(k_full(j % ks), (j / ks) & 1, &no_abort, nullptr);
      const int nl = one ? min(kp, 1) : it;
      for (int j = max(0, nl - qs); j < nl; ++j) mbar_wait_bounded(q_full(j % qs), (j / qs) & 1, &no_abort, nullptr);
    }
  } else if (warp == 1) {
    if (nrt > 0 && elect_one()) {
      // ---------------- MMA issuer
      constexpr int bf = std::is_same<T, __nv_bfloat16>::value ? 1 : 0;
      const uint64_t kd = smem_desc_sw128(smem_u32(smem)), qd = smem_desc_sw128(smem_u32(smem_q));
      int it = 0, kp = 0;
      bool ok = true;
      for (int kt = split; ok && kt < ktiles; kt += (int)gridDim.z, ++kp) {
        const int s = kp % ks;
        if (!mbar_wait_bounded(k_full(s), (kp / ks) & 1, abort_flag, a.err)) break;
        for (int rt = first_tile(kt); ok && rt < nrt; ++rt, ++it) {
          const int slot = one ? 0 : it % qs, sb = it % kSBufs;
          ok = mbar_wait_bounded(q_full(slot), one ? 0 : (it / qs) & 1, abort_flag, a.err) &&
               (it < kSBufs || mbar_wait_bounded(s_empty(sb), ((it / kSBufs) - 1) & 1, abort_flag, a.err));
          if (!ok) break;
          tc_fence_after();
          const int n = (min(queries, count - rt * queries) * a.group + 15) / 16 * 16;
          const uint32_t idesc = idesc_f16(bf, 128, n);
          const uint64_t kk = kd + (uint64_t)(s * (F::kTile >> 4)), qq = qd + (uint64_t)(slot * (F::kTile >> 4));
#pragma unroll
          for (int h = 0; h < F::kHalves; ++h)
#pragma unroll
            for (int k = 0; k < 4; ++k)
              tc_mma_f16(tmem + (uint32_t)sb * 128u, kk + (uint64_t)(h * (F::kBox >> 4) + 2 * k),
                         qq + (uint64_t)(h * (F::kBox >> 4) + 2 * k), idesc, (h | k) != 0);
          tc_commit(s_full(sb));
          if (!one) tc_commit(q_empty(slot));
        }
        tc_commit(k_empty(s));
      }
      tc_commit(done_bar);  // every MMA issued must have finished before TMEM is freed
      volatile int no_abort = 0;
      mbar_wait_bounded(done_bar, 0, &no_abort, nullptr);
    }
  } else {
    // ---------------- sums: warps 2..9, a key per thread and half of the rows
    const int q4 = warp & 3, half = (warp - 2) >> 2, slot = q4 * 32 + lane;
    const int aid = (warp - 2) * 32 + lane;
    const uint32_t lane_off = (uint32_t)(q4 * 32) << 16;
    auto pair_sync = [&]() { asm volatile("bar.sync %0, 64;" ::"r"(1 + q4) : "memory"); };
    auto all_sync = [&]() { asm volatile("bar.sync 5, 256;" ::: "memory"); };
    const int64_t at = ((int64_t)b * a.kv_heads + kvh) * a.max_seq;
    // thread aid < 128 has row aid of a tile of rows' lse copied to shared memory
    const int row_q = aid / a.group;
    const float* row_lse = a.lse + ((int64_t)b * a.heads + kvh * a.group + aid % a.group) * a.tokens;
    auto fetch = [&](int rt, int buf) {
      if (aid < 128) {
        const int t = rt * queries + row_q;
        bool have = row_q < queries && t < count;
        int q = t;
        if (LIST && have) {
          q = a.rows[(int64_t)b * a.rows_step + t];
          have = q >= 0 && q < a.tokens;
          if (!have) atomicExch(a.err, kDevErrBounds);
        }
        if (LIST) {
          const uint32_t none = __ballot_sync(0xffffffffu, !have && row_q < queries && t < count);
          if (lane == 0) none_rows[buf * 4 + (aid >> 5)] = none;
        }
        if (have)
          asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(lse + buf * 128 + aid)), "l"(row_lse + q) : "memory");
        else
          lse[buf * 128 + aid] = INFINITY;  // (adds nothing)
      }
      cp_async_commit();
    };
    if (nrt > 0) {
      fetch(first_tile(split), 0);
      cp_async_wait<0>();
      all_sync();
    }
    const float2 scale2 = make_float2(a.scale_log2, a.scale_log2), log2e = make_float2(-1.4426950408889634f, -1.4426950408889634f);
    const float2 zero2 = make_float2(0.f, 0.f);
    int it = 0, kp = 0;
    bool ok = true;
    for (int kt = split; kt < ktiles; kt += (int)gridDim.z, ++kp) {
      const int j = kt * kKeys + slot;
      const float before = half == 0 && j < len && a.weights_in ? a.weights_in[at + j] : 0.f;
      float2 sum2[2] = {zero2, zero2};
      for (int rt = first_tile(kt); rt < nrt; ++rt, ++it) {
        const int sb = it % kSBufs, buf = one ? 0 : it & 1;
        const bool last = rt + 1 == nrt && kt + (int)gridDim.z >= ktiles;
        if (!one && !last) fetch(rt + 1 < nrt ? rt + 1 : first_tile(kt + (int)gridDim.z), buf ^ 1);
        ok = ok && mbar_wait_bounded(s_full(sb), (it / kSBufs) & 1, abort_flag, a.err);
        ok = __all_sync(0xffffffffu, ok);
        tc_fence_after();
        if (ok) {
          const int rows = min(queries, count - rt * queries) * a.group, nch = (rows + 15) / 16;
          // the tile's rows from `low` on see this thread's key; from `low_all`
          // on, all of the tile's keys
          const int ahead = kt * kKeys - (len - count) - rt * queries;
          // (clamped first: far behind the queries, rows times heads pass 32 bits)
          const int low = max(ahead + slot, 0) * a.group, low_all = max(ahead + kKeys - 1, 0) * a.group;
          const uint32_t tS = tmem + (uint32_t)sb * 128u + lane_off;
          const uint32_t* none = none_rows + buf * 4;
          const bool some_none = LIST && (none[0] | none[1] | none[2] | none[3]);
#pragma unroll
          for (int c2 = 0; c2 < 4; c2 += 2) {  // two of the half's chunks of 16 rows at a time
            uint32_t s[2][16];
#pragma unroll
            for (int c = 0; c < 2; ++c)
              if (half + 2 * (c2 + c) < nch) tmem_ld_32x32b_x16(tS + (uint32_t)((half + 2 * (c2 + c)) * 16), s[c]);
            tmem_ld_wait();
            if (c2 == 2) {  // all has been read
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(s_empty(sb));
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              const int c0 = (half + 2 * (c2 + c)) * 16;
              if (c0 >= rows) break;
              const float* le = lse + buf * 128 + c0;
              float2 p[8];
#pragma unroll
              for (int e = 0; e < 8; e += 2) {
                const float4 l4 = *reinterpret_cast<const float4*>(le + 2 * e);
                p[e] = fma2(make_float2(l4.x, l4.y), log2e, fma2(make_float2(__uint_as_float(s[c][2 * e]), __uint_as_float(s[c][2 * e + 1])), scale2, zero2));
                p[e + 1] = fma2(make_float2(l4.z, l4.w), log2e, fma2(make_float2(__uint_as_float(s[c][2 * e + 2]), __uint_as_float(s[c][2 * e + 3])), scale2, zero2));
              }
#pragma unroll
              for (int e = 0; e < 8; ++e) p[e] = make_float2(ex2(p[e].x), ex2(p[e].y));
              if (c0 < low_all || c0 + 16 > rows) {  // hidden keys, or rows behind the last
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                  const int r = c0 + 2 * e;
                  if (r < low || r >= rows) p[e].x = 0.f;
                  if (r + 1 < low || r + 1 >= rows) p[e].y = 0.f;
                }
              }
              if (some_none) {
                const uint32_t here = none[c0 >> 5] >> (c0 & 31);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                  if (here >> (2 * e) & 1u) p[e].x = 0.f;
                  if (here >> (2 * e + 1) & 1u) p[e].y = 0.f;
                }
              }
#pragma unroll
              for (int e = 0; e < 8; ++e) sum2[e & 1] = add2(sum2[e & 1], p[e]);
            }
          }
        }
        if (!one && !last) {
          cp_async_wait<0>();
          all_sync();
        }
      }
      const float sum = (sum2[0].x + sum2[0].y) + (sum2[1].x + sum2[1].y);
      float* x = xch + (kp & 1) * 128;
      if (half == 1) x[slot] = sum;
      pair_sync();
      if (half == 0 && j < len && ok) a.weights[at + j] = before + (sum + x[slot]);
    }
    tc_fence_before();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, kWtTmemCols);
  }
}

int done(cudaError_t e, const char* what) {
  if (e == cudaSuccess) e = cudaGetLastError();
  if (e != cudaSuccess) SN_FAIL(SWAPNET_ERR_CUDA, std::string(what) + ": " + cudaGetErrorString(e));
  return SWAPNET_OK;
}

// Maps of the queries (64 dims x the heads of a group x queries) and of a
// cache or a draft (64 dims x 128 rows of one sequence).
int query_map(CUtensorMap* m, const CachedArgs& a, int queries) {
  const uint64_t dims[3] = {(uint64_t)a.dim, (uint64_t)a.heads, (uint64_t)a.n_seq * a.tokens};
  const uint64_t strides[2] = {(uint64_t)a.dim * 2, (uint64_t)a.q_stride * 2};
  const uint32_t box[3] = {64, (uint32_t)a.group, (uint32_t)queries};
  return make_tmap_3d(m, a.dtype, a.q, dims, strides, box);
}
int rows_map(CUtensorMap* m, const CachedArgs& a, const void* base, int64_t rows, int64_t row_stride, int64_t seq_stride) {
  const uint64_t dims[3] = {(uint64_t)a.kv_heads * a.dim, (uint64_t)rows, (uint64_t)a.n_seq};
  // (a single sequence's stride is never used, but has to be a valid one)
  const uint64_t strides[2] = {(uint64_t)row_stride * 2, (uint64_t)(a.n_seq > 1 ? seq_stride : row_stride) * 2};
  const uint32_t box[3] = {64, kKeys, 1};
  return make_tmap_3d(m, a.dtype, base, dims, strides, box);
}

// The join of the units that several CTAs shared: blockIdx.y is the CTA that
// begins one.  A CTA holds at most two pieces that are not whole units: the
// rest of one that began before its run (slot 2 c) and the start of one that
// goes on behind it (slot 2 c + 1).  A warp per row, or all eight warps of the
// block where that takes fewer rounds of loads, each of four pieces (a unit of
// hundreds of pieces, or a block per row).
constexpr int kRjWarps = 8;
template <typename T>
__global__ void __launch_bounds__(32 * kRjWarps)
    attention_runs_join_kernel(const __grid_constant__ CachedArgs a, int queries, int row_tile) {
  __shared__ float4 so[kRjWarps][32];
  __shared__ float2 sm[kRjWarps];
  pdl_wait();
  const int c = blockIdx.y, lane = threadIdx.x & 31, warp = warp_index();
  const int4 u = a.units[c];
  if (u.w == 0) return;
  const int b = u.x, t0 = u.y * queries, kvh = u.z & 0xffff, rows = u.z >> 16, pieces = u.w;
  const int blocks = gridDim.x, per_warp = (rows + kRjWarps * blocks - 1) / (kRjWarps * blocks), per_block = (rows + blocks - 1) / blocks;
  const bool many = per_block * ((pieces + 4 * kRjWarps - 1) / (4 * kRjWarps) + 1) < per_warp * ((pieces + 3) / 4);  // (+ 1: the warps' results meet)
  const int V = a.dim / 4, first = many ? warp : 0, step = many ? kRjWarps : 1;
  const float2* ml = reinterpret_cast<const float2*>(a.ml);
  const float4* part = reinterpret_cast<const float4*>(a.part);
  for (int r0 = blockIdx.x * (many ? 1 : kRjWarps); r0 < rows; r0 += gridDim.x * (many ? 1 : kRjWarps)) {
    const int rl = many ? r0 : r0 + warp;
    const bool own = rl < rows;
    auto slot = [&](int p) { return ((int64_t)2 * (c + p * a.kv_heads) + (p == 0 ? 1 : 0)) * row_tile + rl; };
    float M = -INFINITY, L = 0.f;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    auto take = [&](float2 s, float4 y) {  // (m = -inf: nothing was seen, and y may be anything)
      const float m = fmaxf(M, s.x), base = m == -INFINITY ? 0.f : m;
      const float f = ex2(M - base), g = ex2(s.x - base);
      M = m;
      L = fmaf(L, f, s.y * g);
      if (s.x == -INFINITY) y = make_float4(0.f, 0.f, 0.f, 0.f);
      x.x = fmaf(x.x, f, y.x * g);
      x.y = fmaf(x.y, f, y.y * g);
      x.z = fmaf(x.z, f, y.z * g);
      x.w = fmaf(x.w, f, y.w * g);
    };
    for (int p0 = first; own && p0 < pieces; p0 += 4 * step) {
      float2 s[4];
      float4 y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int p = p0 + i * step;
        s[i] = p < pieces ? ml[slot(p)] : make_float2(-INFINITY, 0.f);
        y[i] = p < pieces && lane < V ? part[slot(p) * V + lane] : make_float4(0.f, 0.f, 0.f, 0.f);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) take(s[i], y[i]);
    }
    if (many) {
      so[warp][lane] = x;
      if (lane == 0) sm[warp] = make_float2(M, L);
      __syncthreads();
      if (warp == 0) {
#pragma unroll
        for (int i = 1; i < kRjWarps; ++i) take(sm[i], so[i][lane]);
      }
      __syncthreads();
    }
    if (own && (!many || warp == 0)) {
      const int t = t0 + rl / a.group, hd = kvh * a.group + rl % a.group;
      const float inv = L > 0.f ? 1.0f / L : (L == 0.f ? 0.f : L);
      if (lane < V) {
        T* to = static_cast<T*>(a.out) + ((int64_t)b * a.tokens + t) * a.out_stride + (int64_t)hd * a.dim + lane * 4;
        *reinterpret_cast<uint2*>(to) = make_uint2(pack_pair<T>(x.x * inv, x.y * inv), pack_pair<T>(x.z * inv, x.w * inv));
      }
      if (lane == 0 && a.lse)
        a.lse[((int64_t)b * a.heads + hd) * a.tokens + t] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
    }
  }
}

template <typename T, int D, int REP> int rows_t(const CachedArgs& a, bool early, cudaStream_t s) {
  static std::atomic<uint64_t> known{0};
  const auto kern = attention_rows_kernel<T, D, REP>;
  if (attr_needed(known)) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, TcCfg<D>::kSmem);
    if (e != cudaSuccess) return done(e, "cached attention: shared memory");
    attr_set(known);
  }
  const int queries = std::min(128 / REP / a.group, a.tokens);
  CUtensorMap q, k, v, kn, vn;
  int rc = query_map(&q, a, queries);
  if (!rc) rc = rows_map(&k, a, a.k, a.max_seq, a.kv_stride, a.seq_stride);
  if (!rc) rc = rows_map(&v, a, a.v, a.max_seq, a.kv_stride, a.seq_stride);
  kn = k;
  vn = v;
  if (a.k_new) {
    if (!rc) rc = rows_map(&kn, a, a.k_new, a.tokens, a.new_stride, a.new_stride * a.tokens);
    if (!rc) rc = rows_map(&vn, a, a.v_new, a.tokens, a.new_stride, a.new_stride * a.tokens);
  }
  if (rc) return rc;
  cudaLaunchConfig_t cfg;
  std::memset(&cfg, 0, sizeof(cfg));
  const int nrt = (a.tokens + queries - 1) / queries;
  const int ctas = run_ctas(a.kv_heads);
  cfg.gridDim = dim3(a.splits == 1 ? a.n_seq * nrt * a.kv_heads : ctas);
  cfg.blockDim = dim3(kAtThreads);
  cfg.dynamicSmemBytes = TcCfg<D>::kSmem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = early ? 1 : 0;
  rc = done(cudaLaunchKernelEx(&cfg, kern, q, k, v, kn, vn, a, queries, nrt), "cached attention launch");
  if (rc || a.splits == 1) return rc;
  // eight blocks per SM that find work, but at least a warp and at most a block
  // for a row (20 units of 28 tiles and 48 rows, up to 9 pieces each: 37.6 us
  // with 6 blocks for a unit's rows, 25.5 with 48)
  const int64_t units = std::min<int64_t>((int64_t)a.n_seq * nrt * a.kv_heads, ctas);
  const int rows = queries * a.group, least = (rows + kRjWarps - 1) / kRjWarps;
  cfg.gridDim = dim3(std::min(rows, std::max(least, (int)(8 * kSms / units))), ctas);
  cfg.blockDim = dim3(32 * kRjWarps);
  cfg.dynamicSmemBytes = 0;
  cfg.numAttrs = 1;
  return done(cudaLaunchKernelEx(&cfg, attention_runs_join_kernel<T>, a, queries, 128 / REP), "cached attention join launch");
}
template <typename T, int D> int rows_d(const CachedArgs& a, bool early, cudaStream_t s) {
  return a.tokens * a.group <= 64 ? rows_t<T, D, 2>(a, early, s) : rows_t<T, D, 1>(a, early, s);
}

template <typename T, int D, bool LIST> int weights_t(const CachedArgs& a, int splits, bool early, cudaStream_t s) {
  static std::atomic<uint64_t> known{0};
  const auto kern = weights_rows_kernel<T, D, LIST>;
  if (attr_needed(known)) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, WtCfg<D>::kSmem);
    if (e != cudaSuccess) return done(e, "cache weights: shared memory");
    attr_set(known);
  }
  const int queries = std::min(128 / a.group, a.tokens);
  CUtensorMap q, k;
  int rc = query_map(&q, a, LIST ? 1 : queries);
  if (!rc) rc = rows_map(&k, a, a.k, a.max_seq, a.kv_stride, a.seq_stride);
  if (rc) return rc;
  cudaLaunchConfig_t cfg;
  std::memset(&cfg, 0, sizeof(cfg));
  cfg.gridDim = dim3(a.kv_heads, a.n_seq, splits);
  cfg.blockDim = dim3(kTcThreads);
  cfg.dynamicSmemBytes = WtCfg<D>::kSmem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = early ? 1 : 0;
  return done(cudaLaunchKernelEx(&cfg, kern, q, k, a, queries), "cache weights launch");
}
template <typename T, int D> int weights_d(const CachedArgs& a, int splits, bool early, cudaStream_t s) {
  return a.rows ? weights_t<T, D, true>(a, splits, early, s) : weights_t<T, D, false>(a, splits, early, s);
}

}  // namespace

int launch_weights(const CachedArgs& a, int splits, bool early, cudaStream_t s) {
  if (a.dtype == SWAPNET_BF16)
    return a.dim == 128 ? weights_d<__nv_bfloat16, 128>(a, splits, early, s) : weights_d<__nv_bfloat16, 64>(a, splits, early, s);
  return a.dim == 128 ? weights_d<__half, 128>(a, splits, early, s) : weights_d<__half, 64>(a, splits, early, s);
}

int launch_attention_rows(const CachedArgs& a, bool early, cudaStream_t s) {
  if (a.dtype == SWAPNET_BF16)
    return a.dim == 128 ? rows_d<__nv_bfloat16, 128>(a, early, s) : rows_d<__nv_bfloat16, 64>(a, early, s);
  return a.dim == 128 ? rows_d<__half, 128>(a, early, s) : rows_d<__half, 64>(a, early, s);
}

}  // namespace swapnet
