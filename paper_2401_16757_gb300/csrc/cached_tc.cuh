// Device-side pieces that the tensor-core attention kernels share: operands in
// tensor memory, which tiles a CTA takes, rows written side by side.
#pragma once
#include "cached.cuh"

namespace swapnet {

constexpr int kKeys = 128;       // keys of a tile
constexpr int kNear = 64;        // sequences whose sizes a CTA keeps

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

}  // namespace swapnet
