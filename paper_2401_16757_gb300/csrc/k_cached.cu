// Attention of a few queries over a long key-value cache (decode steps, small
// drafted trees), and the join of its splits, with the weights that the cached
// rows got.  fp16 / bf16 storage, fp32 arithmetic, fixed orders of summation.
//
// Rows of a (sequence, key head) are its queries times the heads that share
// the key head: they read the same keys, so one warp-level product serves up
// to 16 of them.
#include <algorithm>
#include <cstring>
#include <string>
#include <type_traits>

#include "cached.cuh"
#include "internal.h"
#include "kernels.h"

namespace swapnet {

namespace {

constexpr int kFwWarps = 4, kFwThreads = 32 * kFwWarps;
constexpr int kGk = 16;      // keys of a group: one step of a warp
constexpr int kFwStages = 3;
// log2 of the largest p: fp16 has no step below 2^-24, so that its two parts of
// p <= 1 would lose the keys below 2^-25 of the largest; with p <= 2^15 a key is
// off by at most 2^-40.  bf16 has fp32's exponents.  (Part of the reference m, so
// that it costs one subtraction per row and group.)
template <typename T> constexpr float kPTop = std::is_same<T, __half>::value ? 15.0f : 0.0f;

template <int D> struct FewCfg {
  static constexpr int kGroup = kGk * D * 2;          // bytes of a group's keys (or values)
  static constexpr int kWarpRing = kFwStages * 2 * kGroup;
  static constexpr int kRing = kFwWarps * kWarpRing;
  static constexpr int kRows = kFewAttnRows;
  static constexpr int kQ = kRows * D * 2;
  static constexpr int kP = kFwWarps * kRows * kGk * 4;
  static constexpr int kOffQ = kRing;
  static constexpr int kOffP = kOffQ + kQ;
  static constexpr int kOffMl = kOffP + kP;
  static constexpr int kOffAnc = kOffMl + kFwWarps * kRows * 8;
  static constexpr int kOffPar = kOffAnc + kTreeMax * 16;
  static constexpr int kSmem = kOffPar + kTreeMax * 4;
  static_assert(kFwWarps * kRows * D * 4 <= kRing, "the warps' outputs overlay the ring");
};

// Byte offset of 16-byte chunk `c` of row `r` in a tile of D-element rows:
// chunks are exchanged within 128 bytes so that the eight rows of an
// 8 x 8 matrix lie in different banks.
template <int D> __device__ __forceinline__ uint32_t swz(int r, int c) { return (uint32_t)(r * (D * 2) + ((c ^ (r & 7)) << 4)); }

// The rows' queries into shared memory (zeros behind the last row).
template <typename T, int D>
__device__ __forceinline__ void load_queries(const CachedArgs& a, int b, int kvh, int rows, uint8_t* dst) {
  constexpr int C = D / 8;
  for (int i = threadIdx.x; i < kFewAttnRows * C; i += kFwThreads) {
    const int r = i / C, c = i % C;
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (r < rows)
      v = *reinterpret_cast<const uint4*>(static_cast<const T*>(a.q) + ((int64_t)b * a.tokens + r / a.group) * a.q_stride +
                                          (int64_t)(kvh * a.group + r % a.group) * D + c * 8);
    *reinterpret_cast<uint4*>(dst + swz<D>(r, c)) = v;
  }
}

// ---------------------------------------------------------- few-row attention
// One CTA: the keys [split] of a (sequence, key head) for up to 16 rows.
// Its warps take groups of 16 keys in turn and keep a softmax of their own
// (running maximum m, sum l, output O in registers), so nothing waits for
// another warp until the end:
//   S = Q K^T          8 mma.m16n8k16 a 16 rows for 128 dims
//   p = 2^(S - m)      handed to the next product as parts of the storage type:
//                      three of bf16, all 24 bits of p, two of fp16, 22 bits
//   O = O 2^(m' - m) + p V
// Keys and values pass through a ring of three groups a warp (cp.async; rows
// behind the sequence's end arrive as zeros, whatever the cache holds there).
// The parts cost a second and a third product, which are free here; one part
// would leave 8 (bf16) or 11 (fp16) bits of p, less than the fp32 that the sums
// keep, two of bf16 17.
// The kernel is bound by reading the cache: a group's 8 KB takes 48 products
// of 16 rows, and the warp-level ones do that at several times DRAM's rate,
// without the fixed costs (TMEM, barriers, 128-row tiles) of tcgen05.
// Measured: one token of 64 sequences, 8 key heads (group 4) of 128 wide bf16
// heads, up to 16384 rows (3.2 GB): 452 us, 7.0 TB/s; with the weights (SPILL: the
// scaled scores are stored for the join, 0.13 GB written and read) 531, 6.1
// TB/s; 7 nodes of 8 heads on 100 rows: 7.2 us, all of it latency (two launches,
// lengths, a tile's round trip, the join).  The second pass over the keys that
// stored scores replace would read 1.6 GB again.
template <typename T, int D, bool SPILL>
__global__ void __launch_bounds__(kFwThreads, 2) attention_few_kernel(const __grid_constant__ CachedArgs a) {
  using F = FewCfg<D>;
  extern __shared__ __align__(128) uint8_t smem[];
  uint32_t(*anc)[4] = reinterpret_cast<uint32_t(*)[4]>(smem + F::kOffAnc);
  int* par = reinterpret_cast<int*>(smem + F::kOffPar);
  float2* mls = reinterpret_cast<float2*>(smem + F::kOffMl);
  const int split = blockIdx.x;
  const int kvh = blockIdx.y, b = blockIdx.z;
  const int warp = warp_index(), lane = threadIdx.x & 31;
  pdl_wait();
  pdl_launch_dependents();
  int len, count;
  if (!seq_sizes(a, b, &len, &count)) return;
  const int rows = count * a.group;
  if (rows == 0) return;
  const int kmax = visible_limit(a, len, count, count - 1), lim_min = visible_limit(a, len, count, 0);
  const int gp = (kmax + kGk - 1) / kGk, groups = gp + (a.k_new ? (count + kGk - 1) / kGk : 0);
  const int g_begin = (int)((int64_t)groups * split / a.splits), g_end = (int)((int64_t)groups * (split + 1) / a.splits);

  uint8_t* ring = smem + warp * F::kWarpRing;
  const uint32_t ring_u = smem_u32(ring);
  auto load = [&](int g, int slot) {
    if (g < g_end) {
      const bool nw = g >= gp;
      const int j0 = (nw ? g - gp : g) * kGk, have = (nw ? count : len) - j0;
      const int64_t stride = nw ? a.new_stride : a.kv_stride;
      const int64_t at = (nw ? (int64_t)b * a.tokens * a.new_stride : (int64_t)b * a.seq_stride) + j0 * stride + kvh * D;
      const T* kb = static_cast<const T*>(nw ? a.k_new : a.k) + at;
      const T* vb = static_cast<const T*>(nw ? a.v_new : a.v) + at;
      const uint32_t dst = ring_u + (uint32_t)slot * 2 * F::kGroup;
      constexpr int C = D / 8;
#pragma unroll
      for (int i = 0; i < kGk * C / 32; ++i) {
        const int r = (lane + 32 * i) / C, c = (lane + 32 * i) % C;
        const bool ok = r < have;
        const int64_t off = ok ? r * stride + c * 8 : 0;
        cp_async_16(dst + swz<D>(r, c), kb + off, ok);
        cp_async_16(dst + F::kGroup + swz<D>(r, c), vb + off, ok);
      }
    }
    cp_async_commit();
  };
#pragma unroll
  for (int i = 0; i < kFwStages - 1; ++i) load(g_begin + warp + i * kFwWarps, i);

  load_queries<T, D>(a, b, kvh, rows, smem + F::kOffQ);
  if (a.k_new && !build_ancestors(a, b, count, anc, par)) {  // (while the first groups arrive)
    cp_async_wait<0>();
    return;
  }
  __syncthreads();
  const uint32_t q_u = smem_u32(smem + F::kOffQ);
  uint32_t qf[D / 16][4];
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) ldmatrix_x4(q_u + swz<D>(lane & 15, 2 * ks + (lane >> 4)), qf[ks]);
  // this lane's rows: lane / 4 and 8 behind it
  int lim[2], node[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = 8 * h + (lane >> 2);
    node[h] = r < rows ? r / a.group : -1;
    lim[h] = r < rows ? visible_limit(a, len, count, r / a.group) : 0;
  }
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, o[D / 8][4];
#pragma unroll
  for (int n = 0; n < D / 8; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[n][e] = 0.f;
  int slot = 0;
  for (int g = g_begin + warp; g < g_end; g += kFwWarps) {
    int ahead = slot + kFwStages - 1;
    if (ahead >= kFwStages) ahead -= kFwStages;
    load(g + (kFwStages - 1) * kFwWarps, ahead);
    cp_async_wait<kFwStages - 1>();
    __syncwarp();
    const uint32_t ks_u = ring_u + (uint32_t)slot * 2 * F::kGroup, vs_u = ks_u + F::kGroup;
    const bool nw = g >= gp;
    const int j0 = (nw ? g - gp : g) * kGk;
    float s[2][4];
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[n][e] = 0.f;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      uint32_t kf[4];
      ldmatrix_x4(ks_u + swz<D>((lane & 7) + ((lane >> 4) << 3), 2 * ks + ((lane >> 3) & 1)), kf);
      mma_16816<T>(s[0], qf[ks], kf[0], kf[1]);
      mma_16816<T>(s[1], qf[ks], kf[2], kf[3]);
    }
    const bool masked = nw || j0 + kGk > lim_min;  // some of these keys are hidden from some rows
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[n][e] *= a.scale_log2;
        if (masked) {
          const int h = e >> 1, j = j0 + n * 8 + (lane & 3) * 2 + (e & 1);
          const bool sees = nw ? node[h] >= 0 && (anc[node[h]][j >> 5] >> (j & 31) & 1u) : j < lim[h];
          if (!sees) s[n][e] = -INFINITY;
        }
      }
    if (SPILL) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = 8 * h + (lane >> 2);
        if (r < rows) {
          float* to = a.scores + (((int64_t)b * a.kv_heads + kvh) * a.tokens * a.group + r) * a.score_ld + j0 + (lane & 3) * 2;
#pragma unroll
          for (int n = 0; n < 2; ++n) *reinterpret_cast<float2*>(to + n * 8) = make_float2(s[n][2 * h], s[n][2 * h + 1]);
        }
      }
    }
    constexpr int kParts = std::is_same<T, __half>::value ? 2 : 3;
    uint32_t pp[kParts][4];
    float al[2], base[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float mx = fmaxf(fmaxf(s[0][2 * h], s[0][2 * h + 1]), fmaxf(s[1][2 * h], s[1][2 * h + 1]));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2)) - kPTop<T>;
      const float mn = fmaxf(m[h], mx);
      base[h] = mn == -INFINITY ? 0.f : mn;  // (nothing seen yet)
      al[h] = ex2(m[h] - base[h]);
      m[h] = mn;
    }
    float sum[2] = {0.f, 0.f};
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float p0 = ex2(s[n][2 * h] - base[h]), p1 = ex2(s[n][2 * h + 1] - base[h]);
        sum[h] += p0 + p1;
        s[n][2 * h] = p0;
        s[n][2 * h + 1] = p1;
        float2 left = make_float2(p0, p1);
#pragma unroll
        for (int i = 0; i < kParts; ++i) {
          const uint32_t part = pp[i][2 * n + h] = pack_pair<T>(left.x, left.y);
          const float2 back = unpack_pair<T>(part);
          left = make_float2(left.x - back.x, left.y - back.y);
        }
      }
#pragma unroll
    for (int h = 0; h < 2; ++h) l[h] = l[h] * al[h] + sum[h];
    if (__any_sync(0xffffffffu, al[0] != 1.f || al[1] != 1.f)) {
#pragma unroll
      for (int n = 0; n < D / 8; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[n][e] *= al[e >> 1];
    }
    if (masked) {
      // A hidden value row that is infinite or not a number must not reach
      // the rows that do not see it (0 x inf): such rows are added by hand,
      // where they are seen, and zeroed for the product.
      uint8_t* vs = ring + slot * 2 * F::kGroup + F::kGroup;
      uint32_t odd = 0;  // bit per value row
#pragma unroll
      for (int i = 0; i < kGk * (D / 8) / 32; ++i) {
        const int r = (lane + 32 * i) / (D / 8), c = (lane + 32 * i) % (D / 8);
        const uint4 v = *reinterpret_cast<const uint4*>(vs + swz<D>(r, c));
        if (odd_chunk<T>(v)) odd |= 1u << r;
      }
      odd = __reduce_or_sync(0xffffffffu, odd);
      if (odd) {
        float* pb = reinterpret_cast<float*>(smem + F::kOffP) + warp * F::kRows * kGk;
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) pb[(8 * (e >> 1) + (lane >> 2)) * kGk + n * 8 + (lane & 3) * 2 + (e & 1)] = s[n][e];
        __syncwarp();
        while (odd) {
          const int j = __ffs(odd) - 1;
          odd &= odd - 1;
#pragma unroll
          for (int n = 0; n < D / 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float p = pb[(8 * (e >> 1) + (lane >> 2)) * kGk + j];
              const T v = *reinterpret_cast<const T*>(vs + swz<D>(j, n) + ((lane & 3) * 2 + (e & 1)) * 2);
              if (p != 0.f) o[n][e] = fmaf(p, to_f<T>(v), o[n][e]);
            }
          __syncwarp();
          if (lane < D / 8) *reinterpret_cast<uint4*>(vs + swz<D>(j, lane)) = make_uint4(0u, 0u, 0u, 0u);
          __syncwarp();
        }
      }
    }
#pragma unroll
    for (int n = 0; n < D / 16; ++n) {
      uint32_t vf[4];
      ldmatrix_x4_trans(vs_u + swz<D>(lane & 15, 2 * n + (lane >> 4)), vf);
#pragma unroll
      for (int i = 0; i < kParts; ++i) {
        mma_16816<T>(o[2 * n], pp[i], vf[0], vf[1]);
        mma_16816<T>(o[2 * n + 1], pp[i], vf[2], vf[3]);
      }
    }
    __syncwarp();  // the group has been read before its slot is filled again
    if (++slot == kFwStages) slot = 0;
  }
  // the warps' results meet in shared memory, in warp order
  cp_async_wait<0>();
  __syncthreads();
  float* ow = reinterpret_cast<float*>(smem) + warp * F::kRows * D;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float x = l[h];
    x += __shfl_xor_sync(0xffffffffu, x, 1);
    x += __shfl_xor_sync(0xffffffffu, x, 2);
    const int rl = 8 * h + (lane >> 2);
    if ((lane & 3) == 0) mls[warp * F::kRows + rl] = make_float2(m[h], x);
#pragma unroll
    for (int n = 0; n < D / 8; ++n)
      *reinterpret_cast<float2*>(ow + rl * D + n * 8 + (lane & 3) * 2) = make_float2(o[n][2 * h], o[n][2 * h + 1]);
  }
  __syncthreads();
  constexpr int V = D / 4;  // float4 per row
  for (int i = threadIdx.x; i < F::kRows * V; i += kFwThreads) {
    const int r = i / V, c = i % V;
    if (r >= rows) break;
    float M = -INFINITY, L = 0.f;
#pragma unroll
    for (int w = 0; w < kFwWarps; ++w) M = fmaxf(M, mls[w * F::kRows + r].x);
    const float base = M == -INFINITY ? 0.f : M;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kFwWarps; ++w) {
      const float2 ml = mls[w * F::kRows + r];
      const float f = ex2(ml.x - base);
      const float4 y = reinterpret_cast<const float4*>(smem)[(w * F::kRows + r) * V + c];
      L = fmaf(ml.y, f, L);
      if (f != 0.f) {
        x.x = fmaf(y.x, f, x.x);
        x.y = fmaf(y.y, f, x.y);
        x.z = fmaf(y.z, f, x.z);
        x.w = fmaf(y.w, f, x.w);
      }
    }
    const int64_t slot_r = (((int64_t)b * a.kv_heads + kvh) * a.splits + split) * a.tokens * a.group + r;
    if (c == 0 && (a.splits > 1 || SPILL)) reinterpret_cast<float2*>(a.ml)[slot_r] = make_float2(M, L);
    if (a.splits > 1) {
      if (M != -INFINITY) reinterpret_cast<float4*>(a.part)[slot_r * V + c] = x;
      continue;
    }
    const int t = r / a.group, hd = kvh * a.group + r % a.group;
    const float inv = L > 0.f ? 1.0f / L : (L == 0.f ? 0.f : L);  // (a NaN stays one)
    T* to = static_cast<T*>(a.out) + ((int64_t)b * a.tokens + t) * a.out_stride + (int64_t)hd * D + c * 4;
    *reinterpret_cast<uint2*>(to) = make_uint2(pack_pair<T>(x.x * inv, x.y * inv), pack_pair<T>(x.z * inv, x.w * inv));
    if (c == 0 && a.lse) a.lse[((int64_t)b * a.heads + hd) * a.tokens + t] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
  }
}

// ----------------------------------------------------------------- the join
// Blocks [0, join_blocks): a warp per row, the splits in order:
//   M = max m_s, L = sum l_s 2^(m_s - M), out = sum O_s 2^(m_s - M) / L.
// The blocks behind them: weights_j = weights_in_j + sum over the rows that
// see row j of 2^(score - log2 L - M), from the stored scores.  The scores of
// the 531 us call above take it 33 us, 6 TB/s of scores and weights.
constexpr int kJoinThreads = 256, kJoinKeys = 4 * kJoinThreads;

// log2 of a row's softmax sum, over its splits.
__device__ __forceinline__ float2 join_stats(const CachedArgs& a, int64_t first, int64_t step) {
  float M = -INFINITY, L = 0.f;
  for (int s = 0; s < a.splits; ++s) M = fmaxf(M, reinterpret_cast<const float2*>(a.ml)[first + s * step].x);
  const float base = M == -INFINITY ? 0.f : M;
  for (int s = 0; s < a.splits; ++s) {
    const float2 ml = reinterpret_cast<const float2*>(a.ml)[first + s * step];
    L = fmaf(ml.y, ex2(ml.x - base), L);
  }
  return make_float2(M, L);
}

template <typename T>
__global__ void __launch_bounds__(kJoinThreads) attention_join_kernel(const __grid_constant__ CachedArgs a, int join_blocks) {
  extern __shared__ float lse2[];  // of the scores' rows, then the keys that they see
  pdl_wait();
  const int kvh = blockIdx.y, b = blockIdx.z;
  int len, count;
  if (!seq_sizes(a, b, &len, &count)) return;
  const int rows = count * a.group;
  const int64_t step = (int64_t)a.tokens * a.group;
  const int64_t first = ((int64_t)b * a.kv_heads + kvh) * a.splits * step;
  if ((int)blockIdx.x < join_blocks) {
    if (a.k_new && a.parents) {  // the splits of such a sequence were not computed
      bool bad = false;
      for (int t = threadIdx.x; t < count; t += blockDim.x) {
        const int p = a.parents[(int64_t)b * a.tokens + t];
        bad = bad || p < -1 || p >= t;
      }
      if (__syncthreads_or(bad)) return;
    }
    const int r = (int)blockIdx.x * (kJoinThreads / 32) + warp_index(), lane = threadIdx.x & 31;
    if (r >= rows) return;
    const float2 st = join_stats(a, first + r, step);
    const float base = st.x == -INFINITY ? 0.f : st.x;
    const int t = r / a.group, hd = kvh * a.group + r % a.group;
    const float inv = st.y > 0.f ? 1.0f / st.y : (st.y == 0.f ? 0.f : st.y);
    const int V = a.dim / 4;
    if (lane < V) {
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int s = 0; s < a.splits; ++s) {
        const float ms = reinterpret_cast<const float2*>(a.ml)[first + s * step + r].x;
        if (ms == -INFINITY) continue;
        const float f = ex2(ms - base);
        const float4 y = reinterpret_cast<const float4*>(a.part)[(first + s * step + r) * V + lane];
        x.x = fmaf(y.x, f, x.x);
        x.y = fmaf(y.y, f, x.y);
        x.z = fmaf(y.z, f, x.z);
        x.w = fmaf(y.w, f, x.w);
      }
      T* to = static_cast<T*>(a.out) + ((int64_t)b * a.tokens + t) * a.out_stride + (int64_t)hd * a.dim + lane * 4;
      *reinterpret_cast<uint2*>(to) = make_uint2(pack_pair<T>(x.x * inv, x.y * inv), pack_pair<T>(x.z * inv, x.w * inv));
    }
    if (lane == 0 && a.lse)
      a.lse[((int64_t)b * a.heads + hd) * a.tokens + t] = st.y == 0.f ? -INFINITY : (st.x + log2f(st.y)) * 0.6931471805599453f;
    return;
  }
  const int j0 = ((int)blockIdx.x - join_blocks) * kJoinKeys;
  if (j0 >= len) return;
  const int64_t at = ((int64_t)b * a.kv_heads + kvh) * a.max_seq;
  const float* sc = a.scores + ((int64_t)b * a.kv_heads + kvh) * step * a.score_ld + j0;
  const bool all = j0 + kJoinKeys <= visible_limit(a, len, count, 0);  // every row sees every key of the block
  // four keys per thread, the loads of four rows before their arithmetic
  constexpr int K = kJoinKeys / kJoinThreads;
  float w[K], x[4][K];
  auto load = [&](int r0) {
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int i = 0; i < K; ++i) {
        const int j = i * kJoinThreads + threadIdx.x;
        x[u][i] = r0 + u < rows && j0 + j < len ? sc[(int64_t)(r0 + u) * a.score_ld + j] : -INFINITY;
      }
  };
  load(0);
#pragma unroll
  for (int i = 0; i < K; ++i) {
    const int j = j0 + i * kJoinThreads + threadIdx.x;
    w[i] = j < len && a.weights_in ? a.weights_in[at + j] : 0.f;
  }
  int* lim = reinterpret_cast<int*>(lse2 + rows);
  for (int r = threadIdx.x; r < rows; r += kJoinThreads) {
    const float2 st = join_stats(a, first + r, step);
    lse2[r] = st.x + log2f(st.y);
    lim[r] = visible_limit(a, len, count, r / a.group);
  }
  __syncthreads();
  float sum[K];
#pragma unroll
  for (int i = 0; i < K; ++i) sum[i] = 0.f;
  for (int r0 = 0; r0 < rows; r0 += 4) {
    if (r0 > 0) load(r0);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (r0 + u >= rows) break;
      const float l2 = lse2[r0 + u];
      const int lm = lim[r0 + u];
#pragma unroll
      for (int i = 0; i < K; ++i)
        if (all || j0 + i * kJoinThreads + (int)threadIdx.x < lm) sum[i] += ex2(x[u][i] - l2);
    }
  }
#pragma unroll
  for (int i = 0; i < K; ++i) {
    const int j = j0 + i * kJoinThreads + threadIdx.x;
    if (j < len) a.weights[at + j] = w[i] + sum[i];
  }
}

int done(cudaError_t e, const char* what) {
  if (e == cudaSuccess) e = cudaGetLastError();
  if (e != cudaSuccess) SN_FAIL(SWAPNET_ERR_CUDA, std::string(what) + ": " + cudaGetErrorString(e));
  return SWAPNET_OK;
}

template <typename... KArgs, typename... Args>
cudaError_t launch(void (*kern)(KArgs...), dim3 grid, int threads, size_t smem, bool early, cudaStream_t s, Args... args) {
  cudaLaunchConfig_t cfg;
  std::memset(&cfg, 0, sizeof(cfg));
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = early ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kern, static_cast<KArgs>(args)...);
}

// Shared memory above 48 KB is allowed per function and device, once.
template <typename K> int allow_smem(K kern, int bytes, std::atomic<uint64_t>& known) {
  if (!attr_needed(known)) return SWAPNET_OK;
  const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e != cudaSuccess) return done(e, "cached attention: shared memory");
  attr_set(known);
  return SWAPNET_OK;
}

template <typename T, int D, bool SPILL> int few_t(const CachedArgs& a, bool early, cudaStream_t s) {
  static std::atomic<uint64_t> known{0};
  using F = FewCfg<D>;
  if (int rc = allow_smem(attention_few_kernel<T, D, SPILL>, F::kSmem, known)) return rc;
  return done(launch(attention_few_kernel<T, D, SPILL>, dim3(a.splits, a.kv_heads, a.n_seq), kFwThreads, F::kSmem, early, s, a),
              "cached attention launch");
}
template <typename T, int D> int few_d(const CachedArgs& a, bool early, cudaStream_t s) {
  return a.scores ? few_t<T, D, true>(a, early, s) : few_t<T, D, false>(a, early, s);
}
}  // namespace

int launch_attention_few(const CachedArgs& a, bool early, cudaStream_t s) {
  if (a.dtype == SWAPNET_BF16) return a.dim == 128 ? few_d<__nv_bfloat16, 128>(a, early, s) : few_d<__nv_bfloat16, 64>(a, early, s);
  return a.dim == 128 ? few_d<__half, 128>(a, early, s) : few_d<__half, 64>(a, early, s);
}

int launch_attention_join(const CachedArgs& a, cudaStream_t s) {
  const int rows = a.tokens * a.group;
  const int jb = a.splits > 1 ? (rows + kJoinThreads / 32 - 1) / (kJoinThreads / 32) : 0;
  const int wb = a.scores ? (a.max_seq + kJoinKeys - 1) / kJoinKeys : 0;
  if (jb + wb == 0) return SWAPNET_OK;
  const dim3 grid(jb + wb, a.kv_heads, a.n_seq);
  const size_t smem = a.scores ? rows * 2 * sizeof(float) : 0;
  return done(a.dtype == SWAPNET_BF16
                  ? launch(attention_join_kernel<__nv_bfloat16>, grid, kJoinThreads, smem, true, s, a, jb)
                  : launch(attention_join_kernel<__half>, grid, kJoinThreads, smem, true, s, a, jb),
              "cached attention join launch");
}

}  // namespace swapnet
