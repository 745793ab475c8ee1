// Attention of queries over a key-value cache held in 8 bits: few rows (decode
// steps, short runs) on warp-level matrix products.  fp32 arithmetic, fixed
// orders of summation.
//
// A value is code * scale with a scale for each block of rows and head.  The
// codes are exact as fp16 numbers, so they enter the products as they are; a
// key block's scale multiplies its scores, a value block's its probabilities.
#include <algorithm>
#include <cstring>
#include <string>
#include <type_traits>

#include "cached.cuh"
#include "internal.h"
#include "kernels.h"
#include "quant.cuh"

namespace swapnet {

namespace {

constexpr int kQfWarps = 4, kQfThreads = 32 * kQfWarps;
constexpr int kStep = 32;     // keys of a warp's step
constexpr int kQfStages = 2;
constexpr float kTop = 14.0f; // log2 of the largest p: times its scale's fraction below 2 it stays within fp16

template <int D, int NR> struct QfCfg {
  static constexpr int kTile = kStep * D;                 // bytes of a step's keys (or values)
  static constexpr int kSlot = 2 * kTile + 16;            // and the scales of its two 16-row parts
  static constexpr int kWarpRing = kQfStages * kSlot;
  static constexpr int kRows = 8 * NR;
  static constexpr int kOut = kQfWarps * kRows * D * 4;   // the warps' outputs, over the ring
  static constexpr int kRing = kQfWarps * kWarpRing > kOut ? kQfWarps * kWarpRing : kOut;
  static constexpr int kOffMl = kRing;
  static constexpr int kSmem = kOffMl + kQfWarps * kRows * 8;
};

// ---------------------------------------------------------- few-row attention
// One CTA: the keys [split] of a (sequence, key head) for up to 8 NR rows (row
// r: query r / group, head r % group of the group).  Its warps take steps of 32
// keys in turn and keep a softmax of their own (reference m, sum l, output O in
// registers), so nothing waits for another warp until the end.  The products
// have the keys as their 16 rows, S^T = K Q^T and O^T = V^T P^T, so that eight
// query rows fill a product's columns (queries as its rows would be half
// padding for up to eight of them):
//   S^T      codes of a 16-byte chunk of eight keys from one 8 x 8 matrix load: a
//            lane gets four neighbouring dims, whose fp16 pairs are the operand
//            of a product over 16 dims in another order, the same for Q
//   y        S^T * (key scale * query scale) + e, with value scale = 2^e * f
//   p        2^(y - m), m = the largest y so far less 14: at most 2^14; l adds
//            p 2^-e, and p f, at most 2^15, meets the values as two fp16 parts
//            (22 bits; what is below 2^-24 of them is lost, 2^-39 of the largest)
//   O^T      V^T from transposing 8 x 8 loads of byte pairs: a register holds
//            two keys of two dims, whose even and odd dims become rows of the
//            operand; P^T by transposing S^T's fragments (movmatrix)
// m grows only where a score passes the largest so far; until then nothing is
// rescaled and no lane asks another.
template <typename T, int D, int CODE, int NR>
__global__ void __launch_bounds__(kQfThreads, NR == 1 ? 3 : 2) attention_quant_few_kernel(const __grid_constant__ QuantArgs a, int row_tiles) {
  using F = QfCfg<D, NR>;
  extern __shared__ __align__(128) uint8_t smem[];
  float2* mls = reinterpret_cast<float2*>(smem + F::kOffMl);
  const int split = blockIdx.x / row_tiles, rt = blockIdx.x % row_tiles;
  const int kvh = blockIdx.y, b = blockIdx.z;
  const int warp = warp_index(), lane = threadIdx.x & 31;
  pdl_wait();
  pdl_launch_dependents();
  int len, count;
  if (!seq_sizes(a, b, &len, &count)) return;
  const int row0 = rt * F::kRows, rows = min(count * a.group - row0, F::kRows);
  if (rows <= 0) return;
  const int kmax = visible_limit(a, len, count, (row0 + rows - 1) / a.group), lim_min = visible_limit(a, len, count, row0 / a.group);
  const int steps = (kmax + kStep - 1) / kStep;
  const int g_begin = (int)((int64_t)steps * split / a.splits), g_end = (int)((int64_t)steps * (split + 1) / a.splits);

  uint8_t* ring = smem + warp * F::kWarpRing;
  const uint32_t ring_u = smem_u32(ring);
  constexpr int C = D / 16;  // 16-byte chunks of a row
  const int lr = lane / C, lc = lane % C;
  const int64_t head_at = (int64_t)b * a.seq_stride + (int64_t)kvh * D + lc * 16;
  const uint8_t *kb = static_cast<const uint8_t*>(a.k) + head_at, *vb = static_cast<const uint8_t*>(a.v) + head_at;
  const int64_t scale_at = ((int64_t)b * a.kv_heads + kvh) * a.blocks;
  auto load = [&](int g, int slot) {
    if (g < g_end) {
      const int j0 = g * kStep;
      const uint32_t dst = ring_u + (uint32_t)slot * F::kSlot;
#pragma unroll
      for (int i = 0; i < kStep * C / 32; ++i) {
        const int r = lr + i * (32 / C);
        const bool ok = j0 + r < len;
        const int64_t off = ok ? (int64_t)(j0 + r) * a.kv_stride : 0;
        cp_async_16(dst + swz8<D>(r, lc), kb + off, ok);
        cp_async_16(dst + F::kTile + swz8<D>(r, lc), vb + off, ok);
      }
      if (lane < 4) {  // key scales of the two parts, then the value scales
        const int j = j0 + (lane & 1) * 16;
        cp_async_4(dst + 2 * F::kTile + lane * 4, (lane < 2 ? a.k_scale : a.v_scale) + scale_at + (j < len ? j / a.block : 0), j < len);
      }
    }
    cp_async_commit();
  };
#pragma unroll
  for (int i = 0; i < kQfStages - 1; ++i) load(g_begin + warp + i * kQfWarps, i);

  // queries: the columns of S^T's products, as fp16
  uint32_t qf[NR][C][2];
  float qs[NR][2];  // of this lane's two rows of an output: log2(e) * scale * the query's own scale
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    const int r = 8 * n + (lane >> 2);
    const bool on = r < rows;
    const int t = on ? (row0 + r) / a.group : 0, h = on ? (row0 + r) % a.group : 0;
    const T* q = static_cast<const T*>(a.q) + ((int64_t)b * a.tokens + t) * a.q_stride + (int64_t)(kvh * a.group + h) * D + (lane & 3) * 4;
    uint2 raw[C];
#pragma unroll
    for (int c = 0; c < C; ++c) raw[c] = on ? *reinterpret_cast<const uint2*>(q + c * 16) : make_uint2(0u, 0u);
    const float s = query_fp16<T, C>(raw, qf[n]);
#pragma unroll
    for (int e = 0; e < 2; ++e) qs[n][e] = __shfl_sync(0xffffffffu, s, ((lane & 3) * 2 + e) * 4) * a.scale_log2;
  }
  int lim[NR][2];
#pragma unroll
  for (int n = 0; n < NR; ++n)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int r = 8 * n + (lane & 3) * 2 + e;
      lim[n][e] = r < rows ? visible_limit(a, len, count, (row0 + r) / a.group) : 0;
    }
  float m[NR][2], l[NR][2], o[D / 16][NR][4];
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    m[n][0] = m[n][1] = -INFINITY;
    l[n][0] = l[n][1] = 0.f;
#pragma unroll
    for (int d = 0; d < D / 16; ++d)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[d][n][e] = 0.f;
  }
  const uint32_t lrow = (lane & 7) + ((lane >> 3) & 1) * 8, lchunk = lane >> 4;  // of a four-matrix load
  int slot = 0;
  for (int g = g_begin + warp; g < g_end; g += kQfWarps) {
    int ahead = slot + kQfStages - 1;
    if (ahead >= kQfStages) ahead -= kQfStages;
    load(g + (kQfStages - 1) * kQfWarps, ahead);
    cp_async_wait<kQfStages - 1>();
    __syncwarp();
    const uint32_t ks_u = ring_u + (uint32_t)slot * F::kSlot, vs_u = ks_u + F::kTile;
    const float4 sc = *reinterpret_cast<const float4*>(ring + slot * F::kSlot + 2 * F::kTile);
    const int j0 = g * kStep;
    float y[2][NR][4];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) y[u][n][e] = 0.f;
#pragma unroll
      for (int c = 0; c < C; c += 2) {
        uint32_t kf[4];
        ldmatrix_x4(ks_u + swz8<D>(u * 16 + lrow, c + lchunk), kf);
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          const uint2 lo = pairs_near<CODE>(kf[2 * w]), hi = pairs_near<CODE>(kf[2 * w + 1]);
          const uint32_t af[4] = {lo.x, hi.x, lo.y, hi.y};
#pragma unroll
          for (int n = 0; n < NR; ++n) mma_16816<__half>(y[u][n], af, qf[n][c + w][0], qf[n][c + w][1]);
        }
      }
    }
    const bool masked = j0 + kStep > lim_min;  // some of these keys are hidden from some rows
    float ve[2], vf[2], vi[2];  // value scale = 2^ve * vf; 2^-ve
#pragma unroll
    for (int u = 0; u < 2; ++u) split_scale(u ? sc.w : sc.z, &ve[u], &vf[u], &vi[u]);
    float mx[NR][2];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      mx[n][0] = mx[n][1] = -INFINITY;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float x = fmaf(y[u][n][e], qs[n][e & 1] * (u ? sc.y : sc.x), ve[u]);
          if (masked && j0 + u * 16 + (lane >> 2) + 8 * (e >> 1) >= lim[n][e & 1]) x = -INFINITY;
          y[u][n][e] = x;
          mx[n][e & 1] = fmaxf(mx[n][e & 1], x);
        }
    }
    bool grow = false;
#pragma unroll
    for (int n = 0; n < NR; ++n) grow = grow || mx[n][0] - kTop > m[n][0] || mx[n][1] - kTop > m[n][1];
    if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        float al[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float x = mx[n][e];
          x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
          x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
          x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
          const float mn = fmaxf(m[n][e], x - kTop);
          al[e] = mn == -INFINITY ? 1.f : ex2(m[n][e] - mn);
          m[n][e] = mn;
          l[n][e] *= al[e];
        }
#pragma unroll
        for (int d = 0; d < D / 16; ++d)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[d][n][e] *= al[e & 1];
      }
    }
    if (CODE == kCodeE4M3 && masked) {
      // a hidden value row must not reach the rows that do not see it: its
      // codes may be no numbers (0 x NaN); a seen one's scale says so
      uint8_t* vs = ring + slot * F::kSlot + F::kTile;
#pragma unroll
      for (int i = 0; i < kStep * C / 32; ++i) {
        uint4* at = reinterpret_cast<uint4*>(vs + (lane + i * 32) * 16);
        const uint4 v = *at;
        *at = make_uint4(numbers_only(v.x), numbers_only(v.y), numbers_only(v.z), numbers_only(v.w));
      }
      __syncwarp();
    }
    uint32_t pt[2][NR][2][2];  // P^T: [part of the keys][rows][hi, lo][keys 0..7, 8..15]
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      const float base[2] = {m[n][0] == -INFINITY ? 0.f : m[n][0], m[n][1] == -INFINITY ? 0.f : m[n][1]};  // (nothing seen yet)
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float w[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float p = ex2(y[u][n][2 * h + e] - base[e]);
            l[n][e] = fmaf(p, vi[u], l[n][e]);
            w[e] = p * vf[u];
            if (masked && y[u][n][2 * h + e] == -INFINITY) w[e] = 0.f;  // (whatever the scale is)
          }
          const uint32_t hi = pack_pair<__half>(w[0], w[1]);
          const float2 back = unpack_pair<__half>(hi);
          pt[u][n][0][h] = transpose8(hi);
          pt[u][n][1][h] = transpose8(pack_pair<__half>(w[0] - back.x, w[1] - back.y));
        }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int c = 0; c < C; c += 2) {
        uint32_t vr[4];
        ldmatrix_x4_trans(vs_u + swz8<D>(u * 16 + lrow, c + lchunk), vr);
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          const uint2 lo = pairs_apart<CODE>(vr[2 * w]), hi = pairs_apart<CODE>(vr[2 * w + 1]);
          const uint32_t af[4] = {lo.x, lo.y, hi.x, hi.y};
#pragma unroll
          for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) mma_16816<__half>(o[c + w][n], af, pt[u][n][i][0], pt[u][n][i][1]);
        }
      }
    __syncwarp();  // the step has been read before its slot is filled again
    if (++slot == kQfStages) slot = 0;
  }
  // the warps' results meet in shared memory, in warp order
  cp_async_wait<0>();
  __syncthreads();
  float* ow = reinterpret_cast<float*>(smem) + warp * F::kRows * D;
#pragma unroll
  for (int n = 0; n < NR; ++n)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float x = l[n][e];
      x += __shfl_xor_sync(0xffffffffu, x, 4);
      x += __shfl_xor_sync(0xffffffffu, x, 8);
      x += __shfl_xor_sync(0xffffffffu, x, 16);
      const int r = 8 * n + (lane & 3) * 2 + e;
      if (lane < 4) mls[warp * F::kRows + r] = make_float2(m[n][e], x);
#pragma unroll
      for (int d = 0; d < D / 16; ++d)
        *reinterpret_cast<float2*>(ow + r * D + d * 16 + (lane >> 2) * 2) =
            make_float2(o[d][n][e], o[d][n][e + 2]);
    }
  __syncthreads();
  constexpr int V = D / 4;  // float4 per row
  for (int i = threadIdx.x; i < rows * V; i += kQfThreads) {
    const int r = i / V, c = i % V;
    float M = -INFINITY, L = 0.f;
#pragma unroll
    for (int w = 0; w < kQfWarps; ++w) M = fmaxf(M, mls[w * F::kRows + r].x);
    const float base = M == -INFINITY ? 0.f : M;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kQfWarps; ++w) {
      const float2 ml = mls[w * F::kRows + r];
      const float f = ex2(ml.x - base);
      const float4 z = reinterpret_cast<const float4*>(smem)[(w * F::kRows + r) * V + c];
      L = fmaf(ml.y, f, L);
      if (f != 0.f) {
        x.x = fmaf(z.x, f, x.x);
        x.y = fmaf(z.y, f, x.y);
        x.z = fmaf(z.z, f, x.z);
        x.w = fmaf(z.w, f, x.w);
      }
    }
    const int rr = row0 + r;
    const int64_t slot_r = (((int64_t)b * a.kv_heads + kvh) * a.splits + split) * a.tokens * a.group + rr;
    if (a.splits > 1) {
      if (c == 0) reinterpret_cast<float2*>(a.ml)[slot_r] = make_float2(M, L);
      if (M != -INFINITY) reinterpret_cast<float4*>(a.part)[slot_r * V + c] = x;
      continue;
    }
    const int t = rr / a.group, hd = kvh * a.group + rr % a.group;
    const float inv = L > 0.f ? 1.0f / L : (L == 0.f ? 0.f : L);  // (a NaN stays one)
    T* to = static_cast<T*>(a.out) + ((int64_t)b * a.tokens + t) * a.out_stride + (int64_t)hd * D + c * 4;
    *reinterpret_cast<uint2*>(to) = make_uint2(pack_pair<T>(x.x * inv, x.y * inv), pack_pair<T>(x.z * inv, x.w * inv));
    if (c == 0 && a.lse) a.lse[((int64_t)b * a.heads + hd) * a.tokens + t] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
  }
}

template <typename T, int D, int CODE, int NR> int few_t(const QuantArgs& a, cudaStream_t s) {
  static std::atomic<uint64_t> known{0};
  using F = QfCfg<D, NR>;
  const auto kern = attention_quant_few_kernel<T, D, CODE, NR>;
  if (attr_needed(known)) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, F::kSmem);
    if (e != cudaSuccess) SN_FAIL(SWAPNET_ERR_CUDA, std::string("quantised attention: ") + cudaGetErrorString(e));
    attr_set(known);
  }
  const int row_tiles = (a.tokens * a.group + F::kRows - 1) / F::kRows;
  kern<<<dim3(a.splits * row_tiles, a.kv_heads, a.n_seq), kQfThreads, F::kSmem, s>>>(a, row_tiles);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) SN_FAIL(SWAPNET_ERR_CUDA, std::string("quantised attention launch: ") + cudaGetErrorString(e));
  return SWAPNET_OK;
}
template <typename T, int D, int CODE> int few_r(const QuantArgs& a, cudaStream_t s) {
  return a.tokens * a.group <= 8 ? few_t<T, D, CODE, 1>(a, s) : few_t<T, D, CODE, 2>(a, s);
}
template <typename T, int D> int few_c(const QuantArgs& a, cudaStream_t s) {
  return a.code == kCodeI8 ? few_r<T, D, kCodeI8>(a, s) : few_r<T, D, kCodeE4M3>(a, s);
}

}  // namespace

int launch_quant_few(const QuantArgs& a, cudaStream_t s) {
  if (a.dtype == SWAPNET_BF16) return a.dim == 128 ? few_c<__nv_bfloat16, 128>(a, s) : few_c<__nv_bfloat16, 64>(a, s);
  return a.dim == 128 ? few_c<__half, 128>(a, s) : few_c<__half, 64>(a, s);
}

}  // namespace swapnet
