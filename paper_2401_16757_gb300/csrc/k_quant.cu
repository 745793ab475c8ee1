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

#include "internal.h"
#include "kernels.h"
#include "quant.cuh"

namespace swapnet {

namespace {

constexpr int kStep = 32;     // keys of a warp's step
constexpr int kQfStages = 2;

// W warps; up to 8 NR rows.
template <int D, int NR, int W> struct QfCfg {
  static constexpr int kThreads = 32 * W;
  static constexpr int kTile = kStep * D;                 // bytes of a step's keys (or values)
  static constexpr int kSlot = 2 * kTile + 16;            // and the scales of its two 16-row parts
  static constexpr int kWarpRing = kQfStages * kSlot;
  static constexpr int kRows = 8 * NR;
  static constexpr int kOut = W * kRows * D * 4;          // the warps' outputs, over the ring
  static constexpr int kRing = W * kWarpRing > kOut ? W * kWarpRing : kOut;
  static constexpr int kOffMl = kRing;
  static constexpr int kOffQ = kOffMl + W * kRows * 8;    // NR 4: queries as operands, a lane's 8 bytes side by side
  static constexpr int kOffQs = kOffQ + (NR > 2 ? NR * (D / 16) * 256 : 0);
  static constexpr int kOffNear = kOffQs + (NR > 2 ? kRows * 4 : 0);
  static constexpr int kSmem = kOffNear + kNear * 8;
  // CTAs of an SM, by registers and shared memory
  static constexpr int kResident = quant_few_resident(kRows, D);
};

// ---------------------------------------------------------- few-row attention
// A unit is up to 8 NR rows of a (sequence, key head) (row r: query r / group,
// head r % group of the group).  A CTA takes one unit, or an equal run of all
// units' tiles of 128 keys, whose shared units meet in the join (as the
// tensor-core kernel's runs do).  Its warps take steps of 32 keys in turn and
// keep a softmax of their own (reference m, sum l, output O in registers), so
// nothing waits for another warp until the end of a piece.  The products have
// the keys as their 16 rows, S^T = K Q^T and O^T = V^T P^T, so that eight query
// rows fill a product's columns (queries as its rows would be half padding for
// up to eight of them):
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
// Keys and values pass through two places a warp each, which are filled again
// as soon as they have been read: the keys once the scores are there, so that
// one and a half steps' loads are on the way while a step is computed.
// m grows only where a score passes the largest so far; until then nothing is
// rescaled and no lane asks another.  With NR 4 the outputs fill half of the
// registers, and the queries stay in shared memory.
// Measured: one token of 64 sequences, 8 key heads (group 4) of 128, I8, up to
// 16384 rows (1.57 GB): 254 to 268 us by the card, 5.8 to 6.2 TB/s; the same loads without
// any product take 252, a copy of as many bytes 238, so that DRAM bounds it.  12
// rows of 4 key heads of 64, E4M3, on 131001 rows: 26.6 us, of which start, end
// and join are 11.  32 rows of 32 x 8 (sequence, head)s on up to 8000 rows (0.34
// GB): 131 us: two warps a scheduler (255 registers), whose products fill the
// pipe to 0.46 and whose instructions issue in 0.41 of the cycles
// (k_quant_keys.cu takes that call: 112).  One row of 32
// heads on 543 rows: 9.2 us, five tiles of 1.2 us and the launch; one row of 8 heads on
// 100 rows 5.0, all of it latency.  Consecutive products of the same sums are kept
// apart (decode 274 to 262 us, in the same form).
template <typename T, int D, int CODE, int NR, int W>
__global__ void __launch_bounds__(32 * W, QfCfg<D, NR, W>::kResident)
    attention_quant_few_kernel(const __grid_constant__ QuantArgs a, int queries, int nrt) {
  using F = QfCfg<D, NR, W>;
  extern __shared__ __align__(128) uint8_t smem[];
  float2* mls = reinterpret_cast<float2*>(smem + F::kOffMl);
  int2* near = reinterpret_cast<int2*>(smem + F::kOffNear);
  int64_t* sched = reinterpret_cast<int64_t*>(smem);
  const int warp = warp_index(), lane = threadIdx.x & 31;
  pdl_wait();
  pdl_launch_dependents();
  Cursor cur;
  const Run r_ = start_run(a, cur, near, sched, queries, nrt);
  const int kvh = r_.kvh;
  __syncthreads();  // (sched's place is the ring's)

  uint8_t* ring = smem + warp * F::kWarpRing;
  const uint32_t ring_u = smem_u32(ring);
  constexpr int C = D / 16;  // 16-byte chunks of a row
  const int lr = lane / C, lc = lane % C;
  const uint32_t lrow = (lane & 7) + ((lane >> 3) & 1) * 8, lchunk = lane >> 4;  // of a four-matrix load
  int64_t at_tile = r_.first;
#pragma unroll 1
  while (cur.step(a, nrt, queries)) {
    const int b = cur.b, len = cur.z.len, count = cur.z.count, t0 = cur.rt * queries;
    const int rows = min(queries, count - t0) * a.group;
    const bool whole = cur.i0 == 0 && cur.n == cur.z.tiles;
    const int kmax = visible_limit(a, len, count, t0 + (rows - 1) / a.group), lim_min = visible_limit(a, len, count, t0);
    const int k_end = min((cur.i0 + cur.n) * kKeys, kmax), k_begin = cur.i0 * kKeys;
    const int steps = k_end > k_begin ? (k_end - k_begin + kStep - 1) / kStep : 0;
    const int64_t head_at = (int64_t)b * a.seq_stride + (int64_t)k_begin * a.kv_stride + (int64_t)kvh * D + lc * 16;
    const uint8_t *kb = static_cast<const uint8_t*>(a.k) + head_at, *vb = static_cast<const uint8_t*>(a.v) + head_at;
    const int64_t scale_at = ((int64_t)b * a.kv_heads + kvh) * a.blocks;
    auto load = [&](int g, int slot, bool keys) {
      if (g < steps) {
        const int j0 = g * kStep;
        const uint32_t dst = ring_u + (uint32_t)slot * F::kSlot;
#pragma unroll
        for (int i = 0; i < kStep * C / 32; ++i) {
          const int r = lr + i * (32 / C);
          const bool ok = k_begin + j0 + r < len;
          const int64_t off = ok ? (int64_t)(j0 + r) * a.kv_stride : 0;
          if (keys)
            cp_async_16(dst + swz8<D>(r, lc), kb + off, ok);
          else
            cp_async_16(dst + F::kTile + swz8<D>(r, lc), vb + off, ok);
        }
        if (keys && lane < 4) {  // key scales of the two parts, then the value scales
          const int j = k_begin + j0 + (lane & 1) * 16;
          cp_async_4(dst + 2 * F::kTile + lane * 4, (lane < 2 ? a.k_scale : a.v_scale) + scale_at + (j < len ? j >> a.block_log2 : 0), j < len);
        }
      }
      cp_async_commit();
    };
#pragma unroll
    for (int i = 0; i < kQfStages; ++i) {
      load(warp + i * W, i, true);
      load(warp + i * W, i, false);
    }

    // queries: the columns of S^T's products, as fp16
    uint32_t qf[NR > 2 ? 1 : NR][C][2];
    float qs[NR][2];  // of this lane's two rows of an output: log2(e) * scale * the query's own scale
    auto query = [&](int n, uint32_t (&to)[C][2]) {
      const int r = 8 * n + (lane >> 2);
      const bool on = r < rows;
      const int t = t0 + (on ? r / a.group : 0), h = on ? r % a.group : 0;
      const T* q = static_cast<const T*>(a.q) + ((int64_t)b * a.tokens + t) * a.q_stride + (int64_t)(kvh * a.group + h) * D + (lane & 3) * 4;
      uint2 raw[C];
#pragma unroll
      for (int c = 0; c < C; ++c) raw[c] = on ? *reinterpret_cast<const uint2*>(q + c * 16) : make_uint2(0u, 0u);
      return query_fp16<T, C>(raw, to) * a.scale_log2;
    };
    uint2* q_frags = reinterpret_cast<uint2*>(smem + F::kOffQ) + lane;  // [n][c][lane]
    if (NR > 2) {
      float* q_scales = reinterpret_cast<float*>(smem + F::kOffQs);
#pragma unroll 1
      for (int n = warp; n < NR; n += W) {
        const float s = query(n, qf[0]);
#pragma unroll
        for (int c = 0; c < C; ++c) q_frags[(n * C + c) * 32] = make_uint2(qf[0][c][0], qf[0][c][1]);
        if ((lane & 3) == 0) q_scales[8 * n + (lane >> 2)] = s;
      }
      __syncthreads();
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        const float2 x = *reinterpret_cast<const float2*>(q_scales + 8 * n + (lane & 3) * 2);
        qs[n][0] = x.x;
        qs[n][1] = x.y;
      }
    } else {
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        const float s = query(n, qf[n]);
#pragma unroll
        for (int e = 0; e < 2; ++e) qs[n][e] = __shfl_sync(0xffffffffu, s, ((lane & 3) * 2 + e) * 4);
      }
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
    int slot = 0;
#pragma unroll 1
    for (int g = warp; g < steps; g += W) {
      cp_async_wait<2 * kQfStages - 1>();  // (all but these values and the keys and values of the steps ahead)
      __syncwarp();
      const uint32_t ks_u = ring_u + (uint32_t)slot * F::kSlot, vs_u = ks_u + F::kTile;
      const float4 sc = *reinterpret_cast<const float4*>(ring + slot * F::kSlot + 2 * F::kTile);
      const int j0 = k_begin + g * kStep;
      float y[2][NR][4];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) y[u][n][e] = 0.f;
#pragma unroll
      for (int c = 0; c < C; c += 2) {
        uint32_t kf[2][4];
#pragma unroll
        for (int u = 0; u < 2; ++u) ldmatrix_x4(ks_u + swz8<D>(u * 16 + lrow, c + lchunk), kf[u]);
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          uint2 q[NR];
#pragma unroll
          for (int n = 0; n < NR; ++n) q[n] = NR > 2 ? q_frags[(n * C + c + w) * 32] : make_uint2(qf[NR > 2 ? 0 : n][c + w][0], qf[NR > 2 ? 0 : n][c + w][1]);
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const uint2 lo = pairs_near<CODE>(kf[u][2 * w]), hi = pairs_near<CODE>(kf[u][2 * w + 1]);
            const uint32_t af[4] = {lo.x, hi.x, lo.y, hi.y};
#pragma unroll
            for (int n = 0; n < NR; ++n) mma_16816<__half>(y[u][n], af, q[n].x, q[n].y);
          }
        }
      }
      __syncwarp();  // the keys have been read before their place is filled again
      load(g + kQfStages * W, slot, true);
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
          for (int e = 0; e < 4; ++e) y[u][n][e] = fmaf(y[u][n][e], qs[n][e & 1] * (u ? sc.y : sc.x), ve[u]);
        if (masked) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int r = 8 * n + (lane & 3) * 2 + (e & 1);
            const int lim = r < rows ? visible_limit(a, len, count, t0 + r / a.group) : 0;
#pragma unroll
            for (int u = 0; u < 2; ++u)
              if (j0 + u * 16 + (lane >> 2) + 8 * (e >> 1) >= lim) y[u][n][e] = -INFINITY;
          }
        }
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e) mx[n][e & 1] = fmaxf(mx[n][e & 1], y[u][n][e]);
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
      cp_async_wait<2 * kQfStages - 1>();
      __syncwarp();
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
          uint32_t af[2][4];
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            const uint2 lo = pairs_apart<CODE>(vr[2 * w]), hi = pairs_apart<CODE>(vr[2 * w + 1]);
            af[w][0] = lo.x, af[w][1] = lo.y, af[w][2] = hi.x, af[w][3] = hi.y;
          }
          // (the parts apart: a product waits for the one before it of the same sums)
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int w = 0; w < 2; ++w)
#pragma unroll
              for (int n = 0; n < NR; ++n) mma_16816<__half>(o[c + w][n], af[w], pt[u][n][i][0], pt[u][n][i][1]);
        }
      __syncwarp();  // and the values before theirs
      load(g + kQfStages * W, slot, false);
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
          *reinterpret_cast<float2*>(ow + r * D + d * 16 + (lane >> 2) * 2) = make_float2(o[d][n][e], o[d][n][e + 2]);
      }
    __syncthreads();
    constexpr int V = D / 4;  // float4 per row
    for (int i = threadIdx.x; i < rows * V; i += F::kThreads) {
      const int r = i / V, c = i % V;
      float M = -INFINITY, L = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) M = fmaxf(M, mls[w * F::kRows + r].x);
      const float base = M == -INFINITY ? 0.f : M;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < W; ++w) {
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
      if (!whole) {
        const int64_t at = ((int64_t)2 * blockIdx.x + (cur.i0 == 0 ? 1 : 0)) * F::kRows + r;
        if (c == 0) reinterpret_cast<float2*>(a.ml)[at] = make_float2(M, L);
        if (M != -INFINITY) reinterpret_cast<float4*>(a.part)[at * V + c] = x;
        continue;
      }
      const int t = t0 + r / a.group, hd = kvh * a.group + r % a.group;
      const float inv = L > 0.f ? 1.0f / L : (L == 0.f ? 0.f : L);  // (a NaN stays one)
      T* to = static_cast<T*>(a.out) + ((int64_t)b * a.tokens + t) * a.out_stride + (int64_t)hd * D + c * 4;
      *reinterpret_cast<uint2*>(to) = make_uint2(pack_pair<T>(x.x * inv, x.y * inv), pack_pair<T>(x.z * inv, x.w * inv));
      if (c == 0 && a.lse) a.lse[((int64_t)b * a.heads + hd) * a.tokens + t] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
    }
    if (a.splits != 1 && cur.i0 == 0 && threadIdx.x == 0) record_unit(a, r_, cur, nrt, at_tile);
    at_tile += cur.n;
    __syncthreads();  // the results have been read before the ring is filled again
  }
}

// ----------------------------------------------------------------- the join
// A unit (blockIdx.y) that several runs shared: their pieces in order, from the
// CTA that began it, each with m, l and O relative to its m.  A CTA holds at
// most two pieces that are not whole units: the rest of one that began before
// its run (slot 2 c) and the start of one that goes on behind it (slot 2 c + 1).
// A warp per row, or all warps of the block where that takes fewer rounds of
// loads, each of eight pieces.  Bound by its chain (launch, record, pieces, the
// warps' results): 5 to 6 us for 4 units of 114 pieces.
constexpr int kQjWarps = 16, kQjAhead = 8;
template <typename T>
__global__ void __launch_bounds__(32 * kQjWarps)
    attention_quant_join_kernel(const __grid_constant__ QuantArgs a, int queries, int row_tile, int nrt) {
  __shared__ float4 so[kQjWarps][32];
  __shared__ float2 sm[kQjWarps];
  const int lane = threadIdx.x & 31, warp = warp_index();
  const int kvh = blockIdx.y % a.kv_heads, pair = blockIdx.y / a.kv_heads, b = pair / nrt, rt = pair % nrt;
  pdl_wait();
  const int2 size = seq_size(a, b), u = reinterpret_cast<const int2*>(a.units)[blockIdx.y];
  if (pair_size(a, size, rt, queries).tiles == 0 || u.y == 0) return;  // (an empty unit has no record)
  const int t0 = rt * queries, rows = min(queries, size.y - t0) * a.group, pieces = u.y;
  const int blocks = gridDim.x, per_warp = (rows + kQjWarps * blocks - 1) / (kQjWarps * blocks), per_block = (rows + blocks - 1) / blocks;
  const bool many = per_block * ((pieces + kQjAhead * kQjWarps - 1) / (kQjAhead * kQjWarps) + 1) < per_warp * ((pieces + kQjAhead - 1) / kQjAhead);  // (+ 1: the warps' results meet)
  const int V = a.dim / 4, first = many ? warp : 0, step = many ? kQjWarps : 1;
  const float2* ml = reinterpret_cast<const float2*>(a.ml);
  const float4* part = reinterpret_cast<const float4*>(a.part);
  for (int r0 = blockIdx.x * (many ? 1 : kQjWarps); r0 < rows; r0 += gridDim.x * (many ? 1 : kQjWarps)) {
    const int rl = many ? r0 : r0 + warp;
    const bool own = rl < rows;
    auto slot = [&](int p) { return ((int64_t)2 * (u.x + (int64_t)p * a.kv_heads) + (p == 0 ? 1 : 0)) * row_tile + rl; };
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
    for (int p0 = first; own && p0 < pieces; p0 += kQjAhead * step) {
      float2 s[kQjAhead];
      float4 y[kQjAhead];
#pragma unroll
      for (int i = 0; i < kQjAhead; ++i) {
        const int p = p0 + i * step;
        s[i] = p < pieces ? ml[slot(p)] : make_float2(-INFINITY, 0.f);
        y[i] = p < pieces && lane < V ? part[slot(p) * V + lane] : make_float4(0.f, 0.f, 0.f, 0.f);
      }
#pragma unroll
      for (int i = 0; i < kQjAhead; ++i) take(s[i], y[i]);
    }
    if (many) {
      so[warp][lane] = x;
      if (lane == 0) sm[warp] = make_float2(M, L);
      __syncthreads();
      if (warp == 0) {
#pragma unroll
        for (int i = 1; i < kQjWarps; ++i) take(sm[i], so[i][lane]);
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

template <typename T, int D, int CODE, int NR, int W> int few_t(const QuantArgs& a, int ctas, cudaStream_t s) {
  static std::atomic<uint64_t> known{0};
  using F = QfCfg<D, NR, W>;
  const auto kern = attention_quant_few_kernel<T, D, CODE, NR, W>;
  if (attr_needed(known)) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, F::kSmem);
    if (e != cudaSuccess) SN_FAIL(SWAPNET_ERR_CUDA, std::string("quantised attention: ") + cudaGetErrorString(e));
    attr_set(known);
  }
  const int queries = std::min(F::kRows / a.group, a.tokens), nrt = (a.tokens + queries - 1) / queries;
  kern<<<ctas, F::kThreads, F::kSmem, s>>>(a, queries, nrt);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) SN_FAIL(SWAPNET_ERR_CUDA, std::string("quantised attention launch: ") + cudaGetErrorString(e));
  return a.splits == 1 ? SWAPNET_OK : launch_quant_join(a, queries, F::kRows, nrt, s);
}
template <typename T, int D, int CODE> int few_r(const QuantArgs& a, int ctas, int row_tile, cudaStream_t s) {
  return row_tile == 8 ? few_t<T, D, CODE, 1, 4>(a, ctas, s) : row_tile == 16 ? few_t<T, D, CODE, 2, 4>(a, ctas, s) : few_t<T, D, CODE, 4, 4>(a, ctas, s);
}
template <typename T, int D> int few_c(const QuantArgs& a, int ctas, int row_tile, cudaStream_t s) {
  return a.code == kCodeI8 ? few_r<T, D, kCodeI8>(a, ctas, row_tile, s) : few_r<T, D, kCodeE4M3>(a, ctas, row_tile, s);
}

}  // namespace

int launch_quant_join(const QuantArgs& a, int queries, int row_tile, int nrt, cudaStream_t s) {
  // about four blocks per SM, but at least a warp and at most a block for a row
  const int64_t units = (int64_t)a.n_seq * nrt * a.kv_heads;
  const int rows = queries * a.group, least = (rows + kQjWarps - 1) / kQjWarps;
  cudaLaunchConfig_t cfg;
  std::memset(&cfg, 0, sizeof(cfg));
  cfg.gridDim = dim3(std::min(rows, std::max(least, (int)(4 * kSms / units))), (unsigned)units);
  cfg.blockDim = dim3(32 * kQjWarps);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const auto kern = a.dtype == SWAPNET_BF16 ? attention_quant_join_kernel<__nv_bfloat16> : attention_quant_join_kernel<__half>;
  cudaError_t e = cudaLaunchKernelEx(&cfg, kern, a, queries, row_tile, nrt);
  if (e == cudaSuccess) e = cudaGetLastError();
  if (e != cudaSuccess) SN_FAIL(SWAPNET_ERR_CUDA, std::string("quantised attention join launch: ") + cudaGetErrorString(e));
  return SWAPNET_OK;
}

int launch_quant_few(const QuantArgs& a, int ctas, int row_tile, cudaStream_t s) {
  if (a.dtype == SWAPNET_BF16) return a.dim == 128 ? few_c<__nv_bfloat16, 128>(a, ctas, row_tile, s) : few_c<__nv_bfloat16, 64>(a, ctas, row_tile, s);
  return a.dim == 128 ? few_c<__half, 128>(a, ctas, row_tile, s) : few_c<__half, 64>(a, ctas, row_tile, s);
}

}  // namespace swapnet
