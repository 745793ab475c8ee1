// Rows appended to a key-value cache: norms of queries and keys, position
// rotation, and for a cache of 8 bits the codes and scales of the blocks that
// the rows lie in, all in one launch.  fp32 arithmetic, fixed orders of
// summation.
//
// What a row needs is its own (norm, rotation), what a code needs is its
// block's largest magnitude; so a CTA holds a whole block of one head in
// registers between the two, and the rows are read once and written once.
//
// Measured (launches of a CUDA graph, inputs larger than L2 or in turn): 28600
// rows of 8 heads of 128 bf16 put into I8 31 us, 5.7 TB/s; 12000 tokens of 16
// query and 2 key heads, norms, three position axes, blocks of 128 rows 29 us,
// 4.1 TB/s; 512 tokens of 32 heads 9.0; one token of 64 sequences, 32 query and
// 8 key heads, blocks of 64 rows 8.5; 10200 tokens of 12 and 4 heads of 64 into
// a 16-bit cache 14.2, 3.7 TB/s; one token of one sequence 3.1, of which the
// launch is 2.  Bound by instructions beside the memory: a warp's row (8 elements a lane) takes about
// 100 with norm and rotation, which is why arithmetic is two numbers at a time,
// a pair of the rotation lies in one lane, and angles come from a series and
// serve eight heads (rows of 12000 tokens: 96 us with a function call for every
// pair and head, one element at a time).
#include <algorithm>
#include <string>
#include <type_traits>

#include "device.cuh"
#include "internal.h"
#include "kernels.h"
#include "quant.h"

namespace swapnet {

namespace {

constexpr int kMaxThreads = 256;

// Two fp32 numbers at a time (one instruction each).
__device__ __forceinline__ float2 fma2(float2 x, float2 y, float2 z) {
  float2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(reinterpret_cast<unsigned long long&>(r))
      : "l"(reinterpret_cast<unsigned long long&>(x)), "l"(reinterpret_cast<unsigned long long&>(y)),
        "l"(reinterpret_cast<unsigned long long&>(z)));
  return r;
}
__device__ __forceinline__ float2 mul2(float2 x, float2 y) {
  float2 r;
  asm("mul.rn.f32x2 %0, %1, %2;"
      : "=l"(reinterpret_cast<unsigned long long&>(r))
      : "l"(reinterpret_cast<unsigned long long&>(x)), "l"(reinterpret_cast<unsigned long long&>(y)));
  return r;
}
__device__ __forceinline__ float2 add2(float2 x, float2 y) {
  float2 r;
  asm("add.rn.f32x2 %0, %1, %2;"
      : "=l"(reinterpret_cast<unsigned long long&>(r))
      : "l"(reinterpret_cast<unsigned long long&>(x)), "l"(reinterpret_cast<unsigned long long&>(y)));
  return r;
}
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// A row of D elements is held by D / 8 neighbouring lanes, in each four pairs
// (u, v), 4 chunk .. 4 chunk + 3, a 32-bit word each: of neighbouring elements,
// or for a rotation of halves of one element of each half, which are brought
// together when they are read.
struct Place {
  int a, b;     // where the two quads of elements are
  bool halves;  // the first holds the u, the second the v (else pairs of neighbours)
};
__device__ __forceinline__ Place place_of(const AppendArgs& g, int chunk, bool turned) {
  if (turned && g.halves && chunk * 8 < g.rope_dim) return Place{chunk * 4, g.rope_dim / 2 + chunk * 4, true};
  return Place{chunk * 8, chunk * 8 + 4, false};
}
// (split: whether some lane's quads are no neighbours)
__device__ __forceinline__ uint4 load8(const void* row, const Place& p, bool split) {
  const uint2* at = static_cast<const uint2*>(row);
  if (!split) return *reinterpret_cast<const uint4*>(at + p.a / 4);
  const uint2 x = at[p.a / 4], y = at[p.b / 4];
  return make_uint4(x.x, x.y, y.x, y.y);
}
__device__ __forceinline__ uint4 to_pairs(const uint4& v, bool halves) {
  if (!halves) return v;
  return make_uint4(__byte_perm(v.x, v.z, 0x5410), __byte_perm(v.x, v.z, 0x7632), __byte_perm(v.y, v.w, 0x5410), __byte_perm(v.y, v.w, 0x7632));
}
__device__ __forceinline__ uint4 from_pairs(const uint4& v, bool halves) {
  if (!halves) return v;
  return make_uint4(__byte_perm(v.x, v.y, 0x5410), __byte_perm(v.z, v.w, 0x5410), __byte_perm(v.x, v.y, 0x7632), __byte_perm(v.z, v.w, 0x7632));
}
__device__ __forceinline__ void store8(void* row, const Place& p, bool split, uint4 v) {
  uint2* at = static_cast<uint2*>(row);
  if (!split) {
    *reinterpret_cast<uint4*>(at + p.a / 4) = v;
    return;
  }
  at[p.a / 4] = make_uint2(v.x, v.y);
  at[p.b / 4] = make_uint2(v.z, v.w);
}

template <typename T> __device__ __forceinline__ float2 unpack2(uint32_t x);
template <> __device__ __forceinline__ float2 unpack2<__half>(uint32_t x) { return __half22float2(reinterpret_cast<const __half2&>(x)); }
template <> __device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t x) {
  return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
}
template <typename T> __device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// The pairs of four words, u and v apart, two pairs to a register pair.
struct Pairs {
  float2 u[2], v[2];
};
template <typename T> __device__ __forceinline__ Pairs pairs_of(const uint4& w) {
  const float2 a = unpack2<T>(w.x), b = unpack2<T>(w.y), c = unpack2<T>(w.z), d = unpack2<T>(w.w);
  return Pairs{{make_float2(a.x, b.x), make_float2(c.x, d.x)}, {make_float2(a.y, b.y), make_float2(c.y, d.y)}};
}
template <typename T> __device__ __forceinline__ uint4 words_of(const Pairs& p) {
  return make_uint4(pack2<T>(p.u[0].x, p.v[0].x), pack2<T>(p.u[0].y, p.v[0].y), pack2<T>(p.u[1].x, p.v[1].x), pack2<T>(p.u[1].y, p.v[1].y));
}

// Norm of a row: x / sqrt(mean + eps) * gain.  All lanes of the warp.
template <int D> __device__ __forceinline__ void norm(Pairs& x, const Pairs& gain, float eps) {
  float2 q = mul2(x.u[0], x.u[0]);
  q = fma2(x.u[1], x.u[1], q);
  q = fma2(x.v[0], x.v[0], q);
  q = fma2(x.v[1], x.v[1], q);
  float s = q.x + q.y;
#pragma unroll
  for (int off = D / 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
  const float2 r = both(rsqrtf(s * (1.0f / D) + eps));
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    x.u[i] = mul2(mul2(x.u[i], r), gain.u[i]);
    x.v[i] = mul2(mul2(x.v[i], r), gain.v[i]);
  }
}

// cos and sin of the angles of this lane's pairs at a token's position.  The
// angle in turns is position * (hi + lo), |hi| at most 1/2: the product with hi
// is split into what it rounds to (below 2^23) and the rest (fma, at most 1/4),
// whole turns are taken off, and only then is it an angle.  Off by: the last sum
// of turns, up to 3/4, 2^-25; the one before it, up to 1/4, 2^-26; lo's rounding
// times the position 2^-26; 2 pi and the product with it 2^-24 in all: below
// 2^-21 (2^-22 for positions below 4096), beside 2^-49 of position * frequency
// that the frequency in 64 bits is off by.  Less the
// nearest quarter turn it is at most pi / 4, where Taylor's series for sine
// (to x^9) and cosine (to x^8) are within 2^-25; the quarters exchange and
// negate the two.  Two pairs at a time: sincosf's share of the rows of 12000
// tokens was a third of their time.
struct Turn {
  float2 c[2], s[2];
};
__device__ __forceinline__ void turn_of(const AppendArgs& a, const float2* turns_of, int b, int t, int pos, int chunk, Turn* w) {
  int at_axis[3] = {pos, pos, pos};
  const bool axes = a.positions && a.axis1 < a.rope_dim / 2;
  if (a.positions) {
    const int* from = a.positions + (int64_t)b * a.tokens + t;
    const int64_t step = (int64_t)a.n_seq * a.tokens;
    at_axis[0] = from[0];
    if (axes) {
      at_axis[1] = from[step];
      at_axis[2] = from[2 * step];
    } else {
      at_axis[1] = at_axis[2] = at_axis[0];
    }
    if ((unsigned)(at_axis[0] | at_axis[1] | at_axis[2]) >= (unsigned)kMaxPosition) {  // (a power of two)
      atomicExch(a.err, kDevErrBounds);
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if ((unsigned)at_axis[i] >= (unsigned)kMaxPosition) at_axis[i] = 0;
    }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float4 f = reinterpret_cast<const float4*>(turns_of)[2 * chunk + i];
    float at[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int pair = 4 * chunk + 2 * i + e;
      at[e] = (float)(!axes || pair < a.axis1 ? at_axis[0] : pair < a.axis2 ? at_axis[1] : at_axis[2]);
    }
    const float2 p = make_float2(at[0], at[1]), minus = both(-1.0f), half = both(12582912.0f);  // 1.5 * 2^23: adding it rounds to whole numbers
    const float2 h = make_float2(f.x, f.z), whole = mul2(p, h), rest = fma2(p, h, mul2(whole, minus));
    const float2 turns = add2(fma2(make_float2(rintf(whole.x), rintf(whole.y)), minus, whole), fma2(p, make_float2(f.y, f.w), rest));
    const float2 k = fma2(turns, both(4.0f), half);  // the nearest quarter in the low bits
    const float2 x = mul2(fma2(add2(k, mul2(half, minus)), both(-0.25f), turns), both(6.283185307179586f));
    const float2 y = mul2(x, x);
    float2 sn = fma2(y, both(1.0f / 362880), both(-1.0f / 5040)), cs = fma2(y, both(1.0f / 40320), both(-1.0f / 720));
    sn = fma2(y, sn, both(1.0f / 120));
    cs = fma2(y, cs, both(1.0f / 24));
    sn = fma2(y, sn, both(-1.0f / 6));
    cs = fma2(y, cs, both(-0.5f));
    sn = fma2(mul2(x, y), sn, x);
    cs = fma2(y, cs, both(1.0f));
    float c[2] = {cs.x, cs.y}, s[2] = {sn.x, sn.y};
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const uint32_t q = __float_as_uint(e ? k.y : k.x);
      const float u = q & 1 ? s[e] : c[e], v = q & 1 ? c[e] : s[e];
      c[e] = __uint_as_float(__float_as_uint(u) ^ ((q + 1) << 30 & 0x80000000u));
      s[e] = __uint_as_float(__float_as_uint(v) ^ (q << 30 & 0x80000000u));
    }
    w->c[i] = make_float2(c[0], c[1]);
    w->s[i] = make_float2(s[0], s[1]);
  }
}
__device__ __forceinline__ void rotate(Pairs& x, const Turn& w) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float2 u = x.u[i], v = x.v[i], minus = both(-1.0f);
    x.u[i] = fma2(u, w.c[i], mul2(mul2(v, minus), w.s[i]));
    x.v[i] = fma2(v, w.c[i], mul2(u, w.s[i]));
  }
}

// A sequence's rows before and its new ones; false (reported) where they are out of range.
__device__ __forceinline__ bool append_sizes(const AppendArgs& a, int b, int* len, int* count) {
  const int n = a.lens[b], c = a.counts ? a.counts[b] : a.tokens;
  *len = n;
  *count = c;
  if (n < 0 || c < 0 || c > a.tokens || n > a.max_seq || c > a.max_seq - n) {
    if (threadIdx.x == 0) atomicExch(a.err, kDevErrBounds);
    return false;
  }
  return true;
}

// ---------------------------------------------------------- rows in 16 bits
// Queries, and for a 16-bit cache keys and values, kind after kind in CTAs of
// their own.  D / 8 lanes take kHeads heads of one token, so that its angles
// serve all of them: eight beside blocks of codes (12000 tokens 29 us, with four
// 35), four in a 16-bit cache's call (14.2 us; with eight, which leave too few
// CTAs, 21; with two 18).
template <typename T, int D, int kHeads>
__device__ __forceinline__ void append_rows(const AppendArgs& a, const float2* turns_of, int b, int len, int count, int cta) {
  constexpr int L = D / 8;
  const int chunk = threadIdx.x % L;
  const int kind = cta < a.q_ctas ? 0 : cta < a.q_ctas + a.kv_ctas ? 1 : 2;  // queries, keys, values
  const int n = kind == 0 ? a.heads : a.kv_heads, groups = (n + kHeads - 1) / kHeads;
  const int own = cta - (kind == 0 ? 0 : a.q_ctas + (kind - 1) * a.kv_ctas), mine = threadIdx.x / L, sets = blockDim.x / L;
  // one head: the sets of lanes take a token's heads; more: tokens, the heads are the CTA's
  int t = kHeads == 1 ? (own * sets + mine) / groups : own / groups * sets + mine;
  const int h0 = (kHeads == 1 ? (own * sets + mine) % groups : own % groups) * kHeads;
  const bool on = t < count;  // (lanes of a warp may differ: the shuffles are for all of them)
  if (!on) t = 0;
  const int64_t row = (int64_t)b * a.tokens + t;
  const T* src = kind == 0 ? static_cast<const T*>(a.q) + row * a.q_stride
                           : static_cast<const T*>(kind == 1 ? a.k_new : a.v_new) + row * a.new_stride;
  T* dst = kind == 0 ? static_cast<T*>(a.q_out) + row * a.out_stride
                     : static_cast<T*>(kind == 1 ? a.k : a.v) + (int64_t)b * a.seq_stride + (int64_t)(len + t) * a.kv_stride;
  const bool turned = kind < 2 && a.rope_dim > 0, split = turned && a.halves;
  const Place p = place_of(a, chunk, turned);
  uint4 v[kHeads];
#pragma unroll
  for (int i = 0; i < kHeads; ++i) {
    v[i] = make_uint4(0u, 0u, 0u, 0u);
    if (on && h0 + i < n) v[i] = load8(src + (int64_t)(h0 + i) * D, p, split);
  }
  const void* gain = kind == 0 ? a.q_gain : kind == 1 ? a.k_gain : nullptr;
  Pairs gn;
  if (gain) gn = pairs_of<T>(to_pairs(load8(gain, p, split), p.halves));
  Turn w;
  const bool turns = turned && on && chunk * 8 < a.rope_dim;
  if (turns) turn_of(a, turns_of, b, t, len + t, chunk, &w);
#pragma unroll
  for (int i = 0; i < kHeads; ++i) {
    if (kHeads > 1 && h0 + i >= n) break;
    if (gain || turned) {
      Pairs x = pairs_of<T>(to_pairs(v[i], p.halves));
      if (gain) norm<D>(x, gn, a.eps);
      if (turns) rotate(x, w);
      v[i] = from_pairs(words_of<T>(x), p.halves);
    }
    if (on && h0 + i < n) store8(dst + (int64_t)(h0 + i) * D, p, split, v[i]);
  }
}

// ------------------------------------------------------------ blocks of codes
// The larger magnitudes of packed 16-bit numbers; what is no number stays one.
template <typename T> __device__ __forceinline__ uint32_t larger2(uint32_t a, uint32_t b);
template <> __device__ __forceinline__ uint32_t larger2<__half>(uint32_t a, uint32_t b) {
  const __half2 r = __hmax2_nan(reinterpret_cast<const __half2&>(a), __habs2(reinterpret_cast<const __half2&>(b)));
  return reinterpret_cast<const uint32_t&>(r);
}
template <> __device__ __forceinline__ uint32_t larger2<__nv_bfloat16>(uint32_t a, uint32_t b) {
  const __nv_bfloat162 r = __hmax2_nan(reinterpret_cast<const __nv_bfloat162&>(a), __habs2(reinterpret_cast<const __nv_bfloat162&>(b)));
  return reinterpret_cast<const uint32_t&>(r);
}

// 8 codes of x / scale, to nearest even; inv = 1 / scale.
// E4M3: the product with the reciprocal of a power of two is the quotient.  I8:
// the product's rest x - q scale, times the reciprocal, makes it the quotient as
// a division rounds it (Markstein's correction; for every pair of 16-bit x and largest magnitude), at a
// third of a division's instructions; adding 1.5 * 2^23 rounds it to a whole
// number in the low bits.
template <typename T, int CODE> __device__ __forceinline__ uint2 codes8(const uint4& w, float scale, float inv) {
  const uint32_t words[4] = {w.x, w.y, w.z, w.w};
  uint32_t p[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 x = unpack2<T>(words[i]);
    float2 q = mul2(x, both(inv));
    if (CODE == kCodeE4M3) {
      unsigned short c;
      asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(c) : "f"(q.y), "f"(q.x));
      p[i] = c;
    } else {
      q = fma2(fma2(q, both(-scale), x), both(inv), q);
      q = add2(q, both(12582912.0f));
      p[i] = __byte_perm(__float_as_uint(q.x), __float_as_uint(q.y), 0x0040);
    }
  }
  return make_uint2(__byte_perm(p[0], p[1], 0x5410), __byte_perm(p[2], p[3], 0x5410));
}
template <int CODE> __device__ __forceinline__ float scale_of(float most) {
  float s;
  if (CODE == kCodeE4M3) {
    // least power of two >= most / 448: 448 = 1.75 * 2^8
    const uint32_t u = __float_as_uint(most);
    const int e = (int)(u >> 23) - 127;
    const int up = (u & 0x7fffffu) > 0x600000u;
    s = __uint_as_float((uint32_t)max(e - 8 + up + 127, 127 - 100) << 23);
  } else {
    s = fmaxf(__fdiv_rn(most, 127.0f), kLeastScale);
  }
  return most <= 3.402823466e38f ? s : __uint_as_float(0x7fc00000u);
}

// One head's keys or values of one block: its rows into registers (P of them
// per lane), norm and rotation of the new ones, the block's largest magnitude,
// codes and scale; the rows of the block that stays open also to open_out.
// FULL: all rows are new ones.
template <typename T> struct BlockPlace {
  const T *fresh, *open;  // the block's first row among the new ones (may lie before them), among the open ones
  T* open_out;
  uint8_t* codes;
  float* scale;
  int old, rows;    // rows of before, all rows
  bool stays, writes;  // not full; codes and scale are written
};
template <typename T, int D, int CODE, int P, bool FULL>
__device__ __forceinline__ void append_block(const AppendArgs& a, const float2* turns_of, const BlockPlace<T>& k, int b, int t0, int pos0,
                                             bool values, uint32_t* most) {
  constexpr int L = D / 8;
  const int RP = blockDim.x / L;  // rows of a pass
  const int chunk = threadIdx.x % L, r0 = threadIdx.x / L;
  const bool turned = !values && a.rope_dim > 0, split = turned && a.halves, normed = !values && a.k_gain;
  const bool turns = turned && chunk * 8 < a.rope_dim;
  const Place at = place_of(a, chunk, turned);
  const int64_t width = (int64_t)a.kv_heads * D;
  uint4 v[P];
  {
    const T *fresh = k.fresh + r0 * a.new_stride, *open = k.open + r0 * width;
    const int64_t fresh_step = RP * a.new_stride, open_step = RP * width;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int r = p * RP + r0;
      if (FULL) {
        v[p] = load8(fresh, at, split);
      } else {
        v[p] = make_uint4(0u, 0u, 0u, 0u);
        if (r < k.rows) v[p] = load8(r < k.old ? open : fresh, at, split);
        open += open_step;
      }
      fresh += fresh_step;
    }
  }
  if (normed || turned) {
    Pairs gn;
    if (normed) gn = pairs_of<T>(to_pairs(load8(a.k_gain, at, split), at.halves));
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int r = p * RP + r0;
      const bool fresh = FULL || (r >= k.old && r < k.rows);  // (rows of before were made when they came)
      if (!FULL && !__any_sync(0xffffffffu, fresh)) continue;
      Pairs x = pairs_of<T>(to_pairs(v[p], at.halves));
      if (normed) norm<D>(x, gn, a.eps);
      if (turns && fresh) {
        Turn w;
        turn_of(a, turns_of, b, t0 + r, pos0 + r, chunk, &w);
        rotate(x, w);
      }
      if (fresh) v[p] = from_pairs(words_of<T>(x), at.halves);
    }
  }
  uint32_t mx = 0u;
#pragma unroll
  for (int p = 0; p < P; ++p) mx = larger2<T>(larger2<T>(larger2<T>(larger2<T>(mx, v[p].x), v[p].y), v[p].z), v[p].w);
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) mx = larger2<T>(mx, __shfl_xor_sync(0xffffffffu, mx, off));
  if ((threadIdx.x & 31) == 0) most[threadIdx.x >> 5] = mx;
  __syncthreads();
  mx = most[threadIdx.x & (blockDim.x / 32 - 1)];  // (4 or 8 warps)
#pragma unroll
  for (int off = kMaxThreads / 64; off > 0; off >>= 1) mx = larger2<T>(mx, __shfl_xor_sync(0xffffffffu, mx, off));
  const float2 tops = unpack2<T>(mx);
  const float top = tops.x > tops.y || tops.x != tops.x ? tops.x : tops.y;  // (what is no number stays one)
  const float scale = scale_of<CODE>(top), inv = 1.0f / scale;
  const bool finite = scale <= 3.402823466e38f;
  if (threadIdx.x == 0 && (FULL || k.writes)) *k.scale = scale;
  uint8_t* codes = k.codes + r0 * a.kv_stride;
  const int64_t step = RP * a.kv_stride;
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int r = p * RP + r0;
    if (!FULL && r >= k.rows) break;
    if (FULL || k.writes) {
      uint2 c = codes8<T, CODE>(v[p], scale, inv);
      if (CODE == kCodeI8 && !finite) c = make_uint2(0u, 0u);
      uint32_t* to = reinterpret_cast<uint32_t*>(codes);
      if (split) {
        to[at.a / 4] = c.x;
        to[at.b / 4] = c.y;
      } else {
        *reinterpret_cast<uint2*>(to + at.a / 4) = c;
      }
    }
    if (!FULL && k.stays) store8(k.open_out + r * width, at, split, v[p]);
    codes += step;
  }
}

// The blocks that a sequence's new rows lie in, a block of a head's keys or
// values per CTA.  The last block's open rows may go where the first one's come
// from: then one CTA takes both.  Eight rows a lane where a block has them: the
// CTA's own steps (places, maximum, scale: about 250 instructions a warp) weigh
// as much as two rows (28600 rows x 8 heads 81 us with four rows a lane and a
// division for every code, 35 with eight and none).
template <typename T, int D, int CODE, int P>
__device__ __forceinline__ void append_blocks(const AppendArgs& a, const float2* turns_of, int b, int len, int count, int cta) {
  __shared__ uint32_t most[kMaxThreads / 32];
  const int B = a.block;
  const int head = cta % a.kv_heads, values = cta / a.kv_heads % 2, step = cta / a.kv_heads / 2;
  const int end = len + count, first = len / B, last = (end + B - 1) / B - 1;
  const bool joint = a.k_open == a.k_open_out && len % B != 0;
  const int64_t width = (int64_t)a.kv_heads * D, open_at = (int64_t)b * B * width + (int64_t)head * D;
#pragma unroll 1
  for (int i = 0; i < (joint && step == 0 ? 2 : 1); ++i) {
    const int blk = i == 1 ? last : first + step;
    if (blk > last || last < first || (i == 1 && last == first) || (joint && step > 0 && blk == last)) continue;
    const int row0 = blk * B;
    BlockPlace<T> k;
    k.fresh = static_cast<const T*>(values ? a.v_new : a.k_new) + ((int64_t)b * a.tokens + (row0 - len)) * a.new_stride + (int64_t)head * D;
    k.open = static_cast<const T*>(values ? a.v_open : a.k_open) + open_at;
    k.open_out = static_cast<T*>(values ? a.v_open_out : a.k_open_out) + open_at;
    k.codes = static_cast<uint8_t*>(values ? a.v : a.k) + (int64_t)b * a.seq_stride + (int64_t)row0 * a.kv_stride + (int64_t)head * D;
    k.scale = (values ? a.v_scale : a.k_scale) + ((int64_t)b * a.kv_heads + head) * a.blocks + blk;
    k.old = len - row0;
    k.rows = min(B, end - row0);
    k.stays = k.rows < B;
    k.writes = count > 0;
    if (i == 1) __syncthreads();  // (the first block's maxima have been read, and its rows)
    if (k.old <= 0 && k.rows == B)
      append_block<T, D, CODE, P, true>(a, turns_of, k, b, row0 - len, row0, values, most);
    else
      append_block<T, D, CODE, P, false>(a, turns_of, k, b, row0 - len, row0, values, most);
  }
}

// CTAs of a sequence: block_ctas, a (block, keys or values, head) each, then
// row_ctas for rows in 16 bits, which take less time; CTA by CTA of all
// sequences.
template <typename T, int D, int CODE, int kHeads, int P>
__global__ void __launch_bounds__(kMaxThreads, 4) cache_append_kernel(const __grid_constant__ AppendArgs a) {
  const int cta = blockIdx.x / a.n_seq, b = blockIdx.x % a.n_seq;
  __shared__ __align__(16) float2 turns_of[64];  // (lanes that read different kernel arguments wait for one another)
  if (a.rope_dim && threadIdx.x < a.rope_dim / 2) turns_of[threadIdx.x] = a.turns[threadIdx.x];
  int len, count;
  if (!append_sizes(a, b, &len, &count)) return;
  if (a.rope_dim) __syncthreads();
  if (cta == 0 && threadIdx.x == 0 && a.lens_out) a.lens_out[b] = len + count;
  if (CODE == kCode16 || cta >= a.block_ctas)
    append_rows<T, D, kHeads>(a, turns_of, b, len, count, cta - a.block_ctas);
  else
    append_blocks<T, D, CODE == kCode16 ? kCodeI8 : CODE, P>(a, turns_of, b, len, count, cta);
}

template <typename T, int D, int CODE, int kHeads, int P> int append_go(const AppendArgs& a, int threads, cudaStream_t s) {
  cache_append_kernel<T, D, CODE, kHeads, P><<<(unsigned)((int64_t)(a.row_ctas + a.block_ctas) * a.n_seq), threads, 0, s>>>(a);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) SN_FAIL(SWAPNET_ERR_CUDA, std::string("cache append launch: ") + cudaGetErrorString(e));
  return SWAPNET_OK;
}
template <typename T, int D, int CODE, int kHeads> int append_p(const AppendArgs& a, int threads, int p, cudaStream_t s) {
  if constexpr (CODE != kCode16) {
    if (p == 2) return append_go<T, D, CODE, kHeads, 2>(a, threads, s);
    if (p == 4) return append_go<T, D, CODE, kHeads, 4>(a, threads, s);
    if (p == 8) return append_go<T, D, CODE, kHeads, 8>(a, threads, s);
  }
  return append_go<T, D, CODE, kHeads, 1>(a, threads, s);
}
template <typename T, int D, int CODE> int append_t(AppendArgs a, cudaStream_t s) {
  constexpr int L = D / 8, kMany = CODE == kCode16 ? 4 : 8;
  // a block's rows: up to eight per lane (they hide the CTA's own steps), in 128
  // threads or, where that is not enough, 256
  const int threads = a.block * L > 8 * 128 || CODE == kCode16 ? 256 : 128, p = (a.block * L + threads - 1) / threads;
  const int rows_per_cta = threads / L;
  // few rows: a head per thread group, so that the call is over sooner; many:
  // four or eight, which share the token's angles and the CTA's own steps
  const int64_t rows = (int64_t)a.n_seq * a.tokens * (a.heads + (CODE == kCode16 ? 2 * a.kv_heads : 0));
  const int kh = rows >= 16384 && a.tokens >= 64 ? kMany : 1;
  auto ctas = [&](int heads) -> int64_t {
    if (kh == 1) return ((int64_t)heads * a.tokens + rows_per_cta - 1) / rows_per_cta;
    return (int64_t)(heads + kh - 1) / kh * ((a.tokens + rows_per_cta - 1) / rows_per_cta);
  };
  const int64_t q_ctas = ctas(a.heads), kv_ctas = CODE == kCode16 ? ctas(a.kv_heads) : 0;
  int64_t block_ctas = 0;
  if (CODE != kCode16) {
    const int64_t blocks = ((int64_t)a.tokens + 2 * a.block - 2) / a.block;  // that the rows may lie in
    block_ctas = blocks * a.kv_heads * 2;
  }
  const int64_t all = q_ctas + 2 * kv_ctas + block_ctas;
  if ((int64_t)std::max(a.heads, a.kv_heads) * a.tokens > (1 << 30) || all * a.n_seq > 0x7fffffff)
    SN_FAIL(SWAPNET_ERR_UNSUPPORTED, "cache append: shape beyond the kernels' limits");
  a.q_ctas = (int)q_ctas;
  a.kv_ctas = (int)kv_ctas;
  a.row_ctas = (int)(q_ctas + 2 * kv_ctas);
  a.block_ctas = (int)block_ctas;
  return kh > 1 ? append_p<T, D, CODE, kMany>(a, threads, p, s) : append_p<T, D, CODE, 1>(a, threads, p, s);
}
template <typename T, int D> int append_d(const AppendArgs& a, cudaStream_t s) {
  return a.code == kCodeI8 ? append_t<T, D, kCodeI8>(a, s) : a.code == kCodeE4M3 ? append_t<T, D, kCodeE4M3>(a, s) : append_t<T, D, kCode16>(a, s);
}

}  // namespace

int launch_cache_append(AppendArgs a, cudaStream_t s) {
  if (a.dtype == SWAPNET_BF16) return a.dim == 128 ? append_d<__nv_bfloat16, 128>(a, s) : append_d<__nv_bfloat16, 64>(a, s);
  return a.dim == 128 ? append_d<__half, 128>(a, s) : append_d<__half, 64>(a, s);
}

}  // namespace swapnet
