// Rows appended to a key-value cache: norms of queries and keys, position
// rotation, and for a cache of 8 bits the codes and scales of the blocks that
// the rows lie in, all in one launch.  fp32 arithmetic, fixed orders of
// summation.
//
// What a row needs is its own (norm, rotation), what a code needs is its
// block's largest magnitude; so a CTA holds a whole block of one head in
// registers between the two, and the rows are read once and written once.
#include <algorithm>
#include <string>
#include <type_traits>

#include "device.cuh"
#include "internal.h"
#include "kernels.h"
#include "quant.h"

namespace swapnet {

namespace {

constexpr int kApThreads = 256;

// A row of D elements is held by D / 8 neighbouring lanes, 8 elements each.
template <typename T> __device__ __forceinline__ void unpack8(const uint4& v, float (&f)[8]) {
  const T* e = reinterpret_cast<const T*>(&v);
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = to_f<T>(e[i]);
}
template <typename T> __device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
  uint4 v;
  T* e = reinterpret_cast<T*>(&v);
#pragma unroll
  for (int i = 0; i < 8; ++i) e[i] = from_f<T>(f[i]);
  return v;
}

// Norm of a row's 8 elements per lane: x / sqrt(mean + eps) * gain.
template <int D> __device__ __forceinline__ void norm8(float (&x)[8], const float (&gain)[8], float eps) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) s = fmaf(x[i], x[i], s);
#pragma unroll
  for (int off = D / 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
  const float r = 1.0f / sqrtf(s * (1.0f / D) + eps);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = x[i] * r * gain[i];
}

// cos and sin of the angles of this lane's pairs at a token's position:
// adjacent pairs: 4, halves: 8 (both lanes of the pairs have them).  The angle
// in turns is position * (hi + lo): the product with hi is split into what it
// rounds to and the rest (fma), whole turns are taken off, and only then is it
// an angle; far positions keep an error below 2^-24.
struct Turn {
  float c[8], s[8];
};
__device__ __forceinline__ void turn_of(const AppendArgs& a, int b, int t, int pos, int pair0, int n, Turn* w) {
  int axis = -1;
  float at = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (i >= n) break;
    const int pair = pair0 + i;
    const int ax = a.positions ? (pair >= a.axis1) + (pair >= a.axis2) : 0;
    if (ax != axis) {
      axis = ax;
      int p = a.positions ? a.positions[((int64_t)ax * a.n_seq + b) * a.tokens + t] : pos;
      if ((unsigned)p >= (unsigned)kMaxPosition) {
        atomicExch(a.err, kDevErrBounds);
        p = 0;
      }
      at = (float)p;
    }
    const float2 f = a.turns[pair];
    const float whole = at * f.x, rest = fmaf(at, f.x, -whole);
    const float turns = (whole - rintf(whole)) + fmaf(at, f.y, rest);
    sincospif(2.0f * turns, &w->s[i], &w->c[i]);
  }
}
// Turns a row; chunk: which 8 elements this lane has.  All lanes of the warp.
template <int D> __device__ __forceinline__ void rotate8(const AppendArgs& a, float (&x)[8], const Turn& w, int chunk) {
  if (!a.halves) {
    if (chunk * 8 >= a.rope_dim) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float u = x[2 * i], v = x[2 * i + 1];
      x[2 * i] = u * w.c[i] - v * w.s[i];
      x[2 * i + 1] = v * w.c[i] + u * w.s[i];
    }
    return;
  }
  const int half = a.rope_dim / 16;  // lanes of a half
  const bool turns = chunk < 2 * half, second = chunk >= half;
  const int lane = threadIdx.x & 31, other = turns ? (second ? lane - half : lane + half) : lane;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float y = __shfl_sync(0xffffffffu, x[i], other);
    if (turns) x[i] = second ? x[i] * w.c[i] + y * w.s[i] : x[i] * w.c[i] - y * w.s[i];
  }
}
// The first pair and the number of pairs that lane `chunk` turns (0: none).
__device__ __forceinline__ int pairs_of(const AppendArgs& a, int chunk, int* first) {
  const int n = a.rope_dim ? (a.halves ? 8 : 4) : 0;
  *first = a.halves ? chunk * 8 % max(a.rope_dim / 2, 1) : chunk * 4;
  return chunk * 8 < a.rope_dim ? n : 0;
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

template <typename T> __device__ __forceinline__ void load_gain(const void* gain, int chunk, float (&g)[8]) {
  if (gain) unpack8<T>(reinterpret_cast<const uint4*>(gain)[chunk], g);
}

// ---------------------------------------------------------- rows in 16 bits
// Queries, and for a 16-bit cache keys and values.  D / 8 lanes take kHeads
// heads of one token, so that its angles serve all of them.
template <typename T, int D, int kHeads>
__device__ __forceinline__ void append_rows(const AppendArgs& a, int b, int len, int count, int cta) {
  constexpr int L = D / 8;
  const int chunk = threadIdx.x % L;
  const int qg = (a.heads + kHeads - 1) / kHeads, kg = a.code == kCode16 ? (a.kv_heads + kHeads - 1) / kHeads : 0;
  const int groups = qg + 2 * kg;
  const int id = cta * (kApThreads / L) + threadIdx.x / L;
  const bool on = id / groups < count;  // (lanes of a warp may differ: the shuffles are for all of them)
  const int t = on ? id / groups : 0, g = id % groups;
  const int kind = g < qg ? 0 : g < qg + kg ? 1 : 2;  // queries, keys, values
  const int h0 = (kind == 0 ? g : kind == 1 ? g - qg : g - qg - kg) * kHeads, n = kind == 0 ? a.heads : a.kv_heads;
  const int64_t row = (int64_t)b * a.tokens + t;
  const T* src = kind == 0 ? static_cast<const T*>(a.q) + row * a.q_stride
                           : static_cast<const T*>(kind == 1 ? a.k_new : a.v_new) + row * a.new_stride;
  T* dst = kind == 0 ? static_cast<T*>(a.q_out) + row * a.out_stride
                     : static_cast<T*>(kind == 1 ? a.k : a.v) + (int64_t)b * a.seq_stride + (int64_t)(len + t) * a.kv_stride;
  uint4 v[kHeads];
#pragma unroll
  for (int i = 0; i < kHeads; ++i) {
    v[i] = make_uint4(0u, 0u, 0u, 0u);
    if (on && h0 + i < n) v[i] = *reinterpret_cast<const uint4*>(src + (int64_t)(h0 + i) * D + chunk * 8);
  }
  const void* gain = kind == 0 ? a.q_gain : kind == 1 ? a.k_gain : nullptr;
  float gn[8];
  load_gain<T>(gain, chunk, gn);
  int first;
  const int pairs = kind < 2 ? pairs_of(a, chunk, &first) : 0;
  Turn w;
  if (on && pairs) turn_of(a, b, t, len + t, first, pairs, &w);
  const bool any_gain = a.q_gain || a.k_gain;
#pragma unroll
  for (int i = 0; i < kHeads; ++i) {
    if (kHeads > 1 && !__any_sync(0xffffffffu, on && h0 + i < n)) break;
    uint4 y = v[i];
    if (any_gain || a.rope_dim) {
      float x[8], z[8];
      unpack8<T>(v[i], x);
      if (any_gain) {
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = x[e];
        norm8<D>(z, gn, a.eps);
        if (gain) {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = z[e];
        }
      }
      if (a.rope_dim) {
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = x[e];
        rotate8<D>(a, z, w, chunk);
        if (kind < 2) {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = z[e];
        }
      }
      if (kind < 2) y = pack8<T>(x);
    }
    if (on && h0 + i < n) *reinterpret_cast<uint4*>(dst + (int64_t)(h0 + i) * D + chunk * 8) = y;
  }
}

// ------------------------------------------------------------ blocks of codes
// The largest magnitude of packed 16-bit numbers by their bits: infinities and
// what is no number come out largest.
__device__ __forceinline__ uint32_t larger2(uint32_t a, uint32_t b) { return __vmaxu2(a, b & 0x7fff7fffu); }

// 8 codes of x / scale, to nearest even.
template <int CODE> __device__ __forceinline__ uint2 codes8(const float (&x)[8], float scale) {
  uint2 out;
  if (CODE == kCodeE4M3) {
    const float inv = 1.0f / scale;  // (a power of two: exact)
    uint32_t p[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      unsigned short c;
      asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(c) : "f"(x[2 * i + 1] * inv), "f"(x[2 * i] * inv));
      p[i] = c;
    }
    out = make_uint2(p[0] | p[1] << 16, p[2] | p[3] << 16);
  } else {
    uint32_t p[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int c = __float2int_rn(__fdiv_rn(x[i], scale));  // (not a number: 0)
      p[i >> 2] |= (uint32_t)(c & 0xff) << (8 * (i & 3));
    }
    out = make_uint2(p[0], p[1]);
  }
  return out;
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

// One head's keys or values of the blocks that a sequence's new rows lie in, a
// block per CTA: its rows into registers (those of the open block from 16
// bits), norm and rotation, the block's largest magnitude, codes and scale;
// the rows of the block that stays open also to k_open_out.  The first and the
// last block share a CTA: the last one's rows may go where the first one's come
// from.
template <typename T, int D, int CODE>
__device__ __forceinline__ void append_block(const AppendArgs& a, int b, int len, int count, int cta) {
  constexpr int L = D / 8, RP = kApThreads / L, P = 128 / RP;  // rows of a pass, passes of the largest block
  __shared__ uint32_t most[kApThreads / 32];
  const int B = a.block, chunk = threadIdx.x % L, r0 = threadIdx.x / L;
  const int head = cta % a.kv_heads, values = cta / a.kv_heads % 2, step = cta / a.kv_heads / 2;
  const int end = len + count, first = len / B, last = (end + B - 1) / B - 1;
  if (last < first) return;  // (nothing there)
  const T* fresh = static_cast<const T*>(values ? a.v_new : a.k_new) + (int64_t)b * a.tokens * a.new_stride + (int64_t)head * D + chunk * 8;
  const int64_t width = (int64_t)a.kv_heads * D, open_at = (int64_t)b * B * width + (int64_t)head * D + chunk * 8;
  const T* open = static_cast<const T*>(values ? a.v_open : a.k_open) + open_at;
  T* open_out = static_cast<T*>(values ? a.v_open_out : a.k_open_out) + open_at;
  uint8_t* codes = static_cast<uint8_t*>(values ? a.v : a.k) + (int64_t)b * a.seq_stride + (int64_t)head * D + chunk * 8;
  float* scales = (values ? a.v_scale : a.k_scale) + ((int64_t)b * a.kv_heads + head) * a.blocks;
  const void* gain = values ? nullptr : a.k_gain;
  float gn[8];
  load_gain<T>(gain, chunk, gn);
  int pair0;
  const int pairs = values ? 0 : pairs_of(a, chunk, &pair0);
  for (int i = 0; i < (step == 0 ? 2 : 1); ++i) {
    const int blk = i == 1 ? last : first + step;
    if (blk > last || (i == 1 && last == first) || (step > 0 && blk == last)) continue;
    const int row0 = blk * B;
    uint4 v[P];
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int r = p * RP + r0, j = row0 + r;
      v[p] = make_uint4(0u, 0u, 0u, 0u);
      if (r < B && j < end)
        v[p] = j < len ? *reinterpret_cast<const uint4*>(open + (int64_t)r * width)
                       : *reinterpret_cast<const uint4*>(fresh + (int64_t)(j - len) * a.new_stride);
    }
    uint32_t mx = 0u;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      if (p * RP >= B) break;
      const int r = p * RP + r0, j = row0 + r;
      const bool is_new = r < B && j >= len && j < end;
      if (!values && (a.k_gain || a.rope_dim)) {
        float x[8];
        unpack8<T>(v[p], x);
        if (a.k_gain) norm8<D>(x, gn, a.eps);
        if (a.rope_dim) {
          Turn w;
          if (is_new && pairs) turn_of(a, b, j - len, j, pair0, pairs, &w);
          rotate8<D>(a, x, w, chunk);
        }
        if (is_new) v[p] = pack8<T>(x);  // (rows of the open block were made when they came)
      }
      mx = larger2(larger2(larger2(larger2(mx, v[p].x), v[p].y), v[p].z), v[p].w);
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) mx = __vmaxu2(mx, __shfl_xor_sync(0xffffffffu, mx, off));
    if (i == 1) __syncthreads();  // (the first block's maxima have been read)
    if ((threadIdx.x & 31) == 0) most[threadIdx.x >> 5] = mx;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kApThreads / 32; ++w) mx = __vmaxu2(mx, most[w]);
    mx = max(mx & 0xffffu, mx >> 16);
    const T top = *reinterpret_cast<const T*>(&mx);
    const float scale = scale_of<CODE>(to_f<T>(top));
    if (threadIdx.x == 0 && count > 0) scales[blk] = scale;
    const bool stays = blk == end / B;  // (not full)
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int r = p * RP + r0, j = row0 + r;
      if (r >= B || j >= end) break;
      float x[8];
      unpack8<T>(v[p], x);
      if (count > 0) *reinterpret_cast<uint2*>(codes + (int64_t)j * a.kv_stride) = codes8<CODE>(x, scale);
      if (stays) *reinterpret_cast<uint4*>(open_out + (int64_t)r * width) = v[p];
    }
  }
}

// CTAs of a sequence: row_ctas for rows in 16 bits, then block_ctas, a (head,
// keys or values, block) each.
template <typename T, int D, int CODE, int kHeads>
__global__ void __launch_bounds__(kApThreads) cache_append_kernel(const __grid_constant__ AppendArgs a) {
  const int per = a.row_ctas + a.block_ctas;
  const int b = blockIdx.x / per, cta = blockIdx.x % per;
  int len, count;
  if (!append_sizes(a, b, &len, &count)) return;
  if (cta == 0 && threadIdx.x == 0 && a.lens_out) a.lens_out[b] = len + count;
  if (cta < a.row_ctas)
    append_rows<T, D, kHeads>(a, b, len, count, cta);
  else if (CODE != kCode16)
    append_block<T, D, CODE == kCode16 ? kCodeI8 : CODE>(a, b, len, count, cta - a.row_ctas);
}

template <typename T, int D, int CODE> int append_t(AppendArgs a, cudaStream_t s) {
  // few rows: a head per thread group, so that the call is over sooner; many:
  // four, which share the token's angles
  const int64_t rows = (int64_t)a.n_seq * a.tokens * (a.heads + (CODE == kCode16 ? 2 * a.kv_heads : 0));
  const int kh = rows >= 16384 ? 4 : 1;
  auto groups = [&](int heads) { return (int64_t)(heads + kh - 1) / kh; };
  const int64_t per_token = groups(a.heads) + (CODE == kCode16 ? 2 * groups(a.kv_heads) : 0);
  const int64_t row_ctas = (per_token * a.tokens + kApThreads / (D / 8) - 1) / (kApThreads / (D / 8));
  int64_t block_ctas = 0;
  if (CODE != kCode16) {
    const int64_t blocks = ((int64_t)a.tokens + 2 * a.block - 2) / a.block;  // that the rows may lie in
    block_ctas = std::max<int64_t>(1, blocks - 1) * a.kv_heads * 2;
  }
  if (per_token * a.tokens > (1 << 30) || (row_ctas + block_ctas) * a.n_seq > 0x7fffffff) SN_FAIL(SWAPNET_ERR_UNSUPPORTED, "cache append: shape beyond the kernels' limits");
  a.row_ctas = (int)row_ctas;
  a.block_ctas = (int)block_ctas;
  const unsigned grid = (unsigned)((row_ctas + block_ctas) * a.n_seq);
  if (kh == 4)
    cache_append_kernel<T, D, CODE, 4><<<grid, kApThreads, 0, s>>>(a);
  else
    cache_append_kernel<T, D, CODE, 1><<<grid, kApThreads, 0, s>>>(a);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) SN_FAIL(SWAPNET_ERR_CUDA, std::string("cache append launch: ") + cudaGetErrorString(e));
  return SWAPNET_OK;
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
