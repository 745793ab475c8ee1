// Device-side pieces of the attention over a cache of 8-bit codes: codes to
// fp16, queries to fp16, scales.
#pragma once
#include "cached_tc.cuh"
#include "kernels.h"
#include "quant.h"

namespace swapnet {

// Byte offset of 16-byte chunk `c` of row `r` in a tile of D-byte rows: chunks
// are exchanged so that the eight rows of an 8 x 8 matrix lie in different
// banks.
template <int D> __device__ __forceinline__ uint32_t swz8(uint32_t r, uint32_t c) {
  if (D == 128) return r * 128 + ((c ^ (r & 7)) << 4);
  return r * 64 + ((c ^ ((r >> 1) & 3)) << 4);
}
__device__ __forceinline__ void cp_async_4(uint32_t dst, const void* src, bool valid) {
  const int n = valid ? 4 : 0;  // 0: write zeros, read nothing
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
// An 8 x 8 matrix of 16-bit elements, transposed across the warp.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// Two codes as fp16 numbers: bytes of x that `sel` (a byte permutation with a
// second word of 0x64) brings into place.
// I8: 1024 + (code + 128) as the byte below an exponent, less 1152: exact.
// E4M3: converted by the instruction for it, two codes in 2 cycles of a
// scheduler (moving the bits takes 8).
__device__ __forceinline__ uint32_t i8_pair(uint32_t flipped, uint32_t sel) {
  const uint32_t u = __byte_perm(flipped, 0x64646464u, sel);
  const __half2 r = __hsub2(reinterpret_cast<const __half2&>(u), __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480)));
  return reinterpret_cast<const uint32_t&>(r);
}
__device__ __forceinline__ uint2 e4m3_pairs(uint32_t x) {
  uint2 r;
  asm("{\n\t.reg .b16 l, h;\n\t"
      "mov.b32 {l, h}, %2;\n\t"
      "cvt.rn.f16x2.e4m3x2 %0, l;\n\t"
      "cvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
      : "=r"(r.x), "=r"(r.y)
      : "r"(x));
  return r;
}
// bytes (0, 1) and (2, 3)
template <int CODE> __device__ __forceinline__ uint2 pairs_near(uint32_t x) {
  if (CODE == kCodeI8) {
    const uint32_t f = x ^ 0x80808080u;
    return make_uint2(i8_pair(f, 0x4140), i8_pair(f, 0x4342));
  }
  return e4m3_pairs(x);
}
// bytes (0, 2) and (1, 3)
template <int CODE> __device__ __forceinline__ uint2 pairs_apart(uint32_t x) {
  if (CODE == kCodeI8) {
    const uint32_t f = x ^ 0x80808080u;
    return make_uint2(i8_pair(f, 0x4240), i8_pair(f, 0x4341));
  }
  return e4m3_pairs(__byte_perm(x, 0u, 0x3120));
}
// The bytes of x with those cleared that are E4M3's codes for no number.
__device__ __forceinline__ uint32_t numbers_only(uint32_t x) {
  const uint32_t none = ((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
  return x & ~(none | (none - (none >> 7)));
}

// A value scale = 2^e * f with f in [1, 2), and inv = 2^-e; scales below 2^-48
// have e = -48 and smaller f, those that are no number or infinite keep f so.
// The softmax takes p = 2^(score + e - m) with p <= 2^14, adds p inv to its sum
// and gives p f, at most 2^15, to the products.  A key loses its weight only
// where p falls below 2^-126: one of a block of zeros beside value scales of
// 2^64 where it is below 2^-28 of the largest on warp products, whose m leaves
// the largest p at 2^14, and 2^-21 on the tensor cores, where it may be 2^7 (a
// least e of -100 left nothing of zeros beside scales of 2^40).
constexpr float kTop = 14.0f;  // log2 of the largest p
__device__ __forceinline__ void split_scale(float scale, float* e, float* f, float* inv) {
  const int x = min(max((int)(__float_as_uint(scale) >> 23 & 0xffu), 127 - 48), 253);
  *inv = __uint_as_float((uint32_t)(254 - x) << 23);
  *f = scale * *inv;
  *e = (float)(x - 127);
}

// A query's C x 4 elements of this lane (four lanes of a row) as fp16 pairs,
// and the power of two that they were divided by: fp16 as it is, bf16 with the
// largest element of the row in [2^14, 2^15), so that what fp16 loses is below
// 2^-39 of it.
template <typename T, int C> __device__ __forceinline__ float query_fp16(const uint2 (&raw)[C], uint32_t (&out)[C][2]) {
  if (std::is_same<T, __half>::value) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      out[c][0] = raw[c].x;
      out[c][1] = raw[c].y;
    }
    return 1.0f;
  }
  uint32_t most = 0u;
#pragma unroll
  for (int c = 0; c < C; ++c) most = __vmaxu2(__vmaxu2(most, raw[c].x & 0x7fff7fffu), raw[c].y & 0x7fff7fffu);
  most = max(most & 0xffffu, most >> 16);
  most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
  most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
  // exponent field of the largest: 2^(x - 127) <= it < 2^(x - 126); infinities keep theirs
  const int x = min(max((int)(most >> 7), 28), 254);
  const float by = __uint_as_float((uint32_t)(127 + 14 - (x - 127)) << 23);
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const float2 u = unpack_pair<__nv_bfloat16>(raw[c].x), w = unpack_pair<__nv_bfloat16>(raw[c].y);
    out[c][0] = pack_pair<__half>(u.x * by, u.y * by);
    out[c][1] = pack_pair<__half>(w.x * by, w.y * by);
  }
  return __uint_as_float((uint32_t)(127 + (x - 127) - 14) << 23);
}

// The power of two that a BF16 query row is divided by: its largest element
// comes to lie in [2^14, 2^15).  From the bits of the largest magnitude its
// exponent field, kept where both factors are normal numbers.
__device__ __forceinline__ uint32_t largest_bits(const uint4& v) {
  const uint32_t m = __vmaxu2(__vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu), __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu));
  return max(m & 0xffffu, m >> 16);
}
__device__ __forceinline__ int query_exponent(uint32_t most) { return min(max((int)(most >> 7), 28), 254); }
__device__ __forceinline__ uint32_t query_pair(uint32_t x, float by) {
  const float2 u = unpack_pair<__nv_bfloat16>(x);
  return pack_pair<__half>(u.x * by, u.y * by);
}
__device__ __forceinline__ float2 mul2(float2 x, float2 y) {
  float2 r;
  asm("mul.rn.f32x2 %0, %1, %2;"
      : "=l"(reinterpret_cast<unsigned long long&>(r))
      : "l"(reinterpret_cast<unsigned long long&>(x)), "l"(reinterpret_cast<unsigned long long&>(y)));
  return r;
}

// ------------------------------------------------------------------ runs
// Which tiles a CTA of an attention launch takes: with a.splits == 1 unit
// blockIdx / kv_heads of its key head, otherwise an equal run of all the head's
// tiles (see Cursor).  near: sizes of sequences, sched: scratch of at least
// blockDim / 32 + 2 words, both in shared memory.  All threads of the block.
struct Run {
  int kvh, run, runs;      // the run's number and how many there are
  int64_t first, total;    // its first tile in the order of all; their number
};
__device__ __forceinline__ Run start_run(const CachedArgs& a, Cursor& cur, int2* near, int64_t* sched, int queries, int nrt) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x / 32;
  Run r;
  r.kvh = blockIdx.x % a.kv_heads;
  r.run = blockIdx.x / a.kv_heads;
  r.runs = 1;
  r.first = r.total = 0;
  cur.next = 0;
  cur.near = near;
  const bool all_near = a.splits != 1 && a.n_seq <= kNear;
  cur.b0 = a.splits == 1 ? r.run / nrt : 0;
  if ((a.splits == 1 || all_near) && threadIdx.x < kNear && cur.b0 + (int)threadIdx.x < a.n_seq) near[threadIdx.x] = seq_size(a, cur.b0 + threadIdx.x);
  __syncthreads();
  if (a.splits == 1) {
    cur.pair = r.run;
    cur.left = pair_size(a, near[0], r.run % nrt, queries).tiles;
    if (cur.left == 0 && r.kvh == 0) {
      int len, count;
      seq_sizes(a, r.run / nrt, &len, &count);  // (reports what is out of range)
    }
    return r;
  }
  // every thread adds up some pairs, then the threads' sums
  auto size_of = [&](int b) { return all_near ? near[b] : seq_size(a, b); };
  const int pairs = a.n_seq * nrt, per = (pairs + blockDim.x - 1) / blockDim.x;
  const int p0 = min((int)threadIdx.x * per, pairs), p1 = min(p0 + per, pairs);
  int64_t sum = 0;
  for (int p = p0; p < p1; ++p) {
    const int2 size = size_of(p / nrt);
    sum += pair_size(a, size, p % nrt, queries).tiles;
    if (blockIdx.x == 0 && (size.x < 0 || size.x > a.max_seq || size.y < 0 || size.y > a.tokens)) atomicExch(a.err, kDevErrBounds);
  }
  int64_t before = sum;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const int64_t o = __shfl_up_sync(0xffffffffu, before, off);
    if (lane >= off) before += o;
  }
  if (lane == 31) sched[warp] = before;
  before -= sum;
  __syncthreads();
  for (int w = 0; w < warps; ++w) {
    if (w < warp) before += sched[w];
    r.total += sched[w];
  }
  r.runs = (int)min((int64_t)(gridDim.x / a.kv_heads), (r.total + kRunTiles - 1) / kRunTiles);
  r.first = r.run < r.runs ? r.total * r.run / r.runs : r.total;
  cur.left = r.run < r.runs ? r.total * (r.run + 1) / r.runs - r.first : 0;
  cur.pair = 0;
  if (cur.left > 0 && before <= r.first && r.first < before + sum) {
    int64_t at = before;
    for (int p = p0; p < p1; ++p) {
      const int tiles = pair_size(a, size_of(p / nrt), p % nrt, queries).tiles;
      if (r.first < at + tiles) {
        sched[warps] = p;
        sched[warps + 1] = r.first - at;
        break;
      }
      at += tiles;
    }
  }
  __syncthreads();
  if (cur.left > 0) {
    cur.pair = (int)sched[warps];
    cur.next = (int)sched[warps + 1];
  }
  if (!all_near) {
    cur.b0 = cur.pair / nrt;
    if (threadIdx.x < kNear && cur.b0 + (int)threadIdx.x < a.n_seq) near[threadIdx.x] = seq_size(a, cur.b0 + threadIdx.x);
  }
  return r;
}
// One thread, for a unit whose first piece this CTA has had (tile `at` of the
// run's order on): the CTA, and how many runs share the unit (0: it is whole).
__device__ __forceinline__ void record_unit(const CachedArgs& a, const Run& r, const Cursor& cur, int nrt, int64_t at) {
  int pieces = 0;
  if (cur.n < cur.z.tiles) {
    const int64_t end = at + cur.z.tiles - 1;  // its last tile
    int c = (int)(end * r.runs / r.total);  // whose run that is, up to the rounding
    while (r.total * (c + 1) / r.runs <= end) ++c;
    while (r.total * c / r.runs > end) --c;
    pieces = c - r.run + 1;
  }
  reinterpret_cast<int2*>(a.units)[((int64_t)cur.b * nrt + cur.rt) * a.kv_heads + r.kvh] = make_int2(blockIdx.x, pieces);
}

// Tensor maps of a call's codes, in tiles of kKeys rows of a head; swizzled: the
// keys' 16-byte chunks by the 128-byte pattern (rows of 128 codes).
inline int quant_maps(const QuantArgs& a, CUtensorMap* k, CUtensorMap* v, bool swizzled) {
  const uint64_t dims[3] = {(uint64_t)a.kv_heads * a.dim, (uint64_t)a.max_seq, (uint64_t)a.n_seq};
  // (a single sequence's stride is never used, but has to be a valid one)
  const uint64_t strides[2] = {(uint64_t)a.kv_stride, (uint64_t)(a.n_seq > 1 ? a.seq_stride : a.kv_stride)};
  const uint32_t box[3] = {(uint32_t)a.dim, kKeys, 1};
  if (int rc = make_tmap_codes(k, a.k, dims, strides, box, swizzled)) return rc;
  return make_tmap_codes(v, a.v, dims, strides, box, false);
}

}  // namespace swapnet
