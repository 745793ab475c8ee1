// Device-side pieces that the cached-attention kernels share: what a sequence
// holds, which keys a query sees, warp-level matrix products.
#pragma once
#include "cached.h"
#include "device.cuh"

namespace swapnet {

// Sequence b's cached rows and queries in use; false (and the device error
// word set) where they are out of range: such a sequence is left alone.
__device__ __forceinline__ bool seq_sizes(const CachedArgs& a, int b, int* len, int* count) {
  const int n = a.lens[b * a.lens_step] + a.len_add, c = a.counts ? a.counts[b * a.counts_step] : a.tokens;
  *len = n;
  *count = c;
  if (n < 0 || n > a.max_seq || c < 0 || c > a.tokens) {
    if (threadIdx.x == 0) atomicExch(a.err, kDevErrBounds);
    return false;
  }
  return true;
}

// Keys of the cache that query t sees: all of them beside a draft, else those
// up to its own row (the queries are the cache's last rows).
__device__ __forceinline__ int visible_limit(const CachedArgs& a, int len, int count, int t) {
  return a.k_new ? len : max(0, len - count + t + 1);
}

// Ancestor bits (itself included) of every drafted node, in shared memory:
// anc[t][w]: nodes 32w .. 32w + 31.  All threads of the block; false if a
// parent is not an earlier node or -1.
__device__ __forceinline__ bool build_ancestors(const CachedArgs& a, int b, int count, uint32_t (*anc)[4], int* par) {
  bool bad = false;
  if (a.parents)
    for (int t = threadIdx.x; t < count; t += blockDim.x) {
      const int p = a.parents[(int64_t)b * a.tokens + t];
      par[t] = p;
      bad = bad || p < -1 || p >= t;
    }
  bad = __syncthreads_or(bad) != 0;
  if (bad) {
    if (threadIdx.x == 0) atomicExch(a.err, kDevErrBounds);
    return false;
  }
  for (int t = threadIdx.x; t < count; t += blockDim.x) {
    uint32_t m[4] = {0u, 0u, 0u, 0u};
    if (a.parents) {
      for (int i = t; i >= 0; i = par[i]) {  // (each step goes to a lower node)
#pragma unroll
        for (int w = 0; w < 4; ++w)
          if (i >> 5 == w) m[w] |= 1u << (i & 31);
      }
    } else {
#pragma unroll
      for (int w = 0; w < 4; ++w) m[w] = t >= 32 * w + 31 ? 0xffffffffu : t >= 32 * w ? (2u << (t & 31)) - 1u : 0u;
    }
#pragma unroll
    for (int w = 0; w < 4; ++w) anc[t][w] = m[w];
  }
  __syncthreads();
  return true;
}

// 2^x to 2 ulp; results below the normal range are 0.
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// ------------------------------------------------------ warp matrix products
__device__ __forceinline__ void ldmatrix_x4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
template <typename T> __device__ __forceinline__ void mma_16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma_16816<__half>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma_16816<__nv_bfloat16>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <typename T> __device__ __forceinline__ uint32_t pack_pair(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack_pair<__half>(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
template <> __device__ __forceinline__ uint32_t pack_pair<__nv_bfloat16>(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
template <typename T> __device__ __forceinline__ float2 unpack_pair(uint32_t u);
template <> __device__ __forceinline__ float2 unpack_pair<__half>(uint32_t u) {
  return make_float2(__half2float(__ushort_as_half((unsigned short)(u & 0xffffu))),
                     __half2float(__ushort_as_half((unsigned short)(u >> 16))));
}
template <> __device__ __forceinline__ float2 unpack_pair<__nv_bfloat16>(uint32_t u) {
  return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
}
// Whether one of eight elements is infinite or not a number: only then is the
// sum of their products with 0 not 0.
__device__ __forceinline__ bool odd_sum(__half2 x, __half2 y, __half2 z, __half2 w) {
  const __half2 o = __float2half2_rn(0.f), s = __hfma2(x, o, __hfma2(y, o, __hfma2(z, o, __hmul2(w, o))));
  return !__hbeq2(s, o);
}
__device__ __forceinline__ bool odd_sum(__nv_bfloat162 x, __nv_bfloat162 y, __nv_bfloat162 z, __nv_bfloat162 w) {
  const __nv_bfloat162 o = __float2bfloat162_rn(0.f), s = __hfma2(x, o, __hfma2(y, o, __hfma2(z, o, __hmul2(w, o))));
  return !__hbeq2(s, o);
}
template <typename T> __device__ __forceinline__ bool odd_chunk(uint4 v) {
  using P = typename std::conditional<std::is_same<T, __half>::value, __half2, __nv_bfloat162>::type;
  return odd_sum(reinterpret_cast<const P&>(v.x), reinterpret_cast<const P&>(v.y), reinterpret_cast<const P&>(v.z), reinterpret_cast<const P&>(v.w));
}

}  // namespace swapnet
