// Keeping a decoder's key-value cache within its rows: eviction of the rows
// that got the least attention, and acceptance of a drafted path (its keys
// and values appended to every layer's cache).
#include <algorithm>
#include <cstring>
#include <string>

#include "cached.h"
#include "device.cuh"
#include "internal.h"
#include "kernels.h"

namespace swapnet {

namespace {

int done(cudaError_t e, const char* what) {
  if (e == cudaSuccess) e = cudaGetLastError();
  if (e != cudaSuccess) SN_FAIL(SWAPNET_ERR_CUDA, std::string(what) + ": " + cudaGetErrorString(e));
  return SWAPNET_OK;
}

// ------------------------------------------------------------------ eviction
// A weight as an unsigned number of the same order: -0 is 0, NaN the largest.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 0xffffffffu;
  const uint32_t u = __float_as_uint(w + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr int kEvBins = 2048;

// Inclusive sum over the block's N threads of x, and the sum of all; wtot: a
// word per warp in shared memory, free again after the next barrier.
template <int N> __device__ __forceinline__ uint32_t block_scan(uint32_t x, uint32_t* wtot, uint32_t* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const uint32_t o = __shfl_up_sync(0xffffffffu, x, off);
    if (lane >= off) x += o;
  }
  if (lane == 31) wtot[warp] = x;
  __syncthreads();
  const uint32_t own = lane < N / 32 ? wtot[lane] : 0u;
  uint32_t ws = own;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const uint32_t o = __shfl_up_sync(0xffffffffu, ws, off);
    if (lane >= off) ws += o;
  }
  *total = __shfl_sync(0xffffffffu, ws, 31);
  return x + __shfl_sync(0xffffffffu, ws - own, warp);
}

// One CTA per (sequence, key head): the rows to keep, in row order, into
// kept.  The candidates (all rows but the first `sink` and the last `recent`)
// give `need` rows: the need-th largest key by three histogram passes over 11,
// 11 and 10 of its bits, then one pass in row order that takes every larger key
// and the first of the equal ones.
// Bound by the latency of its passes: about 20 us for 256 pairs of up to 8001
// rows (the first round trip 1.7 us, three passes of 1 to 2 us with their sums,
// 4 us of the last pass's instructions), two CTAs per SM.  Keys kept in registers
// between the passes took the same, four passes over bytes 0.6 us more; clusters
// of eight CTAs per pair, reading each other's histograms, took 50 in place of 76
// us for 4 pairs of 84570 rows and 28 in place of 13 for 8 of 8000.
template <int N>
__global__ void __launch_bounds__(N) evict_select_kernel(const __grid_constant__ EvictArgs a) {
  __shared__ uint32_t hist[kEvBins], wtot[32];
  __shared__ uint32_t sh_prefix, sh_need;
  pdl_launch_dependents();  // (the rows' kernel may take its place on idle SMs; it waits for this one's end)
  const int kvh = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
  const int len = a.lens[b * a.lens_step];
  if (len < 0 || len > a.max_seq) {
    if (tid == 0) atomicExch(a.err, kDevErrBounds);
    return;
  }
  const int64_t pair = (int64_t)b * a.kv_heads + kvh;
  const float* w = a.weights + pair * a.max_seq;
  int* kept = a.kept + pair * a.keep;
  const int keep = min(len, a.keep);
  if (kvh == 0 && tid == 0 && a.lens_out) a.lens_out[b] = keep;
  const int c0 = len > keep ? a.sink : len, c1 = len > keep ? len - a.recent : len;  // candidates [c0, c1)
  uint32_t need = len > keep ? keep - a.sink - a.recent : 0, prefix = 0, all;
  if (need == 0) {
    prefix = 0xffffffffu;  // nothing but the protected rows
  } else {
    for (int shift = 21; shift >= 0; shift = shift == 10 ? 0 : shift - 11) {  // bits 31..21, 20..10, 9..0
      const uint32_t mask = shift == 0 ? 1023u : kEvBins - 1;
      const int known = shift == 21 ? 32 : shift == 10 ? 21 : 10;  // bits above are the prefix's
      for (int i = tid; i < kEvBins; i += N) hist[i] = 0;
      __syncthreads();
      for (int64_t j0 = c0 + tid; j0 < c1; j0 += 4 * N) {  // four loads on their way
        float x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = j0 + i * N < c1 ? w[j0 + i * N] : 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t key = weight_key(x[i]);
          if (j0 + i * N < c1 && (known == 32 || key >> known == prefix >> known)) atomicAdd(&hist[(key >> shift) & mask], 1u);
        }
      }
      __syncthreads();
      // from the largest bin down, kEvBins / N per thread
      constexpr int B = kEvBins / N;
      const int top = kEvBins - 1 - B * tid;
      uint32_t h[B], sum = 0;
#pragma unroll
      for (int i = 0; i < B; ++i) sum += h[i] = hist[top - i];
      uint32_t before = block_scan<N>(sum, wtot, &all) - sum;
      if (before < need && need <= before + sum) {
#pragma unroll
        for (int i = 0; i < B; ++i) {
          if (before < need && need <= before + h[i]) {
            sh_prefix = prefix | (uint32_t)(top - i) << shift;
            sh_need = need - before;
          }
          before += h[i];
        }
      }
      __syncthreads();
      prefix = sh_prefix;
      need = sh_need;
    }
  }
  // keys above `prefix` are taken, and the first `need` equal ones
  uint32_t taken = 0, equal = 0;  // before this tile
  for (int t0 = 0; t0 < len; t0 += 4 * N) {
    bool gt[4], eq[4];
    uint32_t mine = 0;  // taken in the low half, equal in the high half
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int j = t0 + 4 * tid + i;
      gt[i] = eq[i] = false;
      if (j < len) {
        if (j < c0 || j >= c1) {
          gt[i] = true;
        } else {
          const uint32_t key = weight_key(w[j]);
          gt[i] = key > prefix;
          eq[i] = need != 0 && key == prefix;
        }
      }
      mine += (gt[i] ? 1u : 0u) + (eq[i] ? 0x10000u : 0u);
    }
    const uint32_t before = block_scan<N>(mine, wtot, &all) - mine;
    uint32_t g = taken + (before & 0xffffu), e = equal + (before >> 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (gt[i] || (eq[i] && e < need)) kept[g + min(e, need)] = t0 + 4 * tid + i;
      g += gt[i];
      e += eq[i];
    }
    taken += all & 0xffffu;
    equal += all >> 16;
    __syncthreads();  // wtot is written again
  }
}

// Out of place: 16 bytes per thread, rows in any order.  Bound by DRAM: 0.53 GB
// read and written in 152 us, 7.0 TB/s (32 sequences, 8 heads of 128, half of
// up to 8001 rows; 173 us with the selection).
__global__ void __launch_bounds__(256) evict_copy_kernel(const __grid_constant__ EvictArgs a, int chunks) {
  pdl_wait();
  const int kvh = blockIdx.y, b = blockIdx.z;
  const int len = a.lens[b * a.lens_step];
  if (len < 0 || len > a.max_seq) return;
  const int n = min(len, a.keep) * chunks;
  const int* kept = a.kept + ((int64_t)b * a.kv_heads + kvh) * a.keep;
  const int64_t src0 = (int64_t)b * a.seq_stride + kvh * a.dim, dst0 = (int64_t)b * a.out_seq_stride + kvh * a.dim;
  for (int i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) {
    const int r = i / chunks, c = i % chunks;
    const int64_t from = src0 + (int64_t)kept[r] * a.kv_stride + c * 8, to = dst0 + (int64_t)r * a.out_stride + c * 8;
    const uint4 x = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.k) + from);
    const uint4 y = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.v) + from);
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.k_out) + to) = x;
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.v_out) + to) = y;
  }
  const int64_t pair = (int64_t)b * a.kv_heads + kvh;
  const float* w = a.weights + pair * a.max_seq;
  float* wo = a.weights_out + pair * a.out_seq;
  // (rows appended later start from nothing)
  for (int j = blockIdx.x * 256 + threadIdx.x; j < min(len, a.out_seq); j += gridDim.x * 256) wo[j] = j < a.keep ? w[kept[j]] : 0.f;
}

// In place: rows only move to lower ones, so a CTA that owns some columns of
// the keys or the values (or, the last one, the weights) moves them tile by
// tile in row order, every load of a tile before its stores.
constexpr int kEvMove = 4;  // rows per thread and tile
__global__ void __launch_bounds__(512) evict_move_kernel(const __grid_constant__ EvictArgs a, int slice) {
  pdl_wait();
  const int kvh = blockIdx.y, b = blockIdx.z;
  const int len = a.lens[b * a.lens_step];
  if (len <= a.keep || len > a.max_seq) return;  // (nothing moves)
  const int* kept = a.kept + ((int64_t)b * a.kv_heads + kvh) * a.keep;
  const int parts = gridDim.x / 2;
  if ((int)blockIdx.x == 2 * parts) {  // the weights
    float* w = a.weights_out + ((int64_t)b * a.kv_heads + kvh) * a.max_seq;
    for (int t0 = 0; t0 < a.keep; t0 += 512 * kEvMove) {
      float x[kEvMove];
#pragma unroll
      for (int i = 0; i < kEvMove; ++i) {
        const int r = t0 + (int)threadIdx.x + i * 512;
        if (r < a.keep) x[i] = w[kept[r]];
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kEvMove; ++i) {
        const int r = t0 + (int)threadIdx.x + i * 512;
        if (r < a.keep) w[r] = x[i];
      }
      __syncthreads();
    }
    for (int j = a.keep + (int)threadIdx.x; j < len; j += 512) w[j] = 0.f;  // (rows appended later start from nothing)
    return;
  }
  uint16_t* base = static_cast<uint16_t*>((int)blockIdx.x < parts ? a.k_out : a.v_out) + (int64_t)b * a.out_seq_stride +
                   kvh * a.dim + (int)(blockIdx.x % parts) * slice * 8;
  const int per = 512 / slice, c = threadIdx.x % slice, r0 = threadIdx.x / slice;
  const bool own = c + (int)(blockIdx.x % parts) * slice < a.dim / 8 && r0 < per;
  for (int t0 = 0; t0 < a.keep; t0 += per * kEvMove) {
    uint4 x[kEvMove];
#pragma unroll
    for (int i = 0; i < kEvMove; ++i) {
      const int r = t0 + r0 + i * per;
      if (own && r < a.keep) x[i] = *reinterpret_cast<const uint4*>(base + (int64_t)kept[r] * a.out_stride + c * 8);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kEvMove; ++i) {
      const int r = t0 + r0 + i * per;
      if (own && r < a.keep) *reinterpret_cast<uint4*>(base + (int64_t)r * a.out_stride + c * 8) = x[i];
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------- acceptance
// Every CTA walks its sequence's tree itself: after[i] is the lowest child of
// node i whose token is what the model chose at node i; the path starts at
// node 0.  Then it copies the path's rows of its cache.  Cache 0's CTA (or
// the only one, without caches) writes the results.  4.5 us for 64 caches of
// one sequence as for 32 caches of 32: a launch and four dependent loads.
__global__ void __launch_bounds__(256) tree_accept_kernel(const __grid_constant__ AcceptArgs a) {
  __shared__ int after[kTreeMax], path[kTreeMax], sh_n;
  const int b = blockIdx.y, cache = blockIdx.x, tid = threadIdx.x;
  const int len = a.lens[b], count = a.counts ? a.counts[b] : a.tokens;
  const int64_t row = (int64_t)b * a.tokens;
  bool bad = len < 0 || len > a.max_seq || count < 1 || count > a.tokens;
  int parent = -1;
  if (!bad && tid < count) {
    parent = a.parents ? a.parents[row + tid] : tid - 1;
    bad = parent < -1 || parent >= tid;
    after[tid] = kTreeMax;
  }
  if (__syncthreads_or(bad)) {
    if (tid == 0 && cache == 0) atomicExch(a.err, kDevErrBounds);
    return;
  }
  if (parent >= 0 && a.ids[row + tid] == a.targets[row + parent]) atomicMin(&after[parent], tid);
  __syncthreads();
  if (tid == 0) {
    int n = 0;
    for (int i = 0; i < kTreeMax; i = after[i]) path[n++] = i;  // (each step goes to a higher node)
    sh_n = n;
  }
  __syncthreads();
  const int n = sh_n;
  if (n > a.max_seq - len) {  // the cache has no room: nothing is accepted
    if (tid == 0 && cache == 0) atomicExch(a.err, kDevErrBounds);
    return;
  }
  if (cache == 0) {
    for (int i = tid; i < a.tokens; i += blockDim.x) a.path[row + i] = i < n ? path[i] : -1;
    if (tid == 0) {
      a.accepted[b] = n;
      a.next[b] = a.targets[row + path[n - 1]];
      a.lens_out[b] = len + n;
    }
  }
  if (cache >= a.n_caches) return;
  const int chunks = a.width / 8;
  uint16_t* to = static_cast<uint16_t*>(a.caches[cache]) + (int64_t)b * a.seq_stride + (int64_t)len * a.cache_stride;
  const uint16_t* from = static_cast<const uint16_t*>(a.drafts[cache]) + row * a.new_stride;
  for (int i = tid; i < n * chunks; i += blockDim.x) {
    const int r = i / chunks, c = i % chunks;
    *reinterpret_cast<uint4*>(to + (int64_t)r * a.cache_stride + c * 8) =
        *reinterpret_cast<const uint4*>(from + (int64_t)path[r] * a.new_stride + c * 8);
  }
}

template <typename A, typename... Args>
cudaError_t launch_after(void (*kern)(A, Args...), dim3 grid, int threads, cudaStream_t s, const A& a, Args... more) {
  cudaLaunchConfig_t cfg;
  std::memset(&cfg, 0, sizeof(cfg));
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, a, more...);
}

}  // namespace

int launch_cache_evict(const EvictArgs& a, cudaStream_t s) {
  const int64_t pairs = (int64_t)a.n_seq * a.kv_heads;
  const dim3 grid(a.kv_heads, a.n_seq);
  // Threads of a CTA, 256 / 1024 (us, with the copy): 352 pairs of 25 rows 9.3 / 13.0,
  // 256 of 200 rows 10.0 / 11.4, of 1000 19.5 / 21.4, of 8000 103 / 98; 8 of 2000 rows 9.6 /
  // 8.8, of 16000 32.5 / 20.0.
  if (a.max_seq <= 1024)
    evict_select_kernel<256><<<grid, 256, 0, s>>>(a);
  else
    evict_select_kernel<1024><<<grid, 1024, 0, s>>>(a);
  if (int rc = done(cudaGetLastError(), "eviction select launch")) return rc;
  const int chunks = a.dim / 8;
  if (a.k == a.k_out) {
    const int slice = std::min(4, chunks);  // 64 bytes of a row: whole sectors
    const int parts = (chunks + slice - 1) / slice;
    return done(launch_after(evict_move_kernel, dim3(2 * parts + 1, a.kv_heads, a.n_seq), 512, s, a, slice), "eviction move launch");
  }
  const int64_t full = ((int64_t)a.keep * chunks + 255) / 256;
  const int blocks = (int)std::max<int64_t>(1, std::min<int64_t>(full, (152 * 32 + pairs - 1) / pairs));
  return done(launch_after(evict_copy_kernel, dim3(blocks, a.kv_heads, a.n_seq), 256, s, a, chunks), "eviction copy launch");
}

int launch_tree_accept(const AcceptArgs& a, cudaStream_t s) {
  tree_accept_kernel<<<dim3(std::max(1, a.n_caches), a.n_seq), 256, 0, s>>>(a);
  return done(cudaGetLastError(), "tree acceptance launch");
}

}  // namespace swapnet
