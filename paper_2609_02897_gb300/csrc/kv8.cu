// The 8-bit K/V cache: conversion of a bf16 context and commit of an accepted path
// (include/asd8.h).  One warp per scale block (up to 32 tokens x D of K or V of one KV
// head): it holds the block in registers, 8 values a lane and step, reduces the largest
// magnitude with a packed maximum and a warp reduction, and writes each value once.
//
// Bound by memory traffic: the conversion reads two bytes and writes one per value, with
// all of a lane's loads (up to 16 of 16 bytes, 512 contiguous bytes a warp) in flight at
// once: 8 x 9000 to 16384 tokens of 8 heads x 128 101.5 us, 6.2 TB/s (0.92 of the measured
// copy rate; 245 us with 16 values a lane apart and every value looked at for infinities).
// The commit is pure latency: a few blocks per sequence and head.  Calls of few blocks run as
// one cluster that clears the status word itself; a kernel for it is what they would cost
// most, on the host (commit of 16 sequences 16.4 -> 13.5 us).
#include <algorithm>

#include "fp8.cuh"
#include "kernels8.h"

namespace asd {
namespace {

__device__ __forceinline__ float warp_max(float m) {
  // magnitudes: non-negative floats order as integers
  return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(m)));
}

// First row (of D values) and scale index of block j of sequence b, KV head g: false when
// the page id is outside the pool.
__device__ __forceinline__ bool block_at(const Kv8Params& p, int b, int g, int j, size_t& row,
                                         size_t& scale) {
  if (p.page_size == 0) {
    const size_t bg = static_cast<size_t>(b) * p.Hkv + g;
    row = bg * p.ctx_max + static_cast<size_t>(j) * p.block;
    scale = bg * p.blocks + j;
    return true;
  }
  const int per = p.blocks;   // blocks of a page
  const int page = p.page_table[static_cast<size_t>(b) * p.pages_per_seq + j / per];
  if (page < 0 || page >= p.num_pages) return false;
  const size_t pg = static_cast<size_t>(page) * p.Hkv + g;
  row = pg * p.page_size + static_cast<size_t>(j % per) * p.block;
  scale = pg * per + j % per;
  return true;
}

// A call's only kernel: its cluster's first CTA clears the status word before any CTA may
// set it.
__device__ __forceinline__ void begin(const Kv8Params& p) {
  pdl_wait();
  if (p.clear_status) {
    if (blockIdx.x == 0 && threadIdx.x == 0) p.status[0] = p.status[1] = 0;
    cluster_barrier();
  }
  pdl_launch_dependents();
}

// Scale exponent of a block from its packed maximum `m` of every lane; `again(finite)`
// gives a lane's largest finite magnitude where the block holds an infinity.
template <typename F>
__device__ __forceinline__ int warp_exponent(uint32_t m, bool& infinite, F again) {
  float a = warp_max(max_of(m));
  infinite = !finite(a);
  if (infinite) a = warp_max(again());   // uniform
  return block_exponent(a);
}

constexpr int kQuantThreads = 512;

// NC: 8-value chunks of a block per lane (block * D / 256).
template <int NC>
__global__ void __launch_bounds__(kQuantThreads) kv8_quantize_kernel(const Kv8Params p) {
  begin(p);
  const int lane = threadIdx.x & 31;
  const long long warps = static_cast<long long>(gridDim.x) * (kQuantThreads / 32);
  // items of the sequences one after another, dealt out to the warps in turn
  long long next = static_cast<long long>(blockIdx.x) * (kQuantThreads / 32) + (threadIdx.x >> 5);
  const int rsh = p.D == 64 ? 3 : 4;   // log2 of the chunks of a row
  for (int b0 = 0; b0 < p.B; b0 += 32) {
    const int mine = b0 + lane < p.B ? p.ctx_len[b0 + lane] : 0;
    for (int k = 0; k < 32 && b0 + k < p.B; ++k) {
      const int b = b0 + k, ctx = __shfl_sync(0xffffffffu, mine, k);
      if (ctx < 0 || ctx > p.ctx_max) {
        if (lane == 0) set_status(p.status, ASD_ERR_CTX_RANGE);
        continue;
      }
      const long long items =
          static_cast<long long>((ctx + p.block - 1) / p.block) * p.Hkv * 2;
      for (; next < items; next += warps) {
        const bool is_v = next & 1;
        const int j = static_cast<int>(next / (2 * p.Hkv));
        const int g = static_cast<int>(next / 2 - static_cast<long long>(j) * p.Hkv);
        size_t row, scale;
        if (!block_at(p, b, g, j, row, scale)) {
          if (lane == 0) set_status(p.status, ASD_ERR_CTX_RANGE);
          continue;
        }
        // chunks of the rows below the context's end
        const int chunks = min(p.block, ctx - j * p.block) << rsh;
        const uint4* src = reinterpret_cast<const uint4*>(
                               static_cast<const uint8_t*>(is_v ? p.v_src : p.k_src) + row * p.D * 2) +
                           lane;
        uint4 x[NC];
#pragma unroll
        for (int i = 0; i < NC; ++i)
          x[i] = i * 32 + lane < chunks ? __ldcs(src + i * 32) : make_uint4(0u, 0u, 0u, 0u);
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < NC; ++i) m = max8(m, x[i]);
        bool infinite;
        const int e = warp_exponent(m, infinite, [&] {
          float a = 0.f;
#pragma unroll
          for (int i = 0; i < NC; ++i) a = fmaxf(a, finite_max8(x[i]));
          return a;
        });
        const float inv = pow2(-e);
        uint2* dst = reinterpret_cast<uint2*>((is_v ? p.v : p.k) + row * p.D) + lane;
#pragma unroll
        for (int i = 0; i < NC; ++i)
          if (i * 32 + lane < chunks)
            dst[i * 32] = infinite ? quantize8<true>(x[i], inv) : quantize8(x[i], inv);
        if (lane == 0) (is_v ? p.v_exp : p.k_exp)[scale] = static_cast<uint8_t>(e + kExpBias);
      }
      next -= items;
    }
  }
}

constexpr int kCommitThreads = 1024;

// 4 e4m3 values times a power of two <= 1, rounded once more.
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float f) {
  const float2 a = e4m3x2_f32(w), b = e4m3x2_f32(w >> 16);
  return e4m3x2(a.x, a.y, f) | (e4m3x2(b.x, b.y, f) << 16);
}

// One CTA per sequence; the path and the pages that it is written to are checked once, then
// every warp takes blocks.
template <int NC>
__global__ void __launch_bounds__(kCommitThreads) kv8_compact_kernel(const Kv8Params p) {
  __shared__ int s_path[kMaxNodes];
  __shared__ int s_bad;
  begin(p);
  const int b = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int s0 = p.cu_nodes[b], n = p.cu_nodes[b + 1] - s0;
  const int ctx = p.ctx_len[b];
  int len = p.path_len[b];
  const bool tree_ok = s0 >= 0 && n > 0 && n <= p.max_nodes && n <= p.T && s0 <= p.T - n;
  if (threadIdx.x == 0) s_bad = 0;
  __syncthreads();
  const bool len_ok = tree_ok && len >= 0 && len <= p.max_path && len <= n;
  if (len_ok)
    for (int k = threadIdx.x; k < len; k += kCommitThreads) {
      const int u = p.path[static_cast<size_t>(b) * p.max_path + k];
      if (u < 0 || u >= n) s_bad = 1;
      s_path[k] = u;
    }
  __syncthreads();
  const bool path_ok = len_ok && !s_bad;
  bool ctx_ok = ctx >= 0 && path_ok && ctx <= p.ctx_max - len;
  if (p.page_size) {   // nothing is written where one of the pages is outside the pool
    bool bad = false;
    if (ctx_ok && len > 0) {
      const int first = ctx / p.page_size, last = (ctx + len - 1) / p.page_size;
      for (int k = first + threadIdx.x; k <= last; k += kCommitThreads) {
        const int page = p.page_table[static_cast<size_t>(b) * p.pages_per_seq + k];
        bad = bad || page < 0 || page >= p.num_pages;
      }
    }
    if (__syncthreads_or(bad)) ctx_ok = false;
  }
  if (!ctx_ok) len = 0;
  if (threadIdx.x == 0) {
    if (!tree_ok) set_status(p.status, ASD_ERR_TREE);
    else if (!path_ok) set_status(p.status, ASD_ERR_SHAPE);
    else if (!ctx_ok) set_status(p.status, ASD_ERR_CTX_RANGE);
    p.ctx_len_out[b] = ctx + len;
  }
  if (len == 0) return;
  const int rsh = p.D == 64 ? 3 : 4;   // log2 of the 8-value chunks of a row
  const int j0 = ctx / p.block, nj = (ctx + len - 1) / p.block - j0 + 1;
  for (int i0 = warp; i0 < nj * p.Hkv * 2; i0 += kCommitThreads / 32) {
    const bool is_v = i0 & 1;
    const int g = (i0 >> 1) % p.Hkv, j = j0 + (i0 >> 1) / p.Hkv;
    size_t row, scale;
    if (!block_at(p, b, g, j, row, scale)) continue;   // (no page: checked above)
    const int old = max(0, min(p.block, ctx - j * p.block));          // earlier rows of the block
    const int end = min(p.block, ctx + len - j * p.block);            // first row behind the path
    uint8_t* exps = (is_v ? p.v_exp : p.k_exp) + scale;
    const int e_old = old > 0 ? static_cast<int>(*exps) - kExpBias : kMinExp;
    const uint8_t* src = static_cast<const uint8_t*>(is_v ? p.v_src : p.k_src);
    uint2* dst = reinterpret_cast<uint2*>((is_v ? p.v : p.k) + row * p.D);
    uint4 x[NC];   // a new row's 8 bf16 values, or an earlier row's 8 bytes
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int c = i * 32 + lane, r = c >> rsh;
      x[i] = make_uint4(0u, 0u, 0u, 0u);
      if (r >= end) continue;
      if (r < old) {
        const uint2 q = dst[c];
        x[i].x = q.x;
        x[i].y = q.y;
      } else {
        const int u = s_path[j * p.block + r - ctx];
        x[i] = *reinterpret_cast<const uint4*>(
            src + ((static_cast<size_t>(s0 + u) * p.Hkv + g) * p.D + (c - (r << rsh)) * 8) * 2);
      }
    }
    auto fresh = [&](int i) { return (i * 32 + lane) >> rsh >= old; };
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < NC; ++i)
      if (fresh(i)) m = max8(m, x[i]);
    bool infinite;
    const int need = warp_exponent(m, infinite, [&] {
      float a = 0.f;
#pragma unroll
      for (int i = 0; i < NC; ++i)
        if (fresh(i)) a = fmaxf(a, finite_max8(x[i]));
      return a;
    });
    const int e = max(need, e_old);
    const float inv = pow2(-e), shift = e - e_old > 126 ? 0.f : pow2(e_old - e);
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int c = i * 32 + lane, r = c >> rsh;
      if (r >= end) continue;
      if (r >= old)
        dst[c] = infinite ? quantize8<true>(x[i], inv) : quantize8(x[i], inv);
      else if (e != e_old)
        dst[c] = make_uint2(rescale4(x[i].x, shift), rescale4(x[i].y, shift));
    }
    if (lane == 0) *exps = static_cast<uint8_t>(e + kExpBias);
  }
}

// 8-value chunks of a block per lane: 2, 4, 8 or 16.
int chunks_per_lane(const Kv8Params& p) { return p.block * p.D / 256; }

constexpr int kMaxCluster = 16;   // more than 8: not portable

// `ctas` (at most 16) as one cluster that clears the status word; a device that does not
// take it, or more CTAs, get a kernel for the word first.
template <typename K>
cudaError_t launch_clearing(K* kernel, long long ctas, int threads, Kv8Params p, bool one,
                            cudaStream_t s) {
  if (one && ctas <= kMaxCluster) {
    cudaError_t err = cudaSuccess;
    if (ctas > 8)
      err = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (err == cudaSuccess) {
      p.clear_status = 1;
      cudaLaunchConfig_t cfg = {};
      cfg.gridDim = dim3(static_cast<unsigned>(ctas));
      cfg.blockDim = dim3(static_cast<unsigned>(threads));
      cfg.stream = s;
      cudaLaunchAttribute attr[2];
      attr[0].id = cudaLaunchAttributeClusterDimension;
      attr[0].val.clusterDim.x = static_cast<unsigned>(ctas);
      attr[0].val.clusterDim.y = 1;
      attr[0].val.clusterDim.z = 1;
      attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
      attr[1].val.programmaticStreamSerializationAllowed = 1;
      cfg.attrs = attr;
      cfg.numAttrs = 2;
      err = cudaLaunchKernelEx(&cfg, kernel, p);
      if (err == cudaSuccess) return err;
    }
    cudaGetLastError();
    p.clear_status = 0;
  }
  const cudaError_t err = launch_clear_status(p.status, s);
  if (err != cudaSuccess) return err;
  return launch_pdl(kernel, dim3(static_cast<unsigned>(ctas)), dim3(static_cast<unsigned>(threads)), 0,
                    s, p);
}

}  // namespace

cudaError_t launch_kv8_quantize(const Kv8Params& p, int nsm, cudaStream_t s) {
  const int nc = chunks_per_lane(p);
  auto* k = nc == 16  ? kv8_quantize_kernel<16>
            : nc == 8 ? kv8_quantize_kernel<8>
            : nc == 4 ? kv8_quantize_kernel<4>
                      : kv8_quantize_kernel<2>;
  const int warps = kQuantThreads / 32;
  const long long items =
      static_cast<long long>(p.B) * ((p.ctx_max + p.block - 1) / p.block) * p.Hkv * 2;
  // one cluster up to four blocks a warp
  const bool one = items <= 4LL * warps * kMaxCluster;
  const long long ctas = std::max(1LL, std::min<long long>((items + warps - 1) / warps,
                                                           one ? kMaxCluster : 2LL * nsm));
  return launch_clearing(k, ctas, kQuantThreads, p, one, s);
}

cudaError_t launch_kv8_compact(const Kv8Params& p, cudaStream_t s) {
  const int nc = chunks_per_lane(p);
  auto* k = nc == 16  ? kv8_compact_kernel<16>
            : nc == 8 ? kv8_compact_kernel<8>
            : nc == 4 ? kv8_compact_kernel<4>
                      : kv8_compact_kernel<2>;
  if (p.in_step)
    return launch_pdl(k, dim3(static_cast<unsigned>(p.B)), dim3(kCommitThreads), 0, s, p);
  return launch_clearing(k, p.B, kCommitThreads, p, true, s);
}

}  // namespace asd
