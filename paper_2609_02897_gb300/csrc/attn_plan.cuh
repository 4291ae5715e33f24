// What the tensor-core attention kernels share: the plan that gives every CTA its query
// rows and keys (attention_tc.cu describes it), ancestor masks and the softmax warps'
// barriers.
#pragma once

#include <algorithm>

#include "kernels.h"
#include "tc.cuh"

namespace asd {
namespace {

constexpr int kRows = kAttnTcRows;   // query rows per CTA = TMEM lanes
constexpr int kKeys = kAttnTcKeys;   // keys per tile
constexpr int kThreads = 384;   // twelve warps (each kernel names their roles)
constexpr int kSoftmaxThreads = 256;   // eight warps: two per TMEM lane quarter

// Named barrier 1 of the softmax warps (N threads).
template <int N = kSoftmaxThreads>
__device__ __forceinline__ void softmax_sync() {
  asm volatile("bar.sync 1, %0;" ::"n"(N) : "memory");
}

// AND of `v` over the softmax warps (named barrier 1); uniform result.
template <int N = kSoftmaxThreads>
__device__ __forceinline__ bool softmax_all(bool v) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 q, %1, 0;\n\t"
      "barrier.cta.red.and.pred p, 1, %2, q;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(r)
      : "r"(v ? 1u : 0u), "n"(N)
      : "memory");
  return r != 0;
}

// OR of `v` over the softmax warps (named barrier 1); uniform result.
template <int N = kSoftmaxThreads>
__device__ __forceinline__ bool softmax_any(bool v) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 q, %1, 0;\n\t"
      "barrier.cta.red.or.pred p, 1, %2, q;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(r)
      : "r"(v ? 1u : 0u), "n"(N)
      : "memory");
  return r != 0;
}

// Every lane polls (bounded by `budget` cycles); the result is lane 0's,
// uniform over the warp.
__device__ __forceinline__ bool wait_all(uint64_t* bar, uint32_t parity, long long budget) {
  return __shfl_sync(0xffffffffu, mbar_wait(smem_u32(bar), parity, budget) ? 1 : 0, 0) != 0;
}

__device__ __forceinline__ bool aborted_warp(volatile int* s_abort) {
  return __shfl_sync(0xffffffffu, *s_abort, 0) != 0;
}

struct Item {
  int b, g, s0, n, r0, nrows, R;
  int key_base;              // first context key of the chunk (a multiple of kKeys)
  int ctx;                   // context length past key_base
  int nctx, ntree, ntiles;   // context, tree and all key tiles of the chunk
  int chunks, chunk, part0;  // chunks of the sequence, this one, the sequence's partial rows
};

constexpr int kOrderMax = 256;   // batches ordered by work in-kernel (larger ones: index order)

// Forms of the kernels compiled apart, since code that a call skips still costs it
// up to 1 %: calls of up to 128 nodes hand half of P over in two bf16 terms and may
// be the mma.sync kernel's (AttnParams::p_two, co_tiles); calls of about one wave of
// pairs go to either form by their context lengths (pair_ratio).
enum Mode { kPlain, kTwoTerms, kByContext };

constexpr int kMaxChunks = 32;   // chunks per sequence: one lane of the merging warp each
constexpr int kMergeOverhead = 3;   // cost of the merge in key tiles of ~1 us

// Shared-memory scratch of make_item, one entry per sequence.
struct PlanSmem {
  int s0[kOrderMax], n[kOrderMax], ctx[kOrderMax];   // first node, nodes, context length
  int tiles[kOrderMax];    // key tiles (0: no query rows)
  int items[kOrderMax];    // query row blocks x KV heads
  int key[kOrderMax];      // key tiles of the longest chunk
  int2 order[kOrderMax];   // larger first: by key, then by index; the sequence's CTAs
  int part[kOrderMax];     // partial rows (0: one chunk)
  int chunks[kOrderMax];
  int cut_ctas[kMaxChunks];   // CTAs and partial rows when the longest sequence is
  int cut_part[kMaxChunks];   // cut into 1, 2, ... chunks
  AloneTiles alone[kMaxNodes / 32];   // a call by itself: sums over 32 sequences each
  int past;                // items in all where they are more than the grid's CTAs, else 0
  int seq, first, part0;   // the sequence of this CTA, its first CTA and partial row
};

// ceil(t / len) and a / b for quotients up to about 2^12, from an approximate
// reciprocal (the estimate is then off by one at most).
__device__ __forceinline__ int ceil_div_est(int t, int len, float inv) {
  int c = static_cast<int>(static_cast<float>(t) * inv);
  c -= (c - 1) * len >= t ? 1 : 0;
  c += c * len < t ? 1 : 0;
  c += c * len < t ? 1 : 0;
  return c;
}
__device__ __forceinline__ int div_est(int a, int b) {
  int q = static_cast<int>(static_cast<float>(a) * __frcp_rn(static_cast<float>(b)));
  q -= q * b > a ? 1 : 0;
  q += (q + 1) * b <= a ? 1 : 0;
  return q;
}

// Sort key of a sequence: the length of its chunks, then its index, ascending.
__device__ __forceinline__ int order_key(int tiles, int q) {
  static_assert(kOrderMax <= 512, "9 bits of index");
  return (min(tiles, 1 << 21) << 9) | (511 - q);
}

// Key tiles per chunk.  Lane k weighs cutting the longest sequence into k + 1
// chunks (and the others into chunks no longer than its), each warp adding up
// some of the sequences.  The chunks run at once, one CTA per SM (a second wave
// would pay a CTA's overhead again), so a step takes its longest chunk: the
// shortest length that fits, unless the merge costs more than the cut saves.
// Every thread of the CTA calls it (it synchronises the CTA) and returns the
// same length; s.cut_* are zero on entry.  It stands between the start of every
// CTA and its first copy: 1.0 us (1.9 with three candidates per warp, a lane per
// sequence).
template <int WARPS>
__device__ __forceinline__ int chunk_length(const AttnParams& p, PlanSmem& s) {
  static_assert(kMaxChunks == 32, "a lane per candidate");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int longest = 1, items = 0;
  for (int q = lane; q < p.B; q += 32) {
    longest = max(longest, s.tiles[q]);
    items += s.items[q];
  }
  longest = __reduce_max_sync(0xffffffffu, longest);
  items = __reduce_add_sync(0xffffffffu, items);
  if (items == 0 || items > p.nsm) return longest;   // uniform over the CTA
  const int len = (longest + lane) / (lane + 1);
  const float inv = __frcp_rn(static_cast<float>(len));
  int ctas = 0, part = 0;
  for (int q = warp; q < p.B; q += WARPS) {
    const int c = ceil_div_est(s.tiles[q], len, inv);
    ctas += s.items[q] * c;
    part += c > 1 ? s.n[q] * p.Hq * c : 0;
  }
  if (warp < p.B) {
    atomicAdd(&s.cut_ctas[lane], ctas);
    atomicAdd(&s.cut_part[lane], part);
  }
  __syncthreads();
  ctas = s.cut_ctas[lane];
  part = s.cut_part[lane];
  // one chunk each (lane 0) is always possible
  const unsigned cost = lane > 0 && (part > p.part_cap || ctas > p.nsm)
                            ? 0xffffffffu
                            : static_cast<unsigned>(len + (part > 0 ? kMergeOverhead : 0));
  const unsigned best = __reduce_min_sync(0xffffffffu, cost);
  return __shfl_sync(0xffffffffu, len, __ffs(__ballot_sync(0xffffffffu, cost == best)) - 1);
}

// The chunk of CTA blockIdx.x: sequences in decreasing order of their chunks'
// length (ties by index), within one its KV heads, its chunks, its blocks of
// query rows (which read the same keys) innermost.  The hardware dispatches
// CTAs in blockIdx order, so the longest run first and the short ones fill the
// last wave.  False when the CTA has none.  Every thread of the CTA calls it (it
// synchronises the CTA).
template <int ROWS, int MODE, int WARPS = kThreads / 32>
__device__ __forceinline__ bool make_item(const AttnParams& p, Item& it, PlanSmem& s) {
  const int idx = blockIdx.x;
  int local, ctx, longest;   // longest: key tiles of the sequence's longest chunk
  if (ROWS == kRows && threadIdx.x == 0) s.past = 0;
  if (p.B > kOrderMax) {   // index order, unsplit
    const int rbmax = (p.max_nodes * p.G + ROWS - 1) / ROWS;
    it.b = idx / (rbmax * p.Hkv);
    if (it.b >= p.B) {
      __syncthreads();
      return false;
    }
    local = idx - it.b * rbmax * p.Hkv;
    it.g = local / rbmax;
    it.r0 = (local - it.g * rbmax) * ROWS;
    it.chunks = 1;
    it.chunk = 0;
    it.part0 = 0;
    it.s0 = p.cu_nodes[it.b];
    it.n = p.cu_nodes[it.b + 1] - it.s0;
    ctx = min(max(p.ctx_len[it.b], 0), p.ctx_max);
    longest = 0x3fffffff;
    __syncthreads();
  } else {
    // sequence extents and context lengths are caller inputs (the tree
    // preparation reports bad ones): a malformed sequence gets no CTA
    if (threadIdx.x == 0) s.seq = -1;
    if (threadIdx.x < kMaxChunks) s.cut_ctas[threadIdx.x] = s.cut_part[threadIdx.x] = 0;
    for (int q = threadIdx.x; q < p.B; q += blockDim.x) {
      const int s0 = p.cu_nodes[q], n = p.cu_nodes[q + 1] - s0;
      const int c = min(max(p.ctx_len[q], 0), p.ctx_max);
      const bool okq = n > 0 && n <= kMaxNodes && s0 >= 0 && s0 + n <= p.T;
      s.s0[q] = s0;
      s.n[q] = n;
      s.ctx[q] = c;
      s.tiles[q] = okq ? (c + kKeys - 1) / kKeys + (n + kKeys - 1) / kKeys : 0;
      s.items[q] = okq ? (n * p.G + ROWS - 1) / ROWS * p.Hkv : 0;
      s.key[q] = s.tiles[q];
      s.part[q] = 0;
      s.chunks[q] = 1;
      s.order[q] = make_int2(order_key(s.tiles[q], q), s.items[q]);
    }
    // B <= 128 here: a sequence per thread
    const bool choice = MODE == kTwoTerms && p.alone && p.co_tiles >= 0;
    if (choice && threadIdx.x < kMaxNodes) {
      const int q = threadIdx.x;
      AloneTiles a{0, 0, 0};
      if (q < p.B) a = alone_tiles(p, min(max(s.n[q], 0), kMaxNodes), s.ctx[q]);
      a = {__reduce_max_sync(0xffffffffu, a.longest), __reduce_add_sync(0xffffffffu, a.total),
           __reduce_add_sync(0xffffffffu, a.blocks)};
      if ((q & 31) == 0) s.alone[q >> 5] = a;
    }
    __syncthreads();
    // The mma.sync kernel's call: decided here, where the extents are at hand,
    // since in front of every CTA's set-up (attention_takes_mma) it cost the several
    // waves of such a call 1.3 us each.
    if (choice) {
      AloneTiles a = s.alone[0];
#pragma unroll
      for (int w = 1; w < kMaxNodes / 32; ++w)
        a = {max(a.longest, s.alone[w].longest), a.total + s.alone[w].total,
             a.blocks + s.alone[w].blocks};
      if (alone_takes_mma(p, a)) return false;
    }
    if (p.part_cap > 0) {
      const int len = chunk_length<WARPS>(p, s);
      const float inv = __frcp_rn(static_cast<float>(len));
      for (int q = threadIdx.x; q < p.B; q += blockDim.x) {
        const int t = s.tiles[q], c = ceil_div_est(t, len, inv);
        s.chunks[q] = c;
        if (c > 1) {
          s.key[q] = (t + c - 1) / c;
          s.part[q] = s.n[q] * p.Hq * c;
          s.order[q] = make_int2(order_key(s.key[q], q), s.items[q] * c);
        }
      }
      __syncthreads();
    }
    // the CTAs (and partial rows) of the sequences before each one, a thread per
    // sequence: on the way of every CTA's first copy (a warp per sequence, its
    // lanes over the others, was slower: 64 sequences of 8 nodes at contexts 300
    // to 1000, 3.4 waves of CTAs, 68.5 us against 61.2)
    for (int q = threadIdx.x; q < p.B; q += blockDim.x) {
      const int2 mine = s.order[q];
      int first = 0, part = 0;
#pragma unroll 8
      for (int j = 0; j < p.B; ++j) {
        const int2 o = s.order[j];
        first += o.x > mine.x ? o.y : 0;
      }
      if (ROWS == kRows && first + mine.y > static_cast<int>(gridDim.x))
        atomicMax(&s.past, first + mine.y);
      if (idx < first || idx >= first + mine.y) continue;
      if (p.part_cap > 0) {
        for (int j = 0; j < p.B; ++j) part += s.order[j].x > mine.x ? s.part[j] : 0;
        if (idx == first) p.plan[q] = make_int2(part, s.chunks[q]);
      }
      s.seq = q;
      s.first = first;
      s.part0 = part;
    }
    __syncthreads();
    it.b = s.seq;
    if (it.b < 0) return false;
    it.s0 = s.s0[it.b];
    it.n = s.n[it.b];
    ctx = s.ctx[it.b];
    it.chunks = s.chunks[it.b];
    it.part0 = s.part0;
    const int rb = (it.n * p.G + ROWS - 1) / ROWS;
    local = idx - s.first;
    const int gz = div_est(local, rb);
    it.r0 = (local - gz * rb) * ROWS;
    it.g = div_est(gz, it.chunks);
    it.chunk = gz - it.g * it.chunks;
    longest = s.key[it.b];
  }
  it.R = it.n * p.G;
  if (it.n <= 0 || it.n > kMaxNodes || it.s0 < 0 || it.s0 + it.n > p.T || it.r0 >= it.R)
    return false;
  it.nrows = min(ROWS, it.R - it.r0);
  const int nctx = (ctx + kKeys - 1) / kKeys, all = nctx + (it.n + kKeys - 1) / kKeys;
  // of the context's tiles, then the tree's, the first chunks take one more
  // than the others where they do not divide
  const int few = it.chunks == 1 ? all : (longest * it.chunks == all ? longest : longest - 1);
  const int more = all - few * it.chunks;
  const int t0 = it.chunk * few + min(it.chunk, more);
  const int t1 = t0 + few + (it.chunk < more ? 1 : 0);
  it.ntiles = t1 - t0;
  it.nctx = min(t1, nctx) - t0;
  it.ntree = it.ntiles - it.nctx;
  it.key_base = t0 * kKeys;
  it.ctx = ctx - it.key_base;
  return true;
}

__device__ __forceinline__ size_t grow_of(const AttnParams& p, const Item& it, int r) {
  const int rr = it.r0 + r;
  const int i = rr / p.G;
  return static_cast<size_t>(it.s0 + i) * p.Hq + it.g * p.G + (rr - i * p.G);
}

constexpr int kPageChunk = 512;   // page-table entries staged in shared memory

// Ancestor bitmasks (self included) of the sequence's nodes for the tree tile,
// by the softmax warps (N threads, tid: thread among them); a malformed parent ends
// the walk, so it is bounded.
template <int N = kSoftmaxThreads>
__device__ __forceinline__ void tree_masks(const AttnParams& p, const Item& it, int tid, int* s_par,
                                           uint64_t (*s_anc)[2]) {
  for (int i = tid; i < it.n; i += N) s_par[i] = p.parent[it.s0 + i];
  softmax_sync<N>();
  for (int i = tid; i < it.n; i += N) {
    uint64_t lo = 0, hi = 0;
    int u = i;
    while (true) {
      if (u < 64) lo |= 1ull << u; else hi |= 1ull << (u - 64);
      const int pu = s_par[u];
      if (pu < 0 || pu >= u) break;
      u = pu;
    }
    s_anc[i][0] = lo;
    s_anc[i][1] = hi;
  }
  softmax_sync<N>();
}

// Cache row of context position j of sequence b, KV head g; false (and reported) when its page
// id is outside the pool.
__device__ __forceinline__ bool context_row(const AttnParams& p, int b, int g, int j, size_t& at) {
  if (p.page_size == 0) {
    at = (static_cast<size_t>(b) * p.Hkv + g) * p.ctx_max + j;
    return true;
  }
  const int page = p.page_table[static_cast<size_t>(b) * p.pages_per_seq + j / p.page_size];
  if (page < 0 || page >= p.num_pages) {
    set_status(p.status, ASD_ERR_CTX_RANGE);
    return false;
  }
  at = (static_cast<size_t>(page) * p.Hkv + g) * p.page_size + j % p.page_size;
  return true;
}

// A lane's columns of a row of D = 32 V bf16 values.
template <int V>
__device__ __forceinline__ void load_columns(const __nv_bfloat16* row, int lane, float (&x)[V]) {
#pragma unroll
  for (int k = 0; k < V; ++k) x[k] = __bfloat162float(row[lane * V + k]);
}

// One-tile form: the items past the grid, which has a CTA for every item of
// sequences that do not overlap.  A batch whose cu_nodes run backwards (reported as
// ASD_ERR_TREE) can make more, and its well-formed sequences keep their outputs.
// Plain loops over the keys, a warp per query row, by the eight softmax warps (tid:
// thread among them) of every CTA when it is done; `context` gives a lane's columns of
// a context position's K and V.  (In the ping-pong form the branch cost the tile loop
// 2 %; its grid covers every item instead.)
template <int D, typename Context>
__device__ __forceinline__ void items_past_grid(const AttnParams& p, PlanSmem& s, int tid,
                                                const Context& context) {
  constexpr int kV = D / 32;   // a lane's columns
  const int lane = tid & 31;
  for (int idx = gridDim.x + blockIdx.x; idx < s.past; idx += gridDim.x) {
    softmax_sync();   // everyone is done with the last item's sequence
    for (int q = tid; q < p.B; q += kSoftmaxThreads) {
      int first = 0;
      for (int j = 0; j < p.B; ++j) first += s.order[j].x > s.order[q].x ? s.order[j].y : 0;
      if (idx < first || idx >= first + s.order[q].y) continue;
      s.seq = q;
      s.first = first;
      if (idx == first && p.part_cap > 0) p.plan[q] = make_int2(0, 1);   // nothing to merge
    }
    softmax_sync();
    const int b = s.seq, s0 = s.s0[b], R = s.n[b] * p.G, rb = (R + kRows - 1) / kRows;
    const int g = (idx - s.first) / rb, r0 = (idx - s.first - g * rb) * kRows;
    for (int r = r0 + (tid >> 5); r < min(r0 + kRows, R); r += kSoftmaxThreads / 32) {
      const int node = r / p.G;
      const size_t row = static_cast<size_t>(s0 + node) * p.Hq + g * p.G + (r - node * p.G);
      float q[kV], o[kV], kx[kV], vx[kV], m = -INFINITY, l = 0.f;
      load_columns(static_cast<const __nv_bfloat16*>(p.q) + row * D, lane, q);
#pragma unroll
      for (int k = 0; k < kV; ++k) {
        q[k] *= p.scale_log2;
        o[k] = 0.f;
      }
      auto key = [&] {
        float x = 0.f;
#pragma unroll
        for (int k = 0; k < kV; ++k) x = fmaf(q[k], kx[k], x);
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
        const float mn = fmaxf(m, x);
        const float al = m == -INFINITY ? 0.f : exp2f(m - mn);
        const float pe = x == -INFINITY ? 0.f : exp2f(x - mn);
        l = l * al + pe;
#pragma unroll
        for (int k = 0; k < kV; ++k) o[k] = fmaf(pe, vx[k], o[k] * al);
        m = mn;
      };
      for (int j = 0; j < s.ctx[b]; ++j)
        if (context(b, g, j, lane, kx, vx)) key();
      for (int u = node; u >= 0;) {   // the node and its ancestors
        const size_t at = (static_cast<size_t>(s0 + u) * p.Hkv + g) * D;
        load_columns(static_cast<const __nv_bfloat16*>(p.tree_k) + at, lane, kx);
        load_columns(static_cast<const __nv_bfloat16*>(p.tree_v) + at, lane, vx);
        key();
        const int pu = p.parent[s0 + u];
        u = pu < u ? pu : -1;
      }
      const float inv = l > 0.f ? 1.f / l : 0.f;
      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.out) + row * D;
#pragma unroll
      for (int k = 0; k < kV; ++k) out[lane * kV + k] = __float2bfloat16_rn(o[k] * inv);
    }
  }
}

}  // namespace
}  // namespace asd
