// LM head on 8-bit operands (include/asd8.h): packing of the weight, quantisation of the
// hidden states, and the matrix product with the margin-rule statistics.
//   logits[i, v] = sum_kb 2^(eh[i, kb] + ew[v / 128, kb]) sum_k h8[i, k] w8[v, k]
#include <algorithm>

#include "fp8.cuh"
#include "kernels8.h"
#include "lm_epilogue.cuh"
#include "tc.cuh"

namespace asd {
namespace {

struct Lm8Header {
  uint32_t magic, version;
  int32_t vocab, hidden, ranges;
};

// ---------------------------------------------------------------- packing W
// One CTA per 128 x 128 block of W: its scale, then its rows into their tiles.
constexpr int kPackThreads = 256;

__global__ void __launch_bounds__(kPackThreads)
    lm8_pack_kernel(const __nv_bfloat16* __restrict__ w, uint8_t* __restrict__ out, int V, int K,
                    int ranges) {
  __shared__ uint32_t s_max[2];
  const int nkb = lm8_kblocks(K), kb = blockIdx.x % nkb, vb = blockIdx.x / nkb;
  if (threadIdx.x < 2) s_max[threadIdx.x] = 0;
  __syncthreads();
  // thread: half a row (64 values as 8 chunks of 8) of the block
  const int r = threadIdx.x >> 1, half = threadIdx.x & 1;
  const int v = vb * 128 + r;
  uint4 x[8];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int k = kb * kLm8KB + half * 64 + i * 8;   // K % 8 == 0: whole chunks
    x[i] = v < V && k < K ? *reinterpret_cast<const uint4*>(w + static_cast<size_t>(v) * K + k)
                          : make_uint4(0u, 0u, 0u, 0u);
    m = max8(m, x[i]);
  }
  atomicMax(&s_max[0], __float_as_uint(max_of(m)));   // magnitudes order as integers
  __syncthreads();
  const bool infinite = !finite(__uint_as_float(s_max[0]));   // uniform over the CTA
  if (infinite) {
    float a = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) a = fmaxf(a, finite_max8(x[i]));
    atomicMax(&s_max[1], __float_as_uint(a));
    __syncthreads();
  }
  const int e = block_exponent(__uint_as_float(s_max[infinite ? 1 : 0]));
  const float inv = pow2(-e);
  if (threadIdx.x == 0) {
    out[kLm8Header + 4 * (static_cast<size_t>(kb / 4) * ((V + 127) / 128) + vb) + kb % 4] =
        static_cast<uint8_t>(e + kExpBias);
    if (blockIdx.x == 0) {
      Lm8Header* h = reinterpret_cast<Lm8Header*>(out);
      h->magic = kLm8Magic;
      h->version = kLm8Version;
      h->vocab = V;
      h->hidden = K;
      h->ranges = ranges;
    }
  }
  const int ngroups = (V + kLmBoxRows - 1) / kLmBoxRows, group = v / kLmBoxRows;
  if (group >= ngroups) return;
  // the row's range, its tile in the range, its row in the tile
  int c = static_cast<int>(static_cast<long long>(group) * ranges / ngroups);
  while (lm_range_begin(c + 1, ranges, ngroups) <= group) ++c;
  while (lm_range_begin(c, ranges, ngroups) > group) --c;
  const int gs = lm_range_begin(c, ranges, ngroups), ge = lm_range_begin(c + 1, ranges, ngroups);
  const int g0 = gs + (group - gs) / kLm8Groups * kLm8Groups, ng = min(kLm8Groups, ge - g0);
  const int row = v - g0 * kLmBoxRows;
  uint8_t* dst = out + lm8_tiles_at(V, K) +
                 static_cast<size_t>(kLm8GroupBytes) *
                     (static_cast<size_t>(nkb) * g0 + static_cast<size_t>(kb) * ng) +
                 static_cast<size_t>(row) * kLm8KB;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint2 lo = infinite ? quantize8<true>(x[2 * i], inv) : quantize8(x[2 * i], inv);
    const uint2 hi = infinite ? quantize8<true>(x[2 * i + 1], inv) : quantize8(x[2 * i + 1], inv);
    *reinterpret_cast<uint4*>(dst + (((half * 4 + i) ^ (row & 7)) << 4)) =
        make_uint4(lo.x, lo.y, hi.x, hi.y);
  }
}

// ------------------------------------------------------- hidden states in e4m3
// One warp per (node, two k-blocks): half a warp holds a block, 8 values a lane.
// Scale byte of row i (of `rows`) and k-block kb: words of four k-blocks, as the tensor
// core takes them.
__device__ __forceinline__ size_t lm8_scale_at(int i, int kb, int rows) {
  return 4 * (static_cast<size_t>(kb / 4) * rows + i) + kb % 4;
}

constexpr int kHidThreads = 256;

__global__ void __launch_bounds__(kHidThreads) lm8_hidden_kernel(const Lm8Params p) {
  // (the stream's work before the call is complete: tree preparation, in front of this kernel,
  // has waited for it and touches none of what is read or written here)
  pdl_launch_dependents();
  const int nkb = lm8_kblocks(p.lm.K), pairs = (nkb + 1) / 2;
  const int lane = threadIdx.x & 31;
  const long long w = static_cast<long long>(blockIdx.x) * (kHidThreads / 32) + (threadIdx.x >> 5);
  const int i = static_cast<int>(w / pairs), kb = static_cast<int>(w % pairs) * 2 + (lane >> 4);
  if (i < p.lm.T && kb < nkb) {
    const int k = kb * kLm8KB + (lane & 15) * 8;
    const uint4 x = k < p.lm.K ? *reinterpret_cast<const uint4*>(
                                     static_cast<const __nv_bfloat16*>(p.lm.hidden) +
                                     static_cast<size_t>(i) * p.lm.K + k)
                               : make_uint4(0u, 0u, 0u, 0u);
    float m = finite_max8(x);
    const unsigned mask = 0xffffu << (lane & 16);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(mask, m, o));
    const int e = block_exponent(m);
    *reinterpret_cast<uint2*>(p.h8 + (static_cast<size_t>(i) * nkb + kb) * kLm8KB + (lane & 15) * 8) =
        quantize8<true>(x, pow2(-e));
    if ((lane & 15) == 0)
      p.h_exp[lm8_scale_at(i, kb, p.t_pad)] = static_cast<uint8_t>(e + kExpBias);
  } else if (i < p.t_pad && kb < nkb) {   // rows of the last node tile that no node owns
    if ((lane & 15) == 0) p.h_exp[lm8_scale_at(i, kb, p.t_pad)] = kExpBias;
  }
  pdl_wait();   // the LM head's wait covers the tree preparation too
}

// ------------------------------------------------------------------ the product
// D[128 nodes, up to 224 vocabulary rows] += h8[128, 128] x w8[224, 128]^T per k-block,
// tcgen05.mma with block scales: the tensor core multiplies every 32 products' sum by
// 2^(eh + ew) before it adds it to the fp32 accumulator in TMEM, so that blocks of unlike
// scale cost nothing.  Its scale operands want a byte per row and 32 columns; a block of
// 128 repeats its byte four times.  As in the bf16 LM head, TMEM lane i holds node row i
// and the thread that owns it reduces the row over the vocabulary; each CTA owns one
// contiguous vocabulary range and streams it once per NT node tiles.
//
// NT = 1 (up to 128 nodes): two 224-column accumulators that take the vocabulary tiles
// in turn.  NT = 2 (more nodes): two node tiles share every W stage, an accumulator each,
// and W is streamed once per 256 nodes.  224 rows is what two accumulators leave of the
// 512 TMEM columns beside the scales, and the more rows share a hidden tile's copy, the
// less of it crosses L2: 16 KB of hidden rows a k-block and node tile, 28 KB of W.
//
// A stage of the ring holds one k-block of W and of the node tiles.  The scale operands
// have a ring of their own: a scale word's four bytes are those of four k-blocks, of which
// an MMA names the one it wants, so they are copied once for four.
//
// Warp roles: warp 0 TMA producer, warp 1 TMEM allocator and MMA issuer of node tile 0,
// warps 2-5 (and 6-9 with NT = 2) epilogue of node tile 0 (1), then the warp that writes
// the scale operands and, with NT = 2, the MMA issuer of node tile 1: one warp's waits and
// 8 MMAs took 1120 cycles a k-block, more than the tensor core does (940).
// What bounds NT = 1 (W 128256 x 4096: 1 node 81 us, 128 85 us, 6.2 TB/s) is the stream of
// W.  NT = 2 (256 nodes 112 us, 512 209 us, 2.6 PFLOP/s) is bound by shared memory: the
// MMAs read 2 x 4 x (4 + 7) KB a k-block and the copies write 60 KB, 1156 cycles at 128 B
// each against 896 of MMAs.  Neither more copies in flight (a ring each for W and the node
// tiles) nor node tiles multicast in clusters of two (44 KB a k-block from L2) moved it.
template <int NT>
struct Lm8Geom {
  static constexpr int kThreads = NT == 1 ? 224 : 384;
  static constexpr int kScaleWarp = NT == 1 ? 6 : 10;
  static constexpr int kWBytes = kLm8TileN * kLm8KB;         // 28 KB
  static constexpr int kMaxStages = NT == 1 ? 6 : 3;
  static constexpr int kSfStages = 2;                        // scale operands of 4 k-blocks
  static constexpr int kSfBytes = NT * 512 + 1024;
  static constexpr int kSfCols = 4 + 8;                      // TMEM columns of an issuer's
  static constexpr uint32_t kSfCol0 = 2 * kLm8TileN;
  static_assert(kSfCol0 + kSfStages * NT * kSfCols <= 512, "TMEM columns");
  __host__ __device__ static constexpr int slot(int a_rows) { return NT * a_rows * kLm8KB + kWBytes; }
  __host__ __device__ static constexpr int stages(int a_rows) {
    return NT == 1 ? (a_rows <= 64 ? 6 : 5) : 3;
  }
  static constexpr size_t smem(int a_rows) {
    return 1024 + static_cast<size_t>(stages(a_rows)) * slot(a_rows) + kSfStages * kSfBytes;
  }
};
constexpr uint32_t kLm8Tmem = 512;

__device__ __forceinline__ void tc_mma_mx8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc,
                                           uint32_t sfa, uint32_t sfb, uint32_t accumulate,
                                           uint32_t on) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.ne.b32 q, %7, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, "
      "[%5], [%6], p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(sfa), "r"(sfb), "r"(on)
      : "memory");
}
template <int NT>
__global__ void __launch_bounds__(Lm8Geom<NT>::kThreads, 1)
    lmhead_fp8_kernel(const __grid_constant__ CUtensorMap tm_h, const Lm8Params p8) {
  using G = Lm8Geom<NT>;
  constexpr int kMax = G::kMaxStages, SF = G::kSfStages;
  const LmParams& p = p8.lm;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t s_full[kMax], s_empty[kMax];
  __shared__ __align__(8) uint64_t s_sf_full[SF], s_sf_empty[SF];
  __shared__ __align__(8) uint64_t s_tfull[2], s_tempty[2];
  __shared__ __align__(8) uint64_t s_mma_done[NT];
  __shared__ uint32_t s_tmem;
  __shared__ volatile int s_abort;
  __shared__ int s_pack_bad;
  __shared__ int s_issued[kMax];

  pdl_launch_dependents();
  const int warp = warp_index(), lane = threadIdx.x & 31;
  const long long budget = wait_budget(p.wait_cycles);
  const int a_rows = NT == 1 ? p.a_rows : 128, S = G::stages(a_rows), slot = G::slot(a_rows);
  const int a_blk = a_rows * kLm8KB;   // a node tile's k-block

  const int ngroups = (p.V + kLmBoxRows - 1) / kLmBoxRows;
  const int gs = lm_range_begin(blockIdx.x, p.g_lm, ngroups);
  const int ge = lm_range_begin(blockIdx.x + 1, p.g_lm, ngroups);
  const int nkb = lm8_kblocks(p.K), nk4 = (nkb + 3) / 4;
  const int nnt = (p.T + 127) / 128, rounds = (nnt + NT - 1) / NT;

  uint32_t base = smem_u32(smem_raw);
  const uint32_t pad = (1024u - (base & 1023u)) & 1023u;
  base += pad;
  const uint32_t sf0 = base + S * slot;
  uint8_t* g_sf = smem_raw + pad + S * slot;

  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) {
      mbar_init(smem_u32(&s_full[s]), 1);
      mbar_init(smem_u32(&s_empty[s]), NT);   // each issuer's MMAs are done with it
      s_issued[s] = 0;
    }
    for (int s = 0; s < SF; ++s) {
      mbar_init(smem_u32(&s_sf_full[s]), 1);
      mbar_init(smem_u32(&s_sf_empty[s]), NT);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(smem_u32(&s_tfull[a]), 1);
      mbar_init(smem_u32(&s_tempty[a]), 4);
    }
    for (int j = 0; j < NT; ++j) mbar_init(smem_u32(&s_mma_done[j]), 1);
    s_abort = 0;
    const Lm8Header* h = reinterpret_cast<const Lm8Header*>(p.w_packed);
    const int bad = h->magic != kLm8Magic || h->version != kLm8Version || h->vocab != p.V ||
                    h->hidden != p.K || h->ranges != p.g_lm;
    if (bad) set_status(p.status, ASD_ERR_SHAPE);
    s_pack_bad = bad;
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(&s_tmem), kLm8Tmem);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s_tmem;
  // vocabulary tiles of this CTA (none when the packed weight does not match)
  const int nvt = ge > gs && !s_pack_bad ? (ge - gs + kLm8Groups - 1) / kLm8Groups : 0;

  if (warp == 0) {
    // ------------------------------------------------------------ TMA producer
    const uint8_t* tiles = p.w_packed + lm8_tiles_at(p.V, p.K);
    const uint64_t pol_w = l2_policy_evict_first(), pol_h = l2_policy_evict_last();
    if (lane == 0) prefetch_tmap(&tm_h);
    auto load_w = [&](int st, int vt, int kb, int n) {   // lane 0; n: node tiles
      const int g0 = gs + vt * kLm8Groups, ng = min(kLm8Groups, ge - g0);
      const uint32_t full = smem_u32(&s_full[st]);
      mbar_expect_tx(full, static_cast<uint32_t>(n * a_blk + ng * kLm8GroupBytes));
      bulk_load(base + st * slot + NT * a_blk,
                tiles + static_cast<size_t>(kLm8GroupBytes) *
                            (static_cast<size_t>(nkb) * g0 + static_cast<size_t>(kb) * ng),
                static_cast<uint32_t>(ng * kLm8GroupBytes), full, pol_w);
      ++s_issued[st];
    };
    auto load_h = [&](int st, int rd, int kb, int n) {   // lane 0
      for (int j = 0; j < n; ++j)
        tma_load_2d(base + st * slot + j * a_blk, &tm_h, smem_u32(&s_full[st]), kb * kLm8KB,
                    (rd * NT + j) * 128, pol_h);
    };
    // The first stages' weights do not wait for the hidden states' quantisation.
    const int pre = nvt > 0 ? min(S, nkb) : 0;
    if (lane == 0)
      for (int i = 0; i < pre; ++i) load_w(i, 0, i, min(NT, nnt));
    pdl_wait();
    if (lane == 0)
      for (int i = 0; i < pre; ++i) load_h(i, 0, i, min(NT, nnt));
    int stage = pre == S ? 0 : pre;
    uint32_t ph = pre == S ? 1u : 0u;
    bool ok = true;
    for (int rd = 0; rd < rounds && ok; ++rd) {
      const int n = min(NT, nnt - rd * NT);
      for (int vt = 0; vt < nvt && ok; ++vt) {
        for (int kb = rd == 0 && vt == 0 ? pre : 0; kb < nkb; ++kb) {
          ok = __shfl_sync(0xffffffffu, mbar_wait(smem_u32(&s_empty[stage]), ph ^ 1u, budget), 0);
          if (!ok || s_abort) {
            ok = false;
            break;
          }
          if (lane == 0) {
            load_w(stage, vt, kb, n);
            load_h(stage, rd, kb, n);
          }
          __syncwarp();
          if (++stage == S) {
            stage = 0;
            ph ^= 1u;
          }
        }
      }
    }
    if (!ok && lane == 0) {
      note_timeout(p.status);
      s_abort = 1;
    }
    // every fill this CTA issued has landed before the CTA may leave
    if (lane == 0)
      for (int s = 0; s < S; ++s)
        if (s_issued[s] > 0)
          mbar_wait(smem_u32(&s_full[s]), static_cast<uint32_t>((s_issued[s] - 1) & 1));
    __syncwarp();
  } else if (warp == 1 || (NT == 2 && warp == 11)) {
    // -------------------------------------------------------------- MMA issuers
    const int j = NT == 2 && warp == 11 ? 1 : 0;   // node tile of the pair
    const uint32_t on = lane == 0 ? 1u : 0u;
    const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
    int stage = 0, sfs = 0;
    uint32_t ph = 0, sph = 0;
    bool ok = true;
    for (int rd = 0; rd < rounds && ok; ++rd) {
      // (tile 1 of an odd last round: nothing but the barriers' arrivals)
      const uint32_t here = rd * NT + j < nnt ? on : 0u;
      for (int vt = 0; vt < nvt && ok; ++vt) {
        const int g0 = gs + vt * kLm8Groups, ng = min(kLm8Groups, ge - g0);
        const int nrows = min(ng * kLmBoxRows, p.V - g0 * kLmBoxRows);
        const uint32_t idesc = idesc_mx8(128, (nrows + 15) & ~15);
        // NT = 1: the accumulators in turn; NT = 2: one for each node tile
        const int acc = NT == 1 ? vt & 1 : j;
        const uint32_t tph = static_cast<uint32_t>(((NT == 1 ? vt >> 1 : rd * nvt + vt) & 1) ^ 1);
        ok = (rd * NT + j >= nnt || wait_warp(&s_tempty[acc], tph, budget)) &&
             __all_sync(0xffffffffu, !s_abort);
        for (int kb = 0; kb < nkb && ok; ++kb) {
          const uint32_t c0 = tm + G::kSfCol0 + (NT * sfs + j) * G::kSfCols, cw = c0 + 4;
          if ((kb & 3) == 0) {
            ok = wait_warp(&s_sf_full[sfs], sph, budget);
            if (!ok) break;
            tc_fence_after();
            const uint32_t sf = sf0 + sfs * G::kSfBytes;
            tc_copy_scales(c0, sf + 512 * j, here);
            tc_copy_scales(cw, sf + NT * 512, here);
            tc_copy_scales(cw + 4, sf + NT * 512 + 512, here);
          }
          ok = wait_warp(&s_full[stage], ph, budget);
          if (!ok) break;
          tc_fence_after();
          const uint32_t a_s = base + stage * slot + j * a_blk, w_s = base + stage * slot + NT * a_blk;
          const uint32_t id = idesc | sf_byte_a(kb & 3) | sf_byte_b(kb & 3);
#pragma unroll
          for (int k = 0; k < 4; ++k)
            tc_mma_mx8(tm + acc * kLm8TileN, sw128_desc(a_s + 32 * k), sw128_desc(w_s + 32 * k), id,
                       c0, cw, (kb | k) != 0 ? 1u : 0u, here);
          tc_commit_on(smem_u32(&s_empty[stage]), on);
          if (++stage == S) {
            stage = 0;
            ph ^= 1u;
          }
          if ((kb & 3) == 3 || kb == nkb - 1) {
            tc_commit_on(smem_u32(&s_sf_empty[sfs]), on);
            if (++sfs == SF) {
              sfs = 0;
              sph ^= 1u;
            }
          }
        }
        if (!ok) break;
        tc_commit_on(smem_u32(&s_tfull[acc]), here);
      }
    }
    if (!ok && lane == 0) {
      note_timeout(p.status);
      s_abort = 1;
    }
    // every tcgen05 operation of this warp is done before TMEM is released
    __syncwarp();
    if (lane == 0) {
      tc_commit(smem_u32(&s_mma_done[j]));
      mbar_wait(smem_u32(&s_mma_done[j]), 0);
    }
    __syncwarp();
  } else if (warp == G::kScaleWarp) {
    // ---------------------------------------------------------- scale operands
    const uint32_t* w_exp = reinterpret_cast<const uint32_t*>(p.w_packed + kLm8Header);
    const uint32_t* h_exp = reinterpret_cast<const uint32_t*>(p8.h_exp);
    const int nvb = (p.V + 127) / 128;
    pdl_wait();
    int sfs = 0;
    uint32_t sph = 0;
    bool ok = true;
    for (int rd = 0; rd < rounds && ok; ++rd) {
      for (int vt = 0; vt < nvt && ok; ++vt) {
        const int g = gs + vt * kLm8Groups + lane;   // lanes 0-6: a 32-row group of W each
        for (int k4 = 0; k4 < nk4; ++k4) {
          const uint32_t w = lane < kLm8Groups && g < ge
                                 ? w_exp[static_cast<size_t>(k4) * nvb + g / 4]
                                 : 0x01010101u * kExpBias;
          uint32_t h[NT][4];
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            const int t0 = (rd * NT + j) * 128;   // (a tile past the last reads the first)
            const uint32_t* src =
                h_exp + static_cast<size_t>(k4) * p8.t_pad + (t0 < p8.t_pad ? t0 : 0) + lane;
#pragma unroll
            for (int k = 0; k < 4; ++k) h[j][k] = src[32 * k];
          }
          uint32_t wc[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) wc[k] = __shfl_sync(0xffffffffu, w, k);
          ok = __shfl_sync(0xffffffffu, mbar_wait(smem_u32(&s_sf_empty[sfs]), sph ^ 1u, budget), 0);
          if (!ok || s_abort) {
            ok = false;
            break;
          }
          uint4* dst = reinterpret_cast<uint4*>(g_sf + sfs * G::kSfBytes) + lane;
#pragma unroll
          for (int j = 0; j < NT; ++j) dst[32 * j] = make_uint4(h[j][0], h[j][1], h[j][2], h[j][3]);
          dst[32 * NT] = make_uint4(wc[0], wc[1], wc[2], wc[3]);
          dst[32 * NT + 32] = make_uint4(wc[4], wc[5], wc[6], wc[7]);
          fence_proxy_async();   // the tensor core's copy reads them
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&s_sf_full[sfs]));
          if (++sfs == SF) {
            sfs = 0;
            sph ^= 1u;
          }
        }
      }
    }
    if (!ok && lane == 0) {
      note_timeout(p.status);
      s_abort = 1;
    }
  } else {
    // ----------------------------------------------------------------- epilogue
    const int j = warp >= 6 ? 1 : 0;   // node tile of the pair
    const int q = warp & 3, row = q * 32 + lane;
    pdl_wait();
    bool ok = true;
    for (int rd = 0; rd < rounds && ok; ++rd) {
      if (rd * NT + j >= nnt) break;
      const int node = (rd * NT + j) * 128 + row;
      const bool active = node < p.T;
      RowState st;
      row_state_init(st, active, node, gs * kLmBoxRows, p.child_start, p.child_cnt, p.child_tok, p.T);
      for (int vt = 0; vt < nvt; ++vt) {
        const int g0 = gs + vt * kLm8Groups, ng = min(kLm8Groups, ge - g0);
        const int v0 = g0 * kLmBoxRows, nrows = min(ng * kLmBoxRows, p.V - v0);
        const int acc = NT == 1 ? vt & 1 : j;
        const int use = NT == 1 ? vt >> 1 : rd * nvt + vt;
        ok = __shfl_sync(0xffffffffu, mbar_wait(smem_u32(&s_tfull[acc]), use & 1, budget), 0);
        if (!ok || s_abort) {
          ok = false;
          break;
        }
        tc_fence_after();
        const uint32_t taddr = tmem + (static_cast<uint32_t>(q * 32) << 16) +
                               static_cast<uint32_t>(acc * kLm8TileN);
        for (int c = 0; c < ng; ++c) {
          float r[32];
          tmem_ld32(taddr + 32 * c, r);
          if (active)
            row_chunk(st, r, v0 + 32 * c, min(32, nrows - 32 * c), p.child_tok, p.child_id,
                      p.l_draft, p.T);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&s_tempty[acc]));
      }
      if (ok && active) {
        LmPartial part;
        part.m = st.m;
        part.s = st.s;
        part.a = st.a;
        part.pad = 0;
        p.part[static_cast<size_t>(node) * p.g_lm + blockIdx.x] = part;
      }
    }
    if (!ok && lane == 0) {
      note_timeout(p.status);
      s_abort = 1;
    }
  }

  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_dealloc(tmem, kLm8Tmem);
}

template <int NT>
cudaError_t launch_nt(const Lm8Params& p, const CUtensorMap& tm_h, cudaStream_t s) {
  const size_t smem = Lm8Geom<NT>::smem(NT == 1 ? p.lm.a_rows : 128);
  const cudaError_t err = set_smem_attrs(lmhead_fp8_kernel<NT>, smem);
  if (err != cudaSuccess) return err;
  return launch_pdl(lmhead_fp8_kernel<NT>, dim3(p.lm.g_lm), dim3(Lm8Geom<NT>::kThreads), smem, s,
                    tm_h, p);
}

}  // namespace

cudaError_t launch_lm8_pack(const void* w, void* w_packed, int vocab, int hidden, int ranges,
                            cudaStream_t s) {
  const long long blocks = static_cast<long long>((vocab + 127) / 128) * lm8_kblocks(hidden);
  if (blocks > 0x7fffffffLL) return cudaErrorInvalidValue;
  lm8_pack_kernel<<<static_cast<unsigned>(blocks), kPackThreads, 0, s>>>(
      static_cast<const __nv_bfloat16*>(w), static_cast<uint8_t*>(w_packed), vocab, hidden, ranges);
  return cudaGetLastError();
}

cudaError_t launch_lm8_hidden(const Lm8Params& p, cudaStream_t s) {
  const long long warps =
      static_cast<long long>(p.t_pad) * ((lm8_kblocks(p.lm.K) + 1) / 2);
  const long long ctas = (warps + kHidThreads / 32 - 1) / (kHidThreads / 32);
  if (ctas > 0x7fffffffLL) return cudaErrorInvalidValue;
  return launch_pdl(lm8_hidden_kernel, dim3(static_cast<unsigned>(ctas)), dim3(kHidThreads), 0, s, p);
}

cudaError_t launch_lmhead_fp8(const Lm8Params& p, const CUtensorMap& tm_h, cudaStream_t s) {
  return p.lm.T <= 128 ? launch_nt<1>(p, tm_h, s) : launch_nt<2>(p, tm_h, s);
}

}  // namespace asd
