// Tree attention over an 8-bit K/V cache (include/asd8.h) on the 5th-generation tensor
// cores, without turning the cache into a wider type: its e4m3 bytes go from TMA to
// shared memory and are operands as they are.
//
//   S = q . K      q = 2^eq (q1 + q2), q1 in e4m3 (4 significant bits, to nearest) and q2, what
//                  that leaves, in e5m2: its 3 bits hold the rest of a bf16 number's 8, and
//                  its exponents reach as far as the number is at least 2^-13 of the row's
//                  largest (smaller ones to 2^-20 of that one); S = q1 K^T + q2 K^T, two MMAs
//                  of half a bf16 MMA's time, products exact, fp32 sums
//   x_j            = S_j log2(e)/sqrt(D) 2^(eq + ek[block of j]): the block scales of K
//                  are factors of the exponent
//   P_j            = 2^(x_j + ev[block of j] - R - d + 7), ev the exponents of V's blocks, R a
//                  reference of the row, d the largest floor(x_j + ev - R) among the 32 keys
//                  that an MMA step takes: at most 2^8, again in two e4m3 terms (2^-8 of P,
//                  2^-16 of the group's largest at least)
//   O += 2^(d-7) P V   two block-scaled MMAs over e4m3 V: the power of two is the MMA's scale byte
//                  of the row and the group, so no weight is small in its own group, however
//                  far the group's lie below the row's largest or its V below the largest V;
//                  output O 2^R / sum_j 2^x_j
//
// (With one reference for all of a row's weights, e4m3's smallest step was 2^-15 of it.  What
// lay below half of that was lost to P.V and not to the sum: a token with 0.9 of the weight
// in front of 16384 others cost them a quarter of what they add.)
//
// R is the largest x + ev of the row's first tile, and of a later one that exceeds it by more
// than kSlack; O is rescaled then, behind the weights, and all rows of the warp that have a larger
// one move at once.  The weight at R is a power of two, which P holds exactly: a token that
// has most of a row's weight keeps it.  (On scores as spread as a model's, the listed cases' outputs
// differ from fp32's by 8e-4 to 1.4e-3 of their norm, two bf16 roundings' flips included;
// 1.5e-3 to 2.2e-3 with whole numbers for R.  kSlack = 5 gives 5e-4 to 1e-3 and costs 8 x 64
// nodes at context 16384 3 %, 32 gives 9e-4 to 1.7e-3 and saves 1 %.)
//
// The last key tile holds the tree's own K and V in bf16: S and P.V of that tile are
// kind::f16 MMAs on a bf16 copy of q and on P = 2^(x - R) <= 2 in bf16 (2^-8 of each weight).
//
// Work items, chunks and their merge are those of attention_tc.cu's one-tile form.  Where
// items have few query rows, TMEM holds copies of them (up to 64 rows two; up to 32 three, four
// with D = 64), and the copies take the key tiles in turn, each with its own maxima, sums and
// O: a copy's softmax has that many tiles' time, and P is 0 in the other copies' lanes.  S of a
// tile is written to its copy's lanes only, so that the copies' S share their columns.
//
// More rows fill the tile, and the softmax is what takes the time.  The two threads of a lane
// then have an O each, the P.V of the tile's first and second 64 keys, and neither waits for
// the other within a tile; the output joins them as it does copies (8 x 64 nodes at context
// 16384 took 4 % less by it).
//
// TMEM (512 columns): with copies O [0, D), S [128, 256), P of copy k [256 + 64 k, 320 + 64 k),
// scales [448, 512) with D = 128 (which leaves room for three copies), [64, 128) with D = 64.
// An O for either key half: O [0, 2 D), then two (D = 64: three) buffers of 128 columns for S;
// each thread's P stands over its 64 columns of S and the tile's scales behind the first
// thread's P, all free when P.V is done.
//
// Warp roles (384 threads): warps 0 and 3 copy the even and the odd key tiles, K and V, and
// their block scales, warp 1 issues the S MMAs, warp 2 allocates TMEM and issues the P.V
// MMAs, warps 4-11 softmax and output.  (With a warp for K and one for V, the lookups and
// eight copies a page-of-16 tile takes, and the scales, were more than a tile's time.)
//
// The block scales are looked up for every BLK = 8, 16 or 32 keys, the cache's block: a
// factor, an addend and a share of the row sum each (all by 8: 168 -> 159 us there).
//
// What bounds it.  Per 128-key tile and SM, D = 128: 32 KB of cache, 1390 cycles at the
// measured copy rate; the tensor core 1080 (four terms of 128 x 128 x 128); shared memory
// 1020 (TMA's writes 256, MMA operands 768); converting K and V to bf16 on the way would
// take 1790 there.  Up to 64 rows that is near the copy rate once the tiles run (one token
// at 8 x 16384 60 us, 4.5 TB/s over the whole call), and short contexts are bound by what
// stands around the tiles: plan, query terms, first copies, output and merge, 12 us (1 x
// 1000 14 us, 8 nodes at 32k 26).  With 128 rows a tile takes 1800 cycles, of which the
// softmax warps issue for 1000 (8 x 64 nodes on 128 of 152 SMs 147 us, 0.94 PFLOP/s, on scores
// as spread as a model's).
#include <algorithm>

#include "attn_plan.cuh"
#include "fp8.cuh"
#include "kernels8.h"

namespace asd {
namespace {

constexpr int kStages = 4;        // tiles of the K ring, and of the V ring
constexpr uint32_t kTmemCols = 512;
constexpr int kSoftmaxWarp = 4, kSplit = 2;   // first softmax warp, threads per TMEM lane
constexpr int kCols = kKeys / kSplit;         // keys of a tile that a thread takes
constexpr int kSoftmax8 = 128 * kSplit;
constexpr int kThreads8 = 128 + kSoftmax8;
constexpr int kRing = 4;          // barriers of S, P and P.V, in turn
constexpr int kGroup = 32;        // keys of an MMA step, under one scale byte of a row
constexpr float kTop = 7.f;       // a group's largest weight is held in [2^7, 2^8]
constexpr float kSlack = 8.f;     // R is moved when a group's largest x + ev exceeds it by more

// Dynamic shared memory, 1024-byte aligned: q1, q2 [128 rows][D bytes], q in bf16
// [D/64][128 rows][128 bytes], the K ring, the V ring.  The tree's bf16 K and V tiles
// take the place of the K ring when every S of the context is done.
template <int D>
struct Geom {
  static constexpr int kTile = kKeys * D;               // K or V of a context tile
  static constexpr int kTreeTile = 2 * kTile;
  static constexpr int kQ8 = kRows * D;
  static constexpr int kQbOff = 2 * kQ8;
  static constexpr int kKOff = kQbOff + 2 * kRows * D;
  static constexpr int kVOff = kKOff + kStages * kTile;
  static constexpr int kBytes = kVOff + kStages * kTile;
  static constexpr int kTreeVOff = kKOff + kTreeTile;
  static_assert(2 * kTreeTile <= kStages * kTile, "the tree's K and V fit the K ring");
};

// Operand rows of D bytes: 128-byte lines with the 128-byte swizzle, or 64-byte lines
// with the 64-byte one; 8 lines form an atom.
template <int D>
__device__ __forceinline__ uint64_t desc8(uint32_t saddr) {
  uint64_t d = static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4);
  d |= static_cast<uint64_t>(1) << 16;
  d |= static_cast<uint64_t>(8 * D >> 4) << 32;
  d |= static_cast<uint64_t>(1) << 46;
  d |= static_cast<uint64_t>(D == 128 ? 2 : 4) << 61;
  return d;
}
// Byte offset of 16-byte chunk c of row r under that swizzle.
template <int D>
__device__ __forceinline__ int swz8(int r, int c) {
  return r * D + ((D == 128 ? c ^ (r & 7) : c ^ ((r >> 1) & 3)) << 4);
}

// kind::f8f6f4 instruction descriptor: A e4m3 or e5m2, B e4m3 -> fp32, both K-major.
__device__ __forceinline__ uint32_t idesc_f8(int m, int n, bool a_e5m2) {
  return (1u << 4) | (a_e5m2 ? (1u << 7) : 0u) | (static_cast<uint32_t>(n >> 3) << 17) |
         (static_cast<uint32_t>(m >> 4) << 24);
}

// MMAs that the issuing warp runs converged, with `on` set in one lane (tc.cuh).
#define ASD_MMA_ON(name, kind, atype, aop, acon)                                              \
  __device__ __forceinline__ void name(uint32_t d, atype a, uint64_t b, uint32_t idesc,       \
                                       uint32_t accumulate, uint32_t on) {                    \
    asm volatile(                                                                             \
        "{\n\t.reg .pred p, q;\n\t"                                                           \
        "setp.ne.b32 p, %4, 0;\n\t"                                                           \
        "setp.ne.b32 q, %5, 0;\n\t"                                                           \
        "@q tcgen05.mma.cta_group::1.kind::" kind " [%0], " aop ", %2, %3, p;\n\t}" ::"r"(d), \
        acon(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(on)                                 \
        : "memory");                                                                          \
  }
ASD_MMA_ON(mma_f8, "f8f6f4", uint64_t, "%1", "l")
ASD_MMA_ON(mma_bf16, "f16", uint64_t, "%1", "l")
ASD_MMA_ON(mma_bf16_ts, "f16", uint32_t, "[%1]", "r")
#undef ASD_MMA_ON
// The same, leaving D as it is in the lanes of quarter k where `skip[k]` is all ones.
#define ASD_MMA_LANES_ON(name, kind)                                                          \
  __device__ __forceinline__ void name(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc,    \
                                       const uint32_t (&skip)[4], uint32_t accumulate,        \
                                       uint32_t on) {                                         \
    asm volatile(                                                                             \
        "{\n\t.reg .pred p, q;\n\t"                                                           \
        "setp.ne.b32 p, %4, 0;\n\t"                                                           \
        "setp.ne.b32 q, %5, 0;\n\t"                                                           \
        "@q tcgen05.mma.cta_group::1.kind::" kind                                             \
        " [%0], %1, %2, %3, {%6, %7, %8, %9}, p;\n\t}" ::"r"(d),                              \
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(on), "r"(skip[0]), "r"(skip[1]),     \
        "r"(skip[2]), "r"(skip[3])                                                            \
        : "memory");                                                                          \
  }
ASD_MMA_LANES_ON(mma_f8_lanes, "f8f6f4")
ASD_MMA_LANES_ON(mma_bf16_lanes, "f16")
#undef ASD_MMA_LANES_ON
// A (TMEM) x B with a scale byte per row and 32 columns of A, and of B.
__device__ __forceinline__ void mma_mx8_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc,
                                           uint32_t sfa, uint32_t sfb, uint32_t accumulate,
                                           uint32_t on) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.ne.b32 q, %7, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], [%1], %2, %3, "
      "[%5], [%6], p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(sfa), "r"(sfb), "r"(on)
      : "memory");
}
// ------------------------------------------------------------------- producers
// Where this lane's box of a context tile starts: the cache row, or -1 where it has none.
// Contiguous: one box of 128 keys, lane 0's; paged: a box of min(page, 128) rows for each
// page the tile touches, lane j taking page j, its id from a piece of the sequence's
// page-table row staged in shared memory.  Pages past the context are not loaded; an id
// outside the pool is reported and not loaded.
struct Pages {
  const AttnParams& p;
  const Item& it;
  int* staged;
  const int32_t* table;
  int psh, br, chunk0 = -kPageChunk;
  __device__ __forceinline__ Pages(const AttnParams& pp, const Item& i, int* s)
      : p(pp), it(i), staged(s), table(pp.page_table + static_cast<size_t>(i.b) * pp.pages_per_seq) {
    psh = pp.page_size ? 31 - __clz(pp.page_size) : 0;
    br = pp.page_size ? min(pp.page_size, kKeys) : kKeys;
  }
  // The pages of the 128 keys from `key0`, and of the tile before, are staged afterwards
  // (tiles come in order).
  __device__ __forceinline__ void stage(int key0, int lane) {
    if (p.page_size == 0 || ((key0 + kKeys - 1) >> psh) < chunk0 + kPageChunk) return;
    chunk0 = max(it.key_base, key0 - kKeys) >> psh;
    // the entries the item needs, all loads in flight at once
    const int end = min(p.pages_per_seq, ((it.key_base + it.nctx * kKeys - 1) >> psh) + 1);
    int v[kPageChunk / 32];
#pragma unroll
    for (int i = 0; i < kPageChunk / 32; ++i) {
      v[i] = -1;
      if (chunk0 + 32 * i + lane < end) v[i] = table[chunk0 + 32 * i + lane];
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < kPageChunk / 32; ++i) staged[32 * i + lane] = v[i];
    __syncwarp();
  }
  // the page of a staged key, -1 if it is outside the pool
  __device__ __forceinline__ int page(int key) const {
    const int g = staged[(key >> psh) - chunk0];
    return g >= 0 && g < p.num_pages ? g : -1;
  }
  __device__ __forceinline__ int row(int t, int lane) {
    const int key0 = it.key_base + t * kKeys;
    if (p.page_size == 0) return lane == 0 ? (it.b * p.Hkv + it.g) * p.ctx_max + key0 : -1;
    stage(key0, lane);
    const int key = key0 + lane * br;
    if (lane * br >= kKeys || key >= it.key_base + it.ctx) return -1;
    const int g = page(key);
    if (g < 0) set_status(p.status, ASD_ERR_CTX_RANGE);
    return g < 0 ? -1 : (g * p.Hkv + it.g) * p.page_size + (key & (p.page_size - 1));
  }
};
// Issues the boxes at `row` (the whole warp).
template <int D>
__device__ __forceinline__ void issue_tile(int row, int br, uint32_t dst, uint32_t bar,
                                           const CUtensorMap* tm, uint64_t pol, int lane) {
  const uint32_t valid = __ballot_sync(0xffffffffu, row >= 0);
  if (lane == 0) mbar_expect_tx(bar, static_cast<uint32_t>(__popc(valid) * br * D));
  __syncwarp();
  if (row >= 0) tma_load_2d(dst + lane * br * D, tm, bar, 0, row, pol);
}

// ---------------------------------------------------------------- block scales
// Factors of context tile t for every 8 of its keys, in a ring of kScaleSlots tiles;
// they are written once the tile's K slot was free.  (Then the ring's slot is: S of
// tile t - 4 was issued, so the copies had read S up to tile t - 8 at least, and each had
// finished its tile before, t - 12 or later.)
constexpr int kScaleSlots = 16;
constexpr int kGroups = kKeys / 8;
struct TileScales {
  float fk[kGroups];   // 2^ek
  float ev[kGroups];   // ev
  float gi[kGroups];   // 2^-ev, for the row sum
};

// A producer writes them behind its tile's copy: lane j < 16 K's byte for keys [8 j,
// 8 j + 8), lane 16 + j V's.
struct Scales {
  const Attn8Params& p8;
  const Item& it;
  Pages& pages;
  const uint8_t* exps;   // of this lane's tensor and KV head (paged: page 0's)
  int bsh, lane;
  __device__ __forceinline__ Scales(const Attn8Params& p, const Item& i, Pages& pg)
      : p8(p), it(i), pages(pg), lane(threadIdx.x & 31) {
    bsh = 31 - __clz(p8.block);
    exps = (lane < 16 ? p8.k_exp : p8.v_exp) +
           (static_cast<size_t>(p8.a.page_size ? 0 : it.b) * p8.a.Hkv + it.g) * p8.blocks;
  }
  // The byte of the lane's keys of tile t; the smallest scale's past the context and in pages
  // outside the pool.  Nothing is done with what is loaded, so that it can stay on its way.
  __device__ __forceinline__ int fetch(int t) {
    constexpr int kNone = kMinExp + kExpBias;
    if (t >= it.nctx) return kNone;
    pages.stage(it.key_base + t * kKeys, lane);
    const int k = t * kKeys + 8 * (lane & 15);
    if (k >= it.ctx) return kNone;
    const int key = it.key_base + k;
    if (p8.a.page_size == 0) return exps[key >> bsh];
    const int g = pages.page(key);
    return g < 0 ? kNone
                 : exps[static_cast<size_t>(g) * p8.a.Hkv * p8.blocks + ((key & (p8.a.page_size - 1)) >> bsh)];
  }
  // A tile's factors from its bytes.
  __device__ __forceinline__ void write(int byte, TileScales& s) {
    const int e = min(max(byte - kExpBias, kMinExp), 126);
    if (lane < 16) {
      s.fk[lane] = pow2(e);
    } else {
      s.ev[lane - 16] = static_cast<float>(e);
      s.gi[lane - 16] = pow2(-e);
    }
    __syncwarp();
  }
};

// ---------------------------------------------------------------------- softmax
// Four values of at most 448 -> words of their two e4m3 terms: the value rounded to fp16 (11
// bits), its 4 leading bits, to nearest, ties away from zero (an addition to the magnitudes:
// cheaper than converting e4m3 back, 159 -> 155 us for 8 x 64 nodes), and what that leaves
// (exact in fp16), both in e4m3.  A NaN, 0x7fff in fp16, stays one in the second term.
__device__ __forceinline__ void two_terms(const float (&w)[4], uint32_t& hi, uint32_t& lo) {
  asm("{\n\t.reg .b16 a, b, c, d;\n\t.reg .b32 p, q, r, s;\n\t"
      "cvt.rn.f16x2.f32 p, %3, %2;\n\t"
      "cvt.rn.f16x2.f32 q, %5, %4;\n\t"
      "add.u32 r, p, 0x00400040;\n\t"
      "add.u32 s, q, 0x00400040;\n\t"
      "and.b32 r, r, 0xff80ff80;\n\t"
      "and.b32 s, s, 0xff80ff80;\n\t"
      "cvt.rn.satfinite.e4m3x2.f16x2 a, r;\n\t"
      "cvt.rn.satfinite.e4m3x2.f16x2 b, s;\n\t"
      "mov.b32 %0, {a, b};\n\t"
      "sub.rn.f16x2 r, p, r;\n\t"
      "sub.rn.f16x2 s, q, s;\n\t"
      "cvt.rn.satfinite.e4m3x2.f16x2 c, r;\n\t"
      "cvt.rn.satfinite.e4m3x2.f16x2 d, s;\n\t"
      "mov.b32 %1, {c, d};\n\t}"
      : "=r"(hi), "=r"(lo)
      : "f"(w[0]), "f"(w[1]), "f"(w[2]), "f"(w[3]));
}

// Four values of at most 448 with 8 significant bits -> words of e4m3 and of what that leaves,
// in e5m2.  (A value is exact in fp16, and so is the rest.)
__device__ __forceinline__ void two_terms_wide(const float (&q)[4], uint32_t& hi, uint32_t& lo) {
  asm("{\n\t.reg .b16 a, b, c, d;\n\t.reg .b32 p, q, r, s;\n\t"
      "cvt.rn.f16x2.f32 p, %3, %2;\n\t"
      "cvt.rn.f16x2.f32 q, %5, %4;\n\t"
      "cvt.rn.satfinite.e4m3x2.f16x2 a, p;\n\t"
      "cvt.rn.satfinite.e4m3x2.f16x2 b, q;\n\t"
      "mov.b32 %0, {a, b};\n\t"
      "cvt.rn.f16x2.e4m3x2 r, a;\n\t"
      "cvt.rn.f16x2.e4m3x2 s, b;\n\t"
      "sub.rn.f16x2 r, p, r;\n\t"
      "sub.rn.f16x2 s, q, s;\n\t"
      "cvt.rn.satfinite.e5m2x2.f16x2 c, r;\n\t"
      "cvt.rn.satfinite.e5m2x2.f16x2 d, s;\n\t"
      "mov.b32 %1, {c, d};\n\t}"
      : "=r"(hi), "=r"(lo)
      : "f"(q[0]), "f"(q[1]), "f"(q[2]), "f"(q[3]));
}

// bf16 pairs: a word with every value that is not finite as 0.
__device__ __forceinline__ uint32_t only_finite2(uint32_t w) {
  const uint32_t keep = ((w & 0x7f80u) == 0x7f80u ? 0u : 0xffffu) |
                        ((w & 0x7f800000u) == 0x7f800000u ? 0u : 0xffff0000u);
  return w & keep;
}
__device__ __forceinline__ uint4 only_finite(uint4 v) {
  return make_uint4(only_finite2(v.x), only_finite2(v.y), only_finite2(v.z), only_finite2(v.w));
}

struct Shared {   // what the roles share, beside the tiles
  uint64_t k_full[kStages], k_empty[kStages], v_full[kStages], v_empty[kStages];
  // tile t's are those of index t % kRing (s_empty: t % copies)
  uint64_t s_full[kRing];    // S in TMEM (MMA -> softmax)
  uint64_t s_empty[4];       // S of a copy in registers (softmax -> MMA)
  uint64_t p_full[kRing];    // P in TMEM (softmax -> MMA)
  uint64_t pv_done[kRing];   // O += P V done (MMA -> softmax)
  uint64_t q_ready, mma_done[2];
  uint64_t ctx_done;         // S of every context tile done: the K ring is free
  uint64_t tree_k, tree_v;   // the tree's K and V have landed
  uint64_t tree_clean;       // V's rows of no node, and values that are not finite, are 0
  uint64_t anc[kMaxNodes][2];
  TileScales sc[kScaleSlots];
  // scale bytes of the tiles' P (index t % kRing) as tc_copy_scales takes them, and V's, 2^0
  __align__(16) uint32_t sfa[kRing][kRows];
  __align__(16) uint32_t sfb[kRows];
  float mx[2][kSplit][kRows]; // [parity][key half][TMEM lane]: partial row max
  float l[kSplit][kRows];     // partial row sum
  float m[kRows], unit[kRows];
  uint32_t tmem;
  int odd_v;                 // the tree's V rows hold values that are not finite
  int abort;
  int par[kMaxNodes];
  int pages[2][kPageChunk];   // producers: staged page-table entries
  int issued[2][kStages];     // fills of K and V per stage
  int tree_issued;
};

// How an item's copies use TMEM.  REP: their number, 0 where it is each item's own.  A number
// that the code knows is worth 5 to 10 %; code for several numbers in one kernel costs calls
// that mix them more (fetched anew by every CTA of another number: ragged trees of 64 columns
// 52 -> 72 us).  So the host chooses (kernel_of_rows).
constexpr int kManyCopies = 4;   // REP: as many as TMEM has room for
template <int D, int REP>
struct Copies {
  static constexpr int kMost = D == 64 ? 4 : 3;
  int own;   // 1, 2 or kMost
  __device__ __forceinline__ explicit Copies(int nrows)
      : own(__all_sync(0xffffffffu, nrows <= 32) ? kMost : (__all_sync(0xffffffffu, nrows <= 64) ? 2 : 1)) {}
  __device__ __forceinline__ int rep() const { return REP == 0 ? own : (REP == kManyCopies ? kMost : REP); }
  // TMEM lane quarters of a copy (log2), and lanes
  __device__ __forceinline__ int quarters_log() const { return rep() > 2 ? 0 : 2 - (rep() >> 1); }
  __device__ __forceinline__ int span() const { return 32 << quarters_log(); }
  __device__ __forceinline__ int warps() const { return kSplit << quarters_log(); }   // softmax, of a copy
  // Each key half has an O of its own, the second at column D; P then takes the place of S,
  // in kOverBufs buffers.
  static constexpr bool kHalves = REP == 1;
  static constexpr int kOverBufs = D == 64 ? 3 : 2;
  __device__ __forceinline__ int p_bufs() const { return kHalves ? kOverBufs : max(rep(), 2); }
  __device__ __forceinline__ uint32_t s_col(int t) const {
    return kHalves ? 2 * D + 128 * (t % kOverBufs) : 128;
  }
  // The buffer of tile t's P, which is copy `copy`'s (t modulo their number; a division that
  // is not by a constant would stand in every tile's chain).
  __device__ __forceinline__ int p_buf(int t, int copy) const { return rep() == 1 ? t & 1 : copy; }
  __device__ __forceinline__ uint32_t p_col(int t, int copy) const {
    return kHalves ? s_col(t) : 256 + 64 * p_buf(t, copy);
  }
  // scale words of P and of V
  __device__ __forceinline__ uint32_t sfa_col(int t, int copy) const {
    return kHalves ? s_col(t) + kCols / 2 : sfb_col(t) + 4 + 4 * p_buf(t, copy);
  }
  __device__ __forceinline__ uint32_t sfb_col(int t) const {
    return kHalves ? s_col(t) + kCols / 2 + 4 : (D == 64 ? 64 : 448);
  }
};

// AND of `v` over the softmax warps of a TMEM lane quarter; uniform result.
__device__ __forceinline__ bool quarter_all(int quarter, bool v) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 q, %1, 0;\n\t"
      "barrier.cta.red.and.pred p, %2, %3, q;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(r)
      : "r"(v ? 1u : 0u), "r"(2 + quarter), "n"(32 * kSplit)
      : "memory");
  return r != 0;
}

// A softmax thread: keys [64 cq, 64 cq + 64) of the tiles of its copy, for one TMEM lane.
template <int D, int BLK, int REP>
struct Softmax {
  const Attn8Params& p8;
  const Item& it;
  Shared& sh;
  const Copies<D, REP> cp;
  uint8_t* gbase;
  uint32_t lane_base;
  int cq, row, copy;
  bool busy;                 // some row of this warp is a query's
  float c_row;
  uint64_t anc;              // the row's ancestors among the thread's keys of the tree tile
  long long budget;
  float R;                   // O is in units of 2^R; -infinity before the row's first key
  float m, l;                // sum of the weights 2^(x - m), m an integer

  __device__ __forceinline__ void mask(float (&x)[kCols], bool tree, int valid) const {
    const int own = min(max(valid - kCols * cq, 0), kCols);
    uint64_t am = own == 64 ? ~0ull : (1ull << own) - 1ull;
    if (tree) am &= anc;
    const uint32_t w[2] = {static_cast<uint32_t>(am), static_cast<uint32_t>(am >> 32)};
#pragma unroll
    for (int k = 0; k < kCols; ++k) x[k] = (w[k >> 5] >> (k & 31)) & 1u ? x[k] : -INFINITY;
  }
  // The largest x, and the largest x + ev of either group of keys (of the tree tile x).
  __device__ __forceinline__ float maximum(const float (&x)[kCols], const TileScales& sc, bool tree,
                                           float (&u)[kCols / kGroup]) const {
    const int s0 = cq * (kCols / 8);
    float mt = -INFINITY;
#pragma unroll
    for (int h = 0; h < kCols / kGroup; ++h) {
      u[h] = -INFINITY;
#pragma unroll
      for (int g = h * kGroup; g < (h + 1) * kGroup; g += BLK) {
        float mg = fmaxf(x[g], x[g + 1]);
#pragma unroll
        for (int k = 2; k < BLK; k += 2) mg = fmaxf(fmaxf(mg, x[g + k]), x[g + k + 1]);
        mg *= tree ? p8.a.scale_log2 : c_row * sc.fk[s0 + g / 8];
        mt = fmaxf(mt, mg);
        u[h] = fmaxf(u[h], tree ? mg : mg + sc.ev[s0 + g / 8]);
      }
    }
    return mt;
  }
  // The weights, as P: words of 4 e4m3 of either term (the second `lo_at` columns behind), the
  // groups' scale bytes at `sf`; the tree tile's as bf16 pairs.  p_at: the thread's keys'.
  // mt, u: from maximum.
  __device__ __forceinline__ void weights(const float (&x)[kCols], float mt, const float (&u)[kCols / kGroup],
                                          uint32_t p_at, uint32_t lo_at, const TileScales& sc,
                                          uint32_t* sf, bool tree) {
    const float rz = R == -INFINITY ? 0.f : R, mn = fmaxf(m, floorf(mt)), mz = mn == -INFINITY ? 0.f : mn;
    l *= ex2_approx(m - mz);   // (0 before the first key, with l)
    m = mn;
    if (!tree) {
      uint32_t bytes = 0;
#pragma unroll
      for (int h = 0; h < kCols / kGroup; ++h) {
        uint32_t hi[8], lo[8];
        // powers of two from R to the group's largest (finite where it has no key); the MMA's
        // scale, as little as a byte holds where it is less
        const float d = fmaxf(floorf(u[h] - rz), -1e6f) - kTop;
        bytes |= static_cast<uint32_t>(fminf(fmaxf(d + 127.f, 0.f), 254.f)) << (8 * h);
        const float top = rz + d, to_sum = ex2_approx(top - mz);
#pragma unroll
        for (int g = 0; g < kGroup / BLK; ++g) {
          const int at = kGroup * h + BLK * g, sg = (cq * kCols + at) / 8;
          const float f = c_row * sc.fk[sg], nb = sc.ev[sg] - top;
          const uint64_t f2 = pack_f32x2(f, f), nb2 = pack_f32x2(nb, nb);
          uint64_t sum = 0ull;
#pragma unroll
          for (int k = 0; k < BLK; k += 4) {
            float w[4];
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
              float y0, y1;
              unpack_f32x2(fma_f32x2(pack_f32x2(x[at + k + i], x[at + k + i + 1]), f2, nb2), y0, y1);
              w[i] = ex2_approx(y0);
              w[i + 1] = ex2_approx(y1);
              sum = add_f32x2(sum, pack_f32x2(w[i], w[i + 1]));
            }
            two_terms(w, hi[(BLK * g + k) / 4], lo[(BLK * g + k) / 4]);
          }
          float s0, s1;
          unpack_f32x2(sum, s0, s1);
          l = fmaf((s0 + s1) * sc.gi[sg], to_sum, l);
        }
        tmem_st8u(p_at + 8 * h, hi);
        tmem_st8u(p_at + lo_at + 8 * h, lo);
      }
      reinterpret_cast<uint16_t*>(sf)[((row & 31) * 4 + (row >> 5)) * 2 + cq] = static_cast<uint16_t>(bytes);
      fence_proxy_async();   // the tensor core's copy reads them
    } else {
      const float f = p8.a.scale_log2;
      float s = 0.f;
#pragma unroll
      for (int h = 0; h < kCols / 32; ++h) {
        uint32_t pk[16];
#pragma unroll
        for (int k = 0; k < 32; k += 2) {
          const float p0 = ex2_approx(fmaf(x[32 * h + k], f, -rz));
          const float p1 = ex2_approx(fmaf(x[32 * h + k + 1], f, -rz));
          s += p0 + p1;
          __nv_bfloat162 v = __floats2bfloat162_rn(p0, p1);
          pk[k / 2] = *reinterpret_cast<uint32_t*>(&v);
        }
        tmem_st16u(p_at + 16 * h, pk);
      }
      // (beyond 2^126 nothing of s is left: this thread's keys are as far below the row's)
      l = fmaf(s, ex2_approx(fminf(rz - mz, 126.f)), l);
    }
  }
  // O += P V of tile t is done.  (The caller knows that tile t - 4's is, and that tile
  // t + 4's cannot be.)
  __device__ __forceinline__ bool wait_pv(int t) const {
    return wait_warp(&sh.pv_done[t % kRing], (t / kRing) & 1, budget);
  }

  // Every tile of the copy; false when a bounded wait gave up.
  // HALVES: the two threads of a lane do not know of each other: their key halves have
  // maxima, sums and an O each, and P is written over the half's S.
  __device__ __forceinline__ bool run() {
    constexpr bool HALVES = Copies<D, REP>::kHalves;
    using G = Geom<D>;
    const int quarter = warp_index() & 3, lane = threadIdx.x & 31;
    bool bad = false;
    int e = 0;
    R = m = -INFINITY;
    l = 0.f;
    if (copy >= cp.rep()) return true;   // lanes of no copy
    for (int t = copy; t < it.ntiles; t += cp.rep(), e ^= 1) {
      const bool tree = t >= it.nctx;
      const int valid = tree ? it.n : min(kKeys, it.ctx - t * kKeys);
      const TileScales& sc = sh.sc[t % kScaleSlots];
      const bool here = !bad && wait_warp(&sh.s_full[t % kRing], (t / kRing) & 1, budget);
      float x[kCols], mt = -INFINITY, u[kCols / kGroup], top = -INFINITY;
      if (here) {
        if (busy) {
          tc_fence_after();
          tmem_ld64(lane_base + cp.s_col(t) + kCols * cq, x);
          tc_fence_before();
        }
        if (!HALVES) {
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&sh.s_empty[copy]));
        }
        if (busy) {
          if (tree || valid < kKeys) mask(x, tree, valid);
          mt = maximum(x, sc, tree, u);
          top = fmaxf(u[0], u[1]);
          if (!HALVES) sh.mx[e][cq][row] = top;
        }
      }
      if (HALVES) {
        if (!here) return false;
      } else {
        // the quarter's warps decide together whether to go on, and the maxima become visible
        if (!quarter_all(quarter, here)) return false;
        top = fmaxf(sh.mx[e][0][row], sh.mx[e][1][row]);
      }
      // P's columns are free (HALVES: S of tile t came behind the P.V before)
      if (!HALVES && t >= cp.p_bufs() && !wait_pv(t - cp.p_bufs())) bad = true;
      if (busy) {
        // (the tree's weights are not scaled: none above 2)
        const bool had = R != -INFINITY;
        bool need = had ? top > R + (tree ? 0.f : kSlack) : top != -INFINITY;
        const bool rescale = t >= cp.rep() && __any_sync(0xffffffffu, need && had);
        // where one of the warp's rows moves its reference all do: the next that has to is
        // then many tiles away (the tree's tile, the last, keeps rows apart)
        if (rescale && !tree) need = need || top > R;
        const float alpha = need && had ? exp2f(R - top) : 1.f;
        if (need) R = top;
        const uint32_t p_at = lane_base + cp.p_col(t, copy) +
                              cq * (HALVES ? kCols : tree ? kCols / 2 : kCols / 4);
        weights(x, mt, u, p_at, HALVES ? kCols / 4 : kCols / 2, sc, sh.sfa[t % kRing], tree);
        if (rescale) {
          // O holds earlier tiles: rescale this thread's half of the row's columns, or its own
          // O.  (The other copies' P.V adds 0 to them, so it has to be done too.)  P.V of the
          // tile before has had the weights' time to finish.
          if (!wait_pv(t - 1)) {
            bad = true;
          } else {
            tc_fence_after();
#pragma unroll 1
            for (int cc = 0; cc < (HALVES ? D : D / kSplit) / 32; ++cc) {
              float o[32];
              const uint32_t oc = lane_base + cq * (HALVES ? D : D / kSplit) + 32 * cc;
              tmem_ld32(oc, o);
              uint32_t f[32];
#pragma unroll
              for (int i = 0; i < 32; ++i) f[i] = __float_as_uint(o[i] * alpha);
              tmem_st16u(oc, reinterpret_cast<const uint32_t(&)[16]>(f[0]));
              tmem_st16u(oc + 16, reinterpret_cast<const uint32_t(&)[16]>(f[16]));
            }
          }
        }
      }
      if (!tree && valid < kKeys) {
        // the context's last tile: V rows past the last valid key may hold anything; zero them
        // so that 0 * V stays 0, once the V tile has landed.  (Its slot was that of tile
        // t - 4, consumed: P.V of tile t - 4 is done.)
        if (!bad && wait_warp(&sh.v_full[t % kStages], (t / kStages) & 1, budget)) {
          // thread among those of the copy
          const int per = 1 << cp.quarters_log(), tid = (cq * per + (quarter & (per - 1))) * 32 + lane;
          const int of = kSplit * 32 * per;
          uint8_t* vt = gbase + G::kVOff + t % kStages * G::kTile;
          constexpr int kChunks = D / 16;
          for (int i = tid; i < (kKeys - valid) * kChunks; i += of)
            *reinterpret_cast<uint4*>(vt + valid * D + i * 16) = make_uint4(0u, 0u, 0u, 0u);
          fence_proxy_async();  // the zeroed rows are read by the tensor cores
        } else {
          bad = true;
        }
      }
      tmem_wait_st();   // P is in place
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&sh.p_full[t % kRing]));
    }
    return !bad;
  }
};

// The tree's V tile in shared memory: rows past the last node as 0, and of the nodes' rows
// what is not finite, since 0 * V has to stay 0: it belongs only to the rows that have the
// node as an ancestor, and the output adds it there.  Thread `tid` of 64; true if it met any.
template <int D>
__device__ __forceinline__ bool clean_tree_v(uint8_t* vt, int n, int tid) {
  constexpr int kChunks = D / 8;
  static_assert(64 % kChunks == 0, "a thread keeps to one chunk of the rows");
  const int rem = tid % kChunks;
  uint8_t* col = vt + (rem >> 3) * (kKeys * 128) + (rem & 7) * 16;
  bool odd = false;
#pragma unroll 8
  for (int r = tid / kChunks; r < n; r += 64 / kChunks) {
    const uint4 v = *reinterpret_cast<const uint4*>(col + r * 128), f = only_finite(v);
    if (f.x != v.x || f.y != v.y || f.z != v.z || f.w != v.w) {
      odd = true;
      *reinterpret_cast<uint4*>(col + r * 128) = f;
    }
  }
  for (int r = n + tid / kChunks; r < kKeys; r += 64 / kChunks)
    *reinterpret_cast<uint4*>(col + r * 128) = make_uint4(0u, 0u, 0u, 0u);
  return odd;
}

// Adds to 8 columns of row q the values of its ancestors' V rows that are not finite: any
// positive weight leaves an infinity or a NaN what it is.
__device__ __forceinline__ void add_odd(const AttnParams& p, const Item& it, const Shared& sh, int q, int c,
                                     float (&o)[8]) {
  const uint64_t* anc = sh.anc[(it.r0 + q) / p.G];
#pragma unroll 1
  for (int u = 0; u < it.n; ++u) {
    if (!((anc[u >> 6] >> (u & 63)) & 1u)) continue;
    const uint4 v = *reinterpret_cast<const uint4*>(
        static_cast<const __nv_bfloat16*>(p.tree_v) +
        (static_cast<size_t>(it.s0 + u) * p.Hkv + it.g) * p.D + c);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 f = bf16x2_f32(w[k]);
      if (!finite(f.x)) o[2 * k] += f.x;
      if (!finite(f.y)) o[2 * k + 1] += f.y;
    }
  }
}

// Softmax warps: warp w handles TMEM lane quarter w % 4 and key half cq = (w - 4) / 4 of its
// copy's tiles, two threads per TMEM lane.
template <int D, int BLK, int REP>
__device__ __forceinline__ bool softmax_role8(const Attn8Params& p8, const Item& it, Shared& sh,
                                              const Copies<D, REP> cp, uint32_t tmem, uint8_t* gbase,
                                              long long budget) {
  using G = Geom<D>;
  const int rep = cp.rep();
  const AttnParams& p = p8.a;
  const int warp = warp_index(), lane = threadIdx.x & 31;
  const int cq = (warp - kSoftmaxWarp) >> 2;
  const int row = (warp & 3) * 32 + lane;      // = TMEM lane
  const int tid = threadIdx.x - 32 * kSoftmaxWarp;
  const uint32_t lane_base = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
  const int span = cp.span();                  // rows of a copy
  const int r = row & (span - 1), copy = row >> (5 + cp.quarters_log());
  const bool mine = r < it.nrows;
  const bool busy = (((warp & 3) * 32) & (span - 1)) < it.nrows;

  // This half of the row's query: a bf16 copy, and two 8-bit terms under the row's scale.
  float c_row = p.scale_log2;
  {
    const uint4* qg = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.q) +
                                                     (mine ? grow_of(p, it, r) : 0) * D);
    uint4 v[D / 8 / kSplit];
    float m = 0.f;
#pragma unroll
    for (int k = 0; k < D / 8 / kSplit; ++k)
      v[k] = mine ? qg[cq * (D / 8 / kSplit) + k] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int k = 0; k < D / 8 / kSplit; ++k) {
      const uint32_t w[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 x = bf16x2_f32(w[i]);
        m = fmaxf(m, fmaxf(fabsf(x.x), fabsf(x.y)));
      }
    }
    sh.mx[1][cq][row] = m;
    softmax_sync();
    m = fmaxf(sh.mx[1][0][row], sh.mx[1][1][row]);
    const int e = min(block_exponent(m), 120);
    const float inv = pow2(-e);
    // (an infinity, which e4m3 does not hold, makes the row's scores NaN; a NaN stays one)
    c_row = finite(m) ? c_row * pow2(e) : __uint_as_float(0x7fffffffu);
#pragma unroll
    for (int k = 0; k < D / 8 / kSplit; ++k) {
      const int c = cq * (D / 8 / kSplit) + k;
      *reinterpret_cast<uint4*>(gbase + G::kQbOff + (c >> 3) * (kRows * 128) + row * 128 +
                                (((c & 7) ^ (row & 7)) << 4)) = v[k];
    }
#pragma unroll
    for (int k = 0; k < D / 8 / kSplit; k += 2) {
      uint32_t hi[4], lo[4];
      const uint32_t w[8] = {v[k].x,     v[k].y,     v[k].z,     v[k].w,
                             v[k + 1].x, v[k + 1].y, v[k + 1].z, v[k + 1].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 x = bf16x2_f32(w[2 * i]), y = bf16x2_f32(w[2 * i + 1]);
        const float q[4] = {x.x * inv, x.y * inv, y.x * inv, y.y * inv};
        two_terms_wide(q, hi[i], lo[i]);
      }
      const int at = swz8<D>(row, (cq * (D / 8 / kSplit) + k) / 2);
      *reinterpret_cast<uint4*>(gbase + at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
      *reinterpret_cast<uint4*>(gbase + G::kQ8 + at) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    }
    fence_proxy_async();   // the tensor cores read these rows
    // P of the other copies' tiles is 0 in this one's lanes
    uint32_t z[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = 0u;
    for (int k = 0; rep > 1 && k < rep; ++k)
      if (k != copy)
        for (int c = 0; c < 64 / kSplit; c += 16)
          tmem_st16u(lane_base + cp.p_col(k, k) + (64 / kSplit) * cq + c, z);
    tmem_wait_st();
    tc_fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&sh.q_ready));
  }

  // (only the chunk with the tree tile has a use for the masks)
  uint64_t anc = 0;
  if (it.ntree > 0) {
    tree_masks<kSoftmax8>(p, it, tid, sh.par, sh.anc);
    if (mine) anc = sh.anc[(it.r0 + r) / p.G][cq];
  }
  Softmax<D, BLK, REP> sm{p8, it, sh, cp, gbase, lane_base, cq, row, copy, busy, c_row, anc, budget, 0.f, 0.f, 0.f};
  bool ok = sm.run();
  // O is complete once every P.V is done
  if (ok) {
    ok = wait_warp(&sh.mma_done[1], 0, budget) && !aborted_warp(&sh.abort) &&
         (it.ntree == 0 || wait_warp(&sh.tree_clean, 0, budget));   // (for odd_v)
    if (ok) tc_fence_after();
  }
  if (softmax_any<kSoftmax8>(!ok)) {
    if (tid == 0) {
      note_timeout(p.status);
      *const_cast<volatile int*>(&sh.abort) = 1;
    }
    return false;
  }
  sh.l[cq][row] = sm.l;
  sh.mx[0][cq][row] = sm.m;
  sh.mx[1][cq][row] = sm.R;   // (of the copies' two threads the same)
  softmax_sync<kSoftmax8>();
  // O of every copy -> shared memory [128][D + 4] (the tiles are free), all in units of the
  // row's largest 2^R
  float R = -INFINITY, M = -INFINITY;
  for (int k = 0; k < rep; ++k)
#pragma unroll
    for (int h = 0; h < kSplit; ++h) {
      M = fmaxf(M, sh.mx[0][h][k * span + r]);
      R = fmaxf(R, sh.mx[1][h][k * span + r]);
    }
  auto weight = [&](float x) { return x == -INFINITY ? 0.f : exp2f(x - R); };
  const float w = weight(cp.kHalves ? sh.mx[1][0][row] : sm.R), w1 = weight(sh.mx[1][1][row]);
  float* stage = reinterpret_cast<float*>(gbase) + row * (D + 4) + cq * (D / kSplit);
#pragma unroll
  for (int cc = 0; cc < D / kSplit / 16; ++cc) {
    uint32_t o[16];
    tmem_ld16(lane_base + cq * (D / kSplit) + 16 * cc, o);
    float f[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) f[i] = __uint_as_float(o[i]) * w;
    if (cp.kHalves) {
      tmem_ld16(lane_base + D + cq * (D / kSplit) + 16 * cc, o);
#pragma unroll
      for (int i = 0; i < 16; ++i) f[i] = fmaf(__uint_as_float(o[i]), w1, f[i]);
    }
#pragma unroll
    for (int i = 0; i < 16; i += 4)
      *reinterpret_cast<float4*>(stage + 16 * cc + i) = make_float4(f[i], f[i + 1], f[i + 2], f[i + 3]);
  }
  float lt = 0.f;
  const bool first = cq == 0 && copy == 0;
  if (first)
    for (int k = 0; k < rep; ++k) {
      const int at = k * span + r;
#pragma unroll
      for (int h = 0; h < kSplit; ++h) {
        const float mk = sh.mx[0][h][at];
        lt += mk == -INFINITY ? 0.f : sh.l[h][at] * exp2f(mk - M);
      }
    }
  softmax_sync<kSoftmax8>();
  if (first) {
    sh.l[0][r] = lt;
    sh.m[r] = M;
    sh.unit[r] = R == -INFINITY ? 0.f : exp2f(R - M);
  }
  softmax_sync<kSoftmax8>();
  // the copies' sum: the output, or (one of several chunks) the fp32 partial that the
  // merge combines
  const size_t part = static_cast<size_t>(it.part0) +
                      static_cast<size_t>(it.g * it.chunks + it.chunk) * it.R + it.r0;
  if (it.chunks > 1 && tid < it.nrows) p.part_ml[part + tid] = make_float2(sh.m[tid], sh.l[0][tid]);
  constexpr int kPerRow = D / 8;
  for (int i = tid; i < it.nrows * kPerRow; i += kSoftmax8) {
    const int q = i / kPerRow, c = (i % kPerRow) * 8;
    float o[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) o[k] = 0.f;
    for (int k = 0; k < rep; ++k) {
      const float4* src =
          reinterpret_cast<const float4*>(reinterpret_cast<const float*>(gbase) + (k * span + q) * (D + 4) + c);
      const float4 x = src[0], y = src[1];
      o[0] += x.x; o[1] += x.y; o[2] += x.z; o[3] += x.w;
      o[4] += y.x; o[5] += y.y; o[6] += y.z; o[7] += y.w;
    }
    if (sh.odd_v) add_odd(p, it, sh, q, c, o);
    const float unit = sh.unit[q];
    if (it.chunks > 1) {
      float4* dst = reinterpret_cast<float4*>(p.part_o + (part + q) * D + c);
      dst[0] = make_float4(o[0] * unit, o[1] * unit, o[2] * unit, o[3] * unit);
      dst[1] = make_float4(o[4] * unit, o[5] * unit, o[6] * unit, o[7] * unit);
    } else {
      const float lr = sh.l[0][q], inv = lr > 0.f ? unit / lr : 0.f;
      uint32_t h[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        __nv_bfloat162 v = __floats2bfloat162_rn(o[2 * k] * inv, o[2 * k + 1] * inv);
        h[k] = *reinterpret_cast<uint32_t*>(&v);
      }
      *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.out) + grow_of(p, it, q) * D + c) =
          make_uint4(h[0], h[1], h[2], h[3]);
    }
  }
  return true;
}

// Key j of sequence b's context, KV head g, for items_past_grid.
static_assert(kSoftmax8 == kSoftmaxThreads, "the softmax warps take the items past the grid");
template <int D>
struct Context8 {
  const Attn8Params& p8;
  __device__ __forceinline__ bool operator()(int b, int g, int j, int lane, float (&k)[D / 32],
                                             float (&v)[D / 32]) const {
    const AttnParams& p = p8.a;
    size_t at;
    if (!context_row(p, b, g, j, at)) return false;
    // the row's scale block: a page's rows, or a sequence's, are p8.blocks of them
    const int slots = p.page_size ? p.page_size : p.ctx_max;
    const size_t block = at / slots * p8.blocks + at % slots / p8.block;
    load(static_cast<const uint8_t*>(p.k_cache) + at * D, p8.k_exp[block], lane, k);
    load(static_cast<const uint8_t*>(p.v_cache) + at * D, p8.v_exp[block], lane, v);
    return true;
  }
  __device__ __forceinline__ static void load(const uint8_t* row, int byte, int lane, float (&x)[D / 32]) {
    const float f = pow2(min(max(byte - kExpBias, kMinExp), 126));
#pragma unroll
    for (int k = 0; k < D / 32; k += 2) {
      const float2 y = e4m3x2_f32(*reinterpret_cast<const uint16_t*>(row + lane * (D / 32) + k));
      x[k] = y.x * f;
      x[k + 1] = y.y * f;
    }
  }
};

// The item's values by shuffles, which makes them uniform to the compiler: with the warp's index
// alike, loops and branches on them need no reconvergence and what they steer stays in uniform
// registers (32 adaptive trees 78 -> 69 us, 8 x 64 nodes at context 16384 167 -> 156).
__device__ __forceinline__ void uniform(Item& it) {
  int* const v[] = {&it.b, &it.g, &it.s0, &it.n, &it.r0, &it.nrows, &it.R, &it.key_base, &it.ctx, &it.nctx,
                    &it.ntree, &it.ntiles, &it.chunks, &it.chunk, &it.part0};
#pragma unroll
  for (int k = 0; k < 15; ++k) *v[k] = __shfl_sync(0xffffffffu, *v[k], 0);
}

template <int D, int BLK, int REP>
__global__ void __launch_bounds__(kThreads8, 1)
    attn_kv8_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                    const __grid_constant__ CUtensorMap tm_tk, const __grid_constant__ CUtensorMap tm_tv,
                    const Attn8Params p8) {
  using G = Geom<D>;
  const AttnParams& p = p8.a;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(16) Shared sh;
  __shared__ PlanSmem s_plan;

  pdl_launch_dependents();
  const int warp = warp_index(), lane = threadIdx.x & 31;
  const long long budget = wait_budget(p.wait_cycles);
  volatile int* s_abort = &sh.abort;

  uint32_t base = smem_u32(smem_raw);
  const uint32_t pad = (1024u - (base & 1023u)) & 1023u;
  uint8_t* gbase = smem_raw + pad;
  base += pad;

  if (threadIdx.x == 32 * 3) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(smem_u32(&sh.k_full[s]), 2);   // the copy and its scales
      mbar_init(smem_u32(&sh.k_empty[s]), 1);
      mbar_init(smem_u32(&sh.v_full[s]), 1);
      mbar_init(smem_u32(&sh.v_empty[s]), 1);
      sh.issued[0][s] = sh.issued[1][s] = 0;
    }
    for (int b = 0; b < kRing; ++b) {
      mbar_init(smem_u32(&sh.s_full[b]), 1);
      mbar_init(smem_u32(&sh.pv_done[b]), 1);
    }
    mbar_init(smem_u32(&sh.q_ready), kSoftmax8 / 32);
    mbar_init(smem_u32(&sh.mma_done[0]), 1);
    mbar_init(smem_u32(&sh.mma_done[1]), 1);
    sh.abort = sh.tree_issued = sh.odd_v = 0;
    mbar_init(smem_u32(&sh.ctx_done), 1);
    mbar_init(smem_u32(&sh.tree_k), 1);
    mbar_init(smem_u32(&sh.tree_v), 1);
    mbar_init(smem_u32(&sh.tree_clean), 2);   // either producer's half
    fence_mbar_init();
  }
  if (warp == 2) {
    tmem_alloc(smem_u32(&sh.tmem), kTmemCols);
    tmem_relinquish();
    tc_fence_before();
  }
  Item it;
  const bool some = make_item<kRows, kPlain, kThreads8 / 32>(p, it, s_plan);   // uniform over the CTA
  tc_fence_after();
  if (!some) {   // no query rows here
    if (warp == 2) tmem_dealloc(sh.tmem, kTmemCols);
    pdl_wait();
    return;
  }
  uniform(it);
  const uint32_t tmem = __shfl_sync(0xffffffffu, sh.tmem, 0);
  const Copies<D, REP> cp(it.nrows);
  if (threadIdx.x == 32 * 3) {   // the copies' own arrivals
    for (int b = 0; b < kRing; ++b) mbar_init(smem_u32(&sh.p_full[b]), cp.warps());
    for (int b = 0; b < 4; ++b) mbar_init(smem_u32(&sh.s_empty[b]), cp.warps());
    fence_mbar_init();
  }
  // scale bytes of 2^0 (of rows without keys, whose P is 0 or of no use, no NaN)
  static_assert(sizeof(sh.sfa) == kRing * sizeof(sh.sfb), "");
  for (int i = threadIdx.x; i < (kRing + 1) * kRows; i += kThreads8)
    (i < kRows ? sh.sfb[i] : sh.sfa[i / kRows - 1][i % kRows]) = 0x01010101u * kExpBias;
  fence_proxy_async();   // the tensor core's copy reads them
  __syncthreads();
  bool ok = true;

  if (warp == 0 || warp == 3) {
    // ------------------------------------------- producers of every second tile
    const int odd = warp == 0 ? 0 : 1;
    if (lane == 0) {
      prefetch_tmap(&tm_k);
      prefetch_tmap(&tm_v);
      prefetch_tmap(&tm_tk);
      prefetch_tmap(&tm_tv);
    }
    const uint64_t pol = l2_policy_evict_first();
    Pages pages(p, it, sh.pages[odd]);
    Scales scales(p8, it, pages);
    // K (which = 0) or V of context tile t, once its slot is free
    auto copy = [&](int which, int t, int row) {
      uint64_t* full = which ? sh.v_full : sh.k_full;
      uint64_t* empty = which ? sh.v_empty : sh.k_empty;
      const int stage = t % kStages;
      ok = wait_warp(&empty[stage], ((t / kStages) & 1) ^ 1u, budget);
      if (!ok) return;
      issue_tile<D>(row, pages.br, base + (which ? G::kVOff : G::kKOff) + stage * G::kTile,
                    smem_u32(&full[stage]), which ? &tm_v : &tm_k, pol, lane);
      if (lane == 0) ++sh.issued[which][stage];
    };
    auto factors = [&](int t, int e) {
      scales.write(e, sh.sc[t % kScaleSlots]);
      if (lane == 0) mbar_arrive(smem_u32(&sh.k_full[t % kStages]));
    };
    // the scales of the first two tiles are on their way first (a small loop: code that runs
    // once costs its fetch; 8 nodes at context 32k 27.8 -> 26.3 us)
    const int e0 = scales.fetch(odd), e1 = scales.fetch(odd + 2);
    int nk = odd, nv;   // next tile of K, of V
#pragma unroll 1
    for (int e = e0; nk < min(it.nctx, kStages); nk += 2, e = e1) {
      const int row = pages.row(nk, lane);
      copy(0, nk, row);
      copy(1, nk, row);
      factors(nk, e);
    }
    nv = nk;
    int next = scales.fetch(nk);   // scale bytes of the next tile, fetched a tile ahead
    int last = -1;         // cache row of K's last tile
    while (nv < it.nctx) {
      int row = last;
      if (nk < it.nctx) {
        row = pages.row(nk, lane);
        copy(0, nk, row);
        if (!ok) break;
        factors(nk, next);
        nk += 2;
        next = scales.fetch(nk);
      }
      // V a tile behind K: K's slots are free as soon as S is done
      if (nv + 2 < nk || nk >= it.nctx) {
        copy(1, nv, nv + 2 < nk ? last : row);
        if (!ok) break;
        nv += 2;
      }
      last = row;
    }
    if (ok && it.ntree > 0 && (it.nctx & 1) == odd) {   // nk is the tree's tile
      ok = it.nctx == 0 || wait_warp(&sh.ctx_done, 0, budget);
      if (ok && lane == 0) {
        mbar_expect_tx(smem_u32(&sh.tree_k), G::kTreeTile);
        mbar_expect_tx(smem_u32(&sh.tree_v), G::kTreeTile);
#pragma unroll
        for (int h = 0; h < D / 64; ++h) {
          tma_load_3d(base + G::kKOff + h * (kKeys * 128), &tm_tk, smem_u32(&sh.tree_k), h * 64, it.g,
                      it.s0, pol);
          tma_load_3d(base + G::kTreeVOff + h * (kKeys * 128), &tm_tv, smem_u32(&sh.tree_v), h * 64,
                      it.g, it.s0, pol);
        }
        sh.tree_issued = 1;
      }
    }
    if (ok && it.ntree > 0) {
      ok = wait_warp(&sh.tree_v, 0, budget);
      if (ok) {
        if (clean_tree_v<D>(gbase + G::kTreeVOff, it.n, odd * 32 + lane)) sh.odd_v = 1;
        fence_proxy_async();   // the tensor cores read the tile
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sh.tree_clean));
      }
    }
    if (!ok && lane == 0) {
      note_timeout(p.status);
      *s_abort = 1;
    }
    __syncwarp();
  } else if (warp == 1 || warp == 2) {
    // ------------------------------------------------------------ MMA issuers
    const uint32_t on = lane == 0 ? 1u : 0u;
    const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
    if (warp == 1) {
      const uint32_t idesc_s[2] = {idesc_f8(kRows, kKeys, false), idesc_f8(kRows, kKeys, true)};
      const uint32_t idesc_t = idesc_bf16(kRows, kKeys);
      ok = wait_warp(&sh.q_ready, 0, budget);
      tc_fence_after();
      int copy = 0;          // of tile t, and the parity of its tiles before
      uint32_t use = 0;
      for (int t = 0; ok && t < it.ntiles; ++t) {
        const bool tree = t >= it.nctx;
        const int stage = tree ? 0 : t % kStages, b = t % kRing;
        ok = (tree ? wait_warp(&sh.tree_k, 0, budget)
                   : wait_warp(&sh.k_full[stage], (t / kStages) & 1, budget)) &&
             (cp.kHalves ? t < cp.kOverBufs || wait_warp(&sh.pv_done[(t - cp.kOverBufs) % kRing],
                                                         ((t - cp.kOverBufs) / kRing) & 1, budget)
                         : wait_warp(&sh.s_empty[copy], use ^ 1u, budget));
        if (!ok) break;
        tc_fence_after();
        const uint32_t kst = base + G::kKOff + stage * G::kTile, sb = tm + cp.s_col(t);
        // the copy's lanes only
        uint32_t skip[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) skip[k] = k >> cp.quarters_log() == copy ? 0u : 0xffffffffu;
        if (!tree) {
#pragma unroll
          for (int term = 0; term < 2; ++term)
#pragma unroll
            for (int ks = 0; ks < D / 32; ++ks) {
              const uint64_t a = desc8<D>(base + term * G::kQ8 + 32 * ks), k = desc8<D>(kst + 32 * ks);
              if (cp.kHalves) mma_f8(sb, a, k, idesc_s[term], term + ks > 0 ? 1u : 0u, on);
              else mma_f8_lanes(sb, a, k, idesc_s[term], skip, term + ks > 0 ? 1u : 0u, on);
            }
        } else {
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks) {
            const int h = ks >> 2, kk = ks & 3;
            const uint64_t a = sw128_desc(base + G::kQbOff + h * (kRows * 128) + 32 * kk),
                           k = sw128_desc(kst + h * (kKeys * 128) + 32 * kk);
            if (cp.kHalves) mma_bf16(sb, a, k, idesc_t, ks > 0 ? 1u : 0u, on);
            else mma_bf16_lanes(sb, a, k, idesc_t, skip, ks > 0 ? 1u : 0u, on);
          }
        }
        if (++copy == cp.rep()) {
          copy = 0;
          use ^= 1u;
        }
        tc_commit_on(smem_u32(&sh.s_full[b]), on);
        tc_commit_on(smem_u32(t == it.nctx - 1 ? &sh.ctx_done : &sh.k_empty[stage]), on);
      }
    } else {
      ok = wait_warp(&sh.q_ready, 0, budget);   // P is 0 where the copies do not write it
      tc_fence_after();
      const uint32_t idesc_o = idesc_mx8(kRows, D, true), idesc_t = idesc_bf16(kRows, D, true);
      if (!cp.kHalves) tc_copy_scales(tm + cp.sfb_col(0), smem_u32(sh.sfb), on);
      int copy = 0;   // of tile j
      for (int j = 0; ok && j < it.ntiles; ++j, copy = copy + 1 == cp.rep() ? 0 : copy + 1) {
        const bool tree = j >= it.nctx;
        const int stage = j % kStages, b = j % kRing;
        ok = wait_warp(&sh.p_full[b], (j / kRing) & 1, budget) &&
             (tree ? wait_warp(&sh.tree_clean, 0, budget)
                   : wait_warp(&sh.v_full[stage], (j / kStages) & 1, budget));
        // MMAs of another kind follow on O: the earlier ones are done first
        if (ok && tree && j > 0)
          ok = wait_warp(&sh.pv_done[(j - 1) % kRing], ((j - 1) / kRing) & 1, budget);
        if (!ok) break;
        tc_fence_after();
        const uint32_t vst = base + (tree ? G::kTreeVOff : G::kVOff + stage * G::kTile);
        // P's columns of MMA step kk: in a row, or behind the start of either key half's S
        const uint32_t pb = tm + cp.p_col(j, copy);
        const uint32_t half = cp.kHalves ? 1u : 0u, o1 = half * D;
        const uint32_t lo = half ? kCols / 4 : kCols / 2;
        if (!tree) {
          const uint32_t skip = half * (kCols - kCols / 4);
          const uint32_t sfa = tm + cp.sfa_col(j, copy), sfb = tm + cp.sfb_col(j);
          tc_copy_scales(sfa, smem_u32(sh.sfa[b]), on);
          if (half) tc_copy_scales(sfb, smem_u32(sh.sfb), on);
#pragma unroll
          for (int term = 0; term < 2; ++term)
#pragma unroll
            for (int kk = 0; kk < kKeys / kGroup; ++kk) {
              const uint32_t h = kk / 2;
              mma_mx8_ts(tm + h * o1, pb + lo * term + 8 * kk + h * skip, desc8<D>(vst + kk * kGroup * D),
                         idesc_o | sf_byte_a(kk), sfa, sfb,
                         (j > 0 || term > 0 || kk > (kk == 2 && half ? 2 : 0)) ? 1u : 0u, on);
            }
        } else {
          const uint32_t skip = half * (kCols - kCols / 2);
#pragma unroll
          for (int kk = 0; kk < kKeys / 16; ++kk) {
            const uint32_t h = kk / 4;
            mma_bf16_ts(tm + h * o1, pb + kk * 8 + h * skip, sw128_desc_mn(vst + kk * 2048, kKeys * 128, 1024),
                        idesc_t, (j > 0 || kk > (kk == 4 && half ? 4 : 0)) ? 1u : 0u, on);
          }
        }
        tc_commit_on(smem_u32(&sh.pv_done[b]), on);
        if (!tree) tc_commit_on(smem_u32(&sh.v_empty[stage]), on);
      }
    }
    if (!ok && lane == 0) {
      note_timeout(p.status);
      *s_abort = 1;
    }
    __syncwarp();
    // every MMA this warp issued has finished before TMEM or the buffers are reused
    if (lane == 0) {
      uint64_t* done = &sh.mma_done[warp == 1 ? 0 : 1];
      tc_commit(smem_u32(done));
      mbar_wait(smem_u32(done), 0);
    }
    __syncwarp();
  } else {
    softmax_role8<D, BLK, REP>(p8, it, sh, cp, tmem, gbase, budget);
  }
  tc_fence_before();
  __syncthreads();   // the tensor cores are idle from here on
  tc_fence_after();
  // A CTA that gave up may have left copies in flight (otherwise every tile was consumed):
  // they land before it leaves.
  if (sh.abort && threadIdx.x == 0) {
    if (sh.tree_issued) {
      mbar_wait(smem_u32(&sh.tree_k), 0);
      mbar_wait(smem_u32(&sh.tree_v), 0);
    }
    for (int st = 0; st < kStages; ++st) {
      if (sh.issued[0][st] > 0)
        mbar_wait(smem_u32(&sh.k_full[st]), static_cast<uint32_t>((sh.issued[0][st] - 1) & 1));
      if (sh.issued[1][st] > 0)
        mbar_wait(smem_u32(&sh.v_full[st]), static_cast<uint32_t>((sh.issued[1][st] - 1) & 1));
    }
  }
  if (warp == 2) tmem_dealloc(tmem, kTmemCols);
  if (s_plan.past > 0 && warp >= kSoftmaxWarp)
    items_past_grid<D>(p, s_plan, threadIdx.x - 32 * kSoftmaxWarp, Context8<D>{p8});
  pdl_wait();   // the next kernel's wait covers every earlier kernel
}

using Kernel = void(const CUtensorMap, const CUtensorMap, const CUtensorMap, const CUtensorMap,
                    const Attn8Params);

// By the largest sequence's rows of a KV head (the items' then are no more): at most 32 fit three
// or four copies, at most 64 two.  8 sequences at context 16384, four heads to a KV head, one / 8 /
// 16 nodes: three copies 60 / 63 / - us, two 67 / 69 / 71, one - / - / 83.  Where sequences have
// few rows on average beside a larger one, the items' own number: 32 of 2 to 24 nodes at contexts
// 1000 to 8000 70 (one copy 82), 64 of 1 and 17 at 2000 84 (98).  (It costs a call whose time
// the large ones set: 64 nodes beside 15 trees of 4 at 4000 58 (53).)  Otherwise one copy, an O
// for each key half, whatever an item's rows: 16 trees of 16 to 96 nodes of 64 columns 51 (60),
// 8 x 64 nodes at 16384, pages of 16, 152 (173).
template <int D, int BLK>
Kernel* kernel_of_rows(int most, double mean) {
  return most <= 32   ? attn_kv8_kernel<D, BLK, kManyCopies>
         : most <= 64 ? attn_kv8_kernel<D, BLK, 2>
         : mean <= 64 ? attn_kv8_kernel<D, BLK, 0>
                      : attn_kv8_kernel<D, BLK, 1>;
}
template <int D>
Kernel* kernel_of(const Attn8Params& p8) {
  const AttnParams& p = p8.a;
  const int most = p.max_nodes * p.G;
  const double mean = static_cast<double>(p.T) * p.G / p.B;
  return p8.block == 32   ? kernel_of_rows<D, 32>(most, mean)
         : p8.block == 16 ? kernel_of_rows<D, 16>(most, mean)
                          : kernel_of_rows<D, 8>(most, mean);
}

}  // namespace

cudaError_t launch_attention_kv8(const Attn8Params& p8, const CUtensorMap& tm_k,
                                 const CUtensorMap& tm_v, const CUtensorMap& tm_tk,
                                 const CUtensorMap& tm_tv, cudaStream_t s) {
  const AttnParams& p = p8.a;
  if (p.D != 64 && p.D != 128) return cudaErrorInvalidValue;
  const size_t smem = 1024 + static_cast<size_t>(p.D == 64 ? Geom<64>::kBytes : Geom<128>::kBytes);
  // row blocks: at most max_nodes * G rows of each of B sequences (index order, B >
  // kOrderMax, numbers these), and T * G rows of which every sequence may leave one block
  // ragged
  const long long full = static_cast<long long>((p.max_nodes * p.G + kRows - 1) / kRows) * p.B;
  const long long blocks =
      p.B > kOrderMax ? full : std::min(full, static_cast<long long>(p.T) * p.G / kRows + p.B);
  const long long ctas = std::max<long long>(blocks * p.Hkv, p.part_cap > 0 ? p.nsm : 0);
  if (ctas > 0x7fffffffLL) return cudaErrorInvalidValue;
  auto* k = p.D == 64 ? kernel_of<64>(p8) : kernel_of<128>(p8);
  cudaError_t err = set_smem_attrs(k, smem);
  if (err != cudaSuccess) return err;
  err = launch_pdl(k, dim3(static_cast<unsigned>(ctas)), dim3(kThreads8), smem, s, tm_k, tm_v, tm_tk,
                   tm_tv, p8);
  return err != cudaSuccess || p.part_cap == 0 ? err : launch_attention_merge(p, s);
}

}  // namespace asd
