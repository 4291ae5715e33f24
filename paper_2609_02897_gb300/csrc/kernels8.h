// Internal interface between the C-ABI layer of the 8-bit calls (asd8_api.cu) and
// their kernels.
#pragma once

#include "asd8.h"
#include "kernels.h"

namespace asd {

// ------------------------------------------------- K/V: conversion and commit
struct Kv8Params {
  const void* k_src;          // quantize: bf16 cache; compact: tree K [T, Hkv, D]
  const void* v_src;
  uint8_t* k;
  uint8_t* v;
  uint8_t* k_exp;
  uint8_t* v_exp;
  const int32_t* page_table;
  const int32_t* ctx_len;
  const int32_t* cu_nodes;    // compact
  const int32_t* path;        // [B, max_path]
  const int32_t* path_len;
  int32_t* ctx_len_out;
  int* status;
  int in_step;                // compact: behind a step's tail, whose call's status word it adds to
  int clear_status;           // set by the launch: the grid is one cluster, whose first CTA
                              // clears the status word
  int B, T, Hkv, D, ctx_max, page_size, pages_per_seq, num_pages, block, max_nodes, max_path;
  int blocks;                 // scale blocks per sequence (contiguous) or page
};
cudaError_t launch_kv8_quantize(const Kv8Params& p, int nsm, cudaStream_t s);
cudaError_t launch_kv8_compact(const Kv8Params& p, cudaStream_t s);

// ------------------------------------------------------------------ attention
struct Attn8Params {
  AttnParams a;               // k_cache, v_cache: e4m3
  const uint8_t* k_exp;
  const uint8_t* v_exp;
  int block;                  // tokens per scale
  int blocks;                 // scale blocks per sequence (contiguous) or page
};
// tm_k / tm_v: 2D maps over the cache rows of D bytes with boxes of min(kAttnTcKeys, rows
// per page) rows; tm_tk / tm_tv as in launch_attention_tc.
cudaError_t launch_attention_kv8(const Attn8Params& p, const CUtensorMap& tm_k,
                                 const CUtensorMap& tm_v, const CUtensorMap& tm_tk,
                                 const CUtensorMap& tm_tv, cudaStream_t s);

// -------------------------------------------------------------------- LM head
// Packed 8-bit weight: a header of kLm8Header bytes, the scale bytes as words of four
// k-blocks [ceil(nkb / 4)][ceil(V / 128)] rounded up to 256 bytes, then for every tile of up to kLm8Groups
// 32-row groups in range order and every k-block kb of 128 columns, the tile's rows
// (whole groups, zeros past V and past K) x 128 bytes with the 128-byte swizzle
// applied (16-byte chunk c of row r at chunk c ^ (r & 7)).  The block of the tile
// starting at group g0 (ng groups) for k-block kb begins 4096 * (nkb * g0 + kb * ng)
// bytes into the tiles, so that an SM's whole range is one stream.
constexpr uint32_t kLm8Magic = 0x38445341u;   // "ASD8"
constexpr uint32_t kLm8Version = 1;
constexpr int kLm8Header = 256;
constexpr int kLm8KB = ASD8_LM_BLOCK;         // columns of a k-block = bytes of a row
constexpr int kLm8Groups = 7;                 // 32-row groups of a tile: 224 rows
constexpr int kLm8TileN = kLm8Groups * kLmBoxRows;
constexpr int kLm8GroupBytes = kLmBoxRows * kLm8KB;
__host__ __device__ inline int lm8_kblocks(int hidden) { return (hidden + kLm8KB - 1) / kLm8KB; }
__host__ __device__ inline size_t lm8_tiles_at(int vocab, int hidden) {
  const size_t n = static_cast<size_t>((vocab + 127) / 128) * ((lm8_kblocks(hidden) + 3) / 4) * 4;
  return kLm8Header + (n + 255) / 256 * 256;
}
inline size_t lm8_bytes(int vocab, int hidden) {
  return lm8_tiles_at(vocab, hidden) + static_cast<size_t>((vocab + kLmBoxRows - 1) / kLmBoxRows) *
                                           lm8_kblocks(hidden) * kLm8GroupBytes;
}
cudaError_t launch_lm8_pack(const void* w, void* w_packed, int vocab, int hidden, int ranges,
                            cudaStream_t s);

struct Lm8Params {
  LmParams lm;                // w_packed: the 8-bit weight; hidden: bf16
  uint8_t* h8;                // [T][nkb * 128] e4m3 hidden states
  uint8_t* h_exp;             // their scale bytes, words of four k-blocks [ceil(nkb / 4)][t_pad]
  int t_pad;                  // T rounded up to 128
};
// Quantises the hidden states (h8, h_exp).
cudaError_t launch_lm8_hidden(const Lm8Params& p, cudaStream_t s);
cudaError_t launch_lmhead_fp8(const Lm8Params& p, const CUtensorMap& tm_h, cudaStream_t s);

}  // namespace asd
