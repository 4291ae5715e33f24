/*
 * asd8.h - the calls of asd.h with an 8-bit K/V cache and an 8-bit LM head.
 *
 * A decode step that verifies a draft tree reads the whole context cache once per
 * layer and the whole LM-head weight once (Sec. 2 "Verify", Sec. 3.1); both are
 * bound by those bytes, which these calls halve.  Everything said in asd.h about
 * pointers, streams, packing, workspaces, status words and errors holds here; dims
 * must have dtype ASD_BF16 (q, tree K/V, hidden states and attention output stay
 * bf16).
 *
 * The 8-bit format (cache and LM head alike).  The values of a block share one
 * scale 2^e; a value x is held as x / 2^e in e4m3 (1 sign, 4 exponent, 3 mantissa
 * bits, largest 448), rounded to nearest, ties to even.  e is the smallest integer
 * >= -60 with max|x| <= 448 * 2^e over the block's finite values, held as the byte
 * e + 127.  Values that are not finite become NaN.  e4m3 is a floating-point format,
 * so a power of two costs no more precision than any other scale would, dividing by
 * it is exact, a block's bytes can be reproduced bit for bit, and a block can be
 * brought to a larger scale by moving exponents alone.
 */
#ifndef ASD8_H_
#define ASD8_H_

#include "asd.h"

#ifdef __cplusplus
extern "C" {
#endif

#define ASD8_KV_BLOCK 32   /* tokens of a cache block (or the page, if smaller)    */
#define ASD8_LM_BLOCK 128  /* weights: 128 x 128; hidden states: 128 of one node   */
#define ASD8_MIN_EXP (-60)

/* An 8-bit K/V cache (device pointers, caller memory).
 *  k, v          e4m3, laid out as the bf16 cache of the same dims: [B, Hkv,
 *                ctx_max, D], or [P, Hkv, page_size, D] when paged; 16-byte aligned
 *  k_exp, v_exp  scale bytes e + 127, [B, Hkv, ceil(ctx_max / n)] or
 *                [P, Hkv, page_size / n] with n = asd8_kv_block(dims) tokens per
 *                block
 * Only blocks that hold a position below ctx_len are ever read. */
typedef struct asd8_cache {
  void* k;
  void* v;
  uint8_t* k_exp;
  uint8_t* v_exp;
} asd8_cache;

/* Tokens per scale: min(32, page_size), 32 when contiguous; 0 for invalid dims. */
int32_t asd8_kv_block(const asd_dims* dims);

/* Scale bytes of k_exp (and of v_exp); 0 for invalid dims. */
size_t asd8_kv_scales(const asd_dims* dims);

/* Bytes of device workspace that the calls below need: the regions of
 * asd_workspace_bytes, the nodes' hidden states in 8 bits, and partial rows of
 * contexts that are cut over several SMs.  A smaller workspace that holds the first
 * two is taken as well; contexts are then cut less, or not at all. */
size_t asd8_workspace_bytes(const asd_dims* dims, int32_t total_nodes);

/*
 * Converts the context of a bf16 cache (k_cache, v_cache as in asd_tree_attention),
 * as a prefill leaves it: positions 0 .. ctx_len[b] - 1 of every sequence.  A block's
 * scale comes from its positions below ctx_len; slots and blocks at or behind it are
 * left as they were.  Pages shared by sequences are written once for each of them,
 * with the same bytes if the sequences agree on how much of the page they use.
 * A context length outside the cache or a page id outside the pool records
 * ASD_ERR_CTX_RANGE; nothing is written for it.
 */
asd_status asd8_kv_quantize(const asd_dims* dims, const void* k_cache, const void* v_cache,
                            const int32_t* page_table, const int32_t* ctx_len,
                            const asd8_cache* cache, void* workspace, size_t workspace_bytes,
                            void* stream);

/*
 * asd_tree_attention with the context in an 8-bit cache:
 *   K_j = k[j] * 2^e of its block, V_j likewise; tree_k, tree_v, q, out bf16.
 * A NaN or an infinity in tree_k or tree_v reaches only the rows that attend to its node.
 * What is rounded, beside the output: a softmax weight by 2^-8 of it or, in the context, by
 * 2^-16 of the largest product of a weight and a V scale among the 32 positions [32 i, 32 i +
 * 32) it is in, where that is more.  So neither tokens far below the row's largest weight
 * nor blocks of V far below the largest lose what they add.  Components of q below 2^-13
 * of their row's largest are rounded by up to 2^-20 of that one (in the context's scores).
 * With one node per sequence (max_nodes 1, parent -1) it is the attention of a plain
 * decode step.
 */
asd_status asd8_tree_attention(const asd_dims* dims, const void* q, const asd8_cache* cache,
                               const int32_t* page_table, const int32_t* ctx_len,
                               const void* tree_k, const void* tree_v, const int32_t* parent,
                               const int32_t* cu_nodes, int32_t total_nodes, void* out,
                               void* workspace, size_t workspace_bytes, void* stream);

/*
 * asd_kv_compact into an 8-bit cache.  Each block that the path touches takes the
 * larger of its scale (if it holds earlier positions of the sequence) and the one
 * its new rows need; where the scale grows, the block's earlier values are rounded
 * once more, to nearest even (a change only for those that become subnormal).
 * Slots behind the path keep their bytes.  Sequences must not share a block that a
 * path is written to.
 */
asd_status asd8_kv_compact(const asd_dims* dims, const void* tree_k, const void* tree_v,
                           const int32_t* cu_nodes, int32_t total_nodes, const int32_t* path,
                           const int32_t* path_len, const int32_t* ctx_len,
                           const int32_t* page_table, const asd8_cache* cache,
                           int32_t* ctx_len_out, void* workspace, size_t workspace_bytes,
                           void* stream);

/*
 * LM-head weight in 8 bits, in the order the LM head streams it (the counterpart of
 * asd_lm_head_packed_bytes and asd_pack_lm_head, with the same rules: written once
 * at model load, for a device of the same kind and the same vocab and hidden).
 * w [vocab, hidden] bf16 row-major; a scale for each 128 x 128 block of it.
 * dims->lm_head_layout is not looked at.
 */
size_t asd8_lm_head_bytes(const asd_dims* dims);
asd_status asd8_pack_lm_head(const asd_dims* dims, const void* w, void* w_packed,
                             size_t packed_bytes, void* stream);

/*
 * asd_lmhead_margin on 8-bit operands: the weight from asd8_pack_lm_head, and the
 * hidden states quantised inside the call with a scale for each 128 values of a node.
 *   logits[i,v] = sum over blocks kb of 2^(eh[i,kb] + ew[v/128,kb]) *
 *                 sum_k h8[i,k] * w8[v,k]          (products exact, fp32 sums)
 * Rows, verdicts and outputs as in asd_lmhead_margin; a node whose hidden states hold a
 * value that is not finite has no largest logit (row_max -inf, row_argmax 2^31 - 1) and none of
 * its children is accepted.  dims->lm_head_schedule must be
 * ASD_LM_EVERY_ROW (ASD_ERR_SHAPE).
 */
asd_status asd8_lmhead_margin(const asd_dims* dims, const void* hidden, const void* w_packed,
                              const int32_t* tokens, const int32_t* parent,
                              const int32_t* cu_nodes, int32_t total_nodes, float tau,
                              float* row_max, int32_t* row_argmax, float* row_lse,
                              float* l_draft, float* ratio, uint8_t* accept, void* workspace,
                              size_t workspace_bytes, void* stream);

/* Which weight asd8_verify_step is given as step.w_lm. */
typedef enum asd8_weight {
  ASD8_W_BF16 = 0, /* as asd_verify_step takes it (dims->lm_head_layout, schedule)  */
  ASD8_W_E4M3 = 1  /* from asd8_pack_lm_head                                        */
} asd8_weight;

/* asd_verify_step with an 8-bit cache: step.k_cache and step.v_cache must be NULL. */
typedef struct asd8_verify_args {
  asd_verify_args step;
  asd8_cache cache;
  int32_t weight; /* asd8_weight of step.w_lm                                       */
  int32_t reserved; /* must be 0                                                    */
} asd8_verify_args;

asd_status asd8_verify_step(const asd_dims* dims, const asd8_verify_args* args, void* workspace,
                            size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* ASD8_H_ */
