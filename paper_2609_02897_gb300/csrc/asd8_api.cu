// C-ABI entry points of the 8-bit cache and LM head (declared in include/asd8.h):
// host-side argument checks, workspace layout and kernel launches.
#include "host.h"
#include "kernels8.h"

using namespace asd;

namespace {

bool dims8_ok(const asd_dims* d) {
  if (!dims_ok(d) || d->dtype != ASD_BF16) return false;
  // cache rows are counted in 32 bits (TMA coordinates)
  const long long rows = d->page_size
                             ? static_cast<long long>(d->num_pages) * d->num_kv_heads * d->page_size
                             : static_cast<long long>(d->batch) * d->num_kv_heads * d->ctx_max;
  return rows <= 0x7fffffffLL;
}

int kv_block(const asd_dims& d) {
  return d.page_size ? std::min<int>(ASD8_KV_BLOCK, d.page_size) : ASD8_KV_BLOCK;
}

// Scale blocks of a sequence (contiguous) or a page.
int kv_blocks(const asd_dims& d) {
  const int n = kv_block(d);
  return d.page_size ? d.page_size / n : (d.ctx_max + n - 1) / n;
}

// The workspace: the regions of asd_workspace_bytes that every call needs, the hidden
// states in 8 bits, then (optional, as there) the split attention's partial rows.
struct Ws8 {
  size_t h8, h_exp, total, full;
  int t_pad;
};

Ws8 layout8(const asd_dims& d, const WsLayout& L, int T, int nsm) {
  Ws8 w{};
  const size_t nkb = static_cast<size_t>(lm8_kblocks(d.hidden));
  w.t_pad = (T + 127) / 128 * 128;
  size_t off = L.total;
  w.h8 = off;     off = align256(off + nkb * kLm8KB * static_cast<size_t>(T));
  w.h_exp = off;  off = align256(off + (nkb + 3) / 4 * 4 * static_cast<size_t>(w.t_pad));
  w.total = off;
  // 128 query rows of partial results per SM at most, and the plan
  w.full = off + align256(sizeof(int2) * static_cast<size_t>(d.batch)) +
           static_cast<size_t>(nsm) * std::min<long long>(kAttnTcRows, static_cast<long long>(d.max_nodes) *
                                                              (d.num_q_heads / d.num_kv_heads)) *
               (sizeof(float2) + 4 * static_cast<size_t>(d.head_dim));
  return w;
}

asd_status begin_call8(const asd_dims* dims, int32_t total_nodes, void* ws, size_t ws_bytes,
                       void* stream, Ctx* c, Ws8* w) {
  if (!dims) return ASD_ERR_INVALID_ARG;
  if (!dims8_ok(dims)) return ASD_ERR_SHAPE;
  const asd_status st = begin_call(dims, total_nodes, ws, ws_bytes, stream, c);
  if (st != ASD_OK) return st;
  *w = layout8(c->d, c->L, c->T, device_sm_count());
  return ws_bytes < w->total ? ASD_ERR_WORKSPACE : ASD_OK;
}

bool cache_ok(const asd8_cache* c) {
  return c && c->k && c->v && c->k_exp && c->v_exp && aligned16(c->k) && aligned16(c->v);
}

Kv8Params kv8_params(const Ctx& c, const asd8_cache& cache, const void* k_src, const void* v_src,
                     const int32_t* page_table, const int32_t* ctx_len) {
  Kv8Params p{};
  p.k_src = k_src;
  p.v_src = v_src;
  p.k = static_cast<uint8_t*>(cache.k);
  p.v = static_cast<uint8_t*>(cache.v);
  p.k_exp = cache.k_exp;
  p.v_exp = cache.v_exp;
  p.page_table = page_table;
  p.ctx_len = ctx_len;
  p.status = ws_at<int>(c.ws, c.L.status);
  p.B = c.d.batch;
  p.T = c.T;
  p.Hkv = c.d.num_kv_heads;
  p.D = c.d.head_dim;
  p.ctx_max = c.d.ctx_max;
  p.page_size = c.d.page_size;
  p.pages_per_seq = c.d.page_size ? c.d.ctx_max / c.d.page_size : 0;
  p.num_pages = c.d.num_pages;
  p.block = kv_block(c.d);
  p.blocks = kv_blocks(c.d);
  p.max_nodes = c.d.max_nodes;
  p.max_path = c.d.max_path;
  return p;
}

asd_status run_attention8(const Ctx& c, const Ws8& w, const void* q, const asd8_cache& cache,
                          const int32_t* page_table, const int32_t* ctx_len, const void* tree_k,
                          const void* tree_v, const int32_t* parent, const int32_t* cu, void* out,
                          bool in_step) {
  const asd_dims& d = c.d;
  Attn8Params p{};
  AttnParams& a = p.a;
  a.q = q;
  a.k_cache = cache.k;
  a.v_cache = cache.v;
  a.tree_k = tree_k;
  a.tree_v = tree_v;
  a.cu_nodes = cu;
  a.ctx_len = ctx_len;
  a.page_table = page_table;
  a.parent = parent;
  a.status = ws_at<int>(c.ws, c.L.status);
  a.wait_cycles = c.wait_cycles;
  a.out = out;
  a.B = d.batch;
  a.T = c.T;
  a.Hq = d.num_q_heads;
  a.Hkv = d.num_kv_heads;
  a.G = d.num_q_heads / d.num_kv_heads;
  a.D = d.head_dim;
  a.ctx_max = d.ctx_max;
  a.page_size = d.page_size;
  a.pages_per_seq = d.page_size ? d.ctx_max / d.page_size : 0;
  a.num_pages = d.num_pages;
  a.max_nodes = d.max_nodes;
  a.scale_log2 = static_cast<float>(1.4426950408889634 / std::sqrt(static_cast<double>(d.head_dim)));
  a.nsm = device_sm_count();
  a.co_tiles = -1;
  p.k_exp = cache.k_exp;
  p.v_exp = cache.v_exp;
  p.block = kv_block(d);
  p.blocks = kv_blocks(d);
  uint64_t rows = d.page_size ? static_cast<uint64_t>(d.num_pages) * d.num_kv_heads * d.page_size
                              : static_cast<uint64_t>(d.batch) * d.num_kv_heads * d.ctx_max;
  if (rows == 0) rows = 1;   // no context at all: the map is never used
  const uint32_t box = static_cast<uint32_t>(d.page_size ? std::min(d.page_size, kAttnTcKeys) : kAttnTcKeys);
  const uint32_t width = static_cast<uint32_t>(d.head_dim);
  CUtensorMap tk, tv, ttk, ttv;
  if (!make_tmap_u8(&tk, cache.k, width, rows, box, width) ||
      !make_tmap_u8(&tv, cache.v, width, rows, box, width) ||
      !make_tree_tmap_bf16(&ttk, tree_k, d.head_dim, d.num_kv_heads, c.T, kAttnTcKeys) ||
      !make_tree_tmap_bf16(&ttv, tree_v, d.head_dim, d.num_kv_heads, c.T, kAttnTcKeys))
    return ASD_ERR_CUDA;
  // the partial rows of contexts cut into chunks, as far as the workspace holds them; a
  // call by itself has no use for the LM head's regions
  const size_t at = in_step ? w.total : c.L.lm_part;
  const size_t rows_at = at + align256(sizeof(int2) * static_cast<size_t>(d.batch));
  const size_t row_bytes = sizeof(float2) + 4 * static_cast<size_t>(d.head_dim);
  const size_t end = std::min(c.ws_bytes, w.full);
  if (end > rows_at) {
    a.part_cap = std::min<long long>(attention_split_rows(d, c.T, a.nsm),
                                     static_cast<long long>((end - rows_at) / row_bytes)) &
                 ~63LL;   // part_o stays aligned behind part_ml
    a.plan = ws_at<int2>(c.ws, at);
    a.part_ml = ws_at<float2>(c.ws, rows_at);
    a.part_o = ws_at<float>(c.ws, rows_at + sizeof(float2) * static_cast<size_t>(a.part_cap));
  }
  return launch_attention_kv8(p, tk, tv, ttk, ttv, c.st) == cudaSuccess ? ASD_OK : ASD_ERR_CUDA;
}

asd_status run_lmhead8(const Ctx& c, const Ws8& w, const void* hidden, const void* w_packed,
                       float* l_draft) {
  const asd_dims& d = c.d;
  Lm8Params p{};
  p.lm.hidden = hidden;
  p.lm.child_start = ws_at<int32_t>(c.ws, c.L.child_start);
  p.lm.child_cnt = ws_at<int32_t>(c.ws, c.L.child_cnt);
  p.lm.child_tok = ws_at<int32_t>(c.ws, c.L.child_tok);
  p.lm.child_id = ws_at<int32_t>(c.ws, c.L.child_id);
  p.lm.part = ws_at<LmPartial>(c.ws, c.L.lm_part);
  p.lm.l_draft = l_draft;
  p.lm.status = ws_at<int>(c.ws, c.L.status);
  p.lm.wait_cycles = c.wait_cycles;
  p.lm.T = c.T;
  p.lm.K = d.hidden;
  p.lm.V = d.vocab;
  p.lm.g_lm = c.L.g_lm;
  p.lm.a_rows = std::min(128, (c.T + 7) / 8 * 8);
  p.lm.w_packed = static_cast<const uint8_t*>(w_packed);
  p.h8 = ws_at<uint8_t>(c.ws, w.h8);
  p.h_exp = ws_at<uint8_t>(c.ws, w.h_exp);
  p.t_pad = w.t_pad;
  CUtensorMap th;
  if (!make_tmap_u8(&th, p.h8, static_cast<uint64_t>(lm8_kblocks(d.hidden)) * kLm8KB, c.T,
                    static_cast<uint32_t>(p.lm.a_rows), kLm8KB))
    return ASD_ERR_CUDA;
  return launch_lm8_hidden(p, c.st) == cudaSuccess && launch_lmhead_fp8(p, th, c.st) == cudaSuccess
             ? ASD_OK
             : ASD_ERR_CUDA;
}

TailParams finalize_params(const Ctx& c, int mode, const int32_t* parent, const int32_t* tokens,
                           const int32_t* cu, float tau, float* row_max, int32_t* row_argmax,
                           float* row_lse, float* l_draft, float* ratio, uint8_t* accept) {
  TailParams t = tail_params(c, mode);
  t.parent = parent;
  t.tokens = tokens;
  t.cu_nodes = cu;
  t.seq_flags = ws_at<int>(c.ws, c.L.seq_flags);
  t.ln_tau = ln_tau(tau);
  t.row_max = row_max;
  t.row_argmax = row_argmax;
  t.row_lse = row_lse;
  t.l_draft = l_draft;
  t.ratio = ratio;
  t.accept = accept;
  return t;
}

}  // namespace

extern "C" {

int32_t asd8_kv_block(const asd_dims* dims) { return dims8_ok(dims) ? kv_block(*dims) : 0; }

size_t asd8_kv_scales(const asd_dims* dims) {
  if (!dims8_ok(dims)) return 0;
  return static_cast<size_t>(dims->page_size ? dims->num_pages : dims->batch) *
         dims->num_kv_heads * static_cast<size_t>(kv_blocks(*dims));
}

size_t asd8_workspace_bytes(const asd_dims* dims, int32_t total_nodes) {
  if (!dims8_ok(dims) || !nodes_ok(dims, total_nodes)) return 0;
  const int nsm = device_sm_count();
  if (nsm <= 0) return 0;
  return layout8(*dims, layout(*dims, total_nodes, nsm), total_nodes, nsm).full;
}

asd_status asd8_kv_quantize(const asd_dims* dims, const void* k_cache, const void* v_cache,
                            const int32_t* page_table, const int32_t* ctx_len,
                            const asd8_cache* cache, void* workspace, size_t workspace_bytes,
                            void* stream) {
  if (!dims || !k_cache || !v_cache || !ctx_len || !cache_ok(cache)) return ASD_ERR_INVALID_ARG;
  if (dims->page_size && !page_table) return ASD_ERR_INVALID_ARG;
  if (!aligned16(k_cache) || !aligned16(v_cache)) return ASD_ERR_INVALID_ARG;
  Ctx c;
  Ws8 w;
  // the workspace gives the status word only: one node per sequence will do
  const asd_status st = begin_call8(dims, dims->batch, workspace, workspace_bytes, stream, &c, &w);
  if (st != ASD_OK) return st;
  return launch_kv8_quantize(kv8_params(c, *cache, k_cache, v_cache, page_table, ctx_len),
                             device_sm_count(), c.st) == cudaSuccess
             ? ASD_OK
             : ASD_ERR_CUDA;
}

asd_status asd8_tree_attention(const asd_dims* dims, const void* q, const asd8_cache* cache,
                               const int32_t* page_table, const int32_t* ctx_len,
                               const void* tree_k, const void* tree_v, const int32_t* parent,
                               const int32_t* cu_nodes, int32_t total_nodes, void* out,
                               void* workspace, size_t workspace_bytes, void* stream) {
  if (!q || !cache_ok(cache) || !ctx_len || !tree_k || !tree_v || !parent || !cu_nodes || !out)
    return ASD_ERR_INVALID_ARG;
  if (dims && dims->page_size && !page_table) return ASD_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(tree_k) || !aligned16(tree_v) || !aligned16(out))
    return ASD_ERR_INVALID_ARG;
  Ctx c;
  Ws8 w;
  const asd_status st = begin_call8(dims, total_nodes, workspace, workspace_bytes, stream, &c, &w);
  if (st != ASD_OK) return st;
  if (launch_tree_prep(prep_params(c, parent, nullptr, cu_nodes, ctx_len, nullptr), c.st) !=
      cudaSuccess)
    return ASD_ERR_CUDA;
  return run_attention8(c, w, q, *cache, page_table, ctx_len, tree_k, tree_v, parent, cu_nodes, out,
                        false);
}

asd_status asd8_kv_compact(const asd_dims* dims, const void* tree_k, const void* tree_v,
                           const int32_t* cu_nodes, int32_t total_nodes, const int32_t* path,
                           const int32_t* path_len, const int32_t* ctx_len,
                           const int32_t* page_table, const asd8_cache* cache,
                           int32_t* ctx_len_out, void* workspace, size_t workspace_bytes,
                           void* stream) {
  if (!tree_k || !tree_v || !cu_nodes || !path || !path_len || !ctx_len || !cache_ok(cache) ||
      !ctx_len_out)
    return ASD_ERR_INVALID_ARG;
  if (dims && dims->page_size && !page_table) return ASD_ERR_INVALID_ARG;
  if (!aligned16(tree_k) || !aligned16(tree_v)) return ASD_ERR_INVALID_ARG;
  Ctx c;
  Ws8 w;
  const asd_status st = begin_call8(dims, total_nodes, workspace, workspace_bytes, stream, &c, &w);
  if (st != ASD_OK) return st;
  Kv8Params p = kv8_params(c, *cache, tree_k, tree_v, page_table, ctx_len);
  p.cu_nodes = cu_nodes;
  p.path = path;
  p.path_len = path_len;
  p.ctx_len_out = ctx_len_out;
  return launch_kv8_compact(p, c.st) == cudaSuccess ? ASD_OK : ASD_ERR_CUDA;
}

size_t asd8_lm_head_bytes(const asd_dims* dims) {
  return dims8_ok(dims) ? lm8_bytes(dims->vocab, dims->hidden) : 0;
}

asd_status asd8_pack_lm_head(const asd_dims* dims, const void* w, void* w_packed,
                             size_t packed_bytes, void* stream) {
  if (!dims || !w || !w_packed) return ASD_ERR_INVALID_ARG;
  if (!dims8_ok(dims)) return ASD_ERR_SHAPE;
  if (!aligned16(w) || (reinterpret_cast<uintptr_t>(w_packed) & 255u)) return ASD_ERR_INVALID_ARG;
  const size_t need = lm8_bytes(dims->vocab, dims->hidden);
  if (packed_bytes < need) return ASD_ERR_WORKSPACE;
  const uintptr_t a0 = reinterpret_cast<uintptr_t>(w), a1 = a0 + 2ull * dims->vocab * dims->hidden;
  const uintptr_t b0 = reinterpret_cast<uintptr_t>(w_packed), b1 = b0 + need;
  if (a0 < b1 && b0 < a1) return ASD_ERR_INVALID_ARG;
  const int nsm = device_sm_count();
  if (nsm <= 0) return ASD_ERR_CUDA;
  return launch_lm8_pack(w, w_packed, dims->vocab, dims->hidden, lm_ranges(dims->vocab, nsm),
                         static_cast<cudaStream_t>(stream)) == cudaSuccess
             ? ASD_OK
             : ASD_ERR_CUDA;
}

asd_status asd8_lmhead_margin(const asd_dims* dims, const void* hidden, const void* w_packed,
                              const int32_t* tokens, const int32_t* parent,
                              const int32_t* cu_nodes, int32_t total_nodes, float tau,
                              float* row_max, int32_t* row_argmax, float* row_lse,
                              float* l_draft, float* ratio, uint8_t* accept, void* workspace,
                              size_t workspace_bytes, void* stream) {
  if (!hidden || !w_packed || !tokens || !parent || !cu_nodes || !row_max || !row_argmax ||
      !row_lse || !l_draft || !ratio || !accept)
    return ASD_ERR_INVALID_ARG;
  if (!tau_ok(tau)) return ASD_ERR_INVALID_ARG;
  if (!aligned16(hidden) || (reinterpret_cast<uintptr_t>(w_packed) & 255u))
    return ASD_ERR_INVALID_ARG;
  if (dims && dims->lm_head_schedule != ASD_LM_EVERY_ROW) return ASD_ERR_SHAPE;
  Ctx c;
  Ws8 w;
  asd_status st = begin_call8(dims, total_nodes, workspace, workspace_bytes, stream, &c, &w);
  if (st != ASD_OK) return st;
  if (launch_tree_prep(prep_params(c, parent, tokens, cu_nodes, nullptr, l_draft), c.st) !=
      cudaSuccess)
    return ASD_ERR_CUDA;
  st = run_lmhead8(c, w, hidden, w_packed, l_draft);
  if (st != ASD_OK) return st;
  return launch_tail(finalize_params(c, kTailFinalize, parent, tokens, cu_nodes, tau, row_max,
                                     row_argmax, row_lse, l_draft, ratio, accept),
                     c.st) == cudaSuccess
             ? ASD_OK
             : ASD_ERR_CUDA;
}

asd_status asd8_verify_step(const asd_dims* dims, const asd8_verify_args* args, void* workspace,
                            size_t workspace_bytes, void* stream) {
  if (!args) return ASD_ERR_INVALID_ARG;
  const asd_verify_args* a = &args->step;
  const bool w8 = args->weight == ASD8_W_E4M3;
  if (!a->q || !a->tree_k || !a->tree_v || !a->hidden || !a->w_lm || !a->tokens || !a->parent ||
      !a->cu_nodes || !a->ctx_len || a->k_cache || a->v_cache || !a->attn_out || !a->row_max ||
      !a->row_argmax || !a->row_lse || !a->l_draft || !a->ratio || !a->accept || !a->path ||
      !a->path_len || !a->bonus || !a->n_promoted || !a->ctx_len_out || !cache_ok(&args->cache))
    return ASD_ERR_INVALID_ARG;
  if ((!w8 && args->weight != ASD8_W_BF16) || args->reserved) return ASD_ERR_INVALID_ARG;
  if (dims && dims->page_size && !a->page_table) return ASD_ERR_INVALID_ARG;
  if (!tau_ok(a->tau)) return ASD_ERR_INVALID_ARG;
  if (!aligned16(a->q) || !aligned16(a->tree_k) || !aligned16(a->tree_v) ||
      !aligned16(a->hidden) || !aligned16(a->w_lm) || !aligned16(a->attn_out) ||
      (w8 && (reinterpret_cast<uintptr_t>(a->w_lm) & 255u)))
    return ASD_ERR_INVALID_ARG;
  const bool lazy = dims && dims->lm_head_schedule == ASD_LM_LAZY_LEVELS;
  if (lazy && w8) return ASD_ERR_SHAPE;
  Ctx c;
  Ws8 w;
  asd_status st = begin_call8(dims, a->total_nodes, workspace, workspace_bytes, stream, &c, &w);
  if (st != ASD_OK) return st;
  record(a->stage_events[0], c.st);
  if (launch_tree_prep(prep_params(c, a->parent, a->tokens, a->cu_nodes, a->ctx_len, a->l_draft),
                       c.st) != cudaSuccess)
    return ASD_ERR_CUDA;
  record(a->stage_events[1], c.st);
  st = w8     ? run_lmhead8(c, w, a->hidden, a->w_lm, a->l_draft)
       : lazy ? run_lmhead_lazy(c, a->hidden, a->w_lm, a->parent, a->tokens, a->cu_nodes, a->tau,
                                a->row_max, a->row_argmax, a->row_lse, a->l_draft, a->ratio,
                                a->accept)
              : run_lmhead(c, a->hidden, a->w_lm, a->l_draft);
  if (st != ASD_OK) return st;
  record(a->stage_events[2], c.st);
  st = run_attention8(c, w, a->q, args->cache, a->page_table, a->ctx_len, a->tree_k, a->tree_v,
                      a->parent, a->cu_nodes, a->attn_out, true);
  if (st != ASD_OK) return st;
  record(a->stage_events[3], c.st);
  TailParams t = finalize_params(c, (lazy ? 0 : kTailFinalize) | kTailWalk, a->parent, a->tokens,
                                 a->cu_nodes, a->tau, a->row_max, a->row_argmax, a->row_lse,
                                 a->l_draft, a->ratio, a->accept);
  t.path = a->path;
  t.path_len = a->path_len;
  t.bonus = a->bonus;
  t.n_promoted = a->n_promoted;
  t.ctx_len = a->ctx_len;   // (a path that does not fit is none)
  t.page_table = a->page_table;
  if (launch_tail(t, c.st) != cudaSuccess) return ASD_ERR_CUDA;
  Kv8Params k = kv8_params(c, args->cache, a->tree_k, a->tree_v, a->page_table, a->ctx_len);
  k.cu_nodes = a->cu_nodes;
  k.path = a->path;
  k.path_len = a->path_len;
  k.ctx_len_out = a->ctx_len_out;
  k.in_step = 1;
  if (launch_kv8_compact(k, c.st) != cudaSuccess) return ASD_ERR_CUDA;
  record(a->stage_events[4], c.st);
  return ASD_OK;
}

}  // extern "C"
