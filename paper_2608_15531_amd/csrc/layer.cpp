// C ABI of the operators around the matmuls in a decoder layer: argument checks
// and dispatch to the HIP launchers.  Every check runs on the host before
// anything is enqueued.
#include "layer.hpp"

#include <climits>
#include <cmath>
#include <cstdint>

#include "internal.hpp"

namespace {

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

bool is_stride(int64_t s, int64_t unit) { return s >= 0 && s % unit == 0; }

// The stride of a dimension of n: that of one place alone is never used, and callers
// keep any number there.
int64_t used(int64_t stride, int64_t n) { return n > 1 ? stride : 0; }

// Rows of `row` units, n of them `stride` apart, lie over one another: different workgroups
// would write the same memory.
bool overlap(int64_t stride, int64_t n, int64_t row) { return n > 1 && stride < row; }

// The same of a cache's rows and words that are to be written.
bool overlap(const fq_kv_cache& c) {
  const int64_t row = c.kind == FQ_KV_BF16 ? 2 * c.head_dim : c.kind == FQ_KV_INT8 ? c.head_dim : c.head_dim / 2;
  if (overlap(c.page_stride, c.n_pages, row) || overlap(c.head_stride, c.n_kv_heads, row) ||
      overlap(c.token_stride, c.page_size, row))
    return true;
  return c.kind != FQ_KV_BF16 && (overlap(c.meta_page_stride, c.n_pages, c.page_size) ||
                                  overlap(c.meta_head_stride, c.n_kv_heads, c.page_size));
}

// Sizes, kind and strides: all that needs no pointer.
fq_status check_cache_sizes(const fq_kv_cache* c) {
  if (!c) return FQ_ERR_NULL;
  if (c->n_pages < 1 || c->page_size < 1 || c->n_kv_heads < 1 || c->head_dim < 1) return FQ_ERR_SHAPE;
  if (c->kind != FQ_KV_BF16 && c->kind != FQ_KV_INT8 && c->kind != FQ_KV_INT4) return FQ_ERR_UNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 128) return FQ_ERR_UNSUPPORTED;
  if (c->page_size % fqi::kKvBlock != 0 || c->page_size > 65536) return FQ_ERR_UNSUPPORTED;
  if (c->n_pages > INT32_MAX || c->n_kv_heads > 65535) return FQ_ERR_UNSUPPORTED;
  const int64_t page_stride = used(c->page_stride, c->n_pages), head_stride = used(c->head_stride, c->n_kv_heads);
  if (page_stride < 0 || head_stride < 0 || c->token_stride < 0) return FQ_ERR_SHAPE;
  // byte offsets inside a 16-token block are 32 bits wide in the kernels
  if (c->token_stride > INT32_MAX / 32) return FQ_ERR_UNSUPPORTED;
  if (page_stride % 16 != 0 || head_stride % 16 != 0 || c->token_stride % 16 != 0) return FQ_ERR_ALIGN;
  if (c->kind != FQ_KV_BF16) {
    const int64_t meta_page = used(c->meta_page_stride, c->n_pages);
    const int64_t meta_head = used(c->meta_head_stride, c->n_kv_heads);
    if (meta_page < 0 || meta_head < 0) return FQ_ERR_SHAPE;
    if (meta_page % 4 != 0 || meta_head % 4 != 0) return FQ_ERR_ALIGN;
  }
  return FQ_OK;
}

fq_status check_cache(const fq_kv_cache* c) {
  const fq_status st = check_cache_sizes(c);
  if (st != FQ_OK) return st;
  if (!c->k || !c->v) return FQ_ERR_NULL;
  if (!aligned(c->k, 16) || !aligned(c->v, 16)) return FQ_ERR_ALIGN;
  if (c->kind != FQ_KV_BF16) {
    if (!c->k_meta || !c->v_meta) return FQ_ERR_NULL;
    if (!aligned(c->k_meta, 16) || !aligned(c->v_meta, 16)) return FQ_ERR_ALIGN;
  }
  return FQ_OK;
}

fq_status check_attention(const fq_attention* a, const fq_kv_cache* c) {
  if (!a) return FQ_ERR_NULL;
  const fq_status st = check_cache_sizes(c);
  if (st != FQ_OK) return st;
  if (a->n_seqs < 1 || a->n_heads < 1 || a->max_q < 1 || a->max_kv < 1 || a->total_q < 0 ||
      a->window < 0 || a->sinks < 0 || a->table_cols < 1 || a->table_stride < 0)
    return FQ_ERR_SHAPE;
  if (a->n_heads % c->n_kv_heads != 0) return FQ_ERR_SHAPE;
  if (int64_t(a->table_cols) * c->page_size < a->max_kv) return FQ_ERR_SHAPE;
  // (the softmax runs in powers of two)
  if (!std::isfinite(a->scale * fqi::kLog2e)) return FQ_ERR_SHAPE;
  const int64_t strides[4] = {used(a->q_token_stride, a->total_q), used(a->q_head_stride, a->n_heads),
                              used(a->o_token_stride, a->total_q), used(a->o_head_stride, a->n_heads)};
  for (int64_t s : strides)
    if (s < 0) return FQ_ERR_SHAPE;
  for (int64_t s : strides)
    if (s % 8 != 0) return FQ_ERR_ALIGN;
  // key numbers below 2^28 (the kernels' division by the page size), positions 32 bits wide
  if (a->max_kv > (1 << 28) || a->max_q > (1 << 28)) return FQ_ERR_UNSUPPORTED;
  return FQ_OK;
}

fq_status hip_status(int e) { return e == 0 ? FQ_OK : FQ_ERR_HIP; }

}  // namespace

extern "C" {

fq_status fq_kv_cache_write(const fq_kv_cache* cache, const uint16_t* K, const uint16_t* V,
                            int64_t k_token_stride, int64_t k_head_stride,
                            int64_t v_token_stride, int64_t v_head_stride, const int64_t* slots,
                            int64_t n_tokens, void* stream) {
  const fq_status st = check_cache(cache);
  if (st != FQ_OK) return st;
  if (n_tokens < 0 || overlap(*cache)) return FQ_ERR_SHAPE;
  k_token_stride = used(k_token_stride, n_tokens);
  v_token_stride = used(v_token_stride, n_tokens);
  k_head_stride = used(k_head_stride, cache->n_kv_heads);
  v_head_stride = used(v_head_stride, cache->n_kv_heads);
  if (k_token_stride < 0 || k_head_stride < 0 || v_token_stride < 0 || v_head_stride < 0) return FQ_ERR_SHAPE;
  if (n_tokens == 0) return FQ_OK;
  if (!K || !V || !slots) return FQ_ERR_NULL;
  if (!is_stride(k_token_stride, 8) || !is_stride(k_head_stride, 8) || !is_stride(v_token_stride, 8) ||
      !is_stride(v_head_stride, 8) || !aligned(K, 16) || !aligned(V, 16) || !aligned(slots, 8))
    return FQ_ERR_ALIGN;
  if (n_tokens > INT32_MAX) return FQ_ERR_UNSUPPORTED;
  return hip_status(fqi::launch_kv_write(*cache, K, V, k_token_stride, k_head_stride, v_token_stride,
                                         v_head_stride, slots, n_tokens, stream));
}

fq_status fq_kv_cache_read(const fq_kv_cache* cache, const int64_t* slots, int64_t n_tokens,
                           void* K, void* V, int32_t dtype, void* stream) {
  const fq_status st = check_cache(cache);
  if (st != FQ_OK) return st;
  if (n_tokens < 0) return FQ_ERR_SHAPE;
  if (dtype != FQ_Y_BF16 && dtype != FQ_Y_F32) return FQ_ERR_UNSUPPORTED;
  if (n_tokens == 0) return FQ_OK;
  if (!K || !V || !slots) return FQ_ERR_NULL;
  if (!aligned(K, 16) || !aligned(V, 16) || !aligned(slots, 8)) return FQ_ERR_ALIGN;
  if (n_tokens > INT32_MAX) return FQ_ERR_UNSUPPORTED;
  return hip_status(fqi::launch_kv_read(*cache, slots, n_tokens, K, V, dtype == FQ_Y_F32, stream));
}

fq_status fq_paged_attention_workspace_bytes(const fq_attention* a, const fq_kv_cache* cache,
                                             size_t* bytes) {
  if (!bytes) return FQ_ERR_NULL;
  const fq_status st = check_attention(a, cache);
  if (st != FQ_OK) return st;
  fqi::AttnPlan pl;
  if (!fqi::plan_attention(*a, *cache, &pl)) return FQ_ERR_UNSUPPORTED;
  *bytes = pl.ws_bytes;
  return FQ_OK;
}

fq_status fq_paged_attention_launch(const fq_attention* a, const fq_kv_cache* cache,
                                    int32_t out[8]) {
  if (!out) return FQ_ERR_NULL;
  const fq_status st = check_attention(a, cache);
  if (st != FQ_OK) return st;
  fqi::AttnPlan pl;
  if (!fqi::plan_attention(*a, *cache, &pl)) return FQ_ERR_UNSUPPORTED;
  out[0] = pl.kernel;
  out[1] = pl.rows;
  out[2] = pl.row_blocks;
  out[3] = pl.split;
  out[4] = pl.split_tiles * pl.tile;   // max_kv <= 2^28
  out[5] = int32_t(pl.workgroups);
  out[6] = int32_t(pl.lds_bytes);
  out[7] = int32_t((pl.partial_bytes + 1023) >> 10);
  return FQ_OK;
}

fq_status fq_paged_attention(const fq_attention* a, const uint16_t* Q, const fq_kv_cache* cache,
                             const int32_t* cu_q, const int32_t* kv_lens,
                             const int32_t* block_table, uint16_t* O, float* lse,
                             void* workspace, size_t workspace_bytes, void* stream) {
  fq_status st = check_attention(a, cache);
  if (st == FQ_OK) st = check_cache(cache);
  if (st != FQ_OK) return st;
  if (overlap(a->o_token_stride, a->total_q, cache->head_dim) || overlap(a->o_head_stride, a->n_heads, cache->head_dim))
    return FQ_ERR_SHAPE;
  if (a->total_q == 0) return FQ_OK;
  if (!Q || !cu_q || !kv_lens || !block_table || !O) return FQ_ERR_NULL;
  if (!aligned(Q, 16) || !aligned(O, 16) || !aligned(lse, 4) || !aligned(cu_q, 4) ||
      !aligned(kv_lens, 4) || !aligned(block_table, 4))
    return FQ_ERR_ALIGN;
  fqi::AttnPlan pl;
  if (!fqi::plan_attention(*a, *cache, &pl)) return FQ_ERR_UNSUPPORTED;
  if (pl.split > 1 && (!workspace || workspace_bytes < pl.ws_bytes || !aligned(workspace, 256)))
    return FQ_ERR_WORKSPACE;
  return hip_status(fqi::launch_attention(pl, *a, *cache, Q, cu_q, kv_lens, block_table, O, lse,
                                          workspace, stream));
}

fq_status fq_gated_residual_norm(const fq_norm* n, const void* x, const void* residual,
                                 const uint16_t* post_weight, const uint16_t* gate,
                                 const uint16_t* pre_weight, void* residual_out, uint16_t* h,
                                 void* stream) {
  if (!n) return FQ_ERR_NULL;
  if (n->rows < 0 || n->cols < 1 || n->x_stride < 0 || n->residual_stride < 0 || n->gate_stride < 0 ||
      n->residual_out_stride < 0 || n->h_stride < 0)
    return FQ_ERR_SHAPE;
  if (!std::isfinite(n->eps) || n->eps < 0 || !std::isfinite(n->residual_scale)) return FQ_ERR_SHAPE;
  if ((n->x_dtype != FQ_Y_BF16 && n->x_dtype != FQ_Y_F32) ||
      (n->residual_dtype != FQ_Y_BF16 && n->residual_dtype != FQ_Y_F32) || n->cols > 32768 ||
      n->rows > INT32_MAX)
    return FQ_ERR_UNSUPPORTED;
  if ((residual_out && overlap(n->residual_out_stride, n->rows, n->cols)) || (h && overlap(n->h_stride, n->rows, n->cols)))
    return FQ_ERR_SHAPE;
  if (n->rows == 0) return FQ_OK;
  if (!residual_out && !h) return FQ_ERR_NULL;
  if (!x || (h && !pre_weight)) return FQ_ERR_NULL;
  const uintptr_t xa = n->x_dtype == FQ_Y_F32 ? 4 : 2, ra = n->residual_dtype == FQ_Y_F32 ? 4 : 2;
  if (!aligned(x, xa) || !aligned(residual, ra) || !aligned(residual_out, ra) || !aligned(post_weight, 2) ||
      !aligned(gate, 2) || !aligned(pre_weight, 2) || !aligned(h, 2))
    return FQ_ERR_ALIGN;
  return hip_status(fqi::launch_norm(*n, x, residual, post_weight, gate, pre_weight, residual_out, h, stream));
}

}  // extern "C"
