// C ABI of the decode-layer operators: argument checks before any launch.
#include <math.h>

#include "hbf.h"
#include "hbf_ops.h"

using namespace hbf;

namespace {

bool aligned(const void *p, uintptr_t a) { return (uintptr_t)p % a == 0; }
bool dtype_ok(uint32_t d) { return d == HBF_BF16 || d == HBF_FP16; }
int status_of(hipError_t e) { return e == hipSuccess ? HBF_OK : HBF_EHIP; }

int check_kv_sizes(const hbf_kv *kv) {
  if (!kv || kv->planes < 1 || kv->planes > 65535 || kv->pages < 1 || kv->pages > KV_MAX_PAGES || kv->page_tokens < 1 ||
      kv->page_tokens > 65536 || kv->slots < 1 || kv->slots > KV_MAX_SLOTS || kv->table_cols < 1 ||
      kv->table_cols > 1 << 24 || kv->table_stride < kv->table_cols)
    return HBF_EINVAL;
  if ((int64_t)kv->table_cols * kv->page_tokens > INT32_MAX) return HBF_EINVAL;
  if (kv->token_bytes < 16 || kv->token_bytes > 1 << 20 || kv->token_bytes % 16 || kv->page_stride % 16 ||
      kv->plane_stride % 16 || kv->page_stride < kv->token_bytes * kv->page_tokens)
    return HBF_EINVAL;
  return HBF_OK;
}

// What every call on a cache needs of its description.
int check_kv(const hbf_kv *kv) {
  const int rc = check_kv_sizes(kv);
  if (rc) return rc;
  if (!kv->dev_pool || !kv->dev_refs || !kv->dev_tables || !kv->dev_lens || !kv->dev_ws) return HBF_EINVAL;
  if (!aligned(kv->dev_pool, 16) || !aligned(kv->dev_refs, 4) || !aligned(kv->dev_tables, 4) ||
      !aligned(kv->dev_lens, 4) || !aligned(kv->dev_ws, 256))
    return HBF_EINVAL;
  return HBF_OK;
}

int check_list(const void *a, const void *b, int n) {
  if (n < 0 || n > KV_MAX_LIST) return HBF_EINVAL;
  if (n > 0 && (!a || !b || !aligned(a, 4) || !aligned(b, 4))) return HBF_EINVAL;
  return HBF_OK;
}

// A layer's pages, as attention reads them.
int check_layer(const hbf_kv_layer *kv) {
  if (!dtype_ok(kv->dtype) || (kv->head_dim != 64 && kv->head_dim != 128) || kv->kv_heads < 1 ||
      kv->kv_heads > 1024 || kv->pages < 1 || kv->pages > KV_MAX_PAGES || kv->page_tokens < 1 ||
      kv->page_tokens > 65536)
    return HBF_EINVAL;
  if (kv->page_stride < 0 || kv->token_stride < 0 || kv->head_stride < 0 || kv->page_stride % 8 ||
      kv->token_stride % 8 || kv->head_stride % 8)
    return HBF_EINVAL;
  return HBF_OK;
}

int check_attention(const hbf_kv_layer *kv, const hbf_attention *at) {
  if (!kv || !at) return HBF_EINVAL;
  const int rc = check_layer(kv);
  if (rc) return rc;
  if (at->rows < 0 || at->rows > 65535 || at->heads < kv->kv_heads || at->heads > 1024 ||
      at->heads % kv->kv_heads || (int64_t)at->rows * at->heads > 1 << 22)
    return HBF_EINVAL;
  if (!isfinite(at->scale)) return HBF_EINVAL;
  if (at->prefix_len < 0 || at->prefix_len > INT32_MAX || at->max_own < 0) return HBF_EINVAL;
  if (at->q_row_stride % 8 || at->q_head_stride % 8 || at->out_row_stride % 8 || at->out_head_stride % 8)
    return HBF_EINVAL;
  return HBF_OK;
}

int check_chunk(const hbf_kv *kv, const hbf_kv_layer *layer, const hbf_chunk *ch) {
  if (!layer || !ch) return HBF_EINVAL;
  int rc = check_kv_sizes(kv);
  if (rc || (rc = check_layer(layer))) return rc;
  if (kv->page_tokens != layer->page_tokens) return HBF_EINVAL;
  if (ch->tokens < 0 || ch->tokens > 1 << 20 || ch->rows < 0 || ch->rows > 65535 || ch->heads < layer->kv_heads ||
      ch->heads > 1024 || ch->heads % layer->kv_heads || (int64_t)ch->tokens * ch->heads > 1 << 24)
    return HBF_EINVAL;
  // a workgroup of 256 threads for each row's and KV head's 16 queries, all in one launch, which has fewer than 2^32 threads
  if ((int64_t)ch->rows * layer->kv_heads * 16 + (int64_t)ch->tokens * ch->heads >= 1 << 28) return HBF_EINVAL;
  if (!isfinite(ch->scale) || ch->window < 0 || ch->sinks < 0) return HBF_EINVAL;
  if (ch->q_row_stride % 8 || ch->q_head_stride % 8 || ch->out_row_stride % 8 || ch->out_head_stride % 8)
    return HBF_EINVAL;
  if (ch->weights_slot_stride < 0 || ch->weights_head_stride < 0 || ch->weights_tokens < 0) return HBF_EINVAL;
  return HBF_OK;
}

int check_new_tokens(const hbf_kv *kv, const hbf_new_tokens *nt) {
  if (!nt || !dtype_ok(nt->dtype) || (nt->flags & ~HBF_ROT_PAIRS)) return HBF_EINVAL;
  if (nt->head_dim != 64 && nt->head_dim != 128) return HBF_EINVAL;
  if (nt->n < 0 || nt->n > 1 << 20 || nt->heads < 1 || nt->heads > 1024 || nt->kv_heads < 1 || nt->kv_heads > 1024 ||
      kv->token_bytes != (uint64_t)nt->kv_heads * nt->head_dim * 2)
    return HBF_EINVAL;
  if (!isfinite(nt->eps) || nt->eps < 0 || nt->pairs < 0 || nt->pairs > nt->head_dim / 2 || nt->pairs % 8)
    return HBF_EINVAL;
  const int64_t strides[] = {nt->q_row_stride, nt->q_head_stride, nt->k_row_stride,   nt->k_head_stride,
                             nt->v_row_stride, nt->v_head_stride, nt->out_row_stride, nt->out_head_stride};
  for (int64_t s : strides)
    if (s % 8) return HBF_EINVAL;
  return HBF_OK;
}

int check_moe(const hbf_moe *m) {
  if (!m || !dtype_ok(m->dtype) || (m->flags & ~HBF_MOE_RENORM)) return HBF_EINVAL;
  if (m->experts < 1 || m->experts > MOE_MAX_EXPERTS || m->topk < 1 || m->topk > MOE_MAX_TOPK) return HBF_EINVAL;
  if (m->dev_router && m->topk > m->experts) return HBF_EINVAL;
  if (m->hidden < 8 || m->hidden > 16384 || m->hidden % 8 || m->ffn < 8 || m->ffn > 16384 || m->ffn % 8)
    return HBF_EINVAL;
  return HBF_OK;
}
bool moe_tokens_ok(const hbf_moe *m, int tokens) {
  return tokens >= 0 && tokens <= MOE_MAX_TOKENS && tokens * m->topk <= MOE_MAX_PAIRS;
}

}  // namespace

extern "C" {

int hbf_kv_workspace_bytes(const hbf_kv *kv, int max_list, size_t *bytes) {
  const int rc = check_kv_sizes(kv);
  if (rc) return rc;
  if (!bytes || max_list < 0 || max_list > KV_MAX_LIST) return HBF_EINVAL;
  *bytes = kv_ws_bytes(kv->pages, max_list);
  return HBF_OK;
}

int hbf_kv_extend(const hbf_kv *kv, const int32_t *slots, const int32_t *add, int n, int ws_list, void *stream) {
  int rc = check_kv(kv);
  if (rc || (rc = check_list(slots, add, n))) return rc;
  if (ws_list < n || ws_list > KV_MAX_LIST) return ws_list < n ? HBF_ENOWORKSPACE : HBF_EINVAL;
  return n ? status_of(launch_kv_extend(*kv, slots, add, n, ws_list, (hipStream_t)stream)) : HBF_OK;
}

int hbf_kv_fork(const hbf_kv *kv, const int32_t *parents, const int32_t *children, int n, int ws_list,
                void *stream) {
  int rc = check_kv(kv);
  if (rc || (rc = check_list(parents, children, n))) return rc;
  if (ws_list < n || ws_list > KV_MAX_LIST) return ws_list < n ? HBF_ENOWORKSPACE : HBF_EINVAL;
  return n ? status_of(launch_kv_fork(*kv, parents, children, n, ws_list, (hipStream_t)stream)) : HBF_OK;
}

int hbf_kv_free(const hbf_kv *kv, const int32_t *slots, int n, void *stream) {
  int rc = check_kv(kv);
  if (rc || (rc = check_list(slots, slots, n))) return rc;
  return n ? status_of(launch_kv_free(*kv, slots, n, (hipStream_t)stream)) : HBF_OK;
}

int hbf_kv_copy(const hbf_kv *kv, const int32_t *src, const int32_t *dst, int n, void *stream) {
  int rc = check_kv(kv);
  if (rc || (rc = check_list(src, dst, n))) return rc;
  return n ? status_of(launch_kv_copy(*kv, src, dst, n, (hipStream_t)stream)) : HBF_OK;
}

int hbf_kv_compact(const hbf_kv *kv, int32_t *remap, int32_t *tables_out, int32_t *refs_out, void *stream) {
  int rc = check_kv(kv);
  if (rc) return rc;
  if (!remap || !aligned(remap, 4) || !aligned(tables_out, 4) || !aligned(refs_out, 4)) return HBF_EINVAL;
  return status_of(launch_kv_compact(*kv, remap, tables_out ? tables_out : kv->dev_tables,
                                     refs_out ? refs_out : kv->dev_refs, (hipStream_t)stream));
}

int hbf_kv_write(const hbf_kv *kv, int first_layer, int layers, const void *k, const void *v, const int32_t *slots,
                 const int32_t *pos, int n, void *stream) {
  int rc = check_kv(kv);
  if (rc || (rc = check_list(slots, pos, n))) return rc;
  if (first_layer < 0 || layers < 0 || (int64_t)first_layer + layers > kv->planes / 2) return HBF_EINVAL;
  if (n == 0 || layers == 0) return HBF_OK;
  if (!k || !v || !aligned(k, 16) || !aligned(v, 16)) return HBF_EINVAL;
  if ((uint64_t)n * (kv->token_bytes / 16) > 1u << 31) return HBF_EINVAL;
  return status_of(launch_kv_write(*kv, first_layer, layers, k, v, slots, pos, n, (hipStream_t)stream));
}

int hbf_kv_get_status(const hbf_kv *kv, void *stream) {
  const int rc = check_kv(kv);
  if (rc) return rc;
  if (hipStreamSynchronize((hipStream_t)stream) != hipSuccess) return HBF_EHIP;
  uint32_t s = 0;
  const uint32_t zero = 0;
  uint32_t *word = &((KvCtl *)kv->dev_ws)->sticky;
  if (hipMemcpy(&s, word, 4, hipMemcpyDeviceToHost) != hipSuccess) return HBF_EHIP;
  if (s && hipMemcpy(word, &zero, 4, hipMemcpyHostToDevice) != hipSuccess) return HBF_EHIP;
  if (s & KV_ERR_ARG) return HBF_EINVAL;
  return s & KV_ERR_PAGES ? HBF_ENOMEM : HBF_OK;
}

int hbf_kv_attention_workspace_bytes(const hbf_kv_layer *kv, const hbf_attention *at, size_t *bytes) {
  const int rc = check_attention(kv, at);
  if (rc) return rc;
  if (!bytes) return HBF_EINVAL;
  *bytes = attn_ws_bytes(*kv, *at);
  return HBF_OK;
}

int hbf_kv_attention(const hbf_kv_layer *kv, const hbf_attention *at, int32_t *status, void *ws, size_t ws_bytes,
                     void *stream) {
  const int rc = check_attention(kv, at);
  if (rc) return rc;
  if (at->rows == 0) return HBF_OK;
  if (!kv->dev_k || !kv->dev_v || !at->dev_q || !at->dev_out || !aligned(kv->dev_k, 16) || !aligned(kv->dev_v, 16) ||
      !aligned(at->dev_q, 16) || !aligned(at->dev_out, 16) || !aligned(at->dev_lse, 4) || !aligned(status, 4))
    return HBF_EINVAL;
  if (at->prefix_len > 0 && (!at->dev_prefix_pages || !aligned(at->dev_prefix_pages, 4))) return HBF_EINVAL;
  if (at->max_own > 0 && (!at->dev_tables || !at->dev_own_len || !aligned(at->dev_tables, 4) ||
                          !aligned(at->dev_own_len, 4)))
    return HBF_EINVAL;
  if (!ws || !aligned(ws, 256) || !aligned(at->dev_ctl, 4)) return HBF_EINVAL;
  if (ws_bytes < attn_ws_bytes(*kv, *at)) return HBF_ENOWORKSPACE;
  return status_of(launch_attn(*kv, *at, status, ws, (hipStream_t)stream));
}

int hbf_kv_write_rotated(const hbf_kv *kv, int layer, const hbf_new_tokens *nt, void *stream) {
  int rc = check_kv(kv);
  if (rc || (rc = check_new_tokens(kv, nt))) return rc;
  if (layer < 0 || layer >= kv->planes / 2) return HBF_EINVAL;
  if (nt->n == 0) return HBF_OK;
  if (!nt->dev_q || !nt->dev_k || !nt->dev_v || !nt->dev_q_out || !aligned(nt->dev_q, 16) || !aligned(nt->dev_k, 16) ||
      !aligned(nt->dev_v, 16) || !aligned(nt->dev_q_out, 16) || !aligned(nt->dev_q_weight, 16) ||
      !aligned(nt->dev_k_weight, 16))
    return HBF_EINVAL;
  if ((nt->pairs > 0 && !nt->dev_freqs) || !aligned(nt->dev_freqs, 8) || !nt->dev_slots || !nt->dev_pos ||
      !aligned(nt->dev_slots, 4) || !aligned(nt->dev_pos, 4) || !aligned(nt->dev_positions, 4))
    return HBF_EINVAL;
  return status_of(launch_kv_write_rotated(*kv, layer, *nt, (hipStream_t)stream));
}

int hbf_kv_chunk_workspace_bytes(const hbf_kv *kv, const hbf_kv_layer *layer, const hbf_chunk *ch, size_t *bytes) {
  const int rc = check_chunk(kv, layer, ch);
  if (rc) return rc;
  if (!bytes) return HBF_EINVAL;
  *bytes = chunk_ws_bytes(*kv, *layer, *ch);
  return HBF_OK;
}

int hbf_kv_chunk_attention(const hbf_kv *kv, const hbf_kv_layer *layer, const hbf_chunk *ch, int32_t *status, void *ws,
                           size_t ws_bytes, void *stream) {
  const int rc = check_chunk(kv, layer, ch);
  if (rc) return rc;
  if (ch->rows == 0 || ch->tokens == 0) return HBF_OK;
  if (!kv->dev_tables || !kv->dev_lens || !aligned(kv->dev_tables, 4) || !aligned(kv->dev_lens, 4)) return HBF_EINVAL;
  if (!layer->dev_k || !layer->dev_v || !ch->dev_q || !ch->dev_out || !aligned(layer->dev_k, 16) ||
      !aligned(layer->dev_v, 16) || !aligned(ch->dev_q, 16) || !aligned(ch->dev_out, 16) || !aligned(ch->dev_lse, 4) ||
      !aligned(ch->dev_weights, 4) || !aligned(ch->dev_ctl, 4) || !aligned(status, 4))
    return HBF_EINVAL;
  if (!ch->dev_slots || !ch->dev_starts || !aligned(ch->dev_slots, 4) || !aligned(ch->dev_starts, 4)) return HBF_EINVAL;
  if (!ws || !aligned(ws, 256)) return HBF_EINVAL;
  if (ws_bytes < chunk_ws_bytes(*kv, *layer, *ch)) return HBF_ENOWORKSPACE;
  return status_of(launch_chunk(*kv, *layer, *ch, status, ws, (hipStream_t)stream));
}

int hbf_kv_evict(const hbf_kv *kv, const hbf_eviction *ev, void *stream) {
  const int rc = check_kv(kv);
  if (rc) return rc;
  if (!ev || kv->planes % 2 || ev->n < 0 || ev->n > KV_MAX_LIST || ev->kv_heads < 1 || ev->kv_heads > 1024 ||
      kv->token_bytes % (16 * (uint64_t)ev->kv_heads) || ev->sinks < 0 || ev->recent < 0 || ev->weights_tokens < 0 ||
      ev->max_keep < 0 || ev->max_keep > 1 << 24 || ev->layer_stride < 0 || ev->slot_stride < 0 || ev->head_stride < 0)
    return HBF_EINVAL;
  const int64_t groups = (int64_t)(kv->planes / 2) * ev->n * ev->kv_heads;
  if (groups > 1 << 22 || groups * ev->max_keep > (int64_t)1 << 40) return HBF_EINVAL;
  if (ev->n == 0) return HBF_OK;
  if (!ev->dev_slots || !ev->dev_keep || !ev->dev_weights || (ev->max_keep > 0 && !ev->dev_kept) ||
      !aligned(ev->dev_slots, 4) || !aligned(ev->dev_keep, 4) || !aligned(ev->dev_weights, 4) ||
      !aligned(ev->dev_weights_out, 4) || !aligned(ev->dev_kept, 4))
    return HBF_EINVAL;
  return status_of(launch_kv_evict(*kv, *ev, (hipStream_t)stream));
}

int hbf_moe_workspace_bytes(const hbf_moe *moe, int tokens, size_t *bytes) {
  const int rc = check_moe(moe);
  if (rc) return rc;
  if (!bytes || !moe_tokens_ok(moe, tokens)) return HBF_EINVAL;
  *bytes = moe_ws_bytes(*moe, tokens);
  return HBF_OK;
}

int hbf_moe_layer(const hbf_moe *moe, const void *x, int64_t x_stride, int tokens, int32_t *ids, float *weights,
                  void *y, int64_t y_stride, int32_t *status, void *ws, size_t ws_bytes, void *stream) {
  const int rc = check_moe(moe);
  if (rc) return rc;
  if (!moe_tokens_ok(moe, tokens)) return HBF_EINVAL;
  if (!moe->dev_gate_up || !moe->dev_down || !aligned(moe->dev_gate_up, 16) || !aligned(moe->dev_down, 16) ||
      !aligned(moe->dev_router, 16) || moe->gate_up_stride % 8 || moe->down_stride % 8)
    return HBF_EINVAL;
  if (tokens == 0) return HBF_OK;
  if (!x || !y || !ids || !weights || !aligned(x, 16) || !aligned(y, 16) || !aligned(ids, 4) ||
      !aligned(weights, 4) || !aligned(status, 4) || x_stride % 8 || y_stride % 8)
    return HBF_EINVAL;
  if (!ws || !aligned(ws, 256)) return HBF_EINVAL;
  if (ws_bytes < moe_ws_bytes(*moe, tokens)) return HBF_ENOWORKSPACE;
  return status_of(launch_moe(*moe, x, x_stride, tokens, ids, weights, y, y_stride, status, ws, (hipStream_t)stream));
}

}  // extern "C"
