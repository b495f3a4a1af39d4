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

int check_attention(const hbf_kv_layer *kv, const hbf_attention *at) {
  if (!kv || !at) return HBF_EINVAL;
  if (!dtype_ok(kv->dtype) || (kv->head_dim != 64 && kv->head_dim != 128) || kv->kv_heads < 1 ||
      kv->kv_heads > 1024 || kv->pages < 1 || kv->pages > KV_MAX_PAGES || kv->page_tokens < 1 ||
      kv->page_tokens > 65536)
    return HBF_EINVAL;
  if (kv->page_stride < 0 || kv->token_stride < 0 || kv->head_stride < 0 || kv->page_stride % 8 ||
      kv->token_stride % 8 || kv->head_stride % 8)
    return HBF_EINVAL;
  if (at->rows < 0 || at->rows > 65535 || at->heads < kv->kv_heads || at->heads > 1024 ||
      at->heads % kv->kv_heads || (int64_t)at->rows * at->heads > 1 << 22)
    return HBF_EINVAL;
  if (!isfinite(at->scale)) return HBF_EINVAL;
  if (at->prefix_len < 0 || at->prefix_len > INT32_MAX || at->max_own < 0) return HBF_EINVAL;
  if (at->q_row_stride % 8 || at->q_head_stride % 8 || at->out_row_stride % 8 || at->out_head_stride % 8)
    return HBF_EINVAL;
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
