// Declarations shared by the decode-layer operators (hbf_kv.hip, hbf_attn.hip,
// hbf_chunk.hip, hbf_evict.hip, hbf_rotate.hip, hbf_moe.hip) and their host side (hbf_ops_api.cpp).
#pragma once

#include <hip/hip_runtime.h>

#include "hbf.h"

namespace hbf {

constexpr uint32_t KV_ERR_ARG = 1, KV_ERR_PAGES = 2;
constexpr int KV_MAX_LIST = 65535;
constexpr int KV_MAX_PAGES = 1 << 20;
constexpr int KV_MAX_SLOTS = 1 << 18;

// The head of a cache's workspace: zero before the first call.
struct KvCtl {
  uint32_t sticky;   // KV_ERR_* since the last hbf_kv_get_status
  uint32_t arrived;  // workgroups of a plan that are done; 0 between calls
  uint32_t err;      // KV_ERR_* of the call under way; 0 between calls
  uint32_t pad;
  // what the plan found, for the launches that follow it
  uint32_t go;       // the call may change things
  uint32_t total;    // pages to take, or to move
  uint32_t live;     // pages in use (compact)
};

size_t kv_ws_bytes(int pages, int max_list);
hipError_t launch_kv_extend(const hbf_kv &kv, const int32_t *slots, const int32_t *add, int n, int ws_list,
                            hipStream_t s);
hipError_t launch_kv_fork(const hbf_kv &kv, const int32_t *parents, const int32_t *children, int n, int ws_list,
                          hipStream_t s);
hipError_t launch_kv_free(const hbf_kv &kv, const int32_t *slots, int n, hipStream_t s);
hipError_t launch_kv_copy(const hbf_kv &kv, const int32_t *src, const int32_t *dst, int n, hipStream_t s);
hipError_t launch_kv_compact(const hbf_kv &kv, int32_t *remap, int32_t *tables_out, int32_t *refs_out, hipStream_t s);
hipError_t launch_kv_write(const hbf_kv &kv, int layer0, int layers, const void *k, const void *v,
                           const int32_t *slots, const int32_t *pos, int n, hipStream_t s);

constexpr int ATTN_CTL_WORDS = 64;
size_t attn_ws_bytes(const hbf_kv_layer &kv, const hbf_attention &at);
hipError_t launch_attn(const hbf_kv_layer &kv, const hbf_attention &at, int32_t *status, void *ws, hipStream_t s);

hipError_t launch_kv_write_rotated(const hbf_kv &kv, int layer, const hbf_new_tokens &nt, hipStream_t s);
size_t chunk_ws_bytes(const hbf_kv &kv, const hbf_kv_layer &layer, const hbf_chunk &ch);
hipError_t launch_chunk(const hbf_kv &kv, const hbf_kv_layer &layer, const hbf_chunk &ch, int32_t *status, void *ws,
                        hipStream_t s);
hipError_t launch_kv_evict(const hbf_kv &kv, const hbf_eviction &ev, hipStream_t s);

constexpr int MOE_MAX_TOKENS = 128, MOE_MAX_TOPK = 32, MOE_MAX_EXPERTS = 1024, MOE_MAX_PAIRS = 2048;
size_t moe_ws_bytes(const hbf_moe &m, int tokens);
hipError_t launch_moe(const hbf_moe &m, const void *x, int64_t xs, int tokens, int32_t *ids, float *weights, void *y,
                      int64_t ys, int32_t *status, void *ws, hipStream_t s);

}  // namespace hbf
