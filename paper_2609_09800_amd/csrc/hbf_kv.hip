// The pages of a KV cache between decode steps: growing, forking, freeing,
// copying and compacting sequences, and writing tokens.
//
// Nothing here is arithmetic: a call moves the bytes of whole tokens or pages
// and the whole numbers of the tables.  A call that takes or moves pages is
// two or three launches.  The plan checks every entry and counts the free
// pages by tiles of refs; its last workgroup turns the tiles' counts into
// offsets and decides whether the call goes ahead, so that a refused call has
// changed nothing.  The launches after it find each free page's rank from its
// tile's offset, and the entry that the rank belongs to by a search in the
// entries' offsets: the k-th free page, in page order, serves the k-th need, in
// list order, whatever runs first.
#include "hbf_half.h"
#include "hbf_ops.h"

namespace hbf {
namespace {

constexpr int THREADS = 256;
constexpr int PER_THREAD = 16;
constexpr int TILE = THREADS * PER_THREAD;        // pages per tile
constexpr int MAX_TILES = KV_MAX_PAGES / TILE;
static_assert(MAX_TILES <= THREADS, "one thread per tile in the plan's end");
constexpr int COPY_BYTES = 16384;                 // bytes a workgroup copies at a time
constexpr int MOVE_GROUPS = 2048;

struct KvWs {
  KvCtl *ctl;
  uint32_t *tile_cnt, *tile_off;   // [MAX_TILES]
  uint32_t *need_off;              // [list + 1] pages needed by the entries before
  int32_t *at;                     // [list] extend: pages held before; fork: the child's own page
  int32_t *code, *movers, *holes;  // [pages] compact
};

size_t up256(size_t x) { return (x + 255) & ~size_t(255); }

size_t carve(void *base, int pages, int list, KvWs *w) {
  char *p = (char *)base;
  size_t o = 256;
  auto take = [&](size_t bytes) {
    char *r = p + o;
    o = up256(o + bytes);
    return (void *)r;
  };
  w->ctl = (KvCtl *)p;
  w->tile_cnt = (uint32_t *)take(MAX_TILES * 4);
  w->tile_off = (uint32_t *)take(MAX_TILES * 4);
  w->code = (int32_t *)take((size_t)pages * 4);
  w->movers = (int32_t *)take((size_t)pages * 4);
  w->holes = (int32_t *)take((size_t)pages * 4);
  w->need_off = (uint32_t *)take(((size_t)list + 1) * 4);
  w->at = (int32_t *)take((size_t)list * 4);
  return o;
}

__device__ __forceinline__ int pages_of(int len, int page_tokens) {
  return (int)(((uint32_t)len + (uint32_t)page_tokens - 1) / (uint32_t)page_tokens);
}
__device__ __forceinline__ bool len_fits(const hbf_kv &kv, int len) {
  return len >= 0 && (int64_t)len <= (int64_t)kv.table_cols * kv.page_tokens;
}
__device__ __forceinline__ int32_t *row_of(const hbf_kv &kv, int32_t *tables, int slot) {
  return tables + (int64_t)slot * kv.table_stride;
}

// Exclusive prefix sum over the workgroup; *total: the sum.
__device__ uint32_t block_scan(uint32_t v, uint32_t *total, uint32_t *lds /* [THREADS / 64] */) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  uint32_t x = v;
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  if (lane == 63) lds[w] = x;
  __syncthreads();
  uint32_t before = 0, sum = 0;
  for (int i = 0; i < THREADS / 64; i++) {
    const uint32_t y = lds[i];
    if (i < w) before += y;
    sum += y;
  }
  __syncthreads();
  *total = sum;
  return before + x - v;
}

// This workgroup's part of the plan is done (its errors in `err`, which may
// differ by thread).  True in every thread of the last workgroup to get here,
// which then sees what all of them wrote.
__device__ bool plan_done(KvCtl *ctl, uint32_t err) {
  __shared__ uint32_t last;
  if (err) atomicOr(&ctl->err, err);
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    last = atomicAdd(&ctl->arrived, 1) + 1 == gridDim.x;
    __threadfence();
  }
  __syncthreads();
  return last != 0;
}

// The last workgroup's end of a plan: tile offsets, and the words for the
// launches that follow.
__device__ void plan_end(const KvWs &w, int tiles, uint32_t *scan_lds, uint32_t *count) {
  const uint32_t c = (int)threadIdx.x < tiles ? w.tile_cnt[threadIdx.x] : 0;
  uint32_t total;
  const uint32_t before = block_scan(c, &total, scan_lds);
  if ((int)threadIdx.x < tiles) w.tile_off[threadIdx.x] = before;
  *count = total;
}
__device__ void plan_publish(KvCtl *ctl, uint32_t err, uint32_t total, uint32_t live) {
  if (threadIdx.x) return;
  ctl->go = err == 0;
  ctl->total = total;
  ctl->live = live;
  ctl->arrived = 0;
  ctl->err = 0;
  if (err) atomicOr(&ctl->sticky, err);
}

// refs of this thread's pages of a tile; pages behind the last read as `past`.
__device__ __forceinline__ void load_refs(const hbf_kv &kv, int tile, int32_t past, int32_t *r) {
  const int p0 = tile * TILE + threadIdx.x * PER_THREAD;
#pragma unroll
  for (int i = 0; i < PER_THREAD; i++) r[i] = p0 + i < kv.pages ? kv.dev_refs[p0 + i] : past;
}

__device__ void copy_bytes(char *dst, const char *src, int64_t bytes) {
  constexpr int STEP = THREADS * 16, U = COPY_BYTES / STEP;
  int64_t o = (int64_t)threadIdx.x * 16;
  for (; o + (U - 1) * STEP < bytes; o += COPY_BYTES) {
    u32x4 v[U];
#pragma unroll
    for (int u = 0; u < U; u++) v[u] = *(const u32x4 *)(src + o + u * STEP);
#pragma unroll
    for (int u = 0; u < U; u++) *(u32x4 *)(dst + o + u * STEP) = v[u];
  }
  for (; o < bytes; o += STEP) *(u32x4 *)(dst + o) = *(const u32x4 *)(src + o);
}

// ------------------------------------------------------------ extend and fork

// Workgroups 0 .. tiles-1 count their tile's free pages; the next one checks
// the list and sums its needs; fork's others check one parent's row each.
template <bool FORK>
__global__ __launch_bounds__(THREADS) void k_kv_plan(hbf_kv kv, KvWs w, const int32_t *first, const int32_t *second,
                                                     int n, int tiles) {
  extern __shared__ uint32_t seen[];  // a bit per slot
  __shared__ uint32_t lds[THREADS / 64];
  const int b = blockIdx.x, t = threadIdx.x;
  uint32_t err = 0;
  if (b < tiles) {
    int32_t r[PER_THREAD];
    load_refs(kv, b, 1, r);
    uint32_t c = 0, total;
#pragma unroll
    for (int i = 0; i < PER_THREAD; i++) c += r[i] == 0;
    block_scan(c, &total, lds);
    if (t == 0) w.tile_cnt[b] = total;
  } else if (b == tiles) {
    for (int i = t; i < (kv.slots + 31) / 32; i += THREADS) seen[i] = 0;
    __syncthreads();
    uint64_t sum = 0;
    for (int i0 = 0; i0 < n; i0 += THREADS) {
      const int i = i0 + t;
      uint32_t need = 0;
      if (i < n) {
        const int slot = FORK ? second[i] : first[i];  // the one whose row changes
        bool ok = slot >= 0 && slot < kv.slots;
        if (ok) ok = !(atomicOr(&seen[slot >> 5], 1u << (slot & 31)) >> (slot & 31) & 1);
        if (ok && FORK) {
          const int from = first[i];
          ok = from >= 0 && from < kv.slots && kv.dev_lens[slot] == 0;
          if (ok) {
            const int len = kv.dev_lens[from];
            ok = len_fits(kv, len);
            need = ok && len % kv.page_tokens != 0;
          }
        } else if (ok) {
          const int len = kv.dev_lens[slot], add = second[i];
          const int64_t grown = (int64_t)len + add;
          ok = len_fits(kv, len) && add >= 0 && grown <= (int64_t)kv.table_cols * kv.page_tokens;
          if (ok) {
            const int held = pages_of(len, kv.page_tokens);
            w.at[i] = held;
            need = pages_of((int)grown, kv.page_tokens) - held;
            if (add > 0 && len % kv.page_tokens != 0) {
              const int p = row_of(kv, kv.dev_tables, slot)[held - 1];
              ok = p >= 0 && p < kv.pages && kv.dev_refs[p] == 1;
            }
          }
        }
        if (!ok) {
          err |= KV_ERR_ARG;
          need = 0;
        }
        // (a need past every page is refused below; clamped, the sums stay in range)
        if (need > KV_MAX_PAGES) need = KV_MAX_PAGES + 1;
      }
      uint32_t total;
      const uint32_t before = block_scan(need, &total, lds);
      if (i < n) w.need_off[i] = (uint32_t)sum + before;
      sum += total;
      if (sum > KV_MAX_PAGES) {
        err |= KV_ERR_PAGES;
        sum = KV_MAX_PAGES + 1;
      }
    }
    if (t == 0) w.need_off[n] = (uint32_t)sum;
    if (FORK)  // a parent's row must not change under those that read it
      for (int i = t; i < n; i += THREADS) {
        const int from = first[i];
        if (from >= 0 && from < kv.slots && (seen[from >> 5] >> (from & 31) & 1)) err |= KV_ERR_ARG;
      }
  } else {
    const int from = first[b - tiles - 1];
    if (from >= 0 && from < kv.slots) {
      const int len = kv.dev_lens[from];
      if (len_fits(kv, len)) {
        const int32_t *row = row_of(kv, kv.dev_tables, from);
        for (int c = t; c < pages_of(len, kv.page_tokens); c += THREADS) {
          const int p = row[c];
          if (p < 0 || p >= kv.pages || kv.dev_refs[p] <= 0) err = KV_ERR_ARG;
        }
      }
    }
  }
  if (!plan_done(w.ctl, err)) return;
  uint32_t free_pages;
  plan_end(w, tiles, lds, &free_pages);
  err = atomicOr(&w.ctl->err, 0);
  __syncthreads();  // every thread has read the word that is cleared now
  const uint32_t need = w.need_off[n];
  if (!(err & KV_ERR_ARG) && need > free_pages) err = KV_ERR_PAGES;
  if (err & KV_ERR_ARG) err = KV_ERR_ARG;
  plan_publish(w.ctl, err, need, 0);
}

template <bool FORK>
__global__ __launch_bounds__(THREADS) void k_kv_apply(hbf_kv kv, KvWs w, const int32_t *first, const int32_t *second,
                                                      int n, int tiles) {
  __shared__ uint32_t lds[THREADS / 64];
  if (!w.ctl->go) return;
  const int b = blockIdx.x, t = threadIdx.x;
  if (b < tiles) {
    const uint32_t need = w.ctl->total;
    uint32_t rank = w.tile_off[b];
    if (rank >= need) return;
    int32_t r[PER_THREAD];
    load_refs(kv, b, 1, r);
    uint32_t c = 0, total;
#pragma unroll
    for (int i = 0; i < PER_THREAD; i++) c += r[i] == 0;
    rank += block_scan(c, &total, lds);
#pragma unroll
    for (int i = 0; i < PER_THREAD; i++) {
      if (r[i] != 0) continue;
      if (rank < need) {
        int lo = 0, hi = n;  // the last entry whose offset is at most rank
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (w.need_off[mid] <= rank) lo = mid; else hi = mid;
        }
        const int page = b * TILE + t * PER_THREAD + i;
        const int slot = FORK ? second[lo] : first[lo];
        const int col = FORK ? kv.dev_lens[first[lo]] / kv.page_tokens : w.at[lo] + (int)(rank - w.need_off[lo]);
        row_of(kv, kv.dev_tables, slot)[col] = page;
        kv.dev_refs[page] = 1;
        if (FORK) w.at[lo] = page;
      }
      rank++;
    }
  } else if (FORK) {
    const int i = b - tiles;
    const int from = first[i], to = second[i];
    const int len = kv.dev_lens[from];
    const int32_t *src = row_of(kv, kv.dev_tables, from);
    int32_t *dst = row_of(kv, kv.dev_tables, to);
    for (int c = t; c < len / kv.page_tokens; c += THREADS) {
      const int p = src[c];
      dst[c] = p;
      atomicAdd(&kv.dev_refs[p], 1);  // (never zero here: no free page is taken for used or the other way)
    }
    if (t == 0) kv.dev_lens[to] = len;
  } else {
    const int i = (b - tiles) * THREADS + t;
    if (i < n) kv.dev_lens[first[i]] += second[i];
  }
}

// The part-full pages of a fork: a plane of one child per workgroup.
__global__ __launch_bounds__(THREADS) void k_kv_fork_copy(hbf_kv kv, KvWs w, const int32_t *parents) {
  if (!w.ctl->go) return;
  const int i = blockIdx.y;
  if (w.need_off[i + 1] == w.need_off[i]) return;
  const int len = kv.dev_lens[parents[i]];
  const int src = row_of(kv, kv.dev_tables, parents[i])[len / kv.page_tokens], dst = w.at[i];
  char *plane = (char *)kv.dev_pool + blockIdx.x * kv.plane_stride;
  copy_bytes(plane + dst * kv.page_stride, plane + src * kv.page_stride,
             (int64_t)(len % kv.page_tokens) * kv.token_bytes);
}

// ------------------------------------------------------------ free

__global__ __launch_bounds__(THREADS) void k_kv_free(hbf_kv kv, KvWs w, const int32_t *slots) {
  __shared__ int held_s;
  const int slot = slots[blockIdx.x];
  uint32_t err = 0;
  if (threadIdx.x == 0) {
    int held = 0;
    if (slot < 0 || slot >= kv.slots) {
      err = KV_ERR_ARG;
    } else {
      const int len = kv.dev_lens[slot];
      if (!len_fits(kv, len)) err = KV_ERR_ARG;
      // whoever of several entries with this slot clears the length frees it
      else if (len > 0 && atomicCAS(&kv.dev_lens[slot], len, 0) == len) held = pages_of(len, kv.page_tokens);
    }
    held_s = held;
  }
  __syncthreads();
  const int held = held_s;
  if (held > 0) {
    int32_t *row = row_of(kv, kv.dev_tables, slot);
    for (int c = threadIdx.x; c < held; c += THREADS) {
      const int p = row[c];
      row[c] = -1;
      if (p < 0 || p >= kv.pages) {
        err = KV_ERR_ARG;
      } else if (atomicSub(&kv.dev_refs[p], 1) <= 0) {  // was free: put back
        atomicAdd(&kv.dev_refs[p], 1);
        err = KV_ERR_ARG;
      }
    }
  }
  if (err) atomicOr(&w.ctl->sticky, err);
}

// ------------------------------------------------------------ copy

__global__ __launch_bounds__(1024) void k_kv_copy_check(hbf_kv kv, KvCtl *ctl, const int32_t *src, const int32_t *dst,
                                                        int n) {
  extern __shared__ uint32_t seen[];  // a bit per page: a destination
  __shared__ uint32_t bad;
  if (threadIdx.x == 0) bad = 0;
  for (int i = threadIdx.x; i < (kv.pages + 31) / 32; i += 1024) seen[i] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += 1024) {
    const int d = dst[i], s = src[i];
    bool ok = d >= 0 && d < kv.pages && s >= 0 && s < kv.pages;
    if (ok) ok = !(atomicOr(&seen[d >> 5], 1u << (d & 31)) >> (d & 31) & 1);
    if (!ok) bad = 1;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += 1024) {
    const int s = src[i];
    if (s >= 0 && s < kv.pages && (seen[s >> 5] >> (s & 31) & 1)) bad = 1;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    ctl->go = !bad;
    ctl->total = n;
    if (bad) atomicOr(&ctl->sticky, KV_ERR_ARG);
  }
}

// Pages src[i] to dst[i], total of them, in every plane; units of COPY_BYTES.
__device__ void move_pages(const hbf_kv &kv, const int32_t *src, const int32_t *dst, uint32_t total) {
  const int64_t bytes = (int64_t)kv.page_tokens * kv.token_bytes;
  const uint32_t parts = (uint32_t)((bytes + COPY_BYTES - 1) / COPY_BYTES);
  const uint64_t per_page = (uint64_t)parts * kv.planes, units = per_page * total;
  for (uint64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const uint32_t i = (uint32_t)(u / per_page), rest = (uint32_t)(u - i * per_page);
    const uint32_t plane = rest / parts, part = rest - plane * parts;
    char *base = (char *)kv.dev_pool + plane * kv.plane_stride + (uint64_t)part * COPY_BYTES;
    const int64_t left = bytes - (int64_t)part * COPY_BYTES;
    copy_bytes(base + dst[i] * kv.page_stride, base + src[i] * kv.page_stride, left < COPY_BYTES ? left : COPY_BYTES);
  }
}

__global__ __launch_bounds__(THREADS) void k_kv_copy(hbf_kv kv, KvCtl *ctl, const int32_t *src, const int32_t *dst) {
  if (ctl->go) move_pages(kv, src, dst, ctl->total);
}

// ------------------------------------------------------------ compact

// Workgroups 0 .. tiles-1 count their tile's pages in use; the others check
// the rows, a wave each.
__global__ __launch_bounds__(THREADS) void k_kv_pack_plan(hbf_kv kv, KvWs w, int tiles) {
  __shared__ uint32_t lds[THREADS / 64];
  const int b = blockIdx.x, t = threadIdx.x;
  uint32_t err = 0;
  int32_t r[PER_THREAD];
  if (b < tiles) {
    load_refs(kv, b, 0, r);
    uint32_t c = 0, total;
#pragma unroll
    for (int i = 0; i < PER_THREAD; i++) {
      c += r[i] > 0;
      if (r[i] < 0) err = KV_ERR_ARG;
    }
    block_scan(c, &total, lds);
    if (t == 0) w.tile_cnt[b] = total;
  } else {
    const int slot = (b - tiles) * (THREADS / 64) + (t >> 6);
    if (slot < kv.slots) {
      const int len = kv.dev_lens[slot];
      if (!len_fits(kv, len)) {
        err = KV_ERR_ARG;
      } else {
        const int32_t *row = row_of(kv, kv.dev_tables, slot);
        for (int c = t & 63; c < pages_of(len, kv.page_tokens); c += 64) {
          const int p = row[c];
          if (p < 0 || p >= kv.pages || kv.dev_refs[p] <= 0) err = KV_ERR_ARG;
        }
      }
    }
  }
  if (!plan_done(w.ctl, err)) return;
  uint32_t live;
  plan_end(w, tiles, lds, &live);
  err = atomicOr(&w.ctl->err, 0);
  __syncthreads();  // (and tile_off is written)
  // pages in use below `live` stay; the rest move
  uint32_t stay = live;
  const int tl = (int)live / TILE;
  if (tl < tiles) {
    load_refs(kv, tl, 0, r);
    uint32_t c = 0, total;
#pragma unroll
    for (int i = 0; i < PER_THREAD; i++) c += r[i] > 0 && tl * TILE + t * PER_THREAD + i < (int)live;
    block_scan(c, &total, lds);
    stay = w.tile_off[tl] + total;
  }
  plan_publish(w.ctl, err, live - stay, live);
}

// Number the pages: those that stay, those that move and the places they move to.
__global__ __launch_bounds__(THREADS) void k_kv_pack_number(hbf_kv kv, KvWs w, int32_t *remap, int32_t *refs_out) {
  __shared__ uint32_t lds[THREADS / 64];
  if (!w.ctl->go) return;
  const int live = (int)w.ctl->live, stay = live - (int)w.ctl->total;
  int32_t r[PER_THREAD];
  load_refs(kv, blockIdx.x, 0, r);
  uint32_t c = 0, total;
#pragma unroll
  for (int i = 0; i < PER_THREAD; i++) c += r[i] > 0;
  int before = (int)(w.tile_off[blockIdx.x] + block_scan(c, &total, lds));
#pragma unroll
  for (int i = 0; i < PER_THREAD; i++) {
    const int p = blockIdx.x * TILE + threadIdx.x * PER_THREAD + i;
    if (p >= kv.pages) break;
    if (r[i] > 0) {
      if (p < live) {
        w.code[p] = p;
        remap[p] = p;
      } else {  // the (before - stay)-th to move
        w.code[p] = ~(before - stay);
        w.movers[before - stay] = p;
      }
      before++;
    } else {
      remap[p] = -1;
      if (p < live) w.holes[p - before] = p;
    }
    if (refs_out != kv.dev_refs) refs_out[p] = r[i];
  }
}

__global__ __launch_bounds__(THREADS) void k_kv_pack_move(hbf_kv kv, KvWs w, int32_t *remap, int32_t *tables_out,
                                                          int32_t *refs_out) {
  if (!w.ctl->go) return;
  const uint32_t total = w.ctl->total;
  const bool same = tables_out == kv.dev_tables;
  constexpr int WAVES = THREADS / 64;
  for (int slot = blockIdx.x * WAVES + (threadIdx.x >> 6); slot < kv.slots; slot += gridDim.x * WAVES) {
    const int held = pages_of(kv.dev_lens[slot], kv.page_tokens);
    const int32_t *row = row_of(kv, kv.dev_tables, slot);
    int32_t *out = row_of(kv, tables_out, slot);
    for (int c = threadIdx.x & 63; c < (same ? held : kv.table_cols); c += 64) {
      int p = row[c];
      if (c < held) {
        const int code = w.code[p];
        p = code < 0 ? w.holes[~code] : code;
      }
      out[c] = p;
    }
  }
  for (uint32_t i = blockIdx.x * THREADS + threadIdx.x; i < total; i += gridDim.x * THREADS) {
    const int s = w.movers[i], d = w.holes[i];
    remap[s] = d;
    refs_out[d] = kv.dev_refs[s];
    refs_out[s] = 0;
  }
  move_pages(kv, w.movers, w.holes, total);
}

// ------------------------------------------------------------ write

// A 16-byte piece of one token in one plane per thread.
__global__ __launch_bounds__(THREADS) void k_kv_write(hbf_kv kv, KvCtl *ctl, int layer0, const char *k, const char *v,
                                                      const int32_t *slots, const int32_t *pos, int n) {
  const uint32_t pieces = (uint32_t)(kv.token_bytes / 16);
  const uint32_t x = blockIdx.x * THREADS + threadIdx.x, i = x / pieces;
  if (i >= (uint32_t)n) return;
  const int plane = blockIdx.y;  // of the call's
  const char *src = (plane & 1 ? v : k) + ((uint64_t)(plane >> 1) * n + i) * kv.token_bytes;
  const u32x4 val = *(const u32x4 *)(src + (x - i * pieces) * 16);
  const int slot = slots[i], at = pos[i];
  if (slot >= 0 && slot < kv.slots) {
    const int len = kv.dev_lens[slot];
    if (len_fits(kv, len) && at >= 0 && at < len) {
      const int page = row_of(kv, kv.dev_tables, slot)[at / kv.page_tokens];
      if (page >= 0 && page < kv.pages) {
        char *dst = (char *)kv.dev_pool + (uint64_t)(2 * layer0 + plane) * kv.plane_stride + page * kv.page_stride +
                    (uint64_t)(at % kv.page_tokens) * kv.token_bytes;
        *(u32x4 *)(dst + (x - i * pieces) * 16) = val;
        return;
      }
    }
  }
  atomicOr(&ctl->sticky, KV_ERR_ARG);
}

int tiles_of(int pages) { return (pages + TILE - 1) / TILE; }

template <bool FORK>
hipError_t plan_apply(const hbf_kv &kv, const KvWs &w, const int32_t *first, const int32_t *second, int n,
                      hipStream_t s) {
  const int tiles = tiles_of(kv.pages);
  const size_t lds = (size_t)((kv.slots + 31) / 32) * 4;
  k_kv_plan<FORK><<<tiles + 1 + (FORK ? n : 0), THREADS, lds, s>>>(kv, w, first, second, n, tiles);
  k_kv_apply<FORK><<<tiles + (FORK ? n : (n + THREADS - 1) / THREADS), THREADS, 0, s>>>(kv, w, first, second, n,
                                                                                        tiles);
  return hipGetLastError();
}

}  // namespace

size_t kv_ws_bytes(int pages, int max_list) {
  KvWs w;
  return carve(nullptr, pages, max_list, &w);
}

hipError_t launch_kv_extend(const hbf_kv &kv, const int32_t *slots, const int32_t *add, int n, int ws_list,
                            hipStream_t s) {
  KvWs w;
  carve(kv.dev_ws, kv.pages, ws_list, &w);
  return plan_apply<false>(kv, w, slots, add, n, s);
}

hipError_t launch_kv_fork(const hbf_kv &kv, const int32_t *parents, const int32_t *children, int n, int ws_list,
                          hipStream_t s) {
  KvWs w;
  carve(kv.dev_ws, kv.pages, ws_list, &w);
  const hipError_t e = plan_apply<true>(kv, w, parents, children, n, s);
  if (e != hipSuccess) return e;
  k_kv_fork_copy<<<dim3(kv.planes, n), THREADS, 0, s>>>(kv, w, parents);
  return hipGetLastError();
}

hipError_t launch_kv_free(const hbf_kv &kv, const int32_t *slots, int n, hipStream_t s) {
  KvWs w;
  carve(kv.dev_ws, kv.pages, 0, &w);
  k_kv_free<<<n, THREADS, 0, s>>>(kv, w, slots);
  return hipGetLastError();
}

hipError_t launch_kv_copy(const hbf_kv &kv, const int32_t *src, const int32_t *dst, int n, hipStream_t s) {
  const int lds = (kv.pages + 31) / 32 * 4;
  if (lds > 65536) {
    const hipError_t e = hipFuncSetAttribute((const void *)k_kv_copy_check,
                                             hipFuncAttributeMaxDynamicSharedMemorySize, KV_MAX_PAGES / 8);
    if (e != hipSuccess) return e;
  }
  KvCtl *ctl = (KvCtl *)kv.dev_ws;
  k_kv_copy_check<<<1, 1024, lds, s>>>(kv, ctl, src, dst, n);
  k_kv_copy<<<MOVE_GROUPS, THREADS, 0, s>>>(kv, ctl, src, dst);
  return hipGetLastError();
}

hipError_t launch_kv_compact(const hbf_kv &kv, int32_t *remap, int32_t *tables_out, int32_t *refs_out,
                             hipStream_t s) {
  KvWs w;
  carve(kv.dev_ws, kv.pages, 0, &w);
  const int tiles = tiles_of(kv.pages);
  k_kv_pack_plan<<<tiles + (kv.slots + THREADS / 64 - 1) / (THREADS / 64), THREADS, 0, s>>>(kv, w, tiles);
  k_kv_pack_number<<<tiles, THREADS, 0, s>>>(kv, w, remap, refs_out);
  k_kv_pack_move<<<MOVE_GROUPS, THREADS, 0, s>>>(kv, w, remap, tables_out, refs_out);
  return hipGetLastError();
}

hipError_t launch_kv_write(const hbf_kv &kv, int layer0, int layers, const void *k, const void *v,
                           const int32_t *slots, const int32_t *pos, int n, hipStream_t s) {
  const uint32_t total = (uint32_t)n * (uint32_t)(kv.token_bytes / 16);
  k_kv_write<<<dim3((total + THREADS - 1) / THREADS, 2 * layers), THREADS, 0, s>>>(
      kv, (KvCtl *)kv.dev_ws, layer0, (const char *)k, (const char *)v, slots, pos, n);
  return hipGetLastError();
}

}  // namespace hbf
