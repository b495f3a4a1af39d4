// The pages of a KV cache between decode steps: growing, forking, freeing,
// copying and compacting sequences, and writing tokens.
//
// Nothing here is arithmetic: a call moves the bytes of whole tokens or pages
// and the whole numbers of the tables.  A call that takes or moves pages first
// checks every entry and counts the free pages, and changes something only if
// all of it can be done.  Then each free page's rank, from counts of those
// before it, gives the entry it serves, by a search in the entries' offsets: the
// k-th free page, in page order, serves the k-th need, in list order, whatever
// runs first.
//
// Small calls (SMALL_PAGES, SMALL_ENTRIES) are bound by latency, and one
// workgroup does all of that in one launch (a fork of 8 sequences 8 us, growing
// them 4.5).  Bytes move at 4.7 TB/s, read and written (258 MB in 110 us).  In larger ones many workgroups check
// and count, the last of them to finish turns the counts into offsets and
// decides, and another launch applies.
#include "hbf_half.h"
#include "hbf_kv_rows.h"
#include "hbf_ops.h"

namespace hbf {
namespace {

constexpr int THREADS = 256;
constexpr int ONE = 1024;                         // threads of a workgroup that does a call by itself
constexpr int PER_THREAD = 16;
constexpr int TILE = THREADS * PER_THREAD;        // pages per workgroup in large calls
constexpr int MAX_TILES = KV_MAX_PAGES / TILE;
static_assert(MAX_TILES <= THREADS, "one thread per tile in the plan's end");
constexpr int SMALL_PAGES = ONE * PER_THREAD;
constexpr int SMALL_ENTRIES = 1 << 16;            // table entries that the call can touch
constexpr int SMALL_LIST = 1024;
constexpr int ROW = 16;                           // threads per table row there: many rows' latencies side by side
constexpr uint64_t SMALL_COPY = 256 << 10;        // bytes of pages that one workgroup copies sooner than a launch does
constexpr int COPY_BYTES = 16384;                 // bytes a workgroup copies at a time
constexpr int MOVE_GROUPS = 2048;

struct KvWs {
  KvCtl *ctl;
  uint32_t *tile_cnt, *tile_off;   // [MAX_TILES]
  uint32_t *need_off;              // [list + 1] pages needed by the entries before
  int32_t *at;                     // [list] extend: pages held before; fork: the child's own page
  int32_t *len;                    // [list] fork: the parent's tokens
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
  w->len = (int32_t *)take((size_t)list * 4);
  return o;
}

// This workgroup's part of the plan is done (its errors in `err`, which may
// differ by thread).  True in every thread of the last workgroup to get here,
// which then sees what all of them wrote.
__device__ bool plan_done(KvCtl *ctl, uint32_t err) {
  __shared__ uint32_t last;
  if (err) atomicOr(&ctl->err, err);
  stores_done();  // (of every wave: the barrier waits for no memory, the fence below for its own wave's)
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
  const uint32_t before = block_scan<THREADS>(c, &total, scan_lds);
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

// refs of this thread's PT pages from p0 on; those behind the last page read as `past`.
template <int PT>
__device__ __forceinline__ void load_refs(const hbf_kv &kv, int p0, int32_t past, int32_t (&r)[PT]) {
#pragma unroll
  for (int i = 0; i < PT; i++) r[i] = p0 + i < kv.pages ? kv.dev_refs[p0 + i] : past;
}

// By nt threads (a workgroup, or one wave of it).
__device__ __forceinline__ void copy_bytes(char *dst, const char *src, int64_t bytes, int nt) {
  constexpr int U = COPY_BYTES / (THREADS * 16);
  const int step = nt * 16;
  int64_t o = (int64_t)(threadIdx.x & (nt - 1)) * 16;
  for (; o + (U - 1) * step < bytes; o += U * step) {
    u32x4 v[U];
#pragma unroll
    for (int u = 0; u < U; u++) v[u] = *(const u32x4 *)(src + o + u * step);
#pragma unroll
    for (int u = 0; u < U; u++) *(u32x4 *)(dst + o + u * step) = v[u];
  }
  for (; o < bytes; o += step) *(u32x4 *)(dst + o) = *(const u32x4 *)(src + o);
}

// ------------------------------------------------------------ extend and fork

// What a list's check leaves of it: entry i changes row slot[i]; a fork's
// parent is from[i], its length len[i]; extend's held[i] pages come before
// those it gets, and part[i], if not -1, is a part-full page that must be its own
// (null: checked already); off[i] pages are needed by the entries before i.
struct List {
  int32_t *slot, *from, *len;
  int32_t *held, *part;
  uint32_t *off;
};

// Checks the list (`seen`: a bit per slot, in LDS) and fills `out` (whose
// pointers may be LDS; null ones are left out); the errors this thread met.
template <bool FORK, int N>
__device__ uint32_t check_list(const hbf_kv &kv, const List &out, const int32_t *first, const int32_t *second, int n,
                               uint32_t *seen, uint32_t *lds) {
  const int t = threadIdx.x;
  uint32_t err = 0;
  for (int i = t; i < (kv.slots + 31) / 32; i += N) seen[i] = 0;
  __syncthreads();
  uint64_t sum = 0;
  for (int i0 = 0; i0 < n; i0 += N) {
    const int i = i0 + t;
    uint32_t need = 0;
    if (i < n) {
      int part = -1;
      const int a = first[i], b = second[i];
      const int slot = FORK ? b : a;  // the one whose row changes
      int len = 0, held = 0;
      bool ok = slot >= 0 && slot < kv.slots;
      if (ok) ok = !(atomicOr(&seen[slot >> 5], 1u << (slot & 31)) >> (slot & 31) & 1);
      if (ok && FORK) {
        ok = a >= 0 && a < kv.slots;
        if (ok) {
          len = kv.dev_lens[a];
          ok = kv.dev_lens[slot] == 0 && len_fits(kv, len);
          need = ok && len % kv.page_tokens != 0;
        }
      } else if (ok) {
        len = kv.dev_lens[slot];
        const int64_t grown = (int64_t)len + b;
        ok = len_fits(kv, len) && b >= 0 && grown <= (int64_t)kv.table_cols * kv.page_tokens;
        if (ok) {
          held = pages_of(len, kv.page_tokens);
          need = pages_of((int)grown, kv.page_tokens) - held;
          if (b > 0 && len % kv.page_tokens != 0) {
            part = row_of(kv, kv.dev_tables, slot)[held - 1];
            ok = part >= 0 && part < kv.pages && (out.part || kv.dev_refs[part] == 1);
          }
        }
      }
      if (!ok) {
        err |= KV_ERR_ARG;
        need = 0;
        len = 0;
        part = -1;
      }
      if (out.slot) out.slot[i] = slot;
      if (out.from) out.from[i] = a;
      if (out.len) out.len[i] = len;
      if (out.held) out.held[i] = held;
      if (out.part) out.part[i] = part;
      // (a need past every page is refused below; clamped, the sums stay in range)
      if (need > KV_MAX_PAGES) need = KV_MAX_PAGES + 1;
    }
    uint32_t total;
    const uint32_t before = block_scan<N>(need, &total, lds);
    if (i < n) out.off[i] = (uint32_t)sum + before;
    sum += total;
    if (sum > KV_MAX_PAGES) {
      err |= KV_ERR_PAGES;
      sum = KV_MAX_PAGES + 1;
    }
  }
  if (t == 0) out.off[n] = (uint32_t)sum;
  if (FORK)  // a parent's row must not change under those that read it
    for (int i = t; i < n; i += N) {
      const int from = first[i];
      if (from >= 0 && from < kv.slots && (seen[from >> 5] >> (from & 31) & 1)) err |= KV_ERR_ARG;
    }
  return err;
}

// A fork's parent's row of `len` tokens, by threads t of nt; used(p): page p has holders.
template <typename F>
__device__ uint32_t check_row(const hbf_kv &kv, int from, int len, int t, int nt, F used) {
  uint32_t err = 0;
  const int held = pages_of(len, kv.page_tokens);
  if (held == 0) return 0;
  const int32_t *row = row_of(kv, kv.dev_tables, from);
#pragma unroll 4
  for (int c = t; c < held; c += nt) {
    const int p = row[c];
    if (p < 0 || p >= kv.pages || !used(p)) err = KV_ERR_ARG;
  }
  return err;
}

// The free pages of this thread's (refs r), `at` of the workgroup's before them,
// to the workgroup's list in LDS.
template <int PT>
__device__ __forceinline__ void list_free(const int32_t (&r)[PT], uint32_t at, uint16_t *pages) {
#pragma unroll
  for (int i = 0; i < PT; i++)
    if (r[i] == 0) pages[at++] = (uint16_t)(threadIdx.x * PT + i);
}
// The workgroup's `total` free pages, from p0 on, the first of them of rank
// `rank`, go to the entries that need them.  FORK: taken[i] receives the child's
// page.
template <bool FORK, int N>
__device__ void give_pages(const hbf_kv &kv, const List &list, int n, int p0, uint32_t total, uint32_t rank,
                           uint32_t need, const uint16_t *pages, int32_t *taken) {
  for (uint32_t k = threadIdx.x; k < total && rank + k < need; k += N) {
    const uint32_t mine = rank + k;
    int lo = 0, hi = n;  // the last entry whose offset is at most the rank
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (list.off[mid] <= mine) lo = mid; else hi = mid;
    }
    const int page = p0 + pages[k];
    const int col = FORK ? list.len[lo] / kv.page_tokens : list.held[lo] + (int)(mine - list.off[lo]);
    row_of(kv, kv.dev_tables, list.slot[lo])[col] = page;
    kv.dev_refs[page] = 1;
    if (FORK) taken[lo] = page;
  }
}

// A fork's child gets its parent's full pages; by threads t of nt.
__device__ void share_row(const hbf_kv &kv, int from, int len, int to, int t, int nt) {
  const int full = len / kv.page_tokens;
  const int32_t *src = row_of(kv, kv.dev_tables, from);
  int32_t *dst = row_of(kv, kv.dev_tables, to);
#pragma unroll 4
  for (int c = t; c < full; c += nt) {
    const int p = src[c];
    dst[c] = p;
    atomicAdd(&kv.dev_refs[p], 1);  // (never zero here: no free page is taken for used or the other way)
  }
  if (t == 0) kv.dev_lens[to] = len;
}

// The tokens of a fork's part-full pages, in one plane.
__device__ __forceinline__ void copy_part(const hbf_kv &kv, int plane, int src, int dst, int len, int nt) {
  char *base = (char *)kv.dev_pool + (uint64_t)plane * kv.plane_stride;
  copy_bytes(base + (uint64_t)dst * kv.page_stride, base + (uint64_t)src * kv.page_stride,
             (int64_t)(len % kv.page_tokens) * kv.token_bytes, nt);
}

// PT pages per thread.  copy: fork's rows and part-full pages too; else
// k_kv_fork_copy's many workgroups do both.
template <bool FORK, int PT>
__global__ __launch_bounds__(ONE) void k_kv_one(hbf_kv kv, KvWs w, const int32_t *first, const int32_t *second, int n,
                                                bool copy) {
  extern __shared__ uint32_t seen[];
  __shared__ uint16_t pages[ONE * PT];
  __shared__ int32_t slot[SMALL_LIST], from[SMALL_LIST], len[SMALL_LIST], held[SMALL_LIST];
  __shared__ uint32_t off[SMALL_LIST + 1], lds[ONE / 64], errs;
  // a bit per page: has holders (fork), has one (extend); counts are looked up here, not in memory once more
  __shared__ uint16_t held_by[ONE];
  static_assert(PT <= 16, "bits of a word");
  const List list = {slot, FORK ? from : nullptr, len, held, FORK ? nullptr : from, off};
  const int t = threadIdx.x;
  int32_t r[PT];
  load_refs(kv, t * PT, 1, r);
  if (t == 0) errs = 0;
  uint32_t err = check_list<FORK, ONE>(kv, list, first, second, n, seen, lds);
  uint32_t c = 0, free_pages, bits = 0;
#pragma unroll
  for (int i = 0; i < PT; i++) {
    c += r[i] == 0;
    bits |= (uint32_t)(FORK ? r[i] > 0 : r[i] == 1) << i;
  }
  held_by[t] = (uint16_t)bits;
  const uint32_t before = block_scan<ONE>(c, &free_pages, lds);
  auto has = [&](int p) { return held_by[p / PT] >> (p % PT) & 1; };
  list_free(r, before, pages);
  if (FORK) {
    for (int i = t / ROW; i < n; i += ONE / ROW) err |= check_row(kv, from[i], len[i], t % ROW, ROW, has);
  } else {
    for (int i = t; i < n; i += ONE)
      if (list.part[i] >= 0 && !has(list.part[i])) err |= KV_ERR_ARG;
  }
  if (err) atomicOr(&errs, err);
  __syncthreads();
  const uint32_t need = off[n];
  const bool bad = errs & KV_ERR_ARG, full = errs & KV_ERR_PAGES || need > free_pages;
  if (t == 0) {
    w.ctl->go = !bad && !full;
    if (bad || full) w.ctl->sticky |= bad ? KV_ERR_ARG : KV_ERR_PAGES;
  }
  if (bad || full) return;
  // (the pages that the children get: `held`, which fork has no other use for)
  give_pages<FORK, ONE>(kv, list, n, 0, free_pages, 0, need, pages, held);
  if (!FORK) {
    for (int i = t; i < n; i += ONE) kv.dev_lens[slot[i]] = len[i] + second[i];
    return;
  }
  if (copy) {
    for (int i = t / ROW; i < n; i += ONE / ROW) share_row(kv, from[i], len[i], slot[i], t % ROW, ROW);
    __syncthreads();
    for (int i = t >> 6; i < n * kv.planes; i += ONE / 64) {  // a wave each
      const int e = i / kv.planes;
      if (off[e + 1] != off[e])
        copy_part(kv, i - e * kv.planes, row_of(kv, kv.dev_tables, from[e])[len[e] / kv.page_tokens], held[e], len[e],
                  64);
    }
  } else {
    __syncthreads();
    for (int i = t; i < n; i += ONE) {
      w.len[i] = len[i];
      w.at[i] = held[i];
      w.need_off[i] = off[i];
    }
    if (t == 0) w.need_off[n] = need;
  }
}

// The list as the launches of a large call hand it on.
template <bool FORK>
__device__ List list_of(const KvWs &w) {
  return List{nullptr, nullptr, FORK ? w.len : nullptr, FORK ? nullptr : w.at, nullptr, w.need_off};
}

// Large calls.  Workgroups 0 .. tiles-1 count their tile's free pages; the next
// one checks the list and sums its needs; fork's others check one parent's row
// each.
template <bool FORK>
__global__ __launch_bounds__(THREADS) void k_kv_plan(hbf_kv kv, KvWs w, const int32_t *first, const int32_t *second,
                                                     int n, int tiles) {
  extern __shared__ uint32_t seen[];  // a bit per slot
  __shared__ uint32_t lds[THREADS / 64];
  const int b = blockIdx.x, t = threadIdx.x;
  uint32_t err = 0;
  if (b < tiles) {
    int32_t r[PER_THREAD];
    load_refs(kv, b * TILE + t * PER_THREAD, 1, r);
    uint32_t c = 0, total;
#pragma unroll
    for (int i = 0; i < PER_THREAD; i++) c += r[i] == 0;
    block_scan<THREADS>(c, &total, lds);
    if (t == 0) w.tile_cnt[b] = total;
  } else if (b == tiles) {
    err = check_list<FORK, THREADS>(kv, list_of<FORK>(w), first, second, n, seen, lds);
  } else {
    const int from = first[b - tiles - 1];
    if (from >= 0 && from < kv.slots) {  // (the list's check has the others)
      const int len = kv.dev_lens[from];
      if (len_fits(kv, len)) err = check_row(kv, from, len, t, THREADS, [&](int p) { return kv.dev_refs[p] > 0; });
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
  __shared__ uint16_t pages[TILE];
  __shared__ uint32_t lds[THREADS / 64];
  if (!w.ctl->go) return;
  const int b = blockIdx.x, t = threadIdx.x;
  if (b < tiles) {
    const uint32_t need = w.ctl->total, rank = w.tile_off[b];
    if (rank >= need) return;
    int32_t r[PER_THREAD];
    load_refs(kv, b * TILE + t * PER_THREAD, 1, r);
    List list = list_of<FORK>(w);
    list.slot = (int32_t *)(FORK ? second : first);
    uint32_t c = 0, total;
#pragma unroll
    for (int i = 0; i < PER_THREAD; i++) c += r[i] == 0;
    list_free(r, block_scan<THREADS>(c, &total, lds), pages);
    __syncthreads();
    give_pages<FORK, THREADS>(kv, list, n, b * TILE, total, rank, need, pages, w.at);
  } else if (FORK) {
    share_row(kv, first[b - tiles], w.len[b - tiles], second[b - tiles], t, THREADS);
  } else {
    const int i = (b - tiles) * THREADS + t;
    if (i < n) kv.dev_lens[first[i]] += second[i];
  }
}

// The part-full pages of a fork: a plane of one child per workgroup.  The first
// plane's shares the row too, if `children` says whose.
__global__ __launch_bounds__(THREADS) void k_kv_fork_copy(hbf_kv kv, KvWs w, const int32_t *parents,
                                                          const int32_t *children) {
  if (!w.ctl->go) return;
  const int i = blockIdx.y;
  if (children && blockIdx.x == 0) share_row(kv, parents[i], w.len[i], children[i], threadIdx.x, THREADS);
  if (w.need_off[i + 1] == w.need_off[i]) return;
  const int len = w.len[i];
  copy_part(kv, blockIdx.x, row_of(kv, kv.dev_tables, parents[i])[len / kv.page_tokens], w.at[i], len, THREADS);
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
    copy_bytes(base + dst[i] * kv.page_stride, base + src[i] * kv.page_stride, left < COPY_BYTES ? left : COPY_BYTES, THREADS);
  }
}

__global__ __launch_bounds__(THREADS) void k_kv_copy(hbf_kv kv, KvCtl *ctl, const int32_t *src, const int32_t *dst) {
  if (ctl->go) move_pages(kv, src, dst, ctl->total);
}

// ------------------------------------------------------------ compact

// The rows' entries, N threads a row, by group `group` of `groups`.
template <int N>
__device__ uint32_t check_rows(const hbf_kv &kv, int group, int groups) {
  uint32_t err = 0;
  for (int slot = group; slot < kv.slots; slot += groups) {
    const int len = kv.dev_lens[slot];
    if (!len_fits(kv, len)) {
      err = KV_ERR_ARG;
      continue;
    }
    const int32_t *row = row_of(kv, kv.dev_tables, slot);
    const int held = pages_of(len, kv.page_tokens);
#pragma unroll 4
    for (int c = threadIdx.x % N; c < held; c += N) {
      const int p = row[c];
      if (p < 0 || p >= kv.pages || kv.dev_refs[p] <= 0) err = KV_ERR_ARG;
    }
  }
  return err;
}

// Number this thread's pages from p0 on (refs r, `before` of them in use before
// these): those that stay, those that move and the places they move to.  The
// first `live` pages will be in use; `stay` of the pages in use lie there.
template <int PT>
__device__ void number_pages(const hbf_kv &kv, const KvWs &w, int p0, const int32_t (&r)[PT], int before, int live,
                             int stay, int32_t *remap, int32_t *refs_out) {
#pragma unroll
  for (int i = 0; i < PT; i++) {
    const int p = p0 + i;
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

template <int PT>
__global__ __launch_bounds__(ONE) void k_kv_pack_one(hbf_kv kv, KvWs w, int32_t *remap, int32_t *refs_out) {
  __shared__ uint32_t lds[ONE / 64];
  const int t = threadIdx.x;
  int32_t r[PT];
  load_refs(kv, t * PT, 0, r);
  uint32_t err = check_rows<ROW>(kv, t / ROW, ONE / ROW), c = 0, live, stay;
#pragma unroll
  for (int i = 0; i < PT; i++) {
    c += r[i] > 0;
    if (r[i] < 0) err = KV_ERR_ARG;
  }
  const int before = (int)block_scan<ONE>(c, &live, lds);
  c = 0;
#pragma unroll
  for (int i = 0; i < PT; i++) c += r[i] > 0 && t * PT + i < (int)live;
  block_scan<ONE>(c, &stay, lds);
  const bool bad = __syncthreads_or(err);
  if (t == 0) {
    w.ctl->go = !bad;
    w.ctl->total = live - stay;
    if (bad) w.ctl->sticky |= KV_ERR_ARG;
  }
  if (!bad) number_pages(kv, w, t * PT, r, before, (int)live, (int)stay, remap, refs_out);
}

// Workgroups 0 .. tiles-1 count their tile's pages in use; the others check
// the rows, a wave each.
__global__ __launch_bounds__(THREADS) void k_kv_pack_plan(hbf_kv kv, KvWs w, int tiles) {
  __shared__ uint32_t lds[THREADS / 64];
  const int b = blockIdx.x, t = threadIdx.x;
  uint32_t err = 0;
  int32_t r[PER_THREAD];
  if (b < tiles) {
    load_refs(kv, b * TILE + t * PER_THREAD, 0, r);
    uint32_t c = 0, total;
#pragma unroll
    for (int i = 0; i < PER_THREAD; i++) {
      c += r[i] > 0;
      if (r[i] < 0) err = KV_ERR_ARG;
    }
    block_scan<THREADS>(c, &total, lds);
    if (t == 0) w.tile_cnt[b] = total;
  } else {
    err = check_rows<64>(kv, (b - tiles) * (THREADS / 64) + (t >> 6), (gridDim.x - tiles) * (THREADS / 64));
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
    load_refs(kv, tl * TILE + t * PER_THREAD, 0, r);
    uint32_t c = 0, total;
#pragma unroll
    for (int i = 0; i < PER_THREAD; i++) c += r[i] > 0 && tl * TILE + t * PER_THREAD + i < (int)live;
    block_scan<THREADS>(c, &total, lds);
    stay = w.tile_off[tl] + total;
  }
  plan_publish(w.ctl, err, live - stay, live);
}

__global__ __launch_bounds__(THREADS) void k_kv_pack_number(hbf_kv kv, KvWs w, int32_t *remap, int32_t *refs_out) {
  __shared__ uint32_t lds[THREADS / 64];
  if (!w.ctl->go) return;
  const int live = (int)w.ctl->live, p0 = blockIdx.x * TILE + threadIdx.x * PER_THREAD;
  int32_t r[PER_THREAD];
  load_refs(kv, p0, 0, r);
  uint32_t c = 0, total;
#pragma unroll
  for (int i = 0; i < PER_THREAD; i++) c += r[i] > 0;
  const int before = (int)(w.tile_off[blockIdx.x] + block_scan<THREADS>(c, &total, lds));
  number_pages(kv, w, p0, r, before, live, live - (int)w.ctl->total, remap, refs_out);
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
                      bool *shared, bool *copy /* done */, hipStream_t s) {
  const int tiles = tiles_of(kv.pages);
  const size_t lds = (size_t)((kv.slots + 31) / 32) * 4;
  if (kv.pages <= SMALL_PAGES && kv.slots <= SMALL_ENTRIES && n <= SMALL_LIST &&
      (!FORK || (int64_t)n * kv.table_cols <= SMALL_ENTRIES)) {
    *shared = *copy = FORK && (uint64_t)n * kv.planes * kv.page_tokens * kv.token_bytes <= SMALL_COPY;
    if (kv.pages <= ONE * 4)
      k_kv_one<FORK, 4><<<1, ONE, lds, s>>>(kv, w, first, second, n, *copy);
    else
      k_kv_one<FORK, PER_THREAD><<<1, ONE, lds, s>>>(kv, w, first, second, n, *copy);
    return hipGetLastError();
  }
  *copy = false;
  *shared = true;
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
  bool shared, copied;
  return plan_apply<false>(kv, w, slots, add, n, &shared, &copied, s);
}

hipError_t launch_kv_fork(const hbf_kv &kv, const int32_t *parents, const int32_t *children, int n, int ws_list,
                          hipStream_t s) {
  KvWs w;
  carve(kv.dev_ws, kv.pages, ws_list, &w);
  bool shared, copied;
  const hipError_t e = plan_apply<true>(kv, w, parents, children, n, &shared, &copied, s);
  if (e != hipSuccess || copied) return e;
  k_kv_fork_copy<<<dim3(kv.planes, n), THREADS, 0, s>>>(kv, w, parents, shared ? nullptr : children);
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
  if (lds + (int)sizeof(uint32_t) > 65536) {  // (and the word beside the bits)
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
  if (kv.pages <= SMALL_PAGES && (int64_t)kv.slots * kv.table_cols <= SMALL_ENTRIES) {
    if (kv.pages <= ONE * 4)
      k_kv_pack_one<4><<<1, ONE, 0, s>>>(kv, w, remap, refs_out);
    else
      k_kv_pack_one<PER_THREAD><<<1, ONE, 0, s>>>(kv, w, remap, refs_out);
  } else {
    const int rows = (kv.slots + THREADS / 64 - 1) / (THREADS / 64);
    k_kv_pack_plan<<<tiles + rows, THREADS, 0, s>>>(kv, w, tiles);
    k_kv_pack_number<<<tiles, THREADS, 0, s>>>(kv, w, remap, refs_out);
  }
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
