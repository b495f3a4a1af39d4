// Sequences of a cache are cut down to the tokens of the largest weight, layer
// by layer and head by head.
//
// The choice is exact: the keep-th largest weight is found by its bits, eight at
// a time, in the order of a whole number that grows with the float; equal ones
// are taken from the lowest position on.  The chosen tokens that already lie before the
// new end of the middle stay, the others fill the places between them: fewer
// bytes than closing ranks, and no place is both read and written, so that all
// of it runs at once.  The last tokens, which stay in their order, move over
// places that the others are read from, and over their own where fewer leave than
// stay last: in a launch of their own, 32 KiB of a plane a workgroup, or where they
// move over themselves a workgroup a plane, some tokens at a time from the front.
// Launches: the check of every row beside the choice; the middle's moves; the
// last tokens' and the weights behind them; tables, counts and lengths.  (48 layers,
// 8 sequences of 1,100 to 2,200 tokens cut to 1,024, 4 heads of 128: 23 + 132 + 40 + 5 us,
// the moves of single heads' 256 bytes at about 4.5 TB/s; the last 64 tokens' K and V,
// 100 MB in two workgroups a plane, at half of a copy's rate, and beside them the weights,
// which take 9 by themselves; a layer of 4 sequences of 600: 11.6 + 6.5 + 6.3 + 2.5, each a
// few rounds to memory.  The last launch joined to the one before by its last workgroup:
// 219 / 209 us and 34.3 / 33.7.)
#include <algorithm>

#include "hbf_half.h"
#include "hbf_kv_rows.h"
#include "hbf_ops.h"

namespace hbf {
namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64;
constexpr int HOLES = 4096;      // free places listed at a time
constexpr int MOVE_TILE = 512;   // places that a workgroup of the moves looks at

struct Args {
  hbf_kv kv;
  hbf_eviction ev;
  KvCtl *ctl;
  int layers, moves;   // workgroups of the moves per layer, entry and head
  int lasts;           // of the last tokens, per plane and entry
  int64_t head_bytes;
};

// An entry of the list; where it is out of range, ok is false.
struct Entry {
  int slot, len, keep;
  bool ok, cut;
};
__device__ __forceinline__ Entry get_entry(const Args &a, int i) {
  Entry e;
  e.slot = a.ev.dev_slots[i];
  e.keep = a.ev.dev_keep[i];
  e.ok = e.slot >= 0 && e.slot < a.kv.slots;
  e.len = e.ok ? a.kv.dev_lens[e.slot] : 0;
  e.ok = e.ok && len_fits(a.kv, e.len) && e.len <= a.ev.weights_tokens && e.keep >= 0 && e.keep <= a.ev.max_keep;
  e.cut = e.ok && e.keep < e.len;
  if (e.cut && e.keep < (int64_t)a.ev.sinks + a.ev.recent) e.ok = e.cut = false;
  return e;
}
__device__ __forceinline__ int32_t *kept_of(const Args &a, int layer, int i, int head) {
  return a.ev.dev_kept + (((int64_t)layer * a.ev.n + i) * a.ev.kv_heads + head) * a.ev.max_keep;
}
__device__ __forceinline__ int64_t weights_at(const Args &a, int layer, int slot, int head) {
  return layer * a.ev.layer_stride + slot * a.ev.slot_stride + head * a.ev.head_stride;
}
// A whole number that grows with the weight; NaN is the lowest, -0 equals 0.
__device__ __forceinline__ uint32_t key_of(float w) {
  if (w != w) return 0;
  const uint32_t u = __float_as_uint(w + 0.f);
  return u >> 31 ? ~u : u | 0x80000000u;
}

// The k-th largest (k >= 1) of the workgroup's keys, and how many equal ones are
// among the k.  each(f): f(key) for the thread's own.
template <typename F>
__device__ uint32_t kth_key(F each, uint32_t k, uint32_t *equal) {
  __shared__ uint32_t bins[256], found, rest, lds[WAVES];
  static_assert(THREADS == 256, "a bin a thread");
  uint32_t prefix = 0;
#pragma unroll 1
  for (int shift = 24; shift >= 0; shift -= 8) {
    bins[threadIdx.x] = 0;
    __syncthreads();
    each([&](uint32_t key) {
      if (shift == 24 || key >> (shift + 8) == prefix) atomicAdd(&bins[key >> shift & 255], 1u);
    });
    __syncthreads();
    // the bin that holds it, from the highest down: those above have fewer than k, with it at least k
    uint32_t total;
    const uint32_t mine = bins[255 - threadIdx.x], before = block_scan<THREADS>(mine, &total, lds);
    if (before < k && before + mine >= k) {
      found = 255 - threadIdx.x;
      rest = k - before;
    }
    __syncthreads();
    prefix = prefix << 8 | found;
    k = rest;
  }
  *equal = k;
  return prefix;
}

// The choice between s0 and mid, of which m - s0 stay: up to FEW_KEYS weights are
// read once, into registers, 16 neighbours a thread.
constexpr int KEYS = 16, FEW_KEYS = THREADS * KEYS;
__device__ void choose_few(const float *w, int s0, int m, int mid, int32_t *kept) {
  __shared__ uint32_t lds[WAVES];
  __shared__ int32_t holes[FEW_KEYS / 2];  // (as many as movers)
  const int first = s0 + threadIdx.x * KEYS, n = min(max(mid - first, 0), KEYS);
  uint32_t key[KEYS], equal, total;
#pragma unroll
  for (int u = 0; u < KEYS; u++) key[u] = key_of(w[min(first + u, mid - 1)]);
  const uint32_t least = kth_key([&](auto f) {
#pragma unroll
    for (int u = 0; u < KEYS; u++)
      if (u < n) f(key[u]);
  }, (uint32_t)(m - s0), &equal);
  uint32_t ties = 0, in = 0, count = 0;
#pragma unroll
  for (int u = 0; u < KEYS; u++) ties += u < n && key[u] == least;
  uint32_t rank = block_scan<THREADS>(ties, &total, lds);
  // movers before this thread's in the high half, free places in the low one
#pragma unroll
  for (int u = 0; u < KEYS; u++) {
    const bool tie = key[u] == least, chosen = u < n && (key[u] > least || (tie && rank < equal));
    rank += u < n && tie;
    in |= (uint32_t)chosen << u;
    if (u < n) count += first + u < m ? !chosen : (uint32_t)chosen << 16;
  }
  const uint32_t before = block_scan<THREADS>(count, &total, lds);
  uint32_t hole = before & 0xffff, mover = before >> 16;
#pragma unroll
  for (int u = 0; u < KEYS; u++) {
    if (u >= n || first + u >= m) continue;
    if (in >> u & 1) kept[first + u] = first + u;
    else holes[hole++] = first + u;
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < KEYS; u++)
    if (u < n && first + u >= m && (in >> u & 1)) kept[holes[mover++]] = first + u;
}

// The same for any number, read anew by each step.
__device__ void choose_many(const float *w, int s0, int m, int mid, int32_t *kept) {
  const int t = threadIdx.x;
  uint32_t equal;
  const uint32_t least = kth_key([&](auto f) {
    for (int i = s0 + t; i < mid; i += THREADS) f(key_of(w[i]));
  }, (uint32_t)(m - s0), &equal);
  // In position order: those above the least, and the first `equal` of those equal to it.
  __shared__ uint32_t lds[WAVES];
  __shared__ int32_t holes[HOLES];
  constexpr int PT = 4;
  uint32_t left = 1;
  for (uint32_t base = 0; left; base += HOLES) {  // free places base .. base + HOLES - 1
    uint32_t ties = 0, done = 0;  // ties and free places (then movers) before the tile
    auto tiles = [&](int from, int to, bool want, auto each) {
      for (int p0 = from; p0 < to; p0 += THREADS * PT) {
        uint32_t key[PT], eq = 0, total;
#pragma unroll
        for (int u = 0; u < PT; u++) {
          const int p = p0 + t * PT + u;
          key[u] = p < to ? key_of(w[p]) : 0;
          eq += p < to && key[u] == least;
        }
        uint32_t rank = ties + block_scan<THREADS>(eq, &total, lds);
        ties += total;
        uint32_t count = 0, mask = 0;
#pragma unroll
        for (int u = 0; u < PT; u++) {
          const int p = p0 + t * PT + u;
          const bool tie = key[u] == least, in = key[u] > least || (tie && rank < equal);
          if (p < to) {
            rank += tie;
            mask |= (uint32_t)(in == want) << u;
            count += in == want;
            if (!want && in && base == 0) kept[p] = p;
          }
        }
        uint32_t at = done + block_scan<THREADS>(count, &total, lds);
        done += total;
#pragma unroll
        for (int u = 0; u < PT; u++)
          if (mask >> u & 1) each(at++, p0 + t * PT + u);
      }
    };
    tiles(s0, m, false, [&](uint32_t at, int p) {
      if (at - base < HOLES) holes[at - base] = p;
    });
    left = done > base + HOLES;
    done = 0;
    __syncthreads();
    tiles(m, mid, true, [&](uint32_t at, int p) {
      if (at - base < HOLES) kept[holes[at - base]] = p;
    });
    __syncthreads();
  }
}

// One layer's and head's choice for entry i: dev_kept.
__device__ void choose(const Args &a, const Entry &e, int layer, int i, int head) {
  int32_t *kept = kept_of(a, layer, i, head);
  const int end = e.cut ? e.keep : e.len;
  for (int j = threadIdx.x; j < a.ev.max_keep; j += THREADS) {
    if (j >= end) kept[j] = -1;
    else if (!e.cut || j < a.ev.sinks) kept[j] = j;
    else if (j >= e.keep - a.ev.recent) kept[j] = j + (e.len - e.keep);
  }
  const int s0 = a.ev.sinks, m = e.keep - a.ev.recent, mid = e.len - a.ev.recent;
  if (!e.cut || m == s0) return;
  const float *w = a.ev.dev_weights + weights_at(a, layer, e.slot, head);
  if (mid - s0 <= FEW_KEYS) choose_few(w, s0, m, mid, kept);
  else choose_many(w, s0, m, mid, kept);
}

// Workgroups 0 .. n-1 check a row each, the next one that no slot is listed twice;
// the last of them decides.  The others choose.
__global__ __launch_bounds__(THREADS) void k_evict_plan(Args a) {
  extern __shared__ uint32_t seen[];  // a bit per slot
  const int t = threadIdx.x, n = a.ev.n;
  int b = blockIdx.x;
  if (b > n) {
    b -= n + 1;
    const int head = b % a.ev.kv_heads, i = b / a.ev.kv_heads % n, layer = b / a.ev.kv_heads / n;
    const Entry e = get_entry(a, i);
    if (e.ok) choose(a, e, layer, i, head);
    return;
  }
  bool bad = false;
  if (b < n) {
    const Entry e = get_entry(a, b);
    bad = !e.ok;
    if (e.cut) {
      const int32_t *row = row_of(a.kv, a.kv.dev_tables, e.slot);
      const int held = pages_of(e.len, a.kv.page_tokens), first = a.ev.sinks / a.kv.page_tokens;
      const int last = pages_of(e.keep, a.kv.page_tokens);
      for (int c = t; c < held; c += THREADS) {
        const int p = row[c];
        if (p < 0 || p >= a.kv.pages) bad = true;
        else {
          const int r = a.kv.dev_refs[p];
          bad |= r < 1 || (c >= first && c < last && e.keep > a.ev.sinks && r != 1);
        }
      }
    }
  } else {
    for (int i = t; i < (a.kv.slots + 31) / 32; i += THREADS) seen[i] = 0;
    __syncthreads();
    for (int i = t; i < n; i += THREADS) {
      const int s = a.ev.dev_slots[i];
      if (s >= 0 && s < a.kv.slots) bad |= atomicOr(&seen[s >> 5], 1u << (s & 31)) >> (s & 31) & 1;
    }
  }
  if (bad) atomicOr(&a.ctl->err, KV_ERR_ARG);
  stores_done();
  if (!last_of(&a.ctl->arrived, (uint32_t)n + 1)) return;
  if (t == 0) {
    const uint32_t err = __hip_atomic_load(&a.ctl->err, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    a.ctl->go = err == 0;
    a.ctl->err = 0;
    if (err) atomicOr(&a.ctl->sticky, err);
  }
}

// Bytes from a plane's first page to token j of the row, which has it.
__device__ __forceinline__ int64_t token_at(const Args &a, const int32_t *row, int j) {
  const int c = j / a.kv.page_tokens;
  return (int64_t)row[c] * (int64_t)a.kv.page_stride + (int64_t)(j - c * a.kv.page_tokens) * (int64_t)a.kv.token_bytes;
}

// The middle: the places of MOVE_TILE that another token comes to.
__global__ __launch_bounds__(THREADS) void k_evict_move(Args a) {
  if (!a.ctl->go) return;
  __shared__ int64_t from[MOVE_TILE], to[MOVE_TILE];
  __shared__ uint32_t count;
  int b = blockIdx.x;
  const int head = b % a.ev.kv_heads;
  b /= a.ev.kv_heads;
  const int part = b % a.moves;
  b /= a.moves;
  const int i = b % a.ev.n, layer = b / a.ev.n;
  const Entry e = get_entry(a, i);
  const bool out = a.ev.dev_weights_out != a.ev.dev_weights;
  const int end = e.cut ? e.keep - a.ev.recent : out ? e.len : 0;
  const int32_t *kept = kept_of(a, layer, i, head), *row = row_of(a.kv, a.kv.dev_tables, e.slot);
  const int64_t wat = weights_at(a, layer, e.slot, head);
  const uint32_t pieces = (uint32_t)(a.head_bytes / 16);
  char *base = (char *)a.kv.dev_pool + (uint64_t)(2 * layer) * a.kv.plane_stride + head * a.head_bytes;
  for (int j0 = part * MOVE_TILE; j0 < end; j0 += a.moves * MOVE_TILE) {
    if (threadIdx.x == 0) count = 0;
    __syncthreads();
    for (int j = j0 + threadIdx.x; j < min(end, j0 + MOVE_TILE); j += THREADS) {
      const int src = kept[j];
      if (src != j || out) a.ev.dev_weights_out[wat + j] = a.ev.dev_weights[wat + src];
      if (src == j) continue;
      const uint32_t at = atomicAdd(&count, 1u);
      from[at] = token_at(a, row, src);
      to[at] = token_at(a, row, j);
    }
    __syncthreads();
    const uint32_t all = count * pieces;
    for (uint32_t x = threadIdx.x; x < all; x += THREADS) {
      const uint32_t at = x / pieces, piece = (x - at * pieces) * 16;
      const char *k = base + from[at] + piece;
      const u32x4 kv = *(const u32x4 *)k, vv = *(const u32x4 *)(k + a.kv.plane_stride);
      char *o = base + to[at] + piece;
      *(u32x4 *)o = kv;
      *(u32x4 *)(o + a.kv.plane_stride) = vv;
    }
    __syncthreads();
  }
}

// The last tokens: of one plane, all heads together, LAST_BYTES a workgroup where
// the new places are before the old ones, and else by one workgroup, some at a
// time from the front.  And, a workgroup a head, a layer's weights of them and behind.
constexpr int LAST_U = 8, LAST_BYTES = THREADS * LAST_U * 16;
__global__ __launch_bounds__(THREADS) void k_evict_last(Args a) {
  if (!a.ctl->go) return;
  int b = blockIdx.x;
  const int each = 2 * a.lasts + a.ev.kv_heads, what = b % each;  // K's parts, V's, weights
  b /= each;
  const int i = b % a.ev.n, layer = b / a.ev.n;
  const Entry e = get_entry(a, i);
  if (!e.cut) return;
  const int m = e.keep - a.ev.recent, by = e.len - e.keep;
  if (what >= 2 * a.lasts) {
    const int64_t wat = weights_at(a, layer, e.slot, what - 2 * a.lasts);
    const float *from = a.ev.dev_weights + wat;
    float *to = a.ev.dev_weights_out + wat;
    const bool over = to == from;  // (then place j + by, which becomes something else in this step or a later one, is read first)
    for (int j0 = m; j0 < e.len; j0 += THREADS) {
      const int j = j0 + threadIdx.x;
      const float v = j < e.keep ? from[j + by] : 0.f;
      if (over) {
        loads_done();
        __syncthreads();
      }
      if (j < e.len) to[j] = v;
    }
    return;
  }
  const int kv = what / a.lasts, part = what % a.lasts;
  char *plane = (char *)a.kv.dev_pool + (uint64_t)(2 * layer + kv) * a.kv.plane_stride;
  const int32_t *row = row_of(a.kv, a.kv.dev_tables, e.slot);
  const uint32_t pieces = (uint32_t)(a.kv.token_bytes / 16);
  const uint64_t all = (uint64_t)a.ev.recent * pieces;
  const bool over = by < a.ev.recent;
  if (over && part) return;
  for (uint64_t x0 = (uint64_t)part * THREADS * LAST_U; x0 < all; x0 += (uint64_t)(over ? 1 : a.lasts) * THREADS * LAST_U) {
    const int j0 = (int)(x0 / pieces);  // the first piece is `rest` of token j0
    const uint32_t rest = (uint32_t)(x0 - (uint64_t)j0 * pieces);
    u32x4 v[LAST_U];
#pragma unroll
    for (int u = 0; u < LAST_U; u++) {
      const uint32_t x = rest + u * THREADS + threadIdx.x, j = x / pieces;
      if (x0 + x - rest < all) v[u] = *(const u32x4 *)(plane + token_at(a, row, m + by + j0 + (int)j) + (x - j * pieces) * 16);
    }
    if (over) {
      loads_done();  // (of every wave, before any stores: the barrier waits for no memory)
      __syncthreads();
    }
#pragma unroll
    for (int u = 0; u < LAST_U; u++) {
      const uint32_t x = rest + u * THREADS + threadIdx.x, j = x / pieces;
      if (x0 + x - rest < all) *(u32x4 *)(plane + token_at(a, row, m + j0 + (int)j) + (x - j * pieces) * 16) = v[u];
    }
  }
}

__global__ __launch_bounds__(THREADS) void k_evict_end(Args a) {
  if (!a.ctl->go) return;
  const Entry e = get_entry(a, blockIdx.x);
  if (!e.cut) return;
  __syncthreads();  // every wave has read the length
  int32_t *row = row_of(a.kv, a.kv.dev_tables, e.slot);
  const int held = pages_of(e.len, a.kv.page_tokens);
  for (int c = pages_of(e.keep, a.kv.page_tokens) + threadIdx.x; c < held; c += THREADS) {
    atomicSub(&a.kv.dev_refs[row[c]], 1);
    row[c] = -1;
  }
  if (threadIdx.x == 0) a.kv.dev_lens[e.slot] = e.keep;
}

}  // namespace

hipError_t launch_kv_evict(const hbf_kv &kv, const hbf_eviction &ev, hipStream_t s) {
  Args a{};
  a.kv = kv;
  a.ev = ev;
  if (!a.ev.dev_weights_out) a.ev.dev_weights_out = const_cast<float *>(ev.dev_weights);
  a.ctl = (KvCtl *)kv.dev_ws;
  a.layers = kv.planes / 2;
  a.head_bytes = (int64_t)(kv.token_bytes / ev.kv_heads);
  const int64_t groups = (int64_t)a.layers * ev.n * ev.kv_heads;
  a.moves = (int)std::max<int64_t>(1, std::min<int64_t>((ev.max_keep + MOVE_TILE - 1) / MOVE_TILE, (1 << 14) / groups));
  k_evict_plan<<<(uint32_t)(ev.n + 1 + groups), THREADS, (size_t)((kv.slots + 31) / 32) * 4, s>>>(a);
  k_evict_move<<<(uint32_t)(groups * a.moves), THREADS, 0, s>>>(a);
  const int64_t entries = (int64_t)a.layers * ev.n, bytes = (int64_t)ev.recent * kv.token_bytes;
  a.lasts = (int)std::max<int64_t>(1, std::min<int64_t>((bytes + LAST_BYTES - 1) / LAST_BYTES, (1 << 14) / entries));
  k_evict_last<<<(uint32_t)(entries * (2 * a.lasts + ev.kv_heads)), THREADS, 0, s>>>(a);
  k_evict_end<<<(uint32_t)ev.n, THREADS, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace hbf
