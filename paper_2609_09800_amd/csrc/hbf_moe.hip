// A whole mixture-of-experts layer for a few tokens.
//
//   logits = x Wr^T; the topk largest, their softmax weights;
//   h = silu(Wg x) * (Wu x) per chosen expert; y = sum_j w_j Wd_j h_j.
//
// With few tokens the layer is bound by reading each chosen expert's weights
// once: 3 F H 16-bit values against 2 flops per value and token.  So the tokens
// are gathered by expert, a tile of 16 of them being the narrow side of the
// matrix instruction, and the weights are its wide side, loaded straight from
// memory into the operand (16 rows of 64 bytes at a time; a row's next 64 follow
// at once).  Four launches or three, each a pass over one kind of weights:
//  - route: logits by tiles of 16 experts and 16 tokens; a token tile's last
//    workgroup chooses, and the last of these sorts the (token, choice) pairs
//    by expert, in tiles of up to 16 (an expert with more is read once per
//    tile, by workgroups that run beside each other).  For up to four tokens
//    the logits only: up chooses;
//  - up: 8 gate rows and the 8 up rows of the same channels per tile of weights,
//    so that its products give 8 channels of h;
//  - down: 32 rows of y per tile and unit, each pair's product to a place of its
//    own;
//  - sum: a token's products in the order of its choices, so that the result
//    does not depend on who computed them (in down's launch where that has a
//    workgroup per unit, or one wave of a workgroup per token tile).
// Up and down are one scheme: a workgroup goes through consecutive units (a
// token tile's rows, then the next tile's) with the tile's tokens kept in
// registers, so that only weights are loaded, the next unit's while this one
// ends; its four waves split the inner axis and meet in LDS once per unit.  At 64
// tokens of 128 experts of 2,048 x 768 they read 6.7 TB/s (up 69 us, down 38, the
// route 14); at one token 3.5 and 2.3, where the launches' chain bounds them (14 and
// 11 us).
#include <math.h>

#include <algorithm>

#include "hbf_half.h"
#include "hbf_ops.h"

namespace hbf {
namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64;  // up and down
constexpr int GROUPS = 768;             // three workgroups per CU
constexpr int ROUTE_THREADS = 1024, ROUTE_WAVES = ROUTE_THREADS / 64;
constexpr int SUM_THREADS = 256;
constexpr int MAX_PAIRS = MOE_MAX_PAIRS;
constexpr int MAX_TILES = MOE_MAX_EXPERTS + MAX_PAIRS / 16;
constexpr int TOKEN_TILES = MOE_MAX_TOKENS / 16;
constexpr int FEW_TOKENS = WAVES, FEW_PAIRS = FEW_TOKENS * MOE_MAX_TOPK, FEW_EXPERTS = 256;

struct Tile {                           // up to 16 pairs of one expert
  int32_t expert;
  uint16_t start, count;                // start: first entry of Lists::pair
};
struct Lists {                          // what the route leaves for the others
  uint32_t n_tiles;
  uint32_t pad[63];
  Tile tile[MAX_TILES];
  int32_t pair[MAX_PAIRS];              // token * topk + choice, by expert
};
struct Ctl {                            // 0 between calls
  uint32_t arrived[TOKEN_TILES];        // a token tile's workgroups that are done
  uint32_t chosen;                      // token tiles whose choices are made
};

struct Args {
  hbf_moe m;
  const char *x;
  int64_t xs;
  int tokens;
  int32_t *ids;
  float *weights;
  char *y;
  int64_t ys;
  int32_t *status;
  Ctl *ctl;
  Lists *lists;
  float *logits;                        // [tokens][e_pad]
  int e_pad;
  char *h_hi, *h_lo;                    // [pairs][F], in the order of `pair`
  float *part;                          // [pairs][H] products, by token and choice
  uint32_t *block_done;                 // [H / 16] token tiles whose products of these rows are there
  bool choose_in_up;                    // few tokens: every workgroup of up makes the choices for itself
  bool sum_in_down;                     // few units: the last workgroup of a block of rows sums it
};

size_t up256(size_t v) { return (v + 255) & ~size_t(255); }

size_t carve(const hbf_moe &m, int tokens, char *base, Args *a) {
  size_t o = 256;
  auto take = [&](size_t bytes) {
    char *r = base + o;
    o = up256(o + bytes);
    return r;
  };
  a->e_pad = (m.experts + 15) / 16 * 16;
  a->ctl = (Ctl *)base;
  a->lists = (Lists *)take(sizeof(Lists));
  a->logits = (float *)take((size_t)tokens * a->e_pad * 4);
  a->h_hi = take((size_t)tokens * m.topk * m.ffn * 2);
  a->h_lo = take((size_t)tokens * m.topk * m.ffn * 2);
  a->part = (float *)take((size_t)tokens * m.topk * m.hidden * 4);
  a->block_done = (uint32_t *)take((size_t)m.hidden / 16 * 4 + 4);
  return o;
}

__device__ __forceinline__ u32x4 load16(const char *p) { return *(const u32x4 *)p; }
constexpr u32x4 ZERO4 = {0, 0, 0, 0};

// ------------------------------------------------------------ route

// The topk choices of token t by one wave; lane l holds experts l EPL .. + EPL-1.
// ids: in LDS.  HANDED: the logits are of this launch, and so may be the readers
// of a.ids.  write: to the caller's arrays too.
template <int EPL, bool HANDED>
__device__ void choose(const Args &a, int t, int32_t *ids, bool write = true) {
  const int lane = threadIdx.x & 63, E = a.m.experts, k = a.m.topk;
  float v[EPL];
  uint32_t key[EPL];
#pragma unroll
  for (int i = 0; i < EPL; i++) {
    const int e = lane * EPL + i;
    const float *from = a.logits + (int64_t)t * a.e_pad + min(e, E - 1);
    v[i] = HANDED ? handed(from) : *from;
    const uint32_t u = __float_as_uint(v[i]);
    // the floats' order as that of whole numbers; NaN below all, 0 for none (left)
    key[i] = e >= E ? 0 : isnan(v[i]) ? 1 : u & 0x80000000u ? ~u : u | 0x80000000u;
    if (key[i] == 0x7fffffffu) key[i] = 0x80000000u;  // -0 ties with 0
  }
  float mine = 0.f, top = 0.f;  // top: the largest logit
  int chosen = 0;
  for (int j = 0; j < k; j++) {
    uint32_t best = key[0];
#pragma unroll
    for (int i = 1; i < EPL; i++) best = max(best, key[i]);
    const uint32_t all = across_wave(best, [](uint32_t x, uint32_t y) { return max(x, y); });
    const int from = __ffsll((unsigned long long)__ballot(best == all)) - 1;  // ties: the lowest index
    int e = 0;
    float val = 0.f;
    if (lane == from) {
      bool done = false;
#pragma unroll
      for (int i = 0; i < EPL; i++)
        if (!done && key[i] == all) {
          e = lane * EPL + i;
          val = v[i];
          key[i] = 0;
          done = true;
        }
    }
    e = __builtin_amdgcn_readlane(e, from);
    val = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(val), from));
    if (j == 0) top = val;
    if (lane == j) {
      chosen = e;
      mine = val;
    }
  }
  float w = lane < k ? expf(mine - top) : 0.f, sum = 0.f;
  if (a.m.flags & HBF_MOE_RENORM) {
    sum = w;
  } else {
#pragma unroll
    for (int i = 0; i < EPL; i++)
      if (lane * EPL + i < E) sum += expf(v[i] - top);
  }
  sum = across_wave(sum, [](float x, float y) { return x + y; });
  if (lane < k) {
    ids[t * k + lane] = chosen;
    if (!write) return;
    __hip_atomic_store(a.ids + t * k + lane, chosen, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    a.weights[t * k + lane] = w / sum;
  }
}

template <typename T>
__global__ __launch_bounds__(ROUTE_THREADS) void k_moe_route(Args a) {
  __shared__ f32x4 red[ROUTE_WAVES][64];
  __shared__ int32_t ids[MAX_PAIRS];
  __shared__ int32_t cnt[MOE_MAX_EXPERTS];
  __shared__ uint32_t wsum[ROUTE_WAVES];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, col = lane & 15, kg = lane >> 4;
  const int E = a.m.experts, H = a.m.hidden, pairs = a.tokens * a.m.topk;
  if (a.m.dev_router) {
    const int e_tiles = a.e_pad / 16;
    const int e0 = blockIdx.x % e_tiles * 16, t0 = blockIdx.x / e_tiles * 16;
    const int e = min(e0 + col, E - 1), t = min(t0 + col, a.tokens - 1);
    const int steps = (H + 31) / 32, per = (steps + ROUTE_WAVES - 1) / ROUTE_WAVES;
    const char *rp = (const char *)a.m.dev_router + 2 * ((int64_t)e * H + kg * 8);
    const char *xp = a.x + 2 * ((int64_t)t * a.xs + kg * 8);
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    constexpr int U = 8;
    for (int s0 = w * per; s0 < min((w + 1) * per, steps); s0 += U) {
      u32x4 rv[U], xv[U];
#pragma unroll
      for (int u = 0; u < U; u++) {
        const int s = s0 + u;
        const bool on = s < (w + 1) * per && s * 32 + kg * 8 < H;
        rv[u] = on ? load16(rp + s * 64) : ZERO4;
        xv[u] = on ? load16(xp + s * 64) : ZERO4;
      }
#pragma unroll
      for (int u = 0; u < U; u++) acc = T::mfma(rv[u], xv[u], acc);
    }
    red[w][lane] = acc;
    __syncthreads();
    if (w == 0) {
#pragma unroll
      for (int i = 1; i < ROUTE_WAVES; i++) acc += red[i][lane];
      if (t0 + col < a.tokens)
#pragma unroll
        for (int i = 0; i < 4; i++) hand_over(a.logits + (int64_t)(t0 + col) * a.e_pad + e0 + kg * 4 + i, acc[i]);
      stores_done();
    }
    if (a.choose_in_up) return;
    const int tile = blockIdx.x / e_tiles;
    if (!last_of(&a.ctl->arrived[tile], e_tiles)) return;
    for (int tt = t0 + w; tt < min(t0 + 16, a.tokens); tt += ROUTE_WAVES) {
      if (E <= 64) choose<1, true>(a, tt, ids);
      else if (E <= 128) choose<2, true>(a, tt, ids);
      else if (E <= 256) choose<4, true>(a, tt, ids);
      else choose<16, true>(a, tt, ids);
    }
    const int t_tiles = gridDim.x / e_tiles;
    if (t_tiles > 1) {
      stores_done();
      if (!last_of(&a.ctl->chosen, t_tiles)) return;
      for (int p = threadIdx.x; p < pairs; p += ROUTE_THREADS)
        ids[p] = __hip_atomic_load(a.ids + p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  } else {
    for (int p = threadIdx.x; p < pairs; p += ROUTE_THREADS) {
      const int e = a.ids[p];
      const bool ok = e >= -1 && e < E;
      if (!ok && a.status) *a.status = HBF_EINVAL;
      ids[p] = ok ? e : -1;
    }
  }
  // pairs by expert
  for (int i = threadIdx.x; i < MOE_MAX_EXPERTS; i += ROUTE_THREADS) cnt[i] = 0;
  if (a.sum_in_down)
    for (int i = threadIdx.x; i <= H / 16; i += ROUTE_THREADS) a.block_done[i] = 0;
  __syncthreads();
  for (int p = threadIdx.x; p < pairs; p += ROUTE_THREADS)
    if (ids[p] >= 0) atomicAdd(&cnt[ids[p]], 1);
  __syncthreads();
  constexpr int PER = MOE_MAX_EXPERTS / ROUTE_THREADS;
  int c[PER];
  uint32_t sum = 0;  // pairs, and tiles above them
#pragma unroll
  for (int i = 0; i < PER; i++) {
    c[i] = cnt[threadIdx.x * PER + i];
    sum += c[i] + ((uint32_t)(c[i] + 15) / 16 << 16);
  }
  uint32_t x = sum;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  if (lane == 63) wsum[w] = x;
  __syncthreads();
  x -= sum;
#pragma unroll
  for (int i = 0; i < ROUTE_WAVES; i++) x += i < w ? wsum[i] : 0;
  uint32_t at = x & 0xffff, ti = x >> 16;
#pragma unroll
  for (int i = 0; i < PER; i++) {
    for (int j = 0; j < c[i]; j += 16)
      a.lists->tile[ti++] = Tile{(int)threadIdx.x * PER + i, (uint16_t)(at + j), (uint16_t)min(c[i] - j, 16)};
    cnt[threadIdx.x * PER + i] = at;
    at += c[i];
  }
  if (threadIdx.x == ROUTE_THREADS - 1) a.lists->n_tiles = ti;
  __syncthreads();
  // (an expert's pairs in any order: they are columns of its product, which do not meet)
  for (int p = threadIdx.x; p < pairs; p += ROUTE_THREADS)
    if (ids[p] >= 0) a.lists->pair[atomicAdd(&cnt[ids[p]], 1)] = p;
}

// ------------------------------------------------------------ up

// The route of at most FEW_TOKENS tokens from their logits, made by each
// workgroup for itself in LDS; the first one leaves it for the others' launch.
// All of them sort the pairs the same way: by expert, then token and choice.
struct FewLists {
  int32_t ids[FEW_PAIRS], pair[FEW_PAIRS], rank[FEW_PAIRS];
  Tile tile[FEW_PAIRS];
  int32_t n_tiles;
};
__device__ void route_few(const Args &a, FewLists &f) {
  const int w = threadIdx.x >> 6, p = threadIdx.x, pairs = a.tokens * a.m.topk;
  if (w < a.tokens) choose<FEW_EXPERTS / 64, false>(a, w, f.ids, blockIdx.x == 0);
  if (p == 0) f.n_tiles = 0;
  __syncthreads();
  int before = 0, rank = 0, count = 0;  // pairs of lower experts; of mine, those before me and all
  if (p < pairs) {
    const int e = f.ids[p];
    for (int q = 0; q < pairs; q++) {
      before += f.ids[q] < e;
      rank += f.ids[q] == e && q < p;
      count += f.ids[q] == e;
    }
    f.pair[before + rank] = p;
    f.rank[p] = rank;
  }
  __syncthreads();
  if (p < pairs && rank % 16 == 0) {
    int tile = rank / 16;
    for (int q = 0; q < pairs; q++) tile += f.ids[q] < f.ids[p] && f.rank[q] % 16 == 0;
    f.tile[tile] = Tile{f.ids[p], (uint16_t)(before + rank), (uint16_t)min(count - rank, 16)};
    atomicAdd(&f.n_tiles, 1);
  }
  __syncthreads();
  if (blockIdx.x) return;
  if (p < pairs) a.lists->pair[p] = f.pair[p];
  if (p < f.n_tiles) a.lists->tile[p] = f.tile[p];
  if (p == 0) a.lists->n_tiles = f.n_tiles;
  if (a.sum_in_down)
    for (int i = p; i <= a.m.hidden / 16; i += THREADS) a.block_done[i] = 0;
}

// KS steps of 32 per wave and pass; EXACT: the hidden size is one pass of them.
template <typename T, int KS, bool EXACT>
__global__ __launch_bounds__(THREADS) void k_moe_up(Args a) {
  __shared__ f32x4 red[2][WAVES][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, col = lane & 15, kg = lane >> 4;
  const int H = a.m.hidden, F = a.m.ffn, blocks = F / 8;
  __shared__ FewLists few;
  const Tile *tiles = a.lists->tile;
  const int32_t *pairs = a.lists->pair;
  if (a.choose_in_up) {
    route_few(a, few);
    tiles = few.tile;
    pairs = few.pair;
  }
  const int64_t units = (int64_t)(a.choose_in_up ? few.n_tiles : (int)a.lists->n_tiles) * blocks;
  const int u0 = (int)(units * blockIdx.x / gridDim.x), u1 = (int)(units * (blockIdx.x + 1) / gridDim.x);
  if (u0 >= u1) return;
  const int passes = EXACT ? 1 : (H + WAVES * KS * 32 - 1) / (WAVES * KS * 32);
  u32x4 av[KS], bv[KS];
  auto k_of = [&](int pass, int s) { return ((pass * WAVES + w) * KS + s) * 32 + kg * 8; };
  auto load_w = [&](int expert, int block, int pass) {
    const int r = block * 8 + (col & 7) + (col & 8 ? F : 0);
    const char *p = (const char *)a.m.dev_gate_up + 2 * ((int64_t)expert * a.m.gate_up_stride + (int64_t)r * H);
#pragma unroll
    for (int s = 0; s < KS; s++) {
      const int k = k_of(pass, s);
      av[s] = EXACT || k < H ? load16(p + 2 * k) : ZERO4;
    }
  };
  auto load_x = [&](int token, int pass) {
    const char *p = a.x + 2 * (token * a.xs);
#pragma unroll
    for (int s = 0; s < KS; s++) {
      const int k = k_of(pass, s);
      bv[s] = EXACT || k < H ? load16(p + 2 * k) : ZERO4;
    }
  };
  int ti = u0 / blocks, block = u0 - ti * blocks, buf = 0;
  Tile tile = tiles[ti];
  load_w(tile.expert, block, 0);
  // columns past the tokens repeat the last
  int token = pairs[tile.start + min(col, (int)tile.count - 1)] / a.m.topk;
  if (passes == 1) load_x(token, 0);  // kept for all of the tile's units
  for (int u = u0; u < u1; u++) {
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int pass = 0; pass < passes; pass++) {
      if (pass) load_w(tile.expert, block, pass);
      if (passes > 1) load_x(token, pass);
#pragma unroll
      for (int s = 0; s < KS; s++) acc = T::mfma(av[s], bv[s], acc);
    }
    const Tile done = tile;
    const int b8 = block * 8;
    if (u + 1 < u1) {  // the next loads are in flight while this unit ends
      if (++block == blocks) {
        block = 0;
        tile = tiles[++ti];
        token = pairs[tile.start + min(col, (int)tile.count - 1)] / a.m.topk;
        if (passes == 1) load_x(token, 0);
      }
      load_w(tile.expert, block, 0);
    }
    red[buf][w][lane] = acc;
    __syncthreads();
    const int n = threadIdx.x >> 3, r = threadIdx.x & 7;
    if (n < done.count) {
      float g = 0.f, up = 0.f;
#pragma unroll
      for (int i = 0; i < WAVES; i++) {
        g += red[buf][i][(r >> 2) * 16 + n][r & 3];
        up += red[buf][i][(2 + (r >> 2)) * 16 + n][r & 3];
      }
      const float h = g / (1.f + expf(-g)) * up;
      // two words: what rounding h to one would lose shows in y as much as y's own rounding
      const typename T::elem hi = (typename T::elem)h;
      const float rest = h - (float)hi;
      const int64_t at = (int64_t)(done.start + n) * F + b8 + r;
      ((typename T::elem *)a.h_hi)[at] = hi;
      ((typename T::elem *)a.h_lo)[at] = (typename T::elem)(isfinite(rest) ? rest : 0.f);
    }
    buf ^= 1;  // (the next unit writes the other half: one barrier per unit)
  }
}

// ------------------------------------------------------------ down

__device__ __forceinline__ bool used(const Args &a, int pair) {
  return a.m.dev_router || (uint32_t)a.ids[pair] < (uint32_t)a.m.experts;
}

// y of rows r0 .. r0 + rows - 1 of every token, from products that others of this
// launch handed over.
__device__ void sum_handed(const Args &a, int r0, int rows, void (*store)(char *, float)) {
  const int k = a.m.topk, H = a.m.hidden;
  for (int i = threadIdx.x; i < a.tokens * rows; i += THREADS) {
    const int t = i / rows, r = r0 + i - t * rows;
    if (r >= H) continue;
    float y = 0.f;
#pragma unroll 8
    for (int j = 0; j < k; j++) {
      const int p = t * k + j;
      if (used(a, p)) y += a.weights[p] * handed(a.part + (int64_t)p * H + r);
    }
    store(a.y + 2 * (t * a.ys + r), y);
  }
}
template <typename T>
__device__ void store_elem(char *to, float v) {
  *(typename T::elem *)to = (typename T::elem)v;
}

// Few token tiles: 16 rows of y per workgroup, a tile's products by one wave of
// it, summed in its LDS.  KS steps of 32 per pass; EXACT: F is one pass and H whole
// workgroups.
constexpr int DOWN_FEW_THREADS = 512, DOWN_FEW_WAVES = DOWN_FEW_THREADS / 64, DOWN_FEW_TILES = 2 * DOWN_FEW_WAVES;
constexpr int DOWN_FEW_PAIRS = 128;
template <typename T, int KS, bool EXACT>
__global__ __launch_bounds__(DOWN_FEW_THREADS, 2) void k_moe_down_few(Args a) {
  __shared__ float part[DOWN_FEW_PAIRS][17];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, col = lane & 15, kg = lane >> 4;
  const int H = a.m.hidden, F = a.m.ffn, r0 = blockIdx.x * 16, k = a.m.topk;
  const int passes = EXACT ? 1 : (F + KS * 32 - 1) / (KS * 32);
  Tile tile = a.lists->tile[w];  // (there may be fewer: asked for beside their number)
  const int n_tiles = a.lists->n_tiles;
  for (int ti = w; ti < n_tiles; ti += DOWN_FEW_WAVES) {
    if (ti != w) tile = a.lists->tile[ti];
    const int n = min(col, (int)tile.count - 1);  // columns past the tokens repeat the last
    const int pair = a.lists->pair[tile.start + n], r = EXACT ? r0 + col : min(r0 + col, H - 1);
    const char *wp = (const char *)a.m.dev_down + 2 * ((int64_t)tile.expert * a.m.down_stride + (int64_t)r * F);
    const int64_t h0 = 2 * (int64_t)(tile.start + n) * F;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int pass = 0; pass < passes; pass++) {
      u32x4 av[KS];
#pragma unroll
      for (int s = 0; s < KS; s++) {
        const int at = (pass * KS + s) * 32 + kg * 8;
        av[s] = EXACT || at < F ? load16(wp + 2 * at) : ZERO4;
      }
      constexpr int HS = 8;  // steps of h at a time
#pragma unroll
      for (int s0 = 0; s0 < KS; s0 += HS) {
        u32x4 hi[HS], lo[HS];
#pragma unroll
        for (int s = 0; s < HS; s++) {
          const int at = (pass * KS + s0 + s) * 32 + kg * 8;
          const bool on = EXACT || at < F;
          hi[s] = on ? load16(a.h_hi + h0 + 2 * at) : ZERO4;
          lo[s] = on ? load16(a.h_lo + h0 + 2 * at) : ZERO4;
        }
#pragma unroll
        for (int s = 0; s < HS; s++) {
          acc = T::mfma(av[s0 + s], hi[s], acc);
          acc = T::mfma(av[s0 + s], lo[s], acc);
        }
      }
    }
    if (col < tile.count)
#pragma unroll
      for (int i = 0; i < 4; i++) part[pair][kg * 4 + i] = acc[i];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < a.tokens * 16; i += DOWN_FEW_THREADS) {
    const int t = i >> 4, r = r0 + (i & 15);
    if (!EXACT && r >= H) continue;
    float y = 0.f;
    for (int j = 0; j < k; j++) {
      const int p = t * k + j;
      if (used(a, p)) y += a.weights[p] * part[p][i & 15];
    }
    ((typename T::elem *)a.y)[t * a.ys + r] = (typename T::elem)y;
  }
}

// KS steps of 32 per wave and pass, RB tiles of 16 rows per unit; EXACT: F is one
// pass and H whole units.
template <typename T, int KS, int RB, bool EXACT>
__global__ __launch_bounds__(THREADS) void k_moe_down(Args a) {
  __shared__ f32x4 red[2][WAVES][RB][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, col = lane & 15, kg = lane >> 4;
  const int H = a.m.hidden, F = a.m.ffn, blocks = (H + 16 * RB - 1) / (16 * RB);
  const int n_tiles = a.lists->n_tiles;
  const int64_t units = (int64_t)n_tiles * blocks;
  if (a.sum_in_down && n_tiles == 0) {  // no choice at all: y is 0
    if ((int)blockIdx.x < blocks) sum_handed(a, blockIdx.x * 16 * RB, 16 * RB, store_elem<T>);
    return;
  }
  const int u0 = (int)(units * blockIdx.x / gridDim.x), u1 = (int)(units * (blockIdx.x + 1) / gridDim.x);
  if (u0 >= u1) return;
  const int passes = EXACT ? 1 : (F + WAVES * KS * 32 - 1) / (WAVES * KS * 32);
  u32x4 av[RB][KS], hi[KS], lo[KS];
  auto k_of = [&](int pass, int s) { return ((pass * WAVES + w) * KS + s) * 32 + kg * 8; };
  auto load_w = [&](int expert, int block, int pass) {
#pragma unroll
    for (int b = 0; b < RB; b++) {
      const int r = (block * RB + b) * 16 + col;
      const char *p = (const char *)a.m.dev_down +
                      2 * ((int64_t)expert * a.m.down_stride + (int64_t)(EXACT ? r : min(r, H - 1)) * F);
#pragma unroll
      for (int s = 0; s < KS; s++) {
        const int k = k_of(pass, s);
        av[b][s] = EXACT || k < F ? load16(p + 2 * k) : ZERO4;
      }
    }
  };
  auto load_h = [&](int entry, int pass) {
#pragma unroll
    for (int s = 0; s < KS; s++) {
      const int k = k_of(pass, s);
      const int64_t at = 2 * ((int64_t)entry * F + k);
      hi[s] = EXACT || k < F ? load16(a.h_hi + at) : ZERO4;
      lo[s] = EXACT || k < F ? load16(a.h_lo + at) : ZERO4;
    }
  };
  int ti = u0 / blocks, block = u0 - ti * blocks, buf = 0;
  Tile tile = a.lists->tile[ti];
  load_w(tile.expert, block, 0);
  int entry = tile.start + min(col, (int)tile.count - 1);  // columns past the tokens repeat the last
  if (passes == 1) load_h(entry, 0);
  for (int u = u0; u < u1; u++) {
    f32x4 acc[RB];
#pragma unroll
    for (int b = 0; b < RB; b++) acc[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int pass = 0; pass < passes; pass++) {
      if (pass) load_w(tile.expert, block, pass);
      if (passes > 1) load_h(entry, pass);
#pragma unroll
      for (int s = 0; s < KS; s++)
#pragma unroll
        for (int b = 0; b < RB; b++) {
          acc[b] = T::mfma(av[b][s], hi[s], acc[b]);
          acc[b] = T::mfma(av[b][s], lo[s], acc[b]);
        }
    }
    const Tile done = tile;
    const int row0 = block * RB * 16;
    if (u + 1 < u1) {
      if (++block == blocks) {
        block = 0;
        tile = a.lists->tile[++ti];
        entry = tile.start + min(col, (int)tile.count - 1);
        if (passes == 1) load_h(entry, 0);
      }
      load_w(tile.expert, block, 0);
    }
#pragma unroll
    for (int b = 0; b < RB; b++) red[buf][w][b][lane] = acc[b];
    __syncthreads();
    const int n = threadIdx.x >> 4, r = threadIdx.x & 15;
    if (n < done.count) {
      const int64_t to = (int64_t)a.lists->pair[done.start + n] * H + row0 + r;
#pragma unroll
      for (int b = 0; b < RB; b++) {
        float o = 0.f;
#pragma unroll
        for (int i = 0; i < WAVES; i++) o += red[buf][i][b][(r >> 2) * 16 + n][r & 3];
        if (EXACT || row0 + b * 16 + r < H) {
          if (a.sum_in_down) hand_over(a.part + to + b * 16, o);
          else a.part[to + b * 16] = o;
        }
      }
    }
    if (a.sum_in_down) {
      stores_done();
      if (last_of(a.block_done + row0 / (16 * RB), n_tiles)) sum_handed(a, row0, 16 * RB, store_elem<T>);
    }
    buf ^= 1;
  }
}

// ------------------------------------------------------------ sum

// Four channels of one token per thread.
template <typename T>
__global__ __launch_bounds__(SUM_THREADS) void k_moe_sum(Args a) {
  const int quads = a.m.hidden / 4, k = a.m.topk;
  const int i = blockIdx.x * SUM_THREADS + threadIdx.x, t = i / quads, r = (i - t * quads) * 4;
  if (t >= a.tokens) return;
  f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int j = 0; j < k; j++) {
    const int p = t * k + j;
    if (used(a, p)) y += a.weights[p] * *(const f32x4 *)(a.part + (int64_t)p * a.m.hidden + r);
  }
  *(u32x2 *)(a.y + 2 * (t * a.ys + r)) = u32x2{pack2<T>(y[0], y[1]), pack2<T>(y[2], y[3])};
}

template <typename T, int KS>
void up(const Args &a, int groups, hipStream_t s) {
  if (a.m.hidden == WAVES * KS * 32)
    k_moe_up<T, KS, true><<<groups, THREADS, 0, s>>>(a);
  else
    k_moe_up<T, KS, false><<<groups, THREADS, 0, s>>>(a);
}
template <typename T, int KS, int RB>
void down(const Args &a, int tiles, hipStream_t s) {
  const int64_t units = (int64_t)tiles * ((a.m.hidden + 16 * RB - 1) / (16 * RB));
  const int groups = (int)std::min<int64_t>(units, GROUPS);
  if (a.m.ffn == WAVES * KS * 32 && a.m.hidden % (16 * RB) == 0)
    k_moe_down<T, KS, RB, true><<<groups, THREADS, 0, s>>>(a);
  else
    k_moe_down<T, KS, RB, false><<<groups, THREADS, 0, s>>>(a);
}

template <typename T, int KS>
void down_few(const Args &a, hipStream_t s) {
  const int groups = (a.m.hidden + 15) / 16;
  if (a.m.ffn == KS * 32 && a.m.hidden % 16 == 0)
    k_moe_down_few<T, KS, true><<<groups, DOWN_FEW_THREADS, 0, s>>>(a);
  else
    k_moe_down_few<T, KS, false><<<groups, DOWN_FEW_THREADS, 0, s>>>(a);
}

template <typename T>
hipError_t run(Args a, hipStream_t s) {
  const int pairs = a.tokens * a.m.topk;
  const int tiles = std::min(pairs, a.m.experts + pairs / 16);  // at most
  // A workgroup per unit: summed there, the layer is a launch shorter (one token of the 128-expert layer: 31.8 us, 33.0
  // with it).  Where workgroups have several units, waiting for each one's stores would cost more.
  a.sum_in_down = (int64_t)tiles * ((a.m.hidden + 31) / 32) <= GROUPS;
  // A workgroup's four waves choose for four tokens side by side, which takes it 3 us, the route's hand-over from
  // workgroup to workgroup 5 (one token of the 128-expert layer: 30.8 us, 32.6 without it).
  a.choose_in_up = a.m.dev_router && a.tokens <= FEW_TOKENS && a.m.experts <= FEW_EXPERTS;
  const int route = a.m.dev_router ? a.e_pad / 16 * ((a.tokens + 15) / 16) : 1;
  k_moe_route<T><<<route, ROUTE_THREADS, 0, s>>>(a);
  const int groups = (int)std::min<int64_t>((int64_t)tiles * (a.m.ffn / 8), GROUPS);
  // steps per wave
  const int up_steps = ((a.m.hidden + 31) / 32 + WAVES - 1) / WAVES;
  if (up_steps <= 2) up<T, 2>(a, groups, s);
  else if (up_steps <= 4) up<T, 4>(a, groups, s);
  else if (up_steps <= 8) up<T, 8>(a, groups, s);
  else up<T, 16>(a, groups, s);
  // Up to 16 token tiles can be summed in the workgroups of 16 rows, but with few rows these leave CUs idle, and above 256
  // channels a wave's weights are not one pass of its registers.  In us, so and by all units' workgroups:
  //   rows x channels: 6 tiles     8 tiles     16 tiles       rows x channels: 6 tiles     8 tiles     16 tiles
  //   512 x 256        13.3 13.8   15.9 17.1   19.6 19.6      2,048 x 256      16.3 17.9   19.9 22.8   24.9 26.2
  //   512 x 512        16.0 15.0   19.9 18.5   25.5 21.3      2,048 x 512      20.8 21.4   25.4 26.1   35.8 33.8
  //   1,024 x 256      14.2 15.0   17.5 18.9   21.4 22.0      2,048 x 768      23.0 24.4   30.4 30.1   47.5 44.1
  //   1,024 x 512      18.0 16.9   22.1 21.3   28.6 25.1      4,096 x 1,536                83   92
  if (tiles <= DOWN_FEW_TILES && pairs <= DOWN_FEW_PAIRS &&
      (a.m.ffn <= 256 || a.m.hidden >= 4096 || (a.m.hidden >= 2048 && (int64_t)tiles * 16 * a.m.ffn <= 65536))) {
    if (a.m.ffn <= 256) down_few<T, 8>(a, s);
    else down_few<T, 24>(a, s);
    return hipGetLastError();
  }
  const int down_steps = ((a.m.ffn + 31) / 32 + WAVES - 1) / WAVES;
  if (down_steps <= 2) down<T, 2, 2>(a, tiles, s);
  else if (down_steps <= 4) down<T, 4, 2>(a, tiles, s);
  else if (down_steps <= 6) down<T, 6, 2>(a, tiles, s);
  else down<T, 8, 2>(a, tiles, s);
  if (!a.sum_in_down)
    k_moe_sum<T><<<(a.tokens * (a.m.hidden / 4) + SUM_THREADS - 1) / SUM_THREADS, SUM_THREADS, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

size_t moe_ws_bytes(const hbf_moe &m, int tokens) {
  Args a{};
  return carve(m, tokens, nullptr, &a);
}

hipError_t launch_moe(const hbf_moe &m, const void *x, int64_t xs, int tokens, int32_t *ids, float *weights, void *y,
                      int64_t ys, int32_t *status, void *ws, hipStream_t s) {
  Args a{};
  carve(m, tokens, (char *)ws, &a);
  a.m = m;
  a.x = (const char *)x;
  a.xs = xs;
  a.tokens = tokens;
  a.ids = ids;
  a.weights = weights;
  a.y = (char *)y;
  a.ys = ys;
  a.status = status;
  return m.dtype == HBF_BF16 ? run<Bf16>(a, s) : run<Fp16>(a, s);
}

}  // namespace hbf
