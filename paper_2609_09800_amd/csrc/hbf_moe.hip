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
// at once).  Three launches, each a pass over one kind of weights:
//  - route: logits by tiles of 16 experts; the last workgroup chooses, and sorts
//    the (token, choice) pairs by expert;
//  - up: 8 gate rows and the 8 up rows of the same channels per tile, so that
//    one tile's products give 8 channels of h;
//  - down: 16 rows of y per workgroup, its waves dealing the experts out among
//    them; each pair's product has a place of its own in LDS, and a token's are
//    summed in the order of its choices, whoever computed them.
#include <math.h>

#include <algorithm>

#include "hbf_half.h"
#include "hbf_ops.h"

namespace hbf {
namespace {

constexpr int UP_THREADS = 256, UP_WAVES = UP_THREADS / 64;
constexpr int UP_GROUPS = 768;          // three workgroups of 4 waves per CU
constexpr int ROUTE_THREADS = 512, ROUTE_WAVES = ROUTE_THREADS / 64;
constexpr int DOWN_THREADS = 512, DOWN_WAVES = DOWN_THREADS / 64;
constexpr int MAX_PAIRS = MOE_MAX_PAIRS;

struct Lists {                          // what the route leaves for the others
  uint32_t n_active;
  uint32_t pad[63];
  int32_t expert[MOE_MAX_EXPERTS];      // of the n_active experts with tokens, ascending
  int32_t start[MOE_MAX_EXPERTS + 1];   // their first entry of `pair`
  int32_t pair[MAX_PAIRS];              // token * topk + choice, by expert
};
struct Ctl {
  uint32_t arrived;                     // 0 between calls
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
  return o;
}

__device__ __forceinline__ u32x4 load16(const char *p) { return *(const u32x4 *)p; }
constexpr u32x4 ZERO4 = {0, 0, 0, 0};

// ------------------------------------------------------------ route

// Maximum over the wave, in every lane.
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#define HBF_DPP_MAX(ctrl) v = max(v, (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, ctrl, 0xf, 0xf, false))
  HBF_DPP_MAX(0xb1);   // quad_perm 1,0,3,2
  HBF_DPP_MAX(0x4e);   // quad_perm 2,3,0,1
  HBF_DPP_MAX(0x141);  // row_half_mirror
  HBF_DPP_MAX(0x140);  // row_mirror
#undef HBF_DPP_MAX
  v = max(v, (uint32_t)__shfl_xor((int)v, 16));
  return max(v, (uint32_t)__shfl_xor((int)v, 32));
}

// The topk choices of token t by one wave; lane l holds experts l EPL .. + EPL-1.
template <int EPL>
__device__ void choose(const Args &a, int t, int32_t *ids_lds) {
  const int lane = threadIdx.x & 63, E = a.m.experts, k = a.m.topk;
  float v[EPL];
  uint32_t key[EPL];
  float top = -INFINITY;
#pragma unroll
  for (int i = 0; i < EPL; i++) {
    const int e = lane * EPL + i;
    v[i] = e < E ? a.logits[(int64_t)t * a.e_pad + e] : 0.f;
    const uint32_t u = __float_as_uint(v[i]);
    // the floats' order as that of whole numbers; NaN below all, 0 for none (left)
    key[i] = e >= E ? 0 : isnan(v[i]) ? 1 : u & 0x80000000u ? ~u : u | 0x80000000u;
    if (key[i] == 0x7fffffffu) key[i] = 0x80000000u;  // -0 ties with 0
    if (e < E) top = fmaxf(top, v[i]);
  }
  float mine = 0.f;
  int chosen = 0;
  for (int j = 0; j < k; j++) {
    uint32_t best = key[0];
#pragma unroll
    for (int i = 1; i < EPL; i++) best = max(best, key[i]);
    const uint32_t all = wave_max(best);
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
    if (lane == j) {
      chosen = e;
      mine = val;
    }
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
  float w = lane < k ? expf(mine - top) : 0.f, sum = 0.f;
  if (a.m.flags & HBF_MOE_RENORM) {
    sum = w;
  } else {
#pragma unroll
    for (int i = 0; i < EPL; i++)
      if (lane * EPL + i < E) sum += expf(v[i] - top);
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
  if (lane < k) {
    ids_lds[t * k + lane] = chosen;
    a.ids[t * k + lane] = chosen;
    a.weights[t * k + lane] = w / sum;
  }
}

template <typename T>
__global__ __launch_bounds__(ROUTE_THREADS) void k_moe_route(Args a) {
  __shared__ f32x4 red[ROUTE_WAVES][64];
  __shared__ int32_t ids[MAX_PAIRS];
  __shared__ int32_t cnt[MOE_MAX_EXPERTS];
  __shared__ uint32_t wsum[ROUTE_WAVES], asum[ROUTE_WAVES];
  __shared__ uint32_t last;
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
      if (t0 + col < a.tokens) *(f32x4 *)(a.logits + (int64_t)(t0 + col) * a.e_pad + e0 + kg * 4) = acc;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      __threadfence();
      last = atomicAdd(&a.ctl->arrived, 1) + 1 == gridDim.x;
      __threadfence();
    }
    __syncthreads();
    if (!last) return;
    if (threadIdx.x == 0) a.ctl->arrived = 0;
    for (int tt = w; tt < a.tokens; tt += ROUTE_WAVES) {
      if (E <= 64) choose<1>(a, tt, ids);
      else if (E <= 128) choose<2>(a, tt, ids);
      else if (E <= 256) choose<4>(a, tt, ids);
      else choose<16>(a, tt, ids);
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
  __syncthreads();
  for (int p = threadIdx.x; p < pairs; p += ROUTE_THREADS)
    if (ids[p] >= 0) atomicAdd(&cnt[ids[p]], 1);
  __syncthreads();
  constexpr int PER = MOE_MAX_EXPERTS / ROUTE_THREADS;
  int c[PER];
  uint32_t sum = 0, act = 0;
#pragma unroll
  for (int i = 0; i < PER; i++) {
    c[i] = cnt[threadIdx.x * PER + i];
    sum += c[i];
    act += c[i] > 0;
  }
  uint32_t xs = sum, xa = act;
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t ys = __shfl_up(xs, d), ya = __shfl_up(xa, d);
    if (lane >= d) {
      xs += ys;
      xa += ya;
    }
  }
  if (lane == 63) {
    wsum[w] = xs;
    asum[w] = xa;
  }
  __syncthreads();
  uint32_t at = xs - sum, ai = xa - act;
  for (int i = 0; i < w; i++) {
    at += wsum[i];
    ai += asum[i];
  }
#pragma unroll
  for (int i = 0; i < PER; i++) {
    if (c[i] > 0) {
      a.lists->expert[ai] = threadIdx.x * PER + i;
      a.lists->start[ai++] = at;
    }
    cnt[threadIdx.x * PER + i] = at;
    at += c[i];
  }
  if (threadIdx.x == ROUTE_THREADS - 1) {
    a.lists->n_active = ai;
    a.lists->start[ai] = at;
  }
  __syncthreads();
  // (an expert's pairs in any order: they are columns of its product, which do not meet)
  for (int p = threadIdx.x; p < pairs; p += ROUTE_THREADS)
    if (ids[p] >= 0) a.lists->pair[atomicAdd(&cnt[ids[p]], 1)] = p;
}

// ------------------------------------------------------------ up

// KS steps of 32 per wave and pass; EXACT: the hidden size is one pass of them.
template <typename T, int KS, bool EXACT>
__global__ __launch_bounds__(UP_THREADS) void k_moe_up(Args a) {
  __shared__ f32x4 red[2][UP_WAVES][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, col = lane & 15, kg = lane >> 4;
  const int H = a.m.hidden, F = a.m.ffn, blocks = F / 8;
  const int64_t units = (int64_t)a.lists->n_active * blocks;
  const int u0 = (int)(units * blockIdx.x / gridDim.x), u1 = (int)(units * (blockIdx.x + 1) / gridDim.x);
  const int passes = EXACT ? 1 : (H + UP_WAVES * KS * 32 - 1) / (UP_WAVES * KS * 32);
  u32x4 av[KS], bv[KS];
  auto k_of = [&](int pass, int s) { return ((pass * UP_WAVES + w) * KS + s) * 32 + kg * 8; };
  auto load_w = [&](int u, int pass) {
    const int e = a.lists->expert[u / blocks], r = u % blocks * 8 + (col & 7) + (col & 8 ? F : 0);
    const char *p = (const char *)a.m.dev_gate_up + 2 * ((int64_t)e * a.m.gate_up_stride + (int64_t)r * H);
#pragma unroll
    for (int s = 0; s < KS; s++) {
      const int k = k_of(pass, s);
      av[s] = EXACT || k < H ? load16(p + 2 * k) : ZERO4;
    }
  };
  auto load_x = [&](int pair, int pass) {
    const char *p = a.x + 2 * ((int64_t)(a.lists->pair[pair] / a.m.topk) * a.xs);
#pragma unroll
    for (int s = 0; s < KS; s++) {
      const int k = k_of(pass, s);
      bv[s] = EXACT || k < H ? load16(p + 2 * k) : ZERO4;
    }
  };
  int held = -1, buf = 0;  // the active expert whose (only) tile of tokens bv holds
  if (u0 < u1) load_w(u0, 0);
  for (int u = u0; u < u1; u++) {
    const int act = u / blocks, p0 = a.lists->start[act], p1 = a.lists->start[act + 1];
    for (int p = p0; p < p1; p += 16) {
      const int mine = min(p + col, p1 - 1);  // columns past the tokens repeat the last
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
      for (int pass = 0; pass < passes; pass++) {
        if (passes > 1 && (pass || p > p0)) load_w(u, pass);
        if (passes > 1 || p1 - p0 > 16 || held != act) load_x(mine, pass);
#pragma unroll
        for (int s = 0; s < KS; s++) acc = T::mfma(av[s], bv[s], acc);
      }
      held = p1 - p0 > 16 ? -1 : act;
      if (p + 16 >= p1 && u + 1 < u1) load_w(u + 1, 0);  // in flight while this tile ends
      red[buf][w][lane] = acc;
      __syncthreads();
      const int n = threadIdx.x >> 3, r = threadIdx.x & 7;
      if (threadIdx.x < 128 && p + n < p1) {
        float g = 0.f, up = 0.f;
#pragma unroll
        for (int i = 0; i < UP_WAVES; i++) {
          g += red[buf][i][(r >> 2) * 16 + n][r & 3];
          up += red[buf][i][(2 + (r >> 2)) * 16 + n][r & 3];
        }
        const float h = g / (1.f + expf(-g)) * up;
        // two words: what rounding h to one would lose shows in y as much as y's own rounding
        const typename T::elem hi = (typename T::elem)h;
        const float rest = h - (float)hi;
        const int64_t at = (int64_t)(p + n) * F + u % blocks * 8 + r;
        ((typename T::elem *)a.h_hi)[at] = hi;
        ((typename T::elem *)a.h_lo)[at] = (typename T::elem)(isfinite(rest) ? rest : 0.f);
      }
      buf ^= 1;  // (the next tile writes the other half; one barrier per tile)
    }
  }
}

// ------------------------------------------------------------ down

template <typename T>
__global__ __launch_bounds__(DOWN_THREADS) void k_moe_down(Args a) {
  extern __shared__ __align__(16) float part[];  // [pairs][16] products of this workgroup's rows
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, col = lane & 15, kg = lane >> 4;
  const int H = a.m.hidden, F = a.m.ffn, k = a.m.topk, r0 = blockIdx.x * 16;
  constexpr int KS = 8;
  const int chunks = (F + KS * 32 - 1) / (KS * 32), n_act = a.lists->n_active;
  for (int i = threadIdx.x; i < a.tokens * k * 4; i += DOWN_THREADS) ((f32x4 *)part)[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  __syncthreads();
  const char *wp = (const char *)a.m.dev_down + 2 * ((int64_t)min(r0 + col, H - 1) * F + kg * 8);
  u32x4 next[KS], av[KS];
  auto load_w = [&](int act, int c) {
    const char *p = wp + 2 * (int64_t)a.lists->expert[act] * a.m.down_stride;
#pragma unroll
    for (int s = 0; s < KS; s++) {
      const int kk = (c * KS + s) * 32;
      next[s] = kk + kg * 8 < F ? load16(p + 2 * kk) : ZERO4;
    }
  };
  if (w < n_act) load_w(w, 0);
  for (int act = w; act < n_act; act += DOWN_WAVES) {
    const int p0 = a.lists->start[act], p1 = a.lists->start[act + 1];
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int c = 0; c < chunks; c++) {
#pragma unroll
      for (int s = 0; s < KS; s++) av[s] = next[s];
      if (c + 1 < chunks)
        load_w(act, c + 1);
      else if (act + DOWN_WAVES < n_act)
        load_w(act + DOWN_WAVES, 0);
      for (int p = p0; p < p1; p += 16) {
        const int64_t row = (int64_t)min(p + col, p1 - 1) * F + c * KS * 32 + kg * 8;
        if (p1 - p0 > 16) acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < KS; s++) {
          const bool on = (c * KS + s) * 32 + kg * 8 < F;
          const u32x4 hi = on ? load16(a.h_hi + 2 * (row + s * 32)) : ZERO4;
          const u32x4 lo = on ? load16(a.h_lo + 2 * (row + s * 32)) : ZERO4;
          acc = T::mfma(av[s], hi, acc);
          acc = T::mfma(av[s], lo, acc);
        }
        if ((p1 - p0 > 16 || c + 1 == chunks) && p + col < p1) {
          f32x4 *to = (f32x4 *)(part + a.lists->pair[p + col] * 16 + kg * 4);
          *to = p1 - p0 > 16 ? *to + acc : acc;
        }
      }
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < a.tokens * 16; i += DOWN_THREADS) {
    const int t = i >> 4, r = i & 15;
    float y = 0.f;
    for (int j = 0; j < k; j++) {
      const int p = t * k + j;
      if (a.m.dev_router || (uint32_t)a.ids[p] < (uint32_t)a.m.experts) y += a.weights[p] * part[p * 16 + r];
    }
    if (r0 + r < H) ((typename T::elem *)a.y)[t * a.ys + r0 + r] = (typename T::elem)y;
  }
}

template <typename T, int KS>
void up(const Args &a, int groups, hipStream_t s) {
  if (a.m.hidden == UP_WAVES * KS * 32)
    k_moe_up<T, KS, true><<<groups, UP_THREADS, 0, s>>>(a);
  else
    k_moe_up<T, KS, false><<<groups, UP_THREADS, 0, s>>>(a);
}

template <typename T>
hipError_t run(const Args &a, hipStream_t s) {
  const int route = a.m.dev_router ? a.e_pad / 16 * ((a.tokens + 15) / 16) : 1;
  k_moe_route<T><<<route, ROUTE_THREADS, 0, s>>>(a);
  const int64_t units = (int64_t)std::min(a.m.experts, a.tokens * a.m.topk) * (a.m.ffn / 8);
  const int groups = (int)std::min<int64_t>(units, UP_GROUPS);
  const int per = ((a.m.hidden + 31) / 32 + UP_WAVES - 1) / UP_WAVES;  // steps per wave
  if (per <= 2) up<T, 2>(a, groups, s);
  else if (per <= 4) up<T, 4>(a, groups, s);
  else if (per <= 8) up<T, 8>(a, groups, s);
  else up<T, 16>(a, groups, s);
  const int lds = a.tokens * a.m.topk * 64;
  if (lds > 65536) {
    const hipError_t e = hipFuncSetAttribute((const void *)k_moe_down<T>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                             MAX_PAIRS * 64);
    if (e != hipSuccess) return e;
  }
  k_moe_down<T><<<(a.m.hidden + 15) / 16, DOWN_THREADS, lds, s>>>(a);
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
