// New tokens of a layer enter the cache: each head's query and key is normed and
// turned, and K and V go to their places in the pages.
//
// One pass: a value is read and written once, and both steps happen in between,
// in 32 bits.  A head is held by D / 16 neighbouring lanes, two pieces of 8 values
// each, chosen so that the values of a pair meet in one lane whichever way pairs
// are laid out: lanes l < pairs / 8 hold the pieces l and l + pairs / 8, the rest
// the values that stay.  A wave's 64 / (D / 16) heads are whole cache lines.
// The angle position * freq is taken in 64 bits (a position of 2^20 leaves 32 bits
// less than four digits of it), reduced to [-pi, pi] there, and its sine and cosine once
// per token and pair, by a lane each, handed to the token's heads through LDS.
// Bound by the memory: 8,192 tokens of 32 + 4 + 4 heads of 128, 168 MB, 35 us, 4.8
// TB/s; one token 3.6 us, a launch.
#include "hbf_half.h"
#include "hbf_kv_rows.h"
#include "hbf_ops.h"

namespace hbf {
namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64;

struct Args {
  hbf_kv kv;
  hbf_new_tokens nt;
  char *k_pages, *v_pages;  // the layer's planes
  int groups;               // a token's heads, 64 / (head_dim / 16) at a time: those of q, k and v
  int per_wave;             // groups that one wave takes
  int waves;                // waves per token
};

struct Pieces {
  u32x4 a, b;
};

template <typename T>
__device__ __forceinline__ void unpack(u32x4 v, float *x) {
  typename T::x8 e = __builtin_bit_cast(typename T::x8, v);
#pragma unroll
  for (int i = 0; i < 8; i++) x[i] = (float)e[i];
}
template <typename T>
__device__ __forceinline__ u32x4 pack(const float *x) {
  return u32x4{pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3]), pack2<T>(x[4], x[5]), pack2<T>(x[6], x[7])};
}

template <typename T, int D, bool PAIRS>
__global__ __launch_bounds__(THREADS) void k_rotate(Args a) {
  constexpr int LANES = D / 16, HEADS = 64 / LANES;
  __shared__ __align__(16) float2 turns[WAVES][D / 2];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, l = lane % LANES;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(blockIdx.x * WAVES + w);
  const int i = (int)(wave / (uint32_t)a.waves), g0 = (int)(wave - (uint32_t)i * a.waves) * a.per_wave;
  if (i >= a.nt.n) return;  // (a whole wave; no barrier follows)
  const int H = a.nt.heads, Hk = a.nt.kv_heads, all = H + 2 * Hk, g1 = min(g0 + a.per_wave, a.groups);
  const int h8 = a.nt.pairs / 8;
  // this lane's pieces
  const int pa = l < h8 ? l : 2 * h8 + 2 * (l - h8), pb = l < h8 ? l + h8 : pa + 1;
  const char *src[3] = {(const char *)a.nt.dev_q + 2 * (i * a.nt.q_row_stride),
                        (const char *)a.nt.dev_k + 2 * (i * a.nt.k_row_stride),
                        (const char *)a.nt.dev_v + 2 * (i * a.nt.v_row_stride)};
  auto load = [&](int g) {
    const int h = min(g * HEADS + lane / LANES, all - 1);
    const char *p = h < H ? src[0] + 2 * (h * a.nt.q_head_stride)
                  : h < H + Hk ? src[1] + 2 * ((h - H) * a.nt.k_head_stride)
                               : src[2] + 2 * ((h - H - Hk) * a.nt.v_head_stride);
    return Pieces{*(const u32x4 *)(p + pa * 16), *(const u32x4 *)(p + pb * 16)};
  };
  Pieces next = load(g0);
  // the token's place
  const int slot = a.nt.dev_slots[i], pos = a.nt.dev_pos[i];
  int64_t at = -1;
  if ((g1 * HEADS > H)) {
    if (slot >= 0 && slot < a.kv.slots) {
      const int len = a.kv.dev_lens[slot];
      if (len_fits(a.kv, len) && pos >= 0 && pos < len) {
        const int page = row_of(a.kv, a.kv.dev_tables, slot)[pos / a.kv.page_tokens];
        if (page >= 0 && page < a.kv.pages)
          at = page * (int64_t)a.kv.page_stride + (int64_t)(pos % a.kv.page_tokens) * (int64_t)a.kv.token_bytes;
      }
    }
    if (at < 0 && lane == 0) atomicOr(&((KvCtl *)a.kv.dev_ws)->sticky, KV_ERR_ARG);
  }
  if (lane < a.nt.pairs) {
    const double angle = (double)(a.nt.dev_positions ? a.nt.dev_positions[i] : pos) * a.nt.dev_freqs[lane];
    // less the nearest multiple of 2 pi, in two words (2^-106 of it is left out)
    const double k = rint(angle * 0.15915494309189533577);
    const float r = (float)fma(-k, 2.4492935982947064e-16, fma(-k, 6.283185307179586477, angle));
    float sn, cs;
    sincosf(r, &sn, &cs);
    turns[w][lane] = make_float2(cs, sn);
  }
  float weight[2][16];
  const bool norm[2] = {a.nt.dev_q_weight != nullptr, a.nt.dev_k_weight != nullptr};
  const void *wp[2] = {a.nt.dev_q_weight, a.nt.dev_k_weight};
#pragma unroll
  for (int j = 0; j < 2; j++)
    if (norm[j]) {
      unpack<T>(*(const u32x4 *)((const char *)wp[j] + pa * 16), weight[j]);
      unpack<T>(*(const u32x4 *)((const char *)wp[j] + pb * 16), weight[j] + 8);
    }
  wave_lds_fence();
  float2 turn[8];
  if (l < h8) {
#pragma unroll
    for (int j = 0; j < 8; j++) turn[j] = turns[w][PAIRS ? (j < 4 ? pa * 4 + j : pb * 4 + j - 4) : pa * 8 + j];
  }
  for (int g = g0; g < g1; g++) {
    const Pieces now = next;
    if (g + 1 < g1) next = load(g + 1);
    const int h = g * HEADS + lane / LANES;
    const bool key = h >= H, value = h >= H + Hk;
    u32x4 ya = now.a, yb = now.b;
    float x[16], sum = 0.f;
    unpack<T>(now.a, x);
    unpack<T>(now.b, x + 8);
#pragma unroll
    for (int j = 0; j < 16; j++) sum = fmaf(x[j], x[j], sum);
#pragma unroll
    for (int d = 1; d < LANES; d <<= 1) sum += __shfl_xor(sum, d);
    if (!value) {
      if (norm[key]) {
        const float f = 1.f / sqrtf(sum * (1.f / D) + a.nt.eps);
#pragma unroll
        for (int j = 0; j < 16; j++) x[j] = x[j] * f * (key ? weight[1][j] : weight[0][j]);
      }
      if (l < h8) {
#pragma unroll
        for (int j = 0; j < 8; j++) {
          const int p = PAIRS ? 2 * j : j, q = PAIRS ? 2 * j + 1 : j + 8;
          const float u = x[p], v = x[q];
          x[p] = u * turn[j].x - v * turn[j].y;
          x[q] = u * turn[j].y + v * turn[j].x;
        }
      }
      ya = pack<T>(x);
      yb = pack<T>(x + 8);
    }
    char *to = nullptr;
    if (!key)
      to = (char *)a.nt.dev_q_out + 2 * (i * a.nt.out_row_stride + h * a.nt.out_head_stride);
    else if (h < all && at >= 0)
      to = (value ? a.v_pages : a.k_pages) + at + (h - H - (value ? Hk : 0)) * (D * 2);
    if (to) {
      *(u32x4 *)(to + pa * 16) = ya;
      *(u32x4 *)(to + pb * 16) = yb;
    }
  }
}

template <typename T>
hipError_t run(const Args &a, hipStream_t s) {
  const uint32_t blocks = (uint32_t)(((int64_t)a.nt.n * a.waves + WAVES - 1) / WAVES);
  const bool pairs = a.nt.flags & HBF_ROT_PAIRS;
  if (a.nt.head_dim == 128) {
    if (pairs) k_rotate<T, 128, true><<<blocks, THREADS, 0, s>>>(a);
    else k_rotate<T, 128, false><<<blocks, THREADS, 0, s>>>(a);
  } else {
    if (pairs) k_rotate<T, 64, true><<<blocks, THREADS, 0, s>>>(a);
    else k_rotate<T, 64, false><<<blocks, THREADS, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_write_rotated(const hbf_kv &kv, int layer, const hbf_new_tokens &nt, hipStream_t s) {
  Args a{};
  a.kv = kv;
  a.nt = nt;
  a.k_pages = (char *)kv.dev_pool + (uint64_t)(2 * layer) * kv.plane_stride;
  a.v_pages = a.k_pages + kv.plane_stride;
  const int at_once = 64 / (nt.head_dim / 16);
  a.groups = (nt.heads + 2 * nt.kv_heads + at_once - 1) / at_once;
  // Few tokens: a wave for each group of heads, so that they wait side by side (5 groups a token; 256 tokens 4.2 us, by
  // a wave a token 6.9; 1,638 10.1 and 10.1; 8,192 38.9 and 30.2, in a graph).
  a.per_wave = (int64_t)nt.n * a.groups <= 8192 ? 1 : a.groups;
  a.waves = (a.groups + a.per_wave - 1) / a.per_wave;
  return nt.dtype == HBF_BF16 ? run<Bf16>(a, s) : run<Fp16>(a, s);
}

}  // namespace hbf
