// Attention of new tokens, one or a chunk of a prompt per row, over cache pages,
// with an optional window and first tokens that stay visible; and the weight
// that the new queries give each cached token.
//
// o = sum_j p_j v_j / sum_j p_j with p_j = exp(s_j - m), s_j = scale q.k_j, m a
// running maximum, in one pass over the tokens, as in the attention over a shared
// prefix, whose tiles and softmax these kernels use.
//
// A row's queries of one KV head, token after token and in each the G heads of
// the group, are cut into tiles; a workgroup takes one tile and the tokens that
// some query of it sees, as one axis x: the first tokens that stay visible, then
// those of the window.  Only steps at the ends of what a tile sees compare
// positions.  Where tiles are too few to fill the card the axis is cut into
// parts, by the tile's own length as the device finds it, and the last
// workgroup of a tile to finish joins them: one launch, whatever the lengths.
// Tiles of 16 queries are bound by the memory (64 rows of 4,096 tokens, 8 heads
// for each of 4 KV heads of 128: 108 us, 5.0 TB/s of K and V; one row of 4,396: 13.4
// us, of rounds to memory), those of 256 by the matrix cores and the vector
// units together (4,096 tokens behind 4,096: 402 to 433 us by the card, 950 to
// 1,030 TFLOP/s of the pairs that are seen).
//
// A token that one query of a tile sees and another does not has p = 0 for the
// other, and 0 * infinity would be NaN: where a step of that kind holds a value of V
// that is not finite, its products are taken one by one; a tile of 256 that meets
// one is done again, 16 queries at a time.
//
// Weights take each score a second time, once the row's sums are known: tiles
// of 16 leave their scores in scratch (64 rows of up to 4,096 tokens: attention 69 us
// without them, 80 with, and 14 to add them up, 44 from K again), for rows of many
// queries they are computed again.
#include <float.h>
#include <math.h>

#include <algorithm>
#include <numeric>

#include "hbf_attn_tile.h"
#include "hbf_kv_rows.h"
#include "hbf_ops.h"

namespace hbf {
namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64;
constexpr int FEW_TILE = 32;   // tokens of a wave's step where queries are few
constexpr int MANY_TILE = 64;  // tokens staged at a time where they are many
constexpr int HALF = 32;       // tokens of a step there
constexpr int RING = 4;        // staged tiles
constexpr int MANY_Q = 256;    // queries of a tile there
constexpr int MANY_WAVES = MANY_Q / 32, MANY_THREADS = 64 * MANY_WAVES;

constexpr int64_t SCORES_BYTES = 512 << 20;  // most that scores are kept in
constexpr int SCORES_QUERIES = 256;          // and the queries of a row and KV head whose are, as a rule

constexpr float LARGE = 1 << 22;  // of a score, times c: beyond, its rounding shows in exp2

struct Args {
  hbf_kv kv;
  hbf_kv_layer layer;
  hbf_chunk ch;
  int group;          // query heads per KV head
  uint32_t group_mul;  // query / group = query * group_mul >> group_shift, for queries below 2^31
  int group_shift;
  float c;            // |scale| * log2(e), not 0
  uint32_t flip;      // sign bits of two 16-bit values if the scale is negative
  uint32_t window;    // of positions, or all of them
  uint32_t page_mul;  // token / page_tokens = token * page_mul >> page_shift, for tokens below 2^31
  int page_shift;
  int tile_q, tile_shift;  // queries per tile, 16 or MANY_Q, and its logarithm
  int slots;          // places for tiles: tokens * group / tile_q + rows
  int splits;         // most parts of a tile
  bool one_tile;      // a row's queries are one tile of 16, as a rule
  uint32_t spread;    // tiles of few queries: workgroup b takes place and head b * spread % their number
  int part_steps;     // least steps of a part
  float *part;        // [slots][kv_heads][splits][tile_q][head_dim] sums of p v
  float2 *part_ml;    // [slots][kv_heads][splits][tile_q] maximum (of q.k, its sign the scale's) and sum
  float2 *query_ml;   // [tokens][heads] the same of each query, 1 / sum; with weights only
  float *part_w;      // [WEIGH_GROUPS][512] sums of a split's queries
  float *scores;      // [tokens][heads][score_tokens] of few queries with weights, along a tile's axis; or null
  int64_t score_tokens;
  bool keep_scores;
  int32_t *status;
};

__device__ __forceinline__ int token_of(const Args &a, int query) {  // of a row's
  return (int)((uint64_t)(uint32_t)query * a.group_mul >> a.group_shift);
}
__device__ __forceinline__ uint32_t page_index(const Args &a, uint32_t token) {
  return (uint32_t)((uint64_t)token * a.page_mul >> a.page_shift);
}

// One row of the call.
struct Row {
  int start, n;          // its queries
  int slot, len;
  bool ok;               // slot and length are in range
  const int32_t *pages;
};

// Row i's first place among the tiles: rows' tiles lie one behind the other, as
// a row of n tokens that starts at token s has at most (s + n) G / Q - s G / Q + 1.
__device__ __forceinline__ int first_tile(const Args &a, int i, int start) {
  return (int)((int64_t)start * a.group >> a.tile_shift) + i;
}
// The row that place `slot` belongs to: the last whose first place is at most that.  A
// wave asks 64 rows at a time.
__device__ __forceinline__ int find_row(const Args &a, int slot) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = a.ch.rows;  // the answer is in [lo, lo + n)
  while (n > 1) {
    const int step = (n + 63) / 64, i = min(lo + lane * step, lo + n - 1);
    const uint64_t below = __ballot(first_tile(a, i, a.ch.dev_starts[i]) <= slot);
    const int k = max(__builtin_popcountll(below) - 1, 0);  // (lanes past the end ask the last row again)
    const int at = min(k * step, n - 1);
    n = min(step, n - at);
    lo += at;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

__device__ __forceinline__ Row get_row(const Args &a, int i) {
  Row r;
  r.start = a.ch.dev_starts[i];
  r.n = a.ch.dev_starts[i + 1] - r.start;
  if (r.start < 0 || r.n < 0 || r.n > a.ch.tokens || r.start > a.ch.tokens - r.n) r.n = 0;  // (refused elsewhere)
  r.slot = a.ch.dev_slots[i];
  r.ok = r.slot >= 0 && r.slot < a.kv.slots;
  r.len = r.ok ? a.kv.dev_lens[r.slot] : 0;
  r.ok = r.ok && len_fits(a.kv, r.len) && (!a.ch.dev_weights || r.len <= a.ch.weights_tokens);
  r.pages = row_of(a.kv, a.kv.dev_tables, r.ok ? r.slot : 0);
  return r;
}

// What the queries [q0, q1) of a row see, as one axis x of `total` tokens: x < first is
// token x, the others are lo + x - first.
struct View {
  int p0, p1;        // positions of the first and the last query's token
  uint32_t first, lo, total;
  __device__ __forceinline__ uint32_t token(uint32_t x) const { return x < first ? x : lo + (x - first); }
};
__device__ __forceinline__ View view_of(const Args &a, const Row &r, int q0, int q1) {
  View v;
  v.p0 = r.len - r.n + token_of(a, q0);
  v.p1 = r.len - r.n + token_of(a, q1 - 1);
  v.first = v.lo = 0;
  if (a.ch.window > 0 && (int64_t)v.p0 - a.ch.window >= a.ch.sinks) {
    v.first = (uint32_t)a.ch.sinks;
    v.lo = (uint32_t)(v.p0 - a.ch.window + 1);
  }
  v.total = v.p1 < 0 ? 0 : v.first + (uint32_t)(v.p1 + 1) - v.lo;
  return v;
}
__device__ __forceinline__ bool sees(const Args &a, int p, int token) {
  return (token <= p) & (((uint32_t)p - (uint32_t)token < a.window) | (token < a.ch.sinks));
}
// Whether every query of the tile sees all of x .. x + n - 1 (which are below total).
__device__ __forceinline__ bool all_see(const Args &a, const View &v, uint32_t x, uint32_t n) {
  if ((int)v.token(x + n - 1) > v.p0) return false;
  if (a.ch.window == 0 || x + n <= v.first) return true;
  const int t = (int)v.token(max(x, v.first));
  return t > v.p1 - a.ch.window;
}

// A wave's share of the staging: NT tokens, a row of D values each by D / 8
// neighbouring lanes.  Lane i looks up where token i lies, the others ask it.
template <int D, int NT>
struct Places {
  static constexpr int LANES = D / 8, AT_ONCE = 64 / LANES, PASSES = NT / AT_ONCE;
  int page = 0;
  bool bad = false;

  // x .. of [.., x1): their page ids (past x1: of its last token).
  __device__ __forceinline__ void find(const Args &a, const View &v, const int32_t *pages, uint32_t x, uint32_t x1) {
    if (NT < 64 && (threadIdx.x & 63) >= NT) return;
    page = pages[page_index(a, v.token(min(x + (threadIdx.x & 63), x1 - 1)))];
  }
  // Bytes from page 0 to this lane's token's row.
  __device__ __forceinline__ int64_t place(const Args &a, const View &v, uint32_t x, uint32_t x1, int head) {
    if (page < 0 || page >= a.layer.pages) {  // noted; page 0 is read instead
      bad = true;
      page = 0;
    }
    const uint32_t token = v.token(min(x + (threadIdx.x & 63), x1 - 1));
    const uint32_t in_page = token - page_index(a, token) * (uint32_t)a.layer.page_tokens;
    return 2 * (page * a.layer.page_stride + in_page * a.layer.token_stride + head * a.layer.head_stride);
  }
};
__device__ __forceinline__ int64_t from_lane(int64_t v, int lane) {
  return (int64_t)((uint64_t)(uint32_t)__shfl((int)(v >> 32), lane) << 32 | (uint32_t)__shfl((int)v, lane));
}

template <int D, int NT, bool V, bool ONCE>
struct Stage : Places<D, NT> {
  using P = Places<D, NT>;
  u32x4 k[P::PASSES], v[P::PASSES];

  __device__ __forceinline__ void load(const Args &a, const View &vw, uint32_t x, uint32_t x1, int head) {
    const int lane = threadIdx.x & 63;
    const int64_t at = P::place(a, vw, x, x1, head);
#pragma unroll
    for (int j = 0; j < P::PASSES; j++) {
      const int64_t mine = from_lane(at, j * P::AT_ONCE + lane / P::LANES) + lane % P::LANES * 16;
      const u32x4 *kp = (const u32x4 *)((const char *)a.layer.dev_k + mine);
      const u32x4 *vp = (const u32x4 *)((const char *)a.layer.dev_v + mine);
      if (ONCE) {  // past the caches' order, as nobody else reads them (64 rows of 4,096 tokens 122 -> 110 us)
        k[j] = __builtin_nontemporal_load(kp);
        if (V) v[j] = __builtin_nontemporal_load(vp);
      } else {  // a row's tiles find them there (4 rows of 32 tokens in 4,096: 51 us, 59 the other way)
        k[j] = *kp;
        if (V) v[j] = *vp;
      }
    }
  }
  // To tiles of K and V.  What lies behind the last token may be anything: 0 * NaN
  // must not reach the sums.
  __device__ __forceinline__ void store(char *kt, char *vt, uint32_t x, uint32_t x1) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int j = 0; j < P::PASSES; j++) {
      const int t = j * P::AT_ONCE + lane / P::LANES;
      *(u32x4 *)(kt + k_at<D>(t, lane % P::LANES)) = k[j];
      if (V) *(u32x4 *)(vt + v_at<D>(t, lane % P::LANES)) = x + t < x1 ? v[j] : u32x4{0, 0, 0, 0};
    }
  }
};

// Byte offset of 16-byte piece `piece` of a token in a staged tile of V whose
// readers take four pieces of 4 tokens in one cycle.
template <int D>
__device__ __forceinline__ int v4_at(int token, int piece) {
  return token * (D * 2) + ((piece ^ (D == 128 ? (token & 3) << 2 : (token >> 1 & 1) << 2)) << 4);
}

// The tile that a workgroup works on.
struct Tile {
  Row row;
  View view;
  int q0, q1;       // its queries, of the row's n * G
  int head;         // KV head
  int place, parts, split;
  uint32_t x0, x1;  // its part of the axis
  // Query q0 + i: its token of the call and its head; row i of out and lse.
  __device__ __forceinline__ bool has(int i) const { return q0 + i < q1; }
};
struct Query {
  int token, head, pos;  // head < 0: none
};
__device__ __forceinline__ Query query_of(const Args &a, const Tile &t, int i) {
  if (!t.has(i)) return Query{0, -1, 0};
  const int q = t.q0 + i, tok = token_of(a, q);
  return Query{t.row.start + tok, t.head * a.group + q - tok * a.group, t.row.len - t.row.n + tok};
}

template <typename T, int D>
__device__ __forceinline__ void load_query(const Args &a, Query q, int kgroup, u32x4 *out) {
  const bool none = q.head < 0;
  const char *p = (const char *)a.ch.dev_q + 2 * (none ? 0 : q.token * a.ch.q_row_stride + q.head * a.ch.q_head_stride);
#pragma unroll
  for (int k = 0; k < D / 32; k++) {
    const u32x4 v = *(const u32x4 *)(p + (k * 32 + kgroup * 8) * 2) ^ a.flip;
    out[k] = none ? u32x4{0, 0, 0, 0} : v;
  }
}

// What a query's sums are multiplied with: 1 / l, or 0 where it sees no token, or
// NaN where it met a bad page.
__device__ __forceinline__ float one_over(Query q, float l, bool bad) { return bad ? NAN : q.pos < 0 ? 0.f : 1.f / l; }
// Four of a query's values, from d0 on.
template <typename T>
__device__ __forceinline__ void write_out(const Args &a, Query q, int d0, f32x4 o) {
  typename T::elem *out = (typename T::elem *)a.ch.dev_out + q.token * a.ch.out_row_stride + q.head * a.ch.out_head_stride + d0;
  *(u32x2 *)out = u32x2{pack2<T>(o[0], o[1]), pack2<T>(o[2], o[3])};
}
// A query's lse, and what its weights are computed from; by one thread.
template <typename T>
__device__ __forceinline__ void write_sums(const Args &a, Query q, float m, float l, bool bad) {
  const int64_t at = (int64_t)q.token * a.ch.heads + q.head;
  const bool none = q.pos < 0 && !bad;
  const float sum = l * exp2f(-SHIFT<T>);
  if (a.ch.dev_lse) a.ch.dev_lse[at] = bad ? NAN : none ? -INFINITY : m * a.c * LN2 + logf(sum);
  // a query in error or that sees nothing gives no weight
  if (a.query_ml) a.query_ml[at] = bad || none ? make_float2(0.f, 0.f) : make_float2(m, 1.f / sum);
}

// The products of a step's 32 tokens with V one by one, in 32 bits: a value that a
// query does not see must not meet its 0.  p: the lane's probabilities as they are
// multiplied otherwise; pos: its query's position; at: 1 KiB of LDS of the wave's own.
template <typename T, int D>
__device__ __forceinline__ void products_one_by_one(const Args &a, const View &v, const char *vt, uint32_t x, uint32_t x1,
                                                    u32x4 p, int pos, f32x4 (&o)[D / 16], char *at) {
  typedef typename T::elem e4 __attribute__((ext_vector_type(4)));
  const int lane = threadIdx.x & 63, col = lane & 15, kg = lane >> 4;
#pragma unroll
  for (int u = 0; u < 2; u++)  // [tokens / 4][16 queries][4 tokens]
    *(u32x2 *)(at + ((u * 4 + kg) * 16 + col) * 8) = u32x2{p[u * 2], p[u * 2 + 1]};
  wave_lds_fence();
#pragma unroll 1
  for (int t = 0; t < FEW_TILE && x + t < x1; t++) {
    if (!sees(a, pos, (int)v.token(x + t))) continue;
    const float w = (float)*(const typename T::elem *)(at + ((t >> 2) * 16 + col) * 8 + (t & 3) * 2);
#pragma unroll
    for (int d = 0; d < D / 16; d++) {
      const int n = d * 16 + kg * 4;
      const e4 e = *(const e4 *)(vt + v_at<D>(t, n / 8) + (n % 8) * 2);
#pragma unroll
      for (int k = 0; k < 4; k++) o[d][k] = fmaf(w, (float)e[k], o[d][k]);
    }
  }
  wave_lds_fence();
}
// Whether 16 bytes hold a value that is not finite.
template <typename T>
__device__ __forceinline__ bool not_finite(u32x4 v) {
  constexpr uint32_t E = __is_same(T, Bf16) ? 0x7f80u : 0x7c00u;
  bool f = false;
#pragma unroll
  for (int i = 0; i < 4; i++) f |= (v[i] & E) == E || (v[i] >> 16 & E) == E;
  return f;
}

// A part's sums of query i, four values from d0 on, handed to the workgroup that joins.
__device__ __forceinline__ int64_t part_at(const Args &a, const Tile &t, int split, int i) {
  return (((int64_t)t.place * a.layer.kv_heads + t.head) * a.splits + split) * a.tile_q + i;
}

// The tile's last workgroup joins its parts: D / 4 lanes a query, R queries at
// a time, U parts of each asked for at once (a trip to memory each: of two queries 8, where there are more, 16 of
// one; one row of 8 queries in 79 parts 28.3 -> 22.5 us a call).
template <typename T, int D, int R, int U>
__device__ void join(const Args &a, const Tile &t) {
  constexpr int LANES = D / 4;
  const int AT_ONCE = blockDim.x / LANES;
  const int d0 = threadIdx.x % LANES * 4, mine = threadIdx.x / LANES;
  for (int i0 = mine; i0 < t.q1 - t.q0; i0 += AT_ONCE * R) {
    float m[R], l[R];
    f32x4 o[R];
    bool bad[R] = {};  // a part with a bad page (its maximum is NaN, which no other is)
#pragma unroll
    for (int r = 0; r < R; r++) {
      m[r] = -INFINITY;
      l[r] = 0.f;
      o[r] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    for (int s0 = 0; s0 < t.parts; s0 += U) {
      float2 ml[R][U];
      f32x4 x[R][U];
#pragma unroll
      for (int r = 0; r < R; r++)
#pragma unroll
        for (int u = 0; u < U; u++) {
          const int64_t at = part_at(a, t, min(s0 + u, t.parts - 1), min(i0 + r * AT_ONCE, t.q1 - t.q0 - 1));
          ml[r][u] = a.part_ml[at];
          x[r][u] = *(const f32x4 *)(a.part + at * D + d0);
        }
#pragma unroll
      for (int r = 0; r < R; r++) {
#pragma unroll
        for (int u = 0; u < U; u++) bad[r] |= ml[r][u].x != ml[r][u].x;
        leave_out(ml[r], x[r], s0, 1, t.parts);
        take_parts(a.c, ml[r], x[r], m[r], l[r], o[r]);
      }
    }
#pragma unroll
    for (int r = 0; r < R; r++) {
      const Query q = query_of(a, t, i0 + r * AT_ONCE);
      if (q.head < 0) continue;
      write_out<T>(a, q, d0, o[r] * one_over(q, l[r], bad[r]));
      if (d0 == 0) write_sums<T>(a, q, m[r], l[r], bad[r]);
    }
  }
}
// This workgroup's part is handed over; joined by the tile's last one.
template <typename T, int D>
__device__ void end_part(const Args &a, const Tile &t) {
  stores_done();
  if (!last_of(a.ch.dev_ctl + t.place * a.layer.kv_heads + t.head, (uint32_t)t.parts)) return;
  see_handed();
  if (t.parts <= 8) join<T, D, 2, 8>(a, t);
  else join<T, D, 1, 16>(a, t);
}

// ------------------------------------------------------------ few queries

// 16 queries of a tile, from i0 on, one per column: each of W waves takes 32 tokens
// at a time through LDS of its own, the next ones' loads in flight; the waves
// meet once, at the end.
template <typename T, int D, int W, bool ONCE>
__device__ __forceinline__ void few(const Args &a, const Tile &t, int i0, char *lds) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, col = lane & 15, kg = lane >> 4;
  constexpr int KS = D / 32, DT = D / 16;
  u32x4 qv[KS];
  const Query mine = query_of(a, t, i0 + col);
  const int pos = mine.head < 0 ? t.view.p1 : mine.pos;
  load_query<T, D>(a, mine, kg, qv);
  float *scores = a.scores && mine.head >= 0  // the lane's part of its query's
                      ? a.scores + ((int64_t)mine.token * a.ch.heads + mine.head) * a.score_tokens + kg * 4 : nullptr;
  f32x4 o[1][DT];
  float m[1] = {-INFINITY}, l[1] = {0.f};
#pragma unroll
  for (int d = 0; d < DT; d++) o[0][d] = f32x4{0.f, 0.f, 0.f, 0.f};
  char *kt = lds + w * FEW_TILE * D * 4, *vt = kt + FEW_TILE * D * 2;
  const int32_t *pages = t.row.pages;
  const uint32_t x1 = t.x1;
  uint32_t x = t.x0 + w * FEW_TILE;
  Stage<D, FEW_TILE, true, ONCE> st;
  constexpr uint32_t STEP = W * FEW_TILE;
  if (x < x1) {
    st.find(a, t.view, pages, x, x1);
    st.load(a, t.view, x, x1, t.head);
    st.find(a, t.view, pages, x + STEP, x1);
    while (true) {
      const bool more = x1 - x > STEP;
      const bool whole = x1 - x >= FEW_TILE && all_see(a, t.view, x, FEW_TILE);
      bool odd = false;  // V holds what is not finite, in a step that some query sees in part
      if (!whole) {
#pragma unroll
        for (int j = 0; j < st.PASSES; j++) odd |= x + j * st.AT_ONCE + lane / st.LANES < x1 && not_finite<T>(st.v[j]);
        odd = __any(odd);
      }
      st.store(kt, vt, x, x1);
      wave_lds_fence();
      if (more) {
        st.load(a, t.view, x + STEP, x1, t.head);
        st.find(a, t.view, pages, x + 2 * STEP, x1);
      }
      f32x4 s[1][2];
#pragma unroll
      for (int u = 0; u < 2; u++) {
        s[0][u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < KS; k++) s[0][u] = T::mfma(*(const u32x4 *)(kt + k_at<D>(u * 16 + col, k * 4 + kg)), qv[k], s[0][u]);
      }
      if (!whole)
#pragma unroll
        for (int u = 0; u < 2; u++)
#pragma unroll
          for (int i = 0; i < 4; i++) {
            const uint32_t xx = x + u * 16 + kg * 4 + i;
            if (xx >= x1 || !sees(a, pos, (int)t.view.token(xx))) s[0][u][i] = -INFINITY;
          }
      if (scores) {
        *(f32x4 *)(scores + x) = s[0][0];
        *(f32x4 *)(scores + x + 16) = s[0][1];
      }
      softmax_step<T, 1, 2, DT>(s, a.c, m, l, o);
      const u32x4 p = p_operand<T>(s[0][0], s[0][1]);
      if (odd) {  // (in the wave's own K, which is done with)
        products_one_by_one<T, D>(a, t.view, vt, x, x1, p, pos, o[0], kt);
      } else {
#pragma unroll
        for (int d = 0; d < DT; d++) o[0][d] = T::mfma(v_operand<D>(vt, kg * 4, 16 + kg * 4, d, lane), p, o[0][d]);
      }
      wave_lds_fence();
      if (!more) break;
      x += STEP;
    }
  }
  // the waves' parts become one, through LDS
  constexpr int RS = D + 4;  // a query's row, padded against bank conflicts
  float *ro = (float *)lds;  // [W][16][RS], then the maxima and sums
  float2 *rml = (float2 *)(lds + W * 16 * RS * 4);
  const bool any_bad = __syncthreads_or(st.bad);
  if (any_bad && threadIdx.x == 0 && a.status) *a.status = HBF_EINVAL;
  const float lq = across_rows(l[0], SUM_OP);
  if (kg == 0) rml[w * 16 + col] = make_float2(m[0], lq);
#pragma unroll
  for (int d = 0; d < DT; d++) *(f32x4 *)(ro + (w * 16 + col) * RS + d * 16 + kg * 4) = o[0][d];
  __syncthreads();
  constexpr int PER = W * 64 / 16;  // threads per query
  const int n = threadIdx.x / PER, d0 = threadIdx.x % PER * 4;
  const Query qq = query_of(a, t, i0 + n);
  if (qq.head >= 0) {
    float mx = -INFINITY, sum = 0.f;
#pragma unroll
    for (int i = 0; i < W; i++) mx = fmaxf(mx, rml[i * 16 + n].x);
    const float ref = mx == -INFINITY ? 0.f : mx;
    float f[W];
#pragma unroll
    for (int i = 0; i < W; i++) {
      f[i] = __builtin_amdgcn_exp2f((rml[i * 16 + n].x - ref) * a.c);
      sum += f[i] * rml[i * 16 + n].y;
    }
    const int64_t at = t.parts > 1 ? part_at(a, t, t.split, i0 + n) : 0;
#pragma unroll
    for (int d = d0; d < D; d += PER * 4) {
      f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < W; i++) v += f[i] * *(const f32x4 *)(ro + (i * 16 + n) * RS + d);
      if (t.parts > 1) hand_over((f32x4 *)(a.part + at * D + d), v);
      else write_out<T>(a, qq, d, v * one_over(qq, sum, any_bad));
    }
    if (d0 == 0 && t.parts == 1) write_sums<T>(a, qq, mx, sum, any_bad);
    if (d0 == 0 && t.parts > 1) hand_over(a.part_ml + at, any_bad ? make_float2(NAN, NAN) : make_float2(mx, sum));
  }
  __syncthreads();
}

// ------------------------------------------------------------ many queries

// op over the two lanes that hold the same column of a 32 x 32 tile, in both of them.
template <typename F>
__device__ __forceinline__ float across_halves(float x, F op) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto both = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const uint32_t a = both[0], b = both[1];
  return op(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}

// A tile of up to MANY_Q queries, 32 for each of eight waves, two on each SIMD, and 64
// tokens staged for all of them (128 queries, four waves, 32 tokens at a time and two
// workgroups a CU: 173 us instead of 180 on windows of 1,024, 442 instead of 417 on
// 4,096 tokens behind 4,096).  Steps of 32 tokens are one ahead of each other:
// while the scores of step h become probabilities on the vector units, the matrix
// cores multiply h - 1's probabilities with V, then K of h + 1 with the queries.
template <typename T, int D>
struct Many {
  static constexpr int KS = D / 16, DT = D / 32;
  static constexpr int TILE_BYTES = MANY_TILE * D * 2;      // of K, then as much of V
  static constexpr int NT = MANY_TILE / MANY_WAVES;         // tokens of a tile that a wave stages
  static constexpr int GROUP = 64 / NT;                     // tiles whose places it looks up at a time, a lane a token
  static constexpr int LANES = D / 8, AT_ONCE = 64 / LANES, PASSES = NT / AT_ONCE;
  const Args &a;
  const Tile &t;
  char *lds;
  uint32_t lds0;
  int lane, w, col, hf;
  int page = 0;
  int from, last;   // the query sees x < a.ch.sinks and from <= x, both below last
  bool bad = false, odd = false;
  int64_t at;       // bytes to the row of this lane's token of the group
  u32x4 qv[KS], p[2], kk[KS], vv[DT][2];
  f32x16 o[DT];
  float m = -INFINITY, ref = 0.f, l = 0.f;

  __device__ __forceinline__ Many(const Args &a, const Tile &t, char *lds) : a(a), t(t), lds(lds) {
    lane = threadIdx.x & 63, w = threadIdx.x >> 6, col = lane & 31, hf = lane >> 5;
    lds0 = lds_address(lds);
  }
  __device__ __forceinline__ void load_queries() {
    const Query qq = query_of(a, t, w * 32 + col);
    const bool none = qq.head < 0;
    const int pos = none ? t.view.p1 : qq.pos;
    last = (int)min((int64_t)pos + 1 - t.view.lo + t.view.first, (int64_t)t.x1);
    from = a.ch.window ? (int)max((int64_t)pos + 1 - a.ch.window - t.view.lo + t.view.first, (int64_t)0) : 0;
    const char *from = (const char *)a.ch.dev_q + 2 * (none ? 0 : qq.token * a.ch.q_row_stride + qq.head * a.ch.q_head_stride);
#pragma unroll
    for (int k = 0; k < KS; k++) {
      const u32x4 v = *(const u32x4 *)(from + (k * 16 + hf * 8) * 2) ^ a.flip;
      qv[k] = none ? u32x4{0, 0, 0, 0} : v;
    }
#pragma unroll
    for (int d = 0; d < DT; d++)
#pragma unroll
      for (int i = 0; i < 16; i++) o[d][i] = 0.f;
  }
  // This lane's token of the tiles from `tile` on (past the part: its last one).
  __device__ __forceinline__ uint32_t token(int tile) const {
    return t.view.token(min(t.x0 + (tile + lane / NT) * MANY_TILE + w * NT + lane % NT, t.x1 - 1));
  }
  __device__ __forceinline__ void find(int tile) { page = t.row.pages[page_index(a, token(tile))]; }
  __device__ __forceinline__ void place(int tile) {
    if (page < 0 || page >= a.layer.pages) {  // noted; page 0 is read instead
      bad = true;
      page = 0;
    }
    const uint32_t tok = token(tile), in_page = tok - page_index(a, tok) * (uint32_t)a.layer.page_tokens;
    at = 2 * (page * a.layer.page_stride + in_page * a.layer.token_stride + t.head * a.layer.head_stride);
  }
  // A tile on its way to LDS: 2 PASSES loads of the wave.
  __device__ __forceinline__ void stage(int tile) {
    if (tile % GROUP == 0 && tile > 0) {
      place(tile);
      find(tile + GROUP);
    }
    const uint32_t kt = lds0 + tile % RING * 2 * TILE_BYTES, vt = kt + TILE_BYTES;
    int64_t row[PASSES];
#pragma unroll
    for (int j = 0; j < PASSES; j++) row[j] = from_lane(at, tile % GROUP * NT + j * AT_ONCE + lane / LANES);
#pragma unroll
    for (int j = 0; j < PASSES; j++) {
      const int first = w * NT + j * AT_ONCE;  // of the wave's first lanes
      const int mine = first + lane / LANES, piece = lane % LANES * 16;
      to_lds((const char *)a.layer.dev_k + row[j] + (piece ^ (k_at<D>(mine, 0) - mine * (D * 2))), kt + first * (D * 2));
      to_lds((const char *)a.layer.dev_v + row[j] + (piece ^ (v4_at<D>(mine, 0) - mine * (D * 2))), vt + first * (D * 2));
    }
  }
  __device__ __forceinline__ void read_k(int tile, int first) {
    const char *kt = lds + tile % RING * 2 * TILE_BYTES;
#pragma unroll
    for (int k = 0; k < KS; k++) kk[k] = *(const u32x4 *)(kt + k_at<D>(first + col, k * 2 + hf));
  }
  __device__ __forceinline__ void read_v(int tile, int first) {
    const char *vt = lds + tile % RING * 2 * TILE_BYTES + TILE_BYTES;
    const int i = lane & 15, half = (i & 1) << 3, r = first + hf * 4 + (i >> 2);
#pragma unroll
    for (int d = 0; d < DT; d++)
#pragma unroll
      for (int k = 0; k < 2; k++) {
        const int piece = d * 4 + ((lane >> 4 & 1) << 1) + ((i & 3) >> 1);
        const u32x2 x = read_transposed(vt + v4_at<D>(r + k * 16, piece) + half);
        const u32x2 y = read_transposed(vt + v4_at<D>(r + k * 16 + 8, piece) + half);
        vv[d][k] = u32x4{x[0], x[1], y[0], y[1]};
      }
  }
  __device__ __forceinline__ void scores(f32x16 &s) {
#pragma unroll
    for (int i = 0; i < 16; i++) s[i] = 0.f;
#pragma unroll
    for (int k = 0; k < KS; k++) s = T::mfma32(kk[k], qv[k], s);
  }
  __device__ __forceinline__ void add_values() {
#pragma unroll
    for (int k = 0; k < 2; k++)
#pragma unroll
      for (int d = 0; d < DT; d++) o[d] = T::mfma32(vv[d][k], p[k], o[d]);
  }
  __device__ __forceinline__ void nothing_pending() {
    p[0] = p[1] = u32x4{0, 0, 0, 0};
#pragma unroll
    for (int d = 0; d < DT; d++) vv[d][0] = vv[d][1] = u32x4{0, 0, 0, 0};
  }
  // Whether every query sees all of tile i.
  __device__ __forceinline__ bool whole(int i) const {
    const uint32_t x = t.x0 + i * MANY_TILE;
    return t.x1 - x >= MANY_TILE && all_see(a, t.view, x, MANY_TILE);
  }
  // Scores of the tokens from x on that their query does not see, or that are none.
  __device__ __forceinline__ void mask(f32x16 &s, uint32_t x) const {
    const uint32_t first = below(a.ch.sinks - (int)min(x, (uint32_t)INT32_MAX));
    const uint32_t keep = (below(last - (int)x) & (~below(from - (int)x) | first)) >> 4 * hf;
#pragma unroll
    for (int i = 0; i < 16; i++) {
      const float v = s[i];
      const uint32_t k = (uint32_t)__builtin_amdgcn_sbfe((int)keep, i / 4 * 8 + i % 4, 1);
      s[i] = __uint_as_float((__float_as_uint(v) & k) | (0xff800000u & ~k));
    }
  }
  // Bits 0 .. n - 1 of 32.
  static __device__ __forceinline__ uint32_t below(int n) { return (uint32_t)((uint64_t(1) << min(max(n, 0), 32)) - 1); }
  // A tile that is not whole: whether its V holds what is not finite (0 * infinity would reach the sums).
  __device__ __forceinline__ void look(int tile) {
    const char *vt = lds + tile % RING * 2 * TILE_BYTES + TILE_BYTES;
#pragma unroll 1
    for (int i = threadIdx.x * 16; i < TILE_BYTES; i += MANY_THREADS * 16) odd |= not_finite<T>(*(const u32x4 *)(vt + i));
  }
  // The running maximum takes the scores in, as in softmax_step: a probability is
  // exp2(s c + ref) with ref = SHIFT - m c, rounded; o and l are relative to ref as it is, so that its rounding
  // cancels, but for scores so large that it passes exp2's range: these go the slow way.  PENDING: of the step
  // before, probabilities and values wait in p and vv; they are relative to the old maximum.
  template <bool PENDING>
  __device__ __forceinline__ void maximum(const f32x16 &s) {
    float mx = s[0];
#pragma unroll
    for (int i = 1; i < 16; i++) mx = fmaxf(mx, s[i]);
    if (__any((mx - m) * a.c > LAZY)) {  // (none seen, none here: NaN, false)
      if (PENDING) add_values();
      const float top = fmaxf(m, across_halves(mx, MAX_OP));
      const float now = top == -INFINITY ? 0.f : fmaf(-top, a.c, SHIFT<T>);  // nothing seen yet: every p is exp2(-infinity)
      odd |= fabsf(now) > LARGE;
      const float alpha = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(now - ref);  // (0: nothing is summed yet)
      m = top;
      ref = now;
      l *= alpha;
#pragma unroll
      for (int d = 0; d < DT; d++) o[d] *= alpha;
      if (PENDING) nothing_pending();
    }
  }
  // What o and l are multiplied with to be relative to the maximum itself.
  __device__ __forceinline__ float to_maximum() const {
    return m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(fmaf(-m, a.c, SHIFT<T> - ref));
  }
  // Of 16 tokens of the step, k = 0 or 1.
  __device__ __forceinline__ void probabilities(const f32x16 &s, int k) {
    float e[8];
#pragma unroll
    for (int i = 0; i < 8; i++) {
      e[i] = __builtin_amdgcn_exp2f(fmaf(s[k * 8 + i], a.c, ref));
      l += e[i];
    }
    p[k] = u32x4{pack2<T>(e[0], e[1]), pack2<T>(e[2], e[3]), pack2<T>(e[4], e[5]), pack2<T>(e[6], e[7])};
  }
  // One step, of tokens first .. of a tile: its scores are in s and its maximum is
  // known; the next one's (there are more), of a tile that is `whole` or not, go to sn.
  __device__ __forceinline__ void step(const f32x16 &s, f32x16 &sn, int tile, int first, bool more, bool whole) {
    const int next = first ? tile + 1 : tile;
    read_k(next, HALF - first);
    add_values();
    probabilities(s, 0);
    scores(sn);
    read_v(tile, first);
    probabilities(s, 1);
    // a product, what it needs from LDS, some of the vector units' work, and so on: left to itself the compiler puts
    // most of the products side by side
#pragma unroll
    for (int z = 0; z < KS + 2 * DT; z++) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      __builtin_amdgcn_sched_group_barrier(0x002, 6, 0);
      __builtin_amdgcn_sched_group_barrier(0x400, 1, 0);
    }
    if (!more) return;
    if (!whole) mask(sn, t.x0 + next * MANY_TILE + HALF - first);
    maximum<true>(sn);
  }
  // Waits until at most `tiles` (0 .. 2) of the staged tiles are on their way, in every wave.
  __device__ __forceinline__ void arrived(int tiles) {
    constexpr int N = 2 * PASSES;
    if (tiles <= 0) loads_left<0>();
    else if (tiles == 1) loads_left<N>();
    else loads_left<2 * N>();
    __syncthreads();
  }
  // All of the part's tokens.
  __device__ __forceinline__ void run() {
    const int n = (int)((t.x1 - t.x0 + MANY_TILE - 1) / MANY_TILE);
    find(0);
    load_queries();  // (on their way beside the page ids)
    place(0);
    find(GROUP);
    for (int i = 0; i < min(n, RING - 1); i++) stage(i);
    nothing_pending();
    f32x16 sa, sb;
    arrived(min(n, RING - 1) - 1);
    bool now = whole(0);
    if (!now) look(0);
    read_k(0, 0);
    scores(sa);
    if (!now) mask(sa, t.x0);
    maximum<false>(sa);
    for (int i = 0; i < n; i++) {
      step(sa, sb, i, 0, true, now);
      // the next tile is there, the one behind it may be on its way, and one more goes where all are done with
      arrived(min(n - 2 - i, 1));
      if (i + RING - 1 < n) stage(i + RING - 1);
      const bool more = i + 1 < n;
      now = more && whole(i + 1);
      if (more && !now) look(i + 1);
      step(sb, sa, i, HALF, more, now);
    }
    add_values();
  }
};

// Returns whether the tile has to be done again, the slow way.
template <typename T, int D>
__device__ __forceinline__ bool many(const Args &a, const Tile &t, char *lds) {
  Many<T, D> z(a, t, lds);
  constexpr int DT = D / 32;
  z.run();
  bool any_bad = false;
  if (__syncthreads_or(z.odd || z.bad)) {
    if (__syncthreads_or(z.odd)) return true;
    any_bad = __syncthreads_or(z.bad);
  }
  if (any_bad && threadIdx.x == 0 && a.status) *a.status = HBF_EINVAL;
  const int i = z.w * 32 + z.col;
  const Query qq = query_of(a, t, i);
  const float fix = z.to_maximum(), l = across_halves(z.l, SUM_OP);
  auto four = [&](int d, int g) { return f32x4{z.o[d][g * 4], z.o[d][g * 4 + 1], z.o[d][g * 4 + 2], z.o[d][g * 4 + 3]}; };
  if (t.parts > 1) {
    if (qq.head < 0) return false;
    const int64_t at = part_at(a, t, t.split, i);
#pragma unroll
    for (int d = 0; d < DT; d++)
#pragma unroll
      for (int g = 0; g < 4; g++) hand_over((f32x4 *)(a.part + at * D + d * 32 + g * 8 + z.hf * 4), four(d, g) * fix);
    if (z.hf == 0) hand_over(a.part_ml + at, any_bad ? make_float2(NAN, NAN) : make_float2(z.m, l * fix));
  } else {
    if (z.hf == 0 && qq.head >= 0) write_sums<T>(a, qq, z.m, l * fix, any_bad);
    // by way of LDS, of which every wave is done with its own eighth's tiles: a lane holds parts of a row, and a
    // store of 8 bytes a row takes as long as one of all of it
    const float f = one_over(qq, l, any_bad);
    char *mine = lds + z.w * 32 * D * 2;
#pragma unroll
    for (int d = 0; d < DT; d++)
#pragma unroll
      for (int g = 0; g < 4; g++) {
        const f32x4 v = four(d, g) * f;
        *(u32x2 *)(mine + k_at<D>(z.col, d * 4 + g) + z.hf * 8) = u32x2{pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3])};
      }
    wave_lds_fence();
    constexpr int LANES = D / 8;
#pragma unroll
    for (int j = 0; j < 32; j += 64 / LANES) {
      const int row = j + z.lane / LANES, piece = z.lane % LANES;
      const u32x4 v = *(const u32x4 *)(mine + k_at<D>(row, piece));
      const Query to = query_of(a, t, z.w * 32 + row);
      if (to.head >= 0)
        *(u32x4 *)((typename T::elem *)a.ch.dev_out + to.token * a.ch.out_row_stride + to.head * a.ch.out_head_stride +
                   piece * 8) = v;
    }
  }
  return false;
}

template <int D, int W>
constexpr int few_bytes() {  // K and V of each wave; or the waves' join
  return W * FEW_TILE * D * 4 > W * 16 * ((D + 4) * 4 + 8) ? W * FEW_TILE * D * 4 : W * 16 * ((D + 4) * 4 + 8);
}
template <int D, bool MANY>
constexpr int lds_bytes() {
  return !MANY ? few_bytes<D, WAVES>() : std::max(RING * 2 * MANY_TILE * D * 2, few_bytes<D, MANY_WAVES>());
}

// Tiles of 16 queries (ONCE: one a row, as a rule), or of MANY_Q.
template <typename T, int D, bool MANY, bool ONCE>
__global__ __launch_bounds__(MANY ? MANY_THREADS : THREADS, MANY ? 1 : 2) void k_chunk(Args a) {
  __shared__ __align__(16) char lds[lds_bytes<D, MANY>()];
  const int kv_heads = a.layer.kv_heads;
  uint32_t b = blockIdx.x;
  if (b == 0) {  // starts that decrease or leave the queries
    bool bad = false;
    for (int i = threadIdx.x; i < a.ch.rows; i += blockDim.x) {
      const int s = a.ch.dev_starts[i], e = a.ch.dev_starts[i + 1];
      bad |= s < 0 || e < s || e > a.ch.tokens;
    }
    if (bad && a.status) *a.status = HBF_EINVAL;
  }
  Tile t;
  const uint32_t groups = (uint32_t)a.slots * kv_heads;
  t.split = b / groups;
  b -= t.split * groups;
  if (!MANY) b = (uint32_t)((uint64_t)b * a.spread % groups);
  t.place = a.slots - 1 - (int)(b / kv_heads);  // the longest first
  t.head = b % kv_heads;
  const int i = find_row(a, t.place);
  t.row = get_row(a, i);
  const int64_t q0 = (int64_t)(t.place - first_tile(a, i, t.row.start)) * a.tile_q, n = (int64_t)t.row.n * a.group;
  if (q0 < 0 || q0 >= n) return;
  t.q0 = (int)q0;
  t.q1 = (int)min(n, q0 + a.tile_q);
  t.view = view_of(a, t.row, t.q0, t.q1);
  constexpr uint32_t step = MANY ? MANY_TILE : WAVES * FEW_TILE;
  const uint32_t steps = t.row.ok ? (t.view.total + step - 1) / step : 0;
  if (steps == 0) {  // nothing is seen, or the row is in error
    if (t.split) return;
    if (!t.row.ok && threadIdx.x == 0 && a.status) *a.status = HBF_EINVAL;
    for (int j = threadIdx.x; j < (t.q1 - t.q0) * (D / 4); j += blockDim.x) {
      Query q = query_of(a, t, j / (D / 4));
      const float v = t.row.ok ? 0.f : NAN;
      write_out<T>(a, q, j % (D / 4) * 4, f32x4{v, v, v, v});
      if (j % (D / 4) == 0) write_sums<T>(a, q, 0.f, 0.f, !t.row.ok);
    }
    return;
  }
  uint32_t most = (steps + a.part_steps - 1) / a.part_steps;
  // (a part's steps and the trips that its join takes: as many of one as of the other, about; one row of 20,000 tokens
  // 22.5 -> 19 us)
  if (!MANY) most = min(most, (uint32_t)(3.5f * __builtin_sqrtf((float)steps)) + 1);
  const uint32_t parts = min(most, (uint32_t)a.splits);
  const uint32_t each = (steps + parts - 1) / parts;
  t.parts = (int)((steps + each - 1) / each);
  if (t.split >= t.parts) return;
  t.x0 = (uint32_t)t.split * each * step;
  t.x1 = min(t.view.total, t.x0 + each * step);
  if constexpr (!MANY) {
    few<T, D, WAVES, ONCE>(a, t, 0, lds);
  } else if (many<T, D>(a, t, lds)) {
    for (int i = 0; i < t.q1 - t.q0; i += 16) few<T, D, MANY_WAVES, false>(a, t, i, lds);
  }
  if (t.parts > 1) end_part<T, D>(a, t);
}

// ------------------------------------------------------------ weights

// The last row that names row i0's slot, or -1 where i0 is not the first; for a workgroup, by way of `after` in LDS.
__device__ __forceinline__ int last_of_slot(const Args &a, int i0, int slot, int *after) {
  if (threadIdx.x == 0) *after = i0;
  bool before = false;
  int last = i0;
  for (int j = threadIdx.x; j < a.ch.rows; j += THREADS)
    if (a.ch.dev_slots[j] == slot) {
      before |= j < i0;
      last = max(last, j);
    }
  if (__syncthreads_or(before)) return -1;
  if (last > i0) atomicMax(after, last);
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(*after);
}

// What a row's queries gave each token, from the scores that attention left: a
// thread a token, with W = 4 a thread of each wave, whose queries are every fourth
// 8 (14 us of rounds to memory for 64 rows of up to 4,096 tokens, 17 MB).  A slot's
// rows are taken by the first of them, one after another, and their queries in
// order.
template <int W>
__global__ __launch_bounds__(THREADS) void k_weigh_scores(Args a, int blocks) {
  constexpr int AHEAD = 8;  // queries whose scores are on their way together; of one tile
  constexpr int TOKENS = THREADS / W;
  __shared__ int after;
  __shared__ float part[W][TOKENS];
  const int w = W == 1 ? 0 : threadIdx.x / TOKENS, mine = threadIdx.x % TOKENS;
  int b = blockIdx.x;
  const int head = b % a.layer.kv_heads;
  b /= a.layer.kv_heads;
  const int i0 = b % a.ch.rows, block = b / a.ch.rows;
  const int slot = a.ch.dev_slots[i0];
  const Row first = get_row(a, i0);
  if (!first.ok || block * TOKENS >= first.len) return;
  const int last = last_of_slot(a, i0, slot, &after);
  if (last < 0) return;
  float *out = a.ch.dev_weights + slot * a.ch.weights_slot_stride + head * a.ch.weights_head_stride;
  for (int64_t j0 = (int64_t)block * TOKENS; j0 < first.len; j0 += (int64_t)blocks * TOKENS) {
    const uint32_t j = (uint32_t)j0 + mine;
    const bool there = j < (uint32_t)first.len;
    const float old = there && w == 0 ? out[j] : 0.f;
    float sum = 0.f;
    for (int i = i0; i <= last; i++) {
      if (i > i0 && a.ch.dev_slots[i] != slot) continue;
      const Row r = i == i0 ? first : get_row(a, i);
      const int n = r.n * a.group;
      for (int q = w * AHEAD; q < n; q += W * AHEAD) {
        const int q0 = q & ~(a.tile_q - 1);  // its tile, whose axis the scores lie along
        const View v = view_of(a, r, q0, min(q0 + a.tile_q, n));
        const uint32_t x = j < v.first ? j : j - v.lo + v.first;
        const bool has = there && (j < v.first || j >= v.lo) && x < v.total;
        if (!__any(has)) continue;
        const float *from = a.scores + x;
        float s[AHEAD];
        float2 ml[AHEAD];
        bool seen[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; k++) {
          const int qq = min(q + k, n - 1), tok = token_of(a, qq);
          const int64_t at = (int64_t)(r.start + tok) * a.ch.heads + head * a.group + qq - tok * a.group;
          ml[k] = a.query_ml[at];
          s[k] = has ? from[at * a.score_tokens] : 0.f;
          seen[k] = has & (q + k < n) & sees(a, r.len - r.n + tok, (int)j);
        }
#pragma unroll
        for (int k = 0; k < AHEAD; k++)  // (not seen: the score is -infinity, but the query's sums may be NaN)
          sum += seen[k] && ml[k].y != 0.f ? __builtin_amdgcn_exp2f((s[k] - ml[k].x) * a.c) * ml[k].y : 0.f;
      }
    }
    if (W > 1) {
      part[w][mine] = sum;
      __syncthreads();
      sum = 0.f;
      if (w == 0)
        for (int k = 0; k < W; k++) sum += part[k][mine];
      __syncthreads();
    }
    if (w == 0 && there && sum != 0.f) out[j] = old + sum;  // (NaN too; a token that nobody sees has 0)
  }
}

// The same from K, where scores would take too much, and for more rows of many
// queries than k_weigh_many takes: a wave takes 32 tokens at a time, through LDS of
// its own, the next ones on their way, and meets 16 queries at a time; a token's
// sum over the lanes that hold its scores is taken once.  (64 rows of up to 4,096
// tokens: 44 us, 3.1 TB/s of K.)
template <typename T, int D>
__global__ __launch_bounds__(THREADS, 3) void k_weigh(Args a, int blocks) {
  constexpr int KS = D / 32, NT = FEW_TILE;
  __shared__ __align__(16) char lds[WAVES * NT * D * 2];
  __shared__ int after;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, col = lane & 15, kg = lane >> 4;
  int b = blockIdx.x;
  const int head = b % a.layer.kv_heads;
  b /= a.layer.kv_heads;
  const int i0 = b % a.ch.rows, block = b / a.ch.rows;
  const int slot = a.ch.dev_slots[i0], last = last_of_slot(a, i0, slot, &after);
  if (last < 0) return;
  const Row first = get_row(a, i0);
  if (!first.ok) return;
  const uint32_t len = (uint32_t)first.len, step = (uint32_t)blocks * WAVES * NT;
  char *kt = lds + w * NT * D * 2;
  float *out = a.ch.dev_weights + slot * a.ch.weights_slot_stride + head * a.ch.weights_head_stride;
  View all;
  all.first = all.lo = 0;
  all.total = len;
  // The queries, 16 of a row from q0 on: theirs of this lane's column, and the row's own.
  struct Queries {
    u32x4 v[KS];
    float2 ml;
    int pos;
  };
  auto load = [&](const Tile &t, int q0) {
    Queries z;
    const Query q = query_of(a, t, q0 + col);
    load_query<T, D>(a, q, kg, z.v);
    z.ml = q.head < 0 ? make_float2(0.f, 0.f) : a.query_ml[(int64_t)q.token * a.ch.heads + q.head];
    z.pos = q.pos;
    return z;
  };
  auto tile_of = [&](int i) {
    Tile t;
    t.row = get_row(a, i);
    t.head = head;
    t.q0 = 0;
    t.q1 = t.row.n * a.group;
    return t;
  };
  const Tile own = tile_of(i0);
  const bool one = last == i0 && own.q1 <= 16;  // as a rule: they are loaded once
  Queries mine = load(own, 0);
  uint32_t x = ((uint32_t)block * WAVES + w) * NT;
  if (x >= len) return;  // (a whole wave; no barrier follows)
  Stage<D, NT, false, true> st;
  st.find(a, all, first.pages, x, len);
  st.load(a, all, x, len, head);
  st.find(a, all, first.pages, min(x + step, len - 1), len);
  while (true) {
    const bool more = len - x > step;
    const uint32_t x1 = min(x + NT, len);
    // lane col < 8 of a group of 16 answers for token x + 16 (col / 4) + 4 kg + col % 4
    const uint32_t at = x + (col >> 2 & 1) * 16 + kg * 4 + (col & 3);
    const bool writes = col < 8 && at < x1;
    const float old = writes ? out[at] : 0.f;
    st.store(kt, nullptr, x, len);
    wave_lds_fence();
    if (more) {
      st.load(a, all, x + step, len, head);
      st.find(a, all, first.pages, min(x + 2 * step, len - 1), len);
    }
    f32x4 sum[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    bool seen = false;
    auto meet = [&](const Queries &z) {
      f32x4 s[2];
#pragma unroll
      for (int u = 0; u < 2; u++) {
        s[u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < KS; k++) s[u] = T::mfma(*(const u32x4 *)(kt + k_at<D>(u * 16 + col, k * 4 + kg)), z.v[k], s[u]);
      }
#pragma unroll
      for (int u = 0; u < 2; u++)
#pragma unroll
        for (int i = 0; i < 4; i++) {
          const uint32_t j = x + u * 16 + kg * 4 + i;
          const float p = __builtin_amdgcn_exp2f((s[u][i] - z.ml.x) * a.c) * z.ml.y;
          sum[u][i] += ((z.ml.y != 0.f) & (j < x1) & sees(a, z.pos, (int)j)) ? p : 0.f;
        }
    };
    for (int i = i0; i <= last; i++) {
      if (i > i0 && a.ch.dev_slots[i] != slot) continue;
      const Tile t = i == i0 ? own : tile_of(i);
      const int p = t.row.len - t.row.n;  // the first query's position
      // queries of tokens [t0, t1) may see one of these
      const int t0 = max(0, (int)x - p);
      int t1 = t.row.n;
      if (a.ch.window > 0 && (int)x >= a.ch.sinks) t1 = (int)min((int64_t)t1, (int64_t)x1 - 1 + a.ch.window - p);
      if (t0 >= t1) continue;
      seen = true;
      if (one) meet(mine);
      else
        for (int q0 = t0 * a.group & ~15; q0 < t1 * a.group; q0 += 16) meet(load(t, q0));
    }
    float v = 0.f;
#pragma unroll
    for (int u = 0; u < 2; u++)
#pragma unroll
      for (int i = 0; i < 4; i++) {
        const float all16 = sum_of_row(sum[u][i]);
        v = col == u * 4 + i ? all16 : v;
      }
    if (writes && seen) out[at] = old + v;
    wave_lds_fence();
    if (!more) break;
    x += step;
  }
}

// And for rows of many queries.  A workgroup holds 512 tokens' K in
// registers, 64 a wave, and meets 64 queries at a time, which all waves read from
// LDS.  A block's queries are cut into `splits` as far as the card has room; the last
// split to finish adds their sums up, in order.  Bound by issue, products and
// exponentials by turns (2,048 tokens behind 2,048, 32 heads of 128: 108 us, the
// products alone 41).
constexpr int BLOCK = 64 * MANY_WAVES, Q_TILE = 64, Q_RING = 3;
constexpr int WEIGH_GROUPS = 256;      // workgroups: one for each CU
constexpr int WEIGH_ROWS = 512;        // most rows that it takes; more go the way of few queries

template <typename T, int D>
struct Weigh {
  static constexpr int KS = D / 16, TILE_BYTES = Q_TILE * D * 2;
  static constexpr int LANES = D / 8, AT_ONCE = 64 / LANES, NT = Q_TILE / MANY_WAVES, PASSES = NT / AT_ONCE;
  const Args &a;
  char *lds;
  uint32_t lds0;
  int lane, w, col, hf;
  u32x4 kk[2][KS];
  f32x16 sum[2];
  uint32_t j0, j1;  // this wave's tokens
  bool seen;

  __device__ __forceinline__ Weigh(const Args &a, char *lds) : a(a), lds(lds) {
    lane = threadIdx.x & 63, w = threadIdx.x >> 6, col = lane & 31, hf = lane >> 5;
    lds0 = lds_address(lds);
  }
  // K of the wave's tokens, by way of its own part of the LDS.
  __device__ __forceinline__ void load_k(const int32_t *pages, int len, int head) {
    View all;
    all.first = all.lo = 0;
    Places<D, 64> pl;
    const uint32_t x1 = max(j1, j0 + 1), last = (uint32_t)len;  // (a wave without tokens reads some of the row's)
    pl.find(a, all, pages, min(j0, last - 1), min(x1, last));
    const int64_t at = pl.place(a, all, min(j0, last - 1), min(x1, last), head);
    const uint32_t to = lds0 + w * 32 * D * 2;
#pragma unroll
    for (int t = 0; t < 2; t++) {
#pragma unroll
      for (int j = 0; j < 32 / AT_ONCE; j++) {
        const int mine = j * AT_ONCE + lane / LANES;
        to_lds((const char *)a.layer.dev_k + from_lane(at, t * 32 + mine) +
                   (lane % LANES * 16 ^ (k_at<D>(mine, 0) - mine * (D * 2))), to + j * AT_ONCE * D * 2);
      }
      loads_done();
#pragma unroll
      for (int k = 0; k < KS; k++) kk[t][k] = *(const u32x4 *)(lds + w * 32 * D * 2 + k_at<D>(col, k * 2 + hf)) ^ a.flip;
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (read before the next are on their way)
    }
  }
  // Queries base .. of [.., q1) of the row (past them: the last one again) on their way to LDS.
  __device__ __forceinline__ void stage(int start, int head, int base, int q1, int buf) {
#pragma unroll
    for (int j = 0; j < PASSES; j++) {
      const int first = w * NT + j * AT_ONCE, mine = first + lane / LANES;
      const int q = min(base + mine, q1 - 1), tok = token_of(a, q);
      const char *row = (const char *)a.ch.dev_q +
                        2 * ((start + tok) * a.ch.q_row_stride + (head * a.group + q - tok * a.group) * a.ch.q_head_stride);
      to_lds(row + (lane % LANES * 16 ^ (k_at<D>(mine, 0) - mine * (D * 2))), lds0 + buf * TILE_BYTES + first * D * 2);
    }
  }
  __device__ __forceinline__ float2 sums_of(int start, int head, int q, int q1) const {
    if (q >= q1) return make_float2(0.f, 0.f);
    const int tok = token_of(a, q);
    return a.query_ml[(start + tok) * a.ch.heads + head * a.group + q - tok * a.group];
  }
  // 32 tokens' scores with the queries of qv.
  __device__ __forceinline__ f32x16 scores(const u32x4 (&k)[KS], const u32x4 (&qv)[KS]) {
    f32x16 s;
#pragma unroll
    for (int e = 0; e < 16; e++) s[e] = 0.f;
#pragma unroll
    for (int i = 0; i < KS; i++) s = T::mfma32(k[i], qv[i], s);
    return s;
  }
  // Their weights exp2((s - m) c) / l, as ml = (-m c, 1 / l); of a tile that is not WHOLE, ml = (m, 1 / l), and only
  // those whose bit (16 r + e) the lane's query sees.
  template <bool WHOLE>
  __device__ __forceinline__ void add(const f32x16 &s, int r, float2 ml, uint32_t sees) {
#pragma unroll
    for (int e = 0; e < 16; e++) {
      if (WHOLE) {
        sum[r][e] = fmaf(__builtin_amdgcn_exp2f(fmaf(s[e], a.c, ml.x)), ml.y, sum[r][e]);
      } else {
        const float p = __builtin_amdgcn_exp2f((s[e] - ml.x) * a.c) * ml.y;
        sum[r][e] += __int_as_float(__float_as_int(p) & __builtin_amdgcn_sbfe((int)sees, r * 16 + e, 1));
      }
    }
  }
  // Bits 0 .. n - 1.
  static __device__ __forceinline__ uint64_t first_bits(int n) { return n <= 0 ? 0 : ~uint64_t(0) >> (64 - min(n, 64)); }
  // What a query at `pos` sees of the wave's tokens, a bit for each of this lane's scores.
  __device__ __forceinline__ uint32_t seen_bits(int pos) const {
    const int behind = a.ch.window == 0 ? 0 : (int)max((int64_t)pos - a.ch.window + 1 - j0, (int64_t)0);  // tokens before the window
    uint64_t v = first_bits(min(pos + 1, (int)j1) - (int)j0) & (~first_bits(behind) | first_bits(a.ch.sinks - (int)j0));
    v >>= 4 * hf;  // scores of 4 tokens of each 8
    auto pack = [](uint32_t x) {
      x &= 0x0f0f0f0f;
      x = (x | x >> 4) & 0x00ff00ff;
      return (x | x >> 8) & 0xffff;
    };
    return pack((uint32_t)v) | pack((uint32_t)(v >> 32)) << 16;
  }
  // One staged tile: products of 32 tokens and 32 queries, each beside the vector units' work on the one before.
  template <bool WHOLE>
  __device__ __forceinline__ void tile(const char *qt, const float2 (&ml)[2], const uint32_t (&sees)[2]) {
    u32x4 qv[KS];
    auto read = [&](int u) {
#pragma unroll
      for (int k = 0; k < KS; k++) qv[k] = *(const u32x4 *)(qt + k_at<D>(u * 32 + col, k * 2 + hf));
    };
    read(0);
    f32x16 x = scores(kk[0], qv);
    f32x16 y = scores(kk[1], qv);
    add<WHOLE>(x, 0, ml[0], sees[0]);
    read(1);
    x = scores(kk[0], qv);
    add<WHOLE>(y, 1, ml[0], sees[0]);
    y = scores(kk[1], qv);
    add<WHOLE>(x, 0, ml[1], sees[1]);
    add<WHOLE>(y, 1, ml[1], sees[1]);
  }
  // Queries q0 .. q1 - 1 of a row that starts at query `start`, at position p.
  __device__ __forceinline__ void meet(int start, int p, int head, int q0, int q1) {
    const int n = (q1 - q0 + Q_TILE - 1) / Q_TILE;
    __syncthreads();  // (all are done with the LDS)
    stage(start, head, q0, q1, 0);
    if (n > 1) stage(start, head, q0 + Q_TILE, q1, 1);
    float2 ml[2] = {sums_of(start, head, q0 + col, q1), sums_of(start, head, q0 + 32 + col, q1)};
    for (int i = 0, buf = 0; i < n; i++, buf = buf + 1 == Q_RING ? 0 : buf + 1) {
      const int base = q0 + i * Q_TILE, last = min(base + Q_TILE, q1) - 1;
      float2 now[2] = {ml[0], ml[1]};
      loads_done();
      __syncthreads();
      asm volatile("" : "+v"(now[0].x), "+v"(now[0].y), "+v"(now[1].x), "+v"(now[1].y));  // (waited for here, not behind the next loads)
      if (i + 2 < n) stage(start, head, base + 2 * Q_TILE, q1, buf == 0 ? Q_RING - 1 : buf - 1);
      if (i + 1 < n) {
        ml[0] = sums_of(start, head, base + Q_TILE + col, q1);
        ml[1] = sums_of(start, head, base + Q_TILE + 32 + col, q1);
      }
      const int pa = p + token_of(a, base), pb = p + token_of(a, last);  // positions of the first and the last
      // (all that follows is of one wave: no barrier)
      if (j0 >= j1 || (int)j0 > pb) continue;
      if (a.ch.window > 0 && (int)j0 >= a.ch.sinks && (int64_t)j1 - 1 <= (int64_t)pa - a.ch.window) continue;
      seen = true;
      uint32_t sees[2] = {0, 0};
      // where every query sees every token and none is to be left out, nothing is compared
      const float far = fmaxf(fabsf(now[0].x), fabsf(now[1].x)) * a.c;
      if (j1 - j0 == 64 && (int)j1 - 1 <= pa && !__any(now[0].y == 0.f || now[1].y == 0.f || far > LARGE) &&
          (a.ch.window == 0 || (int)j1 <= a.ch.sinks || (int64_t)j0 > (int64_t)pb - a.ch.window)) {
#pragma unroll
        for (int u = 0; u < 2; u++) {  // -m c is rounded: what it is off by goes to the factor
          const float ref = -now[u].x * a.c;
          now[u].y *= __builtin_amdgcn_exp2f(-fmaf(now[u].x, a.c, ref));
          now[u].x = ref;
        }
        tile<true>(lds + buf * TILE_BYTES, now, sees);
      } else {
#pragma unroll
        for (int u = 0; u < 2; u++)
          sees[u] = now[u].y == 0.f ? 0 : seen_bits(p + token_of(a, min(base + u * 32 + col, last)));
        tile<false>(lds + buf * TILE_BYTES, now, sees);
      }
    }
  }
};

template <typename T, int D>
__global__ __launch_bounds__(MANY_THREADS, 1) void k_weigh_many(Args a) {
  using Z = Weigh<T, D>;
  constexpr int LDS = Q_RING * Z::TILE_BYTES > MANY_WAVES * 32 * D * 2 ? Q_RING * Z::TILE_BYTES : MANY_WAVES * 32 * D * 2;
  __shared__ __align__(16) char lds[LDS];
  __shared__ int row_blocks[WEIGH_ROWS], slots[WEIGH_ROWS];
  __shared__ uint32_t scan[MANY_THREADS / 64];
  static_assert(WEIGH_ROWS == MANY_THREADS, "a row a thread");
  const int kv_heads = a.layer.kv_heads;
  // The blocks of rows whose slot no row before names.
  uint32_t units;
  int splits = 1;
  {
    const int i = threadIdx.x;
    int mine = 0;
    slots[i] = i < a.ch.rows ? a.ch.dev_slots[i] : -1;
    __syncthreads();
    if (i < a.ch.rows) {
      const Row r = get_row(a, i);
      mine = r.ok ? (int)(((uint32_t)r.len + BLOCK - 1) / BLOCK) : 0;
      for (int j = 0; j < i; j++)
        if (slots[j] == slots[i]) mine = 0;
    }
    uint32_t total;
    row_blocks[i] = (int)block_scan<MANY_THREADS>((uint32_t)mine, &total, scan);
    __syncthreads();
    units = total * kv_heads;  // (below 2^32: the weights of as many blocks take more memory than the card has)
    if (a.part_w) splits = max(1, min((int)(gridDim.x / max(units, 1u)), 64));
  }
  for (uint32_t u = blockIdx.x; u < units * splits; u += gridDim.x) {
    const int split = u / units, unit = u - split * units, head = unit % kv_heads, b = unit / kv_heads;
    int i0 = 0;  // the last row whose first block is at most b
    for (int hi = a.ch.rows; hi - i0 > 1;) {
      const int mid = (i0 + hi) >> 1;
      if (row_blocks[mid] <= b) i0 = mid; else hi = mid;
    }
    i0 = __builtin_amdgcn_readfirstlane(i0);
    const int slot = __builtin_amdgcn_readfirstlane(slots[i0]);
    const uint32_t base = (uint32_t)__builtin_amdgcn_readfirstlane(b - row_blocks[i0]) * BLOCK;
    const int len = a.kv.dev_lens[slot];  // (in range, or the row has no blocks)
    Z z(a, lds);
    z.j0 = min(base + z.w * 64, (uint32_t)len);
    z.j1 = min(base + z.w * 64 + 64, (uint32_t)len);
    __syncthreads();  // (all are done with the LDS)
    z.load_k(row_of(a.kv, a.kv.dev_tables, slot), len, head);
#pragma unroll
    for (int r = 0; r < 2; r++)
#pragma unroll
      for (int e = 0; e < 16; e++) z.sum[r][e] = 0.f;
    z.seen = false;
    const int end = (int)min(base + BLOCK, (uint32_t)len);
#pragma unroll 1
    for (int i = i0; i < a.ch.rows; i++) {
      if (__builtin_amdgcn_readfirstlane(slots[i]) != slot) continue;
      int start = a.ch.dev_starts[i], n = a.ch.dev_starts[i + 1] - start;
      if (start < 0 || n < 0 || n > a.ch.tokens || start > a.ch.tokens - n) n = 0;  // (refused elsewhere)
      const int p = len - n;  // the first query's position
      // the queries that may see one of the block's tokens
      const int t0 = max(0, (int)base - p);
      int t1 = n;
      if (a.ch.window > 0 && (int)base >= a.ch.sinks) t1 = (int)min((int64_t)n, (int64_t)end - 1 + a.ch.window - p);
      if (t0 >= t1) continue;
      const int q0 = t0 * a.group, q1 = t1 * a.group;
      const int each = ((q1 - q0 + Q_TILE - 1) / Q_TILE + splits - 1) / splits * Q_TILE;
      if (split * each < q1 - q0) z.meet(start, p, head, q0 + split * each, min(q1, q0 + (split + 1) * each));
    }
    // a token's sum over the lanes that hold its scores; then every split's
    float mine = 0.f;  // lane's of a half: the one of r = col / 16, e = col % 16
#pragma unroll
    for (int r = 0; r < 2; r++)
#pragma unroll
      for (int e = 0; e < 16; e++) {
        const float v = sum_of_half(z.sum[r][e]);
        mine = z.col == r * 16 + e ? v : mine;
      }
    float *out = a.ch.dev_weights + slot * a.ch.weights_slot_stride + head * a.ch.weights_head_stride;
    const uint32_t at = z.col / 16 * 32 + z.col % 16 / 4 * 8 + z.hf * 4 + z.col % 4;
    if (splits == 1) {
      if (z.seen && z.j0 + at < z.j1) out[z.j0 + at] += mine;
      continue;
    }
    hand_over(a.part_w + (int64_t)u * BLOCK + z.w * 64 + at, z.seen ? mine : 0.f);
    stores_done();
    if (!last_of(a.ch.dev_ctl + unit, (uint32_t)splits)) continue;
    const uint32_t j = base + threadIdx.x;
    float v = 0.f;
    for (int k = 0; k < splits; k++) v += handed(a.part_w + ((int64_t)k * units + unit) * BLOCK + threadIdx.x);
    if (j < (uint32_t)len && v != 0.f) out[j] += v;  // (NaN too; a token that nobody sees has 0)
  }
}

// Sizes of a call.
Args plan(const hbf_kv &kv, const hbf_kv_layer &layer, const hbf_chunk &ch) {
  Args a{};
  a.kv = kv;
  a.layer = layer;
  a.ch = ch;
  a.group = ch.heads / layer.kv_heads;
  // (the least number that is not 0: as flat as 0 is, and -infinity times it stays that)
  a.c = std::min(std::max(fabsf(ch.scale) * LOG2E, FLT_TRUE_MIN), FLT_MAX);
  a.flip = ch.scale < 0 ? 0x80008000u : 0;
  a.window = ch.window ? (uint32_t)ch.window : UINT32_MAX;
  // with M = ceil(2^k / d), k = 31 + ceil(log2 d): x * M / 2^k is at most x / 2^31 < 1 / d above x / d
  auto by = [](int d, uint32_t *mul, int *shift) {
    for (*shift = 0; (1 << *shift) < d; ++*shift) {
    }
    *shift += 31;
    *mul = (uint32_t)(((uint64_t(1) << *shift) + d - 1) / d);
  };
  by(layer.page_tokens, &a.page_mul, &a.page_shift);
  by(a.group, &a.group_mul, &a.group_shift);
  const int64_t queries = (int64_t)ch.tokens * a.group;
  const int64_t rows = std::max(ch.rows, 1);
  const int64_t longest = (int64_t)kv.table_cols * kv.page_tokens;
  // Tiles of 256 queries or of 16.  Those of 256 read K and V a sixteenth as often, but take 15 us to begin and end, and
  // more to join their parts: for calls of more than 16 queries a row and KV head, of at least 450,000 tokens met by
  // tiles of 16 (4 rows of 128 queries in 1,000 tokens, 4 KV heads, in tiles of 16 and of 256: 17 and 36 us; 16 of 64
  // in 2,000: 54 and 47), whose tiles of 256, in parts of 1,024 tokens, take half of the card at least (one row of
  // 2,048 queries in 2,000: 36 and 68; four of 256 in 4,096: 45 and 71, in 8,192: 102 and 79).  As a rule a row is no
  // longer than 16,384, however wide its table is.
  const int64_t likely = std::min<int64_t>(longest, 16384);
  const bool many = queries > 16 * rows && (queries >> 4) * layer.kv_heads * likely >= 450000 &&
                    std::max(rows, queries >> 8) * layer.kv_heads * (likely / 1024 + 1) >= 128;
  a.tile_shift = many ? 8 : 4;
  a.tile_q = 1 << a.tile_shift;
  a.slots = (int)(queries >> a.tile_shift) + ch.rows;
  // Parts, so that the workgroups of all rows, if they are long, have room at once, two on a CU where the tiles are
  // many (8 rows behind 16,000 tokens, 32 tiles: in 160 workgroups 52 us, in 256 65; 24 behind 10,000, 96 tiles: in 480
  // 86, in 672 101); a tile takes as many as its length gives work for.  Where the tiles alone are a card's worth, a
  // part has 8 steps at least (64 rows of 500 tokens 24.1 -> 19.1 us, of 1,500 47.3 -> 48.5).
  const int64_t groups = std::max<int64_t>((int64_t)a.slots * layer.kv_heads, 1);  // (0 without rows)
  // Rows of one tile each: places that no row needs may come at a fixed distance, and in the places' order they would
  // leave some of the XCDs, which take workgroups by turns, idle (64 rows of 16 queries behind 2,048 tokens 91 -> 77
  // us).  A row's tiles stay side by side, as they read the same (one row of 2,048 queries 36 us, spread 54).
  a.one_tile = queries <= 16 * rows;
  a.spread = 1;
  if (a.one_tile)
    for (a.spread = (uint32_t)(groups * 0.618) | 1; std::gcd((uint64_t)a.spread, (uint64_t)groups) != 1; a.spread += 2) {
    }
  const int64_t tiles = std::max(rows, queries >> a.tile_shift) * layer.kv_heads;  // that there are, as a rule
  a.part_steps = many ? 16 : tiles >= 256 ? 8 : 2;
  const int64_t steps = longest / ((many ? MANY_TILE : WAVES * FEW_TILE) * a.part_steps) + 1;
  const int64_t parts = many || tiles < 64 ? 256 / groups : 512 / tiles;
  a.splits = groups > (int64_t)HBF_CHUNK_CTL_WORDS || !ch.dev_ctl ? 1 : (int)std::max<int64_t>(1, std::min(steps, parts));
  // Weights of tiles of 16: from the scores that attention leaves, where they take no more than SCORES_BYTES (64 rows of
  // 8 queries behind 4,096 tokens: 146 us, from K again 173) and are not many for each token (one row of 256 queries
  // behind 4,096: 35, from K by k_weigh_many 39; of 1,024 behind 1,000, the other way: 134 and 42).
  const int64_t held = std::min<int64_t>(longest, ch.weights_tokens);
  a.score_tokens = (held + WAVES * FEW_TILE - 1) / (WAVES * FEW_TILE) * (WAVES * FEW_TILE);
  a.keep_scores = ch.dev_weights && !many && queries <= SCORES_QUERIES * rows &&
                  ch.tokens * (int64_t)ch.heads * a.score_tokens * 4 <= SCORES_BYTES;
  return a;
}

size_t up256(size_t x) { return (x + 255) & ~size_t(255); }
size_t carve(Args &a, char *ws) {
  size_t o = 0;
  auto take = [&](size_t bytes) {
    char *r = ws + o;
    o = up256(o + bytes);
    return (void *)r;
  };
  if (a.splits > 1) {
    const size_t n = (size_t)a.slots * a.layer.kv_heads * a.splits * a.tile_q;
    a.part = (float *)take(n * a.layer.head_dim * 4);
    a.part_ml = (float2 *)take(n * 8);
  }
  if (a.ch.dev_weights) {
    a.query_ml = (float2 *)take((size_t)a.ch.tokens * a.ch.heads * 8);
    if (a.keep_scores) a.scores = (float *)take((size_t)a.ch.tokens * a.ch.heads * a.score_tokens * 4);
    if (!a.keep_scores && !a.one_tile && a.ch.dev_ctl) a.part_w = (float *)take((size_t)WEIGH_GROUPS * BLOCK * 4);
  }
  return std::max(o, size_t(256));
}

template <typename T, int D>
hipError_t run(const Args &a, hipStream_t s) {
  const uint32_t blocks = (uint32_t)((int64_t)a.slots * a.layer.kv_heads * a.splits);
  if (a.tile_q == MANY_Q) k_chunk<T, D, true, false><<<blocks, MANY_THREADS, 0, s>>>(a);
  else if (a.one_tile) k_chunk<T, D, false, true><<<blocks, THREADS, 0, s>>>(a);
  else k_chunk<T, D, false, false><<<blocks, THREADS, 0, s>>>(a);
  if (a.ch.dev_weights) {
    const int64_t groups = (int64_t)a.ch.rows * a.layer.kv_heads;
    const int64_t longest = std::min<int64_t>((int64_t)a.kv.table_cols * a.kv.page_tokens, a.ch.weights_tokens);
    if (a.keep_scores) {
      const int64_t each = std::max<int64_t>(1, std::min<int64_t>(longest / (a.one_tile ? THREADS : 64) + 1, 8192 / groups));
      if (a.one_tile) k_weigh_scores<1><<<(uint32_t)(groups * each), THREADS, 0, s>>>(a, (int)each);
      else k_weigh_scores<WAVES><<<(uint32_t)(groups * each), THREADS, 0, s>>>(a, (int)each);
      return hipGetLastError();
    }
    if (!a.one_tile && a.ch.rows <= WEIGH_ROWS) {
      k_weigh_many<T, D><<<WEIGH_GROUPS, MANY_THREADS, 0, s>>>(a);
      return hipGetLastError();
    }
    const int64_t most = longest / (WAVES * FEW_TILE) + 1;
    const int each = (int)std::max<int64_t>(1, std::min<int64_t>(most, 2048 / groups));
    k_weigh<T, D><<<(uint32_t)(groups * each), THREADS, 0, s>>>(a, each);
  }
  return hipGetLastError();
}

}  // namespace

size_t chunk_ws_bytes(const hbf_kv &kv, const hbf_kv_layer &layer, const hbf_chunk &ch) {
  Args a = plan(kv, layer, ch);
  return carve(a, nullptr);
}

hipError_t launch_chunk(const hbf_kv &kv, const hbf_kv_layer &layer, const hbf_chunk &ch, int32_t *status, void *ws,
                        hipStream_t s) {
  Args a = plan(kv, layer, ch);
  a.status = status;
  carve(a, (char *)ws);
  if (layer.dtype == HBF_BF16) return layer.head_dim == 128 ? run<Bf16, 128>(a, s) : run<Bf16, 64>(a, s);
  return layer.head_dim == 128 ? run<Fp16, 128>(a, s) : run<Fp16, 64>(a, s);
}

}  // namespace hbf
