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
// Tiles of few queries are bound by memory, those of many by the matrix cores
// and the LDS.
//
// A token that one query of a tile sees and another does not has p = 0 for the
// other, and 0 * infinity would be NaN: where a step of that kind holds a value of V
// that is not finite, its products are taken one by one.
#include <float.h>
#include <math.h>

#include <algorithm>

#include "hbf_attn_tile.h"
#include "hbf_kv_rows.h"
#include "hbf_ops.h"

namespace hbf {
namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64;
constexpr int FEW_TILE = 32;   // tokens of a wave's step where queries are few
constexpr int MANY_TILE = 64;  // tokens staged where they are many
constexpr int MANY_Q = 128, FEW_Q = 16;  // queries per tile

struct Args {
  hbf_kv kv;
  hbf_kv_layer layer;
  hbf_chunk ch;
  int group;          // query heads per KV head
  float c;            // |scale| * log2(e), not 0
  uint32_t flip;      // sign bits of two 16-bit values if the scale is negative
  uint32_t page_mul;  // token / page_tokens = token * page_mul >> page_shift, for tokens below 2^31
  int page_shift;
  int tile_q, tile_shift;  // queries per tile, FEW_Q or MANY_Q, and its logarithm
  int slots;          // places for tiles: tokens * group / tile_q + rows
  int splits;         // most parts of a tile
  int part_steps;     // least steps of a part
  float *part;        // [slots][kv_heads][splits][tile_q][head_dim] sums of p v
  float2 *part_ml;    // [slots][kv_heads][splits][tile_q] maximum (of q.k, its sign the scale's) and sum
  float2 *query_ml;   // [tokens][heads] the same of each query, 1 / sum; with weights only
  int32_t *status;
};

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
  v.p0 = r.len - r.n + q0 / a.group;
  v.p1 = r.len - r.n + (q1 - 1) / a.group;
  v.first = v.lo = 0;
  if (a.ch.window > 0 && (int64_t)v.p0 - a.ch.window >= a.ch.sinks) {
    v.first = (uint32_t)a.ch.sinks;
    v.lo = (uint32_t)(v.p0 - a.ch.window + 1);
  }
  v.total = v.p1 < 0 ? 0 : v.first + (uint32_t)(v.p1 + 1) - v.lo;
  return v;
}
__device__ __forceinline__ bool sees(const Args &a, int p, int token) {
  return token <= p && (a.ch.window == 0 || token > p - a.ch.window || token < a.ch.sinks);
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

template <int D, int NT>
struct Stage : Places<D, NT> {
  using P = Places<D, NT>;
  u32x4 k[P::PASSES], v[P::PASSES];

  __device__ __forceinline__ void load(const Args &a, const View &vw, uint32_t x, uint32_t x1, int head) {
    const int lane = threadIdx.x & 63;
    const int64_t at = P::place(a, vw, x, x1, head);
#pragma unroll
    for (int j = 0; j < P::PASSES; j++) {
      const int64_t mine = from_lane(at, j * P::AT_ONCE + lane / P::LANES) + lane % P::LANES * 16;
      k[j] = *(const u32x4 *)((const char *)a.layer.dev_k + mine);
      v[j] = *(const u32x4 *)((const char *)a.layer.dev_v + mine);
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
      *(u32x4 *)(vt + v_at<D>(t, lane % P::LANES)) = x + t < x1 ? v[j] : u32x4{0, 0, 0, 0};
    }
  }
};

// The same share loaded past the registers, straight into LDS; there after loads_done().
template <int D, int NT>
struct StageLds : Places<D, NT> {
  using P = Places<D, NT>;
  // To tokens first .. of a tile (past x1: its last one again).
  __device__ __forceinline__ void load(const Args &a, const View &vw, uint32_t x, uint32_t x1, int head, uint32_t kt,
                                       uint32_t vt, int first) {
    const int lane = threadIdx.x & 63;
    const int64_t at = P::place(a, vw, x, x1, head);
    int64_t row[P::PASSES];
#pragma unroll
    for (int j = 0; j < P::PASSES; j++) row[j] = from_lane(at, j * P::AT_ONCE + lane / P::LANES);
#pragma unroll
    for (int j = 0; j < P::PASSES; j++) {
      const int t = first + j * P::AT_ONCE;  // of the wave's first lanes
      const int mine = t + lane / P::LANES, piece = lane % P::LANES * 16;
      to_lds((const char *)a.layer.dev_k + row[j] + (piece ^ (k_at<D>(mine, 0) - mine * (D * 2))), kt + t * (D * 2));
      to_lds((const char *)a.layer.dev_v + row[j] + (piece ^ (v_at<D>(mine, 0) - mine * (D * 2))), vt + t * (D * 2));
    }
  }
};

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
  const int q = t.q0 + i, tok = q / a.group;
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

// Four of a query's values, from d0 on, from its sums; none: it sees no token.
// lead: the one thread that writes lse.
template <typename T>
__device__ __forceinline__ void write_out(const Args &a, Query q, int d0, f32x4 o, float m, float l, bool bad, bool lead) {
  const bool none = q.pos < 0 && !bad;
  if (bad) l = NAN;
  o *= none ? 0.f : 1.f / l;
  typename T::elem *out = (typename T::elem *)a.ch.dev_out + q.token * a.ch.out_row_stride + q.head * a.ch.out_head_stride + d0;
  *(u32x2 *)out = u32x2{pack2<T>(o[0], o[1]), pack2<T>(o[2], o[3])};
  if (!lead) return;
  const int64_t at = (int64_t)q.token * a.ch.heads + q.head;
  const float sum = l * exp2f(-SHIFT<T>);
  if (a.ch.dev_lse) a.ch.dev_lse[at] = none ? -INFINITY : m * a.c * LN2 + logf(sum);
  // a query in error or that sees nothing gives no weight
  if (a.query_ml) a.query_ml[at] = bad || none ? make_float2(0.f, 0.f) : make_float2(m, 1.f / sum);
}

// A step's products with V one by one, in 32 bits: a value that a query does not see
// must not meet its 0.  s: the lane's probabilities; pos: its queries' positions.
template <typename T, int D, int QT, int U>
__device__ void products_one_by_one(const Args &a, const View &v, const char *vt, uint32_t x, uint32_t x1,
                                    const f32x4 (&s)[QT][U], const int (&pos)[QT], f32x4 (&o)[QT][D / 16]) {
  const int lane = threadIdx.x & 63, col = lane & 15, kg = lane >> 4;
#pragma unroll
  for (int u = 0; u < U; u++)
#pragma unroll
    for (int i = 0; i < 4; i++)
#pragma unroll 1
      for (int g = 0; g < 4; g++) {
        const int t = u * 16 + g * 4 + i;
        if (x + t >= x1) break;
        const int token = (int)v.token(x + t);
#pragma unroll
        for (int q = 0; q < QT; q++) {
          const float p = __shfl(s[q][u][i], g * 16 + col);
          if (!sees(a, pos[q], token)) continue;
#pragma unroll
          for (int d = 0; d < D / 16; d++) {
            const int at = d * 16 + kg * 4;
            const u32x2 w = *(const u32x2 *)(vt + v_at<D>(t, at / 8) + (at % 8) * 2);
            typedef typename T::elem e4 __attribute__((ext_vector_type(4)));
            const e4 e = __builtin_bit_cast(e4, w);
#pragma unroll
            for (int k = 0; k < 4; k++) o[q][d][k] = fmaf(p, (float)e[k], o[q][d][k]);
          }
        }
      }
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
// a time, U parts of each asked for at once.
template <typename T, int D>
__device__ void join(const Args &a, const Tile &t) {
  constexpr int LANES = D / 4, AT_ONCE = THREADS / LANES, R = 2, U = 8;
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
      if (q.head >= 0) write_out<T>(a, q, d0, o[r], m[r], l[r], bad[r], d0 == 0);
    }
  }
}
// This workgroup's part is handed over; joined by the tile's last one.
template <typename T, int D>
__device__ void end_part(const Args &a, const Tile &t) {
  stores_done();
  if (!last_of(a.ch.dev_ctl + t.place * a.layer.kv_heads + t.head, (uint32_t)t.parts)) return;
  see_handed();
  join<T, D>(a, t);
}

// ------------------------------------------------------------ few queries

// A tile of at most 16 QT queries, one per column: each wave takes 32 tokens at a
// time through LDS of its own, the next ones' loads in flight; the waves meet
// once, at the end.
template <typename T, int D, int QT>
__device__ void few(const Args &a, const Tile &t, char *lds) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, col = lane & 15, kg = lane >> 4;
  constexpr int KS = D / 32, DT = D / 16;
  u32x4 qv[QT][KS];
  int pos[QT];
#pragma unroll
  for (int q = 0; q < QT; q++) {
    const Query qq = query_of(a, t, q * 16 + col);
    pos[q] = qq.head < 0 ? t.view.p1 : qq.pos;
    load_query<T, D>(a, qq, kg, qv[q]);
  }
  f32x4 o[QT][DT];
  float m[QT], l[QT];
#pragma unroll
  for (int q = 0; q < QT; q++) {
    m[q] = -INFINITY;
    l[q] = 0.f;
#pragma unroll
    for (int d = 0; d < DT; d++) o[q][d] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  char *kt = lds + w * FEW_TILE * D * 4, *vt = kt + FEW_TILE * D * 2;
  const int32_t *pages = t.row.pages;
  const uint32_t x1 = t.x1;
  uint32_t x = t.x0 + w * FEW_TILE;
  Stage<D, FEW_TILE> st;
  constexpr uint32_t STEP = WAVES * FEW_TILE;
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
      f32x4 s[QT][2];
#pragma unroll
      for (int u = 0; u < 2; u++) {
#pragma unroll
        for (int q = 0; q < QT; q++) s[q][u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < KS; k++) {
          const u32x4 kk = *(const u32x4 *)(kt + k_at<D>(u * 16 + col, k * 4 + kg));
#pragma unroll
          for (int q = 0; q < QT; q++) s[q][u] = T::mfma(kk, qv[q][k], s[q][u]);
        }
      }
      if (!whole)
#pragma unroll
        for (int u = 0; u < 2; u++)
#pragma unroll
          for (int i = 0; i < 4; i++) {
            const uint32_t xx = x + u * 16 + kg * 4 + i;
            const int token = (int)t.view.token(xx);
#pragma unroll
            for (int q = 0; q < QT; q++)
              if (xx >= x1 || !sees(a, pos[q], token)) s[q][u][i] = -INFINITY;
          }
      softmax_step<T, QT, 2, DT>(s, a.c, m, l, o);
      if (odd) {
        products_one_by_one<T, D, QT, 2>(a, t.view, vt, x, x1, s, pos, o);
      } else {
        u32x4 p[QT];
#pragma unroll
        for (int q = 0; q < QT; q++) p[q] = p_operand<T>(s[q][0], s[q][1]);
#pragma unroll
        for (int d = 0; d < DT; d++) {
          const u32x4 v = v_operand<D>(vt, kg * 4, 16 + kg * 4, d, lane);
#pragma unroll
          for (int q = 0; q < QT; q++) o[q][d] = T::mfma(v, p[q], o[q][d]);
        }
      }
      wave_lds_fence();
      if (!more) break;
      x += STEP;
    }
  }
  // the waves' parts become one: 16 queries at a time through LDS
  constexpr int RS = D + 4;  // a query's row, padded against bank conflicts
  float *ro = (float *)lds;  // [WAVES][16][RS], then the maxima and sums
  float2 *rml = (float2 *)(lds + WAVES * 16 * RS * 4);
  const bool any_bad = __syncthreads_or(st.bad);
  if (any_bad && threadIdx.x == 0 && a.status) *a.status = HBF_EINVAL;
#pragma unroll
  for (int q = 0; q < QT; q++) {
    const float lq = across_rows(l[q], SUM_OP);
    if (kg == 0) rml[w * 16 + col] = make_float2(m[q], lq);
#pragma unroll
    for (int d = 0; d < DT; d++) *(f32x4 *)(ro + (w * 16 + col) * RS + d * 16 + kg * 4) = o[q][d];
    __syncthreads();
    constexpr int PER = THREADS / 16;  // threads per query
    const int n = threadIdx.x / PER, d0 = threadIdx.x % PER * 4;
    const Query qq = query_of(a, t, q * 16 + n);
    if (qq.head >= 0) {
      float mx = -INFINITY, sum = 0.f;
#pragma unroll
      for (int i = 0; i < WAVES; i++) mx = fmaxf(mx, rml[i * 16 + n].x);
      const float ref = mx == -INFINITY ? 0.f : mx;
      float f[WAVES];
#pragma unroll
      for (int i = 0; i < WAVES; i++) {
        f[i] = __builtin_amdgcn_exp2f((rml[i * 16 + n].x - ref) * a.c);
        sum += f[i] * rml[i * 16 + n].y;
      }
      const int64_t at = t.parts > 1 ? part_at(a, t, t.split, q * 16 + n) : 0;
#pragma unroll
      for (int d = d0; d < D; d += PER * 4) {
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < WAVES; i++) v += f[i] * *(const f32x4 *)(ro + (i * 16 + n) * RS + d);
        if (t.parts > 1) hand_over((f32x4 *)(a.part + at * D + d), v);
        else write_out<T>(a, qq, d, v, mx, sum, any_bad, d == 0);
      }
      if (d0 == 0 && t.parts > 1) hand_over(a.part_ml + at, any_bad ? make_float2(NAN, NAN) : make_float2(mx, sum));
    }
    __syncthreads();
  }
  if (t.parts > 1) end_part<T, D>(a, t);
}

// ------------------------------------------------------------ many queries

// A tile of up to MANY_Q queries: 64 tokens staged for four waves of 32 queries each.
template <typename T, int D>
__device__ void many(const Args &a, const Tile &t, char *lds) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, col = lane & 15, kg = lane >> 4;
  static_assert(MANY_Q == 32 * WAVES, "queries per wave");
  constexpr int KS = D / 32, DT = D / 16, QT = 2, U = MANY_TILE / 16;
  constexpr int TILE_BYTES = MANY_TILE * D * 2;
  constexpr int NT = MANY_TILE / WAVES;  // tokens of a tile that a wave stages
  constexpr uint32_t STEP = MANY_TILE;
  const int32_t *pages = t.row.pages;
  const uint32_t lds0 = lds_address(lds), x1 = t.x1;
  StageLds<D, NT> st;
  st.find(a, t.view, pages, t.x0 + w * NT, x1);
  u32x4 qv[QT][KS];
  int pos[QT];
#pragma unroll
  for (int q = 0; q < QT; q++) {
    const Query qq = query_of(a, t, w * 32 + q * 16 + col);
    pos[q] = qq.head < 0 ? t.view.p1 : qq.pos;
    load_query<T, D>(a, qq, kg, qv[q]);
  }
  st.load(a, t.view, t.x0 + w * NT, x1, t.head, lds0, lds0 + TILE_BYTES, w * NT);
  f32x4 o[QT][DT];
  float m[QT], l[QT];
#pragma unroll
  for (int q = 0; q < QT; q++) {
    m[q] = -INFINITY;
    l[q] = 0.f;
#pragma unroll
    for (int d = 0; d < DT; d++) o[q][d] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  st.find(a, t.view, pages, t.x0 + STEP + w * NT, x1);
  loads_done();
  __syncthreads();
  int cur = 0;
  for (uint32_t x = t.x0;;) {
    char *kt = lds + cur * 2 * TILE_BYTES, *vt = kt + TILE_BYTES;
    const bool whole = x1 - x >= MANY_TILE && all_see(a, t.view, x, MANY_TILE);
    bool odd = false;
    if (!whole) {  // 0 * infinity must not reach the sums: no V behind the last token, and see what is before it
      for (int i = threadIdx.x * 16; i < TILE_BYTES; i += THREADS * 16) {
        u32x4 *at = (u32x4 *)(vt + i);
        if (x + i / (D * 2) >= x1) *at = u32x4{0, 0, 0, 0};
        else odd |= not_finite<T>(*at);
      }
      odd = __syncthreads_or(odd);
    }
    // Operands come from LDS one group of products ahead of their use: left to
    // itself the compiler waits for each group's reads right before it.
    u32x4 kk[2][KS];
    auto read_k = [&](int u) {
#pragma unroll
      for (int k = 0; k < KS; k++) kk[u & 1][k] = *(const u32x4 *)(kt + k_at<D>(u * 16 + col, k * 4 + kg));
    };
    f32x4 s[QT][U];
    read_k(0);
#pragma unroll
    for (int u = 0; u < U; u++) {
      if (u + 1 < U) read_k(u + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int q = 0; q < QT; q++) s[q][u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KS; k++)
#pragma unroll
        for (int q = 0; q < QT; q++) s[q][u] = T::mfma(kk[u & 1][k], qv[q][k], s[q][u]);
      __builtin_amdgcn_sched_barrier(0);
    }
    const bool more = x1 - x > STEP;
    if (more) {  // the next step's tile, here so that its addresses are found beside the products
      const uint32_t next = lds0 + (cur ^ 1) * 2 * TILE_BYTES;
      st.load(a, t.view, x + STEP + w * NT, x1, t.head, next, next + TILE_BYTES, w * NT);
      if (x1 - x > 2 * STEP) st.find(a, t.view, pages, x + 2 * STEP + w * NT, x1);
    }
    if (!whole)
#pragma unroll
      for (int u = 0; u < U; u++)
#pragma unroll
        for (int i = 0; i < 4; i++) {
          const uint32_t xx = x + u * 16 + kg * 4 + i;
          const int token = (int)t.view.token(xx);
#pragma unroll
          for (int q = 0; q < QT; q++)
            if (xx >= x1 || !sees(a, pos[q], token)) s[q][u][i] = -INFINITY;
        }
    u32x4 vv[2][U / 2];
    auto read_v = [&](int d) {
#pragma unroll
      for (int u = 0; u < U / 2; u++)
        vv[d & 1][u] = v_operand<D>(vt, u * 32 + kg * 4, u * 32 + 16 + kg * 4, d, lane);
    };
    softmax_step<T, QT, U, DT>(s, a.c, m, l, o);
    if (odd) {
      products_one_by_one<T, D, QT, U>(a, t.view, vt, x, x1, s, pos, o);
    } else {
      u32x4 p[QT][U / 2];
#pragma unroll
      for (int q = 0; q < QT; q++)
#pragma unroll
        for (int u = 0; u < U / 2; u++) p[q][u] = p_operand<T>(s[q][2 * u], s[q][2 * u + 1]);
      read_v(0);
#pragma unroll
      for (int d = 0; d < DT; d++) {
        if (d + 1 < DT) read_v(d + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = 0; u < U / 2; u++)
#pragma unroll
          for (int q = 0; q < QT; q++) o[q][d] = T::mfma(vv[d & 1][u], p[q][u], o[q][d]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if (!more) break;
    x += STEP;
    loads_done();
    __syncthreads();
    cur ^= 1;
  }
  const bool any_bad = __syncthreads_or(st.bad);
  if (any_bad && threadIdx.x == 0 && a.status) *a.status = HBF_EINVAL;
#pragma unroll
  for (int q = 0; q < QT; q++) {
    const int i = w * 32 + q * 16 + col;
    const Query qq = query_of(a, t, i);
    const float lq = across_rows(l[q], SUM_OP);
    if (qq.head < 0) continue;
    if (t.parts > 1) {
      const int64_t at = part_at(a, t, t.split, i);
#pragma unroll
      for (int d = 0; d < DT; d++) hand_over((f32x4 *)(a.part + at * D + d * 16 + kg * 4), o[q][d]);
      if (kg == 0) hand_over(a.part_ml + at, any_bad ? make_float2(NAN, NAN) : make_float2(m[q], lq));
    } else {
#pragma unroll
      for (int d = 0; d < DT; d++) write_out<T>(a, qq, d * 16 + kg * 4, o[q][d], m[q], lq, any_bad, d == 0 && kg == 0);
    }
  }
  if (t.parts > 1) end_part<T, D>(a, t);
}

template <int D>
constexpr int lds_bytes() {
  const int many_b = 4 * MANY_TILE * D * 2;    // K and V, twice
  const int few_b = WAVES * FEW_TILE * D * 4;  // K and V of each wave; the waves' join is smaller
  return many_b > few_b ? many_b : few_b;
}

// MANY: tiles of MANY_Q queries; rows that have few in theirs take the other way all the same.
template <typename T, int D, bool MANY>
__global__ __launch_bounds__(THREADS, 2) void k_chunk(Args a) {
  __shared__ __align__(16) char lds[lds_bytes<D>()];
  const int kv_heads = a.layer.kv_heads;
  uint32_t b = blockIdx.x;
  if (b == 0) {  // starts that decrease or leave the queries
    bool bad = false;
    for (int i = threadIdx.x; i < a.ch.rows; i += THREADS) {
      const int s = a.ch.dev_starts[i], e = a.ch.dev_starts[i + 1];
      bad |= s < 0 || e < s || e > a.ch.tokens;
    }
    if (bad && a.status) *a.status = HBF_EINVAL;
  }
  Tile t;
  t.head = b % kv_heads;
  b /= kv_heads;
  t.place = a.slots - 1 - (int)(b % a.slots);  // the longest first
  t.split = b / a.slots;
  const int i = find_row(a, t.place);
  t.row = get_row(a, i);
  const int64_t q0 = (int64_t)(t.place - first_tile(a, i, t.row.start)) * a.tile_q, n = (int64_t)t.row.n * a.group;
  if (q0 < 0 || q0 >= n) return;
  t.q0 = (int)q0;
  t.q1 = (int)min(n, q0 + a.tile_q);
  t.view = view_of(a, t.row, t.q0, t.q1);
  const bool is_few = !MANY || t.q1 - t.q0 <= 2 * FEW_Q;
  const uint32_t step = is_few ? WAVES * FEW_TILE : MANY_TILE;
  const uint32_t steps = t.row.ok ? (t.view.total + step - 1) / step : 0;
  if (steps == 0) {  // nothing is seen, or the row is in error
    if (t.split) return;
    if (!t.row.ok && threadIdx.x == 0 && a.status) *a.status = HBF_EINVAL;
    for (int j = threadIdx.x; j < (t.q1 - t.q0) * (D / 4); j += THREADS) {
      Query q = query_of(a, t, j / (D / 4));
      write_out<T>(a, q, j % (D / 4) * 4, f32x4{0.f, 0.f, 0.f, 0.f}, 0.f, 0.f, !t.row.ok, j % (D / 4) == 0);
    }
    return;
  }
  const uint32_t most = (steps + a.part_steps - 1) / a.part_steps, parts = min(most, (uint32_t)a.splits);
  const uint32_t each = (steps + parts - 1) / parts;
  t.parts = (int)((steps + each - 1) / each);
  if (t.split >= t.parts) return;
  t.x0 = (uint32_t)t.split * each * step;
  t.x1 = min(t.view.total, t.x0 + each * step);
  if (!MANY || t.q1 - t.q0 <= FEW_Q) few<T, D, 1>(a, t, lds);
  else if (is_few) few<T, D, 2>(a, t, lds);
  else many<T, D>(a, t, lds);
}

// ------------------------------------------------------------ weights

// What a row's queries gave each token: a wave takes 64 tokens, as the rows of the
// operand, in registers, and meets 16 queries at a time; the sums of a token stay
// in the four lanes that hold its scores until the end.  A slot's rows are taken
// by the first of them, one after another.
constexpr int WEIGH_TILE = 64;
template <typename T, int D>
__global__ __launch_bounds__(THREADS) void k_weigh(Args a, int blocks) {
  constexpr int KS = D / 32, U = WEIGH_TILE / 16;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, col = lane & 15, kg = lane >> 4;
  int b = blockIdx.x;
  const int head = b % a.layer.kv_heads;
  b /= a.layer.kv_heads;
  const int i0 = b % a.ch.rows, block = b / a.ch.rows;
  const int slot = a.ch.dev_slots[i0];
  bool before = false;
  for (int j = threadIdx.x; j < i0; j += THREADS) before |= a.ch.dev_slots[j] == slot;
  if (__syncthreads_or(before)) return;
  const Row first = get_row(a, i0);
  if (!first.ok) return;
  View all;
  all.first = all.lo = 0;
  all.total = first.len;
  for (uint32_t j0 = ((uint32_t)block * WAVES + w) * WEIGH_TILE; j0 < (uint32_t)first.len;
       j0 += (uint32_t)blocks * WAVES * WEIGH_TILE) {
    const uint32_t j1 = min(j0 + WEIGH_TILE, (uint32_t)first.len);
    Places<D, WEIGH_TILE> pl;
    pl.find(a, all, first.pages, j0, j1);
    const int64_t at = pl.place(a, all, j0, j1, head);
    u32x4 kk[U][KS];
#pragma unroll
    for (int u = 0; u < U; u++) {
      const char *p = (const char *)a.layer.dev_k + from_lane(at, u * 16 + col) + kg * 16;
#pragma unroll
      for (int k = 0; k < KS; k++) kk[u][k] = *(const u32x4 *)(p + k * 64);
    }
    f32x4 sum[U];
#pragma unroll
    for (int u = 0; u < U; u++) sum[u] = f32x4{0.f, 0.f, 0.f, 0.f};
    bool seen = false;
    for (int i = i0; i < a.ch.rows; i++) {
      if (a.ch.dev_slots[i] != slot) continue;
      Tile t;
      t.row = get_row(a, i);
      t.head = head;
      const int p = t.row.len - t.row.n;  // the first query's position
      // tokens [t0, t1) may see one of these
      int t0 = max(0, (int)j0 - p), t1 = t.row.n;
      if (a.ch.window > 0 && (int)j0 >= a.ch.sinks) t1 = (int)min((int64_t)t1, (int64_t)j1 - 1 + a.ch.window - p);
      if (t0 >= t1) continue;
      t.q0 = t0 * a.group;
      t.q1 = t1 * a.group;
      // where every query sees every token, no positions are compared
      const bool whole = j1 - j0 == WEIGH_TILE && (int)j1 - 1 <= p + t0 &&
                         (a.ch.window == 0 || (int)j1 <= a.ch.sinks || (int)j0 > p + t1 - 1 - a.ch.window);
      seen = true;
      for (int q0 = 0; q0 < t.q1 - t.q0; q0 += 16) {
        const Query q = query_of(a, t, q0 + col);
        u32x4 qv[KS];
        load_query<T, D>(a, q, kg, qv);
        const float2 ml = q.head < 0 ? make_float2(0.f, 0.f) : a.query_ml[(int64_t)q.token * a.ch.heads + q.head];
        f32x4 s[U];
#pragma unroll
        for (int u = 0; u < U; u++) {
          s[u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int k = 0; k < KS; k++) s[u] = T::mfma(kk[u][k], qv[k], s[u]);
        }
#pragma unroll
        for (int u = 0; u < U; u++)
#pragma unroll
          for (int j = 0; j < 4; j++) {
            const int token = (int)j0 + u * 16 + kg * 4 + j;
            const bool skip = ml.y == 0.f || (!whole && (token >= (int)j1 || !sees(a, q.pos, token)));
            sum[u][j] += skip ? 0.f : __builtin_amdgcn_exp2f((s[u][j] - ml.x) * a.c) * ml.y;
          }
      }
    }
    if (!seen) continue;
    float *out = a.ch.dev_weights + slot * a.ch.weights_slot_stride + head * a.ch.weights_head_stride;
#pragma unroll
    for (int u = 0; u < U; u++)
#pragma unroll
      for (int i = 0; i < 4; i++) {
        float v = sum[u][i];
#pragma unroll
        for (int d = 1; d < 16; d <<= 1) v += __shfl_xor(v, d);
        const uint32_t j = j0 + u * 16 + kg * 4 + i;
        if (col == 0 && j < j1) out[j] += v;
      }
  }
}

// Sizes of a call.
Args plan(const hbf_kv &kv, const hbf_kv_layer &layer, const hbf_chunk &ch) {
  Args a{};
  a.kv = kv;
  a.layer = layer;
  a.ch = ch;
  a.group = ch.heads / layer.kv_heads;
  // (1e-30: as flat as 0 is, and -infinity times it stays that)
  a.c = std::min(std::max(fabsf(ch.scale) * LOG2E, 1e-30f), FLT_MAX);
  a.flip = ch.scale < 0 ? 0x80008000u : 0;
  // with M = ceil(2^k / d), k = 31 + ceil(log2 d): token * M / 2^k is at most token / 2^31 < 1 / d above token / d
  while ((1 << a.page_shift) < layer.page_tokens) a.page_shift++;
  a.page_shift += 31;
  a.page_mul = (uint32_t)(((uint64_t(1) << a.page_shift) + layer.page_tokens - 1) / layer.page_tokens);
  const int64_t queries = (int64_t)ch.tokens * a.group;
  a.tile_q = queries > (int64_t)FEW_Q * std::max(ch.rows, 1) ? MANY_Q : FEW_Q;
  a.tile_shift = a.tile_q == MANY_Q ? 7 : 4;
  a.slots = (int)(queries >> a.tile_shift) + ch.rows;
  // Parts, so that about 1,024 workgroups have work if all rows are long; a tile takes as many as its length gives work for.
  const int64_t groups = (int64_t)a.slots * layer.kv_heads, longest = (int64_t)kv.table_cols * kv.page_tokens;
  a.part_steps = a.tile_q == FEW_Q ? 2 : 4;
  const int64_t steps = longest / ((a.tile_q == FEW_Q ? WAVES * FEW_TILE : MANY_TILE) * a.part_steps) + 1;
  a.splits = groups > (int64_t)HBF_CHUNK_CTL_WORDS || !ch.dev_ctl ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>(steps, 1024 / groups));
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
  if (a.ch.dev_weights) a.query_ml = (float2 *)take((size_t)a.ch.tokens * a.ch.heads * 8);
  return std::max(o, size_t(256));
}

template <typename T, int D>
hipError_t run(const Args &a, hipStream_t s) {
  const uint32_t blocks = (uint32_t)((int64_t)a.slots * a.layer.kv_heads * a.splits);
  if (a.tile_q == MANY_Q) k_chunk<T, D, true><<<blocks, THREADS, 0, s>>>(a);
  else k_chunk<T, D, false><<<blocks, THREADS, 0, s>>>(a);
  if (a.ch.dev_weights) {
    const int64_t groups = (int64_t)a.ch.rows * a.layer.kv_heads;
    const int64_t longest = std::min<int64_t>((int64_t)a.kv.table_cols * a.kv.page_tokens, a.ch.weights_tokens);
    const int64_t most = longest / (WAVES * WEIGH_TILE) + 1;
    const int each = (int)std::max<int64_t>(1, std::min<int64_t>(most, 4096 / groups));
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
