// Decode attention of a batch whose rows share one prefix, over cache pages.
//
// o = sum_i p_i v_i / sum_i p_i with p_i = exp(s_i - m), s_i = scale q.k_i, m a
// running maximum: one pass over the tokens, and parts of the token axis
// joined afterwards by their maxima and sums.
//
// A KV head's G query heads of all rows meet the same prefix tokens, so the
// prefix is one product of rows * G queries with its K and V: read once for the
// batch.  Own tokens are met by one row's G queries.  Both run in one launch,
// each workgroup taking a part of the token axis for some queries:
//  - few queries (own tokens; a prefix with at most 32 of them): bound by
//    memory.  Each of four waves takes 32 tokens at a time through LDS of its
//    own, the next tokens' loads in flight meanwhile; the waves meet once, at the
//    end.
//  - many queries: bound by the matrix cores and the LDS.  64 tokens are staged
//    for four waves of 32 queries each, loaded past the registers (64 rows over
//    32,771 tokens: 59.6 us, 63.3 by way of them).  Two workgroups on a CU, out of
//    step with each other, keep its matrix cores and its vector units busy by
//    turns (as one workgroup of eight waves, in step, they took half as long
//    again).
// The parts are joined by a launch of their own, or, where they are few, by the
// last workgroup of each KV head.
// Scores are computed transposed, S^T = K Q^T: a lane then holds one query's
// scores of four consecutive tokens per tile of 16, which, rounded, are
// already the operand of O^T = V^T P^T (the order of the tokens within a step
// is free as long as V's are read in the same one), so P never leaves its lane.
// It is rounded to one word of the call's type: with a second word for the rest
// the result's error is 1.7e-3 (its own rounding's) instead of 2.2e-3 in bfloat16, but
// there are half as many products again (64 rows over 32,771 tokens: 70.1 us, 58.7
// so; one row over 4,096: 11.4, 11.1), and an infinite V met by a rest of 0 would make NaN
// of what is infinite.
// K and V are loaded a head's whole row (128 or 256 bytes) by neighbouring lanes
// and take the operands' shape on the way through LDS: loaded straight into it,
// in pieces of 64 bytes, they pass the CU's vector cache at half its rate
// (28 bytes a clock measured), which bound both paths.
#include <float.h>
#include <math.h>

#include <algorithm>

#include "hbf_half.h"
#include "hbf_ops.h"

namespace hbf {
namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64;
constexpr int FEW_TILE = 32;    // tokens of a wave's step where queries are few
constexpr int MANY_TILE = 64;   // tokens staged where they are many
constexpr int MANY_Q = 128;     // queries per workgroup there
constexpr int JOIN_THREADS = 256, JOIN_WAVES = JOIN_THREADS / 64;
constexpr float LN2 = 0.69314718055994530942f, LOG2E = 1.44269504088896340736f;

struct Args {
  hbf_kv_layer kv;
  hbf_attention at;
  int group;            // query heads per KV head
  float c;              // |scale| * log2(e), not 0
  uint32_t flip;        // sign bits of two 16-bit values if the scale is negative
  uint32_t page_mul;    // token / page_tokens = token * page_mul >> page_shift, for tokens below 2^31
  int page_shift;
  int few_q;            // the prefix's queries per workgroup if they are few (16 or 32), else 0
  int m_tiles;          // workgroups across the prefix's queries
  int prefix_splits;
  int prefix_chunk;     // tokens per part
  int prefix_blocks;    // workgroups of the prefix, before the own ones
  int own_splits, own_chunk, own_tiles;  // own_tiles: workgroups across a row's query heads of one KV head
  float *part;          // [splits][rows][heads][head_dim] sums of p v
  float2 *part_ml;      // [splits][rows][heads] maximum (of q.k, its sign the scale's) and sum
  int32_t *status;
  uint32_t *ctl;        // a KV head's workgroups that are done, where the last one joins; else null
  uint32_t arrivals;    // workgroups per KV head
};

template <int D>
__device__ __forceinline__ int swizzle(int token) {  // spreads a column of 16-byte pieces over the banks
  return D == 128 ? token & 15 : (token >> 1) & 7;
}
// Byte offset of 16-byte piece `piece` of a token in a staged tile of K, whose
// readers take one piece of 16 tokens at a time,
template <int D>
__device__ __forceinline__ int k_at(int token, int piece) {
  return token * (D * 2) + ((piece ^ swizzle<D>(token)) << 4);
}
// and of V, whose readers take two pieces of 8 tokens in one cycle.
template <int D>
__device__ __forceinline__ int v_at(int token, int piece) {
  return token * (D * 2) + ((piece ^ (D == 128 ? (token & 7) << 1 : token & 6)) << 4);
}
// The lane's operand of V^T: dimensions 16 dt .. + 15, tokens t0 .. + 3 and t1 .. + 3.
template <int D>
__device__ __forceinline__ u32x4 v_operand(const char *v, int t0, int t1, int dt, int lane) {
  const int i = lane & 15, piece = dt * 2 + ((i & 3) >> 1), half = (i & 1) << 3;
  const u32x2 a = read_transposed(v + v_at<D>(t0 + (i >> 2), piece) + half);
  const u32x2 b = read_transposed(v + v_at<D>(t1 + (i >> 2), piece) + half);
  return u32x4{a[0], a[1], b[0], b[1]};
}

constexpr auto MAX_OP = [](float a, float b) { return fmaxf(a, b); };
constexpr auto SUM_OP = [](float a, float b) { return a + b; };

// One step of the running softmax for QT queries per lane (columns): their
// scores s of U tiles of 16 tokens become probabilities exp2((s - m) c + SHIFT), and l
// collects the lane's own.  m is any number that keeps exp2 in range, the same
// in a column's four lanes: it moves up, to the maximum so far, only where a
// score passes it by more than LAZY / c (then p <= 2^LAZY otherwise), which
// few steps do, and then what was summed before is scaled.  The difference comes
// first and the factor after it: at scores of 2^28 the product s c alone is
// rounded by more than exp2's range.
// p, l and o all carry the same 2^SHIFT.  A half's steps end at 2^-24: at the
// maximum p is 2^7, at most 2^15 on the way up, and what rounds to 0 is below
// 2^-32 of the maximum's (without the 2^7, 2^-25: thousands of such tokens, left
// out of o but not of l, showed).  bfloat16 has float's range.
constexpr float LAZY = 8.f;
template <typename T>
constexpr float SHIFT = 0.f;
template <>
constexpr float SHIFT<Fp16> = 7.f;
template <typename T, int QT, int U, int DT>
__device__ __forceinline__ void softmax_step(f32x4 (&s)[QT][U], float c, float (&m)[QT], float (&l)[QT],
                                             f32x4 (&o)[QT][DT]) {
  float mx[QT];
  bool up = false;
#pragma unroll
  for (int q = 0; q < QT; q++) {
    mx[q] = s[q][0][0];
#pragma unroll
    for (int u = 0; u < U; u++)
#pragma unroll
      for (int i = 0; i < 4; i++) mx[q] = fmaxf(mx[q], s[q][u][i]);
    up |= (mx[q] - m[q]) * c > LAZY;  // (none seen, none here: NaN, false)
  }
  if (__any(up)) {
#pragma unroll
    for (int q = 0; q < QT; q++) {
      const float top = fmaxf(m[q], across_rows(mx[q], MAX_OP));
      const float alpha = top == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m[q] - top) * c);
      m[q] = top;
      l[q] *= alpha;
#pragma unroll
      for (int d = 0; d < DT; d++) o[q][d] *= alpha;
    }
  }
#pragma unroll
  for (int q = 0; q < QT; q++) {
    const float ref = m[q] == -INFINITY ? 0.f : m[q];  // nothing seen yet: every p is 0
#pragma unroll
    for (int u = 0; u < U; u++)
#pragma unroll
      for (int i = 0; i < 4; i++) {
        const float d = s[q][u][i] - ref;
        s[q][u][i] = __builtin_amdgcn_exp2f(SHIFT<T> == 0.f ? d * c : fmaf(d, c, SHIFT<T>));
        l[q] += s[q][u][i];
      }
  }
}

template <typename T>
__device__ __forceinline__ u32x4 p_operand(f32x4 a, f32x4 b) {
  return u32x4{pack2<T>(a[0], a[1]), pack2<T>(a[2], a[3]), pack2<T>(b[0], b[1]), pack2<T>(b[2], b[3])};
}

__device__ __forceinline__ uint32_t page_index(const Args &a, uint32_t token) {
  return (uint32_t)((uint64_t)token * a.page_mul >> a.page_shift);
}

// A wave's share of the staging: NT tokens, a row of D values each by D / 8
// neighbouring lanes.  Lane i looks up where token i lies, the others ask it.
template <int D, int NT>
struct Stage {
  static constexpr int LANES = D / 8, AT_ONCE = 64 / LANES, PASSES = NT / AT_ONCE;
  u32x4 k[PASSES], v[PASSES];
  int page = 0;
  bool bad = false;

  // Tokens base .. of [.., t1): their page ids (past t1: of its last token).
  __device__ __forceinline__ void find(const Args &a, const int32_t *pages, uint32_t base, uint32_t t1) {
    if (NT < 64 && (threadIdx.x & 63) >= NT) return;
    page = pages[page_index(a, min(base + (threadIdx.x & 63), t1 - 1))];
  }
  __device__ __forceinline__ void load(const Args &a, uint32_t base, uint32_t t1, int head) {
    const int lane = threadIdx.x & 63;
    if (page < 0 || page >= a.kv.pages) {  // noted; page 0 is read instead
      bad = true;
      page = 0;
    }
    const uint32_t token = min(base + lane, t1 - 1);
    const uint32_t in_page = token - page_index(a, token) * (uint32_t)a.kv.page_tokens;
    const int64_t at = 2 * (page * a.kv.page_stride + in_page * a.kv.token_stride + head * a.kv.head_stride);
#pragma unroll
    for (int j = 0; j < PASSES; j++) {
      const int from = j * AT_ONCE + lane / LANES;
      const int64_t mine = (int64_t)(((uint64_t)(uint32_t)__shfl((int)(at >> 32), from) << 32) |
                                     (uint32_t)__shfl((int)at, from)) + lane % LANES * 16;
      k[j] = *(const u32x4 *)((const char *)a.kv.dev_k + mine);
      v[j] = *(const u32x4 *)((const char *)a.kv.dev_v + mine);
    }
  }
  // To tiles of K and V, as tokens first .. of them.  What lies behind the last
  // token may be anything: 0 * NaN must not reach the sums.
  __device__ __forceinline__ void store(char *kt, char *vt, int first, uint32_t base, uint32_t t1) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int j = 0; j < PASSES; j++) {
      const int t = j * AT_ONCE + lane / LANES;
      *(u32x4 *)(kt + k_at<D>(first + t, lane % LANES)) = k[j];
      *(u32x4 *)(vt + v_at<D>(first + t, lane % LANES)) = base + t < t1 ? v[j] : u32x4{0, 0, 0, 0};
    }
  }
};

// The same share loaded past the registers: a wave's lanes' 16 bytes each fall
// side by side into LDS, so that the pieces' order within a row is in the
// addresses asked for.
template <int D, int NT>
struct StageLds {
  static constexpr int LANES = D / 8, AT_ONCE = 64 / LANES, PASSES = NT / AT_ONCE;
  int page = 0;
  bool bad = false;

  __device__ __forceinline__ void find(const Args &a, const int32_t *pages, uint32_t base, uint32_t t1) {
    if (NT < 64 && (threadIdx.x & 63) >= NT) return;
    page = pages[page_index(a, min(base + (threadIdx.x & 63), t1 - 1))];
  }
  // Tokens base .. (past t1: its last one again) to tokens first .. of a tile; there after loads_done().
  __device__ __forceinline__ void load(const Args &a, uint32_t base, uint32_t t1, int head, uint32_t kt, uint32_t vt,
                                       int first) {
    const int lane = threadIdx.x & 63;
    if (page < 0 || page >= a.kv.pages) {  // noted; page 0 is read instead
      bad = true;
      page = 0;
    }
    const uint32_t token = min(base + lane, t1 - 1);
    const uint32_t in_page = token - page_index(a, token) * (uint32_t)a.kv.page_tokens;
    const int64_t at = 2 * (page * a.kv.page_stride + in_page * a.kv.token_stride + head * a.kv.head_stride);
    uint32_t hi[PASSES], lo[PASSES];
#pragma unroll
    for (int j = 0; j < PASSES; j++) {
      hi[j] = (uint32_t)__shfl((int)(at >> 32), j * AT_ONCE + lane / LANES);
      lo[j] = (uint32_t)__shfl((int)at, j * AT_ONCE + lane / LANES);
    }
#pragma unroll
    for (int j = 0; j < PASSES; j++) {
      const int t = first + j * AT_ONCE;  // of the wave's first lanes
      const int64_t row = (int64_t)((uint64_t)hi[j] << 32 | lo[j]);
      const int mine = t + lane / LANES, piece = lane % LANES * 16;
      to_lds((const char *)a.kv.dev_k + row + (piece ^ (k_at<D>(mine, 0) - mine * (D * 2))), kt + t * (D * 2));
      to_lds((const char *)a.kv.dev_v + row + (piece ^ (v_at<D>(mine, 0) - mine * (D * 2))), vt + t * (D * 2));
    }
  }
};

struct Query {
  int row, head;  // row < 0: none
};
__device__ __forceinline__ int64_t part_slot(const Args &a, int split, Query q) {
  return ((int64_t)split * a.at.rows + q.row) * a.at.heads + q.head;
}

template <typename T, int D>
__device__ __forceinline__ void load_query(const Args &a, Query q, int kgroup, u32x4 *out) {
  const char *p = (const char *)a.at.dev_q +
                  2 * ((q.row < 0 ? 0 : q.row) * a.at.q_row_stride + (q.row < 0 ? 0 : q.head) * a.at.q_head_stride);
#pragma unroll
  for (int k = 0; k < D / 32; k++) {
    const u32x4 v = *(const u32x4 *)(p + (k * 32 + kgroup * 8) * 2) ^ a.flip;
    out[k] = q.row < 0 ? u32x4{0, 0, 0, 0} : v;
  }
}

// ------------------------------------------------------------ few queries

// Tokens [t0, t1) (t0 < t1) of a page list for 16 QT queries, one per column;
// query(col) names them.
template <typename T, int D, int QT, bool HERE, typename Q>
__device__ void few(const Args &a, const int32_t *pages, uint32_t t0, uint32_t t1, int head, int split, Q query,
                    char *lds) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, col = lane & 15, kg = lane >> 4;
  constexpr int KS = D / 32, DT = D / 16;
  u32x4 qv[QT][KS];
#pragma unroll
  for (int q = 0; q < QT; q++) load_query<T, D>(a, query(q * 16 + col), kg, qv[q]);
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
  uint32_t base = t0 + w * FEW_TILE;
  Stage<D, FEW_TILE> st;
  constexpr uint32_t STEP = WAVES * FEW_TILE;
  if (base < t1) {
    st.find(a, pages, base, t1);
    st.load(a, base, t1, head);
    st.find(a, pages, base + STEP, t1);
    while (true) {
      const bool more = t1 - base > STEP, tail = t1 - base < FEW_TILE;
      st.store(kt, vt, 0, base, t1);
      wave_lds_fence();
      if (more) {
        st.load(a, base + STEP, t1, head);
        st.find(a, pages, base + 2 * STEP, t1);
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
      if (tail)
#pragma unroll
        for (int q = 0; q < QT; q++)
#pragma unroll
          for (int u = 0; u < 2; u++)
#pragma unroll
            for (int i = 0; i < 4; i++)
              if (base + u * 16 + kg * 4 + i >= t1) s[q][u][i] = -INFINITY;
      softmax_step<T, QT, 2, DT>(s, a.c, m, l, o);
      u32x4 p[QT];
#pragma unroll
      for (int q = 0; q < QT; q++) p[q] = p_operand<T>(s[q][0], s[q][1]);
#pragma unroll
      for (int d = 0; d < DT; d++) {
        const u32x4 v = v_operand<D>(vt, kg * 4, 16 + kg * 4, d, lane);
#pragma unroll
        for (int q = 0; q < QT; q++) o[q][d] = T::mfma(v, p[q], o[q][d]);
      }
      wave_lds_fence();
      if (!more) break;
      base += STEP;
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
    const Query qq = query(q * 16 + n);
    if (qq.row >= 0) {
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
      const int64_t slot = part_slot(a, split, qq);
#pragma unroll
      for (int d = d0; d < D; d += PER * 4) {
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < WAVES; i++) x += f[i] * *(const f32x4 *)(ro + (i * 16 + n) * RS + d);
        if (HERE) hand_over((f32x4 *)(a.part + slot * D + d), x);
        else *(f32x4 *)(a.part + slot * D + d) = x;
      }
      if (d0 == 0) {
        const float2 ml = any_bad ? make_float2(NAN, NAN) : make_float2(mx, sum);
        if (HERE) hand_over(a.part_ml + slot, ml);
        else a.part_ml[slot] = ml;
      }
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------ many queries

// Tokens [t0, t1) (t0 < t1) of the prefix for MANY_Q queries from m0 on.
template <typename T, int D>
__device__ void many(const Args &a, uint32_t t0, uint32_t t1, int head, int split, int m0, char *lds) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, col = lane & 15, kg = lane >> 4;
  static_assert(MANY_Q == 32 * WAVES, "queries per wave");
  constexpr int KS = D / 32, DT = D / 16, QT = 2, U = MANY_TILE / 16;
  constexpr int TILE_BYTES = MANY_TILE * D * 2;
  auto query = [&](int n) {
    const int mm = m0 + n;
    const int row = mm / a.group;
    return row < a.at.rows ? Query{row, head * a.group + mm - row * a.group} : Query{-1, 0};
  };
  constexpr int NT = MANY_TILE / WAVES;  // tokens of a tile that a wave stages
  constexpr uint32_t STEP = MANY_TILE;
  const int32_t *pages = a.at.dev_prefix_pages;
  const uint32_t lds0 = lds_address(lds);
  StageLds<D, NT> st;
  st.find(a, pages, t0 + w * NT, t1);
  u32x4 qv[QT][KS];
#pragma unroll
  for (int q = 0; q < QT; q++) load_query<T, D>(a, query(w * 32 + q * 16 + col), kg, qv[q]);
  st.load(a, t0 + w * NT, t1, head, lds0, lds0 + TILE_BYTES, w * NT);
  f32x4 o[QT][DT];
  float m[QT], l[QT];
#pragma unroll
  for (int q = 0; q < QT; q++) {
    m[q] = -INFINITY;
    l[q] = 0.f;
#pragma unroll
    for (int d = 0; d < DT; d++) o[q][d] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  st.find(a, pages, t0 + STEP + w * NT, t1);
  loads_done();
  __syncthreads();
  int cur = 0;
  for (uint32_t base = t0;;) {
    const char *kt = lds + cur * 2 * TILE_BYTES, *vt = kt + TILE_BYTES;
    if (t1 - base < MANY_TILE) {  // 0 * infinity must not reach the sums: no V behind the last token
      const int left = (int)(t1 - base);
      for (int i = left * D * 2 + threadIdx.x * 16; i < TILE_BYTES; i += THREADS * 16)
        *(u32x4 *)(lds + cur * 2 * TILE_BYTES + TILE_BYTES + i) = u32x4{0, 0, 0, 0};
      __syncthreads();
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
    const bool more = t1 - base > STEP;
    if (more) {  // the next step's tile, here so that its addresses are found beside the products
      const uint32_t next = lds0 + (cur ^ 1) * 2 * TILE_BYTES;
      st.load(a, base + STEP + w * NT, t1, head, next, next + TILE_BYTES, w * NT);
      if (t1 - base > 2 * STEP) st.find(a, pages, base + 2 * STEP + w * NT, t1);
    }
    if (t1 - base < MANY_TILE)
#pragma unroll
      for (int q = 0; q < QT; q++)
#pragma unroll
        for (int u = 0; u < U; u++)
#pragma unroll
          for (int i = 0; i < 4; i++)
            if (base + u * 16 + kg * 4 + i >= t1) s[q][u][i] = -INFINITY;
    u32x4 vv2[2][U / 2];
    auto read_v = [&](int d) {
#pragma unroll
      for (int u = 0; u < U / 2; u++)
        vv2[d & 1][u] = v_operand<D>(vt, u * 32 + kg * 4, u * 32 + 16 + kg * 4, d, lane);
    };
    softmax_step<T, QT, U, DT>(s, a.c, m, l, o);
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
        for (int q = 0; q < QT; q++) o[q][d] = T::mfma(vv2[d & 1][u], p[q][u], o[q][d]);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (!more) break;
    base += STEP;
    loads_done();
    __syncthreads();
    cur ^= 1;
  }
  const bool any_bad = __syncthreads_or(st.bad);
  if (any_bad && threadIdx.x == 0 && a.status) *a.status = HBF_EINVAL;
#pragma unroll
  for (int q = 0; q < QT; q++) {
    const Query qq = query(w * 32 + q * 16 + col);
    const float lq = across_rows(l[q], SUM_OP);
    if (qq.row < 0) continue;
    const int64_t slot = part_slot(a, split, qq);
#pragma unroll
    for (int d = 0; d < DT; d++) *(f32x4 *)(a.part + slot * D + d * 16 + kg * 4) = o[q][d];
    if (kg == 0) a.part_ml[slot] = any_bad ? make_float2(NAN, NAN) : make_float2(m[q], lq);
  }
}

// ------------------------------------------------------------ join

// Row `row`'s parts; bad: its length is out of range (then it counts as empty).
__device__ __forceinline__ int parts_of(const Args &a, int len, bool *bad) {
  *bad = len < 0 || len > a.at.max_own;
  const int own = *bad || len == 0 ? 0 : (int)(((uint32_t)len + (uint32_t)a.own_chunk - 1) / (uint32_t)a.own_chunk);
  return a.prefix_splits + own;
}
// Four of a query's values, from d0 on, from its sums; none: it saw no token.  lead: the one thread that writes lse.
template <typename T>
__device__ __forceinline__ void write_out(const Args &a, int row, int head, int d0, f32x4 o, float m, float l, bool none,
                                          bool bad, bool lead) {
  if (bad) {
    l = NAN;
    if (a.status && lead) *a.status = HBF_EINVAL;
  }
  none = none && !bad;
  o *= none ? 0.f : 1.f / l;
  typename T::elem *out = (typename T::elem *)a.at.dev_out + row * a.at.out_row_stride + head * a.at.out_head_stride + d0;
  *(u32x2 *)out = u32x2{pack2<T>(o[0], o[1]), pack2<T>(o[2], o[3])};
  if (a.at.dev_lse && lead) a.at.dev_lse[(int64_t)row * a.at.heads + head] = none ? -INFINITY : m * a.c * LN2 + logf(l * exp2f(-SHIFT<T>));
}

// The running sums (m, l, o) take U parts in, relative to a first maximum, raised
// as parts of larger ones come (NaN, a part of bad pages, stays).
template <int U>
__device__ __forceinline__ void take_parts(float c, const float2 (&ml)[U], const f32x4 (&p)[U], float &m, float &l,
                                           f32x4 &o) {
  float top = m;
#pragma unroll
  for (int u = 0; u < U; u++) top = fmaxf(top, ml[u].x);
  const float ref = top == -INFINITY ? 0.f : top, alpha = __builtin_amdgcn_exp2f((m - ref) * c);
  m = top;
  l *= alpha;
  o *= alpha;
#pragma unroll
  for (int u = 0; u < U; u++) {
    const float f = __builtin_amdgcn_exp2f((ml[u].x - ref) * c);
    l += f * ml[u].y;
    o += f * p[u];
  }
}
// Parts n and above, of those that are u0 .. + step * (U - 1), are none.
template <int U>
__device__ __forceinline__ void leave_out(float2 (&ml)[U], f32x4 (&p)[U], int u0, int step, int n) {
#pragma unroll
  for (int u = 0; u < U; u++)
    if (u0 + u * step >= n) {
      ml[u] = make_float2(-INFINITY, 0.f);
      p[u] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
}

// All queries of one KV head by one workgroup, from parts that others of the
// launch handed over: D / 4 lanes a query, R queries each, at most HERE_PARTS / R
// parts a query, so that a thread asks for all it needs at once (parts past a
// row's own are none, and left out).
constexpr int HERE_PARTS = 24;
template <typename T, int D, int R>
__device__ void join_here(const Args &a, int kv_head) {
  constexpr int LANES = D / 4, U = HERE_PARTS / R;
  const int d0 = threadIdx.x % LANES * 4, all = a.prefix_splits + a.own_splits;
  const int64_t stride = (int64_t)a.at.rows * a.at.heads;
  const int last = a.at.rows * a.group - 1;
  int len[R];
  float2 ml[R][U];
  f32x4 x[R][U];
  auto query = [&](int r) { return (int)threadIdx.x / LANES + r * (THREADS / LANES); };
#pragma unroll
  for (int r = 0; r < R; r++) {  // (no branches: past the last query its own again, past the last part that one)
    const int mm = min(query(r), last), row = mm / a.group;
    const int64_t qi = (int64_t)row * a.at.heads + kv_head * a.group + mm - row * a.group;
    len[r] = a.at.dev_own_len ? a.at.dev_own_len[row] : 0;
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int64_t slot = min(u, all - 1) * stride + qi;
      ml[r][u] = a.part_ml[slot];
      x[r][u] = *(const f32x4 *)(a.part + slot * D + d0);
    }
  }
#pragma unroll
  for (int r = 0; r < R; r++) {
    bool bad;
    const int n = parts_of(a, len[r], &bad);
    float m = -INFINITY, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    leave_out(ml[r], x[r], 0, 1, n);
    take_parts(a.c, ml[r], x[r], m, l, o);
    const int mm = query(r), row = mm / a.group;
    if (mm <= last) write_out<T>(a, row, kv_head * a.group + mm - row * a.group, d0, o, m, l, n == 0, bad, d0 == 0);
  }
}

template <int D>
constexpr int lds_bytes() {
  const int many_b = 4 * MANY_TILE * D * 2;                     // K and V, twice
  const int few_b = WAVES * FEW_TILE * D * 4;                 // K and V of each wave; the waves' join is smaller
  return many_b > few_b ? many_b : few_b;
}

// A workgroup's part is written.
template <typename T, int D, bool HERE>
__device__ void end(const Args &a, int kv_head) {
  if (!HERE) return;
  stores_done();
  if (!last_of(a.ctl + kv_head, a.arrivals)) return;
  see_handed();
  const int m = a.at.rows * a.group, at_once = THREADS / (D / 4);
  if (m <= at_once) join_here<T, D, 1>(a, kv_head);
  else if (m <= 2 * at_once) join_here<T, D, 2>(a, kv_head);
  else join_here<T, D, 4>(a, kv_head);
}

// Workgroups [0, prefix_blocks): the prefix, those of one part and KV head on
// one XCD (block numbers equal modulo 8) so that they share its L2.  Then the
// own tokens'.  HERE: few queries, joined by the last workgroups.
template <typename T, int D, bool HERE>
__global__ __launch_bounds__(THREADS, 2) void k_attn(Args a) {
  __shared__ __align__(16) char lds[lds_bytes<D>()];
  int b = blockIdx.x;
  if (b < a.prefix_blocks) {
    const int sh = b / (8 * a.m_tiles) * 8 + b % 8, mt = b / 8 % a.m_tiles;
    if (sh >= a.prefix_splits * a.kv.kv_heads) return;
    const int head = sh % a.kv.kv_heads, split = sh / a.kv.kv_heads;
    const uint32_t t0 = (uint32_t)split * (uint32_t)a.prefix_chunk;
    const uint32_t t1 = min(t0 + (uint32_t)a.prefix_chunk, (uint32_t)a.at.prefix_len);
    if (!HERE && a.few_q == 0) {
      many<T, D>(a, t0, t1, head, split, mt * MANY_Q, lds);
      return;
    }
    const int m0 = mt * a.few_q;
    auto query = [&](int n) {
      const int mm = m0 + n, row = mm / a.group;
      return row < a.at.rows ? Query{row, head * a.group + mm - row * a.group} : Query{-1, 0};
    };
    if (a.few_q == 16)
      few<T, D, 1, HERE>(a, a.at.dev_prefix_pages, t0, t1, head, split, query, lds);
    else
      few<T, D, 2, HERE>(a, a.at.dev_prefix_pages, t0, t1, head, split, query, lds);
    end<T, D, HERE>(a, head);
    return;
  }
  b -= a.prefix_blocks;
  const int tile = b % a.own_tiles;
  b /= a.own_tiles;
  const int head = b % a.kv.kv_heads;
  b /= a.kv.kv_heads;
  const int row = b % a.at.rows, split = b / a.at.rows;
  const int len = a.at.dev_own_len[row];
  if (len < 0 || len > a.at.max_own) {
    if (threadIdx.x == 0 && a.status) *a.status = HBF_EINVAL;
    end<T, D, HERE>(a, head);
    return;
  }
  const uint32_t t0 = (uint32_t)split * (uint32_t)a.own_chunk;
  if (t0 >= (uint32_t)len) {
    end<T, D, HERE>(a, head);
    return;
  }
  auto query = [&](int n) {
    const int g = tile * 16 + n;
    return g < a.group ? Query{row, head * a.group + g} : Query{-1, 0};
  };
  few<T, D, 1, HERE>(a, a.at.dev_tables + (int64_t)row * a.at.table_stride, t0,
               min(t0 + (uint32_t)a.own_chunk, (uint32_t)len), head, a.prefix_splits + split, query, lds);
  end<T, D, HERE>(a, head);
}

// Join a query's parts by PER waves, D / 4 lanes a part.
template <typename T, int D, int PER>
__global__ __launch_bounds__(JOIN_THREADS) void k_attn_join(Args a) {
  constexpr int LANES = D / 4, ALL = JOIN_THREADS / LANES, GROUPS = ALL * PER / JOIN_WAVES;  // groups of lanes: all, a query's
  constexpr int U = PER == 2 || PER == 1 && D == 128 ? 8 : 4;
  __shared__ f32x4 so[JOIN_THREADS];
  __shared__ float2 sml[ALL];
  const int all = threadIdx.x / LANES, g = all % GROUPS, d0 = threadIdx.x % LANES * 4;
  const int64_t stride = (int64_t)a.at.rows * a.at.heads;
  const int64_t mine = (int64_t)blockIdx.x * (JOIN_WAVES / PER) + all / GROUPS, qi = min(mine, stride - 1);
  const int row = (int)(qi / a.at.heads), head = (int)(qi - (int64_t)row * a.at.heads);
  const int len = a.at.dev_own_len ? a.at.dev_own_len[row] : 0;
  float m = -INFINITY, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float2 ml[U];
  f32x4 p[U];
  auto load = [&](int i0, int end) {
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int i = i0 + u * GROUPS;
      ml[u] = i < end ? a.part_ml[i * stride + qi] : make_float2(-INFINITY, 0.f);
      p[u] = i < end ? *(const f32x4 *)(a.part + (i * stride + qi) * D + d0) : f32x4{0.f, 0.f, 0.f, 0.f};
    }
  };
  load(g, a.prefix_splits + a.own_splits);  // without waiting for the length: parts that are none are left out below
  bool bad;
  const int n = parts_of(a, len, &bad);
  leave_out(ml, p, g, GROUPS, n);
  for (int i0 = g; i0 < n; i0 += GROUPS * U) {
    if (i0 != g) load(i0, n);
    take_parts(a.c, ml, p, m, l, o);
  }
  so[threadIdx.x] = o;
  if (d0 == 0) sml[all] = make_float2(m, l);
  __syncthreads();
  if (g || mine >= stride) return;
  float2 parts[GROUPS];
  f32x4 sums[GROUPS];
#pragma unroll
  for (int i = 0; i < GROUPS; i++) {
    parts[i] = sml[all + i];
    sums[i] = so[threadIdx.x + i * LANES];
  }
  m = -INFINITY;
  l = 0.f;
  o = f32x4{0.f, 0.f, 0.f, 0.f};
  take_parts(a.c, parts, sums, m, l, o);
  write_out<T>(a, row, head, d0, o, m, l, n == 0, bad, d0 == 0);
}

// Sizes of a call: how the token axes are cut.
Args plan(const hbf_kv_layer &kv, const hbf_attention &at) {
  Args a{};
  a.kv = kv;
  a.at = at;
  a.group = at.heads / kv.kv_heads;
  // (1e-30: as flat as 0 is, and -infinity times it stays that)
  a.c = std::min(std::max(fabsf(at.scale) * LOG2E, 1e-30f), FLT_MAX);
  a.flip = at.scale < 0 ? 0x80008000u : 0;
  // with M = ceil(2^k / d), k = 31 + ceil(log2 d): token * M / 2^k is at most token / 2^31 < 1 / d above token / d
  while ((1 << a.page_shift) < kv.page_tokens) a.page_shift++;
  a.page_shift += 31;
  a.page_mul = (uint32_t)(((uint64_t(1) << a.page_shift) + kv.page_tokens - 1) / kv.page_tokens);
  const int64_t m = (int64_t)at.rows * a.group;
  a.few_q = m <= 16 ? 16 : m <= 32 ? 32 : 0;
  a.m_tiles = (int)(a.few_q ? 1 : (m + MANY_Q - 1) / MANY_Q);
  a.own_tiles = (a.group + 15) / 16;
  // Parts: two workgroups per CU, the prefix's and the own ones' shares of the 512 as their shares of the work, in
  // steps of a workgroup (64 tokens for many queries, 128 for few), so that all run at the same time.  A part of many
  // queries has 4 steps at least: its sums, 66 KB, take as long to write and join as two.
  constexpr double SLOTS = 512;
  const int64_t pre_step = a.few_q ? WAVES * FEW_TILE : MANY_TILE, own_step = WAVES * FEW_TILE;
  const int64_t pre_groups = (int64_t)kv.kv_heads * a.m_tiles, own_groups = (int64_t)at.rows * kv.kv_heads * a.own_tiles;
  const int64_t pre_steps = (at.prefix_len + pre_step - 1) / pre_step, own_steps = (at.max_own + own_step - 1) / own_step;
  const double pre_work = (double)pre_groups * pre_steps, own_work = (double)own_groups * own_steps;
  auto cut = [](int64_t tokens, int64_t all, int64_t step, int64_t least, double groups, int *chunk) {
    if (tokens <= 0) return 0;
    const int64_t parts = std::max<int64_t>(1, std::min<int64_t>((all + least - 1) / least, (int64_t)groups)), each = (all + parts - 1) / parts;
    *chunk = (int)std::min<int64_t>(each * step, INT32_MAX / 2 / step * step);
    return (int)((tokens + *chunk - 1) / *chunk);
  };
  const double slots = SLOTS / (pre_work + own_work + 1e-9);
  // max_own is what the table's rows can hold, and a cache's are as wide as a sequence may grow, whatever they hold.
  // Workgroups past a row's length end at once, but a prefix cut into too few parts is slow: against it, no more
  // than 1,024 own tokens count.
  const double pre_slots = SLOTS / (pre_work + std::min(own_work, own_groups * 1024. / own_step) + 1e-9);
  a.prefix_splits = cut(at.prefix_len, pre_steps, pre_step, a.few_q ? 1 : 4, pre_slots * pre_work / pre_groups, &a.prefix_chunk);
  a.own_splits = cut(at.max_own, own_steps, own_step, 1, slots * own_work / std::max<int64_t>(1, own_groups), &a.own_chunk);
  // A KV head's last workgroup joins its queries where a thread can ask for their parts at once: a launch less, 3.4 us
  // of the host's time and 4 of the GPU's (7 rows of 3 queries over 1,003 tokens: 9.1 us, 11.9 with it; one row of 8
  // over 300: 9.0, 11.7; one over 4,096 tokens: 11.1, 11.6).  A part is two steps if that makes them few enough.
  const int64_t at_once = THREADS / (kv.head_dim / 4), each = m <= at_once ? 1 : m <= 2 * at_once ? 2 : 4;
  const int64_t most = HERE_PARTS / each - a.own_splits;
  if (a.few_q && a.prefix_splits > most && (pre_steps + 1) / 2 <= most)
    a.prefix_splits = cut(at.prefix_len, pre_steps, pre_step, 2, INT32_MAX, &a.prefix_chunk);
  a.arrivals = (uint32_t)(a.prefix_splits + (int64_t)at.rows * a.own_splits * a.own_tiles);
  if (a.few_q && a.arrivals && kv.kv_heads <= ATTN_CTL_WORDS && a.prefix_splits <= most) a.ctl = at.dev_ctl;
  a.prefix_blocks = (a.prefix_splits * kv.kv_heads + 7) / 8 * 8 * a.m_tiles;
  return a;
}

template <typename T, int D>
hipError_t run(const Args &a, hipStream_t s) {
  const int64_t blocks =
      a.prefix_blocks + (int64_t)a.own_splits * a.at.rows * a.kv.kv_heads * a.own_tiles;
  if (a.ctl) {
    k_attn<T, D, true><<<(uint32_t)blocks, THREADS, 0, s>>>(a);
    return hipGetLastError();
  }
  if (blocks > 0) k_attn<T, D, false><<<(uint32_t)blocks, THREADS, 0, s>>>(a);
  // A wave per query where its parts are few and the waves fill the card: 512 queries in up to 12 parts took 16.4 us so, 15.9 by
  // a workgroup each.
  const uint32_t queries = (uint32_t)a.at.rows * a.at.heads;
  if (a.prefix_splits + a.own_splits <= 16 && queries > 1024) {
    k_attn_join<T, D, 1><<<(queries + JOIN_WAVES - 1) / JOIN_WAVES, JOIN_THREADS, 0, s>>>(a);
  } else {
    constexpr int PER = D == 128 ? 4 : 2;  // eight groups of lanes a query
    k_attn_join<T, D, PER><<<(queries * PER + JOIN_WAVES - 1) / JOIN_WAVES, JOIN_THREADS, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace

size_t attn_ws_bytes(const hbf_kv_layer &kv, const hbf_attention &at) {
  const Args a = plan(kv, at);
  const size_t slots = (size_t)(a.prefix_splits + a.own_splits) * at.rows * at.heads;
  return slots * ((size_t)kv.head_dim * 4 + 8) + 256;
}

hipError_t launch_attn(const hbf_kv_layer &kv, const hbf_attention &at, int32_t *status, void *ws, hipStream_t s) {
  Args a = plan(kv, at);
  const size_t slots = (size_t)(a.prefix_splits + a.own_splits) * at.rows * at.heads;
  a.part = (float *)ws;
  a.part_ml = (float2 *)((char *)ws + slots * kv.head_dim * 4);
  a.status = status;
  if (kv.dtype == HBF_BF16) return kv.head_dim == 64 ? run<Bf16, 64>(a, s) : run<Bf16, 128>(a, s);
  return kv.head_dim == 64 ? run<Fp16, 64>(a, s) : run<Fp16, 128>(a, s);
}

}  // namespace hbf
