// Pieces that the attention kernels share: staged tiles of K and V, the running
// softmax of a step, the joining of parts.
#pragma once

#include <math.h>

#include "hbf_half.h"

namespace hbf {

constexpr float LN2 = 0.69314718055994530942f, LOG2E = 1.44269504088896340736f;

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
inline constexpr float SHIFT = 0.f;
template <>
inline constexpr float SHIFT<Fp16> = 7.f;
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

// A step's probabilities as the matrix cores take them with V: rounded to the
// 16-bit type, each by half of a step relative to itself at most; the sum l keeps
// them as they are.  (Errors against 64 bits, of the results' size: bfloat16 0.0019
// to 0.0023, 0.0017 from the results' own rounding alone.)
template <typename T>
__device__ __forceinline__ u32x4 p_operand(f32x4 a, f32x4 b) {
  return u32x4{pack2<T>(a[0], a[1]), pack2<T>(a[2], a[3]), pack2<T>(b[0], b[1]), pack2<T>(b[2], b[3])};
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

}  // namespace hbf
