// A cache's table rows and lengths, as its kernels read them.
#pragma once

#include <hip/hip_runtime.h>

#include "hbf.h"

namespace hbf {

__device__ __forceinline__ int pages_of(int len, int page_tokens) {
  return (int)(((uint32_t)len + (uint32_t)page_tokens - 1) / (uint32_t)page_tokens);
}
__device__ __forceinline__ bool len_fits(const hbf_kv &kv, int len) {
  return len >= 0 && (int64_t)len <= (int64_t)kv.table_cols * kv.page_tokens;
}
__device__ __forceinline__ int32_t *row_of(const hbf_kv &kv, int32_t *tables, int slot) {
  return tables + (int64_t)slot * kv.table_stride;
}

// Exclusive prefix sum over a workgroup of N threads; *total: the sum.
template <int N>
__device__ uint32_t block_scan(uint32_t v, uint32_t *total, uint32_t *lds /* [N / 64] */) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  uint32_t x = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  if (lane == 63) lds[w] = x;
  __syncthreads();
  uint32_t before = 0, sum = 0;
#pragma unroll
  for (int i = 0; i < N / 64; i++) {
    const uint32_t y = lds[i];
    before += i < w ? y : 0;
    sum += y;
  }
  __syncthreads();
  *total = sum;
  return before + x - v;
}

}  // namespace hbf
