// The two 16-bit types of the decode-layer operators: conversions, the matrix
// instruction and the transposing LDS read.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace hbf {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

struct Bf16 {
  typedef __bf16 elem;
  typedef __bf16 x8 __attribute__((ext_vector_type(8)));
  typedef __bf16 x2 __attribute__((ext_vector_type(2)));
  // D[16 x 16] += A[16 x 32] B[32 x 16]: lane l holds A's row l % 16 and B's
  // column l % 16 at k = 8 (l / 16) .. + 7, and D's column l % 16 at rows
  // 4 (l / 16) .. + 3.
  static __device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
  }
  // D[32 x 32] += A[32 x 16] B[16 x 32]: lane l holds A's row l % 32 and B's
  // column l % 32 at k = 8 (l / 32) .. + 7, and of D's column l % 32 the rows
  // 8 (i / 4) + 4 (l / 32) + i % 4, i < 16.
  static __device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
  }
};
struct Fp16 {
  typedef _Float16 elem;
  typedef _Float16 x8 __attribute__((ext_vector_type(8)));
  typedef _Float16 x2 __attribute__((ext_vector_type(2)));
  static __device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
  }
};

// Two values rounded to nearest even, the first in the low half.
template <typename T>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  typename T::x2 v;
  v[0] = (typename T::elem)lo;
  v[1] = (typename T::elem)hi;
  return __builtin_bit_cast(uint32_t, v);
}

// A 16-lane group reads a 4 x 16 block of 16-bit values, lane i the 8 bytes at
// `at` (row i / 4, columns 4 (i % 4) .. + 3), and lane i receives column i.
__device__ __forceinline__ u32x2 read_transposed(const void *at) {
  typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)at));
}

// op over the wave, in every lane (op associative and commutative).
template <typename V, typename F>
__device__ __forceinline__ V across_wave(V x, F op) {
  uint32_t u = __builtin_bit_cast(uint32_t, x);
  auto join = [&](uint32_t a, uint32_t b) {
    u = __builtin_bit_cast(uint32_t, op(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b)));
  };
  join(u, __builtin_amdgcn_update_dpp(0, u, 0xb1, 0xf, 0xf, true));   // quad_perm 1,0,3,2
  join(u, __builtin_amdgcn_update_dpp(0, u, 0x4e, 0xf, 0xf, true));   // quad_perm 2,3,0,1
  join(u, __builtin_amdgcn_update_dpp(0, u, 0x141, 0xf, 0xf, true));  // row_half_mirror
  join(u, __builtin_amdgcn_update_dpp(0, u, 0x140, 0xf, 0xf, true));  // row_mirror
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  join(a[0], a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  join(b[0], b[1]);
  return __builtin_bit_cast(V, u);
}

// The sum over each 16 lanes of the wave, in each of them; over each half of it.
__device__ __forceinline__ float sum_of_row(float x) {
  uint32_t u = __builtin_bit_cast(uint32_t, x);
  auto join = [&](uint32_t b) {
    u = __builtin_bit_cast(uint32_t, __builtin_bit_cast(float, u) + __builtin_bit_cast(float, b));
  };
  join(__builtin_amdgcn_update_dpp(0, u, 0xb1, 0xf, 0xf, true));   // quad_perm 1,0,3,2
  join(__builtin_amdgcn_update_dpp(0, u, 0x4e, 0xf, 0xf, true));   // quad_perm 2,3,0,1
  join(__builtin_amdgcn_update_dpp(0, u, 0x141, 0xf, 0xf, true));  // row_half_mirror
  join(__builtin_amdgcn_update_dpp(0, u, 0x140, 0xf, 0xf, true));  // row_mirror
  return __builtin_bit_cast(float, u);
}
__device__ __forceinline__ float sum_of_half(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, sum_of_row(x));
  const auto both = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t a = both[0], b = both[1];
  return __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
}

// op over the four lanes that hold the same column of a tile (l % 16), in each of them.
template <typename F>
__device__ __forceinline__ float across_rows(float x, F op) {
  uint32_t u = __builtin_bit_cast(uint32_t, x);
  auto join = [&](uint32_t a, uint32_t b) {
    u = __builtin_bit_cast(uint32_t, op(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)));
  };
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  join(a[0], a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  join(b[0], b[1]);
  return __builtin_bit_cast(float, u);
}

// Values that workgroups of one launch hand to each other: written past the
// caches of one XCD, and read past them.  A writer waits for its stores
// (stores_done) before it tells of them.
__device__ __forceinline__ void hand_over(float *to, float v) {
  __hip_atomic_store(to, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void hand_over(f32x4 *to, f32x4 v) {
  const u32x4 u = __builtin_bit_cast(u32x4, v);
#pragma unroll
  for (int i = 0; i < 2; i++)
    __hip_atomic_store((uint64_t *)to + i, (uint64_t)u[2 * i + 1] << 32 | u[2 * i], __ATOMIC_RELAXED,
                       __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void hand_over(float2 *to, float2 v) {
  __hip_atomic_store((uint64_t *)to, (uint64_t)__float_as_uint(v.y) << 32 | __float_as_uint(v.x), __ATOMIC_RELAXED,
                     __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float handed(const float *from) {
  return __hip_atomic_load(from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// After last_of: ordinary loads too find what was handed over.
__device__ __forceinline__ void see_handed() { __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent"); }
__device__ __forceinline__ void stores_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// True in every thread of the last of n workgroups to get here; the counter is
// 0 again.  What a workgroup hands over before, its stores done, the last one
// finds.
static __device__ bool last_of(uint32_t *counter, uint32_t n) {
  __shared__ uint32_t last;
  __syncthreads();
  if (n == 1) return true;
  if (threadIdx.x == 0) {
    last = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1 == n;
    if (last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  return last != 0;
}

// 16 bytes of each lane, from an address of its own, to LDS at `to` (the same in
// all lanes) + 16 lane.  In flight until loads_done(); the compiler does not know.
__device__ __forceinline__ uint32_t lds_address(const void *p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char *)p;
}
__device__ __forceinline__ void to_lds(const void *from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(
                   __builtin_amdgcn_readfirstlane((int)to)),
               "v"(from)
               : "memory", "m0");
}
__device__ __forceinline__ void loads_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
// All but the wave's last N are there.
template <int N>
__device__ __forceinline__ void loads_left() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// What the lanes of one wave have written to LDS is read by others of it: the
// LDS serves a wave's accesses in order, so only the compiler is held.
__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

}  // namespace hbf
