// What the products' kernels share.
#pragma once
#include "vvs_e4m3.h"
#include "vvs_qlinear.h"

namespace vvs {

typedef int intx8 __attribute__((ext_vector_type(8)));

constexpr size_t kMostLds = 160 << 10;   // of a workgroup

// n elements of a row's four
template <typename T>
__device__ __forceinline__ void store4(T* y, int n, bool wide, const float (&v)[4]) {
  if (wide && n >= 4) {
    if constexpr (sizeof(T) == 4) *(float4*)y = make_float4(v[0], v[1], v[2], v[3]);
    else *(uint2*)y = make_uint2(pack2bf(v[0], v[1]), pack2bf(v[2], v[3]));
    return;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (j < n) st(y + j, v[j]);
}

__device__ __forceinline__ float silu(float x) { return x / (1.f + expf(-x)); }

// Largest over the 16 lanes of a row of the wave, left in all of them
__device__ __forceinline__ float row16_max(float x) {
  x = fmaxf(x, dpp_move<0x128>(x));         // row_ror:8
  x = fmaxf(x, dpp_move<0x141>(x));         // row_half_mirror
  x = fmaxf(x, dpp_move<0x4E>(x));          // quad_perm:[2,3,0,1]
  return fmaxf(x, dpp_move<0xB1>(x));       // quad_perm:[1,0,3,2]
}

// Rounds a block of 128 elements, 8 in each of 16 lanes of a wave's row: their largest gives the power of two, the product with its inverse is exact (but for elements far below the
// smallest e4m3 number), so that an element is rounded once.
__device__ __forceinline__ void round_block(const float (&v)[8], uint8_t* values, uint8_t* power, bool held, bool first) {
  float top = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) top = fmaxf(top, finite(v[j]) ? fabsf(v[j]) : 0.f);
  const int e = e4m3_exponent(row16_max(top));
  const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
  float w[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) w[j] = v[j] * inv;
  if (held) *(uint2*)values = to_e4m3x8(w);
  if (first) *power = held ? (uint8_t)(e + 127) : 0;
}

// Agent scope: written through to the memory behind the XCDs' L2s, and read from there
__device__ __forceinline__ void put4(float* p, const float (&v)[4]) {
#pragma unroll
  for (int j = 0; j < 4; j += 2)
    __hip_atomic_store((uint64_t*)(p + j), (uint64_t)__float_as_uint(v[j]) | (uint64_t)__float_as_uint(v[j + 1]) << 32, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void get4(const float* p, float* v) {
#pragma unroll
  for (int j = 0; j < 4; j += 2) {
    const uint64_t u = __hip_atomic_load((const uint64_t*)(p + j), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    v[j] = __uint_as_float((uint32_t)u);
    v[j + 1] = __uint_as_float((uint32_t)(u >> 32));
  }
}

// Counts a workgroup in; the last of n goes on, for all.  What it reads was written through to memory before it was counted.  Leaves the counter at zero.  flag: a word of LDS that nobody reads any more
// once all threads are here.
__device__ __forceinline__ bool last_workgroup(uint32_t* counter, int n, int* flag) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) {
    const bool last = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)n - 1;
    if (last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *flag = last;
  }
  __syncthreads();
  return *flag != 0;
}

}  // namespace vvs
