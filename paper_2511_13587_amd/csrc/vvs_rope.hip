// Rotary positions on several axes.
#include "vvs_device.h"
#include "vvs_qcache.h"

namespace vvs {

// A workgroup takes kRopeTokens tokens: first the sines and cosines of all their pairs, once for all heads, then the heads, 8 elements a time.
// The angle is a product in 64 bits, counted in turns, so that taking whole turns off is exact: in 32 bits position 100000 would be off by 0.008 rad.
constexpr int kRopeTokens = 4;

// 8 elements of a row of partial sums
__device__ __forceinline__ void read8_sums(const RopeArgs& a, size_t at, float (&v)[8]) {
  read8(a.sums + at, v);
  for (int s = 1; s < a.splits; ++s) {
    float x[8];
    read8(a.sums + s * a.split_stride + at, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += x[j];
  }
}

template <typename T, bool HALVES, bool SUMS>
__global__ __launch_bounds__(256) void k_rope_axes(RopeArgs a) {
  __shared__ float2 turn[kRopeTokens][128];
  const int m0 = blockIdx.x * kRopeTokens, nm = min(kRopeTokens, a.M - m0);
  for (int i = threadIdx.x; i < nm * a.pairs; i += 256) {
    const int t = i / a.pairs, j = i % a.pairs;
    const double w = (double)a.pos[(size_t)(m0 + t) * a.axes + a.axis[j]] * a.turns[j];
    float sn, cs;
    sincospif((float)(2.0 * (w - rint(w))), &sn, &cs);
    turn[t][j] = make_float2(cs, a.inverse ? -sn : sn);
  }
  __syncthreads();
  // a unit: 8 elements, or two runs of 8 that rotate against each other (HALVES); then what is copied
  const int rot = HALVES ? a.pairs / 8 : a.pairs / 4, units = rot + (a.dh - 2 * a.pairs) / 8, all = (a.heads + (SUMS ? 2 : 1) * a.kv_heads) * units;
  for (int i = threadIdx.x; i < nm * all; i += 256) {
    const int t = i / all, u = i % all, hd = u / units, e = u % units;
    const bool is_k = hd >= a.heads;
    if (SUMS) {                                // a context's heads: adjacent pairs, all dims rotated; values are only added up
      const bool is_v = hd >= a.heads + a.kv_heads;
      const size_t row = m0 + t, d = (size_t)a.heads * a.dh;
      float v[8];
      read8_sums(a, row * (d + 2 * a.kv_heads * a.dh) + (size_t)hd * a.dh + e * 8, v);
      if (!is_v) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 c = turn[t][e * 4 + j];
          const float p = v[2 * j] * c.x - v[2 * j + 1] * c.y;
          v[2 * j + 1] = v[2 * j] * c.y + v[2 * j + 1] * c.x;
          v[2 * j] = p;
        }
      }
      T* y = (T*)(is_v ? a.v_out : is_k ? a.k_out : a.q_out) + row * (is_k ? a.kv_heads : a.heads) * a.dh + (size_t)(is_v ? hd - a.heads - a.kv_heads : is_k ? hd - a.heads : hd) * a.dh;
      write8(y + e * 8, v);
      continue;
    }
    const size_t m = m0 + t, at = (size_t)(is_k ? hd - a.heads : hd) * a.dh;
    const T* x = (const T*)(is_k ? a.k : a.q) + m * (is_k ? a.k_stride : a.q_stride) + at;
    T* y = (T*)(is_k ? a.k_out : a.q_out) + m * (is_k ? a.k_out_stride : a.q_out_stride) + at;
    float v[8];
    if (e >= rot) {
      const int d = 2 * a.pairs + (e - rot) * 8;
      read8(x + d, v);
      write8(y + d, v);
    } else if (HALVES) {
      float b[8], p[8], q[8];
      read8(x + e * 8, v);
      read8(x + a.pairs + e * 8, b);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float2 c = turn[t][e * 8 + j];
        p[j] = v[j] * c.x - b[j] * c.y;
        q[j] = v[j] * c.y + b[j] * c.x;
      }
      write8(y + e * 8, p);
      write8(y + a.pairs + e * 8, q);
    } else {
      read8(x + e * 8, v);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 c = turn[t][e * 4 + j];
        const float p = v[2 * j] * c.x - v[2 * j + 1] * c.y;
        v[2 * j + 1] = v[2 * j] * c.y + v[2 * j + 1] * c.x;
        v[2 * j] = p;
      }
      write8(y + e * 8, v);
    }
  }
}

template <typename T>
static void rope_t(const RopeArgs& a, hipStream_t s) {
  const dim3 grid((a.M + kRopeTokens - 1) / kRopeTokens);
  if (a.sums) hipLaunchKernelGGL((k_rope_axes<T, false, true>), grid, dim3(256), 0, s, a);
  else if (a.halves) hipLaunchKernelGGL((k_rope_axes<T, true, false>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((k_rope_axes<T, false, false>), grid, dim3(256), 0, s, a);
}

void launch_rope_axes(const RopeArgs& a, int dtype, hipStream_t s) {
  if (dtype == VVS_BF16) rope_t<bf16_t>(a, s);
  else rope_t<float>(a, s);
}

}  // namespace vvs
