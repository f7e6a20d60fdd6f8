// Rows in 8 bits: rounding, norm with the residual's addition, reading back.  All three are bound by HBM once there are some hundreds of rows and by the launch before; elements go through once, 8 to a thread,
// so that 16 neighbouring lanes hold a block and its largest value is found by four exchanges inside a row of 16 lanes (round_block), without LDS.
#include "vvs_qlinear_device.h"

namespace vvs {

// 8 elements from `at` on of a row of n; those behind its end are 0
template <typename T>
__device__ __forceinline__ void read_row8(const T* row, int at, int n, bool wide, float (&v)[8]) {
  if (wide && at + 8 <= n) {
    read8(row + at, v);
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = at + j < n ? ld(row + at + j) : 0.f;
}
template <typename T>
__device__ __forceinline__ void write_row8(T* row, int at, int n, bool wide, const float (&v)[8]) {
  if (wide && at + 8 <= n) {
    write8(row + at, v);
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (at + j < n) st(row + at + j, v[j]);
}

// y = e4m3(x / 2^E), E the least power that brings a block's largest value to 448 or less.  One unit of 16 lanes per block; blocks behind a row's last one (their number is rounded up to 4) are powers
// alone.  8191 rows of 4096 in bf16: 101 MB in 18.5 us, 5.5 TB/s (a copy of 4 GiB 4.7; part of these rows is still in the last-level cache); 432 rows of 1280 3.1 us.
template <typename T>
__global__ __launch_bounds__(256) void k_qrows_round(QRound a) {
  const int powers = qrows_powers(a.width), blocks = qrows_blocks(a.width);
  const uint32_t unit = blockIdx.x * 16u + (threadIdx.x >> 4);
  const int m = unit / (uint32_t)powers, b = unit % (uint32_t)powers, sub = threadIdx.x & 15;
  if (m >= a.M) return;
  float v[8];
  const int at = b * kQRowBlock + sub * 8;
  if constexpr (sizeof(T) == 2) {
    if (a.packed && at < a.width) read8((const T*)a.x + pack_index(m, at, a.width), v);      // (a multiple of 64 elements wide)
    else if (a.packed) read_row8((const T*)a.x, at, a.width, 1, v);
    else read_row8((const T*)a.x + (size_t)m * a.stride, at, a.width, a.wide, v);
  } else {
    read_row8((const T*)a.x + (size_t)m * a.stride, at, a.width, a.wide, v);
  }
  round_block(v, a.y.values + (size_t)m * blocks * kQRowBlock + at, a.y.powers + (size_t)m * powers + b, b < blocks, sub == 0);
}

void launch_qrows_round(const QRound& a, hipStream_t s) {
  const size_t units = (size_t)a.M * qrows_powers(a.width);
  const dim3 grid((unsigned)((units + 15) / 16));
  if (a.dtype == VVS_BF16) hipLaunchKernelGGL(k_qrows_round<bf16_t>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(k_qrows_round<float>, grid, dim3(256), 0, s, a);
}

// x = y 2^E, the same units.  8191 rows of 4096 to bf16: 101 MB in 16.6 us, 6.1 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void k_qrows_read(QRowsRead a) {
  const int powers = qrows_powers(a.width), blocks = qrows_blocks(a.width);
  const uint32_t unit = blockIdx.x * 16u + (threadIdx.x >> 4);
  const int m = unit / (uint32_t)blocks, b = unit % (uint32_t)blocks, at = b * kQRowBlock + (threadIdx.x & 15) * 8;
  if (m >= a.M) return;
  float v[8];
  from_e4m3x8(*(const uint2*)(a.x.values + (size_t)m * blocks * kQRowBlock + at), v);
  const float scale = __uint_as_float((uint32_t)a.x.powers[(size_t)m * powers + b] << 23);
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] *= scale;
  write_row8((T*)a.y + (size_t)m * a.stride, at, a.width, a.wide, v);
}

void launch_qrows_read(const QRowsRead& a, hipStream_t s) {
  const size_t units = (size_t)a.M * qrows_blocks(a.width);
  const dim3 grid((unsigned)((units + 15) / 16));
  if (a.dtype == VVS_BF16) hipLaunchKernelGGL(k_qrows_read<bf16_t>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(k_qrows_read<float>, grid, dim3(256), 0, s, a);
}

__device__ __forceinline__ void read_any8(const void* row, int dtype, int at, int n, bool wide, float (&v)[8]) {
  if (dtype == VVS_BF16) read_row8((const bf16_t*)row, at, n, wide, v);
  else read_row8((const float*)row, at, n, wide, v);
}

// x' = x + delta, y = x' g / sqrt(mean(x'^2) + eps), in 8 bits.  One workgroup per row, which stays in registers, V times 8 elements per thread, so that x and delta are read once and nothing is read back; a
// barrier for the sum is the only meeting of the waves (but in rows whose squares fp32 does not hold).  x' is rounded to the residual's type, and what is normalised is what is kept.
// 8192 rows of 4096, x, delta and x' in bf16: 235 MB in 48.1 us, 4.9 TB/s, where a copy of 4 GiB has 4.7; few rows wait for a
// chain of loads, sum, barrier, rounding: 10 rows of 128 3.9 us, 432 rows of 1280 4.6.  Loads of bf16 are turned to fp32 where they are made: each of x, delta and gain that is in bf16 is waited for before the next is asked
// for, and off 16 bytes each element of it.
template <int V, int MOST>
__global__ __launch_bounds__(MOST) void k_qrows_norm(QNorm a) {
  __shared__ float red[16];
  const int m = blockIdx.x, blocks = qrows_blocks(a.width), powers = qrows_powers(a.width);
  const size_t esz = a.x_dtype == VVS_BF16 ? 2 : 4, dsz = a.delta_dtype == VVS_BF16 ? 2 : 4;
  float v[V][8];
#pragma unroll
  for (int j = 0; j < V; ++j) read_any8((const char*)a.x + (size_t)m * a.x_stride * esz, a.x_dtype, (j * blockDim.x + threadIdx.x) * 8, a.width, a.x_wide, v[j]);
  if (a.delta) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      float d[8];
      read_any8((const char*)a.delta + (size_t)m * a.delta_stride * dsz, a.delta_dtype, (j * blockDim.x + threadIdx.x) * 8, a.width, a.delta_wide, d);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[j][i] += d[i];
        if (a.x_dtype == VVS_BF16) v[j][i] = bf2f(f2bf(v[j][i]));
      }
    }
  }
  // the gain is on its way while the sum is taken (but for the widest rows, which fill the registers)
  constexpr bool kAhead = V <= 4;
  float g[kAhead ? V : 1][8];
  if constexpr (kAhead) {
#pragma unroll
    for (int j = 0; j < V; ++j) read_any8(a.gain, a.gain_dtype, (j * blockDim.x + threadIdx.x) * 8, a.width, a.gain_wide, g[j]);
  }
  float ss = 0.f;
#pragma unroll
  for (int j = 0; j < V; ++j) {
#pragma unroll
    for (int i = 0; i < 8; ++i) ss += v[j][i] * v[j][i];
  }
  if (a.x_out) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int at = (j * blockDim.x + threadIdx.x) * 8;
      if (a.x_dtype == VVS_BF16) write_row8((bf16_t*)a.x_out + (size_t)m * a.x_out_stride, at, a.width, a.x_out_wide, v[j]);
      else write_row8((float*)a.x_out + (size_t)m * a.x_out_stride, at, a.width, a.x_out_wide, v[j]);
    }
  }
  // The waves' sums are added, and the factor is taken, in 64 bits, so that it is off by one rounding, not by several that a whole row would share: values end next to a border of e4m3 now and then.
  // (8192 rows of 4096 in bf16: 49.2 us, 49.5 all in fp32; an element's two products exact as well 52.6, in 64 bits 53.4)
  auto sum_of_waves = [&](float mine) {
    mine = wave_sum(mine);
    double all = mine;
    if (blockDim.x > 64) {
      if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = mine;
      __syncthreads();
      all = 0.0;
      for (int w = 0; w < (int)(blockDim.x >> 6); ++w) all += red[w];
    }
    return all;
  };
  double all = sum_of_waves(ss), eps = a.eps;
  // Squares below 2^-126 lose bits and those below 2^-149 vanish (65536 of them are 2^-30 of a sum of 2^-80; an eps from 2^-50 on hides them all), and a sum may overflow.  Then the row is brought to
  // 1 .. 2 by a power of two, exactly, and eps by its square, and summed again: the same quotient.  All threads have the same sum, and go the same way.
  if (!(all < INFINITY) || (all < 0x1p-80 && a.eps < 0x1p-50f)) {
    float top = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) {
#pragma unroll
      for (int i = 0; i < 8; ++i) top = fmaxf(top, finite(v[j][i]) ? fabsf(v[j][i]) : 0.f);
    }
    top = wave_max(top);
    if (blockDim.x > 64) {
      __syncthreads();                                  // (the sums have been read)
      if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = top;
      __syncthreads();
      for (int w = 0; w < (int)(blockDim.x >> 6); ++w) top = fmaxf(top, red[w]);
      __syncthreads();
    }
    const int shift = top > 0.f ? -ilogbf(top) : 0;
    ss = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[j][i] = ldexpf(v[j][i], shift);
        ss += v[j][i] * v[j][i];
      }
    }
    all = sum_of_waves(ss);
    eps = ldexp(eps, 2 * shift);
  }
  // (fp32's reciprocal root and one step of Newton's method)
  const double mean = all * a.per_element + eps;
  double factor = rsqrtf((float)mean);
  factor = factor > 0.0 && factor < INFINITY ? factor * (1.5 - 0.5 * mean * factor * factor) : 1.0 / sqrt(mean);
  const float r = (float)factor;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int at = (j * blockDim.x + threadIdx.x) * 8, b = at / kQRowBlock;
    if (b >= powers) break;
    if constexpr (!kAhead) read_any8(a.gain, a.gain_dtype, at, a.width, a.gain_wide, g[0]);
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = at + i < a.width ? v[j][i] * r * g[kAhead ? j : 0][i] : 0.f;
    round_block(y, a.y.values + (size_t)m * blocks * kQRowBlock + at, a.y.powers + (size_t)m * powers + b, b < blocks, (threadIdx.x & 15) == 0);
  }
}

void launch_qrows_norm(const QNorm& a, hipStream_t s) {
  // 8 elements per thread as long as the row fits (4096 wide: 28 rows 3.5 us, 432 rows 6.8, 8192 rows in bf16 49.0; 16 elements per thread 4.2, 7.5, 50.6; a wave per row 8.0, 11.3, 64.3).  Powers are in
  // fours, so that whole waves cover them.
  const int units = qrows_powers(a.width) * 16;
  auto go = [&](auto kernel, int v) { hipLaunchKernelGGL(kernel, dim3(a.M), dim3(((units + v - 1) / v + 63) & ~63), 0, s, a); };
  if (units <= 512) go(k_qrows_norm<1, 512>, 1);
  else if (units <= 1024) go(k_qrows_norm<1, 1024>, 1);
  else if (units <= 2048) go(k_qrows_norm<2, 1024>, 2);   // (4096 rows of 11008 in bf16 79.9 us, 32 elements per thread 88.6)
  else if (units <= 4096) go(k_qrows_norm<4, 1024>, 4);
  else go(k_qrows_norm<8, 1024>, 8);
}

}  // namespace vvs
