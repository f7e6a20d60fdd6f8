// Products of rows and weights in 8 bits.
#include <algorithm>

#include "vvs_e4m3.h"
#include "vvs_qlinear.h"

namespace vvs {

// ------------------------------------------------------------------------------------------------ weights
// One wave per tile of 16 columns and block of 128 contraction values; lane 16 g + i has values 32 g .. 32 g + 31 of column i.  Once per model.
template <typename T>
__global__ __launch_bounds__(256) void k_qlinear_load(QLoad a) {
  const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
  const uint32_t unit = blockIdx.x * 4 + (threadIdx.x >> 6);
  const int t = unit & 3, block = (unit >> 2) % (uint32_t)a.w.blocks, group = (unit >> 2) / (uint32_t)a.w.blocks;
  if (group >= a.w.groups) return;
  const int col = a.w.column(group, t, i), k0 = block * kQRowBlock + g * 32;
  const T* src = (const T*)(a.w.gated && (t & 1) ? a.b : a.a);
  float v[32], top = 0.f;
#pragma unroll
  for (int j = 0; j < 32; ++j) {
    v[j] = col < a.w.out && k0 + j < a.w.in ? ld(src + (size_t)(k0 + j) * a.w.out + col) : 0.f;
    top = fmaxf(top, finite(v[j]) ? fabsf(v[j]) : 0.f);
  }
  const int e = e4m3_exponent(rows_max(top));
  const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
  uint32_t w[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) w[j] = to_e4m3x4(v[4 * j] * inv, v[4 * j + 1] * inv, v[4 * j + 2] * inv, v[4 * j + 3] * inv);
  uint4* dst = (uint4*)(a.w.data + a.w.tile_at(group, block, t));
  dst[lane] = make_uint4(w[0], w[1], w[2], w[3]);
  dst[64 + lane] = make_uint4(w[4], w[5], w[6], w[7]);
  uint8_t* power = a.w.powers + a.w.power_at(group, block, t) + i * 4;
  if (g == 0) *power = (uint8_t)(e + 127);
  // behind the last block: 0
  if (block == a.w.blocks - 1 && g > block % 4) power[g - block % 4] = 0;
}

template <typename T>
__global__ __launch_bounds__(256) void k_qlinear_read(QWeightsRead a) {
  const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
  const uint32_t unit = blockIdx.x * 4 + (threadIdx.x >> 6);
  const int t = unit & 3, block = (unit >> 2) % (uint32_t)a.w.blocks, group = (unit >> 2) / (uint32_t)a.w.blocks;
  if (group >= a.w.groups) return;
  const int col = a.w.column(group, t, i), k0 = block * kQRowBlock + g * 32;
  if (col >= a.w.out) return;
  T* dst = (T*)(a.w.gated && (t & 1) ? a.b : a.a);
  const uint4* src = (const uint4*)(a.w.data + a.w.tile_at(group, block, t));
  const float scale = __uint_as_float((uint32_t)a.w.powers[a.w.power_at(group, block, t) + i * 4] << 23);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint4 q = src[64 * h + lane];
    float v[8];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      from_e4m3x8(p ? make_uint2(q.z, q.w) : make_uint2(q.x, q.y), v);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int k = k0 + 16 * h + 8 * p + j;
        if (k < a.w.in) st(dst + (size_t)k * a.w.out + col, v[j] * scale);
      }
    }
  }
}

void launch_qlinear_load(const QLoad& a, hipStream_t s) {
  const dim3 grid((unsigned)((size_t)a.w.groups * a.w.blocks));
  if (a.dtype == VVS_BF16) hipLaunchKernelGGL(k_qlinear_load<bf16_t>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(k_qlinear_load<float>, grid, dim3(256), 0, s, a);
}

void launch_qlinear_read(const QWeightsRead& a, hipStream_t s) {
  const dim3 grid((unsigned)((size_t)a.w.groups * a.w.blocks));
  if (a.dtype == VVS_BF16) hipLaunchKernelGGL(k_qlinear_read<bf16_t>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(k_qlinear_read<float>, grid, dim3(256), 0, s, a);
}

// ------------------------------------------------------------------------------------------------ products
// 32 bytes of a lane's operand: 32 contraction values of one row or column
struct Held { uint4 h[2]; };
// ... as the operands of four 16x16x32 MFMAs in bf16, times their power of two (exact)
__device__ __forceinline__ bf16x8 part_of(const Held& x, int j, float scale) {
  const uint4 q = x.h[j >> 1];
  return e4m3_to_bf16(j & 1 ? make_uint2(q.z, q.w) : make_uint2(q.x, q.y), scale);
}

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

// Few rows.  A workgroup of 8 waves makes CT tiles of 16 columns for 16 RT rows; every wave takes each eighth block of the contraction, straight from memory into operand registers, and the
// eight partial sums are added through LDS in the order of the waves.
constexpr int kFewWaves = 8;
template <int RT, int CT, bool GATED, typename T>
__global__ __launch_bounds__(64 * kFewWaves) void k_qlinear_few(QProduct a) {
  extern __shared__ float4 parts[];          // [wave][CT][RT][lane]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4;
  const int group = blockIdx.x / (4 / CT), t0 = blockIdx.x % (4 / CT) * CT, m0 = blockIdx.y * 16 * RT;
  const int blocks = a.w.blocks, powers = qrows_powers(a.w.in);
  const size_t width = (size_t)blocks * kQRowBlock;
  size_t row[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) row[r] = min(m0 + 16 * r + i, a.M - 1);     // rows behind the last one repeat it
  floatx4 acc[CT][RT];
#pragma unroll
  for (int c = 0; c < CT; ++c)
#pragma unroll
    for (int r = 0; r < RT; ++r) acc[c][r] = floatx4{0.f, 0.f, 0.f, 0.f};
  for (int b = wave; b < blocks; b += kFewWaves) {
    Held w[CT], x[RT];
    float ws[CT], xs[RT];
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      const uint4* p = (const uint4*)(a.w.data + a.w.tile_at(group, b, t0 + c));
      w[c].h[0] = p[lane];
      w[c].h[1] = p[64 + lane];
      ws[c] = __uint_as_float((uint32_t)a.w.powers[a.w.power_at(group, b, t0 + c) + i * 4] << 23);
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const uint4* p = (const uint4*)(a.x.values + row[r] * width + (size_t)b * kQRowBlock + g * 32);
      x[r].h[0] = p[0];
      x[r].h[1] = p[1];
      xs[r] = __uint_as_float((uint32_t)a.x.powers[row[r] * powers + b] << 23);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      bf16x8 wj[CT];
#pragma unroll
      for (int c = 0; c < CT; ++c) wj[c] = part_of(w[c], j, ws[c]);
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const bf16x8 xj = part_of(x[r], j, xs[r]);
#pragma unroll
        for (int c = 0; c < CT; ++c) acc[c][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wj[c], xj, acc[c][r], 0, 0, 0);
      }
    }
  }
#pragma unroll
  for (int c = 0; c < CT; ++c)
#pragma unroll
    for (int r = 0; r < RT; ++r) parts[((wave * CT + c) * RT + r) * 64 + lane] = make_float4(acc[c][r][0], acc[c][r][1], acc[c][r][2], acc[c][r][3]);
  __syncthreads();
  auto whole = [&](int c, int r, int l, float (&v)[4]) {
    float4 s = parts[(c * RT + r) * 64 + l];
#pragma unroll
    for (int u = 1; u < kFewWaves; ++u) {
      const float4 p = parts[((u * CT + c) * RT + r) * 64 + l];
      s.x += p.x; s.y += p.y; s.z += p.z; s.w += p.w;
    }
    v[0] = s.x; v[1] = s.y; v[2] = s.z; v[3] = s.w;
  };
  constexpr int kPairs = GATED ? CT / 2 : CT;
  for (int u = threadIdx.x; u < kPairs * RT * 64; u += 64 * kFewWaves) {
    const int l = u & 63, r = (u >> 6) % RT, c = (u >> 6) / RT, m = m0 + 16 * r + (l & 15);
    if (m >= a.M) continue;
    float v[4];
    if constexpr (GATED) {
      float up[4];
      whole(2 * c, r, l, v);
      whole(2 * c + 1, r, l, up);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = silu(v[j]) * up[j];
      *(float4*)(a.act + (size_t)m * a.w.groups * 32 + a.w.column(group, t0 + 2 * c, 4 * (l >> 4))) = make_float4(v[0], v[1], v[2], v[3]);
    } else {
      whole(c, r, l, v);
      const int col = a.w.column(group, t0 + c, 4 * (l >> 4));
      store4((T*)a.y + (size_t)m * a.stride + col, a.w.out - col, a.wide, v);
    }
  }
}

template <int RT, int CT, bool GATED, typename T>
static void few_t(const QProduct& a, hipStream_t s) {
  const size_t lds = (size_t)kFewWaves * CT * RT * 64 * sizeof(float4);
  if (lds > 65536) allow_dynamic_lds((const void*)k_qlinear_few<RT, CT, GATED, T>, lds);
  hipLaunchKernelGGL((k_qlinear_few<RT, CT, GATED, T>), dim3(a.w.groups * (4 / CT), (a.M + 16 * RT - 1) / (16 * RT)), dim3(64 * kFewWaves), lds, s, a);
}

template <bool GATED, typename T>
static void few(const QProduct& a, hipStream_t s) {
  if (a.M <= 16) few_t<1, 2, GATED, T>(a, s);
  else if (a.M <= 32) few_t<2, 2, GATED, T>(a, s);
  else few_t<4, 4, GATED, T>(a, s);
}

void launch_qlinear_product(const QProduct& a, hipStream_t s) {
  if (a.w.gated) {
    few<true, float>(a, s);
    QRound r{};
    r.M = a.M; r.width = a.w.out; r.dtype = VVS_FP32;
    r.x = a.act; r.stride = (size_t)a.w.groups * 32; r.wide = 1;
    r.y = a.y8;
    launch_qrows_round(r, s);
  } else if (a.dtype == VVS_BF16) {
    few<false, bf16_t>(a, s);
  } else {
    few<false, float>(a, s);
  }
}

}  // namespace vvs
