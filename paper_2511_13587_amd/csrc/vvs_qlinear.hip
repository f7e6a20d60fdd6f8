// Products of rows and weights in 8 bits.
#include <algorithm>

#include "vvs_e4m3.h"
#include "vvs_qlinear_device.h"

namespace vvs {

// ------------------------------------------------------------------------------------------------ weights
// One wave per tile of 16 columns and block of 128 contraction values; lane 16 g + i has values 32 g .. 32 g + 31 of column i, whose bytes it stores as the products load them.  Once per model: bound by reads
// of 32 or 64 bytes in a row (4096 x 12288 from fp32 201 MB in 48 us, 4.2 TB/s).
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
// Few rows: Y^T = W^T X^T in tiles of 16 columns x 16 rows.  A workgroup of NW waves makes CT tiles of 16 columns for 16 RT rows; wave w takes blocks w, w + NW, ... of the contraction, straight from
// memory into operand registers, and the partial sums are added through LDS in the order of the waves.  Powers of all blocks lie in LDS, four in a word.  A block is asked for in front of the products of the one before,
// under a condition; where the paths join the compiler waits for the youngest loads, so that of every two blocks one is on its way during products and the other is waited for at once.  The powers are asked for behind the
// first blocks, a word per thread at a time, rows' first: each round is a memory latency (4096 values: two; 11008: four).
// Bound by the weights' bytes where they are many (14 rows, gated, 4096 -> 11008, 91 MB in 18.8 us, 4.8 TB/s), by the latencies of powers, first blocks, every other block, the exchange through LDS and the launch
// where not: 28 rows, 11008 -> 4096, 45 MB in 13.7 us, 3.3 TB/s; 10 rows, 344 -> 128 3.3 us.  Every wave has its part of the contraction, not of the columns: a wave alone with 11008 values would go through 86 blocks one after another.
// Weights pass LDS by: nobody shares them.  Products are those of bf16 operands: an e4m3 number times its power of two is one exactly (8 bits of exponent, 3 of mantissa), so that what is summed in fp32
// are the true products; turning eight of a lane's numbers takes four instructions, and the matrix cores wait for memory anyway (busy 8 % of the time in the gated case above, waves waiting for loads 56 %).
// (Two and three blocks ahead, under the same kind of condition: 28 rows, 4096 -> 12288 18.6, 20.2 us for 17.1.)
template <int NW, int RT, int CT, bool GATED, typename T>
__global__ __launch_bounds__(64 * NW) void k_qlinear_few(QProduct a) {
  extern __shared__ float4 parts[];          // [wave][CT][RT][lane]; until the products are made the powers: rows [16 RT][stride], columns [16 CT][stride]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, g = lane >> 4;
  const int group = blockIdx.x / (4 / CT), t0 = blockIdx.x % (4 / CT) * CT, m0 = blockIdx.y * 16 * RT;
  const int blocks = a.w.blocks, powers = qrows_powers(a.w.in), words = powers / 4, stride = words | 1;
  const size_t width = (size_t)blocks * kQRowBlock;
  const uint8_t* const rows = a.x.values + (size_t)m0 * width;
  uint32_t row[RT];                          // rows behind the last one repeat it
#pragma unroll
  for (int r = 0; r < RT; ++r) row[r] = (uint32_t)(min(16 * r + i, a.M - 1 - m0) * (int)width + g * 32);
  floatx4 acc[CT][RT];
#pragma unroll
  for (int c = 0; c < CT; ++c)
#pragma unroll
    for (int r = 0; r < RT; ++r) acc[c][r] = floatx4{0.f, 0.f, 0.f, 0.f};
  u32x4 w[2][CT][2], x[2][RT][2];
  auto request = [&](int b, u32x4 (&wb)[CT][2], u32x4 (&xb)[RT][2]) {
    const uint8_t* p = a.w.data + a.w.tile_at(group, b, t0);
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      wb[c][0] = *(const u32x4*)(p + c * 2048 + lane * 16);
      wb[c][1] = *(const u32x4*)(p + c * 2048 + 1024 + lane * 16);
    }
    const uint8_t* q = rows + (size_t)b * kQRowBlock;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      xb[r][0] = *(const u32x4*)(q + row[r]);
      xb[r][1] = *(const u32x4*)(q + row[r] + 16);
    }
  };
  int* const xpow = (int*)parts;
  int* const wpow = xpow + 16 * RT * stride;
  const int* const mine_xpow = xpow + i * stride;
  const int* const mine_wpow = wpow + i * stride;
  auto multiply = [&](int b, const u32x4 (&wb)[CT][2], const u32x4 (&xb)[RT][2]) {
    const int at = b >> 2, sh = 8 * (b & 3);
    int ws[CT], xs[RT];
#pragma unroll
    for (int c = 0; c < CT; ++c) ws[c] = mine_wpow[c * 16 * stride + at] >> sh & 0xFF;
#pragma unroll
    for (int r = 0; r < RT; ++r) xs[r] = mine_xpow[r * 16 * stride + at] >> sh & 0xFF;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      bf16x8 wj[CT];
#pragma unroll
      for (int c = 0; c < CT; ++c) wj[c] = e4m3_to_bf16(make_uint2(wb[c][j >> 1][2 * (j & 1)], wb[c][j >> 1][2 * (j & 1) + 1]), __uint_as_float((uint32_t)ws[c] << 23));
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const bf16x8 xj = e4m3_to_bf16(make_uint2(xb[r][j >> 1][2 * (j & 1)], xb[r][j >> 1][2 * (j & 1) + 1]), __uint_as_float((uint32_t)xs[r] << 23));
#pragma unroll
        for (int c = 0; c < CT; ++c) acc[c][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wj[c], xj, acc[c][r], 0, 0, 0);
      }
    }
  };
  // this workgroup's blocks: b0 .. b1 - 1
  const int b0 = (int)((int64_t)blocks * blockIdx.z / gridDim.z), b1 = (int)((int64_t)blocks * (blockIdx.z + 1) / gridDim.z);
  if (b0 + wave < b1) request(b0 + wave, w[0], x[0]);
  for (int u = tid; u < 16 * RT * words; u += 64 * NW) {
    const int r = u / words, d = u % words;
    xpow[r * stride + d] = *(const int*)(a.x.powers + (size_t)min(m0 + r, a.M - 1) * powers + d * 4);
  }
  {
    const int* p = (const int*)(a.w.powers + a.w.power_at(group, 0, t0));
    for (int u = tid; u < 16 * CT * words; u += 64 * NW) wpow[u % (16 * CT) * stride + u / (16 * CT)] = p[u / (16 * CT) * 64 + u % (16 * CT)];
  }
  __syncthreads();
  for (int b = b0 + wave; b < b1; b += 2 * NW) {
    if (b + NW < b1) request(b + NW, w[1], x[1]);
    multiply(b, w[0], x[0]);
    if (b + 2 * NW < b1) request(b + 2 * NW, w[0], x[0]);
    if (b + NW < b1) multiply(b + NW, w[1], x[1]);
  }
  __syncthreads();
#pragma unroll
  for (int c = 0; c < CT; ++c)
#pragma unroll
    for (int r = 0; r < RT; ++r) parts[((wave * CT + c) * RT + r) * 64 + lane] = make_float4(acc[c][r][0], acc[c][r][1], acc[c][r][2], acc[c][r][3]);
  __syncthreads();
  const int busy = min(NW, b1 - b0);
  auto whole = [&](int c, int r, int l, float (&v)[4]) {
    float4 s = parts[(c * RT + r) * 64 + l];
    for (int u = 1; u < busy; ++u) {
      const float4 p = parts[((u * CT + c) * RT + r) * 64 + l];
      s.x += p.x; s.y += p.y; s.z += p.z; s.w += p.w;
    }
    v[0] = s.x; v[1] = s.y; v[2] = s.z; v[3] = s.w;
  };
  auto last_of = [&](uint32_t* counter, int n) { return last_workgroup(counter, n, (int*)parts); };
  if constexpr (GATED) {
    for (int u = tid; u < CT / 2 * RT * 64; u += 64 * NW) {
      const int l = u & 63, r = (u >> 6) % RT, c = (u >> 6) / RT, m = m0 + 16 * r + (l & 15);
      float v[4], up[4];
      whole(2 * c, r, l, v);
      whole(2 * c + 1, r, l, up);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = silu(v[j]) * up[j];
      if (m < a.M) put4(a.act + (size_t)m * a.w.groups * 32 + a.w.column(group, t0 + 2 * c, 4 * (l >> 4)), v);
    }
    // a block of 128 hidden units is that of 16 / CT workgroups
    if (!last_of(a.counters + blockIdx.y * (a.w.groups / 4) + group / 4, 16 / CT)) return;
    const int out_blocks = qrows_blocks(a.w.out), out_powers = qrows_powers(a.w.out), block = group / 4, sub = tid & 15;
    for (int r = tid >> 4; r < 16 * RT; r += 4 * NW) {
      const int m = m0 + r;
      if (m >= a.M || block >= out_blocks) break;
      float v[8];
      const float* p = a.act + (size_t)m * a.w.groups * 32 + block * kQRowBlock + sub * 8;
      get4(p, v);
      get4(p + 4, v + 4);
      // units behind the last one are held as 0, also in a row whose other units are NaN (a product with weights of 0 is not always 0)
      const int left = a.w.out - block * kQRowBlock - sub * 8;
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = j < left ? v[j] : 0.f;
      uint8_t* power = a.y8.powers + (size_t)m * out_powers;
      round_block(v, a.y8.values + ((size_t)m * out_blocks + block) * kQRowBlock + sub * 8, power + block, true, sub == 0);
      if (block == out_blocks - 1 && sub > 0 && block + sub < out_powers) power[block + sub] = 0;
    }
  } else {
    const int splits = gridDim.z, unit = blockIdx.y * gridDim.x + blockIdx.x;
    float* const mine = a.act + (size_t)unit * splits * (CT * RT * 256);      // [split][CT][RT][lane][4]
    if (splits > 1) {
      for (int u = tid; u < CT * RT * 64; u += 64 * NW) {
        float v[4];
        whole((u >> 6) / RT, (u >> 6) % RT, u & 63, v);
        put4(mine + ((size_t)blockIdx.z * CT * RT * 64 + u) * 4, v);
      }
      if (!last_of(a.counters + unit, splits)) return;
    }
    for (int u = tid; u < CT * RT * 64; u += 64 * NW) {
      const int l = u & 63, r = (u >> 6) % RT, c = (u >> 6) / RT, m = m0 + 16 * r + (l & 15);
      if (m >= a.M) continue;
      float v[4];
      if (splits > 1) {
        get4(mine + (size_t)u * 4, v);
        for (int z = 1; z < splits; ++z) {
          float p[4];
          get4(mine + ((size_t)z * CT * RT * 64 + u) * 4, p);
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] += p[j];
        }
      } else {
        whole(c, r, l, v);
      }
      const int col = a.w.column(group, t0 + c, 4 * (l >> 4));
      store4((T*)a.y + (size_t)m * a.stride + col, a.w.out - col, a.wide, v);
    }
  }
}

template <int NW, int RT, int CT, bool GATED, typename T>
static void few_t(const QProduct& a, int splits, hipStream_t s) {
  const size_t parts = (size_t)NW * CT * RT * 64 * sizeof(float4), powers = (size_t)16 * (RT + CT) * ((qrows_powers(a.w.in) / 4) | 1) * 4, lds = std::max(parts, powers);
  auto kernel = k_qlinear_few<NW, RT, CT, GATED, T>;
  if (lds > 65536) allow_dynamic_lds((const void*)kernel, kMostLds);
  hipLaunchKernelGGL(kernel, dim3(a.w.groups * (4 / CT), (a.M + 16 * RT - 1) / (16 * RT), splits), dim3(64 * NW), lds, s, a);
}

template <typename T>
static void few(const QProduct& a, const QPlan& p, hipStream_t s) {
  if (p.rt == 1 && p.ct == 1) few_t<8, 1, 1, false, T>(a, p.splits, s);
  else if (p.rt == 1) few_t<4, 1, 2, false, T>(a, p.splits, s);
  else if (p.ct == 2) few_t<8, 2, 2, false, T>(a, p.splits, s);
  else few_t<8, 2, 4, false, T>(a, p.splits, s);
}

void launch_qlinear_product(const QProduct& a, const QPlan& p, hipStream_t s) {
  if (!p.few) launch_qlinear_tile(a, p.tile, p.splits, s);
  else if (a.w.gated && p.rt == 1) few_t<4, 1, 2, true, float>(a, 1, s);
  else if (a.w.gated) few_t<4, 2, 2, true, float>(a, 1, s);
  else if (a.dtype == VVS_BF16) few<bf16_t>(a, p, s);
  else few<float>(a, p, s);
}

}  // namespace vvs
