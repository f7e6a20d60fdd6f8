// Key/value cache in 8 bits: append, attention with counted weights, eviction, read.
#include <float.h>
#include <limits.h>
#include <algorithm>

#include "vvs_e4m3.h"
#include "vvs_qcache.h"

namespace vvs {

constexpr float kLn2 = 0.6931471805599453f;
constexpr float kQSmall = 0x1p-110f;   // 2^kQLeast

__device__ __forceinline__ int row_len(const QLen& len, int r, int capacity) { return min(max(len.len ? len.len[r >> len.shift] : len.fixed, 0), capacity); }

// Byte of (slot w of a block, dim) in the block's keys and in its values (vvs_qcache.h)
__device__ __forceinline__ int key_byte(int w, int dim) {
  const int i = ((w >> 3) << 2) | (w & 3), t = (w >> 2) & 1;
  return (((dim >> 5) * 64 + ((dim >> 3) & 3) * 16 + i) * 2 + t) * 8 + (dim & 7);
}
__device__ __forceinline__ int value_byte(int w, int dim) { return (((dim >> 5) * 64 + (w >> 3) * 16 + (dim & 15)) * 2 + ((dim >> 4) & 1)) * 8 + (w & 7); }


// Transposes of 8 x 8 elements between the 8 lanes l % 8 (lane: a row, element: a column), in registers: half of what a lane holds is exchanged with the lane 4 on, 2 on, 1 on.
// What the cache wants of the values - 8 slots of one dim in a lane - is the transpose of what memory gives - 8 dims of one slot.
__device__ __forceinline__ uint32_t lane_xor1(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, 0xB1, 0xF, 0xF, false); }
__device__ __forceinline__ uint32_t lane_xor2(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, 0x4E, 0xF, 0xF, false); }
__device__ __forceinline__ uint32_t lane_xor4(uint32_t x) {
  const int y = __builtin_amdgcn_update_dpp((int)x, (int)x, 0x141, 0xF, 0xF, false);             // row_half_mirror, then quad_perm:[3,2,1,0]
  return (uint32_t)__builtin_amdgcn_update_dpp(y, y, 0x1B, 0xF, 0xF, false);
}
__device__ __forceinline__ void swap_rows(uint32_t& a, uint32_t& b, bool odd, uint32_t (*partner)(uint32_t)) {
  const uint32_t got = partner(odd ? a : b);
  a = odd ? got : a;
  b = odd ? b : got;
}
__device__ __forceinline__ uint2 transpose_bytes(uint2 v, int lane) {
  swap_rows(v.x, v.y, lane & 4, lane_xor4);
  const uint32_t half = lane & 2 ? 0x03020706u : 0x05040100u, byte = lane & 1 ? 0x03070105u : 0x06020400u;
  v.x = __builtin_amdgcn_perm(lane_xor2(v.x), v.x, half);
  v.y = __builtin_amdgcn_perm(lane_xor2(v.y), v.y, half);
  v.x = __builtin_amdgcn_perm(lane_xor1(v.x), v.x, byte);
  v.y = __builtin_amdgcn_perm(lane_xor1(v.y), v.y, byte);
  return v;
}
__device__ __forceinline__ uint4 transpose_halves(uint4 v, int lane) {
  swap_rows(v.x, v.z, lane & 4, lane_xor4);
  swap_rows(v.y, v.w, lane & 4, lane_xor4);
  swap_rows(v.x, v.y, lane & 2, lane_xor2);
  swap_rows(v.z, v.w, lane & 2, lane_xor2);
  const uint32_t half = lane & 1 ? 0x03020706u : 0x05040100u;
  v.x = __builtin_amdgcn_perm(lane_xor1(v.x), v.x, half);
  v.y = __builtin_amdgcn_perm(lane_xor1(v.y), v.y, half);
  v.z = __builtin_amdgcn_perm(lane_xor1(v.z), v.z, half);
  v.w = __builtin_amdgcn_perm(lane_xor1(v.w), v.w, half);
  return v;
}

// slot of tile t's row that lane l % 16 = i supplies (keys), and the one whose dims it takes before the transpose (values)
__device__ __forceinline__ int slot_of(int t, int i) { return 8 * (i >> 2) + 4 * t + (i & 3); }
__device__ __forceinline__ int value_slot(int lane) { return 8 * (lane >> 4) + (lane & 7); }

// ------------------------------------------------------------------------------------------------ append
// One wave per (layer, row, head, block that is written into); heads are next to each other in a workgroup, as their elements are in memory.  A lane loads the 16 bytes
// (fp32: 32) of 8 dims of the slots that it stores, all at once; their largest gives E; what the block held already is only read where it shares 8 bytes with new slots, or where E grew.
template <typename T, int DH>
__global__ __launch_bounds__(256) void k_qcache_append(QAppend a, int max_blocks) {
  constexpr int KD = DH / 32;
  const int lane = threadIdx.x & 63, unit = blockIdx.x * 4 + (threadIdx.x >> 6), r = blockIdx.y, layer = blockIdx.z;
  const int head = unit % a.c.kv_heads, nth = unit / a.c.kv_heads;
  if (nth >= max_blocks) return;
  if (a.skip && a.skip[r >> a.len.shift] < 0) return;
  const int len = row_len(a.len, r, a.capacity);
  const int want = a.n_tokens ? min(max(a.n_tokens[r >> a.n_shift] + a.count_plus, 0), a.n) : a.n, n = min(want, a.capacity - len);
  const int block = (len >> 5) + nth, slot0 = block * kQBlock;
  if (n < 1 || slot0 >= len + n) return;
  const int begin = max(len - slot0, 0), end = min(len + n - slot0, kQBlock);   // slots of the block that are written
  const size_t region = a.c.region(a.layer + layer, r, head);
  uint8_t* data = a.c.data + (region * a.c.blocks + block) * a.c.block_bytes();
  float2* scale = a.c.scale + region * a.c.blocks + block;
  const float2 was = *scale;
  if (a.pos && lane >= begin && lane < end) {
    const size_t at = region * a.capacity + slot0 + lane;
    if (a.mass) a.mass[at] = 0.f;
    a.pos[at] = a.pos_base ? a.pos_base[r >> a.len.shift] + a.pos_add + slot0 + lane - len : slot0 + lane;
  }
  // source token of slot w (slot w takes token w + slot0 - len), < 0: zeros
  auto token = [&](int w) {
    const int t = min(max(w, begin), end - 1) + slot0 - len;
    const int p = a.select ? a.select[(size_t)(r >> a.select_shift) * a.select_stride + t] : t;
    return p >= 0 && p < a.src_tokens ? p : -1;
  };
  const int g = lane >> 4, i = lane & 15;
  const int w_k[2] = {slot_of(0, i), slot_of(1, i)}, w_v = value_slot(lane);
  const int tok[3] = {token(w_k[0]), token(w_k[1]), token(w_v)};
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const T* src = (const T*)(half ? a.v : a.k) + (size_t)layer * a.layer_stride[half] + (size_t)r * a.src_tokens * a.stride[half] + (size_t)head * DH;
    float x[KD][2][8];
    float top = 0.f;
#pragma unroll
    for (int c = 0; c < KD; ++c)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int from = half ? tok[2] : tok[t], dim = half ? c * 32 + t * 16 + (i & 8) : c * 32 + 8 * g;
        read8(src + (size_t)max(from, 0) * a.stride[half] + dim, x[c][t]);
      }
#pragma unroll
    for (int c = 0; c < KD; ++c)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int w = half ? w_v : w_k[t];
        const bool is_new = w >= begin && w < end, there = w < end && (half ? tok[2] : tok[t]) >= 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float v = there ? x[c][t][j] : 0.f;
          x[c][t][j] = v;
          const float m = fabsf(v);
          top = fmaxf(top, is_new && m < INFINITY ? m : 0.f);
        }
      }
    const int was_e = exponent_of(half ? was.y : was.x);
    int e = e4m3_exponent(wave_max(top));
    if (begin > 0) e = max(e, was_e);
    const bool grew = begin > 0 && e > was_e;
    uint8_t* out = data + half * kQBlock * DH;
#pragma unroll
    for (int c = 0; c < KD; ++c)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float y = ldexpf(x[c][t][j], -e);
          v[j] = finite(y) ? y : __uint_as_float(0x7FC00000u);
        }
        uint2 bytes = to_e4m3x8(v);
        uint2* at = (uint2*)(out + (c * 64 + lane) * 16) + t;
        // the 8 bytes are one slot's dims (keys), or 8 slots of a dim (values): which of them are old
        const int first = half ? 8 * g : w_k[t], slots = half ? 8 : 1;
        if (half) bytes = transpose_bytes(bytes, lane);
        const bool has_new = first < end && first + slots > begin, has_old = first < begin;
        if (!has_new && !(grew && has_old)) continue;
        if (has_old) {
          uint2 held = *at;
          if (grew) {
            float old[8];
            from_e4m3x8(held, old);
#pragma unroll
            for (int j = 0; j < 8; ++j) old[j] = ldexpf(old[j], was_e - e);
            held = to_e4m3x8(old);
          }
          const int keep = begin - first;                    // leading bytes of the 8 that are old (keys: all)
          const uint64_t mask = !half || keep >= 8 ? ~0ull : (1ull << (8 * keep)) - 1;
          bytes.x = (held.x & (uint32_t)mask) | (bytes.x & ~(uint32_t)mask);
          bytes.y = (held.y & (uint32_t)(mask >> 32)) | (bytes.y & ~(uint32_t)(mask >> 32));
        }
        *at = bytes;
      }
    if (lane == 0) (half ? scale->y : scale->x) = ldexpf(1.f, e);
  }
}

template <typename T>
static void append_t(const QAppend& a, hipStream_t s) {
  const int max_blocks = (int)std::min<int64_t>(((int64_t)a.n + 2 * kQBlock - 2) / kQBlock, a.c.blocks);
  const dim3 grid(((int64_t)a.c.kv_heads * max_blocks + 3) / 4, a.c.rows, a.n_layers);
  if (a.c.dh == 32) hipLaunchKernelGGL((k_qcache_append<T, 32>), grid, dim3(256), 0, s, a, max_blocks);
  else if (a.c.dh == 64) hipLaunchKernelGGL((k_qcache_append<T, 64>), grid, dim3(256), 0, s, a, max_blocks);
  else hipLaunchKernelGGL((k_qcache_append<T, 128>), grid, dim3(256), 0, s, a, max_blocks);
}

void launch_qcache_append(const QAppend& a, int dtype, hipStream_t s) {
  if (dtype == VVS_BF16) append_t<bf16_t>(a, s);
  else append_t<float>(a, s);
}

// ------------------------------------------------------------------------------------------------ read
// One wave per (layer, row, head, block that the window touches): whole 16-byte pieces of the block, the values turned in registers.  The numbers go through LDS (32 slots at a
// time, a wave's own), so that a slot's dims are written side by side: straight from the registers a store covers 32 bytes of each of 32 slots.
template <typename T, int DH>
__global__ __launch_bounds__(256) void k_qcache_read(QRead a, int max_blocks) {
  constexpr int KD = DH / 32, PAD = 16 / sizeof(T), LANES = DH * sizeof(T) / 16;      // LANES: pieces of 16 bytes that make up a slot
  __shared__ __align__(16) T s_out[4][kQBlock][DH + PAD];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, unit = blockIdx.x * 4 + wave, r = blockIdx.y, layer = blockIdx.z;
  const int head = unit % a.c.kv_heads, nth = unit / a.c.kv_heads;
  if (nth >= max_blocks) return;
  const int len = row_len(a.len, r, a.capacity);
  const int64_t first = a.first ? a.first[r] : 0, block = (first >> 5) + nth, slot0 = block * kQBlock;
  if (slot0 >= first + a.n) return;
  const bool held = block >= 0 && slot0 < len;
  const size_t at = a.c.region(a.layer + layer, r, head) * a.c.blocks + (held ? (size_t)block : 0);
  const uint8_t* data = a.c.data + at * a.c.block_bytes();
  const float2 sc = a.c.scale[at];
  const size_t out0 = ((size_t)layer * a.c.rows + r) * a.n;
  const int g = lane >> 4, i = lane & 15;
  uint4 b[2][KD];
#pragma unroll
  for (int half = 0; half < 2; ++half)
#pragma unroll
    for (int c = 0; c < KD; ++c) b[half][c] = held ? *(const uint4*)(data + half * kQBlock * DH + (c * 64 + lane) * 16) : make_uint4(0, 0, 0, 0);
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const float unit_of = half ? sc.y : sc.x;
#pragma unroll
    for (int c = 0; c < KD; ++c)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        uint2 v8 = t ? make_uint2(b[half][c].z, b[half][c].w) : make_uint2(b[half][c].x, b[half][c].y);
        if (half) v8 = transpose_bytes(v8, lane);
        const int w = half ? value_slot(lane) : slot_of(t, i), dim = half ? c * 32 + t * 16 + (i & 8) : c * 32 + 8 * g;
        float v[8];
        from_e4m3x8(v8, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = held && slot0 + w < len ? v[j] * unit_of : 0.f;
        write8(&s_out[wave][w][dim], v);
      }
    __builtin_amdgcn_wave_barrier();
    T* out = (T*)(half ? a.v : a.k);
#pragma unroll
    for (int j = 0; j < kQBlock * LANES / 64; ++j) {
      const int w = (j * 64 + lane) / LANES, dim = lane % LANES * PAD;
      const uint4 x = *(const uint4*)&s_out[wave][w][dim];
      const int64_t slot = slot0 + w;
      if (slot >= first && slot < first + a.n) *(uint4*)(out + ((out0 + (size_t)(slot - first)) * a.c.kv_heads + head) * DH + dim) = x;
    }
    __builtin_amdgcn_wave_barrier();
  }
}

template <typename T>
static void read_t(const QRead& a, hipStream_t s) {
  const int max_blocks = (int)(((int64_t)a.n + 2 * kQBlock - 2) / kQBlock);
  const dim3 grid(((int64_t)a.c.kv_heads * max_blocks + 3) / 4, a.c.rows, a.n_layers);
  if (a.c.dh == 32) hipLaunchKernelGGL((k_qcache_read<T, 32>), grid, dim3(256), 0, s, a, max_blocks);
  else if (a.c.dh == 64) hipLaunchKernelGGL((k_qcache_read<T, 64>), grid, dim3(256), 0, s, a, max_blocks);
  else hipLaunchKernelGGL((k_qcache_read<T, 128>), grid, dim3(256), 0, s, a, max_blocks);
}

void launch_qcache_read(const QRead& a, int dtype, hipStream_t s) {
  if (dtype == VVS_BF16) read_t<bf16_t>(a, s);
  else read_t<float>(a, s);
}

// ------------------------------------------------------------------------------------------------ attention
// One wave takes 32 keys a step (a cached block, or 32 block tokens) against 16 NQB queries; a query is (block token, query head of the key/value head).
//
// Scores S^T = K Q^T: e4m3 numbers are exact in bf16, the block's power of two is multiplied into the softmax's constant.  Values go into O^T += V^T P^T as bf16 too, times their
// block's power of two (exact).  Weights are 2^(score c - M), M at most 2^6 below the largest exponent so far, so that the accumulators are rescaled only when a maximum grows by more
// than that; beside bf16 values they go as sums of two bf16 values (to 2^-17 of themselves, as in the contexts' attention), in fp32 calls as three, as queries, block keys and block values do,
// which hold all 24 bits.  The exponents of bf16 are those of fp32: a weight keeps its bits down to 2^-117 of the largest, and a block's power of two has no say in M.  (Single fp16 weights,
// times their block's power of two, took half of the products, but what lay 2^14 below the largest of them lost bits, and 2^25 below it vanished, beside a normaliser that had
// it: whole outputs behind a first token without value, small values behind a block of zeros.)  The normaliser sums the fp32 weights per lane; lanes, waves and splits are joined at the end,
// in a fixed order.

// x as a sum of NS bf16 values
template <int NS>
__device__ __forceinline__ void split8(const float (&x)[8], bf16x8 (&out)[NS]) {
  float rest[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) rest[i] = x[i];
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i] = pack2bf(rest[2 * i], rest[2 * i + 1]);
      rest[2 * i] -= __uint_as_float(w[i] << 16);
      rest[2 * i + 1] -= __uint_as_float(w[i] & 0xFFFF0000u);
    }
    out[n] = as_bf16x8(make_uint4(w[0], w[1], w[2], w[3]));
  }
}
template <int NS>
__device__ __forceinline__ void load_operand(const float* p, bf16x8 (&out)[NS]) {
  float v[8];
  read8(p, v);
  split8<NS>(v, out);
}
template <int NS>
__device__ __forceinline__ void load_operand(const bf16_t* p, bf16x8 (&out)[NS]) {
  static_assert(NS == 1, "");
  out[0] = as_bf16x8(*(const uint4*)p);
}

template <typename T, int DH>
struct QShape {
  static constexpr int NS = sizeof(T) == 4 ? 3 : 1;     // bf16 values that make up an operand of the caller's type
  static constexpr int NP = sizeof(T) == 4 ? 3 : 2;     // ... and a softmax weight
  static constexpr int KD = DH / 32, DT = DH / 16;
};

// A cached block in registers, as it lies in memory
template <int DH>
struct QRaw {
  uint4 k[DH / 32], v[DH / 32];
  float2 scale;
  __device__ __forceinline__ void load(const uint8_t* data, const float2* sc, int lane) {
#pragma unroll
    for (int c = 0; c < DH / 32; ++c) k[c] = *(const uint4*)(data + (c * 64 + lane) * 16);
#pragma unroll
    for (int c = 0; c < DH / 32; ++c) v[c] = *(const uint4*)(data + kQBlock * DH + (c * 64 + lane) * 16);
    scale = make_float2(fmaxf(sc->x, kQSmall), fmaxf(sc->y, kQSmall));     // (a block never written holds 0)
  }
  // slots from `valid` on are zeros among the values: what lies behind the length may be anything, NaN included
  __device__ __forceinline__ void mask_values(int lane, int valid) {
    const int mine = valid - 8 * (lane >> 4);       // of this lane's 8 slots
    const uint64_t keep = mine >= 8 ? ~0ull : mine <= 0 ? 0ull : (1ull << (8 * mine)) - 1;
#pragma unroll
    for (int c = 0; c < DH / 32; ++c) {
      v[c].x &= (uint32_t)keep; v[c].y &= (uint32_t)(keep >> 32); v[c].z &= (uint32_t)keep; v[c].w &= (uint32_t)(keep >> 32);
    }
  }
};

// Keys of a step of block tokens.  Tokens from n on are the last one again: their scores are masked.
template <typename T, int DH, int NS>
__device__ __forceinline__ void keys_of_tokens(const T* k, size_t stride, int tok0, int n, int lane, bf16x8 (&kf)[2][DH / 32][NS]) {
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const T* p = k + (size_t)min(tok0 + slot_of(t, lane & 15), n - 1) * stride + (lane >> 4) * 8;
#pragma unroll
    for (int kd = 0; kd < DH / 32; ++kd) load_operand<NS>(p + kd * 32, kf[t][kd]);
  }
}
// Values: 8 dims of one slot are loaded, and turned.  Zeros in the place of tokens from n on, and of elements that are not finite; returns whether this lane met any of those.
template <int DH, int NS>
__device__ __forceinline__ bool values_of_tokens(const float* v, size_t stride, int tok0, int n, int lane, bf16x8 (&vf)[DH / 16][NS]) {
  const int tok = tok0 + value_slot(lane);
  const float* p = v + (size_t)min(tok, n - 1) * stride + (lane & 8);
  bool odd = false;
#pragma unroll
  for (int dt = 0; dt < DH / 16; ++dt) {
    float x[8];
    read8(p + dt * 16, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const bool fin = finite(x[j]);
      odd |= !fin && tok < n;
      x[j] = fin && tok < n ? x[j] : 0.f;
    }
    bf16x8 part[NS];
    split8<NS>(x, part);
#pragma unroll
    for (int s = 0; s < NS; ++s) vf[dt][s] = as_bf16x8(transpose_halves(__builtin_bit_cast(uint4, part[s]), lane));
  }
  return odd;
}

// (bf16: one piece of 16 bytes; there: all ones, or 0 behind the last token; odd: not 0 if anything was not finite)
__device__ __forceinline__ uint4 turned_values(uint4 b, uint32_t there, int lane, uint32_t& odd) {
  uint32_t w[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    w[j] &= there;
    // exponents of all ones: the carry of one more into the sign, half by half
    const uint32_t bad = ((w[j] & 0x7F807F80u) + 0x00800080u) & 0x80008000u;
    odd |= bad;
    w[j] &= ~((bad >> 15) * 0xFFFFu);
  }
  return transpose_halves(make_uint4(w[0], w[1], w[2], w[3]), lane);
}
template <int DH, int NS>
__device__ __forceinline__ bool values_of_tokens(const bf16_t* v, size_t stride, int tok0, int n, int lane, bf16x8 (&vf)[DH / 16][NS]) {
  static_assert(NS == 1, "");
  const int tok = tok0 + value_slot(lane);
  const bf16_t* p = v + (size_t)min(tok, n - 1) * stride + (lane & 8);
  uint32_t odd = 0;
#pragma unroll
  for (int dt = 0; dt < DH / 16; ++dt) vf[dt][0] = as_bf16x8(turned_values(*(const uint4*)(p + dt * 16), tok < n ? 0xFFFFFFFFu : 0u, lane, odd));
  return odd != 0;
}

// scores of the step's 32 keys for 16 queries: lane (g, query) gets those of keys 8 g .. 8 g + 7
template <int KD, int NK, int NS>
__device__ __forceinline__ void step_scores(const bf16x8 (&kf)[2][KD][NK], const bf16x8 (&qf)[KD][NS], float (&sv)[8]) {
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    floatx4 s = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int sum = (NK > 1 ? NS - 1 : NS + NK - 2); sum >= 0; --sum)          // small products first; those below the last bit are left out
#pragma unroll
      for (int p = 0; p < NK; ++p) {
        if (sum - p < 0 || sum - p >= NS) continue;
#pragma unroll
        for (int kd = 0; kd < KD; ++kd) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[t][kd][p], qf[kd][sum - p], s, 0, 0, 0);
      }
#pragma unroll
    for (int j = 0; j < 4; ++j) sv[4 * t + j] = s[j];
  }
}

// What a wave carries along for 16 queries (column col of a lane): reference exponent (the same in all four lanes of a query), this lane's part of the normaliser, O^T
template <int DT>
struct QRun {
  float m, l;
  floatx4 o[DT];
  __device__ __forceinline__ void clear() {
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[dt] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  static __device__ __forceinline__ float top(const float (&sv)[8]) {
    return fmaxf(fmaxf(fmaxf(sv[0], sv[1]), fmaxf(sv[2], sv[3])), fmaxf(fmaxf(sv[4], sv[5]), fmaxf(sv[6], sv[7])));
  }
  // the reference follows where the largest exponent to come, `cand` in this lane, is more than 2^6 above it
  __device__ __forceinline__ void follow(float cand) {
    cand = rows_max(cand);
    if (__builtin_amdgcn_ballot_w64(cand > m + 6.f)) {
      const float to = fmaxf(m, cand), alpha = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - to);
      m = to;
      l *= alpha;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[dt][j] *= alpha;
    }
  }
  // weights of 8 keys, e[i] = 2^(sv[i] c - m), and their sum into the normaliser
  __device__ __forceinline__ void exponentials(const float (&sv)[8], float c, float (&e)[8]) {
    const float off = m == -INFINITY ? 0.f : -m;
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = __builtin_amdgcn_exp2f(fmaf(sv[i], c, off));
    l += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
  }
  __device__ __forceinline__ void weights(const float (&sv)[8], float c, float (&e)[8]) {
    follow(top(sv) * c);
    exponentials(sv, c, e);
  }
  template <int NK, int NP>
  __device__ __forceinline__ void add(const float (&e)[8], const bf16x8 (&vf)[DT][NK]) {
    bf16x8 pf[NP];
    split8<NP>(e, pf);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int sum = (NK > 1 ? NP - 1 : NP + NK - 2); sum >= 0; --sum)
#pragma unroll
        for (int p = 0; p < NK; ++p) {
          if (sum - p < 0 || sum - p >= NP) continue;
          o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[dt][p], pf[sum - p], o[dt], 0, 0, 0);
        }
  }
};

// What of the row a wave sees
struct QRow {
  int len, n, blocks;       // cached slots, block tokens, cached blocks
};

__device__ __forceinline__ QRow row_of(const QAttention& a, int r) {
  QRow w;
  w.len = row_len(a.len, r, a.capacity);
  w.n = a.n_tokens ? min(max(a.n_tokens[r], 0), a.T) : a.T;
  w.blocks = (w.len + kQBlock - 1) / kQBlock;
  return w;
}

// Block tokens that the queries in front of query `end` can see: with a chain none behind the last query
__device__ __forceinline__ int seen_by(const QAttention& a, const QRow& w, int end) {
  return !a.k || end < 1 ? 0 : a.causal ? min(w.n, (end - 1) / a.group + 1) : w.n;
}

// Bit i: query token t sees block token tok + i (below `seen`)
__device__ __forceinline__ uint32_t sees8(const QAttention& a, int t, int tok, int seen) {
  const int n = a.causal ? min(seen, t + 1) - tok : seen - tok;
  const uint32_t near = n >= 8 ? 255u : n <= 0 ? 0u : (1u << n) - 1;
  return a.causal ? near : near & (uint32_t)(a.anc[t & (VVS_MAX_T - 1)] >> (tok & (VVS_MAX_T - 1)));
}

// Where query `qi` of key/value head hk (t = qi / group) writes, as an index of [rows][T][heads]
__device__ __forceinline__ size_t query_at(const QAttention& a, int r, int hk, int qi) {
  return ((size_t)r * a.T + qi / a.group) * a.c.heads + (size_t)hk * a.group + qi % a.group;
}

template <typename T, int DH>
__device__ __forceinline__ void store4(const QAttention& a, size_t at, int dim, const float (&v)[4]) {
  if constexpr (sizeof(T) == 4) {
    *(float4*)((float*)a.out + at * DH + dim) = make_float4(v[0], v[1], v[2], v[3]);
  } else {
    const uint2 w = make_uint2(pack2bf(v[0], v[1]), pack2bf(v[2], v[3]));
    if (a.packed) {      // rows of the next projection: tokens, contraction: heads x dims
      const int token = (int)(at / a.c.heads), col = (int)(at % a.c.heads) * DH + dim;
      *(uint2*)((bf16_t*)a.out + pack_index(token, col, a.c.heads * DH)) = w;
    } else {
      *(uint2*)((bf16_t*)a.out + at * DH + dim) = w;
    }
  }
}

// log-sum-exp for the caller, and in units of log2 for the counted weights of many queries: as one number, so that its size takes some of the 24 bits, and weights are off by
// 2^-24 of |norm| relative to themselves (2^-18 at scores 64 powers of two from 0), as they are by the rounding of the scores
__device__ __forceinline__ void tell_norm(const QAttention& a, size_t at, float m, float l) {
  const bool none = l == 0.f;            // a query that sees nothing
  if (a.lse) a.lse[at] = none ? -INFINITY : (m + log2f(l)) * kLn2;
  if (a.norm) a.norm[at] = none ? INFINITY : m + log2f(l);
}

// Scores (times c: units of log2) that the main kernel leaves for the counted weights: [rows][kv heads][steps][counted queries][32 keys]
__device__ __forceinline__ float* kept_scores(const QAttention& a, int r, int hk, int step) {
  return a.scores + (((size_t)r * a.c.kv_heads + hk) * a.score_steps + step) * a.n_kept * kQBlock;
}

// Adds up the weights of one (row, key/value head) from the kept scores, 4 keys at a time: thread `first` of `by`.  norm: [n_queries] (reference exponent, 1 / sum); seen: block tokens that the
// counted queries' tile looked at (the others have weight 0)
__device__ __forceinline__ void mass_of_kept(const QAttention& a, const QRow& w, int r, int hk, const float2* norm, int n_queries, int seen, int first, int by) {
  const int steps = w.blocks + (a.block_mass ? (w.n + 31) / 32 : 0);
  float* mass = a.mass + ((size_t)r * a.c.kv_heads + hk) * a.capacity;
  float* block_mass = a.block_mass + ((size_t)r * a.c.kv_heads + hk) * a.block_stride;
  for (int i = first + (a.mass ? 0 : w.blocks * 8); i < steps * 8; i += by) {
    const int step = i >> 3, at = (i & 7) * 4;
    const bool cached = step < w.blocks;
    const int key = cached ? i * 4 : (i - w.blocks * 8) * 4, end = cached ? w.len : w.n, there = cached ? w.len : seen;
    const float* x = kept_scores(a, r, hk, step) + at;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    if (key < there)
      for (int q = 0; q < n_queries; ++q) {
        const float4 s = *(const float4*)(x + q * kQBlock);
        const float2 n = norm[q];
        sum[0] += __builtin_amdgcn_exp2f(s.x - n.x) * n.y;
        sum[1] += __builtin_amdgcn_exp2f(s.y - n.x) * n.y;
        sum[2] += __builtin_amdgcn_exp2f(s.z - n.x) * n.y;
        sum[3] += __builtin_amdgcn_exp2f(s.w - n.x) * n.y;
      }
    float* out = cached ? mass : block_mass;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (key + j < end) out[key + j] = (cached ? out[key + j] : 0.f) + (key + j < there ? sum[j] : 0.f);
  }
}

// Values of block tokens that are not finite (their places in the product held zeros): only for the queries that see them.  e: the step's weights
template <int DT, typename T>
__device__ __forceinline__ void add_odd_values(const QAttention& a, const T* v, const float (&e)[8], int t, int tok0, int seen, int lane, floatx4 (&o)[DT]) {
  for (int j = 0; j < 32 && tok0 + j < seen; ++j) {
    float p = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float x = __shfl(e[i], (j >> 3) * 16 + (lane & 15), 64);
      p = (j & 7) == i ? x : p;
    }
    const bool vis = sees8(a, t, tok0 + j, seen) & 1;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = ld(v + (size_t)(tok0 + j) * a.v_stride + dt * 16 + 4 * (lane >> 4) + i);
        o[dt][i] += vis && !finite(x) ? p * x : 0.f;
      }
  }
}

// grid (kv_heads * query tiles, splits, rows), 4 waves.  The steps of a split go to its waves in turn; the waves' results are joined through LDS.
template <typename T, int DH, int NQB>
__global__ __launch_bounds__(256, sizeof(T) == 4 && DH == 128 ? 1 : 2) void k_qcache_attention(QAttention a, int q_tiles) {
  using S = QShape<T, DH>;
  constexpr int KD = S::KD, DT = S::DT, NS = S::NS, NP = S::NP, NQ = 16 * NQB;
  __shared__ float s_o[2][NQ][DH + 4];
  __shared__ float s_m[4][NQ], s_l[4][NQ];
  __shared__ float2 s_norm[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, col = lane & 15;
  const int hk = blockIdx.x / q_tiles, q0 = (blockIdx.x % q_tiles) * NQ, r = blockIdx.z, split = blockIdx.y;
  const QRow w = row_of(a, r);
  const int nq = w.n * a.group;
  if (q0 >= nq) return;                       // only tokens behind the row's number
  const T* q = (const T*)a.q + (size_t)r * a.T * a.q_stride + (size_t)hk * a.group * DH;
  const T* k = (const T*)a.k + (size_t)r * a.T * a.k_stride + (size_t)hk * DH;
  const T* v = (const T*)a.v + (size_t)r * a.T * a.v_stride + (size_t)hk * DH;
  const size_t region = a.c.region(a.layer, r, hk) * a.c.blocks;
  bf16x8 qf[NQB][KD][NS];
  int qt[NQB];                                // block token of this lane's query
#pragma unroll
  for (int qb = 0; qb < NQB; ++qb) {
    const int qi = min(q0 + qb * 16 + col, nq - 1);
    qt[qb] = qi / a.group;
#pragma unroll
    for (int kd = 0; kd < KD; ++kd)
      load_operand<NS>(q + (size_t)qt[qb] * a.q_stride + (size_t)(qi % a.group) * DH + kd * 32 + g * 8, qf[qb][kd]);
  }
  QRun<DT> run[NQB];
#pragma unroll
  for (int qb = 0; qb < NQB; ++qb) run[qb].clear();
  // scores of the counted queries, the first ones, are kept by the tile that has them
  const int n_kept = a.n_kept && q0 == 0 ? min(a.n_kept, nq) : 0;
  auto keep_scores = [&](int step, const float (&sv)[8], float c) {
    if (col < n_kept) {
      float* p = kept_scores(a, r, hk, step) + col * kQBlock + 8 * g;
      ((float4*)p)[0] = make_float4(sv[0] * c, sv[1] * c, sv[2] * c, sv[3] * c);
      ((float4*)p)[1] = make_float4(sv[4] * c, sv[5] * c, sv[6] * c, sv[7] * c);
    }
  };
  const int seen = seen_by(a, w, min(q0 + NQ, nq));
  const int steps = w.blocks + (seen + 31) / 32;
  const int s0 = (int)((int64_t)steps * split / a.splits), s1 = (int)((int64_t)steps * (split + 1) / a.splits);
  const int cached_end = min(s1, w.blocks);
  const uint8_t* data = a.c.data + region * a.c.block_bytes();
  QRaw<DH> raw;
  int step = s0 + wave;
  if (step < cached_end) raw.load(data + (size_t)step * a.c.block_bytes(), a.c.scale + region + step, lane);
  for (; step < cached_end; step += 4) {
    const int valid = w.len - step * kQBlock;
    if (valid < kQBlock) raw.mask_values(lane, valid);
    const float2 sc = raw.scale;
    bf16x8 kf[2][KD][1];
#pragma unroll
    for (int c = 0; c < KD; ++c) {
      kf[0][c][0] = e4m3_to_bf16(make_uint2(raw.k[c].x, raw.k[c].y), 1.f);
      kf[1][c][0] = e4m3_to_bf16(make_uint2(raw.k[c].z, raw.k[c].w), 1.f);
    }
    const float c_exp = fmaxf(a.c_exp * sc.x, FLT_MIN);     // above 0: masked scores are -inf
    uint4 vraw[KD];
#pragma unroll
    for (int c = 0; c < KD; ++c) vraw[c] = raw.v[c];
    // the wave's next block is on its way meanwhile
    if (step + 4 < cached_end) raw.load(data + (size_t)(step + 4) * a.c.block_bytes(), a.c.scale + region + step + 4, lane);
    bf16x8 vf[DT][1];
#pragma unroll
    for (int c = 0; c < KD; ++c) {
      vf[2 * c][0] = e4m3_to_bf16(make_uint2(vraw[c].x, vraw[c].y), sc.y);
      vf[2 * c + 1][0] = e4m3_to_bf16(make_uint2(vraw[c].z, vraw[c].w), sc.y);
    }
#pragma unroll
    for (int qb = 0; qb < NQB; ++qb) {
      float sv[8], e[8];
      step_scores<KD, 1, NS>(kf, qf[qb], sv);
      if (valid < kQBlock) {
#pragma unroll
        for (int i = 0; i < 8; ++i) sv[i] = 8 * g + i < valid ? sv[i] : -INFINITY;
      }
      if (qb == 0 && n_kept) keep_scores(step, sv, c_exp);
      run[qb].weights(sv, c_exp, e);
      run[qb].template add<1, NP>(e, vf);
    }
  }
  for (; step < s1; step += 4) {
    const int tok0 = (step - w.blocks) * 32;
    bf16x8 kf[2][KD][NS], vf[DT][NS];
    keys_of_tokens<T, DH, NS>(k, a.k_stride, tok0, seen, lane, kf);
    const bool odd = __builtin_amdgcn_ballot_w64(values_of_tokens<DH, NS>(v, a.v_stride, tok0, seen, lane, vf)) != 0;
#pragma unroll
    for (int qb = 0; qb < NQB; ++qb) {
      float sv[8], e[8];
      step_scores<KD, NS, NS>(kf, qf[qb], sv);
      const uint32_t vis = sees8(a, qt[qb], tok0 + 8 * g, seen);
#pragma unroll
      for (int i = 0; i < 8; ++i) sv[i] = (vis >> i) & 1 ? sv[i] : -INFINITY;
      if (qb == 0 && n_kept) keep_scores(step, sv, a.c_exp);
      run[qb].weights(sv, a.c_exp, e);
      run[qb].template add<NS, NP>(e, vf);
      if (odd) add_odd_values<DT>(a, v, e, qt[qb], tok0, seen, lane, run[qb].o);
    }
  }
  // join the four waves: common reference, then sums in the order (0 + 2) + (1 + 3)
#pragma unroll
  for (int qb = 0; qb < NQB; ++qb) {
    run[qb].l = rows_sum(run[qb].l);
    if (g == 0) { s_m[wave][qb * 16 + col] = run[qb].m; s_l[wave][qb * 16 + col] = run[qb].l; }
  }
  __syncthreads();
  float l_all[NQB], m_all[NQB];
#pragma unroll
  for (int qb = 0; qb < NQB; ++qb) {
    const int qi = qb * 16 + col;
    float m = fmaxf(fmaxf(s_m[0][qi], s_m[1][qi]), fmaxf(s_m[2][qi], s_m[3][qi]));
    m_all[qb] = m;
    if (m == -INFINITY) m = 0.f;
    l_all[qb] = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float f = s_m[i][qi] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(s_m[i][qi] - m);      // (without a maximum: nothing, or NaN)
      l_all[qb] += s_l[i][qi] * f;
    }
    const float f = run[qb].m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(run[qb].m - m);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i) run[qb].o[dt][i] *= f;
  }
#pragma unroll
  for (int round = 0; round < 2; ++round) {
    const bool gives = round == 0 ? wave >= 2 : wave == 1, takes = round == 0 ? wave < 2 : wave == 0;
    if (round) __syncthreads();
    if (gives) {
#pragma unroll
      for (int qb = 0; qb < NQB; ++qb)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) *(floatx4*)&s_o[wave & 1][qb * 16 + col][dt * 16 + 4 * g] = run[qb].o[dt];
    }
    __syncthreads();
    if (takes) {
#pragma unroll
      for (int qb = 0; qb < NQB; ++qb)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) run[qb].o[dt] += *(const floatx4*)&s_o[round ? 1 : wave][qb * 16 + col][dt * 16 + 4 * g];
    }
  }
  if (wave == 0) {
#pragma unroll
    for (int qb = 0; qb < NQB; ++qb) {
      const int qi = q0 + qb * 16 + col;
      if (qi >= nq) continue;
      if (a.splits > 1) {
        float* part = a.parts + ((((size_t)r * gridDim.x + blockIdx.x) * a.splits + split) * NQ + qb * 16 + col) * (DH + 2);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int i = 0; i < 4; i += 2) *(float2*)(part + dt * 16 + 4 * g + i) = make_float2(run[qb].o[dt][i], run[qb].o[dt][i + 1]);
        if (g == 0) *(float2*)(part + DH) = make_float2(m_all[qb], l_all[qb]);
        continue;
      }
      const size_t at = query_at(a, r, hk, qi);
      const float inv = l_all[qb] == 0.f ? 0.f : 1.f / l_all[qb];
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        float x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = run[qb].o[dt][i] * inv;
        store4<T, DH>(a, at, dt * 16 + 4 * g, x);
      }
      if (g == 0) {
        tell_norm(a, at, m_all[qb], l_all[qb]);
        if (qb == 0) s_norm[col] = make_float2(m_all[qb] == -INFINITY ? 0.f : m_all[qb], inv);
      }
    }
  }
  if (a.splits > 1 || !a.n_kept || q0) return;
  // the only split: the counted weights are added up here
  __syncthreads();
  mass_of_kept(a, w, r, hk, s_norm, n_kept, seen, threadIdx.x, 256);
}

// Many queries: a workgroup takes 128 of them, 32 per wave, and all its waves go through the same keys, so that what is done once per key - load, conversion, turning - is
// shared: the waves bring the operands of 64 keys to LDS while those before are at work, from registers that were loaded another 64 keys earlier.  bf16 calls; grid as above.
// 8 rows x 32 query heads on 8 x 512 tokens over 4096 slots, head size 128: 494 us, 591 TFLOP/s (444 with weights of a single product; with those, 16 queries per wave took half as
// long again, every operand read from LDS for half as many); 4 rows over 2048 slots 151 us.  Matrix cores are busy 29 % of the busy CUs' time; of a wave's time vector instructions take
// 33 %, waits for memory, LDS and barriers 32 %, waits to issue 24 %: bound by the chain product - exponential - split - product of two waves per SIMD.
template <int DH>
__global__ __launch_bounds__(256, 2) void k_qcache_attention_many(QAttention a, int q_tiles) {
  constexpr int KD = DH / 32, DT = DH / 16, NQB = 2, NQ = 64 * NQB;
  __shared__ uint4 s_k[2][2][2 * KD][64], s_v[2][2][DT][64];      // [buffer][block of 32 keys]
  __shared__ int s_odd[2][2];                 // block tokens: whether any values are not finite
  __shared__ float2 s_norm[16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, col = lane & 15;
  const int hk = blockIdx.x / q_tiles, q0 = (blockIdx.x % q_tiles) * NQ, r = blockIdx.z, split = blockIdx.y;
  const QRow w = row_of(a, r);
  const int nq = w.n * a.group;
  if (q0 >= nq) return;
  const bf16_t* k = (const bf16_t*)a.k + (size_t)r * a.T * a.k_stride + (size_t)hk * DH;
  const bf16_t* v = (const bf16_t*)a.v + (size_t)r * a.T * a.v_stride + (size_t)hk * DH;
  const size_t region = a.c.region(a.layer, r, hk) * a.c.blocks;
  const int qw = q0 + wave * 16 * NQB;        // this wave's first query
  bf16x8 qf[NQB][KD][1];
  int qt[NQB];
#pragma unroll
  for (int qb = 0; qb < NQB; ++qb) {
    const int qi = min(qw + qb * 16 + col, nq - 1);
    qt[qb] = qi / a.group;
    const bf16_t* q = (const bf16_t*)a.q + ((size_t)r * a.T + qt[qb]) * a.q_stride + ((size_t)hk * a.group + qi % a.group) * DH + g * 8;
#pragma unroll
    for (int kd = 0; kd < KD; ++kd) load_operand<1>(q + kd * 32, qf[qb][kd]);
  }
  const int t_first = min(qw, nq - 1) / a.group, t_last = min(qw + 16 * NQB - 1, nq - 1) / a.group;      // tokens of the wave's queries
  QRun<DT> run[NQB];
#pragma unroll
  for (int qb = 0; qb < NQB; ++qb) run[qb].clear();
  const int n_kept = a.n_kept && qw == 0 ? min(a.n_kept, nq) : 0;
  auto keep_scores = [&](int step, const float (&sv)[8], float c) {
    if (col < n_kept) {
      float* p = kept_scores(a, r, hk, step) + col * kQBlock + 8 * g;
      ((float4*)p)[0] = make_float4(sv[0] * c, sv[1] * c, sv[2] * c, sv[3] * c);
      ((float4*)p)[1] = make_float4(sv[4] * c, sv[5] * c, sv[6] * c, sv[7] * c);
    }
  };
  const int seen = seen_by(a, w, min(q0 + NQ, nq));
  const int steps = w.blocks + (seen + 31) / 32;
  const int s0 = (int)((int64_t)steps * split / a.splits), s1 = (int)((int64_t)steps * (split + 1) / a.splits);
  const int cached_end = min(s1, w.blocks);
  const uint8_t* data = a.c.data + region * a.c.block_bytes();
  const float2* scales = a.c.scale + region;
  auto tail = [&](int step, float (&sv)[8]) {   // slots behind the length
    const int mine = w.len - step * kQBlock - 8 * g;
    const uint32_t vis = mine >= 8 ? 255u : mine <= 0 ? 0u : (1u << mine) - 1;
#pragma unroll
    for (int i = 0; i < 8; ++i) sv[i] = (vis >> i) & 1 ? sv[i] : -INFINITY;
  };

  // ---- cached blocks, two at a time: a wave brings KD of the 4 KD pieces of 1 KiB, the keys or the values of one block
  if (s0 < cached_end) {
    uint4 raw[KD];
    float unit_of = 0.f;                       // power of two of the values on their way
    const int b = wave >> 1;
    auto load_raw = [&](int step) {
      const int at = min(step + b, cached_end - 1);
      unit_of = scales[at].y;
#pragma unroll
      for (int n = 0; n < KD; ++n) raw[n] = *(const uint4*)(data + (size_t)at * a.c.block_bytes() + (((wave & 1) * KD + n) * 64 + lane) * 16);
    };
    auto bring = [&](int step, int buf) {
      const float unit = fmaxf(unit_of, kQSmall);
#pragma unroll
      for (int n = 0; n < KD; ++n) {
        uint2 lo = make_uint2(raw[n].x, raw[n].y), hi = make_uint2(raw[n].z, raw[n].w);
        if (!(wave & 1)) {
          s_k[buf][b][n][lane] = __builtin_bit_cast(uint4, e4m3_to_bf16(lo, 1.f));
          s_k[buf][b][KD + n][lane] = __builtin_bit_cast(uint4, e4m3_to_bf16(hi, 1.f));
        } else {
          if (step + b >= cached_end || w.len - (step + b) * kQBlock < kQBlock) {                 // (a second block that is not there: zeros)
            const int mine = step + b < cached_end ? w.len - (step + b) * kQBlock - 8 * g : 0;
            const uint64_t keep = mine >= 8 ? ~0ull : mine <= 0 ? 0ull : (1ull << (8 * mine)) - 1;
            lo.x &= (uint32_t)keep; lo.y &= (uint32_t)(keep >> 32); hi.x &= (uint32_t)keep; hi.y &= (uint32_t)(keep >> 32);
          }
          s_v[buf][b][2 * n][lane] = __builtin_bit_cast(uint4, e4m3_to_bf16(lo, unit));
          s_v[buf][b][2 * n + 1][lane] = __builtin_bit_cast(uint4, e4m3_to_bf16(hi, unit));
        }
      }
    };
    load_raw(s0);
    bring(s0, 0);
    if (s0 + 2 < cached_end) load_raw(s0 + 2);
    __syncthreads();
    for (int step0 = s0, buf = 0; step0 < cached_end; step0 += 2, buf ^= 1) {
      // both blocks at once: twice the independent work between the waits for the matrix cores and for the maxima.  One that is not there gets weights of 0
      float c_exp[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) c_exp[b] = fmaxf(a.c_exp * fmaxf(scales[min(step0 + b, cached_end - 1)].x, kQSmall), FLT_MIN);
      float sv[2][NQB][8];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        bf16x8 kf[2][KD][1];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int kd = 0; kd < KD; ++kd) kf[t][kd][0] = as_bf16x8(s_k[buf][b][t * KD + kd][lane]);
#pragma unroll
        for (int qb = 0; qb < NQB; ++qb) {
          step_scores<KD, 1, 1>(kf, qf[qb], sv[b][qb]);
          // (in units of log2 from here on: what comes out of a product needs no quieting of NaN in front of a maximum, which costs as much)
#pragma unroll
          for (int i = 0; i < 8; ++i) sv[b][qb][i] *= c_exp[b];
        }
      }
      // the next 64 keys' operands, while the matrix cores work on these (in front of the products: 2 to 5 % more)
      if (step0 + 2 < cached_end) bring(step0 + 2, buf ^ 1);
      if (step0 + 4 < cached_end) load_raw(step0 + 4);
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        if (w.len - (step0 + b) * kQBlock < kQBlock) {
#pragma unroll
          for (int qb = 0; qb < NQB; ++qb) tail(step0 + b, sv[b][qb]);
        }
        if (step0 + b >= cached_end) {
#pragma unroll
          for (int qb = 0; qb < NQB; ++qb)
#pragma unroll
            for (int i = 0; i < 8; ++i) sv[b][qb][i] = -INFINITY;
        } else if (n_kept) {
          keep_scores(step0 + b, sv[b][0], 1.f);
        }
      }
#pragma unroll
      for (int qb = 0; qb < NQB; ++qb) run[qb].follow(fmaxf(QRun<DT>::top(sv[0][qb]), QRun<DT>::top(sv[1][qb])));
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        bf16x8 vf[DT][1];
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) vf[dt][0] = as_bf16x8(s_v[buf][b][dt][lane]);
#pragma unroll
        for (int qb = 0; qb < NQB; ++qb) {
          float e[8];
          run[qb].exponentials(sv[b][qb], 1.f, e);
          run[qb].template add<1, 2>(e, vf);
        }
      }
      __syncthreads();
    }
  }

  // ---- block tokens, 32 at a time: waves 0 and 1 bring the keys of both tiles, waves 2 and 3 half of the values each
  {
    const int f0 = max(s0, w.blocks);
    uint4 raw[KD];
    auto load_raw = [&](int step) {
      const int tok0 = (step - w.blocks) * 32, tok = min(tok0 + (wave < 2 ? slot_of(wave, col) : value_slot(lane)), seen - 1);
      const bf16_t* p = (wave < 2 ? k : v) + (size_t)tok * (wave < 2 ? a.k_stride : a.v_stride) + (wave < 2 ? g * 8 : (wave - 2) * (DH / 2) + (lane & 8));
      const int next = wave < 2 ? 32 : 16;
#pragma unroll
      for (int n = 0; n < KD; ++n) raw[n] = *(const uint4*)(p + n * next);
    };
    auto bring = [&](int step, int buf) {
      if (wave < 2) {
#pragma unroll
        for (int kd = 0; kd < KD; ++kd) s_k[buf][0][wave * KD + kd][lane] = raw[kd];
      } else {
        uint32_t odd = 0;
        const uint32_t there = (step - w.blocks) * 32 + value_slot(lane) < seen ? 0xFFFFFFFFu : 0u;
#pragma unroll
        for (int n = 0; n < KD; ++n) s_v[buf][0][(wave - 2) * KD + n][lane] = turned_values(raw[n], there, lane, odd);
        const bool any = __builtin_amdgcn_ballot_w64(odd != 0) != 0;
        if (lane == 0) s_odd[buf][wave - 2] = any;
      }
    };
    if (f0 < s1) {
      load_raw(f0);
      bring(f0, 0);
      if (f0 + 1 < s1) load_raw(f0 + 1);
    }
    __syncthreads();
    for (int step = f0, buf = 0; step < s1; ++step, buf ^= 1) {
      if (step + 1 < s1) bring(step + 1, buf ^ 1);
      if (step + 2 < s1) load_raw(step + 2);
      const int tok0 = (step - w.blocks) * 32;
      if (!a.causal || tok0 <= t_last) {
        float sv[NQB][8];
        {
          bf16x8 kf[2][KD][1];
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int kd = 0; kd < KD; ++kd) kf[t][kd][0] = as_bf16x8(s_k[buf][0][t * KD + kd][lane]);
#pragma unroll
          for (int qb = 0; qb < NQB; ++qb) step_scores<KD, 1, 1>(kf, qf[qb], sv[qb]);
        }
        if (!a.causal || tok0 + 31 > t_first || tok0 + 31 >= seen) {
#pragma unroll
          for (int qb = 0; qb < NQB; ++qb) {
            const uint32_t vis = sees8(a, qt[qb], tok0 + 8 * g, seen);
#pragma unroll
            for (int i = 0; i < 8; ++i) sv[qb][i] = (vis >> i) & 1 ? sv[qb][i] : -INFINITY;
          }
        }
        if (n_kept) keep_scores(step, sv[0], a.c_exp);
        bf16x8 vf[DT][1];
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) vf[dt][0] = as_bf16x8(s_v[buf][0][dt][lane]);
        const bool odd = s_odd[buf][0] | s_odd[buf][1];
#pragma unroll
        for (int qb = 0; qb < NQB; ++qb) {
          float e[8];
          run[qb].weights(sv[qb], a.c_exp, e);
          run[qb].template add<1, 2>(e, vf);
          if (odd) add_odd_values<DT>(a, v, e, qt[qb], tok0, seen, lane, run[qb].o);
        }
      }
      __syncthreads();
    }
  }

#pragma unroll
  for (int qb = 0; qb < NQB; ++qb) {
    const int qi = qw + qb * 16 + col;
    const float l = rows_sum(run[qb].l), m = run[qb].m;
    if (qi < nq) {
      if (a.splits > 1) {
        float* part = a.parts + ((((size_t)r * gridDim.x + blockIdx.x) * a.splits + split) * NQ + (qi - q0)) * (DH + 2);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int i = 0; i < 4; i += 2) *(float2*)(part + dt * 16 + 4 * g + i) = make_float2(run[qb].o[dt][i], run[qb].o[dt][i + 1]);
        if (g == 0) *(float2*)(part + DH) = make_float2(m, l);
      } else {
        const size_t at = query_at(a, r, hk, qi);
        const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          float x[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] = run[qb].o[dt][i] * inv;
          store4<bf16_t, DH>(a, at, dt * 16 + 4 * g, x);
        }
        if (g == 0) {
          tell_norm(a, at, m, l);
          if (qw == 0 && qb == 0) s_norm[col] = make_float2(m == -INFINITY ? 0.f : m, inv);
        }
      }
    }
  }
  if (a.splits > 1 || !a.n_kept || q0) return;
  __syncthreads();
  mass_of_kept(a, w, r, hk, s_norm, min(a.n_kept, nq), seen_by(a, w, min(16 * NQB, nq)), threadIdx.x, 256);
}

// Joins the splits.  Few of them (up to kQFewSplits): one group of DH / 4 lanes per query goes through them; many (WIDE): a workgroup per query, whose groups take every so-manieth split.
// Workgroups of blockIdx.y >= joins add up the counted weights instead (kept_tile: queries that went through the keys with the counted ones).  us per call of attention, by groups /
// by workgroups: one row of 32768 slots, 8 key/value heads in 64 splits 46 / 21, of 131072 slots and one head 124 / 20; 16 rows of 4000 in 8 splits 36.1 / 37.0.
constexpr int kQFewSplits = 8;

template <typename T, int DH, bool WIDE>
__global__ __launch_bounds__(256) void k_qcache_join(QAttention a, int q_tiles, int nq_tile, int joins, int kept_tile) {
  constexpr int LQ = DH / 4, GROUPS = 256 / LQ;
  __shared__ float2 s_norm[kQKept];
  __shared__ float s_red[16];
  __shared__ float s_x[WIDE ? GROUPS : 1][DH];
  const int r = blockIdx.z, tid = threadIdx.x;
  const QRow w = row_of(a, r);
  const size_t step = (size_t)nq_tile * (DH + 2);
  const float* tile_parts = a.parts + ((size_t)r * gridDim.x + blockIdx.x) * a.splits * step;
  auto scaled = [](float ms, float m) { return ms == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ms - m); };      // (without a maximum: nothing, or NaN)
  if ((int)blockIdx.y >= joins) {
    const int hk = blockIdx.x / q_tiles;
    if (blockIdx.x % q_tiles) return;
    const int n_kept = min(a.n_kept, w.n * a.group), q = tid >> 5;      // 32 threads per kept query
    if (q < n_kept) {
      const float* part = tile_parts + (size_t)q * (DH + 2) + DH;
      float m = -INFINITY, l = 0.f;
      for (int s = tid & 31; s < a.splits; s += 32) m = fmaxf(m, part[s * step]);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 32));
      for (int s = tid & 31; s < a.splits; s += 32) l += part[s * step + 1] * scaled(part[s * step], m);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) l += __shfl_xor(l, o, 32);
      if ((tid & 31) == 0) s_norm[q] = make_float2(m == -INFINITY ? 0.f : m, l == 0.f ? 0.f : 1.f / l);
    }
    __syncthreads();
    mass_of_kept(a, w, r, hk, s_norm, n_kept, seen_by(a, w, min(kept_tile, w.n * a.group)), (blockIdx.y - joins) * 256 + tid, (gridDim.y - joins) * 256);
    return;
  }
  const int hk = blockIdx.x / q_tiles, tile = blockIdx.x % q_tiles, group = tid / LQ, dim = tid % LQ * 4;
  const int in_tile = WIDE ? blockIdx.y : blockIdx.y * GROUPS + group, qi = tile * nq_tile + in_tile;
  if (in_tile >= nq_tile || qi >= w.n * a.group) return;
  const float* part = tile_parts + (size_t)in_tile * (DH + 2);
  float m = -INFINITY, l = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
  for (int s = WIDE ? tid : 0; s < a.splits; s += WIDE ? 256 : 1) m = fmaxf(m, part[s * step + DH]);
  if (WIDE) m = block_max(m, s_red);
  for (int s = WIDE ? tid : 0; s < a.splits; s += WIDE ? 256 : 1) l += part[s * step + DH + 1] * scaled(part[s * step + DH], m);
  if (WIDE) l = block_sum(l, s_red);
#pragma unroll 4
  for (int s = WIDE ? group : 0; s < a.splits; s += WIDE ? GROUPS : 1) {
    const float f = scaled(part[s * step + DH], m);
    const float2 p0 = *(const float2*)(part + s * step + dim), p1 = *(const float2*)(part + s * step + dim + 2);
    x[0] += p0.x * f;
    x[1] += p0.y * f;
    x[2] += p1.x * f;
    x[3] += p1.y * f;
  }
  if (WIDE) {
#pragma unroll
    for (int i = 0; i < 4; ++i) s_x[group][dim + i] = x[i];
    __syncthreads();
    if (group) return;
    for (int g = 1; g < GROUPS; ++g)
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] += s_x[g][dim + i];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = l == 0.f ? 0.f : x[i] / l;
  const size_t at = query_at(a, r, hk, qi);
  store4<T, DH>(a, at, dim, x);
  if (dim == 0) tell_norm(a, at, m, l);
}

// Counted weights of many queries: the scores are made again, now with the normaliser known.  A wave holds the keys of a step of 32 in registers, the queries pass by, 64 at a
// time, through LDS, shared by the four waves; their order is fixed.  Nothing in the loop may wait for the queries that were requested last: with the norms looked at as soon as they were
// requested, and keys on their way when the loop began, 4 rows of 512, 384, 256 and 128 tokens over 2048 slots each, 8 x 4 heads of 128, took 78 us, now 60.  Products and exponentials would be
// some 18 us each: bound by the chain LDS - product - exponential of few waves, the longest row's workgroups last.
template <typename T, int DH>
__global__ __launch_bounds__(256, sizeof(T) == 4 && DH == 128 ? 1 : 2) void k_qcache_mass(QAttention a) {
  using S = QShape<T, DH>;
  constexpr int KD = S::KD, NS = S::NS;
  __shared__ uint4 s_q[2][4][KD * NS][64];
  __shared__ float s_norm[2][4][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, col = lane & 15;
  const int hk = blockIdx.y, r = blockIdx.z;
  const QRow w = row_of(a, r);
  const int seen = a.k ? w.n : 0, steps = w.blocks + (a.block_mass ? (w.n + 31) / 32 : 0), nq = min(a.n_counted, w.n) * a.group;
  const int first = a.mass ? 0 : w.blocks;
  const T* q = (const T*)a.q + (size_t)r * a.T * a.q_stride + (size_t)hk * a.group * DH;
  const T* k = (const T*)a.k + (size_t)r * a.T * a.k_stride + (size_t)hk * DH;
  const size_t region = a.c.region(a.layer, r, hk) * a.c.blocks;
  for (int step0 = first + blockIdx.x * 4; step0 < steps; step0 += gridDim.x * 4) {
    bf16x8 kf[2][KD][NS];
    float sum[8], c_exp = a.c_exp;
    const int step = min(step0 + wave, steps - 1);
    const bool there = step0 + wave < steps, cached = step < w.blocks;
    const int tok0 = cached ? -1 : (step - w.blocks) * 32;                                         // first block token
    const int q_all = cached ? 0 : a.causal ? (tok0 + 31) * a.group : INT_MAX;                      // first query from which on all see all keys
    const int valid = !there ? 0 : cached ? min(w.len - step * kQBlock, 32) : min(seen - tok0, 32);  // keys there
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = 0.f;
    if (cached) {
      const uint8_t* data = a.c.data + (region + step) * a.c.block_bytes();
      c_exp = fmaxf(a.c_exp * a.c.scale[region + step].x, FLT_MIN);
#pragma unroll
      for (int kd = 0; kd < KD; ++kd) {
        const uint4 b = *(const uint4*)(data + (kd * 64 + lane) * 16);
        kf[0][kd][0] = e4m3_to_bf16(make_uint2(b.x, b.y), 1.f);
        kf[1][kd][0] = e4m3_to_bf16(make_uint2(b.z, b.w), 1.f);
#pragma unroll
        for (int p = 1; p < NS; ++p) kf[0][kd][p] = kf[1][kd][p] = as_bf16x8(make_uint4(0, 0, 0, 0));
      }
    } else {
      keys_of_tokens<T, DH, NS>(k, a.k_stride, tok0, seen, lane, kf);
    }
    // Keys that are still on their way here would have every pass of the loop wait for whatever was requested last
    __builtin_amdgcn_s_waitcnt(0x0F70);          // vmcnt(0)
    // (of a chain only the queries from the workgroup's first block token on see anything of block tokens)
    const int q_first = step0 >= w.blocks && a.causal ? (step0 - w.blocks) * 32 * a.group / 64 * 64 : 0;
    // a wave brings 16 of the 64 queries that pass by together: into registers while the ones before are at work, then to LDS; +inf as the norm of what is no query
    bf16x8 next[KD][NS];
    float next_norm = 0.f;
    bool next_there = false;                     // (looked at when the norm is stored: here it would wait for the load)
    auto load_queries = [&](int q0) {
      const int at = q0 + wave * 16 + col, qi = min(at, nq - 1), t = qi / a.group;
#pragma unroll
      for (int kd = 0; kd < KD; ++kd) load_operand<NS>(q + (size_t)t * a.q_stride + (size_t)(qi % a.group) * DH + kd * 32 + g * 8, next[kd]);
      next_norm = a.norm[query_at(a, r, hk, qi)];
      next_there = at < nq;
    };
    auto put_queries = [&](int buf) {
#pragma unroll
      for (int kd = 0; kd < KD; ++kd)
#pragma unroll
        for (int p = 0; p < NS; ++p) s_q[buf][wave][kd * NS + p][lane] = __builtin_bit_cast(uint4, next[kd][p]);
      if (g == 0) s_norm[buf][wave][col] = next_there ? next_norm : INFINITY;
    };
    if (q_first < nq) load_queries(q_first);
    __syncthreads();
    if (q_first < nq) put_queries(0);
    if (q_first + 64 < nq) load_queries(q_first + 64);
    __syncthreads();
    int buf = 0;
    for (int q0 = q_first; q0 < nq; q0 += 64, buf ^= 1) {
      if (q0 + 64 < nq) put_queries(buf ^ 1);
      if (q0 + 128 < nq) load_queries(q0 + 128);
#pragma unroll 2
      for (int b = 0; b < 4; ++b) {
        bf16x8 qf[KD][NS];
#pragma unroll
        for (int kd = 0; kd < KD; ++kd)
#pragma unroll
          for (int p = 0; p < NS; ++p) qf[kd][p] = as_bf16x8(s_q[buf][b][kd * NS + p][lane]);
        const float norm = s_norm[buf][b][col];
        float sv[8];
        step_scores<KD, NS, NS>(kf, qf, sv);
        if (q0 + b * 16 >= q_all) {          // all queries see all keys that there are (the others' sums are left out below)
#pragma unroll
          for (int i = 0; i < 8; ++i) sum[i] += __builtin_amdgcn_exp2f(fmaf(sv[i], c_exp, -norm));
        } else {
          const uint32_t vis = sees8(a, min(q0 + b * 16 + col, nq - 1) / a.group, tok0 + 8 * g, seen);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float p = __builtin_amdgcn_exp2f(fmaf(sv[i], c_exp, -norm));
            sum[i] += (vis >> i) & 1 ? p : 0.f;
          }
        }
      }
      __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {               // over the 16 queries of the lane's row
      float x = sum[i];
      x += dpp_move<0x128>(x);
      x += dpp_move<0x141>(x);
      x += dpp_move<0x4E>(x);
      x += dpp_move<0xB1>(x);
      sum[i] = x;
    }
    if (col < 8) {
      float x = sum[0];
#pragma unroll
      for (int i = 1; i < 8; ++i) x = col == i ? sum[i] : x;
      const int at = 8 * g + col;
      if (at < valid) {
        if (cached) a.mass[((size_t)r * a.c.kv_heads + hk) * a.capacity + (size_t)step * kQBlock + at] += x;
        else a.block_mass[((size_t)r * a.c.kv_heads + hk) * a.block_stride + tok0 + at] = x;
      }
    }
  }
}

template <typename T, int DH, int NQB, bool MANY = false>
static void attention_t(QAttention a, hipStream_t s) {
  constexpr int BLOCKS = MANY ? 4 * NQB : NQB;      // of 16 queries per workgroup
  const int q_tiles = (a.T * a.group + 16 * BLOCKS - 1) / (16 * BLOCKS);
  const int64_t tiles = (int64_t)a.c.rows * a.c.kv_heads * q_tiles;
  // As many splits as give each CU about four workgroups, but at least four steps to each of a split's waves where the cache is full; the partial results have room for kQParts
  const int64_t most = (int64_t)kQParts / (tiles * BLOCKS);
  a.splits = (int)std::max<int64_t>(1, std::min<int64_t>({1024 / tiles, most, a.c.blocks / 16}));
  // Few counted queries: their scores are kept, 4 bytes per query and slot written and read, where reading the keys again is DH bytes per slot (and many times the work)
  const int counted = a.n_counted * a.group;
  a.n_kept = counted <= std::min(kQKept, DH / 16) ? counted : 0;
  if (a.n_kept) a.norm = nullptr;
  const dim3 grid(a.c.kv_heads * q_tiles, a.splits, a.c.rows);
  if constexpr (MANY) hipLaunchKernelGGL((k_qcache_attention_many<DH>), grid, dim3(256), 0, s, a, q_tiles);
  else hipLaunchKernelGGL((k_qcache_attention<T, DH, NQB>), grid, dim3(256), 0, s, a, q_tiles);
  if (a.splits > 1) {
    const int per = a.splits > kQFewSplits ? 1 : 256 / (DH / 4), joins = (16 * BLOCKS + per - 1) / per;
    // (a workgroup first finds the norms: a few workgroups with much to add rather than many with little)
    const int masses = a.n_kept ? (int)std::max<int64_t>(1, std::min<int64_t>(a.c.blocks / 32, 2048 / ((int64_t)a.c.rows * a.c.kv_heads))) : 0;
    const dim3 join_grid(grid.x, joins + masses, grid.z);
    if (a.splits > kQFewSplits) hipLaunchKernelGGL((k_qcache_join<T, DH, true>), join_grid, dim3(256), 0, s, a, q_tiles, 16 * BLOCKS, joins, 16 * NQB);
    else hipLaunchKernelGGL((k_qcache_join<T, DH, false>), join_grid, dim3(256), 0, s, a, q_tiles, 16 * BLOCKS, joins, 16 * NQB);
  }
  if (!a.n_kept && (a.n_counted > 0 || a.block_mass)) {
    const int steps = a.c.blocks + (a.T + 31) / 32, per = 4;
    hipLaunchKernelGGL((k_qcache_mass<T, DH>), dim3(std::min((steps + per - 1) / per, 1024), a.c.kv_heads, a.c.rows), dim3(256), 0, s, a);
  }
}

template <typename T, int DH>
static void attention_d(const QAttention& a, hipStream_t s) {
  // query blocks of 16 per wave: as few as hold the queries; more would not fit the registers beside head size 128 or fp32 operands in three parts
  const int nq = a.T * a.group;
  if constexpr (sizeof(T) == 4) {
    attention_t<T, DH, 1>(a, s);
  } else {
    if (nq <= 16) attention_t<T, DH, 1>(a, s);
    else if (nq <= 32) attention_t<T, DH, 2>(a, s);
    else if (nq <= 64 && DH < 128) attention_t<T, DH < 128 ? DH : 64, 4>(a, s);
    else attention_t<T, DH, 2, true>(a, s);
  }
}

void launch_qcache_attention(const QAttention& a, int dtype, hipStream_t s) {
  if (dtype == VVS_BF16) {
    if (a.c.dh == 32) attention_d<bf16_t, 32>(a, s);
    else if (a.c.dh == 64) attention_d<bf16_t, 64>(a, s);
    else attention_d<bf16_t, 128>(a, s);
  } else {
    if (a.c.dh == 32) attention_d<float, 32>(a, s);
    else if (a.c.dh == 64) attention_d<float, 64>(a, s);
    else attention_d<float, 128>(a, s);
  }
}

// ------------------------------------------------------------------------------------------------ eviction
// Which slots stay: per (layer, row, head) the keep-th largest weight is found by its bits, then the kept slots behind `keep` are dealt to the holes in front of it, in order.
// Order-preserving bits: a weight's sign bit is flipped, or all its bits when it is set; -0 counts as 0, NaN as the largest number, the newest tokens lie above all.
constexpr int kQSelect = 1024;

__device__ __forceinline__ uint32_t mass_bits(float m) {
  const uint32_t u = __float_as_uint(m == 0.f ? 0.f : m);
  if (m != m) return 0xFFFFFFFEu;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

struct QSelect {           // one (layer, row, head)
  int len, left;
  const float* mass;
  float* mass_out;
  const int32_t* pos;
  int32_t *pos_out, *origin;
};
__device__ __forceinline__ QSelect select_of(const QEvict& a, int head, int r, int layer) {
  const size_t region = a.c.region(layer, r, head), base = region * a.capacity;
  const int len = row_len(a.len, r, a.capacity);
  return QSelect{len, min(len, a.keep), a.mass + base, a.mass_out + base, a.pos ? a.pos + base : nullptr, a.pos ? a.pos_out + base : nullptr, a.origin + region * a.c.blocks * kQBlock};
}
// Weights and positions of the slots in front of `left`, from where `origin` says (a slot itself, or one behind all of them, so that the outputs may be the inputs).  Eight at a
// time: outputs that may be inputs keep the loads of a next slot behind the stores of this one (one at a time, 16 x 8 rows of 32768 took 87 us, now 73)
__device__ __forceinline__ void settle(const QSelect& h, int left, int tid, int threads) {
  for (int i0 = tid; i0 < left; i0 += 8 * threads) {
    int from[8], p[8];
    float m[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) from[j] = h.origin[min(i0 + j * threads, left - 1)];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      m[j] = h.mass[from[j]];
      p[j] = h.pos ? h.pos[from[j]] : 0;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int i = i0 + j * threads;
      if (i < left) {
        h.mass_out[i] = m[j];
        if (h.pos) h.pos_out[i] = p[j];
      }
    }
  }
}
// A row that is not shortened
__device__ __forceinline__ void stay(const QSelect& h, int tid, int threads) {
  if (h.mass == h.mass_out && (!h.pos || h.pos == h.pos_out)) return;
  for (int i = tid; i < h.left; i += threads) {
    h.mass_out[i] = h.mass[i];
    if (h.pos) h.pos_out[i] = h.pos[i];
  }
}
__device__ __forceinline__ void clear_behind(const QSelect& h, int capacity, int tid, int threads) {
  for (int i = h.left + tid; i < capacity; i += threads) {
    h.mass_out[i] = 0.f;
    if (h.pos) h.pos_out[i] = 0;
  }
}

// Rows of up to 64 * WAVES * KPT slots: every lane holds the keys of KPT slots (a wave's slots lie together), 32 rounds of counting find the threshold.
// A workgroup of one wave needs no barrier.  Bound by the rounds (KPT comparisons each), not by the 8 bytes per slot: 36 x 16 x 20 rows of 696 slots take 59 us,
// 16 x 8 rows of 32768 73.  (Digits of 8 bits counted in LDS: 1521 and 208 us - most weights share a few exponents, so that the counters collide.)
template <int WAVES, int KPT>
__global__ __launch_bounds__(64 * WAVES) void k_qcache_select(QEvict a) {
  constexpr int THREADS = 64 * WAVES;
  __shared__ uint16_t s_list[THREADS * KPT / 2];
  __shared__ int s_count[2][WAVES], s_equal[WAVES], s_hole[WAVES], s_source[WAVES];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const QSelect h = select_of(a, blockIdx.x, blockIdx.y, blockIdx.z);
  if (h.len <= a.keep) {
    stay(h, tid, THREADS);
    clear_behind(h, a.capacity, tid, THREADS);
    return;
  }
  const int slot0 = wave * 64 * KPT + lane;
  uint32_t key[KPT];
  int newest = h.pos ? INT_MIN : h.len - 1;
  if (h.pos) {
#pragma unroll
    for (int j = 0; j < KPT; ++j) {
      const int i = slot0 + j * 64;
      key[j] = i < h.len ? (uint32_t)h.pos[i] : 0x80000000u;
      newest = max(newest, (int)key[j]);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) newest = max(newest, __shfl_xor(newest, o, 64));
    if (WAVES > 1) {
      if (lane == 0) s_equal[wave] = newest;
      __syncthreads();
      for (int w = 0; w < WAVES; ++w) newest = max(newest, s_equal[w]);
      __syncthreads();
    }
  }
  const int64_t above = (int64_t)newest - a.recent;
#pragma unroll
  for (int j = 0; j < KPT; ++j) {
    const int i = slot0 + j * 64;
    const bool recent = (h.pos ? (int)key[j] : i) > above;
    key[j] = i >= h.len ? 0u : recent ? 0xFFFFFFFFu : mass_bits(h.mass[i]);       // (a slot that is filled has a key above 0: no float is all ones but a NaN)
  }
  // largest bound that `keep` keys reach
  uint32_t bound = 0;
  for (int b = 31; b >= 0; --b) {
    const uint32_t cand = bound | 1u << b;
    int n = 0;
#pragma unroll
    for (int j = 0; j < KPT; ++j) n += __popcll(__builtin_amdgcn_ballot_w64(key[j] >= cand));
    if (WAVES > 1) {
      if (lane == 0) s_count[b & 1][wave] = n;
      __syncthreads();
      n = 0;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) n += s_count[b & 1][w];
    }
    if (n >= a.keep) bound = cand;
    if (n == a.keep) break;
  }
  // kept: keys above the bound, and as many equal ones, from the lowest slot on, as there is room for
  int n_above = 0, n_equal = 0;
#pragma unroll
  for (int j = 0; j < KPT; ++j) {
    n_above += __popcll(__builtin_amdgcn_ballot_w64(key[j] > bound));
    n_equal += __popcll(__builtin_amdgcn_ballot_w64(key[j] == bound && slot0 + j * 64 < h.len));
  }
  int equal_before = 0;
  if (WAVES > 1) {
    if (lane == 0) { s_equal[wave] = n_equal; s_hole[wave] = n_above; }
    __syncthreads();
    n_above = 0;
    for (int w = 0; w < WAVES; ++w) { n_above += s_hole[w]; equal_before += w < wave ? s_equal[w] : 0; }
    __syncthreads();
  }
  const int room = a.keep - n_above;
  const uint64_t below = (1ull << lane) - 1;
  uint32_t kept = 0;
  int n_hole = 0, n_source = 0;
#pragma unroll
  for (int j = 0; j < KPT; ++j) {
    const int i = slot0 + j * 64;
    const bool equal = key[j] == bound && i < h.len;
    const uint64_t eq = __builtin_amdgcn_ballot_w64(equal);
    const bool k = key[j] > bound || (equal && equal_before + __popcll(eq & below) < room);
    equal_before += __popcll(eq);
    kept |= (uint32_t)k << j;
    n_hole += __popcll(__builtin_amdgcn_ballot_w64(!k && i < a.keep));
    n_source += __popcll(__builtin_amdgcn_ballot_w64(k && i >= a.keep));
  }
  int hole = 0, source = 0;
  if (WAVES > 1) {
    if (lane == 0) { s_hole[wave] = n_hole; s_source[wave] = n_source; }
    __syncthreads();
    for (int w = 0; w < wave; ++w) { hole += s_hole[w]; source += s_source[w]; }
  }
#pragma unroll
  for (int j = 0; j < KPT; ++j) {                // the sources, in order
    const int i = slot0 + j * 64;
    const bool s = (kept >> j & 1) && i >= a.keep;
    const uint64_t b = __builtin_amdgcn_ballot_w64(s);
    if (s) s_list[source + __popcll(b & below)] = (uint16_t)i;
    source += __popcll(b);
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < KPT; ++j) {                // the n-th hole takes the n-th source
    const int i = slot0 + j * 64;
    const bool o = !(kept >> j & 1) && i < a.keep;
    const uint64_t b = __builtin_amdgcn_ballot_w64(o);
    if (i < a.keep) h.origin[i] = o ? s_list[hole + __popcll(b & below)] : i;
    hole += __popcll(b);
  }
  __syncthreads();
  settle(h, a.keep, tid, THREADS);
  __syncthreads();                               // the sources' weights have been read
  clear_behind(h, a.capacity, tid, THREADS);
}

// Longer rows: the keys are read again for each digit of 8 bits, counted in LDS, and for the dealing.
// exclusive prefix over the workgroup; *total: the sum.  red: kQSelect / 64 ints
__device__ __forceinline__ int block_rank(bool mine, int* red, int* total) {
  const uint64_t b = __builtin_amdgcn_ballot_w64(mine);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  __syncthreads();
  if (lane == 0) red[wave] = __popcll(b);
  __syncthreads();
  int before = 0, all = 0;
  for (int i = 0; i < kQSelect / 64; ++i) {
    const int n = red[i];
    if (i < wave) before += n;
    all += n;
  }
  *total = all;
  return before + __popcll(b & ((1ull << lane) - 1));
}

__global__ __launch_bounds__(kQSelect) void k_qcache_select_long(QEvict a) {
  __shared__ int s_hist[256], s_red[kQSelect / 64], s_pick[2];
  const int tid = threadIdx.x;
  const QSelect h = select_of(a, blockIdx.x, blockIdx.y, blockIdx.z);
  if (h.len <= a.keep) {
    stay(h, tid, kQSelect);
    clear_behind(h, a.capacity, tid, kQSelect);
    return;
  }
  int newest = h.len - 1;
  if (h.pos) {
    newest = INT_MIN;
    for (int i = tid; i < h.len; i += kQSelect) newest = max(newest, h.pos[i]);
    newest = block_max_int(newest, s_red);
  }
  auto key = [&](int i) {
    const int64_t p = h.pos ? h.pos[i] : i;
    return p > (int64_t)newest - a.recent ? 0xFFFFFFFFu : mass_bits(h.mass[i]);
  };
  uint32_t prefix = 0;
  int room = a.keep;                       // of the keys that share the prefix, how many are kept
  for (int shift = 24; shift >= 0; shift -= 8) {
    __syncthreads();
    if (tid < 256) s_hist[tid] = 0;
    __syncthreads();
    for (int i = tid; i < h.len; i += kQSelect) {
      const uint32_t k = key(i);
      if (shift == 24 || k >> (shift + 8) == prefix) atomicAdd(&s_hist[(k >> shift) & 255], 1);   // whole numbers: in any order the same
    }
    __syncthreads();
    if (tid == 0) {
      int b = 255, above = 0;
      while (above + s_hist[b] < room) above += s_hist[b--];
      s_pick[0] = b;
      s_pick[1] = room - above;
    }
    __syncthreads();
    prefix = prefix << 8 | (uint32_t)s_pick[0];
    room = s_pick[1];
  }
  int equal = 0, holes = 0, sources = 0;
  for (int i0 = 0; i0 < h.len; i0 += kQSelect) {
    const int i = i0 + tid;
    const uint32_t k = i < h.len ? key(i) : 0;
    int total;
    const bool eq = i < h.len && k == prefix;
    const int rank = equal + block_rank(eq, s_red, &total);
    equal += total;
    const bool kept = i < h.len && (k > prefix || (eq && rank < room));
    const bool hole = i < a.keep && !kept, source = i >= a.keep && kept;
    const int o = holes + block_rank(hole, s_red, &total);
    holes += total;
    const int q = sources + block_rank(source, s_red, &total);
    sources += total;
    // a hole notes its number; the sources, as many as there are holes, are listed behind `keep`
    if (i < a.keep) h.origin[i] = kept ? i : -1 - o;
    if (source) h.origin[a.keep + q] = i;
  }
  __syncthreads();
  for (int i = tid; i < a.keep; i += kQSelect) {
    const int o = h.origin[i];
    h.origin[i] = o >= 0 ? i : h.origin[a.keep + (-1 - o)];
  }
  __syncthreads();
  settle(h, a.keep, tid, kQSelect);
  __syncthreads();
  clear_behind(h, a.capacity, tid, kQSelect);
}

// Moves the elements: one wave per (layer, row, head, block below keep).  Of the keys a lane gathers 8 dims of its two slots, 8 bytes in a row.  Of the values it gathers its dims of 8 slots: the
// 16 lanes of a group read the 256 bytes in which a source's dims lie beside those of the 7 slots around it, and each picks its byte.  (Single bytes by the lane that holds the slot: every
// lane touches a segment of its own, 370 us instead of 276 for 36 x 16 x 20 rows of 696 slots cut to 256.)  Bound by HBM: a slot's values share their cache lines with 7 others, so that
// nearly all of them are read: about 1 GB with keys and stores, by arithmetic.
template <int DH>
__global__ __launch_bounds__(256) void k_qcache_move(QEvict a) {
  const int lane = threadIdx.x & 63, unit = blockIdx.x * 4 + (threadIdx.x >> 6), r = blockIdx.y, layer = blockIdx.z;
  const int blocks = a.keep / kQBlock, head = unit / blocks, block = unit % blocks;
  if (head >= a.c.kv_heads) return;
  if (row_len(a.len, r, a.capacity) <= a.keep) return;
  const size_t region = a.c.region(a.layer + layer, r, head) * a.c.blocks;
  const int g = lane >> 4, i = lane & 15, slot0 = block * kQBlock;
  const int32_t* origin = a.origin + a.c.region(layer, r, head) * a.c.blocks * kQBlock + slot0;
  const int from_k[2] = {origin[slot_of(0, i)], origin[slot_of(1, i)]};        // this lane's slots: keys of both tiles
  const int4 o0 = *(const int4*)(origin + 8 * g), o1 = *(const int4*)(origin + 8 * g + 4);
  const int from_v[8] = {o0.x, o0.y, o0.z, o0.w, o1.x, o1.y, o1.z, o1.w};      // ... and values
  if (!__builtin_amdgcn_ballot_w64(from_k[0] != slot0 + slot_of(0, i) || from_k[1] != slot0 + slot_of(1, i))) return;
  float unit_k[2], unit_v[8], tk = 0.f, tv = 0.f;
#pragma unroll
  for (int t = 0; t < 2; ++t) { unit_k[t] = fmaxf(a.c.scale[region + (from_k[t] >> 5)].x, kQSmall); tk = fmaxf(tk, unit_k[t]); }
#pragma unroll
  for (int j = 0; j < 8; ++j) { unit_v[j] = fmaxf(a.c.scale[region + (from_v[j] >> 5)].y, kQSmall); tv = fmaxf(tv, unit_v[j]); }
  tk = wave_max(tk);
  tv = wave_max(tv);
  bool other_v = false;
#pragma unroll
  for (int j = 0; j < 8; ++j) other_v |= unit_v[j] != tv;
  const bool again_k = __builtin_amdgcn_ballot_w64(unit_k[0] != tk || unit_k[1] != tk) != 0, again_v = __builtin_amdgcn_ballot_w64(other_v) != 0;
  uint8_t* data = a.c.data + region * a.c.block_bytes();
  uint8_t* out = data + (size_t)block * a.c.block_bytes();
#pragma unroll
  for (int c = 0; c < DH / 32; ++c) {
    uint2 k[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) k[t] = *(const uint2*)(data + (size_t)(from_k[t] >> 5) * a.c.block_bytes() + key_byte(from_k[t] & 31, c * 32 + 8 * g));
    u32x4 b[8];
#pragma unroll
    for (int j = 0; j < 8; ++j)
      b[j] = *(const u32x4*)(data + (size_t)(from_v[j] >> 5) * a.c.block_bytes() + kQBlock * DH + (c * 64 + (from_v[j] >> 3 & 3) * 16 + i) * 16);
    uint32_t v0[2] = {0, 0}, v1[2] = {0, 0};      // slots 0 .. 3 and 4 .. 7 of both dims
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int at = from_v[j] & 7;
      const u32x4 x = b[j];
      const uint32_t w0 = at & 4 ? x[1] : x[0], w1 = at & 4 ? x[3] : x[2];
      const uint32_t x0 = (w0 >> (at & 3) * 8) & 255u, x1 = (w1 >> (at & 3) * 8) & 255u;
      v0[j >> 2] |= x0 << (j & 3) * 8;
      v1[j >> 2] |= x1 << (j & 3) * 8;
    }
    uint2 v[2] = {make_uint2(v0[0], v0[1]), make_uint2(v1[0], v1[1])};
    if (again_k) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        float x[8];
        from_e4m3x8(k[t], x);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] *= unit_k[t] / tk;
        k[t] = to_e4m3x8(x);
      }
    }
    if (again_v) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        float x[8];
        from_e4m3x8(v[t], x);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] *= unit_v[j] / tv;
        v[t] = to_e4m3x8(x);
      }
    }
    *(uint4*)(out + (c * 64 + lane) * 16) = make_uint4(k[0].x, k[0].y, k[1].x, k[1].y);
    *(uint4*)(out + kQBlock * DH + (c * 64 + lane) * 16) = make_uint4(v[0].x, v[0].y, v[1].x, v[1].y);
  }
  if (lane == 0) a.c.scale[region + block] = make_float2(tk, tv);
}

void launch_qcache_evict(const QEvict& a, hipStream_t s) {
  const dim3 heads(a.c.kv_heads, a.c.rows, a.n_layers);
  if (a.capacity <= 1024) hipLaunchKernelGGL((k_qcache_select<1, 16>), heads, dim3(64), 0, s, a);
  else if (a.capacity <= 8192) hipLaunchKernelGGL((k_qcache_select<4, 32>), heads, dim3(256), 0, s, a);
  else if (a.capacity <= 32768) hipLaunchKernelGGL((k_qcache_select<16, 32>), heads, dim3(1024), 0, s, a);
  else hipLaunchKernelGGL(k_qcache_select_long, heads, dim3(kQSelect), 0, s, a);
  if (a.keep >= a.capacity) return;
  const dim3 grid(((int64_t)a.c.kv_heads * (a.keep / kQBlock) + 3) / 4, a.c.rows, a.n_layers);
  if (a.c.dh == 32) hipLaunchKernelGGL(k_qcache_move<32>, grid, dim3(256), 0, s, a);
  else if (a.c.dh == 64) hipLaunchKernelGGL(k_qcache_move<64>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(k_qcache_move<128>, grid, dim3(256), 0, s, a);
}

}  // namespace vvs
