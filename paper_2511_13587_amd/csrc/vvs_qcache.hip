// Key/value cache in 8 bits: append, attention with counted weights, eviction, read.
#include <algorithm>

#include "vvs_mfma.h"
#include "vvs_qcache.h"

namespace vvs {

constexpr float kLn2 = 0.6931471805599453f;

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ int row_len(const QLen& len, int r, int capacity) { return min(max(len.len[r >> len.shift], 0), capacity); }

// Eight e4m3 numbers times a power of two as bf16 (exact)
__device__ __forceinline__ bf16x8 e4m3_to_bf16(uint2 b, float scale) {
  uint4 r;
  r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b.x, scale, false));
  r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b.x, scale, true));
  r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b.y, scale, false));
  r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b.y, scale, true));
  return as_bf16x8(r);
}

// e4m3 byte <-> float.  The conversion rounds to nearest, ties to even; nothing above 448 is given to it but what is not finite, which becomes NaN.
template <int I>
__device__ __forceinline__ float e4m3_at(uint32_t w) { return __builtin_amdgcn_cvt_f32_fp8(w, I); }
__device__ __forceinline__ uint32_t to_e4m3x4(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
__device__ __forceinline__ uint2 to_e4m3x8(const float (&v)[8]) { return make_uint2(to_e4m3x4(v[0], v[1], v[2], v[3]), to_e4m3x4(v[4], v[5], v[6], v[7])); }
__device__ __forceinline__ void from_e4m3x8(uint2 b, float (&v)[8]) {
  v[0] = e4m3_at<0>(b.x); v[1] = e4m3_at<1>(b.x); v[2] = e4m3_at<2>(b.x); v[3] = e4m3_at<3>(b.x);
  v[4] = e4m3_at<0>(b.y); v[5] = e4m3_at<1>(b.y); v[6] = e4m3_at<2>(b.y); v[7] = e4m3_at<3>(b.y);
}

// Smallest E >= kQLeast with top <= 448 * 2^E = 0.875 * 2^(E + 9)
__device__ __forceinline__ int e4m3_exponent(float top) {
  int e;
  const float m = frexpf(top, &e);
  return top > 0.f ? max(e - 9 + (m > 0.875f), kQLeast) : kQLeast;
}
__device__ __forceinline__ int exponent_of(float scale) { return scale > 0.f ? ilogbf(scale) : kQLeast; }   // (a block never written holds 0)
__device__ __forceinline__ bool finite(float x) { return fabsf(x) < INFINITY; }

// Byte of (slot w of a block, dim) in the block's keys and in its values (vvs_qcache.h)
__device__ __forceinline__ int key_byte(int w, int dim) {
  const int i = ((w >> 3) << 2) | (w & 3), t = (w >> 2) & 1;
  return (((dim >> 5) * 64 + ((dim >> 3) & 3) * 16 + i) * 2 + t) * 8 + (dim & 7);
}
__device__ __forceinline__ int value_byte(int w, int dim) { return (((dim >> 5) * 64 + (w >> 3) * 16 + (dim & 15)) * 2 + ((dim >> 4) & 1)) * 8 + (w & 7); }

// ------------------------------------------------------------------------------------------------ append
// One wave per (layer, row, head, block that is written into), first its keys, then its values.  Two passes over the wave's share: the largest new
// element gives E, then every lane makes the 16 bytes that it stores.  What the block held is rounded to the larger E.
template <typename T>
__device__ __forceinline__ float element(const void* p, size_t at) { return ld((const T*)p + at); }

template <typename T>
__global__ __launch_bounds__(256) void k_qcache_append(QAppend a, int max_blocks) {
  const int lane = threadIdx.x & 63, unit = blockIdx.x * 4 + (threadIdx.x >> 6), r = blockIdx.y, layer = blockIdx.z;
  const int head = unit / max_blocks, nth = unit % max_blocks;
  if (head >= a.c.kv_heads) return;
  if (a.skip && a.skip[r >> a.len.shift] < 0) return;
  const int len = row_len(a.len, r, a.capacity);
  const int want = a.n_tokens ? min(max(a.n_tokens[r >> a.n_shift] + a.count_plus, 0), a.n) : a.n, n = min(want, a.capacity - len);
  const int block = (len >> 5) + nth, slot0 = block * kQBlock;
  if (n < 1 || slot0 >= len + n) return;
  const int begin = max(len - slot0, 0), end = min(len + n - slot0, kQBlock);   // slots of the block that are written
  const int dh = a.c.dh, shift = slot0 - len;                                   // slot w takes token w + shift
  const size_t row0 = (size_t)layer * a.layer_stride + (size_t)r * a.src_tokens * a.stride + (size_t)head * dh;
  const size_t region = a.c.region(a.layer + layer, r, head);
  uint8_t* data = a.c.data + (region * a.c.blocks + block) * a.c.block_bytes();
  float2* scale = a.c.scale + region * a.c.blocks + block;
  // source token of slot w, < 0: none
  auto token = [&](int w) {
    if (w < begin || w >= end) return -1;
    const int t = w + shift;
    if (!a.select) return t;
    const int p = a.select[(size_t)(r >> a.select_shift) * a.select_stride + t];
    return p >= 0 && p < a.src_tokens ? p : -1;
  };
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const void* src = half ? a.v : a.k;
    float top = 0.f;
    for (int i = lane; i < kQBlock * dh; i += 64) {
      const int t = token(i / dh);
      if (t < 0) continue;
      const float x = fabsf(element<T>(src, row0 + (size_t)t * a.stride + i % dh));
      if (finite(x)) top = fmaxf(top, x);
    }
    const int was = exponent_of(half ? scale->y : scale->x);
    int e = e4m3_exponent(wave_max(top));
    if (begin > 0) e = max(e, was);
    uint8_t* out = data + half * kQBlock * dh;
    const int g = lane >> 4, i = lane & 15;
    for (int c = 0; c < dh / 32; ++c) {
      uint2* at = (uint2*)(out + (c * 64 + lane) * 16);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        float old[8], v[8];
        const uint2 held = at[t];
        from_e4m3x8(held, old);
        bool any = false;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int w = half ? 8 * g + j : 8 * (i >> 2) + 4 * t + (i & 3), dim = half ? c * 32 + t * 16 + i : c * 32 + 8 * g + j;
          const int tok = token(w);
          float x = 0.f;
          if (tok >= 0) x = ldexpf(element<T>(src, row0 + (size_t)tok * a.stride + dim), -e);
          v[j] = w < begin ? ldexpf(old[j], was - e) : finite(x) ? x : __uint_as_float(0x7FC00000u);
          any |= w < end;
        }
        if (any) at[t] = to_e4m3x8(v);
      }
    }
    if (lane == 0) (half ? scale->y : scale->x) = ldexpf(1.f, e);
  }
}

void launch_qcache_append(const QAppend& a, int dtype, hipStream_t s) {
  const int max_blocks = (int)std::min<int64_t>(((int64_t)a.n + 2 * kQBlock - 2) / kQBlock, a.c.blocks);
  const dim3 grid(((int64_t)a.c.kv_heads * max_blocks + 3) / 4, a.c.rows, a.n_layers);
  if (dtype == VVS_BF16) hipLaunchKernelGGL(k_qcache_append<bf16_t>, grid, dim3(256), 0, s, a, max_blocks);
  else hipLaunchKernelGGL(k_qcache_append<float>, grid, dim3(256), 0, s, a, max_blocks);
}

// ------------------------------------------------------------------------------------------------ read
template <typename T>
__global__ __launch_bounds__(256) void k_qcache_read(QRead a) {
  const int dh = a.c.dh, r = blockIdx.y, layer = blockIdx.z, per = a.c.kv_heads * (dh / 8);
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= (int64_t)a.n * per) return;
  const int j = (int)(i / per), head = (int)(i % per) / (dh / 8), dim = (int)(i % per) % (dh / 8) * 8;
  const int len = row_len(a.len, r, a.capacity);
  const int64_t slot = (int64_t)(a.first ? a.first[r] : 0) + j;
  float k[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (slot >= 0 && slot < len) {
    const size_t block = a.c.region(a.layer + layer, r, head) * a.c.blocks + (slot >> 5);
    const uint8_t* data = a.c.data + block * a.c.block_bytes();
    const float2 sc = a.c.scale[block];
    const int w = (int)(slot & 31);
    from_e4m3x8(*(const uint2*)(data + key_byte(w, dim)), k);
    const uint8_t* vb = data + kQBlock * dh + value_byte(w, dim);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      k[e] *= sc.x;
      v[e] = e4m3_at<0>(vb[e * 16]) * sc.y;
    }
  }
  const size_t at = (((size_t)layer * a.c.rows + r) * a.n + j) * a.c.kv_heads * dh + (size_t)head * dh + dim;
  if constexpr (sizeof(T) == 4) {
    ((float4*)((T*)a.k + at))[0] = make_float4(k[0], k[1], k[2], k[3]);
    ((float4*)((T*)a.k + at))[1] = make_float4(k[4], k[5], k[6], k[7]);
    ((float4*)((T*)a.v + at))[0] = make_float4(v[0], v[1], v[2], v[3]);
    ((float4*)((T*)a.v + at))[1] = make_float4(v[4], v[5], v[6], v[7]);
  } else {
    *(uint4*)((T*)a.k + at) = make_uint4(pack2bf(k[0], k[1]), pack2bf(k[2], k[3]), pack2bf(k[4], k[5]), pack2bf(k[6], k[7]));
    *(uint4*)((T*)a.v + at) = make_uint4(pack2bf(v[0], v[1]), pack2bf(v[2], v[3]), pack2bf(v[4], v[5]), pack2bf(v[6], v[7]));
  }
}

void launch_qcache_read(const QRead& a, int dtype, hipStream_t s) {
  const int64_t items = (int64_t)a.n * a.c.kv_heads * (a.c.dh / 8);
  const dim3 grid((items + 255) / 256, a.c.rows, a.n_layers);
  if (dtype == VVS_BF16) hipLaunchKernelGGL(k_qcache_read<bf16_t>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(k_qcache_read<float>, grid, dim3(256), 0, s, a);
}

// ------------------------------------------------------------------------------------------------ attention
// One wave takes 32 keys a step (a cached block, or 32 block tokens) against 16 NQB queries; a query is (block token, query head of the key/value head).
// The online softmax keeps the running maximum in units of log2: m = max(score * c), weights 2^(score c - m).  Cached elements are exact in bf16, so scores
// are bf16 products summed in fp32; fp32 queries (and block keys, values and weights) go in as sums of NS bf16 values, which hold all 24 bits.

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
__device__ __forceinline__ void read8(const float* p, float (&v)[8]) {
  const float4 a = ((const float4*)p)[0], b = ((const float4*)p)[1];
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
template <int NS>
__device__ __forceinline__ void load_operand(const float* p, bool there, bf16x8 (&out)[NS]) {
  float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (there) read8(p, v);
  split8<NS>(v, out);
}
template <int NS>
__device__ __forceinline__ void load_operand(const bf16_t* p, bool there, bf16x8 (&out)[NS]) {
  static_assert(NS == 1, "");
  out[0] = as_bf16x8(there ? *(const uint4*)p : make_uint4(0, 0, 0, 0));
}

template <typename T, int DH>
struct QShape {
  static constexpr int NS = sizeof(T) == 4 ? 3 : 1;     // bf16 values that make up an operand of the caller's type
  static constexpr int NP = sizeof(T) == 4 ? 3 : 2;     // ... and a softmax weight (of bf16 calls: to 2^-17)
  static constexpr int KD = DH / 32, DT = DH / 16;
};

// Keys of a step in the operand registers: kf[tile][dims][part]
template <typename T, int DH, int NK>
__device__ __forceinline__ void keys_of_block(const uint8_t* data, float scale, int lane, bf16x8 (&kf)[2][DH / 32][NK]) {
#pragma unroll
  for (int kd = 0; kd < DH / 32; ++kd) {
    const uint4 b = *(const uint4*)(data + (kd * 64 + lane) * 16);
    kf[0][kd][0] = e4m3_to_bf16(make_uint2(b.x, b.y), scale);
    kf[1][kd][0] = e4m3_to_bf16(make_uint2(b.z, b.w), scale);
  }
}
// Values; slots from `valid` on of the block (of the wave's 32) are zeros: what lies behind the length may be anything
template <int DH>
__device__ __forceinline__ void values_of_block(const uint8_t* data, float scale, int lane, int valid, bf16x8 (&vf)[DH / 16][1]) {
  const int mine = valid - 8 * (lane >> 4);       // of this lane's 8 slots
  const uint64_t keep = mine >= 8 ? ~0ull : mine <= 0 ? 0ull : (1ull << (8 * mine)) - 1;
#pragma unroll
  for (int c = 0; c < DH / 32; ++c) {
    uint4 b = *(const uint4*)(data + kQBlock * DH + (c * 64 + lane) * 16);
    b.x &= (uint32_t)keep; b.y &= (uint32_t)(keep >> 32); b.z &= (uint32_t)keep; b.w &= (uint32_t)(keep >> 32);
    vf[2 * c][0] = e4m3_to_bf16(make_uint2(b.x, b.y), scale);
    vf[2 * c + 1][0] = e4m3_to_bf16(make_uint2(b.z, b.w), scale);
  }
}
// slot of tile t's row that lane l % 16 = i supplies
__device__ __forceinline__ int slot_of(int t, int i) { return 8 * (i >> 2) + 4 * t + (i & 3); }

template <typename T, int DH, int NS>
__device__ __forceinline__ void keys_of_tokens(const T* k, size_t stride, int tok0, int n, int lane, bf16x8 (&kf)[2][DH / 32][NS]) {
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int tok = tok0 + slot_of(t, lane & 15);
#pragma unroll
    for (int kd = 0; kd < DH / 32; ++kd) load_operand<NS>(k + (size_t)min(tok, n - 1) * stride + kd * 32 + (lane >> 4) * 8, tok < n, kf[t][kd]);
  }
}
// ... with zeros for elements that are not finite; returns whether this lane met any
template <typename T, int DH, int NS>
__device__ __forceinline__ bool values_of_tokens(const T* v, size_t stride, int tok0, int n, int lane, bf16x8 (&vf)[DH / 16][NS]) {
  bool odd = false;
#pragma unroll
  for (int dt = 0; dt < DH / 16; ++dt) {
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int tok = tok0 + (lane >> 4) * 8 + j;
      x[j] = tok < n ? ld(v + (size_t)min(tok, n - 1) * stride + dt * 16 + (lane & 15)) : 0.f;
      if (!finite(x[j])) { odd = true; x[j] = 0.f; }
    }
    split8<NS>(x, vf[dt]);
  }
  return odd;
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

// Online softmax of 8 scores per lane and O^T += V^T P^T; e: the weights, as they went in
template <int DT, int NK, int NP>
__device__ __forceinline__ void step_softmax(const float (&sv)[8], const bf16x8 (&vf)[DT][NK], float c_exp, float& m_run, float& l_run, floatx4 (&o)[DT], float (&e)[8]) {
  float mx = sv[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) mx = fmaxf(mx, sv[i]);
  const float m_new = fmaxf(m_run, rows_max(mx) * c_exp);
  const float m_safe = m_new == -INFINITY ? 0.f : m_new;
  const float alpha = __builtin_amdgcn_exp2f(m_run - m_safe);
  float rs = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    e[i] = __builtin_amdgcn_exp2f(fmaf(sv[i], c_exp, -m_safe));
    rs += e[i];
  }
  l_run = l_run * alpha + rows_sum(rs);
  m_run = m_new;
  bf16x8 pf[NP];
  split8<NP>(e, pf);
  if (__builtin_amdgcn_ballot_w64(alpha != 1.0f)) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int j = 0; j < 4; ++j) o[dt][j] *= alpha;
  }
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

// log-sum-exp for the caller, maximum and 1 / sum for the counted weights (from the log alone they would lose what its size takes of 24 bits)
__device__ __forceinline__ void tell_norm(const QAttention& a, size_t at, float m, float l) {
  const bool none = m == -INFINITY;
  if (a.lse) a.lse[at] = none ? -INFINITY : (m + log2f(l)) * kLn2;
  if (a.norm) a.norm[at] = make_float2(none ? 0.f : m, none ? 0.f : 1.f / l);
}

// grid (kv_heads * query tiles, splits, rows), 4 waves.  The steps of a split go to its waves in turn; the waves' results are joined through LDS.
template <typename T, int DH, int NQB>
__global__ __launch_bounds__(256) void k_qcache_attention(QAttention a, int q_tiles) {
  using S = QShape<T, DH>;
  constexpr int KD = S::KD, DT = S::DT, NS = S::NS, NP = S::NP, NQ = 16 * NQB;
  __shared__ float s_o[2][NQ][DH + 4];
  __shared__ float s_m[4][NQ], s_l[4][NQ];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, col = lane & 15;
  const int hk = blockIdx.x / q_tiles, q0 = (blockIdx.x % q_tiles) * NQ, r = blockIdx.z, split = blockIdx.y;
  const QRow w = row_of(a, r);
  const int nq = w.n * a.group;
  if (q0 >= nq) return;                       // only tokens behind the row's number
  const T* q = (const T*)a.q + (size_t)r * a.T * a.q_stride + (size_t)hk * a.group * DH;
  const T* k = (const T*)a.k + (size_t)r * a.T * a.kv_stride + (size_t)hk * DH;
  const T* v = (const T*)a.v + (size_t)r * a.T * a.kv_stride + (size_t)hk * DH;
  const size_t region = a.c.region(a.layer, r, hk) * a.c.blocks;
  bf16x8 qf[NQB][KD][NS];
  int qt[NQB];                                // block token of this lane's query
#pragma unroll
  for (int qb = 0; qb < NQB; ++qb) {
    const int qi = min(q0 + qb * 16 + col, nq - 1);
    qt[qb] = qi / a.group;
#pragma unroll
    for (int kd = 0; kd < KD; ++kd)
      load_operand<NS>(q + (size_t)qt[qb] * a.q_stride + (size_t)(qi % a.group) * DH + kd * 32 + g * 8, true, qf[qb][kd]);
  }
  float m_run[NQB], l_run[NQB];
  floatx4 o[NQB][DT];
#pragma unroll
  for (int qb = 0; qb < NQB; ++qb) {
    m_run[qb] = -INFINITY;
    l_run[qb] = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[qb][dt] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  // block tokens that the tile's queries can see: with a chain none behind the last query
  const int seen = !a.k ? 0 : a.causal ? min(w.n, (min(q0 + NQ, nq) - 1) / a.group + 1) : w.n;
  const int steps = w.blocks + (seen + 31) / 32;
  const int s0 = (int)((int64_t)steps * split / a.splits), s1 = (int)((int64_t)steps * (split + 1) / a.splits);
  for (int step = s0 + wave; step < s1; step += 4) {
    float e[8];
    if (step < w.blocks) {
      const uint8_t* data = a.c.data + (region + step) * a.c.block_bytes();
      const float2 sc = a.c.scale[region + step];
      const int valid = w.len - step * kQBlock;
      bf16x8 kf[2][KD][1], vf[DT][1];
      keys_of_block<T, DH, 1>(data, sc.x, lane, kf);
      values_of_block<DH>(data, sc.y, lane, valid, vf);
#pragma unroll
      for (int qb = 0; qb < NQB; ++qb) {
        float sv[8];
        step_scores<KD, 1, NS>(kf, qf[qb], sv);
        if (valid < kQBlock) {
#pragma unroll
          for (int i = 0; i < 8; ++i) sv[i] = 8 * g + i < valid ? sv[i] : -INFINITY;
        }
        step_softmax<DT, 1, NP>(sv, vf, a.c_exp, m_run[qb], l_run[qb], o[qb], e);
      }
    } else {
      const int tok0 = (step - w.blocks) * 32;
      bf16x8 kf[2][KD][NS], vf[DT][NS];
      keys_of_tokens<T, DH, NS>(k, a.kv_stride, tok0, seen, lane, kf);
      const bool odd = __builtin_amdgcn_ballot_w64(values_of_tokens<T, DH, NS>(v, a.kv_stride, tok0, seen, lane, vf)) != 0;
#pragma unroll
      for (int qb = 0; qb < NQB; ++qb) {
        float sv[8];
        step_scores<KD, NS, NS>(kf, qf[qb], sv);
        const uint32_t vis = sees8(a, qt[qb], tok0 + 8 * g, seen);
#pragma unroll
        for (int i = 0; i < 8; ++i) sv[i] = (vis >> i) & 1 ? sv[i] : -INFINITY;
        step_softmax<DT, NS, NP>(sv, vf, a.c_exp, m_run[qb], l_run[qb], o[qb], e);
        if (odd) {                            // values that are not finite: only for the queries that see them
          for (int j = 0; j < 32 && tok0 + j < seen; ++j) {
            float p = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float x = __shfl(e[i], (j >> 3) * 16 + col, 64);
              if ((j & 7) == i) p = x;
            }
            if (sees8(a, qt[qb], tok0 + j, seen) & 1) {
#pragma unroll
              for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  const float x = ld(v + (size_t)(tok0 + j) * a.kv_stride + dt * 16 + 4 * g + i);
                  if (!finite(x)) o[qb][dt][i] += p * x;
                }
            }
          }
        }
      }
    }
  }
  // join the four waves: common maximum, then sums in the order (0 + 2) + (1 + 3)
#pragma unroll
  for (int qb = 0; qb < NQB; ++qb)
    if (g == 0) { s_m[wave][qb * 16 + col] = m_run[qb]; s_l[wave][qb * 16 + col] = l_run[qb]; }
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
    for (int i = 0; i < 4; ++i) l_all[qb] += s_l[i][qi] * __builtin_amdgcn_exp2f(s_m[i][qi] - m);
    const float f = __builtin_amdgcn_exp2f(m_run[qb] - m);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[qb][dt][i] *= f;
  }
#pragma unroll
  for (int round = 0; round < 2; ++round) {
    const bool gives = round == 0 ? wave >= 2 : wave == 1, takes = round == 0 ? wave < 2 : wave == 0;
    if (round) __syncthreads();
    if (gives) {
#pragma unroll
      for (int qb = 0; qb < NQB; ++qb)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) *(floatx4*)&s_o[wave & 1][qb * 16 + col][dt * 16 + 4 * g] = o[qb][dt];
    }
    __syncthreads();
    if (takes) {
#pragma unroll
      for (int qb = 0; qb < NQB; ++qb)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[qb][dt] += *(const floatx4*)&s_o[round ? 1 : wave][qb * 16 + col][dt * 16 + 4 * g];
    }
  }
  if (wave) return;
#pragma unroll
  for (int qb = 0; qb < NQB; ++qb) {
    const int qi = q0 + qb * 16 + col;
    if (qi >= nq) continue;
    if (a.splits > 1) {
      float* part = a.parts + ((((size_t)r * gridDim.x + blockIdx.x) * a.splits + split) * NQ + qb * 16 + col) * (DH + 2);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 4; i += 2) *(float2*)(part + dt * 16 + 4 * g + i) = make_float2(o[qb][dt][i], o[qb][dt][i + 1]);
      if (g == 0) *(float2*)(part + DH) = make_float2(m_all[qb], l_all[qb]);
      continue;
    }
    const size_t at = query_at(a, r, hk, qi);
    const bool none = m_all[qb] == -INFINITY;
    const float inv = none ? 0.f : 1.f / l_all[qb];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      float x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = o[qb][dt][i] * inv;
      store4<T, DH>(a, at, dt * 16 + 4 * g, x);
    }
    if (g == 0) tell_norm(a, at, m_all[qb], l_all[qb]);
  }
}

// Joins the splits: one group of DH / 4 lanes per query
template <typename T, int DH>
__global__ __launch_bounds__(256) void k_qcache_join(QAttention a, int q_tiles, int nq_tile) {
  constexpr int LQ = DH / 4;
  const int hk = blockIdx.x / q_tiles, tile = blockIdx.x % q_tiles, r = blockIdx.z;
  const int in_tile = blockIdx.y * (256 / LQ) + threadIdx.x / LQ, dim = threadIdx.x % LQ * 4;
  const QRow w = row_of(a, r);
  const int qi = tile * nq_tile + in_tile;
  if (in_tile >= nq_tile || qi >= w.n * a.group) return;
  const float* part = a.parts + (((size_t)r * gridDim.x + blockIdx.x) * a.splits * nq_tile + in_tile) * (DH + 2);
  const size_t step = (size_t)nq_tile * (DH + 2);
  float m = -INFINITY;
  for (int s = 0; s < a.splits; ++s) m = fmaxf(m, part[s * step + DH]);
  const bool none = m == -INFINITY;
  float l = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < a.splits && !none; ++s) {
    const float f = __builtin_amdgcn_exp2f(part[s * step + DH] - m);
    l += part[s * step + DH + 1] * f;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] += part[s * step + dim + i] * f;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = none ? 0.f : x[i] / l;
  const size_t at = query_at(a, r, hk, qi);
  store4<T, DH>(a, at, dim, x);
  if (dim == 0) tell_norm(a, at, m, l);
}

// Counted weights: the scores are made again, now with the normaliser known.  One wave per 32 keys, over all counted queries in order.
template <typename T, int DH>
__global__ __launch_bounds__(256) void k_qcache_mass(QAttention a) {
  using S = QShape<T, DH>;
  constexpr int KD = S::KD, NS = S::NS;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, col = lane & 15;
  const int hk = blockIdx.y, r = blockIdx.z;
  const QRow w = row_of(a, r);
  const int seen = a.k ? w.n : 0, steps = w.blocks + (a.block_mass ? (a.T + 31) / 32 : 0), nq = min(a.n_counted, w.n) * a.group;
  const T* q = (const T*)a.q + (size_t)r * a.T * a.q_stride + (size_t)hk * a.group * DH;
  const T* k = (const T*)a.k + (size_t)r * a.T * a.kv_stride + (size_t)hk * DH;
  const size_t region = a.c.region(a.layer, r, hk) * a.c.blocks;
  for (int step = (a.mass ? 0 : w.blocks) + blockIdx.x * 4 + wave; step < steps; step += gridDim.x * 4) {
    const bool cached = step < w.blocks;
    const int tok0 = (step - w.blocks) * 32, valid = cached ? w.len - step * kQBlock : seen - tok0;
    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    bf16x8 kf[2][KD][NS];
    if (cached) {
      bf16x8 one[2][KD][1];
      keys_of_block<T, DH, 1>(a.c.data + (region + step) * a.c.block_bytes(), a.c.scale[region + step].x, lane, one);
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int kd = 0; kd < KD; ++kd) {
          kf[t][kd][0] = one[t][kd][0];
#pragma unroll
          for (int p = 1; p < NS; ++p) kf[t][kd][p] = as_bf16x8(make_uint4(0, 0, 0, 0));
        }
    } else if (valid > 0) {
      keys_of_tokens<T, DH, NS>(k, a.kv_stride, tok0, seen, lane, kf);
    }
    // (of a chain only the queries from the step's first token on see anything)
    for (int q0 = !cached && a.causal ? tok0 * a.group / 16 * 16 : 0; q0 < nq && valid > 0; q0 += 16) {
      const int qi = min(q0 + col, nq - 1), t = qi / a.group;
      bf16x8 qf[KD][NS];
#pragma unroll
      for (int kd = 0; kd < KD; ++kd) load_operand<NS>(q + (size_t)t * a.q_stride + (size_t)(qi % a.group) * DH + kd * 32 + g * 8, true, qf[kd]);
      const float2 norm = a.norm[query_at(a, r, hk, qi)];
      float sv[8];
      step_scores<KD, NS, NS>(kf, qf, sv);
      const int there = valid - 8 * g;
      const uint32_t vis = q0 + col >= nq ? 0u : cached ? (there >= 8 ? 255u : there <= 0 ? 0u : (1u << there) - 1) : sees8(a, t, tok0 + 8 * g, seen);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float p = __builtin_amdgcn_exp2f(fmaf(sv[i], a.c_exp, -norm.x)) * norm.y;
        sum[i] += (vis >> i) & 1 ? p : 0.f;
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {                 // over the 16 queries of the lane's row
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
      if (cached) {
        if (at < valid) a.mass[((size_t)r * a.c.kv_heads + hk) * a.capacity + (size_t)step * kQBlock + at] += x;
      } else if (tok0 + at < w.n) {
        a.block_mass[((size_t)r * a.c.kv_heads + hk) * a.T + tok0 + at] = x;
      }
    }
  }
}

template <typename T, int DH, int NQB>
static void attention_t(QAttention a, hipStream_t s) {
  const int q_tiles = (a.T * a.group + 16 * NQB - 1) / (16 * NQB);
  const int64_t tiles = (int64_t)a.c.rows * a.c.kv_heads * q_tiles;
  // As many splits as give each CU about four workgroups, with at least four steps each where the cache is full; the partial results have room for kQParts
  const int64_t most = (int64_t)kQParts / (tiles * NQB);
  a.splits = (int)std::max<int64_t>(1, std::min<int64_t>({1024 / tiles, most, (a.c.blocks + 3) / 4}));
  const dim3 grid(a.c.kv_heads * q_tiles, a.splits, a.c.rows);
  hipLaunchKernelGGL((k_qcache_attention<T, DH, NQB>), grid, dim3(256), 0, s, a, q_tiles);
  if (a.splits > 1) {
    const int per = 256 / (DH / 4);
    hipLaunchKernelGGL((k_qcache_join<T, DH>), dim3(grid.x, (16 * NQB + per - 1) / per, grid.z), dim3(256), 0, s, a, q_tiles, 16 * NQB);
  }
  if (a.n_counted > 0 || a.block_mass) {
    const int steps = a.c.blocks + (a.T + 31) / 32;
    hipLaunchKernelGGL((k_qcache_mass<T, DH>), dim3(std::min((steps + 3) / 4, 1024), a.c.kv_heads, a.c.rows), dim3(256), 0, s, a);
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
    else if (nq <= 32 || DH == 128) attention_t<T, DH, 2>(a, s);
    else if constexpr (DH < 128) attention_t<T, DH, 4>(a, s);
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
// Which slots stay: one workgroup per (layer, row, head) finds the keep-th largest weight by its bits, 8 at a time, then deals the kept slots behind `keep` to the
// holes in front of it, in order.  Order-preserving bits: a weight's sign bit is flipped, or all its bits when it is set; -0 counts as 0, NaN as the largest.
constexpr int kQSelect = 1024;

__device__ __forceinline__ uint32_t mass_bits(float m) {
  const uint32_t u = __float_as_uint(m == 0.f ? 0.f : m);
  if (m != m) return 0xFFFFFFFEu;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// exclusive prefix over the workgroup; *total: the sum.  red: kQSelect / 64 + 1 ints
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

__global__ __launch_bounds__(kQSelect) void k_qcache_select(QEvict a) {
  __shared__ int s_hist[256], s_red[kQSelect / 64 + 1], s_pick[2];
  const int head = blockIdx.x, r = blockIdx.y, layer = blockIdx.z, tid = threadIdx.x;
  const size_t region = ((size_t)layer * a.c.rows + r) * a.c.kv_heads + head, base = region * a.capacity;
  const int len = row_len(a.len, r, a.capacity), left = min(len, a.keep);
  const float* mass = a.mass + base;
  float* mass_out = a.mass_out + base;
  const int32_t* pos = a.pos ? a.pos + base : nullptr;
  int32_t* pos_out = a.pos ? a.pos_out + base : nullptr;
  int32_t* origin = a.origin + base;
  if (len <= a.keep) {
    for (int i = tid; i < a.capacity; i += kQSelect) {
      if (i < left) origin[i] = i;
      mass_out[i] = i < left ? mass[i] : 0.f;
      if (pos) pos_out[i] = i < left ? pos[i] : 0;
    }
    return;
  }
  int newest = len - 1;
  if (pos) {
    newest = pos[0];
    for (int i = tid; i < len; i += kQSelect) newest = max(newest, pos[i]);
    newest = block_max_int(newest, s_red);
  }
  auto key = [&](int i) {
    const int64_t p = pos ? pos[i] : i;
    return p > (int64_t)newest - a.recent ? 0xFFFFFFFFu : mass_bits(mass[i]);
  };
  uint32_t prefix = 0;
  int need = a.keep;                       // of the keys that share the prefix, how many are kept
  for (int shift = 24; shift >= 0; shift -= 8) {
    __syncthreads();
    if (tid < 256) s_hist[tid] = 0;
    __syncthreads();
    for (int i = tid; i < len; i += kQSelect) {
      const uint32_t k = key(i);
      if (shift == 24 || k >> (shift + 8) == prefix) atomicAdd(&s_hist[(k >> shift) & 255], 1);   // whole numbers: in any order the same
    }
    __syncthreads();
    if (tid == 0) {
      int b = 255, above = 0;
      while (above + s_hist[b] < need) above += s_hist[b--];
      s_pick[0] = b;
      s_pick[1] = need - above;
    }
    __syncthreads();
    prefix = prefix << 8 | (uint32_t)s_pick[0];
    need = s_pick[1];
  }
  // kept: keys above the prefix, and the first `need` equal to it
  int equal = 0, holes = 0, sources = 0;
  for (int i0 = 0; i0 < len; i0 += kQSelect) {
    const int i = i0 + tid;
    const uint32_t k = i < len ? key(i) : 0;
    int total;
    const bool eq = i < len && k == prefix;
    const int rank = equal + block_rank(eq, s_red, &total);
    equal += total;
    const bool kept = i < len && (k > prefix || (eq && rank < need));
    const bool hole = i < a.keep && !kept, source = i >= a.keep && kept;
    const int h = holes + block_rank(hole, s_red, &total);
    holes += total;
    const int q = sources + block_rank(source, s_red, &total);
    sources += total;
    // a hole notes its number; the sources, as many as there are holes, are listed behind `keep`
    if (i < a.keep) origin[i] = kept ? i : -1 - h;
    if (source) origin[a.keep + q] = i;
  }
  __syncthreads();
  for (int i = tid; i < a.keep; i += kQSelect) {
    const int o = origin[i];
    const int from = o >= 0 ? i : origin[a.keep + (-1 - o)];
    origin[i] = from;
    const float m = mass[from];
    mass_out[i] = m;
    if (pos) pos_out[i] = pos[from];
  }
  __syncthreads();
  for (int i = a.keep + tid; i < a.capacity; i += kQSelect) {
    mass_out[i] = 0.f;
    if (pos) pos_out[i] = 0;
  }
}

// Moves the elements: one wave per (layer, row, head, block below keep)
__global__ __launch_bounds__(256) void k_qcache_move(QEvict a) {
  const int lane = threadIdx.x & 63, unit = blockIdx.x * 4 + (threadIdx.x >> 6), r = blockIdx.y, layer = blockIdx.z;
  const int blocks = a.keep / kQBlock, head = unit / blocks, block = unit % blocks;
  if (head >= a.c.kv_heads) return;
  if (row_len(a.len, r, a.capacity) <= a.keep) return;
  const int dh = a.c.dh;
  const size_t base = (((size_t)layer * a.c.rows + r) * a.c.kv_heads + head) * a.capacity, region = a.c.region(a.layer + layer, r, head) * a.c.blocks;
  const int from = a.origin[base + block * kQBlock + (lane & 31)];
  if (!__builtin_amdgcn_ballot_w64(from != block * kQBlock + (lane & 31))) return;
  const float2 sc = a.c.scale[region + (from >> 5)];
  const int ek = exponent_of(sc.x), ev = exponent_of(sc.y);
  int tk = ek, tv = ev;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) { tk = max(tk, __shfl_xor(tk, o, 64)); tv = max(tv, __shfl_xor(tv, o, 64)); }
  uint8_t* data = a.c.data + (region + block) * a.c.block_bytes();
  const int g = lane >> 4, i = lane & 15;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    uint8_t* out = data + half * kQBlock * dh;
    for (int c = 0; c < dh / 32; ++c) {
      uint2* at = (uint2*)(out + (c * 64 + lane) * 16);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        float v[8];
        if (half == 0) {
          const int w = slot_of(t, i), src = __shfl(from, w, 64), e = __shfl(ek, w, 64);
          from_e4m3x8(*(const uint2*)(a.c.data + (region + (src >> 5)) * a.c.block_bytes() + key_byte(src & 31, c * 32 + 8 * g)), v);
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] = ldexpf(v[j], e - tk);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int w = 8 * g + j, src = __shfl(from, w, 64), e = __shfl(ev, w, 64);
            const uint8_t b = a.c.data[(region + (src >> 5)) * a.c.block_bytes() + kQBlock * dh + value_byte(src & 31, c * 32 + t * 16 + i)];
            v[j] = ldexpf(e4m3_at<0>(b), e - tv);
          }
        }
        at[t] = to_e4m3x8(v);
      }
    }
  }
  if (lane == 0) a.c.scale[region + block] = make_float2(ldexpf(1.f, tk), ldexpf(1.f, tv));
}

void launch_qcache_evict(const QEvict& a, hipStream_t s) {
  hipLaunchKernelGGL(k_qcache_select, dim3(a.c.kv_heads, a.c.rows, a.n_layers), dim3(kQSelect), 0, s, a);
  if (a.keep >= a.capacity) return;
  hipLaunchKernelGGL(k_qcache_move, dim3(((int64_t)a.c.kv_heads * (a.keep / kQBlock) + 3) / 4, a.c.rows, a.n_layers), dim3(256), 0, s, a);
}

}  // namespace vvs
