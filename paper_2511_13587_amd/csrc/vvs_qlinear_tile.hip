// Products of many rows in 8 bits: tiles whose rows pass through LDS.
#include <algorithm>
#include <type_traits>

#include "vvs_e4m3.h"
#include "vvs_qlinear_device.h"

namespace vvs {

// Order of the tiles.  Workgroups are dealt to the 8 XCDs round-robin; each takes a run of consecutive tiles of an order that goes through bands of 8 row tiles column by column, so that what an
// XCD's 32 CUs work on at a time - 8 row tiles times 4 column tiles - shares its rows and weights in the XCD's L2.
__device__ __forceinline__ void qtile_of(int id, int MT, int NT, int* tile_m, int* tile_n) {
  const int all = MT * NT, x = id & 7, q = all >> 3, p = x * q + min(x, all & 7) + (id >> 3);
  const int band = p / (8 * NT), rem = p % (8 * NT), h = min(8, MT - 8 * band);
  *tile_n = rem / h;
  *tile_m = band * 8 + rem % h;
}

// Y^T = W^T X^T.  A workgroup of WM x WN waves makes 16 RT WM rows by WN groups of 64 columns; a wave 16 RT rows of one group, whose weights nobody else in the workgroup needs: they come straight into its operand
// registers, NB - 1 blocks of 128 contraction values ahead.  The rows' bytes of a block are every wave's, and pass through LDS (lds_dma16, no registers), two or three blocks ahead.
// Bound by the matrix cores: 8192 rows, 4096 -> 12288, 825 GFLOP in 321 us, 2.6 PFLOP/s (an 8192^3 product in e4m3 by the library 2.7), the matrix cores busy 75 % of the time, waves waiting 24 % of theirs; a
// tile of 128 x 256 reads 48 KB a block for 8.4 MFLOP, and 82 % of the requests to the L2 are hits.
// What is under way: the waits written out let the requests of one block (NB = 2) or two (NB = 4) be.  The compiler adds waits for the weights' loads, which it knows, and cannot count the rows', which it does not: in
// front of the products of every step (NB = 2, where the rows are asked for last), of two steps in four (NB = 4; with shares of three, and in part of the fourth), it waits until all has landed.  What was asked for half a
// step before is then waited for.  Too strict, never too lax: the results do not depend on it.
// Few tiles wait for loads, some 0.6 us per block: NB = 4, and KS shares of the contraction with waves, stages and powers of their own, whose sums the first adds up through LDS in their
// order (432 rows: 1280 -> 3840 in one share 7.7 us; 3456 -> 1280 in four 10.9, one 12.3; 11008 -> 4096 in four 39.5, one 54.8).  Powers of the first blocks are asked for in front of everything else (432 rows, 1280 ->
// 3840 9.3 -> 8.3).
// FAST: the e4m3 numbers go into the matrix cores as they are, with both powers of two as scales (16x16x128, twice the rate of bf16 and fewer instructions).  These products lose what lies 2^13
// below the largest of a few neighbours: 1.3e-5 of the result in the 2-norm for normally distributed operands, 130 times below the rounding of bf16 outputs and 2000 times below that of 8 bits; more of sums that
// cancel.  !FAST: bf16 operands, exact; what up to 64 rows take, and more where the caller wants it (vvs_qlinear_config.products) or outputs are in fp32, but for the sums of bf16 contexts.
constexpr int power_blocks(int shares) { return shares > 1 ? 32 : 64; }                  // whose powers lie in LDS at a time
constexpr int power_stride(int shares) { return power_blocks(shares) / 4 + 1; }          // (an odd number of words: 16 rows on 16 banks)
// LDS of a share: rows [stages][BM][128 bytes], then powers of its next blocks: [BM][stride], [64 WN][stride], four in a word
constexpr int tile_stages(int NB) { return NB == 2 ? 3 : NB; }
constexpr int share_lds(int BM, int WN, int NB, int shares) { return tile_stages(NB) * BM * kQRowBlock + (BM + 64 * WN) * power_stride(shares) * 4; }

// Place of 16 bytes c of row r in LDS: c ^ swizzle(r), so that the lanes that LDS serves at a time read different banks.  It serves a wave's 16-byte reads 16 lanes at a time - lanes 0-3, 12-15, 20-23, 24-27;
// 4-7, 8-11, 16-19, 28-31; and the same 32 on - from 64 banks, two rows of 128 bytes: rows 4 to 11 of a tile go by with the other half of the contraction than the rest.  (r & 7: two lanes on every bank, by
// SQ_LDS_BANK_CONFLICT; so none.)
__device__ __forceinline__ int swizzle(int r) { return ((r >> 1) & 7) ^ (((r + 4) >> 3 & 1) << 1); }

struct __attribute__((aligned(8))) Bytes16 { uint32_t x, y, z, w; };     // (rows of bf16 may lie at multiples of 8 bytes)

template <int WM, int WN, int RT, bool FAST, bool GATED, typename T, int NB, int KS>
__global__ __launch_bounds__(64 * WM * WN * KS, 2) void k_qlinear_tile(QProduct a, int MT, int NT) {
  constexpr int BM = 16 * RT * WM, NW = WM * WN, NQ = BM / 8 / NW, kStages = tile_stages(NB), kPowerBlocks = power_blocks(KS), kPowerStride = power_stride(KS);
  static_assert(BM <= 64 * NW && BM % (8 * NW) == 0 && (!GATED || (WM == 1 && WN == 4 && KS == 1)) && (NW & (NW - 1)) == 0, "");
  extern __shared__ uint4 lds[];
  const int all_waves = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), share = KS == 1 ? 0 : all_waves / NW, wave = KS == 1 ? all_waves : all_waves % NW;
  const int tid = KS == 1 ? threadIdx.x : threadIdx.x & (64 * NW - 1), lane = tid & 63, i = lane & 15, g = lane >> 4;
  char* const my_lds = (char*)lds + share * share_lds(BM, WN, NB, KS);
  int* const xpow = (int*)(my_lds + kStages * BM * kQRowBlock);
  int* const wpow = xpow + BM * kPowerStride;
  const int wm = wave / WN, wn = wave % WN;
  int tile_m, tile_n;
  qtile_of(blockIdx.x, MT, NT, &tile_m, &tile_n);
  // this share's blocks: first .. first + blocks - 1, of `most` at most
  const int m0 = tile_m * BM, powers = qrows_powers(a.w.in), first = KS == 1 ? 0 : share * a.w.blocks / KS, blocks = KS == 1 ? a.w.blocks : (share + 1) * a.w.blocks / KS - first;
  const int most = KS == 1 ? blocks : (a.w.blocks + KS - 1) / KS;
  const int own_group = tile_n * WN + wn, group = min(own_group, a.w.groups - 1);
  const size_t width = (size_t)a.w.blocks * kQRowBlock;
  const uint32_t lds0 = (uint32_t)(uintptr_t)my_lds;

  // rows behind the last one repeat it
  const uint8_t* const tile_rows = a.x.values + (size_t)m0 * width + first * kQRowBlock;
  uint32_t src[NQ];
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    const int r = (wave * NQ + q) * 8 + (lane >> 3);
    src[q] = (uint32_t)(min(r, a.M - 1 - m0) * (int)width + ((lane & 7) ^ swizzle(r)) * 16);
  }
  auto request = [&](int kb, int stage, int q) { lds_dma16(tile_rows + (size_t)kb * kQRowBlock, src[q], lds0 + stage * BM * kQRowBlock + (wave * NQ + q) * 1024); };
  const uint8_t* const wsrc = a.w.data + a.w.tile_at(group, first, 0);
  auto weights = [&](int kb, u32x4 (&w)[4][2], int c, int h) { w[c][h] = *(const u32x4*)(wsrc + (size_t)kb * 8192 + c * 2048 + h * 1024 + lane * 16); };
  // powers of blocks k0 .. k0 + kPowerBlocks - 1 of the share into LDS (bytes from memory at every block cost a large product 6 %).  A share that begins inside a word of four moves the bytes to where they are
  // in its own count.
  constexpr int kLanes = 64 * NW / BM;                           // threads that a row's words are dealt to
  struct Powers { int x[4], w[8]; };
  auto load_powers = [&](int k0, int d0) {                       // words d0 .. d0 + 7 of the columns', d0 / 2 * kLanes and on of the rows'
    const int words = (min(kPowerBlocks, blocks - k0) + 3) / 4, at = (first + k0) / 4, last = powers / 4 - 1, sh = 8 * (first & 3);
    auto word = [&](const int* p, int d, int step) {
      if constexpr (KS == 1) return p[(size_t)(at + d) * step];
      else return (int)(((uint64_t)(uint32_t)p[(size_t)min(at + d + 1, last) * step] << 32 | (uint32_t)p[(size_t)(at + d) * step]) >> sh);
    };
    Powers v;
    const int* const px = (const int*)(a.x.powers + (size_t)min(m0 + tid % BM, a.M - 1) * powers);
    const int* const pw = (const int*)(a.w.powers + a.w.power_at(group, 0, 0)) + lane;
#pragma unroll
    for (int j = 0; j < 4; ++j) v.x[j] = word(px, min(d0 / 2 * kLanes + tid / BM + j * kLanes, words - 1), 1);
#pragma unroll
    for (int j = 0; j < 8; ++j) v.w[j] = word(pw, min(d0 + j, words - 1), 64);
    return v;
  };
  auto store_powers = [&](const Powers& v, int k0, int d0) {
    const int words = (min(kPowerBlocks, blocks - k0) + 3) / 4;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int d = d0 / 2 * kLanes + tid / BM + j * kLanes;
      if (d < words) xpow[tid % BM * kPowerStride + d] = v.x[j];
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (d0 + j < words) wpow[(wn * 64 + lane) * kPowerStride + d0 + j] = v.w[j];
  };
  static_assert(kLanes >= 2, "");
  auto fetch_powers = [&](int k0, int from) {
    for (int d0 = from; d0 * 4 < min(kPowerBlocks, blocks - k0); d0 += 8) store_powers(load_powers(k0, d0), k0, d0);
  };

  floatx4 acc[4][RT];
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int r = 0; r < RT; ++r) acc[c][r] = floatx4{0.f, 0.f, 0.f, 0.f};

  u32x4 w[NB][4][2];
  int ws[4];
  const Powers ahead = load_powers(0, 0);              // (the loads that follow do not wait for these to be in LDS)
  // ahead: blocks 0 and 1 of the rows, 0 of the weights; NB = 4: 0 to 2 of both
#pragma unroll
  for (int k = 0; k < (NB == 2 ? 2 : 3); ++k) {
#pragma unroll
    for (int q = 0; q < NQ; ++q) request(min(k, blocks - 1), k, q);
    if (k == 0 || NB == 4) {
#pragma unroll
      for (int c = 0; c < 8; ++c) weights(min(k, blocks - 1), w[k], c >> 1, c & 1);
    }
  }
  store_powers(ahead, 0, 0);
  fetch_powers(0, 8);

  const char* const mine = my_lds + (wm * RT * 16 + i) * kQRowBlock;
  const int* const mine_xpow = xpow + (wm * RT * 16 + i) * kPowerStride;
  const int* const mine_wpow = wpow + (wn * 64 + i) * kPowerStride;
  const int sw = swizzle(i);
  int st_next = 0;                                   // stage of the next step
  auto step = [&](auto uc, int k4) {                 // block k4 + U, k4 a multiple of 4
    constexpr int U = decltype(uc)::value, B = U & (NB - 1);
    const int st = NB == 2 ? st_next : U;
    const int kb = k4 + U, pw = (k4 & (kPowerBlocks - 1)) >> 2;
    // this block's rows and weights have landed - what may be under way is what later blocks asked for, but see above - and the stage before is free
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(NB == 2 ? NQ : 2 * (NQ + 8)) : "memory");
#pragma unroll
    for (int c = 0; c < 4; ++c) asm volatile("" : "+v"(w[B][c][0]), "+v"(w[B][c][1]));
    const int wnext = min(kb + NB - 1, blocks - 1), xnext = min(kb + (NB == 2 ? 2 : 3), blocks - 1);        // (the last block is requested again)
    const int free = NB == 2 ? (st == 0 ? 2 : st - 1) : (U + 3) & 3;
    constexpr int BF = (B + NB - 1) & (NB - 1);
    if constexpr (U == 0) {
#pragma unroll
      for (int c = 0; c < 4; ++c) ws[c] = mine_wpow[c * 16 * kPowerStride + pw];
    }
    const char* const stage = mine + st * BM * kQRowBlock;
    // requests go out between the products; what the next step waits for first: NB = 2, its weights
    auto later = [&](int r) {
      constexpr int H = RT / 2, PW = (8 + H - 1) / H, PQ = (NQ + H - 1) / H;
      const int h = r < H ? r : r - H;
      if ((r < H) == (NB == 2)) {
#pragma unroll
        for (int p = h * PW; p < min((h + 1) * PW, 8); ++p) weights(wnext, w[BF], p >> 1, p & 1);
      } else {
#pragma unroll
        for (int q = h * PQ; q < min((h + 1) * PQ, NQ); ++q) request(xnext, free, q);
      }
    };
    if constexpr (FAST) {
      // two row tiles are on their way from LDS while one is multiplied, and no more: left to itself the compiler moves the reads to where they spill (8 % of a large product)
      constexpr int NX = RT > 2 ? 3 : 2;
      struct Rows { u32x4 h[2]; } x[NX];
      int xs[NX];
      auto rows = [&](int r) {
        x[r % NX].h[0] = *(const u32x4*)(stage + r * 16 * kQRowBlock + ((2 * g) ^ sw) * 16);
        x[r % NX].h[1] = *(const u32x4*)(stage + r * 16 * kQRowBlock + ((2 * g + 1) ^ sw) * 16);
        xs[r % NX] = mine_xpow[r * 16 * kPowerStride + pw];
      };
#pragma unroll
      for (int r = 0; r < NX - 1; ++r) rows(r);
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        if (r + NX - 1 < RT) rows(r + NX - 1);
        later(r);
#pragma unroll
        for (int c = 0; c < 4; ++c)
          acc[c][r] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(__builtin_bit_cast(intx8, w[B][c]), __builtin_bit_cast(intx8, x[r % NX]), acc[c][r], 0, 0, U, ws[c], U, xs[r % NX]);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
      float wsc[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) wsc[c] = __uint_as_float(((uint32_t)ws[c] >> (8 * U) & 0xFF) << 23);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        bf16x8 wj[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) wj[c] = e4m3_to_bf16(make_uint2(w[B][c][j >> 1][2 * (j & 1)], w[B][c][j >> 1][2 * (j & 1) + 1]), wsc[c]);
        uint2 x[2];
        int xs[2];
        auto rows = [&](int r) {
          x[r & 1] = *(const uint2*)(stage + r * 16 * kQRowBlock + ((2 * g + (j >> 1)) ^ sw) * 16 + (j & 1) * 8);
          xs[r & 1] = mine_xpow[r * 16 * kPowerStride + pw];
        };
        rows(0);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          if (r + 1 < RT) rows(r + 1);
          if (j == 0) later(r);
          const bf16x8 xj = e4m3_to_bf16(x[r & 1], __uint_as_float(((uint32_t)xs[r & 1] >> (8 * U) & 0xFF) << 23));
#pragma unroll
          for (int c = 0; c < 4; ++c) acc[c][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wj[c], xj, acc[c][r], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
    if (NB == 2) st_next = st == 2 ? 0 : st + 1;
  };
  auto step_or_wait = [&](auto uc, int k4) {
    const int k = k4 + decltype(uc)::value;
    if (k < blocks) step(uc, k4);
    else if (KS > 1 && k < most) asm volatile("s_barrier" ::: "memory");        // (another share has one more)
  };
  for (int k4 = 0; k4 < most; k4 += 4) {
    if (k4 && (k4 & (kPowerBlocks - 1)) == 0) {
      asm volatile("s_barrier" ::: "memory");       // all have read the last ones: their products were waited for
      if (k4 < blocks) fetch_powers(k4, 0);
    }
    step_or_wait(std::integral_constant<int, 0>{}, k4);
    step_or_wait(std::integral_constant<int, 1>{}, k4);
    step_or_wait(std::integral_constant<int, 2>{}, k4);
    step_or_wait(std::integral_constant<int, 3>{}, k4);
  }
  // no request may be under way when LDS is used again or given back
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");

  // the shares' sums, added in their order by the first
  constexpr int kJoin = (KS - 1) * NW * 4 * RT * 1024;           // bytes
  if constexpr (KS > 1) {
    float4* const join = (float4*)lds + wave * 4 * RT * 64 + lane;
    if (share) {
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int r = 0; r < RT; ++r) join[((share - 1) * NW * 4 * RT + c * RT + r) * 64] = make_float4(acc[c][r][0], acc[c][r][1], acc[c][r][2], acc[c][r][3]);
    }
    __syncthreads();
    if (share) return;
    for (int k = 0; k < KS - 1; ++k)
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          const float4 p = join[(k * NW * 4 * RT + c * RT + r) * 64];
          acc[c][r] += floatx4{p.x, p.y, p.z, p.w};
        }
  }

  if constexpr (GATED) {
    // a wave's 32 hidden units, 8 in a row per lane; the largest of a block of 128 is that of four waves
    float* const top = (float*)lds;                  // [4][BM], then the bytes of the block: [BM][128], 16 bytes c of row r at place c ^ (r & 7)
    char* const bytes = (char*)lds + 16 * BM;
    float v[RT][8];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      float t = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[r][j] = silu(acc[2 * (j >> 2)][r][j & 3]) * acc[2 * (j >> 2) + 1][r][j & 3];
        t = fmaxf(t, finite(v[r][j]) ? fabsf(v[r][j]) : 0.f);
      }
      t = rows_max(t);
      if (g == 0) top[wn * BM + r * 16 + i] = t;
    }
    __syncthreads();
    const int out_blocks = qrows_blocks(a.w.out), out_powers = qrows_powers(a.w.out);
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const int lm = r * 16 + i, m = m0 + lm;
      const int e = e4m3_exponent(fmaxf(fmaxf(top[lm], top[BM + lm]), fmaxf(top[2 * BM + lm], top[3 * BM + lm])));
      const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[r][j] *= inv;
      *(uint2*)(bytes + lm * kQRowBlock + (((2 * wn + (g >> 1)) ^ (lm & 7)) * 16) + (g & 1) * 8) = to_e4m3x8(v[r]);
      if (m < a.M && lane < 16 && wn == 0) {
        uint8_t* p = a.y8.powers + (size_t)m * out_powers;
        p[tile_n] = (uint8_t)(e + 127);
        if (tile_n == out_blocks - 1)
          for (int b = out_blocks; b < out_powers; ++b) p[b] = 0;
      }
    }
    __syncthreads();
    // (a row's 128 bytes by neighbouring lanes; pieces of 8 bytes from where the products are would be 32 in a row: 4093 rows, 4096 -> 11008 with reading back 330 us, so 322)
    // Bytes of units behind the last one are 0, also in a row whose other units are NaN: a product with weights of 0 is NaN there (and has no part in the largest).
    const int c = tid & 7, left = a.w.out - tile_n * kQRowBlock - c * 16;
    auto keep = [&](int at) { return left >= at + 4 ? ~0u : left <= at ? 0u : ~0u >> (8 * (at + 4 - left)); };
    const uint4 mask = make_uint4(keep(0), keep(4), keep(8), keep(12));
#pragma unroll
    for (int k = 0; k < BM / 32; ++k) {
      const int lm = k * 32 + (tid >> 3);
      uint4 q = *(const uint4*)(bytes + lm * kQRowBlock + (c ^ (lm & 7)) * 16);
      q.x &= mask.x; q.y &= mask.y; q.z &= mask.z; q.w &= mask.w;
      if (m0 + lm < a.M) *(uint4*)(a.y8.values + ((size_t)(m0 + lm) * out_blocks + tile_n) * kQRowBlock + c * 16) = q;
    }
  } else {
    if (own_group >= a.w.groups) return;
    // A lane has 16 columns of a row; 64 whole ones go through LDS, so that a store writes all of a row's, not pieces of 8 or 16 bytes that lie apart (16 bytes c of row i at place c ^ i).
    // 8192 rows, 4096 -> 12288 in bf16 350 -> 331 us, 432 rows, 1280 -> 3840 8.5 -> 8.2, fp32 12.1 -> 9.2
    if (a.wide && a.w.out - own_group * 64 >= 64) {
      constexpr int kChunks = 4 * sizeof(T), kRows = 64 / kChunks;                          // of 16 bytes in a row; rows of a store
      char* const buf = (char*)lds + kJoin + wave * 16 * kChunks * 16;
      const int chunk = lane % kChunks, sub = lane / kChunks;
      T* const y = (T*)a.y + own_group * 64 + chunk * (16 / sizeof(T));
#pragma unroll
      for (int r = 0; r < RT; ++r) {
#pragma unroll
        for (int h = 0; h < kChunks / 4; ++h) {
          Bytes16 v;
          if constexpr (sizeof(T) == 4) v = __builtin_bit_cast(Bytes16, acc[h][r]);
          else v = Bytes16{pack2bf(acc[2 * h][r][0], acc[2 * h][r][1]), pack2bf(acc[2 * h][r][2], acc[2 * h][r][3]), pack2bf(acc[2 * h + 1][r][0], acc[2 * h + 1][r][1]), pack2bf(acc[2 * h + 1][r][2], acc[2 * h + 1][r][3])};
          *(Bytes16*)(buf + (i * kChunks + ((kChunks / 4 * g + h) ^ (i & (kChunks - 1)))) * 16) = v;
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int k = 0; k < 16 / kRows; ++k) {
          const int row = k * kRows + sub, m = m0 + (wm * RT + r) * 16 + row;
          const Bytes16 v = *(const Bytes16*)(buf + (row * kChunks + (chunk ^ (row & (kChunks - 1)))) * 16);
          if (m < a.M) *(Bytes16*)(y + (size_t)m * a.stride) = v;
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      }
      return;
    }
    const int col0 = a.w.column(own_group, 0, 4 * g), left = a.w.out - col0;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const int m = m0 + (wm * RT + r) * 16 + i;
      if (m >= a.M) continue;
      T* y = (T*)a.y + (size_t)m * a.stride + col0;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const float v[4] = {acc[c][r][0], acc[c][r][1], acc[c][r][2], acc[c][r][3]};
        store4(y + 4 * c, left - 4 * c, a.wide, v);
      }
    }
  }
}

template <int WM, int WN, int RT, bool FAST, bool GATED, typename T, int NB, int KS>
static void tile_t(const QProduct& a, hipStream_t s) {
  constexpr int BM = 16 * RT * WM;
  constexpr size_t lds = KS * share_lds(BM, WN, NB, KS);
  static_assert(lds >= (KS - 1) * WM * WN * 4 * RT * 1024 + (GATED ? (16 + kQRowBlock) * BM : 4096 * WM * WN) && lds <= kMostLds, "");
  const int MT = (a.M + BM - 1) / BM, NT = (a.w.groups + WN - 1) / WN;
  auto kernel = k_qlinear_tile<WM, WN, RT, FAST, GATED, T, NB, KS>;
  if (lds > 65536) allow_dynamic_lds((const void*)kernel, lds);
  hipLaunchKernelGGL(kernel, dim3((unsigned)((size_t)MT * NT)), dim3(64 * WM * WN * KS), lds, s, a, MT, NT);
}

template <bool FAST, typename T>
static void tile_least(const QProduct& a, int shares, hipStream_t s) {
  if (shares == 4) tile_t<1, 2, 2, FAST, false, T, 4, 4>(a, s);
  else if (shares == 2) tile_t<1, 2, 2, FAST, false, T, 4, 2>(a, s);
  else tile_t<1, 2, 2, FAST, false, T, 4, 1>(a, s);
}

template <bool FAST, typename T>
static void tile_by(const QProduct& a, QTile t, int shares, hipStream_t s) {
  switch (t) {
    case kTile128x256: return tile_t<1, 4, 8, FAST, false, T, 2, 1>(a, s);
    case kTile64x256: return tile_t<1, 4, 4, FAST, false, T, 4, 1>(a, s);
    case kTile64x128:
      if constexpr (FAST) {
        if (shares == 4) return tile_t<1, 2, 4, FAST, false, T, 4, 4>(a, s);
      }
      if (shares == 2) return tile_t<1, 2, 4, FAST, false, T, 4, 2>(a, s);
      return tile_t<1, 2, 4, FAST, false, T, 4, 1>(a, s);
    default: tile_least<FAST, T>(a, shares, s);
  }
}

void launch_qlinear_tile(const QProduct& a, QTile t, int shares, hipStream_t s) {
  shares = qlinear_shares(a.w, shares);                // (a share without a block would ask for one in front of the first)
  if (a.w.gated && t == kTile32x256) tile_t<1, 4, 2, false, true, float, 4, 1>(a, s);
  else if (a.w.gated && t == kTile64x256) a.fast ? tile_t<1, 4, 4, true, true, float, 4, 1>(a, s) : tile_t<1, 4, 4, false, true, float, 4, 1>(a, s);
  else if (a.w.gated) a.fast ? tile_t<1, 4, 8, true, true, float, 2, 1>(a, s) : tile_t<1, 4, 8, false, true, float, 2, 1>(a, s);
  else if (a.dtype == VVS_BF16 && !a.fast) tile_by<false, bf16_t>(a, t, shares, s);
  else if (a.dtype == VVS_BF16) tile_by<true, bf16_t>(a, t, shares, s);
  else if (a.fast) tile_by<true, float>(a, t, shares, s);
  else tile_by<false, float>(a, t, shares, s);
}

}  // namespace vvs
