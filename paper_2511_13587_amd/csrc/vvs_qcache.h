// Key/value cache in 8 bits: layout, kernel arguments and launchers.
#pragma once
#include "vvs_internal.h"

namespace vvs {

constexpr int kQBlock = VVS_QCACHE_BLOCK;   // slots that share a power of two
constexpr int kQLeast = -110;               // smallest exponent of a block
constexpr int kQParts = 4096;               // partial results of a split attention call that the workspace has room for, of 16 queries each: 512 workgroups of 128 queries, two per
                                            // CU (us with room for 256 / 512 / 1024: 1 row x 32 heads x 512 tokens over 4096 slots 116 / 93 / 105, 4 rows x 256 over 2048 107 / 92 / 108)
constexpr int kQKept = 8;                   // queries per row and key/value head whose scores are kept for the counted weights

// One cache (all layers).  A region is what one (layer, row, key/value head) holds: blocks of 32 slots, each 32 * head_size bytes of keys and
// then as many of values; behind all regions, in the same order, two floats per block: 2^E of its keys and of its values.
//
// Bytes lie in the operand order of the attention's 16x16x32 MFMAs (lane l = 16 g + i), 16 bytes per lane and load:
//   keys (S^T = K Q^T, contraction over dims): [32 dims kd][lane][tile t][dim % 8] with g = dim % 32 / 8; slot w of the block is row i = 4 (w / 8) + w % 4 of
//     tile t = w / 4 % 2, so that a lane's eight scores of both tiles are those of slots 8 g .. 8 g + 7;
//   values (O^T = V^T P^T, contraction over slots): [32 dims][lane][dim % 32 / 16][w % 8] with g = w / 8, i = dim % 16.
struct QLayout {
  int rows, heads, kv_heads, dh, blocks;    // blocks: per region
  uint8_t* data;
  float2* scale;
  __host__ __device__ size_t region(int layer, int row, int head) const { return ((size_t)layer * rows + row) * kv_heads + head; }
  __host__ __device__ size_t block_bytes() const { return (size_t)2 * kQBlock * dh; }
};

// Cached length of row r: len[r >> shift] (a context keeps one per prompt, for two rows), or `fixed` for every row where len is nullptr
struct QLen {
  const int32_t* len;
  int shift, fixed;
};
constexpr size_t qcache_parts_bytes(int dh) { return (size_t)kQParts * 16 * (dh + 2) * sizeof(float); }
constexpr int qcache_score_steps(int blocks, int max_tokens) { return blocks + (max_tokens + kQBlock - 1) / kQBlock; }

struct QAttention {
  QLayout c;
  QLen len;
  int layer, T, group;              // T: block tokens per row; group: query heads per key/value head
  const int32_t* n_tokens;          // [rows] or nullptr
  const void *q, *k, *v;            // k, v: nullptr = the queries see the cache alone
  size_t q_stride, k_stride, v_stride;      // elements between tokens; rows are T tokens apart
  float c_exp;                      // scale * log2(e)
  void* out;
  float* lse;                       // [rows][T][heads] or nullptr
  float* norm;                      // workspace, likewise, in units of log2, or nullptr: nothing is counted
  int n_counted;
  float *mass, *block_mass;         // [rows][kv_heads][capacity], [rows][kv_heads][block_stride]
  int block_stride;
  int capacity;
  int packed;                       // 1: out in the operand order of the projections
  float* parts;                     // partial results: o, then (m, l)
  float* scores;                    // workspace: kept scores of one layer, [rows][kv_heads][score_steps][n_kept][32]
  int score_steps, n_kept;          // (n_kept: the launcher's choice)
  int splits;
  int causal;
  uint64_t anc[VVS_MAX_T];          // !causal: bit j = token sees block token j
};

struct QAppend {
  QLayout c;
  QLen len;
  int layer, n_layers, n, src_tokens;    // n: most tokens taken of a row; src_tokens: tokens per row in k and v
  const int32_t* n_tokens;               // [rows] or nullptr
  const int32_t* select;                 // [rows][select_stride] or nullptr
  int select_stride, select_shift;
  const int32_t* skip;                   // [rows >> len.shift] or nullptr: rows with a negative entry take nothing
  int count_plus;                        // n_tokens[r >> shift] + count_plus tokens are taken
  int n_shift;
  const void *k, *v;
  size_t stride[2], layer_stride[2];     // elements between tokens, between layers: of k, of v
  int capacity;
  float* mass;                           // contexts, or nullptr: weights of the new slots begin at 0 ...
  int32_t* pos;                          // ... and their positions at pos_base[r >> len.shift] + pos_add (pos_base nullptr: a slot's number); [layers][rows][kv_heads][capacity]
  const int32_t* pos_base;
  int pos_add;
};

struct QEvict {
  QLayout c;
  QLen len;
  int layer, n_layers, keep, recent, capacity;
  const float* mass;
  float* mass_out;
  const int32_t* pos;
  int32_t* pos_out;
  int32_t* origin;                  // workspace: [layers of the call][rows][kv_heads][blocks * 32]
};

struct QRead {
  QLayout c;
  QLen len;
  int layer, n_layers, n, capacity;
  const int32_t* first;             // [rows] or nullptr
  void *k, *v;
};

struct RopeArgs {
  const float* sums;                // contexts: queries, keys and values as `splits` partial sums of a projection, rows of (heads + 2 kv_heads) * dh, instead of q and k ...
  int splits;
  size_t split_stride;
  void* v_out;                      // ... and where the values go (nullptr: no sums)
  const int32_t* pos;
  const void *q, *k;
  void *q_out, *k_out;
  size_t q_stride, k_stride, q_out_stride, k_out_stride;
  int M, heads, kv_heads, dh, axes, pairs, halves, inverse;
  double turns[128];                // turns per position of each pair
  uint8_t axis[128];
};

void launch_qcache_attention(const QAttention& a, int dtype, hipStream_t s);
void launch_qcache_append(const QAppend& a, int dtype, hipStream_t s);
void launch_qcache_evict(const QEvict& a, hipStream_t s);
void launch_qcache_read(const QRead& a, int dtype, hipStream_t s);
void launch_rope_axes(const RopeArgs& a, int dtype, hipStream_t s);

// Contexts with VVS_CACHE_E4M3 (vvs_qcache_ctx.hip)
void launch_context_positions(Ctx* c, const TreeDesc& tree, const PosDesc& pos, int T, hipStream_t s);
void launch_context_rope(Ctx* c, int layer, int M, const float* sums, int splits, hipStream_t s);
void launch_context_attention(Ctx* c, int layer, const TreeDesc& tree, const PosDesc& pos, int T, hipStream_t s);
void launch_context_append(Ctx* c, hipStream_t s);
void launch_context_read(Ctx* c, int layer, int row, int n_slots, float* dk, float* dv, hipStream_t s);

}  // namespace vvs
