// Rows and weights in 8 bits: layout, kernel arguments and launchers.
#pragma once
#include "vvs_internal.h"

namespace vvs {

constexpr int kQRowBlock = VVS_QROWS_BLOCK;   // elements that share a power of two

__host__ __device__ constexpr int qrows_blocks(int width) { return width / kQRowBlock + (width % kQRowBlock != 0); }
__host__ __device__ constexpr int qrows_powers(int width) { return (qrows_blocks(width) + 3) & ~3; }   // bytes of a row's powers

// Rows in 8 bits as they lie in the caller's buffers (vvs.h)
struct QRowsIn { const uint8_t *values, *powers; };
struct QRowsOut { uint8_t *values, *powers; };

struct QRound {
  int M, width, dtype;
  const void* x;
  size_t stride;
  int wide;                         // 16-byte loads: pointer and stride allow them
  int packed;                       // contexts: x lies in the operand order of the projections (bf16, pack_index)
  QRowsOut y;
};

struct QNorm {
  int M, width;
  const void* x; int x_dtype; size_t x_stride;
  const void* delta; int delta_dtype; size_t delta_stride;   // delta: nullptr or added
  void* x_out; size_t x_out_stride;                          // nullptr or where x + delta goes, in x's type
  const void* gain; int gain_dtype;
  int x_wide, delta_wide, x_out_wide, gain_wide;             // 16-byte accesses
  float eps;
  double per_element;               // 1 / width
  QRowsOut y;
};

struct QRowsRead {
  int M, width, dtype;
  QRowsIn x;
  void* y;
  size_t stride;
  int wide;
};

// Weights of one linear map.  Columns are taken in groups of 64 - with a gate: 32 gate and 32 up columns - of four tiles of 16; contraction values in blocks of 128.
// Bytes lie in the operand order of the MFMAs, in which the weights are the rows: [group][block][tile t][half h][lane l = 16 g + i][16 bytes], contraction values
// 32 g + 16 h .. + 15 of the block.  Row i of tile t is column 16 (i / 4) + 4 t + i % 4 of the group, so that a lane's results of the four tiles (rows 4 g .. 4 g + 3 of
// each) are 16 columns in a row; with a gate tiles 0 and 2 are gate, 1 and 3 up, row i being hidden unit 8 (i / 4) + 4 (t / 2) + i % 4 of the group: 8 units in a row, gate
// and up in the same lane.  Powers (E + 127): [group][block / 4][tile][i][block % 4].
struct QWeights {
  int in, out, gated, blocks, groups;       // blocks: of 128 contraction values
  uint8_t *data, *powers;
  __host__ __device__ int unit() const { return gated ? 32 : 64; }                                // columns (hidden units) per group
  __host__ __device__ int column(int group, int t, int i) const { return gated ? group * 32 + 8 * (i >> 2) + 4 * (t >> 1) + (i & 3) : group * 64 + 16 * (i >> 2) + 4 * t + (i & 3); }
  __host__ __device__ size_t tile_at(int group, int block, int t) const { return (((size_t)group * blocks + block) * 4 + t) * 2048; }
  __host__ __device__ size_t power_at(int group, int block, int t) const { return (((size_t)group * ((blocks + 3) / 4) + block / 4) * 4 + t) * 64 + block % 4; }
};

constexpr size_t qweights_data_bytes(size_t groups, int blocks) { return groups * blocks * 8192; }
constexpr size_t qweights_bytes(size_t groups, int blocks) { return qweights_data_bytes(groups, blocks) + groups * ((blocks + 3) / 4) * 256; }   // powers behind the data
inline QWeights qweights(int in, int out, int gated, void* base = nullptr) {
  QWeights w{in, out, gated, qrows_blocks(in), 0, (uint8_t*)base, nullptr};
  w.groups = (out + w.unit() - 1) / w.unit();
  if (gated) w.groups = (w.groups + 3) & ~3;                   // whole blocks of 128 hidden units
  w.powers = w.data ? w.data + qweights_data_bytes(w.groups, w.blocks) : nullptr;
  return w;
}
// Workspace of a product that k_qlinear_few makes: counters, in a place of one size, so that maps can share a workspace, then for a contraction in parts their partial sums of 32 rows, with a gate the
// activations in fp32 of up to 32 rows, or of as many as have no more workgroups than kGateWorkgroups (of 32 rows x 32 packed columns).
constexpr int kGateWorkgroups = 704;
constexpr size_t kQlinearCounters = 4096;                      // bytes: a counter per 32 rows x 32 columns of up to 85 groups, or per row tile and block of 128 hidden units of up to 2048 groups
// Parts of the contraction of up to 32 rows x 32 columns: as many as give one or two workgroups to every CU
inline int qlinear_parts(const QWeights& w) { return w.gated ? 1 : w.blocks >= 40 && w.groups > 32 && w.groups <= 64 ? 2 : w.blocks >= 80 && w.groups > 74 && w.groups <= 85 ? 3 : 1; }
inline size_t qlinear_part_bytes(const QWeights& w) {
  const size_t gate = (size_t)(w.groups > kGateWorkgroups / 2 ? w.groups : kGateWorkgroups / 2) * 32 * 32, parts = qlinear_parts(w) > 1 ? (size_t)w.groups * 64 * 32 * qlinear_parts(w) : 0;
  return align_up((w.gated ? gate : parts) * sizeof(float), 256);
}

struct QLoad {
  QWeights w;
  const void *a, *b;                // [in][out]; b: up weights
  int dtype;
};

struct QWeightsRead {
  QWeights w;
  void *a, *b;
  int dtype;
};

// Which kernel makes a product
enum QTile { kTile128x256, kTile64x256, kTile64x128, kTile32x128, kTile32x256 };   // rows x packed columns of a workgroup
struct QPlan {
  bool few;                         // k_qlinear_few: rt tiles of 16 rows, ct of 16 columns, the contraction cut into splits; else k_qlinear_tile, whose workgroups cut it into splits
  int rt, ct, splits;
  QTile tile;
};
QPlan plan_qlinear_product(const QWeights& w, int M, bool fast);   // fast: see QProduct (gated: the same choice for both)

// Shares of the contraction that a workgroup of k_qlinear_tile has waves for: 1, 2 or 4, and each at least a block
inline int qlinear_shares(const QWeights& w, int wanted) { return wanted >= 4 && w.blocks >= 4 ? 4 : wanted >= 2 && w.blocks >= 2 ? 2 : 1; }

// Whether a product may take the matrix instructions for e4m3 (outputs of type `dtype`, or of a context of it; in 8 bits: as VVS_BF16)
inline int qlinear_fast(int products, int dtype, int M) { return M > 64 && (products == VVS_PRODUCTS_E4M3 || (products == VVS_PRODUCTS_AUTO && dtype == VVS_BF16)); }

struct QProduct {
  QWeights w;
  int M;
  QRowsIn x;
  int dtype;                        // of y
  int fast;                         // e4m3 products (k_qlinear_tile; gated tiles of 32 rows: exact ones all the same)
  void* y;                          // !gated
  size_t stride;
  int wide;                         // stores of 4 elements at once
  float* act;                       // workspace: gated, [M][groups * 32]; else partial sums
  uint32_t* counters;               // workspace: zero between calls
  QRowsOut y8;                      // gated
};

void launch_qrows_round(const QRound& a, hipStream_t s);
void launch_qrows_norm(const QNorm& a, hipStream_t s);
void launch_qrows_read(const QRowsRead& a, hipStream_t s);
void launch_qlinear_load(const QLoad& a, hipStream_t s);
void launch_qlinear_read(const QWeightsRead& a, hipStream_t s);
void launch_qlinear_product(const QProduct& a, const QPlan& p, hipStream_t s);
void launch_qlinear_tile(const QProduct& a, QTile t, int shares, hipStream_t s);

// Contexts with their weights in 8 bits (vvs_qlinear_ctx.hip): a layer's maps, in the order of its projections
enum QMap { kMapQkv, kMapO, kMapGate, kMapDown };
inline QWeights context_map(const Ctx* c, QMap m, void* base = nullptr) {
  return m == kMapQkv ? qweights(c->d, 3 * c->d, 0, base) : m == kMapO ? qweights(c->d, c->d, 0, base) : m == kMapGate ? qweights(c->d, c->F, 1, base) : qweights(c->F, c->d, 0, base);
}
void launch_context_load(Ctx* c, int layer, const void* const* tensors, hipStream_t s);          // the layer's tensors in canonical order
void launch_context_norm(Ctx* c, int M, const float* gain, const float* delta, hipStream_t s);   // x (+ delta) -> rows in 8 bits
void launch_context_round(Ctx* c, int M, hipStream_t s);                                         // the attention's output -> rows in 8 bits
void launch_context_product(Ctx* c, int layer, QMap m, int M, float* out, hipStream_t s);        // kMapGate: into the rows of hidden units

}  // namespace vvs
