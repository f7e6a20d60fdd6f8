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
  bool few;                         // k_qlinear_few: rt tiles of 16 rows, ct of 16 columns, the contraction cut into splits; else k_qlinear_tile
  int rt, ct, splits;
  QTile tile;
};
QPlan plan_qlinear_product(const QWeights& w, int M);

struct QProduct {
  QWeights w;
  int M;
  QRowsIn x;
  int dtype;                        // of y
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
void launch_qlinear_tile(const QProduct& a, QTile t, hipStream_t s);

}  // namespace vvs
