// Host side of the rows and weights in 8 bits: argument checks, buffer sizes, entry points.
#include "vvs_qlinear.h"

#include <algorithm>
#include <cmath>
#include <new>

namespace vvs {

struct QLinear {
  vvs_qlinear_config cfg;
  QWeights w;
  size_t weight_bytes, ws_bytes;
  int dev;
  char* ws;
  bool loaded;
  std::string err;
};

// What vvs_last_error(NULL) tells of a failed create or query (vvs_host.cpp)
vvs_status fail_without_context(vvs_status st, const char* msg);

// The calls on rows have no object to keep a message in: one per thread
static thread_local const char* t_rows_error = "";

static vvs_status rows_no(vvs_status st, const char* msg) {
  t_rows_error = msg;
  return st;
}

static vvs_status rows_launched() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? VVS_OK : rows_no(VVS_EHIP, hipGetErrorString(e));
}

static vvs_status no(QLinear* l, vvs_status st, const char* msg) {
  if (!l) return fail_without_context(st, msg);
  l->err = msg;
  return st;
}

static bool known(int dtype) { return dtype == VVS_FP32 || dtype == VVS_BF16; }
static size_t size_of(int dtype) { return dtype == VVS_BF16 ? 2 : 4; }

// Widths and strides of a tensor [n_rows, width]: elements from row to row, 0 where they follow each other; < 0: not allowed
static int64_t stride_of(int64_t given, int width) {
  const int64_t s = given ? given : width;
  return s < width || s > ((int64_t)1 << 31) ? -1 : s;
}
// 16-byte accesses of 8 elements (by: 4, accesses of 4 elements)
static int wide_rows(const void* p, int64_t stride, int dtype, int by = 8) {
  const size_t bytes = by * size_of(dtype) < 16 ? by * size_of(dtype) : 16;
  return ((uintptr_t)p | (uintptr_t)stride * size_of(dtype)) % bytes == 0;
}
static bool off_element(const void* p, int dtype) { return (uintptr_t)p % size_of(dtype) != 0; }
static bool off16(const void* p) { return ((uintptr_t)p & 15) != 0; }

// Rows of `width` bytes, `stride` bytes apart.  Two such tensors share memory unless one lies behind the other or, with the same stride, each row beside the other's
struct Span { uintptr_t at; uint64_t width, stride; int64_t rows; };
static Span span_of(const void* p, int64_t rows, int64_t width, int64_t stride, size_t size) { return Span{(uintptr_t)p, (uint64_t)width * size, (uint64_t)stride * size, rows}; }
static bool share(const Span& a, const Span& b) {
  if (!a.at || !b.at) return false;
  if (a.at + (uint64_t)(a.rows - 1) * a.stride + a.width <= b.at || b.at + (uint64_t)(b.rows - 1) * b.stride + b.width <= a.at) return false;
  if (a.stride != b.stride) return true;
  const uint64_t d = b.at >= a.at ? (b.at - a.at) % a.stride : (a.stride - (a.at - b.at) % a.stride) % a.stride;
  return d < a.width || d + b.width > a.stride;
}
static Span values_span(const void* p, int64_t rows, int width) { const int64_t w = (int64_t)qrows_blocks(width) * kQRowBlock; return span_of(p, rows, w, w, 1); }
static Span powers_span(const void* p, int64_t rows, int width) { const int64_t w = qrows_powers(width); return span_of(p, rows, w, w, 1); }
template <size_t N, size_t K>
static bool share_any(const Span (&outs)[N], const Span (&ins)[K]) {
  for (size_t i = 0; i < N; ++i) {
    for (size_t j = i + 1; j < N; ++j)
      if (share(outs[i], outs[j])) return true;
    for (const Span& b : ins)
      if (share(outs[i], b)) return true;
  }
  return false;
}

constexpr int kWidest = 65536;                                 // of a row that a workgroup keeps in registers
constexpr int64_t kMostThreads = ((int64_t)1 << 32) - 1024;    // of a launch along a dimension

static vvs_status check_rows(int n_rows, int width, const void* values, const void* powers, int threads_per_row) {
  if (n_rows < 1 || width < 1) return rows_no(VVS_EINVAL, "qrows: n_rows and width must be positive");
  if (width > kWidest) return rows_no(VVS_ESIZE, "qrows: at most 65536 elements per row");
  if (!values || !powers) return rows_no(VVS_EINVAL, "qrows: NULL argument");
  if (off16(values) || off16(powers)) return rows_no(VVS_EINVAL, "qrows: values and powers must be 16-byte aligned");
  if ((int64_t)n_rows * threads_per_row > kMostThreads) return rows_no(VVS_ESIZE, "qrows: more rows than a launch holds");
  return VVS_OK;
}

// Which kernel makes a product.  Few rows are bound by the weights' bytes, which every wave streams for itself, and by how many waves there are to do so; more rows share the weights, and themselves pass
// through LDS.  The rule goes by the number of workgroups - the smallest tiles that fit the 256 CUs once, twice or three times, then larger ones - and by the length of the contraction in blocks of 128: where
// tiles are few and it is long, several workgroups (parts) or a workgroup's waves (shares) divide it.  It is 0.5 % behind the best of all variants in the mean over some 900 sizes, 8 to 4000 rows, and 15 %
// at one.  Each border was taken where the kernels, as they are, cross; us per call in a graph, weights rotating through 400 MB, outputs in bf16: as chosen / the next variant.
//   k_qlinear_few
//     16 x 16   up to 256 workgroups                                  28 rows, 4096 -> 2048 6.0 / 32 x 16 7.7
//     16 x 32   up to 16 rows; up to 256 workgroups                   8 rows, 4096 -> 12288 13.3 / 16 x 16 13.6; 64 rows, 4096 -> 2048 7.2 / 32 x 32 8.6
//               up to 768 (640 for 64 rows) and 16 blocks             256 rows, 1280 -> 1280 5.8 / 32 x 64 6.4
//               up to 1152 and 12 blocks, whole products              128 rows, 1536 -> 4608 in fp32 9.4 / tiles 10.6
//     32 x 32   one row tile in two or three parts (qlinear_parts)    28 rows, 11008 -> 4096 15.0 / whole 19.5, 11008 -> 5000 18.0 / whole 20.5
//               up to 256 workgroups; up to 32 rows                   128 rows, 4096 -> 2048 8.6 / 32 x 64 10.0
//               up to 64 rows, 512 workgroups, 23 blocks              40 rows, 2560 -> 6912 8.8 / 32 x 64 10.3
//     32 x 64   up to 256, from 24 blocks, over 64 rows from 10       128 rows, 4096 -> 4096 10.3 / tiles in four shares 11.5
//   k_qlinear_tile, e4m3 products
//     64 x 128  all workgroups on the card at once, three per CU      432 rows, 4096 -> 12288 38.3 / 128 x 256 40.2
//     128 x 256 from 208 workgroups on                                600 rows, 4096 -> 16384 54.3 / 64 x 256 66.5
//     32 x 128  up to 256; in four shares from 24 blocks, two from 16 432 rows, 1280 -> 1280 6.5 / 64 x 128 7.6; 3456 -> 1280 10.9 / one share 12.3; 2048 -> 2048 8.4 / 9.0
//     64 x 128  up to 256, four shares from 40 blocks                 432 rows, 11008 -> 4096 39.5 / two shares 44.3
//     64 x 256  from 150, up to 32 blocks                             600 rows, 1536 -> 4608 10.7 / 64 x 128 11.4
//     64 x 128  up to 512, two shares from 16 blocks; whole from 144  432 rows, 4096 -> 4096 15.8 / one share 17.7; 512 rows, 768 -> 2304 6.4 / 32 x 128 6.9
//   k_qlinear_tile, whole products (twice the instructions, more for smaller tiles to hide)
//     32 x 128  up to 1024 workgroups                                 600 rows, 1280 -> 3840 18.3 / 64 x 256 21.7
//               up to 256: four shares from 24 blocks, two from 8     432 rows, 3456 -> 1280 15.1 / two shares 16.4; 1280 -> 1280 9.8 / one share 11.0
//               up to 512 in two shares                               432 rows, 4096 -> 4096 26.0 / one share 35.6
//     64 x 128  beyond, two shares from 32 blocks                     432 rows, 8192 -> 8192 66.9 / 32 x 128 77.5
//   with a gate (columns counted twice; not in shares: 48 rows, 4096 -> 11008 33.5 / 34.4)
//     16 x 32   up to 16 rows; up to 768 workgroups                   48 rows, 768 -> 2048 8.0 / 32 x 32 8.5
//     32 x 32   up to 32 rows                                         28 rows, 4096 -> 11008 26.0 / 16 x 32 32.1
//               up to 704: up to 64 rows, or from 16 blocks           64 rows, 2048 -> 5632 15.5 / tiles 18.6; 128 rows, 4096 -> 2048 16.7 / tiles 21.6
//     32 x 256  up to 64 rows                                         64 rows, 4096 -> 11008 35.2 / 32 x 32 41.9
//               one or two blocks, over 64 rows up to four            128 rows, 512 -> 1408 7.5 / 16 x 32 8.3
//     128 x 256 from 208 on, else 64 x 256                            432 rows, 4096 -> 11008 55.5 / 64 x 256 64.9; 128 rows 34.6 / 128 x 256 45.7
QPlan plan_qlinear_product(const QWeights& w, int M, bool fast) {
  auto few = [&](int rt, int ct) { return (int64_t)((M + 16 * rt - 1) / (16 * rt)) * w.groups * (4 / ct); };
  auto tiles = [&](int rows, int groups) { return (int64_t)((M + rows - 1) / rows) * ((w.groups + groups - 1) / groups); };
  auto small = [](int rt, int ct, int splits = 1) { return QPlan{true, rt, ct, splits, kTile32x128}; };
  auto large = [&](QTile t, int shares = 1) { return QPlan{false, 2, 2, qlinear_shares(w, shares), t}; };
  if (w.gated) {
    if (M > 32 && w.blocks <= (M > 64 ? 4 : 2) && tiles(32, 4) <= 256) return large(kTile32x256);
    if (M <= 16 || few(1, 2) <= 768) return small(1, 2);
    if (M <= 32 || (few(2, 2) <= kGateWorkgroups && (M <= 64 || w.blocks >= 16))) return small(2, 2);
    return large(M <= 64 ? kTile32x256 : tiles(128, 4) >= 208 ? kTile128x256 : kTile64x256);
  }
  if (few(1, 1) <= 256) return small(1, 1);
  const int parts = M <= 32 ? qlinear_parts(w) : 1;
  if (parts == 3 || (parts == 2 && M > 16)) return small(2, 2, parts);
  if (M <= 16 || few(1, 2) <= 256) return small(1, 2);
  if (w.blocks <= 16 && few(1, 2) <= (M <= 64 ? 640 : 768)) return small(1, 2);
  if (w.blocks <= 12 && few(1, 2) <= 1152 && M > 64 && !fast) return small(1, 2);
  if (few(2, 2) <= 256) return small(2, 2);
  if (few(2, 4) <= 256 && w.blocks >= (M <= 64 ? 24 : 10)) return small(2, 4);
  if (M <= 64 && few(2, 2) <= 512 && w.blocks < 24) return small(2, 2);
  if (M <= 32) return small(2, 2);
  const int64_t least = tiles(32, 2), middle = tiles(64, 2);
  if (!fast && (least <= 1024 || M <= 64)) {
    if (least <= 256) return large(kTile32x128, w.blocks >= 24 ? 4 : w.blocks >= 8 ? 2 : 1);
    if (least <= 512) return large(kTile32x128, 2);
    return w.blocks >= 32 && middle <= 512 && M > 64 ? large(kTile64x128, 2) : large(kTile32x128);
  }
  if (middle > 512 && middle <= 768) return large(kTile64x128);
  if (tiles(128, 4) >= 208) return large(kTile128x256);
  if (least <= 256) return large(kTile32x128, w.blocks >= 24 ? 4 : w.blocks >= 16 ? 2 : 1);
  if (middle <= 256 && w.blocks >= 40) return large(kTile64x128, 4);
  if (tiles(64, 4) >= 150 && (w.blocks <= 32 || middle > 512)) return large(kTile64x256);
  if (middle <= 512 && w.blocks >= 16) return large(kTile64x128, 2);
  return large(middle >= 144 ? kTile64x128 : kTile32x128);
}

static vvs_status plan_qlinear(const vvs_qlinear_config* cfg, QLinear* l) {
  if (!cfg) return no(nullptr, VVS_EINVAL, "qlinear config is NULL");
  const vvs_qlinear_config& g = *cfg;
  if (g.in < 1 || g.out < 1 || g.max_rows < 1) return no(nullptr, VVS_EINVAL, "qlinear config: a dimension is not positive");
  if (!known(g.dtype)) return no(nullptr, VVS_EINVAL, "qlinear config: unknown dtype");
  if (g.products != VVS_PRODUCTS_AUTO && g.products != VVS_PRODUCTS_WHOLE && g.products != VVS_PRODUCTS_E4M3) return no(nullptr, VVS_EINVAL, "qlinear config: unknown products");
  if (g.gated != 0 && g.gated != 1) return no(nullptr, VVS_EINVAL, "qlinear config: gated must be 0 or 1");
  if (g.in > kWidest || (g.gated && g.out > kWidest)) return no(nullptr, VVS_ESIZE, "qlinear config: at most 65536 elements per row");
  if (g.out > (1 << 24) || g.max_rows > (1 << 20)) return no(nullptr, VVS_ESIZE, "qlinear config: at most 2^24 columns and 2^20 rows");
  l->cfg = g;
  QWeights& w = l->w;
  w = qweights(g.in, g.out, g.gated);
  // (a launch of the smallest tiles, a wave per 64 columns and 32 rows)
  if ((int64_t)w.groups * ((g.max_rows + 31) / 32 + 1) * 64 > kMostThreads) return no(nullptr, VVS_ESIZE, "qlinear config: more outputs than a launch holds");
  if ((int64_t)w.groups * w.blocks >= (1 << 24)) return no(nullptr, VVS_ESIZE, "qlinear config: more weights than a launch holds");
  l->weight_bytes = align_up(qweights_bytes(w.groups, w.blocks), 256);
  l->ws_bytes = kQlinearCounters + qlinear_part_bytes(w);
  return VVS_OK;
}

static QLinear* of(vvs_qlinear* l) { return reinterpret_cast<QLinear*>(l); }

static vvs_status check_device(QLinear* l) {
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) return no(l, VVS_EHIP, "qlinear: no current device");
  if (dev != l->dev) return no(l, VVS_EINVAL, "qlinear: created on another device than the current one");
  return VVS_OK;
}

static vvs_status launched(QLinear* l, const char* what) {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return VVS_OK;
  l->err = std::string(what) + ": " + hipGetErrorString(e);
  return VVS_EHIP;
}

// A map's own buffers, and a weight tensor of its config
static Span bytes_span(const void* p, size_t bytes) { return Span{(uintptr_t)p, bytes, bytes, 1}; }
static Span held_span(const QLinear* l) { return bytes_span(l->w.data, l->weight_bytes); }
static Span workspace_span(const QLinear* l) { return bytes_span(l->ws, l->ws_bytes); }
static Span tensor_span(const QLinear* l, const void* p) { return bytes_span(p, (size_t)l->cfg.in * l->cfg.out * size_of(l->cfg.dtype)); }

static vvs_status check_product(QLinear* l, int n_rows, const void* values, const void* powers) {
  if (!l->loaded) return no(l, VVS_ESTATE, "qlinear: call vvs_qlinear_load first");
  if (!values || !powers) return no(l, VVS_EINVAL, "qlinear: NULL argument");
  if (n_rows < 1) return no(l, VVS_EINVAL, "qlinear: n_rows must be positive");
  if (n_rows > l->cfg.max_rows) return no(l, VVS_ESIZE, "qlinear: n_rows exceeds max_rows");
  if (off16(values) || off16(powers)) return no(l, VVS_EINVAL, "qlinear: values and powers must be 16-byte aligned");
  const Span ws[] = {workspace_span(l)}, rows[] = {values_span(values, n_rows, l->cfg.in), powers_span(powers, n_rows, l->cfg.in)};
  if (share_any(ws, rows)) return no(l, VVS_EINVAL, "qlinear: the workspace shares memory with the rows");
  return VVS_OK;
}

}  // namespace vvs

using namespace vvs;

extern "C" {

const char* vvs_qrows_last_error(void) { return t_rows_error; }

vvs_status vvs_qrows_sizes(int32_t width, int32_t n_rows, size_t* value_bytes, size_t* power_bytes) {
  if (n_rows < 1 || width < 1) return rows_no(VVS_EINVAL, "qrows: n_rows and width must be positive");
  if (width > kWidest) return rows_no(VVS_ESIZE, "qrows: at most 65536 elements per row");
  if (value_bytes) *value_bytes = (size_t)n_rows * qrows_blocks(width) * kQRowBlock;
  if (power_bytes) *power_bytes = (size_t)n_rows * qrows_powers(width);
  return VVS_OK;
}

vvs_status vvs_qrows_round(int32_t n_rows, int32_t width, int32_t dtype, const void* d_x, int64_t x_stride, void* d_values, void* d_powers, vvs_stream s) {
  const vvs_status st = check_rows(n_rows, width, d_values, d_powers, width > 0 && width <= kWidest ? 16 * qrows_powers(width) : 16);
  if (st != VVS_OK) return st;
  if (!d_x) return rows_no(VVS_EINVAL, "qrows round: NULL argument");
  if (!known(dtype)) return rows_no(VVS_EINVAL, "qrows round: unknown dtype");
  const int64_t xs = stride_of(x_stride, width);
  if (xs < 0 || off_element(d_x, dtype)) return rows_no(VVS_EINVAL, "qrows round: the stride has to cover a row, the pointer to be aligned to an element");
  const Span outs[] = {values_span(d_values, n_rows, width), powers_span(d_powers, n_rows, width)}, ins[] = {span_of(d_x, n_rows, width, xs, size_of(dtype))};
  if (share_any(outs, ins)) return rows_no(VVS_EINVAL, "qrows round: an output shares memory with the input or with the other");
  QRound a{};
  a.M = n_rows; a.width = width; a.dtype = dtype;
  a.x = d_x; a.stride = (size_t)xs; a.wide = wide_rows(d_x, xs, dtype);
  a.y = QRowsOut{(uint8_t*)d_values, (uint8_t*)d_powers};
  launch_qrows_round(a, (hipStream_t)s);
  return rows_launched();
}

vvs_status vvs_qrows_norm(int32_t n_rows, int32_t width, int32_t x_dtype, const void* d_x, int64_t x_stride, int32_t delta_dtype, const void* d_delta,
                          int64_t delta_stride, void* d_x_out, int64_t x_out_stride, int32_t gain_dtype, const void* d_gain, float eps, void* d_values,
                          void* d_powers, vvs_stream s) {
  const vvs_status st = check_rows(n_rows, width, d_values, d_powers, width > 0 ? std::min(1024, 16 * qrows_powers(std::min(width, kWidest))) : 1024);
  if (st != VVS_OK) return st;
  if (!d_x || !d_gain) return rows_no(VVS_EINVAL, "qrows norm: NULL argument");
  if (!known(x_dtype) || !known(gain_dtype) || (d_delta && !known(delta_dtype))) return rows_no(VVS_EINVAL, "qrows norm: unknown dtype");
  if (!(eps >= 0.f) || !std::isfinite(eps)) return rows_no(VVS_EINVAL, "qrows norm: eps must be finite and not negative");
  const int64_t xs = stride_of(x_stride, width), ds = stride_of(delta_stride, width), os = stride_of(x_out_stride, width);
  if (xs < 0 || (d_delta && ds < 0) || (d_x_out && os < 0) || off_element(d_x, x_dtype) || off_element(d_x_out, x_dtype) || off_element(d_gain, gain_dtype) ||
      (d_delta && off_element(d_delta, delta_dtype)))
    return rows_no(VVS_EINVAL, "qrows norm: strides have to cover a row, pointers to be aligned to an element");
  if (d_x == d_x_out && xs != os) return rows_no(VVS_EINVAL, "qrows norm: in place, both strides are the same");
  Span x = span_of(d_x, n_rows, width, xs, size_of(x_dtype));
  const Span out = span_of(d_x_out, n_rows, width, os, size_of(x_dtype)), outs[] = {values_span(d_values, n_rows, width), powers_span(d_powers, n_rows, width), out};
  if (d_x == d_x_out) x.at = 0;                                // (in place; as an output it is compared with the others)
  const Span ins[] = {x, span_of(d_delta, n_rows, width, ds, d_delta ? size_of(delta_dtype) : 4), span_of(d_gain, 1, width, width, size_of(gain_dtype))};
  if (share_any(outs, ins)) return rows_no(VVS_EINVAL, "qrows norm: an output shares memory with an input or with another output");
  QNorm a{};
  a.M = n_rows; a.width = width;
  a.x = d_x; a.x_dtype = x_dtype; a.x_stride = (size_t)xs; a.x_wide = wide_rows(d_x, xs, x_dtype);
  if (d_delta) { a.delta = d_delta; a.delta_dtype = delta_dtype; a.delta_stride = (size_t)ds; a.delta_wide = wide_rows(d_delta, ds, delta_dtype); }
  if (d_x_out) { a.x_out = d_x_out; a.x_out_stride = (size_t)os; a.x_out_wide = wide_rows(d_x_out, os, x_dtype); }
  a.gain = d_gain; a.gain_dtype = gain_dtype; a.gain_wide = wide_rows(d_gain, 0, gain_dtype);
  a.eps = eps; a.per_element = 1.0 / width;
  a.y = QRowsOut{(uint8_t*)d_values, (uint8_t*)d_powers};
  launch_qrows_norm(a, (hipStream_t)s);
  return rows_launched();
}

vvs_status vvs_qrows_read(int32_t n_rows, int32_t width, const void* d_values, const void* d_powers, int32_t dtype, void* d_out, int64_t out_stride, vvs_stream s) {
  const vvs_status st = check_rows(n_rows, width, d_values, d_powers, width > 0 && width <= kWidest ? 16 * qrows_powers(width) : 16);
  if (st != VVS_OK) return st;
  if (!d_out) return rows_no(VVS_EINVAL, "qrows read: NULL argument");
  if (!known(dtype)) return rows_no(VVS_EINVAL, "qrows read: unknown dtype");
  const int64_t os = stride_of(out_stride, width);
  if (os < 0 || off_element(d_out, dtype)) return rows_no(VVS_EINVAL, "qrows read: the stride has to cover a row, the pointer to be aligned to an element");
  const Span outs[] = {span_of(d_out, n_rows, width, os, size_of(dtype))}, ins[] = {values_span(d_values, n_rows, width), powers_span(d_powers, n_rows, width)};
  if (share_any(outs, ins)) return rows_no(VVS_EINVAL, "qrows read: the output shares memory with the rows");
  QRowsRead a{};
  a.M = n_rows; a.width = width; a.dtype = dtype;
  a.x = QRowsIn{(const uint8_t*)d_values, (const uint8_t*)d_powers};
  a.y = d_out; a.stride = (size_t)os; a.wide = wide_rows(d_out, os, dtype);
  launch_qrows_read(a, (hipStream_t)s);
  return rows_launched();
}

vvs_status vvs_qlinear_query_sizes(const vvs_qlinear_config* cfg, size_t* weight_bytes, size_t* workspace_bytes) {
  QLinear l{};
  const vvs_status st = plan_qlinear(cfg, &l);
  if (st != VVS_OK) return st;
  if (weight_bytes) *weight_bytes = l.weight_bytes;
  if (workspace_bytes) *workspace_bytes = l.ws_bytes;
  return VVS_OK;
}

vvs_status vvs_qlinear_create(const vvs_qlinear_config* cfg, void* d_weights, void* d_workspace, vvs_qlinear** out) {
  if (!out) return no(nullptr, VVS_EINVAL, "qlinear create: out is NULL");
  *out = nullptr;
  if (!d_weights || !d_workspace) return no(nullptr, VVS_EINVAL, "qlinear create: NULL device buffer");
  if (((uintptr_t)d_weights | (uintptr_t)d_workspace) & 255) return no(nullptr, VVS_EINVAL, "qlinear create: device buffers must be 256-byte aligned");
  QLinear plan{};
  const vvs_status st = plan_qlinear(cfg, &plan);
  if (st != VVS_OK) return st;
  if (share(bytes_span(d_weights, plan.weight_bytes), bytes_span(d_workspace, plan.ws_bytes))) return no(nullptr, VVS_EINVAL, "qlinear create: the workspace shares memory with the weights");
  int ndev = 0;
  if (hipGetDeviceCount(&ndev) != hipSuccess || ndev < 1) return no(nullptr, VVS_EHIP, "qlinear create: no HIP device (this library has no CPU path)");
  hipError_t e = hipGetDevice(&plan.dev);
  if (e != hipSuccess) return no(nullptr, VVS_EHIP, hipGetErrorString(e));
  plan.ws = (char*)d_workspace;
  plan.w = qweights(plan.cfg.in, plan.cfg.out, plan.cfg.gated, d_weights);
  QLinear* l = new (std::nothrow) QLinear(plan);
  if (!l) return no(nullptr, VVS_EHIP, "qlinear create: out of memory");
  launch_fill_zero(d_workspace, l->ws_bytes, nullptr);
  e = hipGetLastError();
  if (e == hipSuccess) e = hipDeviceSynchronize();
  if (e != hipSuccess) { delete l; return no(nullptr, VVS_EHIP, hipGetErrorString(e)); }
  *out = reinterpret_cast<vvs_qlinear*>(l);
  return VVS_OK;
}

void vvs_qlinear_destroy(vvs_qlinear* l) { delete of(l); }

const char* vvs_qlinear_last_error(const vvs_qlinear* l) { return l ? reinterpret_cast<const QLinear*>(l)->err.c_str() : ""; }

vvs_status vvs_qlinear_load(vvs_qlinear* ql, const void* d_w, const void* d_w_up, vvs_stream s) {
  QLinear* l = of(ql);
  if (!l) return VVS_EINVAL;
  if (!d_w || !d_w_up != !l->cfg.gated) return no(l, VVS_EINVAL, "qlinear load: one weight tensor, with a gate two");
  if (off_element(d_w, l->cfg.dtype) || off_element(d_w_up, l->cfg.dtype)) return no(l, VVS_EINVAL, "qlinear load: unaligned weights");
  if (share(held_span(l), tensor_span(l, d_w)) || share(held_span(l), tensor_span(l, d_w_up))) return no(l, VVS_EINVAL, "qlinear load: a weight tensor shares memory with the map's buffer");
  vvs_status st = check_device(l);
  if (st != VVS_OK) return st;
  launch_qlinear_load(QLoad{l->w, d_w, d_w_up, l->cfg.dtype}, (hipStream_t)s);
  if ((st = launched(l, "qlinear load")) == VVS_OK) l->loaded = true;
  return st;
}

vvs_status vvs_qlinear_read(vvs_qlinear* ql, void* d_w, void* d_w_up, vvs_stream s) {
  QLinear* l = of(ql);
  if (!l) return VVS_EINVAL;
  if (!l->loaded) return no(l, VVS_ESTATE, "qlinear read: call vvs_qlinear_load first");
  if (!d_w || !d_w_up != !l->cfg.gated) return no(l, VVS_EINVAL, "qlinear read: one weight tensor, with a gate two");
  if (off_element(d_w, l->cfg.dtype) || off_element(d_w_up, l->cfg.dtype)) return no(l, VVS_EINVAL, "qlinear read: unaligned weights");
  const Span outs[] = {tensor_span(l, d_w), tensor_span(l, d_w_up)}, own[] = {held_span(l), workspace_span(l)};
  if (share_any(outs, own)) return no(l, VVS_EINVAL, "qlinear read: a weight tensor shares memory with the map's buffers or with the other");
  const vvs_status st = check_device(l);
  if (st != VVS_OK) return st;
  launch_qlinear_read(QWeightsRead{l->w, d_w, d_w_up, l->cfg.dtype}, (hipStream_t)s);
  return launched(l, "qlinear read");
}

vvs_status vvs_qlinear_apply(vvs_qlinear* ql, int32_t n_rows, const void* d_values, const void* d_powers, int32_t out_dtype, void* d_out, int64_t out_stride, vvs_stream s) {
  QLinear* l = of(ql);
  if (!l) return VVS_EINVAL;
  if (l->cfg.gated) return no(l, VVS_EINVAL, "qlinear apply: created with a gate (vvs_qlinear_gate)");
  vvs_status st = check_product(l, n_rows, d_values, d_powers);
  if (st != VVS_OK) return st;
  if (!d_out) return no(l, VVS_EINVAL, "qlinear apply: NULL argument");
  if (!known(out_dtype)) return no(l, VVS_EINVAL, "qlinear apply: unknown dtype");
  const int64_t os = stride_of(out_stride, l->cfg.out);
  if (os < 0 || off_element(d_out, out_dtype)) return no(l, VVS_EINVAL, "qlinear apply: the stride has to cover a row, the pointer to be aligned to an element");
  const Span outs[] = {span_of(d_out, n_rows, l->cfg.out, os, size_of(out_dtype))},
             ins[] = {values_span(d_values, n_rows, l->cfg.in), powers_span(d_powers, n_rows, l->cfg.in), held_span(l), workspace_span(l)};
  if (share_any(outs, ins)) return no(l, VVS_EINVAL, "qlinear apply: the output shares memory with the rows or the map's buffers");
  if ((st = check_device(l)) != VVS_OK) return st;
  QProduct a{};
  a.w = l->w; a.M = n_rows;
  a.x = QRowsIn{(const uint8_t*)d_values, (const uint8_t*)d_powers};
  a.dtype = out_dtype; a.fast = qlinear_fast(l->cfg.products, out_dtype, n_rows);
  a.y = d_out; a.stride = (size_t)os; a.wide = wide_rows(d_out, os, out_dtype, 4);
  a.counters = (uint32_t*)l->ws; a.act = (float*)(l->ws + kQlinearCounters);
  launch_qlinear_product(a, plan_qlinear_product(l->w, n_rows, a.fast), (hipStream_t)s);
  return launched(l, "qlinear apply");
}

vvs_status vvs_qlinear_gate(vvs_qlinear* ql, int32_t n_rows, const void* d_values, const void* d_powers, void* d_out_values, void* d_out_powers, vvs_stream s) {
  QLinear* l = of(ql);
  if (!l) return VVS_EINVAL;
  if (!l->cfg.gated) return no(l, VVS_EINVAL, "qlinear gate: created without a gate (vvs_qlinear_apply)");
  vvs_status st = check_product(l, n_rows, d_values, d_powers);
  if (st != VVS_OK) return st;
  if (!d_out_values || !d_out_powers) return no(l, VVS_EINVAL, "qlinear gate: NULL argument");
  if (off16(d_out_values) || off16(d_out_powers)) return no(l, VVS_EINVAL, "qlinear gate: values and powers must be 16-byte aligned");
  const Span outs[] = {values_span(d_out_values, n_rows, l->cfg.out), powers_span(d_out_powers, n_rows, l->cfg.out)},
             ins[] = {values_span(d_values, n_rows, l->cfg.in), powers_span(d_powers, n_rows, l->cfg.in), held_span(l), workspace_span(l)};
  if (share_any(outs, ins)) return no(l, VVS_EINVAL, "qlinear gate: an output shares memory with the rows, the map's buffers or the other output");
  if ((st = check_device(l)) != VVS_OK) return st;
  QProduct a{};
  a.w = l->w; a.M = n_rows;
  a.x = QRowsIn{(const uint8_t*)d_values, (const uint8_t*)d_powers};
  a.fast = qlinear_fast(l->cfg.products, VVS_BF16, n_rows);
  a.counters = (uint32_t*)l->ws; a.act = (float*)(l->ws + kQlinearCounters);
  a.y8 = QRowsOut{(uint8_t*)d_out_values, (uint8_t*)d_out_powers};
  launch_qlinear_product(a, plan_qlinear_product(l->w, n_rows, false), (hipStream_t)s);
  return launched(l, "qlinear gate");
}

}  // extern "C"
