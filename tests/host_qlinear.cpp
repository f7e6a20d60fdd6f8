// Host-only exerciser of the rows and weights in 8 bits: argument checks, sizes, which kernel a call takes and what the launchers are handed, under the sanitizers.  The launchers
// are stand-ins that write what the kernels write, so that a buffer that is too small shows.
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>
#include <cmath>
#include <thread>
#include <vector>

#include "vvs_qlinear.h"

static int g_dev = 0;
static std::string g_said;
extern "C" {
hipError_t hipGetDeviceCount(int* n) { *n = 2; return hipSuccess; }
hipError_t hipGetDevice(int* dev) { *dev = g_dev; return hipSuccess; }
hipError_t hipDeviceSynchronize() { return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
const char* hipGetErrorString(hipError_t) { return "an error"; }
}

namespace vvs {
vvs_status fail_without_context(vvs_status st, const char* msg) { g_said = msg; return st; }
void launch_fill_zero(void* p, size_t bytes, hipStream_t) { memset(p, 0, bytes); }

static int g_launches = 0;
static QNorm g_norm;
static QProduct g_product;
static QPlan g_plan;
static void fill(const QRowsOut& y, int M, int width) {
  memset(y.values, 1, (size_t)M * qrows_blocks(width) * kQRowBlock);
  memset(y.powers, 1, (size_t)M * qrows_powers(width));
}
void launch_qrows_round(const QRound& a, hipStream_t) {
  if (a.M < 1 || a.width < 1 || !a.x || a.stride < (size_t)a.width) abort();
  fill(a.y, a.M, a.width);
  ++g_launches;
}
void launch_qrows_norm(const QNorm& a, hipStream_t) {
  if (a.M < 1 || a.x_stride < (size_t)a.width || (a.delta && a.delta_stride < (size_t)a.width) || (a.x_out && a.x_out_stride < (size_t)a.width)) abort();
  fill(a.y, a.M, a.width);
  g_norm = a;
  ++g_launches;
}
void launch_qrows_read(const QRowsRead& a, hipStream_t) {
  if (a.M < 1 || a.stride < (size_t)a.width) abort();
  ++g_launches;
}
void launch_qlinear_load(const QLoad& a, hipStream_t) {
  // the last tile's bytes and powers, as the kernel counts them
  memset(a.w.data, 0, a.w.tile_at(a.w.groups - 1, a.w.blocks - 1, 3) + 2048);
  memset(a.w.powers, 0, a.w.power_at(a.w.groups - 1, (a.w.blocks - 1) / 4 * 4, 3) + 64);
  for (int t = 0; t < 4; ++t)
    for (int i = 0; i < 16; ++i)
      if (a.w.column(a.w.groups - 1, t, i) >= a.w.groups * a.w.unit()) abort();
  ++g_launches;
}
void launch_qlinear_read(const QWeightsRead&, hipStream_t) { ++g_launches; }
void launch_qlinear_product(const QProduct& a, const QPlan& p, hipStream_t) {
  if (a.M < 1 || a.w.blocks != qrows_blocks(a.w.in)) abort();
  if (a.w.gated) fill(a.y8, a.M, a.w.out);
  else if (a.stride < (size_t)a.w.out) abort();
  // maps that share a workspace: no map's sums lie where another's counters do
  if ((char*)a.act - (char*)a.counters != (ptrdiff_t)kQlinearCounters) abort();
  if (p.few) {
    const int rows = (a.M + 16 * p.rt - 1) / (16 * p.rt), columns = a.w.groups * (4 / p.ct);
    if (rows > 65535 || (p.rt != 1 && p.rt != 2) || (p.ct != 1 && p.ct != 2 && p.ct != 4) || p.splits < 1) abort();
    if (a.w.gated) {
      if (p.ct != 2 || p.splits != 1 || a.w.groups % 4) abort();
      if (sizeof(uint32_t) * rows * a.w.groups / 4 > kQlinearCounters) abort();
      memset(a.act, 0, sizeof(float) * a.M * a.w.groups * 32);
    } else if (p.splits > 1) {
      if (sizeof(uint32_t) * rows * columns > kQlinearCounters) abort();
      memset(a.act, 0, sizeof(float) * (size_t)rows * columns * p.splits * p.rt * p.ct * 256);
    }
  } else {
    if (a.w.gated && a.w.groups % 4) abort();
    // every share of the contraction has a block, and the tiles are there in so many shares
    if ((p.splits != 1 && p.splits != 2 && p.splits != 4) || p.splits > a.w.blocks || (p.splits > 1 && (a.w.gated || p.tile == kTile128x256 || p.tile == kTile64x256))) abort();
    if (p.splits == 4 && p.tile == kTile64x128 && !a.fast) abort();
  }
  g_product = a;
  g_plan = p;
  ++g_launches;
}
}  // namespace vvs

using namespace vvs;

static int g_bad = 0;
#define WANT(x, st)                                                                           \
  do {                                                                                        \
    const int got = (x);                                                                      \
    if (got != (st)) { fprintf(stderr, "line %d: %s gave %d, not %d\n", __LINE__, #x, got, (st)); g_bad = 1; } \
  } while (0)
#define CHECK(x) do { if (!(x)) { fprintf(stderr, "line %d: %s\n", __LINE__, #x); g_bad = 1; } } while (0)

struct Rows {
  size_t vb = 0, pb = 0;
  char *v, *p;
  Rows(int n, int width) {
    if (vvs_qrows_sizes(width, n, &vb, &pb) != VVS_OK) abort();
    v = (char*)aligned_alloc(16, (vb + 15) / 16 * 16);
    p = (char*)malloc(pb);            // (malloc: exact, and aligned to 16)
  }
  ~Rows() { free(v); free(p); }
};

static void rows_calls() {
  size_t v = 0, p = 0;
  WANT(vvs_qrows_sizes(0, 1, &v, &p), VVS_EINVAL);
  WANT(vvs_qrows_sizes(1, 0, &v, &p), VVS_EINVAL);
  WANT(vvs_qrows_sizes(-1, -1, &v, &p), VVS_EINVAL);
  WANT(vvs_qrows_sizes(65537, 1, &v, &p), VVS_ESIZE);
  CHECK(strstr(vvs_qrows_last_error(), "65536"));
  WANT(vvs_qrows_sizes(65536, 2147483647, &v, &p), VVS_OK);
  CHECK(v == 65536ull * 2147483647 && p == 512ull * 2147483647);
  WANT(vvs_qrows_sizes(129, 3, &v, nullptr), VVS_OK);
  CHECK(v == 3 * 256);
  WANT(vvs_qrows_sizes(129, 3, nullptr, &p), VVS_OK);
  CHECK(p == 3 * 4);

  const int n = 5, w = 200;
  Rows r(n, w);
  std::vector<float> x(n * 512), d(n * 512), o(n * 512), g(512);
  float* xf = x.data();
  auto round = [&](int rows, int width, int dtype, const void* src, int64_t stride, void* values, void* powers) { return (int)vvs_qrows_round(rows, width, dtype, src, stride, values, powers, nullptr); };
  WANT(round(n, w, VVS_FP32, xf, 0, r.v, r.p), VVS_OK);
  WANT(round(n, w, VVS_FP32, xf, 512, r.v, r.p), VVS_OK);
  WANT(round(n, w, VVS_BF16, (char*)xf + 2, 201, r.v, r.p), VVS_OK);
  for (int bad : {0, -1, -2147483647 - 1}) { WANT(round(bad, w, VVS_FP32, xf, 0, r.v, r.p), VVS_EINVAL); WANT(round(n, bad, VVS_FP32, xf, 0, r.v, r.p), VVS_EINVAL); }
  WANT(round(n, 65537, VVS_FP32, xf, 0, r.v, r.p), VVS_ESIZE);
  WANT(round(2147483647, 65536, VVS_FP32, xf, 0, r.v, r.p), VVS_ESIZE);
  WANT(round(n, w, 2, xf, 0, r.v, r.p), VVS_EINVAL);
  WANT(round(n, w, -1, xf, 0, r.v, r.p), VVS_EINVAL);
  WANT(round(n, w, VVS_FP32, nullptr, 0, r.v, r.p), VVS_EINVAL);
  WANT(round(n, w, VVS_FP32, xf, 0, nullptr, r.p), VVS_EINVAL);
  WANT(round(n, w, VVS_FP32, xf, 0, r.v, nullptr), VVS_EINVAL);
  WANT(round(n, w, VVS_FP32, xf, 199, r.v, r.p), VVS_EINVAL);
  WANT(round(n, w, VVS_FP32, xf, -200, r.v, r.p), VVS_EINVAL);
  WANT(round(n, w, VVS_FP32, xf, (int64_t)1 << 40, r.v, r.p), VVS_EINVAL);
  WANT(round(n, w, VVS_FP32, (char*)xf + 2, 0, r.v, r.p), VVS_EINVAL);
  WANT(round(n, w, VVS_BF16, (char*)xf + 1, 0, r.v, r.p), VVS_EINVAL);
  WANT(round(n, w, VVS_FP32, xf, 0, r.v + 8, r.p), VVS_EINVAL);
  WANT(round(n, w, VVS_FP32, xf, 0, r.v, r.p + 4), VVS_EINVAL);
  WANT(round(n, w, VVS_FP32, xf, 0, xf, r.p), VVS_EINVAL);                       // onto its input
  WANT(round(n, w, VVS_FP32, xf, 0, r.v, xf + 4), VVS_EINVAL);
  WANT(round(n, w, VVS_FP32, xf, 0, r.v, r.v + 16), VVS_EINVAL);                 // one output inside the other
  CHECK(strstr(vvs_qrows_last_error(), "shares memory"));
  {
    // the message is a thread's own
    std::thread other([&] { CHECK(strlen(vvs_qrows_last_error()) == 0); WANT(round(0, w, VVS_FP32, xf, 0, r.v, r.p), VVS_EINVAL); CHECK(strstr(vvs_qrows_last_error(), "positive")); });
    other.join();
    CHECK(strstr(vvs_qrows_last_error(), "shares memory"));
  }

  auto norm = [&](const void* src, int64_t xs, const void* delta, int64_t ds, void* out, int64_t os, float eps = 1e-5f, int xt = VVS_FP32, int dt = VVS_FP32, int gt = VVS_FP32, const void* gain = nullptr,
                  void* values = nullptr, void* powers = nullptr) {
    return (int)vvs_qrows_norm(n, w, xt, src, xs, dt, delta, ds, out, os, gt, gain ? gain : g.data(), eps, values ? values : r.v, powers ? powers : r.p, nullptr);
  };
  WANT(norm(xf, 0, d.data(), 0, o.data(), 0), VVS_OK);
  CHECK(g_norm.x_wide && g_norm.delta_wide && g_norm.x_out_wide && g_norm.gain_wide);
  WANT(norm(xf, 0, d.data(), 0, xf, 0), VVS_OK);                                 // in place
  WANT(norm(xf, 512, d.data(), 0, xf, 0), VVS_EINVAL);                           // ... with another stride
  WANT(norm(xf, 0, nullptr, 0, nullptr, 0), VVS_OK);
  CHECK(!g_norm.delta && !g_norm.x_out);
  WANT(norm(xf, 0, nullptr, -5, nullptr, -5, 0.f, VVS_FP32, 77), VVS_OK);         // of what is not there nothing is asked
  WANT(norm(xf, 201, d.data(), 512, o.data(), 203), VVS_OK);
  CHECK(!g_norm.x_wide && g_norm.delta_wide && !g_norm.x_out_wide);
  for (float bad : {-1e-6f, INFINITY, -INFINITY, NAN}) WANT(norm(xf, 0, nullptr, 0, nullptr, 0, bad), VVS_EINVAL);
  WANT(norm(nullptr, 0, nullptr, 0, nullptr, 0), VVS_EINVAL);
  WANT((int)vvs_qrows_norm(n, w, VVS_FP32, xf, 0, 0, nullptr, 0, nullptr, 0, VVS_FP32, nullptr, 0.f, r.v, r.p, nullptr), VVS_EINVAL);
  WANT(norm(xf, 0, d.data(), 0, nullptr, 0, 0.f, 5), VVS_EINVAL);
  WANT(norm(xf, 0, d.data(), 0, nullptr, 0, 0.f, VVS_FP32, 5), VVS_EINVAL);
  WANT(norm(xf, 0, d.data(), 0, nullptr, 0, 0.f, VVS_FP32, VVS_FP32, 5), VVS_EINVAL);
  WANT(norm(xf, 100, d.data(), 0, nullptr, 0), VVS_EINVAL);
  WANT(norm(xf, 0, d.data(), 100, nullptr, 0), VVS_EINVAL);
  WANT(norm(xf, 0, d.data(), 0, o.data(), 100), VVS_EINVAL);
  WANT(norm((char*)xf + 2, 0, nullptr, 0, nullptr, 0), VVS_EINVAL);
  WANT(norm(xf, 0, (char*)d.data() + 1, 0, nullptr, 0, 0.f, VVS_FP32, VVS_BF16), VVS_EINVAL);
  WANT(norm(xf, 0, nullptr, 0, (char*)o.data() + 2, 0), VVS_EINVAL);
  WANT(norm(xf, 0, nullptr, 0, nullptr, 0, 0.f, VVS_FP32, 0, VVS_FP32, (char*)g.data() + 3), VVS_EINVAL);
  WANT(norm(xf, 0, d.data(), 0, d.data(), 0), VVS_EINVAL);                       // onto delta
  WANT(norm(xf, 0, d.data(), 0, xf + 8, 0), VVS_EINVAL);                         // across x
  WANT(norm(xf, 0, nullptr, 0, o.data(), 0, 0.f, VVS_FP32, 0, VVS_FP32, o.data() + 40), VVS_EINVAL);
  WANT(norm(xf, 0, nullptr, 0, r.v, 0), VVS_EINVAL);                             // onto the rows
  WANT(norm(xf, 512, nullptr, 0, xf + 312, 512), VVS_OK);                        // parts of one tensor, side by side
  WANT(norm(xf, 512, nullptr, 0, xf + 313, 512), VVS_EINVAL);                    // ... the last element is the next row's first
  WANT(norm(xf, 512, nullptr, 0, xf + 199, 512), VVS_EINVAL);
  WANT(norm(xf + 312, 512, nullptr, 0, xf, 512), VVS_OK);
  WANT(norm(xf + 313, 512, nullptr, 0, xf, 512), VVS_EINVAL);
  WANT(norm(xf, 512, xf + 200, 512, xf + 312, 512), VVS_EINVAL);                 // across delta

  auto read = [&](int rows, int width, int dtype, void* out, int64_t os) { return (int)vvs_qrows_read(rows, width, r.v, r.p, dtype, out, os, nullptr); };
  WANT(read(n, w, VVS_FP32, o.data(), 0), VVS_OK);
  WANT(read(n, w, VVS_BF16, o.data(), 300), VVS_OK);
  WANT(read(0, w, VVS_FP32, o.data(), 0), VVS_EINVAL);
  WANT(read(n, 70000, VVS_FP32, o.data(), 0), VVS_ESIZE);
  WANT(read(n, w, 3, o.data(), 0), VVS_EINVAL);
  WANT(read(n, w, VVS_FP32, nullptr, 0), VVS_EINVAL);
  WANT(read(n, w, VVS_FP32, o.data(), 199), VVS_EINVAL);
  WANT(read(n, w, VVS_FP32, (char*)o.data() + 1, 0), VVS_EINVAL);
  WANT(read(n, w, VVS_FP32, r.v, 0), VVS_EINVAL);
}

// One map with exact buffers: the calls in a few sizes of rows
static void map(int in, int out, int max_rows, int gated) {
  vvs_qlinear_config g{in, out, max_rows, gated, VVS_BF16};
  size_t wb = 0, sb = 0;
  WANT(vvs_qlinear_query_sizes(&g, &wb, &sb), VVS_OK);
  char *weights = (char*)aligned_alloc(256, wb), *ws = (char*)aligned_alloc(256, sb);
  vvs_qlinear* l = nullptr;
  WANT(vvs_qlinear_create(&g, weights, ws, &l), VVS_OK);
  alignas(16) static char buf[16];
  Rows x(max_rows, in), y(gated ? max_rows : 1, gated ? out : 1);
  auto call = [&](int n) { return gated ? (int)vvs_qlinear_gate(l, n, x.v, x.p, y.v, y.p, nullptr) : (int)vvs_qlinear_apply(l, n, x.v, x.p, VVS_BF16, buf, 0, nullptr); };
  WANT(call(1), VVS_ESTATE);
  WANT(vvs_qlinear_load(l, buf, gated ? buf : nullptr, nullptr), VVS_OK);
  for (int n : {1, 2, 15, 16, 17, 31, 32, 33, 64, 65, 100, 129, 1000, max_rows})
    if (n <= max_rows) {
      WANT(call(n), VVS_OK);
      CHECK(g_product.M == n && g_product.w.in == in && g_product.w.out == out);
      if (!gated) CHECK(g_product.fast == (n > 64));             // (outputs in bf16)
      if (n <= 64) CHECK(g_plan.few || g_plan.tile == (gated ? kTile32x256 : kTile32x128));    // the tiles that multiply whole
    }
  WANT(call(max_rows + 1), VVS_ESIZE);
  WANT(call(0), VVS_EINVAL);
  vvs_qlinear_destroy(l);
  free(weights);
  free(ws);
}

int main() {
  rows_calls();
  for (int gated : {0, 1}) {
    map(1, 1, 1, gated);
    map(129, 65, 40, gated);
    map(344, 128, 70, gated);
    map(768, 2048, 1000, gated);
    map(11008, 300, 200, gated);
    map(8192, 4096, 33, gated);
    map(65536, 40, 65, gated);
    map(130, 5000, 4200, gated);
    map(5000, 2100, 40, gated);
    map(10300, 5000, 40, gated);
    map(10300, 5440, 33, gated);
    map(2100, 2100, 300, gated);
    map(2100, 5600, 70, gated);
    map(300, 65536, 130, gated);
  }
  // which kernel
  auto plan = [](int in, int out, int gated, int M) { QWeights w{in, out, gated, qrows_blocks(in), 0, nullptr, nullptr}; w.groups = (out + w.unit() - 1) / w.unit(); if (gated) w.groups = (w.groups + 3) & ~3; return plan_qlinear_product(w, M, !gated && M > 64); };
  { QPlan p = plan(11008, 4096, 0, 28); CHECK(p.few && p.splits == 2 && p.rt == 2 && p.ct == 2); }
  { QPlan p = plan(11008, 4096, 0, 8); CHECK(p.few && p.splits == 1 && p.rt == 1 && p.ct == 1); }
  for (int M : {8, 28}) { QPlan p = plan(11008, 5000, 0, M); CHECK(p.few && p.splits == 3 && p.rt == 2 && p.ct == 2); }
  { QPlan p = plan(11008, 5000, 0, 33); CHECK(p.splits == 1); }
  { QPlan p = plan(4096, 12288, 0, 8); CHECK(p.few && p.rt == 1 && p.ct == 2); }
  { QPlan p = plan(1280, 3840, 0, 432); CHECK(!p.few && p.tile == kTile64x128); }
  { QPlan p = plan(1280, 1280, 0, 432); CHECK(!p.few && p.tile == kTile32x128); }
  { QPlan p = plan(1280, 3840, 0, 1000); CHECK(!p.few && p.tile == kTile64x256); }
  { QPlan p = plan(4096, 12288, 0, 8192); CHECK(!p.few && p.tile == kTile128x256); }
  { QPlan p = plan(1280, 3840, 0, 128); CHECK(p.few && p.ct == 4); }
  { QPlan p = plan(11008, 4096, 0, 224); CHECK(!p.few && p.tile == kTile32x128 && p.splits == 4); }
  { QPlan p = plan(11008, 4096, 0, 300); CHECK(!p.few && p.tile == kTile64x128 && p.splits == 4); }
  { QPlan p = plan(4096, 4096, 0, 432); CHECK(!p.few && p.tile == kTile64x128 && p.splits == 2); }
  { QPlan p = plan(3456, 1280, 0, 432); CHECK(!p.few && p.tile == kTile32x128 && p.splits == 4); }
  { QPlan p = plan(2048, 2048, 0, 432); CHECK(!p.few && p.tile == kTile32x128 && p.splits == 2); }
  for (int blocks = 1; blocks < 8; ++blocks) {
    const QWeights w{blocks * 128, 64, 0, blocks, 1, nullptr, nullptr};
    for (int wanted : {0, 1, 2, 3, 4, 8}) CHECK(qlinear_shares(w, wanted) >= 1 && qlinear_shares(w, wanted) <= std::min(4, blocks) && qlinear_shares(w, wanted) != 3);
  }
  { QPlan p = plan(4096, 11008, 1, 14); CHECK(p.few && p.rt == 1); }
  { QPlan p = plan(4096, 11008, 1, 60); CHECK(!p.few && p.tile == kTile32x256); }
  { QPlan p = plan(4096, 11008, 1, 128); CHECK(!p.few && p.tile == kTile64x256); }
  { QPlan p = plan(4096, 11008, 1, 4093); CHECK(!p.few && p.tile == kTile128x256); }
  { QPlan p = plan(1280, 1280, 0, 28); CHECK(p.few && p.rt == 1 && p.ct == 1); }
  { QPlan p = plan(4096, 2048, 0, 60); CHECK(p.few && p.rt == 1 && p.ct == 2); }
  { QPlan p = plan(1280, 1280, 0, 256); CHECK(p.few && p.rt == 1 && p.ct == 2); }
  { QPlan p = plan(4096, 2048, 0, 128); CHECK(p.few && p.rt == 2 && p.ct == 2 && p.splits == 1); }
  { QPlan p = plan(4096, 12288, 0, 28); CHECK(p.few && p.rt == 2 && p.ct == 4); }
  { QPlan p = plan(4096, 16384, 0, 48); CHECK(!p.few && p.tile == kTile32x128 && p.splits == 4); }
  { QPlan p = plan(4096, 32768, 0, 48); CHECK(!p.few && p.tile == kTile32x128 && p.splits == 2); }
  { QPlan p = plan(4096, 12288, 0, 432); CHECK(!p.few && p.tile == kTile64x128); }
  { QPlan p = plan(4096, 16384, 0, 600); CHECK(!p.few && p.tile == kTile128x256); }
  { QPlan p = plan(768, 2048, 1, 48); CHECK(p.few && p.rt == 1); }
  { QPlan p = plan(4096, 11008, 1, 28); CHECK(p.few && p.rt == 2); }
  { QPlan p = plan(4096, 2048, 1, 128); CHECK(p.few && p.rt == 2); }
  { QPlan p = plan(1280, 3456, 1, 128); CHECK(!p.few && p.tile == kTile64x256); }
  { QPlan p = plan(128, 344, 1, 128); CHECK(!p.few && p.tile == kTile32x256); }

  // configs
  vvs_qlinear_config g{256, 128, 40, 0, VVS_FP32};
  size_t wb = 0, sb = 0;
  auto sizes = [&](int32_t vvs_qlinear_config::*f, int v) { vvs_qlinear_config h = g; h.*f = v; return (int)vvs_qlinear_query_sizes(&h, &wb, &sb); };
  WANT(vvs_qlinear_query_sizes(nullptr, &wb, &sb), VVS_EINVAL);
  for (int v : {0, -1, -2147483647 - 1}) {
    WANT(sizes(&vvs_qlinear_config::in, v), VVS_EINVAL);
    WANT(sizes(&vvs_qlinear_config::out, v), VVS_EINVAL);
    WANT(sizes(&vvs_qlinear_config::max_rows, v), VVS_EINVAL);
  }
  WANT(sizes(&vvs_qlinear_config::dtype, 2), VVS_EINVAL);
  WANT(sizes(&vvs_qlinear_config::gated, 2), VVS_EINVAL);
  WANT(sizes(&vvs_qlinear_config::gated, -1), VVS_EINVAL);
  WANT(sizes(&vvs_qlinear_config::in, 65537), VVS_ESIZE);
  WANT(sizes(&vvs_qlinear_config::out, 2147483647), VVS_ESIZE);
  WANT(sizes(&vvs_qlinear_config::max_rows, 2147483647), VVS_ESIZE);
  { vvs_qlinear_config h{65536, 1 << 24, 1, 0, VVS_BF16}; WANT(vvs_qlinear_query_sizes(&h, &wb, &sb), VVS_ESIZE); }
  { vvs_qlinear_config h{128, 1 << 24, 1 << 20, 0, VVS_BF16}; WANT(vvs_qlinear_query_sizes(&h, &wb, &sb), VVS_ESIZE); }
  { vvs_qlinear_config h{128, 65537, 1, 1, VVS_BF16}; WANT(vvs_qlinear_query_sizes(&h, &wb, &sb), VVS_ESIZE); }
  { vvs_qlinear_config h{4096, 11008, 8192, 1, VVS_BF16}; WANT(vvs_qlinear_query_sizes(&h, &wb, &sb), VVS_OK); CHECK(wb >= 2ull * 4096 * 11008 && wb < 2.02 * 4096 * 11008 && sb < (2 << 20)); }

  // create
  WANT(vvs_qlinear_query_sizes(&g, &wb, &sb), VVS_OK);
  CHECK(wb % 256 == 0 && sb % 256 == 0);
  char *weights = (char*)aligned_alloc(256, wb), *ws = (char*)aligned_alloc(256, sb);
  vvs_qlinear* l = nullptr;
  WANT(vvs_qlinear_create(&g, weights, ws, nullptr), VVS_EINVAL);
  WANT(vvs_qlinear_create(&g, nullptr, ws, &l), VVS_EINVAL);
  WANT(vvs_qlinear_create(&g, weights, nullptr, &l), VVS_EINVAL);
  WANT(vvs_qlinear_create(&g, weights + 128, ws, &l), VVS_EINVAL);
  WANT(vvs_qlinear_create(&g, weights, ws + 64, &l), VVS_EINVAL);
  WANT(vvs_qlinear_create(nullptr, weights, ws, &l), VVS_EINVAL);
  CHECK(!l && strstr(g_said.c_str(), "NULL"));
  WANT(vvs_qlinear_create(&g, weights, ws, &l), VVS_OK);
  alignas(16) static char buf[64];
  Rows x(40, 256);
  static float out[40 * 200];
  WANT(vvs_qlinear_load(nullptr, buf, nullptr, nullptr), VVS_EINVAL);
  WANT(vvs_qlinear_read(nullptr, buf, nullptr, nullptr), VVS_EINVAL);
  WANT(vvs_qlinear_apply(nullptr, 1, x.v, x.p, VVS_FP32, out, 0, nullptr), VVS_EINVAL);
  WANT(vvs_qlinear_gate(nullptr, 1, x.v, x.p, buf, buf, nullptr), VVS_EINVAL);
  WANT(vvs_qlinear_read(l, buf, nullptr, nullptr), VVS_ESTATE);
  WANT(vvs_qlinear_apply(l, 1, x.v, x.p, VVS_FP32, out, 0, nullptr), VVS_ESTATE);
  CHECK(strstr(vvs_qlinear_last_error(l), "load"));
  WANT(vvs_qlinear_load(l, nullptr, nullptr, nullptr), VVS_EINVAL);
  WANT(vvs_qlinear_load(l, buf, buf, nullptr), VVS_EINVAL);
  WANT(vvs_qlinear_load(l, buf + 2, nullptr, nullptr), VVS_EINVAL);
  g_dev = 1;
  WANT(vvs_qlinear_load(l, buf, nullptr, nullptr), VVS_EINVAL);
  CHECK(strstr(vvs_qlinear_last_error(l), "device"));
  g_dev = 0;
  WANT(vvs_qlinear_load(l, buf, nullptr, nullptr), VVS_OK);
  WANT(vvs_qlinear_read(l, buf, buf, nullptr), VVS_EINVAL);
  WANT(vvs_qlinear_read(l, buf, nullptr, nullptr), VVS_OK);
  auto apply = [&](int n, const void* v, const void* p, int dtype, void* y, int64_t stride) { return (int)vvs_qlinear_apply(l, n, v, p, dtype, y, stride, nullptr); };
  const int before = g_launches;
  WANT(apply(0, x.v, x.p, VVS_FP32, out, 0), VVS_EINVAL);
  WANT(apply(-3, x.v, x.p, VVS_FP32, out, 0), VVS_EINVAL);
  WANT(apply(41, x.v, x.p, VVS_FP32, out, 0), VVS_ESIZE);
  WANT(apply(4, nullptr, x.p, VVS_FP32, out, 0), VVS_EINVAL);
  WANT(apply(4, x.v, nullptr, VVS_FP32, out, 0), VVS_EINVAL);
  WANT(apply(4, x.v + 8, x.p, VVS_FP32, out, 0), VVS_EINVAL);
  WANT(apply(4, x.v, x.p + 4, VVS_FP32, out, 0), VVS_EINVAL);
  WANT(apply(4, x.v, x.p, 9, out, 0), VVS_EINVAL);
  WANT(apply(4, x.v, x.p, VVS_FP32, nullptr, 0), VVS_EINVAL);
  WANT(apply(4, x.v, x.p, VVS_FP32, out, 127), VVS_EINVAL);
  WANT(apply(4, x.v, x.p, VVS_FP32, (char*)out + 2, 0), VVS_EINVAL);
  WANT(apply(4, x.v, x.p, VVS_BF16, (char*)out + 1, 0), VVS_EINVAL);
  WANT(apply(4, x.v, x.p, VVS_FP32, x.v, 0), VVS_EINVAL);
  WANT(vvs_qlinear_gate(l, 4, x.v, x.p, buf, buf + 32, nullptr), VVS_EINVAL);
  g_dev = 1;
  WANT(apply(4, x.v, x.p, VVS_FP32, out, 0), VVS_EINVAL);
  g_dev = 0;
  CHECK(g_launches == before);
  WANT(apply(4, x.v, x.p, VVS_FP32, out, 0), VVS_OK);
  CHECK(g_product.wide);
  WANT(apply(4, x.v, x.p, VVS_FP32, out + 1, 0), VVS_OK);
  CHECK(!g_product.wide);
  WANT(apply(4, x.v, x.p, VVS_BF16, (char*)out + 8, 132), VVS_OK);
  CHECK(g_product.wide);
  WANT(apply(40, x.v, x.p, VVS_BF16, (char*)out + 2, 129), VVS_OK);
  CHECK(!g_product.wide);
  vvs_qlinear_destroy(l);
  vvs_qlinear_destroy(nullptr);
  CHECK(strlen(vvs_qlinear_last_error(nullptr)) == 0);
  // a gate's output
  g.gated = 1;
  WANT(vvs_qlinear_query_sizes(&g, &wb, &sb), VVS_OK);
  char *weights2 = (char*)aligned_alloc(256, wb), *ws2 = (char*)aligned_alloc(256, sb);
  WANT(vvs_qlinear_create(&g, weights2, ws2, &l), VVS_OK);
  WANT(vvs_qlinear_load(l, buf, nullptr, nullptr), VVS_EINVAL);
  WANT(vvs_qlinear_load(l, buf, buf, nullptr), VVS_OK);
  Rows y(40, 128);
  auto gate = [&](int n, void* v, void* p) { return (int)vvs_qlinear_gate(l, n, x.v, x.p, v, p, nullptr); };
  WANT(gate(40, y.v, y.p), VVS_OK);
  WANT(gate(41, y.v, y.p), VVS_ESIZE);
  WANT(gate(40, nullptr, y.p), VVS_EINVAL);
  WANT(gate(40, y.v, nullptr), VVS_EINVAL);
  WANT(gate(40, y.v + 8, y.p), VVS_EINVAL);
  WANT(gate(40, y.v, y.p + 4), VVS_EINVAL);
  WANT(gate(40, x.v, y.p), VVS_EINVAL);
  WANT(gate(40, y.v, x.p), VVS_EINVAL);
  WANT(gate(40, y.v, y.v + 128), VVS_EINVAL);
  WANT(vvs_qlinear_apply(l, 4, x.v, x.p, VVS_FP32, out, 0, nullptr), VVS_EINVAL);
  vvs_qlinear_destroy(l);
  free(weights); free(ws); free(weights2); free(ws2);
  if (g_bad) return 1;
  printf("host qlinear ok\n");
  return 0;
}
