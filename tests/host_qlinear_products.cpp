// Host-only: which kernel a call of a linear map takes and whether with the matrix instructions for e4m3, by the map's config.  Arguments, nine per case: rows in out gated products dtype fast tile shares.
#include <stdio.h>
#include <stdlib.h>

#include "vvs_qlinear.h"

extern "C" {
hipError_t hipGetDeviceCount(int* n) { *n = 1; return hipSuccess; }
hipError_t hipGetDevice(int* dev) { *dev = 0; return hipSuccess; }
hipError_t hipDeviceSynchronize() { return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
const char* hipGetErrorString(hipError_t) { return ""; }
}

namespace vvs {
static QProduct g_product;
static QPlan g_plan;
static int g_launches = 0;
vvs_status fail_without_context(vvs_status st, const char*) { return st; }
void launch_fill_zero(void*, size_t, hipStream_t) {}
void launch_qrows_round(const QRound&, hipStream_t) {}
void launch_qrows_norm(const QNorm&, hipStream_t) {}
void launch_qrows_read(const QRowsRead&, hipStream_t) {}
void launch_qlinear_load(const QLoad&, hipStream_t) {}
void launch_qlinear_read(const QWeightsRead&, hipStream_t) {}
void launch_qlinear_product(const QProduct& a, const QPlan& p, hipStream_t) { g_product = a; g_plan = p; ++g_launches; }
}  // namespace vvs

using namespace vvs;

int main(int argc, char** argv) {
  int bad = 0;
  // places far from each other; nothing is read or written
  auto at = [](int i) { return (void*)((uintptr_t)(i + 1) << 40); };
  for (int i = 1; i + 8 < argc; i += 9) {
    int v[9];
    for (int j = 0; j < 9; ++j) v[j] = atoi(argv[i + j]);
    const vvs_qlinear_config g{v[1], v[2], v[0], v[3], VVS_BF16, v[4]};
    vvs_qlinear* l = nullptr;
    int st = vvs_qlinear_create(&g, at(0), at(1), &l);
    if (st == VVS_OK) st = vvs_qlinear_load(l, at(2), v[3] ? at(3) : nullptr, nullptr);
    if (st == VVS_OK) st = v[3] ? vvs_qlinear_gate(l, v[0], at(4), at(5), at(6), at(7), nullptr) : vvs_qlinear_apply(l, v[0], at(4), at(5), v[5], at(6), 0, nullptr);
    if (st != VVS_OK || g_plan.few || g_product.fast != v[6] || (int)g_plan.tile != v[7] || g_plan.splits != v[8]) {
      fprintf(stderr, "%d rows, %d -> %d, gated %d, products %d: status %d, few %d, fast %d, tile %d, shares %d\n", v[0], v[1], v[2], v[3], v[4], st, g_plan.few, g_product.fast, (int)g_plan.tile, g_plan.splits);
      bad = 1;
    }
    vvs_qlinear_destroy(l);
  }
  for (int products : {-1, 3, 100}) {
    const vvs_qlinear_config g{128, 128, 1, 0, VVS_BF16, products};
    size_t w = 0, ws = 0;
    vvs_qlinear* l = nullptr;
    if (vvs_qlinear_query_sizes(&g, &w, &ws) != VVS_EINVAL || vvs_qlinear_create(&g, at(0), at(1), &l) != VVS_EINVAL || l) { fprintf(stderr, "products %d taken\n", products); bad = 1; }
  }
  if (bad) return 1;
  printf("host qlinear products ok, %d launches\n", g_launches);
  return 0;
}
