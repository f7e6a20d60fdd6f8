// Host-only: calls of a linear map whose tensors lie over each other or in the map's own buffers are refused before anything is launched; those beside them are taken.
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include "vvs_qlinear.h"

extern "C" {
hipError_t hipGetDeviceCount(int* n) { *n = 1; return hipSuccess; }
hipError_t hipGetDevice(int* dev) { *dev = 0; return hipSuccess; }
hipError_t hipDeviceSynchronize() { return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
const char* hipGetErrorString(hipError_t) { return ""; }
}

namespace vvs {
static int g_launches = 0;
static std::string g_said;
vvs_status fail_without_context(vvs_status st, const char* msg) { g_said = msg; return st; }
void launch_fill_zero(void*, size_t, hipStream_t) { ++g_launches; }
void launch_qrows_round(const QRound&, hipStream_t) { ++g_launches; }
void launch_qrows_norm(const QNorm&, hipStream_t) { ++g_launches; }
void launch_qrows_read(const QRowsRead&, hipStream_t) { ++g_launches; }
void launch_qlinear_load(const QLoad&, hipStream_t) { ++g_launches; }
void launch_qlinear_read(const QWeightsRead&, hipStream_t) { ++g_launches; }
void launch_qlinear_product(const QProduct&, const QPlan&, hipStream_t) { ++g_launches; }
}  // namespace vvs

using namespace vvs;

static int g_bad = 0;
static vvs_qlinear* g_map;
static void want(int line, int got, bool taken, int before) {
  const bool right = taken ? got == VVS_OK && g_launches == before + 1 : got == VVS_EINVAL && g_launches == before && strstr(g_map ? vvs_qlinear_last_error(g_map) : g_said.c_str(), "shares memory");
  if (!right) { fprintf(stderr, "line %d: status %d, %d launches (%s)\n", line, got, g_launches - before, g_map ? vvs_qlinear_last_error(g_map) : g_said.c_str()); g_bad = 1; }
}
#define TAKEN(x) do { const int before = g_launches; want(__LINE__, (x), true, before); } while (0)
#define REFUSED(x) do { const int before = g_launches; want(__LINE__, (x), false, before); } while (0)

int main() {
  // places far from each other; nothing is read or written
  auto at = [](int i, size_t off = 0) { return (void*)(((uintptr_t)(i + 1) << 40) + off); };
  for (int gated : {0, 1}) {
    const int in = 300, out = 200, rows = 20;
    const vvs_qlinear_config g{in, out, rows, gated, VVS_BF16};
    const size_t bytes = (size_t)in * out * 2;              // of a weight tensor
    size_t wb = 0, sb = 0;
    if (vvs_qlinear_query_sizes(&g, &wb, &sb) != VVS_OK) return 1;
    g_map = nullptr;
    vvs_qlinear* l = nullptr;
    REFUSED(vvs_qlinear_create(&g, at(0), at(0), &l));
    REFUSED(vvs_qlinear_create(&g, at(0), at(0, wb - 256), &l));
    REFUSED(vvs_qlinear_create(&g, at(0, sb - 256), at(0), &l));
    TAKEN(vvs_qlinear_create(&g, at(0), at(0, wb), &l));     // side by side
    vvs_qlinear_destroy(l);
    TAKEN(vvs_qlinear_create(&g, at(0), at(1), &l));
    g_map = l;
    auto load = [&](void* a, void* b) { return (int)vvs_qlinear_load(l, a, gated ? b : nullptr, nullptr); };
    auto read = [&](void* a, void* b) { return (int)vvs_qlinear_read(l, a, gated ? b : nullptr, nullptr); };
    REFUSED(load(at(0), at(3)));                             // from the buffer that it goes to
    REFUSED(load(at(0, wb - 2), at(3)));
    if (gated) REFUSED(load(at(2), at(0, wb / 2)));
    TAKEN(load(at(2), at(2)));                               // one tensor for both
    TAKEN(load(at(0, wb), at(3)));                           // behind the buffer
    REFUSED(read(at(0), at(3)));
    REFUSED(read(at(1), at(3)));                             // into the workspace
    REFUSED(read(at(1, sb - 2), at(3)));
    if (gated) {
      REFUSED(read(at(2), at(2)));                           // gate and up over each other
      REFUSED(read(at(2), at(2, bytes - 2)));
      REFUSED(read(at(2, bytes - 2), at(2)));
      REFUSED(read(at(2), at(0, 256)));
      REFUSED(read(at(2), at(1)));
    }
    TAKEN(read(at(2), at(2, bytes)));
    if (gated) {
      auto gate = [&](void* v, void* p, void* ov, void* op) { return (int)vvs_qlinear_gate(l, rows, v, p, ov, op, nullptr); };
      TAKEN(gate(at(4), at(5), at(6), at(7)));
      for (int own : {0, 1}) {
        REFUSED(gate(at(4), at(5), at(own, 16), at(7)));
        REFUSED(gate(at(4), at(5), at(6), at(own, 16)));
      }
      REFUSED(gate(at(1, 4096), at(5), at(6), at(7)));       // rows in the workspace, which a call writes
      REFUSED(gate(at(4), at(1, 4096), at(6), at(7)));
    } else {
      auto apply = [&](void* v, void* p, void* y, int64_t stride) { return (int)vvs_qlinear_apply(l, rows, v, p, VVS_FP32, y, stride, nullptr); };
      TAKEN(apply(at(4), at(5), at(6), 0));
      REFUSED(apply(at(4), at(5), at(0), 0));
      REFUSED(apply(at(4), at(5), at(0, wb - 4), 0));
      REFUSED(apply(at(4), at(5), at(1), 0));
      REFUSED(apply(at(4), at(5), at(1, sb - 4), 0));
      REFUSED(apply(at(1, 4096 - 256), at(5), at(6), 0));
      REFUSED(apply(at(4), at(1), at(6), 0));
      TAKEN(apply(at(1, sb), at(5), at(0, wb), 0));
    }
    vvs_qlinear_destroy(l);
  }
  if (g_bad) return 1;
  printf("host qlinear overlap ok\n");
  return 0;
}
