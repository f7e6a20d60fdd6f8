// Host-only exerciser of the largest calls of the 8-bit cache and the rotary operator: what would not fit a launch's grid is refused before anything is launched.
// Stand-ins: those of host_fuzz.cpp, but for the clearing of buffers, which here are address space without memory.
#define launch_fill_zero clear_everything
#define main host_fuzz_main
#include "host_fuzz.cpp"
#undef main
#undef launch_fill_zero
#include <sys/mman.h>
#include "vvs_qcache.h"

namespace vvs {
static int g_called = 0;
void launch_fill_zero(void* p, size_t bytes, hipStream_t) {
  if (bytes < (size_t)1 << 20) memset(p, 0, bytes);
}
void launch_qcache_attention(const QAttention&, int, hipStream_t) { ++g_called; }
void launch_qcache_append(const QAppend&, int, hipStream_t) { ++g_called; }
void launch_qcache_evict(const QEvict&, hipStream_t) { ++g_called; }
void launch_qcache_read(const QRead&, int, hipStream_t) { ++g_called; }
void launch_evict(Ctx*, int, int, hipStream_t) { ++g_called; }
void launch_rope_axes(const RopeArgs&, int, hipStream_t) { ++g_called; }
}  // namespace vvs

using namespace vvs;

static int g_bad = 0;
#define WANT(x, st)                                                                           \
  do {                                                                                        \
    const int got = (x);                                                                      \
    if (got != (st)) { fprintf(stderr, "line %d: %s gave %d, not %d\n", __LINE__, #x, got, (st)); g_bad = 1; } \
  } while (0)

int main() {
  // 4096 key/value heads of 524352 slots: 2^26 blocks of 32 and some
  const vvs_qcache_config g{1, 1, 4096, 4096, 32, 524352, 1, VVS_BF16};
  size_t cb = 0, wb = 0;
  WANT(vvs_qcache_query_sizes(&g, &cb, &wb), VVS_OK);
  void* cache = mmap(nullptr, cb, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS | MAP_NORESERVE, -1, 0);
  void* ws = mmap(nullptr, wb, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS | MAP_NORESERVE, -1, 0);
  if (cache == MAP_FAILED || ws == MAP_FAILED) { printf("no address space\n"); return 0; }
  vvs_qcache* c = nullptr;
  WANT(vvs_qcache_create(&g, cache, ws, &c), VVS_OK);
  alignas(16) static char buf[64];
  int32_t* i32 = (int32_t*)buf;
  float* f32 = (float*)buf;
  void* p = buf;
  g_called = 0;
  WANT(vvs_qcache_append(c, 0, 1, i32, 1 << 30, nullptr, 1, i32, p, 0, p, 0, nullptr), VVS_ESIZE);
  WANT(vvs_qcache_append(c, 0, 1, i32, 524288, nullptr, 524288, nullptr, p, 0, p, 0, nullptr), VVS_ESIZE);
  WANT(vvs_qcache_evict(c, 0, 1, i32, 524288, 0, f32, f32, nullptr, nullptr, nullptr), VVS_ESIZE);
  WANT(vvs_qcache_read(c, 0, 1, i32, nullptr, 524288, p, p, nullptr), VVS_ESIZE);
  WANT(vvs_qcache_read(c, 0, 1, i32, nullptr, 1 << 30, p, p, nullptr), VVS_ESIZE);
  if (g_called) g_bad = 1;
  WANT(vvs_qcache_append(c, 0, 1, i32, 524224, nullptr, 524224, nullptr, p, 0, p, 0, nullptr), VVS_OK);
  WANT(vvs_qcache_read(c, 0, 1, i32, nullptr, 524224, p, p, nullptr), VVS_OK);
  vvs_qcache_destroy(c);
  vvs_rope* r = nullptr;
  const vvs_rope_config rc{64, 3, {12, 10, 10, 0}, VVS_ROPE_OWN, VVS_ROPE_ADJACENT, VVS_BF16, 10000.f};
  WANT(vvs_rope_create(&rc, &r), VVS_OK);
  if (g_called != 2) g_bad = 1;
  for (int n : {(1 << 26) - 3, 1 << 26, 2147483647}) WANT(vvs_rope_apply(r, n, i32, 1, p, 0, p, 0, 0, nullptr, 0, nullptr, 0, 0, nullptr), VVS_ESIZE);
  WANT(vvs_rope_apply(r, (1 << 26) - 4, i32, 1, p, 0, p, 0, 0, nullptr, 0, nullptr, 0, 0, nullptr), VVS_OK);
  if (g_called != 3) g_bad = 1;
  vvs_rope_destroy(r);
  if (!g_bad) printf("host qcache sizes ok\n");
  return g_bad;
}
