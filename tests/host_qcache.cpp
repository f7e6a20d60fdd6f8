// Host-only exerciser of the 8-bit key/value cache and the rotary operator: argument checks, sizes and what the launchers are handed, under the
// sanitizers.  The HIP runtime and the launchers of the contexts are the stand-ins of host_fuzz.cpp; those of the cache are below.
#define main host_fuzz_main
#include "host_fuzz.cpp"
#undef main
#include <math.h>
#include <string>
#include "vvs_qcache.h"

namespace vvs {
static int g_attention = 0, g_append = 0, g_evict = 0, g_read = 0, g_rope = 0;
static QAttention g_attn_args;
static RopeArgs g_rope_args;
void launch_qcache_attention(const QAttention& a, int, hipStream_t) {
  if (a.T < 1 || a.c.heads % a.c.kv_heads || !a.q || !a.out || !(a.c_exp > 0.f) || !a.k != !a.v || a.n_counted > a.T || a.c.blocks * kQBlock < a.capacity) abort();
  if (a.q_stride < (size_t)a.c.heads * a.c.dh || a.k_stride < (size_t)a.c.kv_heads * a.c.dh || a.v_stride < (size_t)a.c.kv_heads * a.c.dh || (!a.causal && a.T > VVS_MAX_T)) abort();
  if (a.norm) memset(a.norm, 0, sizeof(float) * a.c.rows * a.T * a.c.heads);      // inside the workspace
  if (a.parts) memset(a.parts, 0, sizeof(float) * kQParts * 16 * (a.c.dh + 2));
  g_attn_args = a;
  ++g_attention;
}
void launch_qcache_append(const QAppend& a, int, hipStream_t) {
  if (a.n < 1 || a.layer < 0 || a.n_layers < 1 || (!a.select && a.n > a.src_tokens) || a.stride[0] < (size_t)a.c.kv_heads * a.c.dh || a.stride[1] < (size_t)a.c.kv_heads * a.c.dh) abort();
  // the last block of the last region
  const size_t last = a.c.region(a.layer + a.n_layers - 1, a.c.rows - 1, a.c.kv_heads - 1) * a.c.blocks + a.c.blocks - 1;
  memset(a.c.data + last * a.c.block_bytes(), 0, a.c.block_bytes());
  a.c.scale[last] = float2{0.f, 0.f};
  ++g_append;
}
void launch_qcache_evict(const QEvict& a, hipStream_t) {
  if (a.keep < kQBlock || a.keep % kQBlock || a.recent < 0 || a.recent > a.keep) abort();
  memset(a.origin, 0, sizeof(int32_t) * a.n_layers * a.c.rows * a.c.kv_heads * a.capacity);
  ++g_evict;
}
void launch_qcache_read(const QRead& a, int, hipStream_t) {
  if (a.n < 1 || !a.k || !a.v) abort();
  ++g_read;
}
void launch_evict(Ctx*, int, int, hipStream_t) { ++g_evict; }
void launch_rope_axes(const RopeArgs& a, int, hipStream_t) {
  if (a.M < 1 || a.heads < 1 || a.pairs < 1 || 2 * a.pairs > a.dh || a.pairs > 128) abort();
  for (int j = 0; j < a.pairs; ++j)
    if (a.axis[j] >= a.axes || !(a.turns[j] > 0.0)) abort();
  g_rope_args = a;
  ++g_rope;
}
}  // namespace vvs

using namespace vvs;

static int g_bad = 0;
#define WANT(x, st)                                                                           \
  do {                                                                                        \
    const int got = (x);                                                                      \
    if (got != (st)) { fprintf(stderr, "line %d: %s gave %d, not %d\n", __LINE__, #x, got, (st)); g_bad = 1; } \
  } while (0)

int main() {
  vvs_qcache_config g{2, 3, 8, 2, 64, 100, 70, VVS_BF16};
  size_t cb = 0, wb = 0;
  WANT(vvs_qcache_query_sizes(nullptr, &cb, &wb), VVS_EINVAL);
  auto sizes = [&](int vvs_qcache_config::*f, int v) { vvs_qcache_config h = g; h.*f = v; return (int)vvs_qcache_query_sizes(&h, &cb, &wb); };
  for (auto f : {&vvs_qcache_config::n_layers, &vvs_qcache_config::n_rows, &vvs_qcache_config::n_heads, &vvs_qcache_config::n_kv_heads,
                 &vvs_qcache_config::capacity, &vvs_qcache_config::max_tokens})
    for (int v : {0, -1, -2147483647}) WANT(sizes(f, v), VVS_EINVAL);
  WANT(sizes(&vvs_qcache_config::n_kv_heads, 3), VVS_EINVAL);
  WANT(sizes(&vvs_qcache_config::dtype, 2), VVS_EINVAL);
  for (int v : {0, 16, 48, 96, 256}) WANT(sizes(&vvs_qcache_config::head_size, v), VVS_ESIZE);
  WANT(sizes(&vvs_qcache_config::n_rows, 65536), VVS_ESIZE);
  WANT(sizes(&vvs_qcache_config::capacity, 2147483647), VVS_ESIZE);
  WANT(sizes(&vvs_qcache_config::max_tokens, 65537), VVS_ESIZE);
  WANT(sizes(&vvs_qcache_config::n_layers, 4097), VVS_ESIZE);
  { vvs_qcache_config h = g; h.n_rows = 65535; h.n_layers = 4096; h.capacity = 1 << 20; WANT(vvs_qcache_query_sizes(&h, &cb, &wb), VVS_ESIZE); }
  WANT(vvs_qcache_query_sizes(&g, &cb, &wb), VVS_OK);
  if (cb < 2ull * 3 * 2 * 128 * 64 * 2 || cb % 256 || wb % 256) g_bad = 1;
  char* cache = (char*)aligned_alloc(256, cb);
  char* ws = (char*)aligned_alloc(256, wb);
  vvs_qcache* c = nullptr;
  WANT(vvs_qcache_create(&g, cache, ws, nullptr), VVS_EINVAL);
  WANT(vvs_qcache_create(&g, nullptr, ws, &c), VVS_EINVAL);
  WANT(vvs_qcache_create(&g, cache, nullptr, &c), VVS_EINVAL);
  WANT(vvs_qcache_create(&g, cache + 16, ws, &c), VVS_EINVAL);
  WANT(vvs_qcache_create(&g, cache, ws, &c), VVS_OK);
  alignas(16) static char buf[64];
  int32_t* i32 = (int32_t*)buf;
  float* f32 = (float*)buf;
  void* p = buf;
  // append
  WANT(vvs_qcache_append(nullptr, 0, 1, i32, 5, nullptr, 5, nullptr, p, 0, p, 0, nullptr), VVS_EINVAL);
  WANT(vvs_qcache_append(c, -1, 1, i32, 5, nullptr, 5, nullptr, p, 0, p, 0, nullptr), VVS_EINVAL);
  WANT(vvs_qcache_append(c, 1, 2, i32, 5, nullptr, 5, nullptr, p, 0, p, 0, nullptr), VVS_EINVAL);
  WANT(vvs_qcache_append(c, 2147483647, 2147483647, i32, 5, nullptr, 5, nullptr, p, 0, p, 0, nullptr), VVS_EINVAL);
  WANT(vvs_qcache_append(c, 0, 0, i32, 5, nullptr, 5, nullptr, p, 0, p, 0, nullptr), VVS_EINVAL);
  WANT(vvs_qcache_append(c, 0, 1, nullptr, 5, nullptr, 5, nullptr, p, 0, p, 0, nullptr), VVS_EINVAL);
  WANT(vvs_qcache_append(c, 0, 1, i32, 5, nullptr, 5, nullptr, nullptr, 0, p, 0, nullptr), VVS_EINVAL);
  WANT(vvs_qcache_append(c, 0, 1, i32, 0, nullptr, 5, nullptr, p, 0, p, 0, nullptr), VVS_EINVAL);
  WANT(vvs_qcache_append(c, 0, 1, i32, 6, nullptr, 5, nullptr, p, 0, p, 0, nullptr), VVS_EINVAL);
  WANT(vvs_qcache_append(c, 0, 1, i32, 5, nullptr, 5, nullptr, p, 127, p, 127, nullptr), VVS_EINVAL);
  WANT(vvs_qcache_append(c, 0, 1, i32, 5, nullptr, 5, nullptr, p, 132, p, 132, nullptr), VVS_EINVAL);
  WANT(vvs_qcache_append(c, 0, 1, i32, 5, nullptr, 5, nullptr, p, -128, p, -128, nullptr), VVS_EINVAL);
  WANT(vvs_qcache_append(c, 0, 1, i32, 5, nullptr, 5, nullptr, buf + 8, 0, p, 0, nullptr), VVS_EINVAL);
  WANT(vvs_qcache_append(c, 0, 1, i32, 5, nullptr, 5, nullptr, p, 0, p, 132, nullptr), VVS_EINVAL);
  WANT(vvs_qcache_append(c, 0, 2, i32, 5, nullptr, 5, nullptr, p, 136, p, 136, nullptr), VVS_OK);
  WANT(vvs_qcache_append(c, 1, 1, i32, 6, i32, 5, i32, p, 0, p, 0, nullptr), VVS_OK);
  // attention
  auto attend = [&](int layer, int T, const int32_t* parent, const uint8_t* mask, void* k, void* v, float scale, int counted, float* mass, float* block, int64_t qs = 0,
                    void* out = nullptr) { return (int)vvs_qcache_attention(c, layer, i32, T, nullptr, parent, mask, p, qs, k, 0, v, 0, scale, out ? out : p, nullptr, counted, mass, block, nullptr); };
  const int32_t chain[3] = {0, 1, 2}, fork[3] = {0, 0, 1}, broken[3] = {0, 2, 1};
  uint8_t full[16];
  memset(full, 1, sizeof(full));
  WANT(attend(2, 4, nullptr, nullptr, p, p, 1.f, 0, nullptr, nullptr), VVS_EINVAL);
  WANT(attend(0, 0, nullptr, nullptr, p, p, 1.f, 0, nullptr, nullptr), VVS_EINVAL);
  WANT(attend(0, 71, nullptr, nullptr, p, p, 1.f, 0, nullptr, nullptr), VVS_ESIZE);
  WANT(attend(0, 4, nullptr, nullptr, p, nullptr, 1.f, 0, nullptr, nullptr), VVS_EINVAL);
  for (float s : {0.f, -1.f, INFINITY, NAN}) WANT(attend(0, 4, nullptr, nullptr, p, p, s, 0, nullptr, nullptr), VVS_EINVAL);
  WANT(attend(0, 4, nullptr, nullptr, p, p, 1.f, 5, f32, nullptr), VVS_EINVAL);
  WANT(attend(0, 4, nullptr, nullptr, p, p, 1.f, -1, f32, nullptr), VVS_EINVAL);
  WANT(attend(0, 4, nullptr, nullptr, p, p, 1.f, 4, nullptr, nullptr), VVS_EINVAL);
  WANT(attend(0, 4, nullptr, nullptr, nullptr, nullptr, 1.f, 4, nullptr, f32), VVS_EINVAL);
  WANT(attend(0, 4, fork, nullptr, nullptr, nullptr, 1.f, 0, nullptr, nullptr), VVS_EINVAL);
  WANT(attend(0, 4, broken, nullptr, p, p, 1.f, 0, nullptr, nullptr), VVS_EINVAL);
  WANT(attend(0, 4, fork, full, p, p, 1.f, 0, nullptr, nullptr), VVS_EINVAL);
  WANT(attend(0, 4, nullptr, nullptr, p, p, 1.f, 0, nullptr, nullptr, 504), VVS_EINVAL);
  WANT(attend(0, 4, nullptr, nullptr, p, p, 1.f, 0, nullptr, nullptr, 0, buf + 4), VVS_EINVAL);
  { std::vector<int32_t> par(69, 0); WANT(attend(0, 70, par.data(), nullptr, p, p, 1.f, 0, nullptr, nullptr), VVS_ESIZE); }
  if (g_attention) g_bad = 1;
  WANT(attend(1, 4, chain, nullptr, p, p, 1.f, 0, nullptr, nullptr), VVS_OK);
  if (!g_attn_args.causal || g_attn_args.norm || g_attn_args.group != 4) g_bad = 1;
  WANT(attend(1, 4, fork, nullptr, p, p, 0.25f, 4, f32, f32, 768), VVS_OK);
  if (g_attn_args.causal || !g_attn_args.norm || g_attn_args.anc[3] != 0b1011 || g_attn_args.q_stride != 768) g_bad = 1;
  WANT(attend(1, 70, nullptr, nullptr, nullptr, nullptr, 1.f, 0, f32, nullptr), VVS_OK);
  // eviction, read
  WANT(vvs_qcache_evict(c, 0, 3, i32, 32, 0, f32, f32, nullptr, nullptr, nullptr), VVS_EINVAL);
  for (int keep : {0, -32, 31, 33}) WANT(vvs_qcache_evict(c, 0, 1, i32, keep, 0, f32, f32, nullptr, nullptr, nullptr), VVS_EINVAL);
  for (int recent : {-1, 33}) WANT(vvs_qcache_evict(c, 0, 1, i32, 32, recent, f32, f32, nullptr, nullptr, nullptr), VVS_EINVAL);
  WANT(vvs_qcache_evict(c, 0, 1, i32, 32, 0, nullptr, f32, nullptr, nullptr, nullptr), VVS_EINVAL);
  WANT(vvs_qcache_evict(c, 0, 1, i32, 32, 0, f32, nullptr, nullptr, nullptr, nullptr), VVS_EINVAL);
  WANT(vvs_qcache_evict(c, 0, 1, i32, 32, 0, f32, f32, i32, nullptr, nullptr), VVS_EINVAL);
  WANT(vvs_qcache_evict(c, 0, 1, i32, 32, 0, (float*)(buf + 2), f32, nullptr, nullptr, nullptr), VVS_EINVAL);
  WANT(vvs_qcache_evict(c, 0, 2, i32, 64, 64, f32, f32, i32, i32, nullptr), VVS_OK);
  WANT(vvs_qcache_evict(c, 1, 1, i32, 1 << 20, 0, f32, f32, nullptr, nullptr, nullptr), VVS_OK);
  WANT(vvs_qcache_read(c, 0, 1, i32, nullptr, 0, p, p, nullptr), VVS_EINVAL);
  WANT(vvs_qcache_read(c, 0, 1, nullptr, nullptr, 4, p, p, nullptr), VVS_EINVAL);
  WANT(vvs_qcache_read(c, 0, 1, i32, nullptr, 4, p, buf + 8, nullptr), VVS_EINVAL);
  { vvs_qcache_config h = g; h.n_heads = h.n_kv_heads = 4096; h.n_layers = h.n_rows = h.max_tokens = 1; h.capacity = 32; h.head_size = 32;
    size_t hb = 0, hw = 0;
    WANT(vvs_qcache_query_sizes(&h, &hb, &hw), VVS_OK);
    char *hc = (char*)aligned_alloc(256, hb), *hws = (char*)aligned_alloc(256, hw);
    vvs_qcache* wide = nullptr;
    WANT(vvs_qcache_create(&h, hc, hws, &wide), VVS_OK);
    WANT(vvs_qcache_read(wide, 0, 1, i32, nullptr, 1 << 30, p, p, nullptr), VVS_ESIZE);
    vvs_qcache_destroy(wide); free(hc); free(hws); }
  WANT(vvs_qcache_read(c, 0, 2, i32, i32, 4, p, p, nullptr), VVS_OK);
  if (std::string(vvs_qcache_last_error(c)).empty() || g_append != 2 || g_attention != 3 || g_evict != 2 || g_read != 1) g_bad = 1;
  vvs_qcache_destroy(c);
  vvs_qcache_destroy(nullptr);
  free(cache);
  free(ws);
  // a context with its cache in 8 bits
  {
    vvs_config cc{};
    cc.n_layers = 2; cc.d_model = 128; cc.n_heads = 4; cc.d_ff = 64; cc.vocab = 64; cc.logit_hi = 64; cc.grid_h = cc.grid_w = 4; cc.prefix_len = 1;
    cc.prefix_kind = VVS_PREFIX_CLASS; cc.n_classes = 3; cc.n_prompts = 2; cc.max_nodes = 5; cc.dtype = VVS_FP32; cc.cfg_scale = 2.f; cc.rms_eps = 1e-5f; cc.rope_base = 10000.f;
    cc.feature_slots = 2;
    size_t kv = 0, w = 0, pw = 0, kv_same = 0;
    WANT(vvs_query_sizes(&cc, &kv_same, &w, &pw), VVS_OK);
    cc.cache_kind = 2;
    WANT(vvs_query_sizes(&cc, &kv, &w, &pw), VVS_EINVAL);
    cc.cache_kind = VVS_CACHE_E4M3; cc.draft_input = 1;
    WANT(vvs_query_sizes(&cc, &kv, &w, &pw), VVS_EINVAL);
    cc.draft_input = 0; cc.n_heads = 8;
    WANT(vvs_query_sizes(&cc, &kv, &w, &pw), VVS_ESIZE);
    cc.n_heads = 4;
    WANT(vvs_query_sizes(&cc, &kv, &w, &pw), VVS_OK);
    if (kv >= kv_same / 2) g_bad = 1;                    // a quarter of fp32, and 8 bytes per slot
    char *dkv = (char*)aligned_alloc(256, kv), *dws = (char*)aligned_alloc(256, w), *dpw = (char*)aligned_alloc(256, pw);
    vvs_ctx* x = nullptr;
    WANT(vvs_create(&cc, dkv, dws, dpw, &x), VVS_OK);
    std::vector<const void*> weights(vvs_num_weight_tensors(&cc), buf);
    std::vector<float> probs(2 * 6 * 64), u(2 * 6 * 2);
    std::vector<int32_t> toks(10), acc(2), path(2 * VVS_MAX_T), next(2);
    WANT(vvs_load_weights(x, weights.data(), (int32_t)weights.size(), nullptr), VVS_OK);
    WANT(vvs_kv_evict(nullptr, 32, 0, nullptr), VVS_EINVAL);
    WANT(vvs_kv_evict(x, 32, 0, nullptr), VVS_ESTATE);
    WANT(vvs_prefill(x, toks.data(), nullptr, 3, toks.data(), u.data(), next.data(), nullptr), VVS_OK);
    const int evictions = g_evict;
    for (int keep : {0, 31, -32}) WANT(vvs_kv_evict(x, keep, 0, nullptr), VVS_EINVAL);
    for (int recent : {-1, 33}) WANT(vvs_kv_evict(x, 32, recent, nullptr), VVS_EINVAL);
    WANT(vvs_kv_evict(x, 32, 32, nullptr), VVS_OK);
    WANT(vvs_verify(x, 5, nullptr, nullptr, toks.data(), probs.data(), u.data(), VVS_STRICT, acc.data(), path.data(), next.data(), nullptr), VVS_OK);
    WANT(vvs_kv_evict(x, 32, 0, nullptr), VVS_ESTATE);
    WANT(vvs_kv_commit(x, nullptr), VVS_OK);
    WANT(vvs_kv_evict(x, 64, 0, nullptr), VVS_OK);
    if (g_evict != evictions + 2 || vvs_plan_is_fused(x, 6)) g_bad = 1;
    vvs_destroy(x);
    cc.cache_kind = VVS_CACHE_SAME;
    WANT(vvs_query_sizes(&cc, &kv, &w, &pw), VVS_OK);
    free(dkv); free(dws); free(dpw);
    dkv = (char*)aligned_alloc(256, kv); dws = (char*)aligned_alloc(256, w); dpw = (char*)aligned_alloc(256, pw);
    WANT(vvs_create(&cc, dkv, dws, dpw, &x), VVS_OK);
    WANT(vvs_kv_evict(x, 32, 0, nullptr), VVS_ESTATE);
    vvs_destroy(x);
    free(dkv); free(dws); free(dpw);
  }
  // rotary operator
  vvs_rope* r = nullptr;
  const vvs_rope_config rc{64, 3, {12, 10, 10, 0}, VVS_ROPE_OWN, VVS_ROPE_ADJACENT, VVS_BF16, 10000.f};
  auto rope = [&](auto change) { vvs_rope_config h = rc; change(h); vvs_rope* x = nullptr; const int st = vvs_rope_create(&h, &x); vvs_rope_destroy(x); return st; };
  WANT(vvs_rope_create(nullptr, &r), VVS_EINVAL);
  WANT(vvs_rope_create(&rc, nullptr), VVS_EINVAL);
  WANT(rope([](auto& h) { h.dtype = 7; }), VVS_EINVAL);
  WANT(rope([](auto& h) { h.series = 2; }), VVS_EINVAL);
  WANT(rope([](auto& h) { h.pairing = -1; }), VVS_EINVAL);
  for (float b : {1.f, 0.f, -5.f, INFINITY, NAN}) WANT(rope([=](auto& h) { h.base = b; }), VVS_EINVAL);
  for (int s : {0, -64, 4, 12, 264}) WANT(rope([=](auto& h) { h.head_size = s; }), VVS_ESIZE);
  for (int n : {0, -1, 5}) WANT(rope([=](auto& h) { h.n_axes = n; }), VVS_ESIZE);
  WANT(rope([](auto& h) { h.pairs[1] = 0; }), VVS_EINVAL);
  WANT(rope([](auto& h) { h.pairs[1] = 2147483647; }), VVS_EINVAL);
  WANT(rope([](auto& h) { h.pairs[0] = 14; }), VVS_EINVAL);
  WANT(rope([](auto& h) { h.pairs[0] = 11; }), VVS_ESIZE);
  WANT(rope([](auto& h) { h.pairs[0] = 8; h.pairing = VVS_ROPE_HALVES; }), VVS_ESIZE);
  WANT(vvs_rope_create(&rc, &r), VVS_OK);
  auto apply = [&](int n, int heads, void* q, int64_t qs, void* qo, int64_t qos, int kv, void* k, void* ko, int inverse) {
    return (int)vvs_rope_apply(r, n, i32, heads, q, qs, qo, qos, kv, k, 0, ko, 0, inverse, nullptr); };
  alignas(16) static char other[64];
  WANT(apply(0, 2, p, 0, p, 0, 0, nullptr, nullptr, 0), VVS_EINVAL);
  WANT(apply(3, 0, p, 0, p, 0, 0, nullptr, nullptr, 0), VVS_EINVAL);
  WANT(apply(3, 5000, p, 0, p, 0, 0, nullptr, nullptr, 0), VVS_ESIZE);
  WANT(apply(3, 2, nullptr, 0, p, 0, 0, nullptr, nullptr, 0), VVS_EINVAL);
  WANT(apply(3, 2, p, 0, p, 0, 1, nullptr, nullptr, 0), VVS_EINVAL);
  WANT(apply(3, 2, p, 0, p, 0, 0, p, p, 0), VVS_EINVAL);
  WANT(apply(3, 2, p, 0, p, 0, 0, nullptr, nullptr, 2), VVS_EINVAL);
  WANT(apply(3, 2, p, 120, p, 120, 0, nullptr, nullptr, 0), VVS_EINVAL);
  WANT(apply(3, 2, p, 132, p, 132, 0, nullptr, nullptr, 0), VVS_EINVAL);
  WANT(apply(3, 2, p, 256, p, 0, 0, nullptr, nullptr, 0), VVS_EINVAL);          // in place with two strides
  WANT(apply(3, 2, buf + 8, 0, p, 0, 0, nullptr, nullptr, 0), VVS_EINVAL);
  if (g_rope) g_bad = 1;
  WANT(apply(3, 2, p, 256, other, 0, 1, p, p, 1), VVS_OK);
  if (g_rope != 1 || g_rope_args.q_stride != 256 || g_rope_args.q_out_stride != 128 || g_rope_args.pairs != 32 || g_rope_args.axis[31] != 2 || g_rope_args.axis[11] != 0) g_bad = 1;
  if (fabs(g_rope_args.turns[12] * 2.0 * M_PI - 1.0) > 1e-12 || fabs(g_rope_args.turns[13] * 2.0 * M_PI - pow(10000.0, -0.1)) > 1e-12) g_bad = 1;
  vvs_rope_destroy(r);
  vvs_rope_destroy(nullptr);
  if (!g_bad) printf("host qcache ok\n");
  return g_bad;
}
