// Host side of the 8-bit key/value cache and of the rotary operator: argument checks, buffer sizes, entry points.
#include "vvs_qcache.h"

#include <float.h>
#include <math.h>
#include <string.h>
#include <algorithm>
#include <new>

namespace vvs {

struct QCache {
  vvs_qcache_config cfg;
  QLayout lay;
  size_t cache_bytes, ws_bytes, parts_off, norm_off, origin_off, scores_off;
  int score_steps;
  int dev, cus;
  char* ws;
  std::string err;
};

struct Rope {
  vvs_rope_config cfg;
  RopeArgs args;
  std::string err;
};

// What vvs_last_error(NULL) tells of a failed create or query (vvs_host.cpp)
vvs_status fail_without_context(vvs_status st, const char* msg);

static vvs_status no(std::string* err, vvs_status st, const char* msg) {
  if (!err) return fail_without_context(st, msg);
  *err = msg;
  return st;
}

static vvs_status plan_qcache(const vvs_qcache_config* cfg, QCache* c) {
  if (!cfg) return no(nullptr, VVS_EINVAL, "qcache config is NULL");
  const vvs_qcache_config& g = *cfg;
  if (g.n_layers < 1 || g.n_rows < 1 || g.n_heads < 1 || g.n_kv_heads < 1 || g.capacity < 1 || g.max_tokens < 1)
    return no(nullptr, VVS_EINVAL, "qcache config: a dimension is not positive");
  if (g.dtype != VVS_FP32 && g.dtype != VVS_BF16) return no(nullptr, VVS_EINVAL, "qcache config: unknown dtype");
  if (g.n_heads % g.n_kv_heads) return no(nullptr, VVS_EINVAL, "qcache config: n_heads is not a multiple of n_kv_heads");
  if (g.head_size != 32 && g.head_size != 64 && g.head_size != 128) return no(nullptr, VVS_ESIZE, "qcache config: head size must be 32, 64 or 128");
  if (g.n_rows > 65535 || g.n_layers > 4096 || g.n_heads > 4096 || g.max_tokens > 65536 || g.capacity > (1 << 30))
    return no(nullptr, VVS_ESIZE, "qcache config: at most 65535 rows, 4096 layers, 4096 heads, 65536 tokens and 2^30 slots");
  if ((int64_t)g.max_tokens * g.n_heads > (1 << 24)) return no(nullptr, VVS_ESIZE, "qcache config: max_tokens * n_heads above 2^24");
  c->cfg = g;
  c->lay = QLayout{g.n_rows, g.n_heads, g.n_kv_heads, g.head_size, (g.capacity + kQBlock - 1) / kQBlock, nullptr, nullptr};
  const size_t regions = (size_t)g.n_layers * g.n_rows * g.n_kv_heads, blocks = regions * c->lay.blocks;
  if (blocks > ((size_t)1 << 31) - 1) return no(nullptr, VVS_ESIZE, "qcache config: 2^31 blocks or more");
  c->cache_bytes = align_up(blocks * c->lay.block_bytes(), 256) + align_up(blocks * sizeof(float2), 256);
  size_t off = 0;
  c->parts_off = off;
  off = align_up(off + qcache_parts_bytes(g.head_size), 256);
  c->norm_off = off;
  off = align_up(off + (size_t)g.n_rows * g.max_tokens * g.n_heads * sizeof(float), 256);
  c->origin_off = off;
  off = align_up(off + blocks * kQBlock * sizeof(int32_t), 256);
  c->scores_off = off;
  c->score_steps = qcache_score_steps(c->lay.blocks, g.max_tokens);
  off = align_up(off + (size_t)g.n_rows * g.n_kv_heads * c->score_steps * kQKept * kQBlock * sizeof(float), 256);
  c->ws_bytes = off;
  return VVS_OK;
}

static QCache* of(vvs_qcache* c) { return reinterpret_cast<QCache*>(c); }

static vvs_status check_device(QCache* c) {
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) return no(&c->err, VVS_EHIP, "qcache: no current device");
  if (dev != c->dev) return no(&c->err, VVS_EINVAL, "qcache: the cache was created on another device than the current one");
  return VVS_OK;
}

static vvs_status check_layers(QCache* c, int layer, int n_layers) {
  if (layer < 0 || n_layers < 1 || layer > c->cfg.n_layers - n_layers) return no(&c->err, VVS_EINVAL, "qcache: no such layer");
  return VVS_OK;
}

static vvs_status launched(QCache* c, const char* what) {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return VVS_OK;
  c->err = std::string(what) + ": " + hipGetErrorString(e);
  return VVS_EHIP;
}

static bool unaligned(const void* p) { return ((uintptr_t)p & 15) != 0; }

// Elements between tokens of a tensor of `least` elements per token; < 0: not allowed
static int64_t stride_of(int64_t given, int64_t least, int dtype) {
  const int64_t s = given ? given : least;
  const int per16 = dtype == VVS_BF16 ? 8 : 4;
  return s < least || s % per16 || s > ((int64_t)1 << 31) ? -1 : s;
}

// Units (waves, tokens) that a launch of four per workgroup of 256 threads holds: a grid has fewer than 2^32 threads along a dimension.  Asked in front of a call's first launch, so that none is left half done.
constexpr int64_t kMostUnits = ((int64_t)1 << 26) - 4;

}  // namespace vvs

using namespace vvs;

extern "C" {

vvs_status vvs_qcache_query_sizes(const vvs_qcache_config* cfg, size_t* cache_bytes, size_t* workspace_bytes) {
  QCache c{};
  const vvs_status st = plan_qcache(cfg, &c);
  if (st != VVS_OK) return st;
  if (cache_bytes) *cache_bytes = c.cache_bytes;
  if (workspace_bytes) *workspace_bytes = c.ws_bytes;
  return VVS_OK;
}

vvs_status vvs_qcache_create(const vvs_qcache_config* cfg, void* d_cache, void* d_workspace, vvs_qcache** out) {
  if (!out) return no(nullptr, VVS_EINVAL, "qcache create: out is NULL");
  *out = nullptr;
  if (!d_cache || !d_workspace) return no(nullptr, VVS_EINVAL, "qcache create: NULL device buffer");
  if (((uintptr_t)d_cache | (uintptr_t)d_workspace) & 255) return no(nullptr, VVS_EINVAL, "qcache create: device buffers must be 256-byte aligned");
  QCache plan{};
  const vvs_status st = plan_qcache(cfg, &plan);
  if (st != VVS_OK) return st;
  int ndev = 0;
  if (hipGetDeviceCount(&ndev) != hipSuccess || ndev < 1) return no(nullptr, VVS_EHIP, "qcache create: no HIP device (this library has no CPU path)");
  hipError_t e = hipGetDevice(&plan.dev);
  if (e == hipSuccess) e = hipDeviceGetAttribute(&plan.cus, hipDeviceAttributeMultiprocessorCount, plan.dev);
  if (e != hipSuccess) return no(nullptr, VVS_EHIP, hipGetErrorString(e));
  plan.ws = (char*)d_workspace;
  plan.lay.data = (uint8_t*)d_cache;
  const size_t blocks = (size_t)plan.cfg.n_layers * plan.cfg.n_rows * plan.cfg.n_kv_heads * plan.lay.blocks;
  plan.lay.scale = (float2*)((char*)d_cache + align_up(blocks * plan.lay.block_bytes(), 256));
  QCache* c = new (std::nothrow) QCache(plan);
  if (!c) return no(nullptr, VVS_EHIP, "qcache create: out of memory");
  launch_fill_zero(d_cache, c->cache_bytes, nullptr);
  launch_fill_zero(d_workspace, c->ws_bytes, nullptr);
  e = hipGetLastError();
  if (e == hipSuccess) e = hipDeviceSynchronize();
  if (e != hipSuccess) { delete c; return no(nullptr, VVS_EHIP, hipGetErrorString(e)); }
  *out = reinterpret_cast<vvs_qcache*>(c);
  return VVS_OK;
}

void vvs_qcache_destroy(vvs_qcache* c) { delete of(c); }

const char* vvs_qcache_last_error(const vvs_qcache* c) { return c ? reinterpret_cast<const QCache*>(c)->err.c_str() : ""; }

vvs_status vvs_qcache_append(vvs_qcache* qc, int32_t layer, int32_t n_layers, const int32_t* d_len, int32_t n_tokens, const int32_t* d_n_tokens,
                             int32_t src_tokens, const int32_t* d_select, const void* d_k, int64_t k_stride, const void* d_v, int64_t v_stride, vvs_stream s) {
  QCache* c = of(qc);
  if (!c) return VVS_EINVAL;
  vvs_status st = check_layers(c, layer, n_layers);
  if (st != VVS_OK) return st;
  if (!d_len || !d_k || !d_v) return no(&c->err, VVS_EINVAL, "qcache append: NULL argument");
  if (n_tokens < 1 || src_tokens < 1 || n_tokens > (1 << 30) || src_tokens > (1 << 30)) return no(&c->err, VVS_EINVAL, "qcache append: numbers of tokens must be positive");
  if (!d_select && n_tokens > src_tokens) return no(&c->err, VVS_EINVAL, "qcache append: more tokens than d_k and d_v hold");
  if (c->cfg.n_kv_heads * std::min<int64_t>(((int64_t)n_tokens + 2 * kQBlock - 2) / kQBlock, c->lay.blocks) > kMostUnits) return no(&c->err, VVS_ESIZE, "qcache append: too many tokens");
  const int64_t per = (int64_t)c->cfg.n_kv_heads * c->cfg.head_size, ks = stride_of(k_stride, per, c->cfg.dtype), vs = stride_of(v_stride, per, c->cfg.dtype);
  if (ks < 0 || vs < 0 || unaligned(d_k) || unaligned(d_v)) return no(&c->err, VVS_EINVAL, "qcache append: pointers and strides must be multiples of 16 bytes, strides cover a token");
  if ((st = check_device(c)) != VVS_OK) return st;
  QAppend a{};
  a.c = c->lay;
  a.len = QLen{d_len, 0};
  a.layer = layer; a.n_layers = n_layers; a.n = n_tokens; a.src_tokens = src_tokens;
  a.n_tokens = d_n_tokens;
  a.select = d_select; a.select_stride = n_tokens;
  a.k = d_k; a.v = d_v; a.stride[0] = (size_t)ks; a.stride[1] = (size_t)vs;
  a.layer_stride[0] = (size_t)ks * src_tokens * c->cfg.n_rows; a.layer_stride[1] = (size_t)vs * src_tokens * c->cfg.n_rows;
  a.capacity = c->cfg.capacity;
  launch_qcache_append(a, c->cfg.dtype, (hipStream_t)s);
  return launched(c, "qcache append");
}

vvs_status vvs_qcache_attention(vvs_qcache* qc, int32_t layer, const int32_t* d_len, int32_t n_tokens, const int32_t* d_n_tokens, const int32_t* h_parent,
                                const uint8_t* h_tree_mask, const void* d_q, int64_t q_stride, const void* d_k, int64_t k_stride, const void* d_v, int64_t v_stride, float scale,
                                void* d_out, float* d_lse, int32_t n_counted, float* d_mass, float* d_block_mass, vvs_stream s) {
  QCache* c = of(qc);
  if (!c) return VVS_EINVAL;
  vvs_status st = check_layers(c, layer, 1);
  if (st != VVS_OK) return st;
  const vvs_qcache_config& g = c->cfg;
  if (!d_len || !d_q || !d_out) return no(&c->err, VVS_EINVAL, "qcache attention: NULL argument");
  if (!d_k != !d_v) return no(&c->err, VVS_EINVAL, "qcache attention: d_k and d_v go together");
  if (n_tokens < 1) return no(&c->err, VVS_EINVAL, "qcache attention: n_tokens < 1");
  if (n_tokens > g.max_tokens) return no(&c->err, VVS_ESIZE, "qcache attention: n_tokens exceeds max_tokens of the cache");
  if (!(scale > 0.f) || !std::isfinite(scale)) return no(&c->err, VVS_EINVAL, "qcache attention: scale must be positive and finite");
  if (n_counted < 0 || n_counted > n_tokens) return no(&c->err, VVS_EINVAL, "qcache attention: n_counted must be in [0, n_tokens]");
  if (n_counted > 0 && !d_mass && !d_block_mass) return no(&c->err, VVS_EINVAL, "qcache attention: counted weights have nowhere to go");
  if (d_block_mass && !d_k) return no(&c->err, VVS_EINVAL, "qcache attention: block weights without a block");
  const bool topology = h_parent || h_tree_mask;
  if (topology && !d_k) return no(&c->err, VVS_EINVAL, "qcache attention: a topology without block keys and values");
  if (topology && n_tokens > VVS_MAX_T) return no(&c->err, VVS_ESIZE, "qcache attention: more than VVS_MAX_T tokens only as a chain");
  QAttention a{};
  a.causal = 1;
  if (topology) {
    TreeDesc tree;
    if ((st = build_tree(n_tokens - 1, h_parent, h_tree_mask, &tree, &c->err)) != VVS_OK) return st;
    a.causal = tree.causal;
    memcpy(a.anc, tree.anc, sizeof(a.anc));
  }
  const int64_t qs = stride_of(q_stride, (int64_t)g.n_heads * g.head_size, g.dtype), per = (int64_t)g.n_kv_heads * g.head_size;
  const int64_t ks = stride_of(k_stride, per, g.dtype), vs = stride_of(v_stride, per, g.dtype);
  if (qs < 0 || ks < 0 || vs < 0 || unaligned(d_q) || unaligned(d_k) || unaligned(d_v) || unaligned(d_out))
    return no(&c->err, VVS_EINVAL, "qcache attention: pointers and strides must be multiples of 16 bytes, strides cover a token");
  if (((uintptr_t)d_mass | (uintptr_t)d_block_mass | (uintptr_t)d_lse) & 3) return no(&c->err, VVS_EINVAL, "qcache attention: unaligned weights");
  if ((st = check_device(c)) != VVS_OK) return st;
  a.c = c->lay;
  a.len = QLen{d_len, 0};
  a.layer = layer; a.T = n_tokens; a.group = g.n_heads / g.n_kv_heads;
  a.n_tokens = d_n_tokens;
  a.q = d_q; a.k = d_k; a.v = d_v; a.q_stride = (size_t)qs; a.k_stride = (size_t)ks; a.v_stride = (size_t)vs;
  a.c_exp = std::max((float)((double)scale * 1.4426950408889634), FLT_MIN);   // above 0: masked scores are -inf
  a.out = d_out;
  a.n_counted = n_counted;
  a.mass = d_mass; a.block_mass = d_block_mass;
  a.block_stride = n_tokens;
  a.capacity = g.capacity;
  a.lse = d_lse;
  a.norm = n_counted || d_block_mass ? (float*)(c->ws + c->norm_off) : nullptr;
  a.parts = (float*)(c->ws + c->parts_off);
  a.scores = (float*)(c->ws + c->scores_off);
  a.score_steps = c->score_steps;
  launch_qcache_attention(a, g.dtype, (hipStream_t)s);
  return launched(c, "qcache attention");
}

vvs_status vvs_qcache_evict(vvs_qcache* qc, int32_t layer, int32_t n_layers, const int32_t* d_len, int32_t keep, int32_t recent, const float* d_mass,
                            float* d_mass_out, const int32_t* d_pos, int32_t* d_pos_out, vvs_stream s) {
  QCache* c = of(qc);
  if (!c) return VVS_EINVAL;
  vvs_status st = check_layers(c, layer, n_layers);
  if (st != VVS_OK) return st;
  if (!d_len || !d_mass || !d_mass_out) return no(&c->err, VVS_EINVAL, "qcache evict: NULL argument");
  if (!d_pos != !d_pos_out) return no(&c->err, VVS_EINVAL, "qcache evict: d_pos and d_pos_out go together");
  if (keep < kQBlock || keep % kQBlock) return no(&c->err, VVS_EINVAL, "qcache evict: keep must be a positive multiple of VVS_QCACHE_BLOCK");
  if (recent < 0 || recent > keep) return no(&c->err, VVS_EINVAL, "qcache evict: recent must be in [0, keep]");
  if (keep < c->cfg.capacity && (int64_t)c->cfg.n_kv_heads * (keep / kQBlock) > kMostUnits) return no(&c->err, VVS_ESIZE, "qcache evict: too many slots are kept");
  if (((uintptr_t)d_mass | (uintptr_t)d_mass_out | (uintptr_t)d_pos | (uintptr_t)d_pos_out) & 3) return no(&c->err, VVS_EINVAL, "qcache evict: unaligned weights or positions");
  if ((st = check_device(c)) != VVS_OK) return st;
  QEvict a{};
  a.c = c->lay;
  a.len = QLen{d_len, 0};
  a.layer = layer; a.n_layers = n_layers; a.keep = keep; a.recent = recent; a.capacity = c->cfg.capacity;
  a.mass = d_mass; a.mass_out = d_mass_out; a.pos = d_pos; a.pos_out = d_pos_out;
  a.origin = (int32_t*)(c->ws + c->origin_off);
  launch_qcache_evict(a, (hipStream_t)s);
  return launched(c, "qcache evict");
}

vvs_status vvs_qcache_read(vvs_qcache* qc, int32_t layer, int32_t n_layers, const int32_t* d_len, const int32_t* d_first, int32_t n_slots, void* d_k,
                           void* d_v, vvs_stream s) {
  QCache* c = of(qc);
  if (!c) return VVS_EINVAL;
  vvs_status st = check_layers(c, layer, n_layers);
  if (st != VVS_OK) return st;
  if (!d_len || !d_k || !d_v) return no(&c->err, VVS_EINVAL, "qcache read: NULL argument");
  if (n_slots < 1 || n_slots > (1 << 30)) return no(&c->err, VVS_EINVAL, "qcache read: n_slots must be positive");
  if (c->cfg.n_kv_heads * (((int64_t)n_slots + 2 * kQBlock - 2) / kQBlock) > kMostUnits) return no(&c->err, VVS_ESIZE, "qcache read: too many slots");
  if (unaligned(d_k) || unaligned(d_v)) return no(&c->err, VVS_EINVAL, "qcache read: pointers must be multiples of 16 bytes");
  if ((st = check_device(c)) != VVS_OK) return st;
  QRead a{};
  a.c = c->lay;
  a.len = QLen{d_len, 0};
  a.layer = layer; a.n_layers = n_layers; a.n = n_slots; a.capacity = c->cfg.capacity;
  a.first = d_first; a.k = d_k; a.v = d_v;
  launch_qcache_read(a, c->cfg.dtype, (hipStream_t)s);
  return launched(c, "qcache read");
}

vvs_status vvs_kv_evict(vvs_ctx* ctx, int32_t keep, int32_t recent, vvs_stream s) {
  Ctx* c = reinterpret_cast<Ctx*>(ctx);
  if (!c) return VVS_EINVAL;
  if (c->cfg.cache_kind != VVS_CACHE_E4M3) return no(&c->err, VVS_ESTATE, "kv_evict: the context was created with VVS_CACHE_SAME");
  if (!c->prefilled) return no(&c->err, VVS_ESTATE, "kv_evict: call vvs_prefill first");
  if (c->verify_pending) return no(&c->err, VVS_ESTATE, "kv_evict: the previous verify was not committed");
  if (keep < kQBlock || keep % kQBlock) return no(&c->err, VVS_EINVAL, "kv_evict: keep must be a positive multiple of VVS_QCACHE_BLOCK");
  if (recent < 0 || recent > keep) return no(&c->err, VVS_EINVAL, "kv_evict: recent must be in [0, keep]");
  launch_evict(c, keep, recent, (hipStream_t)s);
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return VVS_OK;
  c->err = std::string("kv_evict: ") + hipGetErrorString(e);
  return VVS_EHIP;
}

vvs_status vvs_rope_create(const vvs_rope_config* cfg, vvs_rope** out) {
  if (!out) return no(nullptr, VVS_EINVAL, "rope create: out is NULL");
  *out = nullptr;
  if (!cfg) return no(nullptr, VVS_EINVAL, "rope create: config is NULL");
  const vvs_rope_config& g = *cfg;
  if (g.dtype != VVS_FP32 && g.dtype != VVS_BF16) return no(nullptr, VVS_EINVAL, "rope config: unknown dtype");
  if (g.series != VVS_ROPE_OWN && g.series != VVS_ROPE_SHARED) return no(nullptr, VVS_EINVAL, "rope config: unknown series");
  if (g.pairing != VVS_ROPE_ADJACENT && g.pairing != VVS_ROPE_HALVES) return no(nullptr, VVS_EINVAL, "rope config: unknown pairing");
  if (!(g.base > 1.f) || !std::isfinite(g.base)) return no(nullptr, VVS_EINVAL, "rope config: base must be above 1 and finite");
  if (g.head_size < 8 || g.head_size > 256 || g.head_size % 8) return no(nullptr, VVS_ESIZE, "rope config: head size must be a multiple of 8, at most 256");
  if (g.n_axes < 1 || g.n_axes > VVS_ROPE_MAX_AXES) return no(nullptr, VVS_ESIZE, "rope config: 1 to VVS_ROPE_MAX_AXES axes");
  int sum = 0;
  for (int i = 0; i < g.n_axes; ++i) {
    if (g.pairs[i] < 1 || g.pairs[i] > g.head_size / 2) return no(nullptr, VVS_EINVAL, "rope config: an axis has between 1 and head_size / 2 pairs");
    sum += g.pairs[i];
  }
  if (sum > g.head_size / 2) return no(nullptr, VVS_EINVAL, "rope config: more pairs than the head has");
  if (sum % (g.pairing == VVS_ROPE_HALVES ? 8 : 4)) return no(nullptr, VVS_ESIZE, "rope config: the sum of pairs must be a multiple of 4 (of 8 with VVS_ROPE_HALVES)");
  Rope* r = new (std::nothrow) Rope{};
  if (!r) return no(nullptr, VVS_EHIP, "rope create: out of memory");
  r->cfg = g;
  RopeArgs& a = r->args;
  a.dh = g.head_size; a.axes = g.n_axes; a.pairs = sum; a.halves = g.pairing == VVS_ROPE_HALVES;
  int j = 0;
  for (int ax = 0; ax < g.n_axes; ++ax)
    for (int i = 0; i < g.pairs[ax]; ++i, ++j) {
      a.axis[j] = (uint8_t)ax;
      const double part = g.series == VVS_ROPE_SHARED ? 2.0 * j / g.head_size : (double)i / g.pairs[ax];
      a.turns[j] = pow((double)g.base, -part) / (2.0 * M_PI);
    }
  *out = reinterpret_cast<vvs_rope*>(r);
  return VVS_OK;
}

void vvs_rope_destroy(vvs_rope* r) { delete reinterpret_cast<Rope*>(r); }

const char* vvs_rope_last_error(const vvs_rope* r) { return r ? reinterpret_cast<const Rope*>(r)->err.c_str() : ""; }

vvs_status vvs_rope_apply(vvs_rope* rope, int32_t n_tokens, const int32_t* d_pos, int32_t n_heads, const void* d_q, int64_t q_stride, void* d_q_out,
                          int64_t q_out_stride, int32_t n_kv_heads, const void* d_k, int64_t k_stride, void* d_k_out, int64_t k_out_stride, int32_t inverse,
                          vvs_stream s) {
  Rope* r = reinterpret_cast<Rope*>(rope);
  if (!r) return VVS_EINVAL;
  const vvs_rope_config& g = r->cfg;
  if (!d_pos || !d_q || !d_q_out) return no(&r->err, VVS_EINVAL, "rope: NULL argument");
  if (n_tokens < 1 || n_heads < 1 || n_kv_heads < 0) return no(&r->err, VVS_EINVAL, "rope: n_tokens and n_heads must be positive, n_kv_heads not negative");
  if (n_heads > 4096 || n_kv_heads > 4096) return no(&r->err, VVS_ESIZE, "rope: at most 4096 heads");
  if (n_tokens > kMostUnits) return no(&r->err, VVS_ESIZE, "rope: at most 2^26 - 4 tokens");
  if (n_kv_heads ? !d_k || !d_k_out : d_k || d_k_out) return no(&r->err, VVS_EINVAL, "rope: d_k, d_k_out and n_kv_heads go together");
  if (inverse != 0 && inverse != 1) return no(&r->err, VVS_EINVAL, "rope: inverse must be 0 or 1");
  const int64_t per = (int64_t)n_heads * g.head_size, kper = (int64_t)n_kv_heads * g.head_size;
  const int64_t qs = stride_of(q_stride, per, g.dtype), qo = stride_of(q_out_stride, per, g.dtype);
  const int64_t ks = stride_of(k_stride, kper, g.dtype), ko = stride_of(k_out_stride, kper, g.dtype);
  if (qs < 0 || qo < 0 || ks < 0 || ko < 0 || unaligned(d_q) || unaligned(d_q_out) || unaligned(d_k) || unaligned(d_k_out) || ((uintptr_t)d_pos & 3))
    return no(&r->err, VVS_EINVAL, "rope: pointers and strides must be multiples of 16 bytes, strides cover a token");
  if ((d_q == d_q_out && qs != qo) || (d_k && d_k == d_k_out && ks != ko)) return no(&r->err, VVS_EINVAL, "rope: in place, both strides are the same");
  RopeArgs a = r->args;
  a.pos = d_pos; a.q = d_q; a.k = d_k; a.q_out = d_q_out; a.k_out = d_k_out;
  a.q_stride = (size_t)qs; a.q_out_stride = (size_t)qo; a.k_stride = (size_t)ks; a.k_out_stride = (size_t)ko;
  a.M = n_tokens; a.heads = n_heads; a.kv_heads = n_kv_heads; a.inverse = inverse;
  launch_rope_axes(a, g.dtype, (hipStream_t)s);
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return VVS_OK;
  r->err = std::string("rope: ") + hipGetErrorString(e);
  return VVS_EHIP;
}

}  // extern "C"
