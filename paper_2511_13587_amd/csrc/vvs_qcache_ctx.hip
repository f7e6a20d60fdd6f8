// The 8-bit key/value cache inside a context: what the forward, the commit and the inspection of a VVS_CACHE_E4M3 context launch.  The operators are those of vvs_qcache.hip and
// vvs_rope.hip; here they get the context's buffers.
#include "vvs_device.h"
#include "vvs_qcache.h"

namespace vvs {

static QLayout layout_of(const Ctx* c) {
  return QLayout{c->R, c->H, c->H, c->dh, c->S_cap / kQBlock, (uint8_t*)c->kv, (float2*)(c->kv + c->q_scale)};
}

// Positions of the forward's tokens on both axes, once for all layers.  Prefix tokens are at (0, 0), where nothing turns.
__global__ void k_context_positions(int32_t* __restrict__ out, TreeDesc tree, PosDesc pos, int T, int M) {
  const int m = blockIdx.x * blockDim.x + threadIdx.x;
  if (m >= M) return;
  int slot, img;
  token_pos(pos, tree, m / T, m % T, &slot, &img);
  out[2 * m] = img >= 0 ? img / pos.grid_w : 0;
  out[2 * m + 1] = img >= 0 ? img % pos.grid_w : 0;
}

void launch_context_positions(Ctx* c, const TreeDesc& tree, const PosDesc& pos, int T, hipStream_t s) {
  const int M = c->R * T;
  hipLaunchKernelGGL(k_context_positions, dim3((M + 255) / 256), dim3(256), 0, s, (int32_t*)(c->ws + c->w.q_pos), tree, pos, T, M);
}

// Staged keys (and values, stage_v further on) of a layer: a verify call's layers lie behind each other, a prefill chunk uses the first one's place
static char* stage_of(const Ctx* c, int layer, int M) { return c->ws + c->w.q_stage + c->esz * (size_t)layer * M * c->d; }

void launch_context_rope(Ctx* c, int layer, int M, const float* sums, int splits, hipStream_t s) {
  RopeArgs a{};
  const bool fits = (size_t)(layer + 1) * M * c->d <= c->stage_v;
  char* k = stage_of(c, fits ? layer : 0, M);
  a.sums = sums; a.splits = splits; a.split_stride = (size_t)M * 3 * c->d;
  a.pos = (const int32_t*)(c->ws + c->w.q_pos);
  a.q_out = c->ws + c->w.q; a.k_out = k; a.v_out = k + c->esz * c->stage_v;
  a.M = M; a.heads = c->H; a.kv_heads = c->H; a.dh = c->dh; a.axes = 2; a.pairs = c->dh / 2;
  for (int j = 0; j < a.pairs; ++j) { a.turns[j] = c->rope_turns[j]; a.axis[j] = j >= a.pairs / 2; }
  launch_rope_axes(a, c->cfg.dtype, s);
}

void launch_context_attention(Ctx* c, int layer, const TreeDesc& tree, const PosDesc& pos, int T, hipStream_t s) {
  const int M = c->R * T;
  const bool verify = pos.kv_len != nullptr, fits = (size_t)(layer + 1) * M * c->d <= c->stage_v;
  char* k = stage_of(c, fits ? layer : 0, M);
  QAttention a{};
  a.c = layout_of(c);
  a.len = QLen{pos.kv_len, 1, pos.kv_base};
  a.layer = layer; a.T = T; a.group = 1;
  a.q = c->ws + c->w.q; a.k = k; a.v = k + c->esz * c->stage_v;
  a.q_stride = a.k_stride = a.v_stride = (size_t)c->d;
  a.c_exp = (float)(1.4426950408889634 / sqrt((double)c->dh));
  a.out = c->ws + c->w.attn;
  a.packed = c->cfg.dtype == VVS_BF16;
  a.capacity = c->S_cap;
  // weights of a prefill's tokens, over the cache and over each other; of a verify call's certain tokens, over the cache
  float* mass = (float*)(c->kv + c->q_mass) + (size_t)layer * c->R * c->H * c->S_cap;
  a.mass = mass;
  a.n_counted = verify ? 1 + tree.n_forced : T;
  if (!verify) { a.block_mass = mass + pos.kv_base; a.block_stride = c->S_cap; }
  a.norm = (float*)(c->ws + c->w.q_norm);
  a.parts = (float*)(c->ws + c->w.q_parts);
  a.scores = (float*)(c->ws + c->w.q_scores);
  a.score_steps = qcache_score_steps(c->S_cap / kQBlock, c->Tmax > c->chunk ? c->Tmax : c->chunk);
  a.causal = tree.causal;
  for (int t = 0; t < VVS_MAX_T; ++t) a.anc[t] = tree.anc[t];
  launch_qcache_attention(a, c->cfg.dtype, s);
  if (verify) return;
  QAppend p{};                 // a prefill's tokens are cached at once
  p.c = a.c;
  p.len = a.len;
  p.layer = layer; p.n_layers = 1; p.n = T; p.src_tokens = T;
  p.k = a.k; p.v = a.v; p.stride[0] = p.stride[1] = (size_t)c->d;
  p.capacity = c->S_cap;
  p.pos = (int32_t*)(c->kv + c->q_slot_pos);
  launch_qcache_append(p, c->cfg.dtype, s);
}

// The pending token and the accepted path of the last verify, of all layers.  Lengths and emitted tokens as the verify found them.
void launch_context_append(Ctx* c, hipStream_t s) {
  const int32_t* oc = (const int32_t*)(c->ws + c->w.outcome);
  const int T = c->last_T;
  QAppend p{};
  p.c = layout_of(c);
  p.len = QLen{oc + kOutcomeSnap * c->B, 1, 0};
  p.layer = 0; p.n_layers = c->L; p.n = T; p.src_tokens = T;
  p.n_tokens = oc; p.n_shift = 1; p.count_plus = 1;
  p.select = oc + 2 * c->B; p.select_stride = VVS_MAX_T; p.select_shift = 1;
  p.skip = oc + c->B;
  p.k = c->ws + c->w.q_stage; p.v = c->ws + c->w.q_stage + c->esz * c->stage_v;
  p.stride[0] = p.stride[1] = (size_t)c->d; p.layer_stride[0] = p.layer_stride[1] = (size_t)c->R * T * c->d;
  p.capacity = c->S_cap;
  p.mass = (float*)(c->kv + c->q_mass);
  p.pos = (int32_t*)(c->kv + c->q_slot_pos);
  p.pos_base = oc + (kOutcomeSnap + 1) * c->B; p.pos_add = c->P - 1;
  launch_qcache_append(p, c->cfg.dtype, s);
}

__global__ void k_shorten(int32_t* __restrict__ len, int B, int keep) {
  const int b = blockIdx.x * blockDim.x + threadIdx.x;
  if (b < B) len[b] = min(len[b], keep);
}

void launch_evict(Ctx* c, int keep, int recent, hipStream_t s) {
  QEvict a{};
  a.c = layout_of(c);
  a.len = QLen{(const int32_t*)(c->ws + c->w.state), 1, 0};
  a.layer = 0; a.n_layers = c->L; a.keep = keep; a.recent = recent; a.capacity = c->S_cap;
  a.mass_out = (float*)(c->kv + c->q_mass);
  a.mass = a.mass_out;
  a.pos_out = (int32_t*)(c->kv + c->q_slot_pos);
  a.pos = a.pos_out;
  a.origin = (int32_t*)(c->ws + c->w.q_origin);
  Timed timed(c, VVS_K_COMMIT, s);
  launch_qcache_evict(a, s);
  hipLaunchKernelGGL(k_shorten, dim3((c->B + 255) / 256), dim3(256), 0, s, (int32_t*)(c->ws + c->w.state), c->B, keep);
}

void launch_context_read(Ctx* c, int layer, int row, int n_slots, float* dk, float* dv, hipStream_t s) {
  QRead a{};
  a.c = layout_of(c);
  const size_t first = a.c.region(layer, row, 0) * a.c.blocks;       // as a cache of one row
  a.c.rows = 1;
  a.c.data += first * a.c.block_bytes();
  a.c.scale += first;
  a.len = QLen{nullptr, 0, c->S_cap};
  a.n_layers = 1; a.n = n_slots; a.capacity = c->S_cap;
  a.k = dk; a.v = dv;
  launch_qcache_read(a, VVS_FP32, s);
}

}  // namespace vvs
