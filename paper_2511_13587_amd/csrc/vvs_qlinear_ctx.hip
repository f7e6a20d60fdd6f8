// Weights in 8 bits inside a context: what the forward of a VVS_WEIGHTS_E4M3 or VVS_WEIGHTS_E4M3_WHOLE context launches.  The operators are those of vvs_qrows.hip and vvs_qlinear.hip; here they get the context's buffers.
// A layer is nine launches: norm into 8 bits, q|k|v, rotary positions and cache, attention, rounding, O, norm, gate|up, down.  Bound by the weights' bytes where they are large (7B shape, 14 rows, us per layer: gate|up 26.0, q|k|v
// 14.6, down 15.0, O 9.2, attention 13.2, two norms 8.0, positions and cache 5.1, rounding 3.9), else by the launches: narrower shapes, whose layers run in few launches with weights in bf16, take longer in
// 8 bits (us per step, bf16 / 8 bits: 7B shape 1 token 3104 / 2592, 2 x 7 tokens 3304 / 3171, 16 x 7 6740 / 6211; 1280 wide, 8 x 27 tokens 2279 / 3073, 32 x 61 9187 / 8973; 768 wide, 4 x 6 tokens 286 / 509).
#include "vvs_device.h"
#include "vvs_qlinear.h"

namespace vvs {

static QWeights map_of(const Ctx* c, int layer, QMap m) {
  const size_t at = m == kMapQkv ? c->p.wqkv : m == kMapO ? c->p.wo : m == kMapGate ? c->p.wgu : c->p.wd;
  return context_map(c, m, c->pw + c->p.layer0 + c->p.layer_stride * layer + at);
}

// q, k and v are one map whose columns come from three tensors: each its own run of groups (d is a multiple of 64)
void launch_context_load(Ctx* c, int layer, const void* const* t, hipStream_t s) {
  const QWeights qkv = map_of(c, layer, kMapQkv);
  for (int i = 0; i < 3; ++i) {
    QWeights part = qkv;
    part.out = c->d; part.groups = c->d / 64;
    part.data += qkv.tile_at(i * part.groups, 0, 0);
    part.powers += qkv.power_at(i * part.groups, 0, 0);
    launch_qlinear_load(QLoad{part, t[1 + i], nullptr, c->cfg.dtype}, s);
  }
  launch_qlinear_load(QLoad{map_of(c, layer, kMapO), t[4], nullptr, c->cfg.dtype}, s);
  launch_qlinear_load(QLoad{map_of(c, layer, kMapGate), t[6], t[7], c->cfg.dtype}, s);
  launch_qlinear_load(QLoad{map_of(c, layer, kMapDown), t[8], nullptr, c->cfg.dtype}, s);
}

static QRowsOut rows_of(const Ctx* c) { return QRowsOut{(uint8_t*)c->ws + c->w.h8, (uint8_t*)c->ws + c->w.h8_powers}; }

void launch_context_norm(Ctx* c, int M, const float* gain, const float* delta, hipStream_t s) {
  QNorm a{};
  a.M = M; a.width = c->d;
  a.x = c->ws + c->w.x; a.x_dtype = VVS_FP32; a.x_stride = c->d; a.x_wide = 1;
  a.delta = delta; a.delta_dtype = VVS_FP32; a.delta_stride = c->d; a.delta_wide = 1;
  if (delta) { a.x_out = c->ws + c->w.x; a.x_out_stride = c->d; a.x_out_wide = 1; }
  a.gain = gain; a.gain_dtype = VVS_FP32; a.gain_wide = 1;
  a.eps = c->cfg.rms_eps; a.per_element = 1.0 / c->d;
  a.y = rows_of(c);
  launch_qrows_norm(a, s);
}

void launch_context_round(Ctx* c, int M, hipStream_t s) {
  QRound a{};
  a.M = M; a.width = c->d; a.dtype = c->cfg.dtype;
  a.x = c->ws + c->w.attn; a.stride = c->d; a.wide = 1;
  a.packed = c->cfg.dtype == VVS_BF16;
  a.y = rows_of(c);
  launch_qrows_round(a, s);
}

void launch_context_product(Ctx* c, int layer, QMap m, int M, float* out, hipStream_t s) {
  const QRowsOut h = rows_of(c), act{(uint8_t*)c->ws + c->w.act8, (uint8_t*)c->ws + c->w.act8_powers};
  QProduct a{};
  a.w = map_of(c, layer, m); a.M = M;
  a.x = m == kMapDown ? QRowsIn{act.values, act.powers} : QRowsIn{h.values, h.powers};
  // (the sums go on in fp32, but what they are of was rounded to 2^-4, and in bf16 contexts what comes of them is to 2^-9)
  a.dtype = VVS_FP32; a.fast = qlinear_fast(c->cfg.weight_kind == VVS_WEIGHTS_E4M3_WHOLE ? VVS_PRODUCTS_WHOLE : VVS_PRODUCTS_AUTO, m == kMapGate ? VVS_BF16 : c->cfg.dtype, M);
  a.y = out; a.stride = a.w.out; a.wide = 1;
  a.y8 = act;
  a.counters = (uint32_t*)(c->ws + c->w.map_counters); a.act = (float*)(c->ws + c->w.map_parts);
  launch_qlinear_product(a, plan_qlinear_product(a.w, M, a.fast), s);
}

}  // namespace vvs
