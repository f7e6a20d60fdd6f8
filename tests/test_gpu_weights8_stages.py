"""Contexts with weights in 8 bits stage by stage, one token per row: keys and values beside their products in 64 bits, and the rows in 8 bits that the second layer starts with - its values, by a unit
matrix - beside those of a layer in 64 bits.  What may be off is bound by what sums are off by, and controls that leave something out are far outside (tests/test_weights8_controls.py)."""
import numpy as np
import pytest
import torch

import qlinear_common as qc
import weights8_common as wc
from paper_2511_13587_amd import binding as vb
from paper_2511_13587_amd import synth
from test_gpu_qlinear import product_error

pytestmark = pytest.mark.gpu

BASE = synth.XL_TREE.replace(n_layers=2, prefix_len=1, grid_h=4, grid_w=4, vocab=1024, logit_hi=1024)
NARROW = BASE.replace(d_model=320, n_heads=5, d_ff=704)                        # 2.5 blocks of 128
WIDE = BASE.replace(d_model=2048, n_heads=16, d_ff=1408)
FP32 = BASE.replace(d_model=256, n_heads=4, d_ff=688, dtype=synth.DTYPE_FP32)
FP32_ODD = BASE.replace(d_model=192, n_heads=6, d_ff=520, dtype=synth.DTYPE_FP32)

# rows: of few-rows kernels, of every tile size that a context's products take; E4M3: e4m3 instructions where a call of these rows may take them, WHOLE: never
E4M3, WHOLE = vb.VVS_WEIGHTS_E4M3, vb.VVS_WEIGHTS_E4M3_WHOLE


@pytest.mark.parametrize("shape,rows,kind", [(NARROW, 10, E4M3), (NARROW, 40, E4M3), (NARROW, 202, E4M3), (NARROW, 202, WHOLE), (BASE, 46, E4M3), (BASE, 216, E4M3), (BASE, 216, WHOLE), (BASE, 434, E4M3),
                                             (BASE, 434, WHOLE), (BASE, 1690, E4M3), (BASE, 1690, WHOLE), (WIDE, 202, E4M3), (WIDE, 202, WHOLE), (FP32, 10, E4M3), (FP32, 202, E4M3), (FP32, 202, WHOLE), (FP32_ODD, 6, E4M3),
                                             (FP32_ODD, 130, E4M3), (FP32_ODD, 130, WHOLE)])
def test_stages(shape, rows, kind):
    shape = shape.replace(n_prompts=rows // 2)
    w = wc.stage_weights(shape)
    pc, pu = synth.make_prefix(shape)
    ctx = vb.Context(vb.make_config(shape, weight_kind=kind))
    ctx.load_weights_from_host(w, synth.weight_names(shape))
    out = torch.zeros(shape.n_prompts, dtype=torch.int32, device="cuda")
    ctx.vvs_prefill(vb.to_device(pc, shape.dtype), vb.to_device(pu, shape.dtype), None, torch.full((shape.n_prompts,), 0.5, device="cuda"), out)
    cached = [[y.double().cpu().reshape(-1) for y in ctx.vvs_debug_kv(layer, row, 1)] for layer in (0, 1) for row in range(rows)]
    k, v = (torch.stack([cached[row][i] for row in range(rows)]) for i in (0, 1))
    behind = torch.stack([cached[rows + row][1] for row in range(rows)])
    ctx.close()
    x = wc.embeddings(shape, pc, pu)
    layer = wc.Layer(shape, w)

    # the first norm's rows by the operator, beside 64 bits; then keys and values of just these rows
    r = vb.QRows(rows, shape.d_model)
    vb.vvs_qrows_norm(torch.from_numpy(x).float().cuda(), torch.from_numpy(w["l0.g1"]).cuda(), shape.rms_eps, r)
    y = torch.from_numpy(x / np.sqrt(np.mean(x * x, axis=1, keepdims=True) + shape.rms_eps) * layer.g[0])
    qc.check_rounded(r, y, y.abs() * 64 * 2.0 ** -24)
    h = qc.values_of(r)
    bf16 = shape.dtype == synth.DTYPE_BF16
    fast = kind == E4M3 and rows > 64
    half = 2.0 ** -8 if bf16 else 2.0 ** -24
    for got, name in ((k, "wk"), (v, "wv")):
        m = torch.from_numpy(np.ascontiguousarray(layer.m[name]))
        want = h @ m
        err = product_error(h, m, fast and bf16)
        worst = ((got - want).abs() - err - half * (want.abs() + err)).max().item()
        assert worst <= 0, (name, worst)

    # all of the layer behind the values.  (Unconditional rows are all the same: one of them)
    once = np.r_[0:rows:2, 1]
    want = layer.rows_behind(x[once], v.numpy()[once])
    off = np.mean(behind.numpy()[once] != want)
    assert off <= (wc.MOST_OFF_E4M3 if fast else wc.MOST_OFF), off
    assert (behind[1::2] == behind[1]).all()
