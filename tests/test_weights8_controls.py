"""The comparison that tests/test_gpu_weights8_stages.py makes tells a layer in 8 bits from one with a rounding point, or 128 values of a contraction, left out: by the 64-bit layer alone."""
import numpy as np
import pytest

import weights8_common as wc
from oracle import vvs_oracle as vo
from paper_2511_13587_amd import synth

BASE = synth.XL_TREE.replace(n_layers=2, prefix_len=1, grid_h=4, grid_w=4, vocab=1024, logit_hi=1024, n_prompts=20)


@pytest.mark.parametrize("shape", [BASE.replace(d_model=320, n_heads=5, d_ff=704), BASE.replace(d_model=256, n_heads=4, d_ff=688, dtype=synth.DTYPE_FP32)], ids=["bf16", "fp32"])
def test_controls(shape):
    w = wc.stage_weights(shape)
    x = wc.embeddings(shape, *synth.make_prefix(shape))
    layer = wc.Layer(shape, w)
    v = layer.first_rows(x) @ layer.m["wv"]
    v = vo.round_bf16(v) if shape.dtype == synth.DTYPE_BF16 else v
    want = layer.rows_behind(x, v)
    off = lambda **kw: np.mean(wc.Layer(shape, w, **kw).rows_behind(x, v) != want)  # noqa: E731
    for seed in range(3):
        assert off(noise=5e-7, seed=seed) < wc.MOST_OFF / 2
        assert off(noise=2e-5, seed=seed) < wc.MOST_OFF_E4M3 / 2
    for what in wc.LEFT_OUT:
        assert off(left_out=what) > 1.5 * wc.MOST_OFF_E4M3, what
