"""A decoder layer with weights and their operands in 8 bits in 64 bits, over one token per row, from its embedding to the rows in 8 bits that the layer behind it starts with; with one of its rounding points
or a part of a contraction left out, for controls."""
import numpy as np
import torch

import qlinear_common as ql
from oracle import vvs_oracle as vo

MATRICES = ("wk", "wv", "wo", "wg", "wu", "wd")
# rounding points behind the values, and blocks of 128 contraction values of a matrix
LEFT_OUT = ("attention", "norm 2", "activations", "weights", "wo", "wg", "wu", "wd")


def held(x):
    return ql.held(torch.from_numpy(np.ascontiguousarray(x)))[0].numpy()


class Layer:
    """left_out: one of LEFT_OUT - a rounding point, that of the weights, or a matrix whose second block of contraction values is taken as zero.  noise: relative, in front of the roundings to 8 bits: what the
    sums in front of them are off by."""

    def __init__(self, shape, w, left_out=None, noise=0.0, seed=5):
        self.eps, self.left_out, self.noise, self.rng = shape.rms_eps, left_out, noise, np.random.default_rng(seed)
        self.g = [np.asarray(w[k], dtype=np.float64) for k in ("l0.g1", "l0.g2", "l1.g1")]
        self.m = {}
        for k in MATRICES:
            v = np.asarray(w[f"l0.{k}"], dtype=np.float64)
            self.m[k] = v if left_out == "weights" else held(v.T).T
            if left_out == k:
                self.m[k] = self.m[k].copy()
                self.m[k][128:256] = 0

    def r8(self, x, point=None, exact=False):
        if self.noise and not exact:
            x = x * (1 + self.noise * self.rng.standard_normal(x.shape))
        return x if point and self.left_out == point else held(x)

    def first_rows(self, x):
        """[R, d] embeddings -> the first norm's rows, from which keys and values are made."""
        return self.r8(vo.rmsnorm(x, self.g[0], self.eps))

    def rows_behind(self, x, v):
        """x [R, d], v [R, d]: the values as they are cached.  A token that sees itself alone has them as its attention's output, without a rounding of its own."""
        x = x + self.r8(v, "attention", exact=True) @ self.m["wo"]
        h = self.r8(vo.rmsnorm(x, self.g[1], self.eps), "norm 2")
        x = x + self.r8(vo.silu(h @ self.m["wg"]) * (h @ self.m["wu"]), "activations") @ self.m["wd"]
        return self.r8(vo.rmsnorm(x, self.g[2], self.eps))


def stage_weights(shape, std=0.05, gain_jitter=0.2):
    """Weights of two layers, the second of which has as its values its norm's rows themselves: a unit matrix for them, and gains of 1."""
    from paper_2511_13587_amd import synth
    w = synth.make_weights(shape, std=std, gain_jitter=gain_jitter)
    w["l1.wv"] = np.eye(shape.d_model, dtype=np.float32)
    w["l1.g1"] = np.ones(shape.d_model, dtype=np.float32)
    return w


def embeddings(shape, pc, pu):
    """[R, d] of a prefill with a dense prefix of one token."""
    x = np.empty((shape.n_rows, shape.d_model))
    x[0::2], x[1::2] = pc[:, 0], pu[0]
    return x


# Share of the rows' elements behind the layer that may be a step off: sums in fp32 are off by 5e-7 of themselves at most, those of the matrix instructions for e4m3 by some 1.3e-5; what that makes of the
# elements is measured in tests/test_weights8_controls.py with 5e-7 and 2e-5 (0.2 % and 9 % at most, over four shapes of 256 to 2048), beside layers with something left out (from 23 % on).
MOST_OFF = 0.02
MOST_OFF_E4M3 = 0.15
