"""Attention over the 8-bit cache where softmax weights and values span many powers of two: no key's part in an output may be lost beside larger ones.

Tolerance, per output element, relative to what the element is made of, S = sum of weight * |value|: a weight is off by 2 * size * 2^-24 * sum |q k| (its own score and the normaliser's) and by the
2^-20 of exponentials and sums; bf16 calls round it to 2^-17 for the product, fp32 calls to 2^-24; n terms added up in fp32, in any order, are off by n * 2^-24 of S at most, the normaliser by as much
relative to itself.  The output is rounded once more, by 2^-8 (bf16) or 2^-24 (fp32) of itself.  Scores are sums of few bf16 and e4m3 numbers here, so that sum |q k| is small where
weights lie far apart."""
import copy

import numpy as np
import pytest
import torch

import qcache_common as qc
from test_gpu_qcache import Both, ints, near, np64

pytestmark = pytest.mark.gpu

SIZE = 64
LN2 = float(np.log(2.0))


def made_of(both, r, length, q, k, v, see):
    """(output, sum of weight * |value|, largest sum of |score products|) of a row in 64 bits."""
    y, _, _, _, top_s, _ = both.ref.attend(0, r, length, q, k, v, see, SIZE ** -0.5, 0)
    sizes = copy.copy(both.ref)
    sizes.v = np.abs(both.ref.v)
    s = sizes.attend(0, r, length, q, k, None if v is None else np.abs(v), see, SIZE ** -0.5, 0)[0]
    return y, s, top_s


def check(both, lens, q, k, v):
    rows, tokens = q.shape[:2]
    out = torch.full(q.shape, 3.0, dtype=both.dtype, device="cuda")
    both.gpu.vvs_qcache_attention(ints(lens), q, k, v, out)
    see = qc.ancestors(None, tokens)
    for r in range(rows):
        y, s, top_s = made_of(both, r, lens[r], np64(q[r]), None if k is None else np64(k[r]), None if v is None else np64(v[r]), see)
        terms = lens[r] + (0 if k is None else tokens)
        bf16 = both.dtype == torch.bfloat16
        part = 2 * SIZE * 2.0 ** -24 * top_s + 2.0 ** -20 + 2 * terms * 2.0 ** -24 + (2.0 ** -17 if bf16 else 2.0 ** -24)
        near(np64(out[r]), y, part * s + (2.0 ** -8 if bf16 else 2.0 ** -23) * np.abs(y))


def biased(rng, rows, tokens, length, dtype, gain, bias, heads=2):
    """Values of 2^gain[block] (None: zeros) and keys whose scores lie bias[block] powers of two above the others': the last dim of every query is 1, the others make up a score of little size."""
    n_blocks = -(-length // 32)
    shape = (1, rows, length, 1, SIZE)
    v, k = rng.standard_normal(shape), rng.standard_normal(shape) * 0.25
    for b in range(n_blocks):
        at = slice(b * 32, min((b + 1) * 32, length))
        v[:, :, at] *= 0.0 if gain[b] is None else 2.0 ** gain[b]
        k[:, :, at, :, -1] = bias[b] * LN2 * SIZE ** 0.5
    q = rng.standard_normal((rows, tokens, heads, SIZE)) * 0.25
    q[..., -1] = 1.0
    return [torch.from_numpy(x.astype(np.float32)).to("cuda", dtype) for x in (k, v, q)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("tokens,length", [(3, 640), (3, 1300), (20, 640), (60, 1300), (150, 640), (150, 1300)])
def test_blocks_of_zeros_take_nothing_from_small_values_behind_them(dtype, tokens, length):
    """Blocks without values (padding, tokens that an append took as zeros) have the smallest power of two there is.  Values of 2^-8, 2^-16, 2^-24 lie behind them, in all four waves' shares, and
    among them; in the last row the zeros have scores 2^10 above the others'."""
    rng = np.random.default_rng(tokens + length)
    n = -(-length // 32)
    both = Both(dtype, rows=4, heads=2, kv_heads=1, size=SIZE, capacity=length, max_tokens=tokens)
    zero = [b < 4 or b % 5 == 2 for b in range(n)]
    ks, vs, qs = [], [], []
    for r, g in enumerate((-8, -16, -24, -8)):
        k, v, q = biased(rng, 1, tokens, length, both.dtype, [None if z else g for z in zero], [10.0 if z and r == 3 else 0.0 for z in zero])
        ks.append(k), vs.append(v), qs.append(q)
    both.append([0] * 4, torch.cat(ks, dim=1), torch.cat(vs, dim=1))
    q = torch.cat(qs)
    lens = [length, length - 5, length - 32, length]
    check(both, lens, q, None, None)
    kk, vv = (torch.from_numpy((rng.standard_normal((4, tokens, 1, SIZE)) * 2.0 ** g).astype(np.float32)).to("cuda", both.dtype) for g in (-2, -20))
    check(both, lens, q, kk, vv)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("tokens,length", [(3, 640), (20, 1300), (150, 640)])
@pytest.mark.parametrize("power", [10, 18, 22, 26, 34])
def test_one_large_value_takes_nothing_from_other_dims(dtype, tokens, length, power):
    """One element of 2^power in the second block: what the other dims of the other blocks come to stays as it is."""
    rng = np.random.default_rng(power + tokens)
    n = -(-length // 32)
    both = Both(dtype, rows=2, heads=2, kv_heads=1, size=SIZE, capacity=length, max_tokens=tokens)
    k, v, q = biased(rng, 2, tokens, length, both.dtype, [0] * n, [0.0] * n)
    v[0, :, 40, 0, 5] = 2.0 ** power
    both.append([0, 0], k, v)
    check(both, [length, length - 3], q, None, None)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("tokens,length", [(2, 4096), (40, 1300), (150, 640)])
@pytest.mark.parametrize("above", [12, 20, 26, 40])
def test_a_key_without_value_leaves_the_others_their_parts(dtype, tokens, length, above):
    """A first token that attention goes to and that holds nothing: its score lies `above` powers of two over the others', whose small weights make up the whole output."""
    rng = np.random.default_rng(above + tokens)
    n = -(-length // 32)
    both = Both(dtype, rows=2, heads=2, kv_heads=1, size=SIZE, capacity=length, max_tokens=tokens)
    k, v, q = biased(rng, 2, tokens, length, both.dtype, [0] * n, [0.0] * n)
    v = v + 1.0                                        # outputs that do not cancel
    k[:, 0, 0, :, -1] = above * LN2 * SIZE ** 0.5       # row 0: the first slot; row 1: one in the middle
    k[:, 1, length // 2, :, -1] = above * LN2 * SIZE ** 0.5
    v[:, 0, 0], v[:, 1, length // 2] = 0.0, 0.0
    both.append([0, 0], k, v)
    check(both, [length, length], q, None, None)


@pytest.mark.parametrize("tokens", [1, 30, 64, 150])
def test_weights_keep_17_bits_beside_cached_values(tokens):
    """Two slots of opposite value and nearly equal score: what is left of them shows what rounding did to the weights."""
    rng = np.random.default_rng(tokens)
    both = Both("bf16", rows=8, heads=2, kv_heads=1, size=SIZE, capacity=64, max_tokens=tokens)
    k, v = (torch.zeros((1, 8, 2, 1, SIZE), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k[:, :, 1, 0, 0] = SIZE ** 0.5
    v[:, :, 0], v[:, :, 1] = 1.0, -1.0
    both.append([0] * 8, k, v)
    q = torch.zeros((8, tokens, 2, SIZE), dtype=torch.bfloat16, device="cuda")
    q[..., 0] = torch.from_numpy((rng.random((8, tokens, 2)) * 0.02).astype(np.float32)).cuda()
    check(both, [2] * 8, q, None, None)
