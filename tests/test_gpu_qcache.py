"""The 8-bit key/value cache on the GPU against its plain 64-bit statement: what is held, attention over it, eviction.

Tolerances.  What the cache holds is defined to the bit, so append, read and eviction are compared for equality.  Attention: a score is a sum of `size`
products in fp32, off by at most size * 2^-24 * sum |q k|; a softmax weight is off by twice that (its own score and the normaliser) relative to itself, by the
2^-22 of the exponential, and by the rounding of the weight in the value product (bf16 calls 2^-17, fp32 calls 2^-24), so that a sum of weights times values is off by at most
their sum times the largest value; 2^-20 covers the sums of weights.  The bf16 output is rounded once, by 2^-8 of itself at most."""
import math

import numpy as np
import pytest
import torch

import qcache_common as qc
from paper_2511_13587_amd import binding as vb

pytestmark = pytest.mark.gpu

DTYPES = {"bf16": (vb.VVS_BF16, torch.bfloat16), "fp32": (vb.VVS_FP32, torch.float32)}


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def np64(t):
    return t.double().cpu().numpy()


def values(rng, dims, dtype, spread=1.5):
    """Normal values with dimensions of different size, rounded to the type; as a device tensor."""
    x = rng.standard_normal(dims) * np.exp2(rng.standard_normal(dims[-2:]) * spread)
    return torch.from_numpy(x.astype(np.float32)).to("cuda", dtype)


class Both:
    """A cache on the GPU and its statement, filled with the same tensors."""

    def __init__(self, dtype, layers=1, rows=2, heads=4, kv_heads=2, size=64, capacity=256, max_tokens=64):
        self.code, self.dtype = DTYPES[dtype]
        self.layers, self.rows, self.heads, self.kv_heads, self.size, self.capacity = layers, rows, heads, kv_heads, size, capacity
        self.gpu = vb.QCache(layers, rows, heads, kv_heads, size, capacity, max_tokens, self.code)
        self.ref = qc.Cache(layers, rows, kv_heads, capacity, size)

    def append(self, lens, k, v, counts=None, select=None, layer=0):
        self.gpu.vvs_qcache_append(ints(lens), k, v, n_tokens=None if counts is None else ints(counts), select=None if select is None else ints(select),
                                   layer=layer, n_layers=k.shape[0])
        kk, vv = np64(k), np64(v)
        for l in range(k.shape[0]):
            for r in range(self.rows):
                pick = list(range(k.shape[2])) if select is None else select[r]
                if counts is not None:
                    pick = pick[:max(0, counts[r])]
                take = [[x[l, r, t] if 0 <= t < k.shape[2] else np.zeros_like(x[l, r, 0]) for t in pick] for x in (kk, vv)]
                if pick:
                    self.ref.append(layer + l, r, lens[r], np.stack(take[0]), np.stack(take[1]))

    def fill(self, rng, lens, layer=0, n_layers=1, spread=1.5):
        n = max(max(lens), 1)
        k, v = (values(rng, (n_layers, self.rows, n, self.kv_heads, self.size), self.dtype, spread) for _ in range(2))
        self.append([0] * self.rows, k, v, counts=lens, layer=layer)

    def check_held(self, lens, layer=0, n_layers=1, first=None, n=None):
        n = n or max(max(lens), 1)
        dims = (n_layers, self.rows, n, self.kv_heads, self.size)
        k, v = torch.full(dims, 7.0, dtype=self.dtype, device="cuda"), torch.full(dims, 7.0, dtype=self.dtype, device="cuda")
        self.gpu.vvs_qcache_read(ints(lens), k, v, first=None if first is None else ints(first), layer=layer, n_layers=n_layers)
        for got, held in ((np64(k), self.ref.k), (np64(v), self.ref.v)):
            for r in range(self.rows):
                f = 0 if first is None else first[r]
                for j in range(n):
                    s = f + j
                    want = held[layer:layer + n_layers, r, :, s] if 0 <= s < min(lens[r], self.capacity) else 0.0 * held[layer:layer + n_layers, r, :, 0]
                    want = np.where(np.isfinite(want) | (s < lens[r]), want, 0.0)
                    with np.errstate(over="ignore"):               # exact in the cache's type, but for what rounds up to 2^128
                        want = want.astype(np.float32)
                    np.testing.assert_array_equal(got[:, r, j], want, err_msg=f"row {r} slot {s}")

    def attend(self, lens, q, k, v, parent=None, counts=None, scale=None, counted=0, layer=0, tree_mask=None):
        """Runs the call into marked buffers and compares everything it writes; returns the output tensor."""
        rows, T, H, D = q.shape
        out = torch.full((rows, T, H, D), 3.0, dtype=self.dtype, device="cuda")
        lse = torch.full((rows, T, H), 3.0, device="cuda")
        rng = np.random.default_rng(99)
        mass = torch.from_numpy(rng.random((rows, self.kv_heads, self.capacity)).astype(np.float32)).cuda() if counted else None
        before = None if mass is None else np64(mass)
        block = torch.full((rows, self.kv_heads, T), 3.0, device="cuda") if counted and k is not None else None
        self.gpu.vvs_qcache_attention(ints(lens), q, k, v, out, n_tokens=None if counts is None else ints(counts), parent=parent, scale=scale, lse=lse,
                                      n_counted=counted, mass=mass, block_mass=block, layer=layer, tree_mask=tree_mask)
        see = qc.ancestors(parent, T)
        sc = D ** -0.5 if scale is None else scale
        for r in range(rows):
            n, t = min(max(lens[r], 0), self.capacity), T if counts is None else min(max(counts[r], 0), T)
            with np.errstate(invalid="ignore", over="ignore"):
                y, z, m, b, top_s, top_v = self.ref.attend(layer, r, n, np64(q[r, :t]), None if k is None else np64(k[r, :t]), None if v is None else np64(v[r, :t]),
                                                           see[:t, :t], sc, counted)
            weight = 2 * D * 2.0 ** -24 * top_s + 2.0 ** -20
            got = np64(out[r])
            near(got[:t], y, weight * top_v + (2.0 ** -17 * top_v + 2.0 ** -8 * np.abs(y) if self.dtype == torch.bfloat16 else 2.0 ** -23 * np.abs(y)))
            assert (got[t:] == 3.0).all(), "tokens behind the row's number were written"
            near(np64(lse[r, :t]), z, weight + 2.0 ** -22 * np.abs(z))
            assert (np64(lse[r, t:]) == 3.0).all()
            if counted:
                per = self.heads // self.kv_heads * min(counted, t)
                near(np64(mass[r])[:, :n], before[r][:, :n] + m, weight * (per * 0 + m) + 2.0 ** -22 * (1 + m))
                assert (np64(mass[r])[:, n:] == before[r][:, n:]).all(), "weights behind the length were touched"
                if block is not None:
                    near(np64(block[r])[:, :t], b, weight * b + 2.0 ** -22)
                    assert (np64(block[r])[:, t:] == 3.0).all()
        return out


def near(got, want, tol):
    with np.errstate(invalid="ignore"):
        bad = ~((np.abs(got - want) <= tol) | (got == want) | (np.isnan(got) & np.isnan(want)))
    assert not bad.any(), f"{int(bad.sum())} of {bad.size} off; first at {np.argwhere(bad)[0]}: got {got[bad][0]}, want {want[bad][0]}, allowed {np.broadcast_to(tol, got.shape)[bad][0]}"


def tree(rng, n, wide=3):
    return np.asarray([int(rng.integers(max(0, j - wide), j)) for j in range(1, n)], dtype=np.int32)


# ------------------------------------------------------------------------------------------------ what is held
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size,kv_heads", [(32, 1), (64, 3), (128, 2)])
def test_appended_values_are_rounded_as_defined(dtype, size, kv_heads):
    rng = np.random.default_rng(size + kv_heads)
    both = Both(dtype, layers=2, rows=3, heads=kv_heads, kv_heads=kv_heads, size=size, capacity=160)
    lens = [0, 0, 0]
    # blocks begun and continued, with larger, smaller and zero values to follow; nothing of a row; more than fits
    for counts, gain in (([1, 31, 32], 1.0), ([33, 2, 0], 300.0), ([7, 0, 40], 1e-3), ([40, 40, 1], 0.0), ([40, 40, 40], 2.0), ([45, 45, 45], 1.0), ([9, 9, 9], 1.0)):
        n = max(counts)
        k, v = (values(rng, (2, 3, n, kv_heads, size), both.dtype) * gain for _ in range(2))
        both.append(lens, k, v, counts=counts)
        lens = [min(160, a + b) for a, b in zip(lens, counts)]
        both.check_held(lens, n_layers=2)


def test_paths_are_appended_to_all_layers():
    rng = np.random.default_rng(1)
    both = Both("bf16", layers=3, rows=4, capacity=96)
    both.fill(rng, [40, 1, 31, 64], n_layers=3)
    k, v = (values(rng, (3, 4, 27, 2, 64), both.dtype) for _ in range(2))
    # (the same token twice, and tokens that the block does not have, are taken as asked)
    both.append([40, 1, 31, 64], k, v, counts=[5, 1, 0, 7],
                select=[[0, 3, 9, 10, 26, 0, 0], [4] * 7, [0] * 7, [0, 0, 5, -1, 27, 26, 1]])
    both.check_held([45, 2, 31, 71], n_layers=3)


def test_appended_parts_of_one_projection_and_windows_of_a_read():
    rng = np.random.default_rng(2)
    both = Both("bf16", rows=2, kv_heads=2, size=64, capacity=100)
    wide = values(rng, (1, 2, 50, 8, 64), both.dtype)
    k, v = wide[:, :, :, 4:6], wide[:, :, :, 6:8]
    both.append([3, 33], k, v)
    both.check_held([53, 83], first=[20, -5], n=70)
    both.check_held([100, 100], first=[90, 2000], n=20)
    both.append([99, 77], k, v)                                     # one fits, 23 fit
    both.check_held([100, 100])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_elements_at_the_ends_of_the_range(dtype):
    both = Both(dtype, rows=1, heads=1, kv_heads=1, size=32, capacity=128)
    dt = both.dtype
    k = torch.zeros((1, 1, 96, 1, 32), dtype=dt, device="cuda")
    v = torch.zeros_like(k)
    k[0, 0, 0, 0, :6] = torch.tensor([math.inf, -math.inf, math.nan, 3.0, 448.0, -0.25], dtype=dt)      # not finite: NaN, the others as without them
    k[0, 0, 33, 0, :3] = torch.tensor([3.3e38, -1e38, 1e-30], dtype=dt)
    k[0, 0, 64, 0, :4] = torch.tensor([1e-38, 2e-38, 1e-34, -3e-33], dtype=dt)                           # below 2^-110 * 2^-9: zeros
    v[0, 0, 0, 0, :5] = torch.tensor([448.0, 449.0, 2.0 ** -7, 1.5 * 2.0 ** -9, 2.0 ** -11], dtype=dt)   # subnormal e4m3, ties
    v[0, 0, 32, 0, :4] = torch.tensor([1.0625, 1.1875, -1.0625, 1.0], dtype=dt)                          # ties to even
    v[0, 0, 64, 0, :2] = torch.tensor([math.nan, math.inf], dtype=dt)                                    # a block of zeros and NaN
    both.append([0], k, v)
    both.check_held([96])


# ------------------------------------------------------------------------------------------------ attention
SHAPES = [
    # dtype, heads, kv heads, size, tokens, tree, lengths, counts, counted
    ("bf16", 4, 4, 64, 1, False, [0, 1, 31, 32, 33, 100], None, 1),
    ("bf16", 4, 2, 64, 6, False, [129, 5, 0, 64], None, 0),
    ("bf16", 4, 1, 64, 27, True, [200, 7, 96, 0], [27, 13, 1, 0], 1),
    ("bf16", 2, 2, 64, 64, True, [70, 31], None, 64),
    ("bf16", 8, 2, 128, 9, True, [333, 1], [9, 5], 9),
    ("bf16", 8, 1, 128, 1, False, [1000, 999, 31], None, 1),
    ("bf16", 3, 1, 32, 33, False, [64, 0], None, 20),
    ("bf16", 4, 2, 64, 130, False, [90, 0, 33], [130, 65, 64], 130),
    ("bf16", 4, 2, 128, 70, False, [15, 64], None, 3),
    ("fp32", 4, 4, 32, 5, False, [33, 0], None, 0),
    ("fp32", 4, 2, 64, 13, True, [100, 31], [13, 2], 13),
    ("fp32", 2, 1, 128, 1, False, [300, 0, 32], None, 1),
    ("fp32", 2, 2, 64, 90, False, [20, 0], [90, 33], 5),
]


@pytest.mark.parametrize("dtype,heads,kv_heads,size,tokens,is_tree,lens,counts,counted", SHAPES)
def test_attention(dtype, heads, kv_heads, size, tokens, is_tree, lens, counts, counted):
    rng = np.random.default_rng(tokens * 7 + size)
    rows = len(lens)
    both = Both(dtype, rows=rows, heads=heads, kv_heads=kv_heads, size=size, capacity=max(lens) + 13, max_tokens=tokens)
    both.fill(rng, lens, spread=0.7)
    qkv = values(rng, (rows, tokens, heads + 2 * kv_heads, size), both.dtype, spread=0.7)
    q, k, v = qkv.split([heads, kv_heads, kv_heads], dim=2)
    parent = tree(rng, tokens) if is_tree else None
    both.attend(lens, q, k, v, parent=parent, counts=counts, counted=counted)
    both.attend(lens, q.contiguous(), None, None, counts=counts, counted=counted, scale=0.3)     # the cache alone: rows of length 0 see nothing


def test_attention_of_a_later_layer_with_a_mask_and_blocks_of_different_size():
    rng = np.random.default_rng(5)
    both = Both("bf16", layers=3, rows=2, heads=4, kv_heads=2, size=64, capacity=140, max_tokens=8)
    for gain in (1e-3, 1.0, 40.0):
        k, v = (values(rng, (3, 2, 40, 2, 64), both.dtype, 0.3) * gain for _ in range(2))
        start = [0 if gain < 1 else 40 if gain == 1 else 80] * 2
        both.append(start, k, v)
    q, k, v = (values(rng, (2, 8, h, 64), both.dtype, 0.3) * 0.2 for h in (4, 2, 2))
    parent = tree(rng, 8)
    mask = qc.ancestors(parent, 8).astype(np.uint8)
    both.attend([120, 77], q, k, v, parent=parent, tree_mask=mask, counted=2, layer=2)
    both.attend([120, 77], q, k, v, parent=parent, tree_mask=mask, counted=8, layer=1)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_what_is_masked_may_be_anything(dtype):
    rng = np.random.default_rng(6)
    both = Both(dtype, rows=2, heads=4, kv_heads=2, size=64, capacity=96, max_tokens=6)
    both.fill(rng, [45, 32], spread=0.5)
    bad = torch.full((1, 2, 30, 2, 64), math.nan, dtype=both.dtype, device="cuda")
    both.gpu.vvs_qcache_append(ints([45, 32]), bad, bad)          # behind the lengths that follow
    q, k, v = (values(rng, (2, 6, h, 64), both.dtype, 0.5) for h in (4, 2, 2))
    parent = np.asarray([0, 0, 1, 2, 2], dtype=np.int32)           # 0 - (1 - 3), (2 - (4, 5))
    for t, what in ((1, math.nan), (3, math.inf)):
        k[:, t], v[:, t] = what, what
    v[:, 3, :, ::2] = -math.inf
    # a row's unused tokens
    k[1, 5], v[1, 5], q[1, 5] = math.nan, math.inf, math.nan
    out = both.attend([45, 32], q, k, v, parent=parent, counts=[6, 5])
    got = np64(out)
    assert np.isfinite(got[:, [0, 2, 4]]).all() and np.isnan(got[:, 1]).all()


def test_visible_values_that_are_not_finite_show():
    rng = np.random.default_rng(7)
    both = Both("bf16", rows=1, heads=1, kv_heads=1, size=64, capacity=64, max_tokens=4)
    both.fill(rng, [10], spread=0.2)
    q, k, v = (values(rng, (1, 4, 1, 64), both.dtype, 0.2) for _ in range(3))
    v[0, 1, 0, 3], v[0, 1, 0, 4], v[0, 2, 0, 3] = math.inf, math.nan, -math.inf
    out = np64(both.attend([10], q, k, v))
    assert out[0, 1, 0, 3] == math.inf and np.isnan(out[0, 2, 0, 3]) and np.isnan(out[0, 1, 0, 4]) and np.isfinite(out[0, 1, 0, 5:]).all()


def test_scores_far_apart_and_equal():
    """One key far above all others, far below, and all the same: running maximum, its rescaling, sums."""
    both = Both("bf16", rows=3, heads=1, kv_heads=1, size=32, capacity=320, max_tokens=2)
    k = torch.zeros((1, 3, 300, 1, 32), dtype=both.dtype, device="cuda")
    v = torch.arange(300, device="cuda").view(1, 1, 300, 1, 1).expand(1, 3, 300, 1, 32).to(both.dtype)
    k[0, 0, 250, 0, 0], k[0, 1, :, 0, 0] = 400.0, -400.0
    k[0, 1, 3, 0, 0] = 0.0
    both.append([0, 0, 0], k, v)
    q = torch.zeros((3, 2, 1, 32), dtype=both.dtype, device="cuda")
    q[..., 0] = 50.0
    both.attend([300, 300, 300], q, None, None, counted=2)


def test_lengths_and_counts_outside_their_range_are_taken_as_the_nearest_inside():
    rng = np.random.default_rng(8)
    both = Both("bf16", rows=3, capacity=70, max_tokens=5)
    both.fill(rng, [70, 70, 70], spread=0.5)
    q, k, v = (values(rng, (3, 5, h, 64), both.dtype, 0.5) for h in (4, 2, 2))
    both.attend([500, -3, 2 ** 31 - 1], q, k, v, counts=[9, -1, 5], counted=5)


def test_the_same_call_gives_the_same_bits_on_another_stream_too():
    rng = np.random.default_rng(9)
    both = Both("bf16", rows=2, heads=8, kv_heads=2, size=128, capacity=4000, max_tokens=3)
    k, v = (values(rng, (1, 2, 4000, 2, 128), both.dtype, 0.5) for _ in range(2))
    both.gpu.vvs_qcache_append(ints([0, 0]), k, v)
    q, k, v = (values(rng, (2, 3, h, 128), both.dtype, 0.5) for h in (8, 2, 2))
    length, got = ints([4000, 3333]), []
    side = torch.cuda.Stream()
    for i in range(6):
        out, mass = torch.empty_like(q), torch.zeros((2, 2, 4000), device="cuda")
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side) if i % 2 else torch.cuda.stream(torch.cuda.current_stream()):
            both.gpu.vvs_qcache_attention(length, q, k, v, out, n_counted=3, mass=mass)
        torch.cuda.synchronize()
        got.append((out, mass))
    for out, mass in got[1:]:
        assert torch.equal(out, got[0][0]) and torch.equal(mass, got[0][1])


def test_offsets_beyond_32_bits():
    """A cache of 5 GiB: the last rows and slots hold what was appended there, and attention sees it."""
    rows, kv_heads, size, capacity = 40, 16, 128, 32768
    both = Both("bf16", rows=1, heads=16, kv_heads=16, size=size, capacity=64, max_tokens=1)
    gpu = vb.QCache(1, rows, 16, kv_heads, size, capacity, 1, vb.VVS_BF16)
    assert gpu.cache_bytes > 5 << 30
    rng = np.random.default_rng(10)
    k, v = (values(rng, (1, 1, 40, kv_heads, size), torch.bfloat16, 0.5) for _ in range(2))
    both.append([0], k, v)
    many = [x.expand(1, rows, 40, kv_heads, size).contiguous() for x in (k, v)]
    start = capacity - 64
    gpu.vvs_qcache_append(ints([start] * rows), *many)
    got = [torch.empty_like(x) for x in many]
    gpu.vvs_qcache_read(ints([capacity] * rows), *got, first=ints([start] * rows))
    ref = [torch.empty((1, 1, 40, kv_heads, size), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    both.gpu.vvs_qcache_read(ints([40]), *ref)
    for x, y in zip(got, ref):
        assert torch.equal(x, y.expand_as(x))
    # all other slots are zeros: scores 0, values 0, so that the weights of 32736 equal keys shrink the output of 40
    q = values(rng, (1, 1, 16, size), torch.bfloat16, 0.5)
    out, lse = torch.empty((rows, 1, 16, size), dtype=torch.bfloat16, device="cuda"), torch.empty((rows, 1, 16), device="cuda")
    gpu.vvs_qcache_attention(ints([start + 40] * rows), q.expand(rows, 1, 16, size).contiguous(), None, None, out, lse=lse)
    y, z, _, _, top_s, top_v = both.ref.attend(0, 0, 40, np64(q[0]), None, None, None, size ** -0.5, 0)
    whole = np.logaddexp(z, math.log(start))
    near(np64(lse), np.broadcast_to(whole, (rows, 1, 16)), 2 * size * 2.0 ** -24 * top_s + 2.0 ** -20 * (1 + np.abs(whole)))
    want = y * np.exp(z - whole)[..., None]
    near(np64(out), np.broadcast_to(want, out.shape), (2 * size * 2.0 ** -24 * top_s + 2.0 ** -16) * top_v * np.exp(z - whole)[..., None] + 2.0 ** -8 * np.abs(want))


# ------------------------------------------------------------------------------------------------ eviction
@pytest.mark.parametrize("dtype,size", [("bf16", 64), ("fp32", 32), ("bf16", 128)])
@pytest.mark.parametrize("keep,recent,in_place,with_pos", [(32, 0, False, True), (64, 17, True, True), (128, 128, False, False), (96, 5, True, False)])
def test_eviction(dtype, size, keep, recent, in_place, with_pos):
    rng = np.random.default_rng(keep + recent + size)
    lens, capacity, layers = [200, 97, keep, 3, 129, 0], 211, 2
    both = Both(dtype, layers=layers, rows=6, heads=2, kv_heads=2, size=size, capacity=capacity)
    # blocks of different size, so that moved elements are rounded again
    for start in (0, 64, 128):
        k, v = (values(rng, (layers, 6, 72, 2, size), both.dtype) * 2.0 ** float(rng.integers(-6, 7)) for _ in range(2))
        both.append([start] * 6, k, v)
    dims = (layers, 6, 2, capacity)
    mass = rng.random(dims).astype(np.float32) ** 8
    mass[rng.random(dims) < 0.2] = 0.0                             # equal weights: the lower slot stays
    mass[0, 0, 0, 150:155] = [np.nan, -0.0, np.inf, -1.0, 0.0]
    pos = np.broadcast_to(rng.permutation(capacity), dims).astype(np.int32) - 50 if with_pos else np.broadcast_to(np.arange(capacity), dims).astype(np.int32)
    m, p = torch.from_numpy(mass).cuda(), torch.from_numpy(np.ascontiguousarray(pos)).cuda()
    m_out, p_out = (m, p) if in_place else (torch.full_like(m, 5.0), torch.full_like(p, 5))
    both.gpu.vvs_qcache_evict(ints(lens), keep, recent, m, m_out, p if with_pos else None, p_out if with_pos else None, n_layers=layers)
    for l in range(layers):
        for r, n in enumerate(lens):
            want_m, want_p = both.ref.evict(l, r, n, keep, recent, mass[l, r], pos[l, r])
            np.testing.assert_array_equal(m_out[l, r].cpu().numpy(), want_m)
            if with_pos:
                np.testing.assert_array_equal(p_out[l, r].cpu().numpy(), want_p)
    both.check_held([min(n, keep) for n in lens], n_layers=layers)


def test_eviction_of_a_long_row_and_of_one_layer():
    rng = np.random.default_rng(11)
    both = Both("bf16", layers=2, rows=1, heads=1, kv_heads=1, size=32, capacity=5000)
    k, v = (values(rng, (2, 1, 5000, 1, 32), both.dtype) for _ in range(2))
    both.append([0], k, v)
    mass = np.exp(rng.standard_normal((1, 1, 1, 5000)) * 3).astype(np.float32)
    pos = rng.permutation(5000).astype(np.int32).reshape(1, 1, 1, 5000)
    m, p = torch.from_numpy(mass).cuda(), torch.from_numpy(pos).cuda()
    both.gpu.vvs_qcache_evict(ints([4999]), 1216, 100, m, m, p, p, layer=1)
    want_m, want_p = both.ref.evict(1, 0, 4999, 1216, 100, mass[0, 0], pos[0, 0])
    np.testing.assert_array_equal(m[0, 0].cpu().numpy(), want_m)
    np.testing.assert_array_equal(p[0, 0].cpu().numpy(), want_p)
    both.check_held([1216], layer=1)
    both.check_held([5000], layer=0)
