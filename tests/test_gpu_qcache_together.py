"""The 8-bit cache's operators as a decoding loop uses them, captured and replayed, and the forms of attention that small sizes do not reach: many queries, rows in splits, blocks of very
different size, values that are not finite among many queries.  Tolerances: test_gpu_qcache.py."""
import math

import numpy as np
import pytest
import torch

import qcache_common as qc
from paper_2511_13587_amd import binding as vb
from test_gpu_qcache import Both, ints, near, np64, tree, values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,heads,kv_heads,size", [("bf16", 4, 4, 64), ("bf16", 8, 2, 128), ("fp32", 4, 2, 32)])
def test_a_decoding_loop(dtype, heads, kv_heads, size):
    """Rotation, attention over cache and tree with counted weights, the accepted path appended to both layers, an eviction now and then."""
    rng = np.random.default_rng(size + heads)
    rows, layers, nodes, capacity, keep = 3, 2, 9, 160, 64
    both = Both(dtype, layers=layers, rows=rows, heads=heads, kv_heads=kv_heads, size=size, capacity=capacity, max_tokens=nodes)
    rope = vb.Rope(size, [size // 4, size // 8, size // 8], 10000.0, both.code)
    lens = [40, 33, 64]
    both.fill(rng, lens, n_layers=layers, spread=0.5)
    mass = torch.zeros((layers, rows, kv_heads, capacity), device="cuda")
    pos = torch.arange(capacity, dtype=torch.int32, device="cuda").expand(layers, rows, kv_heads, capacity).contiguous()
    emitted = list(lens)
    for step in range(7):
        parent = tree(rng, nodes)
        depth = [0]
        for p in parent:
            depth.append(depth[p] + 1)
        paths = [[0] for _ in range(rows)]
        for path in paths:
            while len(path) < 6 and (parent == path[-1]).any() and rng.random() < 0.7:
                path.append(int(np.flatnonzero(parent == path[-1])[0]) + 1)
        counts = [len(p) for p in paths]
        staged = torch.zeros((2, layers, rows, nodes, kv_heads, size), dtype=both.dtype, device="cuda")
        at = torch.tensor([[[(emitted[r] + d) // 64, (emitted[r] + d) // 8 % 8, (emitted[r] + d) % 8] for d in depth] for r in range(rows)], dtype=torch.int32, device="cuda")
        for layer in range(layers):
            qkv = values(rng, (rows, nodes, heads + 2 * kv_heads, size), both.dtype, 0.5)
            q, k, v = qkv.split([heads, kv_heads, kv_heads], dim=2)
            rope.vvs_rope_apply(at, q, k, q, k)                                   # in place, inside the projection's output
            staged[0, layer], staged[1, layer] = k, v
            out, lse, block = torch.zeros((rows, nodes, heads, size), dtype=both.dtype, device="cuda"), torch.zeros((rows, nodes, heads), device="cuda"), torch.zeros((rows, kv_heads, nodes), device="cuda")
            before = np64(mass[layer])
            both.gpu.vvs_qcache_attention(ints(lens), q, k, v, out, parent=parent, lse=lse, n_counted=1, mass=mass[layer], block_mass=block, layer=layer)
            for r in range(rows):
                y, z, m, b, top_s, top_v = both.ref.attend(layer, r, lens[r], np64(q[r]), np64(k[r]), np64(v[r]), qc.ancestors(parent, nodes), size ** -0.5, 1)
                weight = 2 * size * 2.0 ** -24 * top_s + 2.0 ** -20
                near(np64(out[r]), y, weight * top_v + (2.0 ** -17 * top_v + 2.0 ** -8 * np.abs(y) if both.dtype == torch.bfloat16 else 2.0 ** -23 * np.abs(y)))
                near(np64(mass[layer, r])[:, :lens[r]], before[r][:, :lens[r]] + m, weight * m + 2.0 ** -22 * (1 + before[r][:, :lens[r]] + m))
                near(np64(block[r]), b, weight * b + 2.0 ** -22)
        select = [p + [0] * (6 - len(p)) for p in paths]
        both.append(lens, staged[0], staged[1], counts=counts, select=select)
        for layer in range(layers):
            for r in range(rows):
                pos[layer, r, :, lens[r]:lens[r] + counts[r]] = torch.arange(emitted[r], emitted[r] + counts[r], device="cuda", dtype=torch.int32)
        lens, emitted = [a + b for a, b in zip(lens, counts)], [a + b for a, b in zip(emitted, counts)]
        both.check_held(lens, n_layers=layers)
        if step % 3 == 2:
            was_m, was_p = mass.cpu().numpy(), pos.cpu().numpy()
            both.gpu.vvs_qcache_evict(ints(lens), keep, 8, mass, mass, pos, pos, n_layers=layers)
            for layer in range(layers):
                for r in range(rows):
                    want_m, want_p = both.ref.evict(layer, r, lens[r], keep, 8, was_m[layer, r], was_p[layer, r])
                    np.testing.assert_array_equal(mass[layer, r].cpu().numpy(), want_m)
                    np.testing.assert_array_equal(pos[layer, r].cpu().numpy(), want_p)
            lens = [min(n, keep) for n in lens]
            both.check_held(lens, n_layers=layers)


def test_a_captured_step_replays_as_it_runs():
    """Rotation, attention, append, eviction and the lengths' advance in one graph, and a second graph over the same cache: every replay, with eager work between, against the eager run."""
    rng = np.random.default_rng(3)
    rows, heads, kv_heads, size, capacity, tokens = 2, 8, 2, 128, 1600, 5

    class State:
        def __init__(self):
            g = np.random.default_rng(4)
            self.cache = vb.QCache(1, rows, heads, kv_heads, size, capacity, tokens, vb.VVS_BF16)
            k, v = (values(g, (1, rows, 1200, kv_heads, size), torch.bfloat16, 0.5) for _ in range(2))
            self.cache.vvs_qcache_append(ints([0, 0]), k, v)
            self.len = ints([1200, 900])
            self.mass = torch.zeros((1, rows, kv_heads, capacity), device="cuda")
            self.pos = torch.arange(capacity, dtype=torch.int32, device="cuda").expand(1, rows, kv_heads, capacity).contiguous()
            self.out = torch.zeros((rows, tokens, heads, size), dtype=torch.bfloat16, device="cuda")

        def step(self):
            q, k, v = inputs.split([heads, kv_heads, kv_heads], dim=2)
            q_turned, k_turned = torch.empty((rows, tokens, heads, size), dtype=torch.bfloat16, device="cuda"), torch.empty((rows, tokens, kv_heads, size), dtype=torch.bfloat16, device="cuda")
            rope.vvs_rope_apply(where, q, k, q_turned, k_turned)
            self.cache.vvs_qcache_attention(self.len, q_turned, k_turned, v, self.out, parent=parent, n_counted=tokens, mass=self.mass[0])
            self.cache.vvs_qcache_append(self.len, k_turned[None], v[None])
            self.len += tokens

        def shorten(self):
            self.cache.vvs_qcache_evict(self.len, 1024, 64, self.mass, self.mass, self.pos, self.pos)
            self.len.clamp_(max=1024)

        def snapshot(self):
            return [x.clone() for x in (self.cache.cache, self.len, self.mass, self.pos, self.out)]

    rope = vb.Rope(size, [24, 20, 20], 10000.0, vb.VVS_BF16)
    inputs = values(rng, (rows, tokens, heads + 2 * kv_heads, size), torch.bfloat16, 0.5)
    where = torch.zeros((rows, tokens, 3), dtype=torch.int32, device="cuda")
    parent = np.asarray([0, 0, 1, 2], dtype=np.int32)
    eager, taped = State(), State()
    warm = State()                                                    # (a stream's first use and lazy loading stay out of the capture)
    warm.step(), warm.shorten()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    step, shorten = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(step, stream=side):
        taped.step()
    with torch.cuda.graph(shorten, stream=side):
        taped.shorten()
    for i in range(6):
        new = values(np.random.default_rng(20 + i), inputs.shape, torch.bfloat16, 0.5)
        inputs.copy_(new)
        where.copy_(torch.randint(0, 5000, where.shape, device="cuda", dtype=torch.int32))
        eager.step()
        step.replay()
        if i in (2, 4):
            eager.shorten()
            shorten.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager.snapshot(), taped.snapshot()):
            assert torch.equal(a, b), f"replay {i}"


FORMS = [
    # dtype, heads, kv heads, size, tokens, tree, lengths, counts, counted
    ("bf16", 8, 2, 128, 40, True, [100, 31, 0], [40, 17, 40], 1),         # many queries, tree
    ("bf16", 8, 2, 128, 40, True, [100, 31, 0], None, 40),
    ("bf16", 2, 1, 64, 90, False, [1500, 1111], None, 2),                 # many queries, splits, kept scores
    ("bf16", 2, 1, 64, 90, False, [1500, 0], [90, 33], 90),               # ... and counted again
    ("bf16", 4, 1, 32, 64, True, [1100, 640], None, 2),
    ("bf16", 4, 1, 32, 100, False, [1100, 33], None, 0),
    ("bf16", 1, 1, 128, 1, False, [2000, 513], None, 1),                  # splits of a single query
    ("bf16", 4, 2, 64, 20, True, [1536, 1], [20, 20], 1),                 # splits of two query blocks
    ("fp32", 2, 1, 64, 30, True, [1030, 5], None, 2),
    ("fp32", 2, 1, 32, 7, False, [1030, 700], None, 7),
    ("fp32", 2, 1, 128, 20, True, [70, 0], None, 20),                     # fp32, many counted
    ("fp32", 4, 1, 64, 70, False, [40, 33], [70, 5], 60),
    ("bf16", 2, 2, 64, 5, False, [40, 33], None, 0),
]


@pytest.mark.parametrize("dtype,heads,kv_heads,size,tokens,is_tree,lens,counts,counted", FORMS)
def test_forms_of_attention(dtype, heads, kv_heads, size, tokens, is_tree, lens, counts, counted):
    rng = np.random.default_rng(tokens + size + counted)
    rows = len(lens)
    both = Both(dtype, rows=rows, heads=heads, kv_heads=kv_heads, size=size, capacity=max(lens) + 1, max_tokens=tokens)
    both.fill(rng, lens, spread=0.5)
    q, k, v = (values(rng, (rows, tokens, h, size), both.dtype, 0.5) for h in (heads, kv_heads, kv_heads))
    both.attend(lens, q, k, v, parent=tree(rng, tokens) if is_tree else None, counts=counts, counted=counted)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("tokens,length", [(3, 192), (150, 192), (2, 1200)])
def test_blocks_of_very_different_size(dtype, tokens, length):
    """Values of 2^-90, 1 and 2^60 and blocks of zeros in one row; keys likewise, with queries that make all of them count."""
    rng = np.random.default_rng(tokens)
    both = Both(dtype, rows=4, heads=2, kv_heads=1, size=64, capacity=length, max_tokens=tokens)
    v = values(rng, (1, 4, length, 1, 64), both.dtype, 0.5)
    k = values(rng, (1, 4, length, 1, 64), both.dtype, 0.5)
    block = torch.arange(length, device="cuda").view(1, 1, -1, 1, 1) // 32
    gain = torch.tensor([[0, 0, 0], [-90, 0, 60], [-90, -90, -90], [60, 0, -200]], device="cuda", dtype=torch.float64)[:, :, None]      # -200: zeros
    for r in range(4):
        for b in range(3):
            v[:, r] = torch.where(block[0] % 3 == b, (v[:, r].double() * 2.0 ** gain[r, b, 0]).to(both.dtype), v[:, r])
    k[:, 3] = torch.where(block[0] % 3 == 1, torch.zeros_like(k[:, 3]), k[:, 3])
    both.append([0] * 4, k, v)
    q, kk, vv = (values(rng, (4, tokens, h, 64), both.dtype, 0.5) for h in (2, 1, 1))
    both.attend([length, length - 7, length - 32, length], q, kk, vv, counted=2)
    # a row whose values are all tiny keeps them
    out = torch.zeros((4, tokens, 2, 64), dtype=both.dtype, device="cuda")
    both.gpu.vvs_qcache_attention(ints([length] * 4), q, None, None, out)
    y = both.ref.attend(0, 2, length, np64(q[2]), None, None, None, 64 ** -0.5, 0)
    near(np64(out[2]), y[0], (2 * 64 * 2.0 ** -24 * y[4] + 2.0 ** -16) * y[5] + 2.0 ** -8 * np.abs(y[0]))


def test_what_is_masked_may_be_anything_among_many_queries():
    rng = np.random.default_rng(8)
    both = Both("bf16", rows=2, heads=4, kv_heads=1, size=64, capacity=96, max_tokens=100)
    both.fill(rng, [45, 32], spread=0.3)
    q, k, v = (values(rng, (2, 100, h, 64), both.dtype, 0.3) for h in (4, 1, 1))
    v[0, 70, 0, 5], v[0, 75, 0, 6], v[0, 40, 0, 9] = math.inf, math.nan, -math.inf
    k[1, 60:], v[1, 60:], q[1, 60:] = math.nan, math.nan, math.nan               # behind the row's number
    out = np64(both.attend([45, 32], q, k, v, counts=[100, 60], counted=3))
    assert np.isfinite(out[0, :40]).all() and (out[0, 40:, :, 9] == -math.inf).all() and np.isfinite(out[0, 40:70, :, :9]).all()
    assert (out[0, 70:, :, 5] == math.inf).all() and np.isnan(out[0, 75:, :, 6]).all() and np.isfinite(out[1, :60]).all()
    both.gpu.vvs_qcache_append(ints([45, 32]), torch.full((1, 2, 40, 1, 64), math.nan, dtype=both.dtype, device="cuda"), torch.full((1, 2, 40, 1, 64), math.nan, dtype=both.dtype, device="cuda"))
    ok = values(rng, (2, 100, 1, 64), both.dtype, 0.3)
    assert np.isfinite(np64(both.attend([45, 32], values(rng, (2, 100, 4, 64), both.dtype, 0.3), ok, ok, counted=100))).all()


def test_eviction_of_rows_longer_than_registers_hold():
    rng = np.random.default_rng(12)
    n = 40000
    both = Both("bf16", rows=1, heads=1, kv_heads=1, size=32, capacity=n)
    k, v = (values(rng, (1, 1, n, 1, 32), both.dtype) for _ in range(2))
    both.append([0], k, v)
    mass = np.exp(rng.standard_normal((1, 1, 1, n)) * 3).astype(np.float32)
    mass[rng.random(mass.shape) < 0.4] = 0.0
    pos = rng.permutation(n).astype(np.int32).reshape(1, 1, 1, n)
    for keep, recent, length, in_place in ((25600, 1000, n, False), (9600, 0, 25600, True)):
        m, p = torch.from_numpy(mass).cuda(), torch.from_numpy(pos).cuda()
        m_out, p_out = (m, p) if in_place else (torch.full_like(m, 5.0), torch.full_like(p, 5))
        both.gpu.vvs_qcache_evict(ints([length]), keep, recent, m, m_out, p, p_out)
        want_m, want_p = both.ref.evict(0, 0, length, keep, recent, mass[0, 0], pos[0, 0])
        np.testing.assert_array_equal(m_out[0, 0].cpu().numpy(), want_m)
        np.testing.assert_array_equal(p_out[0, 0].cpu().numpy(), want_p)
        both.check_held([keep], first=[keep - 64], n=64)
        mass[0, 0], pos[0, 0] = want_m, want_p


def test_refusals_of_the_binding():
    cache = vb.QCache(1, 2, 4, 2, 64, 64, 8, vb.VVS_BF16)
    x = torch.zeros((2, 8, 4, 64), dtype=torch.bfloat16, device="cuda")
    k = torch.zeros((2, 8, 2, 64), dtype=torch.bfloat16, device="cuda")
    n = ints([0, 0])
    good = dict(length=n, q=x, k=k, v=k, out=torch.zeros_like(x))
    cache.vvs_qcache_attention(**good)
    for bad in (dict(q=x.float()), dict(q=x.cpu()), dict(out=x.transpose(1, 2)), dict(v=k[:, :, :1]), dict(length=n.long()), dict(length=ints([0])), dict(q=x[:, :, ::2]),
                dict(parent=[0, 0]), dict(lse=torch.zeros((2, 8, 4), dtype=torch.bfloat16, device="cuda")), dict(n_counted=1, mass=torch.zeros((2, 2, 63), device="cuda"))):
        with pytest.raises(ValueError):
            cache.vvs_qcache_attention(**{**good, **bad})
    for bad in (dict(parent=[0, 2, 1, 0, 0, 0, 0]), dict(scale=0.0), dict(n_counted=9), dict(n_counted=1), dict(layer=1), dict(k=None, v=None, parent=list(range(7)))):
        with pytest.raises(vb.VvsError):
            cache.vvs_qcache_attention(**{**good, **bad})
    with pytest.raises(vb.VvsError):
        cache.vvs_qcache_attention(**{**good, "k": None})
    rope = vb.Rope(64, [16, 16], 10000.0, vb.VVS_BF16)
    pos = torch.zeros((2, 8, 2), dtype=torch.int32, device="cuda")
    rope.vvs_rope_apply(pos, x, k, x, k)
    for args in ((pos[:, :, :1], x, k, x, k), (pos, x.float(), k, x, k), (pos, x.cpu(), k, x, k), (pos, x, k, x, None), (pos.long(), x, k, x, k), (pos, x[0], k, x, k)):
        with pytest.raises((ValueError, vb.VvsError)):
            rope.vvs_rope_apply(*args)
    torch.cuda.synchronize()
    cache.close()
    cache.close()
