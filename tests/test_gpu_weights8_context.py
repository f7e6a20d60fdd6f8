"""Contexts that hold their layers' weights in 8 bits (VVS_WEIGHTS_E4M3) in lockstep with the oracle, whose layer here has their rounding points: weights held in e4m3 blocks, the norms' outputs, the attention's
(rounded to the dtype first) and the activations as well.  After every call that caches tokens the oracle takes over the context's cache, so that the next forward is compared on the same one.  A value
that fp32 and 64 bits put on two sides of a border of e4m3 moves by a step, 2^-3 of itself, and is amplified by what follows: the bound is that of the bf16 contexts - 3e-2, or three times what the oracle
itself moves by under a perturbation of fp32's size (1e-6 in front of the 8-bit roundings, 1e-7 in front of the bf16 ones)."""
import dataclasses

import numpy as np
import pytest
import torch

import gpu_common as gc
import qlinear_common as ql
from oracle import vvs_oracle as vo
from paper_2511_13587_amd import binding as vb
from paper_2511_13587_amd import synth

pytestmark = pytest.mark.gpu

FP32 = synth.TINY.replace(n_prompts=2, n_nodes=9)
BF16 = synth.XL_TREE.replace(n_layers=2, n_prompts=2, prefix_len=8)
MANY = synth.B_SHAPE.replace(n_layers=2, n_prompts=4, n_nodes=20)              # 168 rows
WIDE = synth.SEVEN_B.replace(n_layers=1, d_model=1024, n_heads=8, d_ff=2816, n_prompts=2, prefix_len=8, vocab=2048, logit_lo=512, logit_hi=1536)


def held(x):
    return ql.held(torch.from_numpy(np.ascontiguousarray(x)))[0].numpy()


class Held8(vo.Oracle):
    """The oracle's layer with weights and their operands in 8 bits; eps: perturbation in front of the rounding to 8 bits."""

    def __init__(self, cfg, weights, eps=0.0):
        super().__init__(cfg, {k: held(v.T).T.astype(np.float32) if k.split(".")[-1] in ("wq", "wk", "wv", "wo", "wg", "wu", "wd") else v for k, v in weights.items()})
        rng = np.random.default_rng(3)
        self.r8 = lambda x: held(x * (1 + eps * rng.standard_normal(x.shape)) if eps else x)

    def forward_block(self, row, x_in, img_index, mask, logits_for=None):
        rb, r8, w = self.rb, self.r8, self.w
        x = np.asarray(x_in, dtype=np.float64).copy()
        T = x.shape[0]
        pos = [self._grid_pos(int(i)) for i in img_index]
        gr, gcol = (np.array([p[i] for p in pos], dtype=np.float64)[:, None, None] for i in (0, 1))
        new_kv = []
        for l in range(self.L):
            q, k, v = self._qkv(l, r8(vo.rmsnorm(x, w[f"l{l}.g1"], self.eps)))
            q, k = (rb(self._rope_block(y.reshape(T, self.H, self.dh), gr, gcol)) for y in (q, k))
            v = rb(v.reshape(T, self.H, self.dh))
            new_kv.append((k, v))
            keys, vals = np.concatenate([self.kc[row][l], k]), np.concatenate([self.vc[row][l], v])
            seen = np.concatenate([np.ones((T, len(keys) - T), dtype=bool), np.asarray(mask).astype(bool)], axis=1)
            o = np.stack([vo.softmax(np.where(seen, q[:, h] @ keys[:, h].T / np.sqrt(self.dh), -np.inf)) @ vals[:, h] for h in range(self.H)], axis=1)
            x = x + r8(rb(o.reshape(T, self.d))) @ w[f"l{l}.wo"]
            h = r8(vo.rmsnorm(x, w[f"l{l}.g2"], self.eps))
            x = x + r8(vo.silu(h @ w[f"l{l}.wg"]) * (h @ w[f"l{l}.wu"])) @ w[f"l{l}.wd"]
        self.block_features = self._feature(x)
        sel = np.arange(T) if logits_for is None else np.asarray(logits_for)
        logits = np.full((T, self.hi - self.lo), np.nan)
        logits[sel] = rb(vo.rmsnorm(x[sel], w["gf"], self.eps)) @ w["wout"][:, self.lo:self.hi]
        return logits, new_kv


class Run:
    def __init__(self, shape, cache_kind=0):
        self.shape = shape
        w = synth.make_weights(shape)
        self.ctx = vb.Context(vb.make_config(shape, weight_kind=vb.VVS_WEIGHTS_E4M3, cache_kind=cache_kind))
        self.ctx.load_weights_from_host(w, synth.weight_names(shape))
        cfg = dict(dataclasses.asdict(shape), feature_slots=5, feature_pre_norm=0)
        self.ora, self.shadow = Held8(cfg, w), Held8(cfg, w, 1e-6)
        if shape.dtype == synth.DTYPE_BF16:
            self.shadow = gc.perturbed_rounding(self.shadow)
        self.out = [torch.zeros(n, dtype=torch.int32, device="cuda") for n in (shape.n_prompts, (shape.n_prompts, vb.VVS_MAX_T), shape.n_prompts)]

    def take_cache(self):
        o = self.ora
        for row in range(o.R):
            n = o.kv_len(row // 2)
            for l in range(o.L):
                k, v = (x.double().cpu().numpy().reshape(n, o.H, o.dh) for x in self.ctx.vvs_debug_kv(l, row, n))
                for x in (o, self.shadow):
                    x.kc[row][l], x.vc[row][l] = k.copy(), v.copy()

    def close_to(self, raw, key):
        want, off = getattr(self.ora, key), getattr(self.shadow, key) - getattr(self.ora, key)
        err = raw.cpu().numpy().reshape(want.shape) - want
        assert np.abs(err).max() <= max(3e-2, 3 * np.abs(off).max())
        assert gc.rms(err) <= max(1e-2, 3 * gc.rms(off))

    def prefill(self, n_forced):
        s = self.shape
        pc, pu = synth.make_prefix(s)
        forced = synth.make_forced_tokens(s, n_forced) if n_forced else None
        self.ora.prefill(pc, pu, forced, np.full(s.n_prompts, 0.5))
        u = np.array([p[:int(np.argmax(p))].sum() + 0.5 * p.max() for p in self.ora.prefill_probs], dtype=np.float32)
        for x in (self.ora, self.shadow):
            x.prefill(pc, pu, forced, u)
        dpc, dpu = (torch.from_numpy(pc).cuda(), None) if s.prefix_kind == synth.PREFIX_CLASS else (vb.to_device(pc, s.dtype), vb.to_device(pu, s.dtype))
        self.ctx.vvs_prefill(dpc, dpu, None if forced is None else torch.from_numpy(forced).cuda(), torch.from_numpy(u).cuda(), self.out[2])
        raw, _, _ = self.ctx.vvs_debug_logits()
        self.close_to(raw[:, 0], "prefill_logits")
        for x in (self.ora, self.shadow):
            x.pending[:] = self.out[2].cpu().numpy()
        self.take_cache()

    def step(self, seed):
        s, n = self.shape, self.shape.n_nodes
        parent = np.asarray([max(0, j - 2) for j in range(n)], dtype=np.int32)
        q, toks = synth.make_draft(s, parent, seed)
        u = synth.make_uniforms(s, n, seed)
        u[:, 1 + seed % 3, 0] = 0.0
        self.ctx.vvs_verify(n, parent, None, torch.from_numpy(toks).cuda(), torch.from_numpy(q).cuda(), torch.from_numpy(u).cuda(), vb.VVS_STRICT, *self.out)
        for x in (self.ora, self.shadow):
            x.verify(parent, toks, q, u, 0, 0)
        raw, _, _ = self.ctx.vvs_debug_logits()
        self.close_to(raw, "raw_logits")
        a, p, t = (x.cpu().numpy() for x in self.out)
        for x in (self.ora, self.shadow):                      # a draw within the noise may fall either way
            x.last["paths"] = [[int(v) for v in p[b, :a[b] + 1]] for b in range(s.n_prompts)]
            x.last["accept_len"], x.last["next_token"] = a.copy(), t.copy()
        self.ctx.vvs_kv_commit()
        for x in (self.ora, self.shadow):
            x.kv_commit()
        state = self.ctx.vvs_read_state()
        assert (state[0] == [self.ora.kv_len(b) for b in range(s.n_prompts)]).all() and (state[1] == self.ora.n_emitted).all()
        self.take_cache()


@pytest.mark.parametrize("shape,forced,cache_kind", [(FP32, 5, 0), (BF16, 9, 0), (MANY, 3, 0), (WIDE, 0, 0), (FP32, 5, 1), (BF16, 9, 1), (WIDE, 0, 1)],
                         ids=["fp32", "bf16", "many", "wide", "fp32-cache8", "bf16-cache8", "wide-cache8"])
def test_context_in_lockstep(shape, forced, cache_kind):
    run = Run(shape, cache_kind)
    assert not run.ctx.vvs_plan_is_fused(shape.n_nodes + 1)
    run.prefill(forced)
    for i in range(2):
        run.step(i)
    run.ctx.close()


def test_a_prefill_of_more_rows_than_a_tile():
    """Chunks of many rows: 2 prompts x 2 rows x 128 prefix tokens and some."""
    run = Run(BF16.replace(prefix_len=130, n_layers=1))
    run.prefill(37)
    run.step(1)
    run.ctx.close()


def test_replayed_calls_have_the_same_bits_and_a_graph_theirs():
    """A verify call and its commit, again and again from the same state, eagerly and from a captured graph."""
    shape = BF16
    run = Run(shape)
    run.prefill(9)
    state = torch.from_numpy(run.ctx.vvs_read_state()).cuda()
    n, parent = shape.n_nodes, np.asarray([max(0, j - 2) for j in range(shape.n_nodes)], dtype=np.int32)
    q, toks = synth.make_draft(shape, parent, 0)
    args = [torch.from_numpy(x).cuda() for x in (toks, q, synth.make_uniforms(shape, n, 0))]

    def call():
        run.ctx.vvs_set_state(state)
        run.ctx.vvs_verify(n, parent, None, *args, vb.VVS_STRICT, *run.out)
        run.ctx.vvs_kv_commit()

    call()
    want = run.ctx.vvs_debug_logits()[0].clone()
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        call()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            call()
    for i in range(6):
        with torch.cuda.stream(stream):
            graph.replay()
        stream.synchronize()
        assert torch.equal(run.ctx.vvs_debug_logits()[0], want)
        call()
        torch.cuda.synchronize()
        assert torch.equal(run.ctx.vvs_debug_logits()[0], want)
    run.ctx.close()


def test_features_and_eviction_go_with_weights_in_8_bits():
    run = Run(BF16, vb.VVS_CACHE_E4M3)
    run.prefill(60)
    run.step(0)
    run.ctx.vvs_kv_evict(32, 8)
    assert (run.ctx.vvs_read_state()[0] == 32).all()
    features, count = run.ctx.vvs_read_features()
    assert np.isfinite(features).all() and (np.asarray(count) >= 2).all()
    run.ctx.close()
