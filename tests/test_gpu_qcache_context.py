"""Contexts that hold their cache in 8 bits (VVS_CACHE_E4M3) in lockstep with the oracle.  After every call that caches tokens, what the context holds is compared with the oracle's
own keys and values rounded as the cache does - a value may lie one e4m3 step off where fp32 and 64 bits fall on two sides of a border - and then becomes the oracle's cache, so
that the next forward is compared on the same cache: fp32 logits to 1e-4 and decisions equal, bf16 logits to the bound of the parity tests (3e-2, or three times what the oracle itself moves
by under a 1e-7 perturbation in front of its rounding points)."""
import dataclasses

import numpy as np
import pytest
import torch

import gpu_common as gc
import qcache_common as qc
from oracle import vvs_oracle as vo
from paper_2511_13587_amd import binding as vb
from paper_2511_13587_amd import synth

pytestmark = pytest.mark.gpu

FP32 = synth.TINY.replace(n_prompts=2, n_nodes=9)
BF16 = synth.XL_TREE.replace(n_layers=2, n_prompts=2, prefix_len=8)


class Run:
    def __init__(self, shape):
        self.shape, self.mixed = shape, False
        self.w = synth.make_weights(shape)
        self.ctx = vb.Context(vb.make_config(shape, cache_kind=vb.VVS_CACHE_E4M3))
        self.ctx.load_weights_from_host(self.w, synth.weight_names(shape))
        cfg = dict(dataclasses.asdict(shape), feature_slots=5, feature_pre_norm=0)
        self.ora = vo.Oracle(cfg, self.w)
        self.shadow = gc.perturbed_rounding(vo.Oracle(cfg, self.w)) if shape.dtype == synth.DTYPE_BF16 else None
        self.out = [torch.zeros(n, dtype=torch.int32, device="cuda") for n in (shape.n_prompts, (shape.n_prompts, vb.VVS_MAX_T), shape.n_prompts)]

    def held(self, layer, row, n):
        k, v = self.ctx.vvs_debug_kv(layer, row, n)
        return [x.double().cpu().numpy().reshape(n, self.ora.H, self.ora.dh) for x in (k, v)]

    def take_cache(self, before):
        """Compares what was cached since the lengths `before` and hands the context's cache to the oracle."""
        o = self.ora
        for row in range(o.R):
            n, m = o.kv_len(row // 2), before[row // 2]
            for l in range(o.L):
                got = self.held(l, row, n)
                for have, own in zip(got, (o.kc[row][l], o.vc[row][l])):
                    ref = qc.Cache(1, 1, o.H, n, o.dh)
                    if m:
                        ref.append(0, 0, 0, own[:m], own[:m])
                    ref.append(0, 0, m, own[m:], own[m:])
                    want = ref.k[0, 0, :, :n].transpose(1, 0, 2)
                    unit = 2.0 ** np.repeat(ref.ke[0, 0], 32, axis=1)[:, :n].T[:, :, None].astype(float)
                    step = np.maximum(np.abs(want) * 2.0 ** -3, unit * 2.0 ** -9)          # largest distance of e4m3 neighbours there, or of two exponents
                    noise = 2e-5 if self.shape.dtype == synth.DTYPE_FP32 else 3e-2
                    assert (np.abs(have - want) <= step + noise).all(), (l, row, np.abs(have - want).max())
                    if self.shape.dtype == synth.DTYPE_FP32:
                        assert (have != want).mean() < 0.01
                for x in (o,) + ((self.shadow,) if self.shadow else ()):
                    x.kc[row][l], x.vc[row][l] = got[0].copy(), got[1].copy()

    def tolerance(self, key):
        if self.shadow is None:
            return 1e-4
        return max(3e-2, 3 * float(np.abs(getattr(self.shadow, key) - getattr(self.ora, key)).max()))

    def prefill(self, n_forced):
        s = self.shape
        pc, pu = synth.make_prefix(s)
        forced = synth.make_forced_tokens(s, n_forced) if n_forced else None
        self.ora.prefill(pc, pu, forced, np.full(s.n_prompts, 0.5))
        u = np.array([p[:int(np.argmax(p))].sum() + 0.5 * p.max() for p in self.ora.prefill_probs], dtype=np.float32)
        self.ora.prefill(pc, pu, forced, u)
        if self.shadow:
            self.shadow.prefill(pc, pu, forced, u)
            self.shadow.pending[:] = self.ora.pending
        dpc, dpu = (torch.from_numpy(pc).cuda(), None) if s.prefix_kind == synth.PREFIX_CLASS else (vb.to_device(pc, s.dtype), vb.to_device(pu, s.dtype))
        self.ctx.vvs_prefill(dpc, dpu, None if forced is None else torch.from_numpy(forced).cuda(), torch.from_numpy(u).cuda(), self.out[2])
        raw, _, _ = self.ctx.vvs_debug_logits()
        err = float(np.abs(raw.cpu().numpy()[:, 0] - self.ora.prefill_logits).max())
        assert err <= self.tolerance("prefill_logits"), err
        assert (self.out[2].cpu().numpy() == self.ora.pending).all()
        self.take_cache([0] * s.n_prompts)

    def step(self, seed, tree=True, n_post=0, mode=0, uneven=False):
        s, n = self.shape, self.shape.n_nodes
        parent = np.asarray([min(j, n_post) if j <= n_post else max(n_post, j - 2) for j in range(n)], dtype=np.int32) if tree else None
        q, toks = synth.make_draft(s, parent if parent is not None else synth.tree_parents(None, n), seed)
        u = synth.make_uniforms(s, n, seed)
        u[:, 1 + seed % 3, 0] = 0.0                                # some tokens are accepted
        if uneven:                                                 # the first prompt takes what it can, the others next to nothing
            u[0, :, 0], u[1:, :, 0] = 0.0, 0.999999
        before = [self.ora.kv_len(b) for b in range(s.n_prompts)]
        args = (torch.from_numpy(toks).cuda(), torch.from_numpy(q).cuda(), torch.from_numpy(u).cuda(), mode, *self.out)
        if n_post:
            self.ctx.vvs_verify_post(n, n_post, parent, None, *args)
        else:
            self.ctx.vvs_verify(n, parent, None, *args)
        acc, paths, nxt = self.ora.verify(parent, toks, q, u, mode, n_post)
        if self.shadow:
            self.shadow.verify(parent, toks, q, u, mode, n_post)
        raw, _, _ = self.ctx.vvs_debug_logits()
        err = float(np.abs(raw.cpu().numpy() - self.ora.raw_logits).max())
        assert err <= self.tolerance("raw_logits"), err
        a, p, t = (x.cpu().numpy() for x in self.out)
        if s.dtype == synth.DTYPE_FP32:
            assert (a == acc).all() and (t == nxt).all() and all((p[b, :acc[b] + 1] == paths[b]).all() for b in range(s.n_prompts))
        else:                                                      # the oracle follows the library's decisions: a draw within the noise may fall either way
            for x in (self.ora, self.shadow):
                x.last["paths"] = [[int(v) for v in p[b, :a[b] + 1]] for b in range(s.n_prompts)]
                x.last["accept_len"], x.last["next_token"] = a.copy(), t.copy()
        self.ctx.vvs_kv_commit()
        self.ora.kv_commit()
        if self.shadow:
            self.shadow.kv_commit()
        state = self.ctx.vvs_read_state()
        assert (state[0] == [self.ora.kv_len(b) for b in range(s.n_prompts)]).all() and (state[1] == self.ora.n_emitted).all()
        self.take_cache(before)
        return a

    def evict(self, keep, recent):
        """Evicts on the GPU, checks that every head keeps `keep` of its slots and the newest, and hands the cache to the oracle."""
        o = self.ora
        lens = [o.kv_len(b) for b in range(o.B)]
        was = {(l, r): self.held(l, r, lens[r // 2]) for l in range(o.L) for r in range(o.R)}
        # before the first eviction the newest tokens are in the last slots; later only the library knows where they are
        newest = [set() if self.mixed else set(range(max(0, n - recent), n)) for n in lens]
        self.ctx.vvs_kv_evict(keep, recent)
        state = self.ctx.vvs_read_state()
        assert (state[0] == np.minimum(lens, keep)).all() and (state[1] == o.n_emitted).all()
        for (l, r), (k, v) in was.items():
            n = min(lens[r // 2], keep)
            k2, v2 = self.held(l, r, n)
            for h in range(o.H):
                # (a moved element may be rounded again, by half a step of the larger power of two: 2^-10 of the largest e4m3 number's unit)
                d = np.abs(k2[:, None, h] - k[None, :, h]).max(axis=2)
                at = d.argmin(axis=1)
                assert (d[np.arange(n), at] <= 2.0 ** -10 * np.abs(k[:, h]).max()).all()
                assert len(set(at.tolist())) == n and newest[r // 2] <= set(at.tolist())
                assert np.abs(v2[:, h] - v[at, h]).max() <= 2.0 ** -10 * np.abs(v[:, h]).max()
            for x in (o,) + ((self.shadow,) if self.shadow else ()):
                x.kc[r][l], x.vc[r][l] = k2, v2
        self.mixed = True


@pytest.mark.parametrize("shape,forced", [(FP32, 5), (FP32.replace(d_model=256, n_heads=4, d_ff=512), 20), (BF16, 5),
                                          (BF16.replace(d_model=512, n_heads=4, d_ff=1024, n_layers=1), 30)], ids=["fp32_32", "fp32_64", "bf16_64", "bf16_128"])
def test_steps_and_eviction_in_lockstep_with_the_oracle(shape, forced):
    run = Run(shape)
    run.prefill(forced)
    for i, kw in enumerate((dict(), dict(tree=False), dict(n_post=2), dict())):
        run.step(i, **kw)
    if run.ora.kv_len(0) > 32 or shape is FP32:
        run.evict(32, 6)
    run.step(7)
    run.step(8, n_post=1)
    run.evict(32, 4)
    run.step(9)
    run.ctx.close()


def test_prefill_in_chunks_sees_what_was_cached():
    """The second chunk of a prefill attends to the first one's keys and values in 8 bits."""
    shape = FP32.replace(grid_h=12, grid_w=12, n_prompts=1)
    run = Run(shape)
    pc, pu = synth.make_prefix(shape)
    forced = synth.make_forced_tokens(shape, 140)
    u = torch.full((1,), 0.5, device="cuda")
    run.ctx.vvs_prefill(torch.from_numpy(pc).cuda(), None, torch.from_numpy(forced).cuda(), u, run.out[2])
    raw, _, _ = run.ctx.vvs_debug_logits()
    o = run.ora
    for row, pre in enumerate(o.prefix_embeddings(pc, pu, 0)):
        x = np.concatenate([pre, o.embed_tokens(forced[0])])
        idx = [-1] * o.P + list(range(140))
        for c in range(0, len(idx), 64):
            t = min(64, len(idx) - c)
            logits, kv = o.forward_block(row, x[c:c + t], idx[c:c + t], np.tril(np.ones((t, t))))
            for l in range(o.L):
                got = run.held(l, row, c + t)
                for have, own in zip(got, kv[l]):
                    ref = qc.Cache(1, 1, o.H, t, o.dh)
                    ref.append(0, 0, 0, own, own)
                    want = ref.k[0, 0, :, :t].transpose(1, 0, 2)
                    assert (np.abs(have[c:] - want) <= np.abs(want) * 2.0 ** -3 + 2e-5).all()
                o.kc[row][l], o.vc[row][l] = got
        assert np.abs(raw.cpu().numpy()[row, 0] - logits[-1]).max() <= 1e-4
    run.ctx.close()


def test_prompts_that_finish_at_different_steps():
    """A finished prompt answers -1 and what it holds stays as it is, bit for bit, while the other goes on; an eviction shortens both."""
    run = Run(FP32)
    total = FP32.grid_h * FP32.grid_w
    run.prefill(total - 12)
    uneven = False
    for i in range(14):
        emitted = run.ora.n_emitted.copy()
        done = [b for b in range(FP32.n_prompts) if emitted[b] >= total]
        was = {(l, r): run.held(l, r, run.ora.kv_len(r // 2)) for l in range(run.ora.L) for r in range(run.ora.R) if r // 2 in done}
        uneven |= len(done) == 1
        a = run.step(i, uneven=True)
        nxt = run.out[2].cpu().numpy()
        assert all(nxt[b] == -1 and a[b] == 0 and run.ora.n_emitted[b] == emitted[b] for b in done)
        for (l, r), held in was.items():
            now = run.held(l, r, len(held[0]))
            assert all((x == y).all() for x, y in zip(now, held))
        if len(done) == FP32.n_prompts:
            break
    assert len(done) == FP32.n_prompts and uneven
    run.evict(32, 6)
    run.ctx.close()


def test_rollback_and_the_feature_cache():
    """A step replayed from a saved state gives the same outcome, and features are those of a context that keeps bf16."""
    shape = BF16
    w = synth.make_weights(shape)
    pc, pu = synth.make_prefix(shape)
    feats = []
    for kind in (vb.VVS_CACHE_E4M3, vb.VVS_CACHE_SAME):
        ctx = vb.Context(vb.make_config(shape, cache_kind=kind, norm_mode=vb.VVS_NORM_SEPARATE))
        ctx.load_weights_from_host(w, synth.weight_names(shape))
        first = torch.zeros(2, dtype=torch.int32, device="cuda")
        ctx.vvs_prefill(vb.to_device(pc, shape.dtype), vb.to_device(pu, shape.dtype), torch.from_numpy(synth.make_forced_tokens(shape, 9)).cuda(),
                        torch.full((2,), 0.5, device="cuda"), first)
        f, n = ctx.vvs_read_features()
        feats.append((f[:, :1], n))
        if kind == vb.VVS_CACHE_E4M3:
            state = torch.from_numpy(ctx.vvs_read_state()).cuda()
            parent = synth.tree_parents(shape.tree_widths, shape.n_nodes)
            q, toks = synth.make_draft(shape, parent, 1)
            u = synth.make_uniforms(shape, shape.n_nodes, 1)
            seen = []
            for _ in range(3):
                ctx.vvs_set_state(state)
                a, p, t = (torch.zeros(d, dtype=torch.int32, device="cuda") for d in (2, (2, vb.VVS_MAX_T), 2))
                ctx.vvs_verify(shape.n_nodes, parent, None, torch.from_numpy(toks).cuda(), torch.from_numpy(q).cuda(), torch.from_numpy(u).cuda(), vb.VVS_STRICT, a, p, t)
                raw = ctx.vvs_debug_logits()[0]
                with pytest.raises(vb.VvsError) as e:
                    ctx.vvs_kv_evict(32, 0)
                assert e.value.status == vb.VVS_ESTATE
                ctx.vvs_kv_commit()
                seen.append((raw.cpu(), a.cpu(), t.cpu(), ctx.vvs_read_state()))
            for x in seen[1:]:
                assert torch.equal(x[0], seen[0][0]) and torch.equal(x[1], seen[0][1]) and torch.equal(x[2], seen[0][2]) and (x[3] == seen[0][3]).all()
        else:
            with pytest.raises(vb.VvsError) as e:
                ctx.vvs_kv_evict(32, 0)
            assert e.value.status == vb.VVS_ESTATE
        ctx.close()
    # the prefix is one chunk, whose tokens see each other unrounded: the two contexts differ by the sums' order alone
    assert (feats[0][1] == feats[1][1]).all()
    assert np.abs(feats[0][0] - feats[1][0]).max() <= 3e-2 * max(1.0, np.abs(feats[1][0]).max())


def test_refusals():
    for kw, status in ((dict(cache_kind=2), vb.VVS_EINVAL), (dict(cache_kind=1, draft_input=1, feature_slots=0), vb.VVS_EINVAL)):
        with pytest.raises(vb.VvsError) as e:
            vb.Context(vb.make_config(BF16, **kw))
        assert e.value.status == status
    with pytest.raises(vb.VvsError) as e:
        vb.Context(vb.make_config(synth.TINY.replace(n_heads=8), cache_kind=1))           # head size 16
    assert e.value.status == vb.VVS_ESIZE
    run = Run(FP32)
    with pytest.raises(vb.VvsError) as e:
        run.ctx.vvs_kv_evict(32, 0)
    assert e.value.status == vb.VVS_ESTATE
    run.prefill(0)
    for keep, recent in ((0, 0), (31, 0), (32, 33), (32, -1)):
        with pytest.raises(vb.VvsError) as e:
            run.ctx.vvs_kv_evict(keep, recent)
        assert e.value.status == vb.VVS_EINVAL
    run.ctx.close()
