"""Contexts with their cache in 8 bits: what a roll-back does to the values of a block that the discarded tokens were rounded into."""
import numpy as np
import pytest
import torch

import qcache_common as qc
from paper_2511_13587_amd import binding as vb
from paper_2511_13587_amd import synth
from test_gpu_qcache_context import FP32, Run

pytestmark = pytest.mark.gpu


def test_rolled_back_tokens_leave_their_power_of_two(monkeypatch):
    """Tokens much larger than those in their block are committed and rolled back: the block keeps the larger power of two and its slots the rounding to it, replays see those values, and from the
    first one on they all give the same bits."""
    shape = FP32.replace(n_layers=1)
    make, big = synth.make_weights, shape.logit_lo + 7

    def weights(s):
        w = make(s)
        w["embed"] = w["embed"].copy()
        w["embed"][:, 0] = 0.0
        w["embed"][big] = 0.0
        w["embed"][big, 0] = 1.0                                     # a token all in dim 0, which only it has, and whose keys and values are large
        for name in ("l0.wk", "l0.wv"):
            w[name] = w[name].copy()
            w[name][0] = np.sign(w[name][0]) * (1.0 + np.abs(w[name][0])) * 8.0
        return w

    monkeypatch.setattr(synth, "make_weights", weights)
    monkeypatch.setattr(synth, "make_forced_tokens", lambda s, n, f=synth.make_forced_tokens: np.where(f(s, n) == big, big + 1, f(s, n)))
    run = Run(shape)
    run.prefill(17)
    o, n = run.ora, run.ora.kv_len(0)
    assert n % 32 and (o.pending != big).all()
    state = torch.from_numpy(run.ctx.vvs_read_state()).cuda()
    before = [run.held(0, r, n) for r in range(o.R)]
    q, toks = synth.make_draft(shape, synth.tree_parents(None, shape.n_nodes), 1)
    toks = np.full_like(toks, big)
    u = np.zeros_like(synth.make_uniforms(shape, shape.n_nodes, 1))
    args = (torch.from_numpy(toks).cuda(), torch.from_numpy(q).cuda(), torch.from_numpy(u).cuda(), vb.VVS_STRICT, *run.out)
    logits = []
    for i in range(4):
        run.ctx.vvs_set_state(state)
        run.ctx.vvs_verify(shape.n_nodes, None, None, *args)
        logits.append(run.ctx.vvs_debug_logits()[0].clone())
        run.ctx.vvs_kv_commit()
        if i == 0:
            o.verify(None, toks, q, u, 0, 0)
            assert (run.out[0].cpu().numpy() >= 1).all()
            lost = 0
            for r in range(o.R):
                k_new, v_new = o.last["node_kv"][r // 2][r % 2][0]
                for new, old, now in zip((k_new, v_new), before[r], run.held(0, r, n)):
                    ref = qc.Cache(1, 1, o.H, n + len(new), o.dh)
                    ref.append(0, 0, 0, old, old)
                    a = int(run.out[0][r // 2])
                    ref.append(0, 0, n, new[:1 + a], new[:1 + a])      # the chain's accepted part
                    np.testing.assert_array_equal(now, ref.k[0, 0, :, :n].transpose(1, 0, 2))
                    lost += int((now != old).sum())
            assert lost > 0
            for r in range(o.R):
                o.kc[r][0], o.vc[r][0] = [x.copy() for x in run.held(0, r, n)]
            o.verify(None, toks, q, u, 0, 0)
        else:
            assert np.abs(logits[i].cpu().numpy() - o.raw_logits).max() <= 1e-4
            assert torch.equal(logits[i], logits[1])
    run.ctx.close()
