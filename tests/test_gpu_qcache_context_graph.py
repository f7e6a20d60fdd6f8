"""Steps of a context with its cache in 8 bits, captured and replayed: verify + commit in one graph, the eviction in a second, against a context that runs them eagerly, with eager work between the
replays.  Everything that a context keeps is compared to the bit."""
import numpy as np
import pytest
import torch

from paper_2511_13587_amd import binding as vb
from paper_2511_13587_amd import synth

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape,n_post", [(synth.TINY.replace(n_prompts=2, n_nodes=9), 2), (synth.XL_TREE.replace(n_layers=2, n_prompts=2, prefix_len=8), 0)], ids=["fp32", "bf16"])
def test_captured_steps_replay_as_they_run(shape, n_post):
    w, n = synth.make_weights(shape), shape.n_nodes
    pc, pu = synth.make_prefix(shape)
    dpc, dpu = (torch.from_numpy(pc).cuda(), None) if shape.prefix_kind == synth.PREFIX_CLASS else (vb.to_device(pc, shape.dtype), vb.to_device(pu, shape.dtype))
    parent = np.asarray([j if j < n_post else max(n_post, j - 2) for j in range(n)], dtype=np.int32)
    toks, q, u = (torch.empty(d, dtype=t, device="cuda") for d, t in (((shape.n_prompts, n), torch.int32), ((shape.n_prompts, n + 1, shape.v_eff), torch.float32),
                                                                      ((shape.n_prompts, n + 1, 2), torch.float32)))

    def inputs(seed):
        dq, dt = synth.make_draft(shape, parent, seed)
        du = synth.make_uniforms(shape, n, seed)
        du[:, :4, 0] = 0.0                                             # some tokens are accepted
        for x, y in ((toks, dt), (q, dq), (u, du)):
            x.copy_(torch.from_numpy(y))

    class Side:
        def __init__(self):
            self.ctx = vb.Context(vb.make_config(shape, cache_kind=vb.VVS_CACHE_E4M3))
            self.ctx.load_weights_from_host(w, synth.weight_names(shape))
            self.out = [torch.zeros(d, dtype=torch.int32, device="cuda") for d in (shape.n_prompts, (shape.n_prompts, vb.VVS_MAX_T), shape.n_prompts)]
            self.ctx.vvs_prefill(dpc, dpu, torch.from_numpy(synth.make_forced_tokens(shape, 33)).cuda(), torch.full((shape.n_prompts,), 0.5, device="cuda"), self.out[2])

        def step(self):
            if n_post:
                self.ctx.vvs_verify_post(n, n_post, parent, None, toks, q, u, vb.VVS_STRICT, *self.out)
            else:
                self.ctx.vvs_verify(n, parent, None, toks, q, u, vb.VVS_STRICT, *self.out)
            self.ctx.vvs_kv_commit()

        def shorten(self):
            self.ctx.vvs_kv_evict(32, 5)

        def snapshot(self):
            return [self.ctx.kv.clone(), *(x.clone() for x in self.out), torch.from_numpy(self.ctx.vvs_read_state())]

    inputs(0)
    warm = Side()                                                       # (a first use's lazy loading stays out of the capture)
    warm.step(), warm.shorten()
    torch.cuda.synchronize()
    warm.ctx.close()
    eager, taped = Side(), Side()
    torch.cuda.synchronize()
    step, shorten = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.graph(step, stream=side):
        taped.step()
    with torch.cuda.graph(shorten, stream=side):
        taped.shorten()
    for i in range(5):
        inputs(i + 1)
        eager.step()
        step.replay()
        if i in (1, 3):
            eager.shorten()
            shorten.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager.snapshot(), taped.snapshot()):
            assert torch.equal(a, b), f"replay {i}"
    eager.ctx.close()
    taped.ctx.close()
