"""Contexts with their cache in 8 bits: vvs_kv_evict keeps the slots of largest accumulated weight and the newest tokens, weights and positions kept by the 64-bit oracle beside the context."""
import numpy as np
import pytest

from oracle import vvs_oracle as vo
from paper_2511_13587_amd import synth
from test_gpu_qcache_context import FP32, Run

pytestmark = pytest.mark.gpu


class Counted(Run):
    """Run, with the weights that the oracle's attention gives to every slot ([layer][heads, slots] per row) and the slots' positions in the sequence."""

    def __init__(self, shape, monkeypatch):
        super().__init__(shape)
        self.mass, self.pos, self.n_post, self.seen = {}, {}, 0, None
        plain, forward = vo.softmax, self.ora.forward_block

        def softmax(z):
            p = plain(z)
            if self.seen is not None:
                self.seen.append(p)
            return p

        def forward_block(row, x_in, img_index, mask, logits_for=None):
            o, n = self.ora, self.ora.kc[row][0].shape[0]
            self.seen = []
            got = forward(row, x_in, img_index, mask, logits_for)
            seen, self.seen = self.seen, None
            weights = np.stack(seen).reshape(o.L, o.H, len(x_in), -1)
            if n == 0:                                              # a prefill: all tokens count, over each other
                self.mass[row], self.pos[row] = weights.sum(axis=2), np.broadcast_to(np.arange(len(x_in)), (o.L, o.H, len(x_in))).copy()
            else:                                                   # a verify call: the tokens certain to be kept, over what is cached
                self.mass[row] = self.mass[row] + weights[:, :, :1 + self.n_post, :n].sum(axis=2)
            return got

        monkeypatch.setattr(vo, "softmax", softmax)
        self.ora.forward_block = forward_block

    def step(self, seed, n_post=0, **kw):
        emitted, self.n_post = self.ora.n_emitted.copy(), n_post
        a = super().step(seed, n_post=n_post, **kw)
        for r in self.mass:
            more = self.ora.kv_len(r // 2) - self.mass[r].shape[2]
            side = (self.ora.L, self.ora.H, more)
            self.mass[r] = np.concatenate([self.mass[r], np.zeros(side)], axis=2)
            self.pos[r] = np.concatenate([self.pos[r], np.broadcast_to(self.ora.P - 1 + emitted[r // 2] + np.arange(more), side)], axis=2)
        return a

    def evict_by_rule(self, keep, recent):
        """Compares what stays with the rule; returns how many slots went by their weight.  Weights of both sides are sums of at most a few dozen softmax weights whose scores agree to 1e-5 of
        themselves: slots whose weights lie within 1e-4 of each other may change places."""
        o, by_weight = self.ora, 0
        lens = [o.kv_len(b) for b in range(o.B)]
        was = {(l, r): self.held(l, r, lens[r // 2]) for l in range(o.L) for r in range(o.R)}
        self.ctx.vvs_kv_evict(keep, recent)
        assert (self.ctx.vvs_read_state()[0] == np.minimum(lens, keep)).all()
        mass, pos = {r: np.zeros((o.L, o.H, min(lens[r // 2], keep))) for r in self.mass}, {r: np.zeros((o.L, o.H, min(lens[r // 2], keep)), dtype=int) for r in self.mass}
        for (l, r), (k, v) in was.items():
            n, left = lens[r // 2], min(lens[r // 2], keep)
            k2, v2 = self.held(l, r, left)
            for h in range(o.H):
                d = np.abs(k2[:, None, h] - k[None, :, h]).max(axis=2)
                origin = d.argmin(axis=1)
                assert (d[np.arange(left), origin] <= 2.0 ** -10 * np.abs(k[:, h]).max()).all() and len(set(origin.tolist())) == left
                assert np.abs(v2[:, h] - v[origin, h]).max() <= 2.0 ** -10 * np.abs(v[:, h]).max()
                m, p = self.mass[r][l, h], self.pos[r][l, h]
                stays = np.zeros(n, dtype=bool)
                stays[origin] = True
                new = p > p.max() - recent
                if n > keep:
                    assert stays[new].all(), "a newest token went"
                    old_kept, gone = stays & ~new, ~stays
                    by_weight += int(gone.sum())
                    if old_kept.any():
                        assert m[old_kept].min() >= m[gone].max() - 1e-4, (l, r, h, m[old_kept].min(), m[gone].max())
                moved = origin != np.arange(left)
                assert (~stays[:left] == moved).all() and (np.diff(origin[moved]) > 0).all() and (origin[moved] >= keep).all()
                mass[r][l, h], pos[r][l, h] = m[origin], p[origin]
            o.kc[r][l], o.vc[r][l] = k2, v2
        self.mass, self.pos = mass, pos
        return by_weight


@pytest.mark.parametrize("shape,forced", [(FP32, 40), (FP32.replace(d_model=256, n_heads=4, d_ff=512), 45)], ids=["heads_of_32", "heads_of_64"])
def test_evictions_keep_the_slots_of_largest_weight(shape, forced, monkeypatch):
    """Prefill, verify calls of every kind, commits, three evictions: the later ones go by weights and positions that moved with their slots, and by the positions that commits noted."""
    make = synth.make_weights
    # queries and keys five times as large: weights that tell slots apart by more than their age
    monkeypatch.setattr(synth, "make_weights", lambda s: {name: w * np.float32(5) if name.endswith((".wq", ".wk")) else w for name, w in make(s).items()})
    run = Counted(shape, monkeypatch)
    run.prefill(forced)
    run.step(1)
    run.step(2, n_post=2)
    assert run.evict_by_rule(32, 6) > 0
    for recent, seeds in ((3, (3, 4)), (0, (5, 6, 7))):
        for s in seeds:
            run.step(s, n_post=s % 2)
        assert all(run.ora.kv_len(b) > 32 for b in range(shape.n_prompts))
        assert run.evict_by_rule(32, recent) > 0
    run.step(9)
    run.ctx.close()
