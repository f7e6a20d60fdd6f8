"""The README's layer with weights in 8 bits, executed as it stands there."""
import os

import pytest
import torch

import qlinear_common as qc
from paper_2511_13587_amd import binding
from test_gpu_qlinear import _normal

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def the_layer():
    with open(os.path.join(ROOT, "README.md")) as f:
        text = f.read()
    return text[text.index("## Weights in 8 bits"):].split("```python\n")[1].split("```")[0]


def test_the_readme_layer():
    """A layer of it for 1, 7 and 40 rows, beside its statement in 64 bits with the weights that are held and rows rounded where the layer rounds them.

    2-norms: a rounding to e4m3 is off by half a step at most, spread over it: 2^-4 / sqrt(3) = 3.6e-2.  Two sides that round operands that differ a little are apart by sqrt(2) of that at most, 5.1e-2, independent
    of what they differed by.  What is added to x behind attention: two roundings, 7.2e-2 of it.  What the layer leaves for the next: the second norm's rows, sqrt(7.2e-2^2 + 5.1e-2^2) = 8.8e-2; of two factors that
    both come from them 17.6e-2; rounded again sqrt(17.6e-2^2 + 5.1e-2^2) = 18.4e-2."""
    d, heads, head_size, d_hidden, max_rows, eps = 256, 4, 64, 700, 40, 1e-5
    e = heads * head_size
    w = {k: (_normal(s, 3 + i) * s[0] ** -0.5).bfloat16() for i, (k, s) in enumerate({"w_qkv": (d, 3 * e), "w_o": (e, d), "w_up": (d, d_hidden), "w_gate": (d, d_hidden), "w_down": (d_hidden, d)}.items())}
    gains = {"gain_1": 1 + 0.2 * _normal((d,), 11, 0), "gain_2": 1 + 0.2 * _normal((d,), 12, 0)}

    def attention(qkv, out):                           # (each token its own value, as a layer over one token each would)
        out.copy_(qkv.view(-1, 3, e)[:, 2])

    scope = dict(torch=torch, binding=binding, d=d, heads=heads, head_size=head_size, d_hidden=d_hidden, max_rows=max_rows, eps=eps, attention=attention,
                 workspace=torch.empty(4 << 20, dtype=torch.uint8, device="cuda"), qkv=torch.empty((max_rows, 3 * e), dtype=torch.bfloat16, device="cuda"),
                 out=torch.empty((max_rows, e), dtype=torch.bfloat16, device="cuda"), summand=torch.empty((max_rows, d), device="cuda"),
                 **{k: v.cuda() for k, v in {**w, **gains}.items()})
    exec(the_layer(), scope)
    held = {k: qc.held(v.t())[0].t() for k, v in w.items()}
    round8 = lambda x: qc.held(x)[0]  # noqa: E731

    def norm(x, gain):
        return round8(x / torch.sqrt((x * x).mean(dim=1, keepdim=True) + eps) * gain.double())

    for n in (1, 7, 40):
        x, delta = _normal((n, d), 20 + n), _normal((n, d), 21 + n)
        gx, gd = x.cuda(), delta.cuda()
        x, delta = x.double(), delta.double()
        gx, gd = scope["layer"](gx, gd)
        x = x + delta
        v = (norm(x, gains["gain_1"]) @ held["w_qkv"])[:, 2 * e:]
        attended = round8(v.bfloat16().double()) @ held["w_o"]
        x = x + attended
        rows = norm(x, gains["gain_2"])
        delta = round8(torch.nn.functional.silu(rows @ held["w_gate"]) * (rows @ held["w_up"])) @ held["w_down"]
        assert (gx.cpu().double() - x).norm() < 7.2e-2 * attended.norm() + 1e-6 * x.norm()
        assert (gd.cpu().double() - delta).norm() < 18.4e-2 * delta.norm()
