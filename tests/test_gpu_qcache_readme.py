"""The README's decoding loop over the 8-bit cache, executed as it stands there: positions of appended slots are the caller's, and an eviction goes by them."""
import os

import numpy as np
import pytest
import torch

from paper_2511_13587_amd import binding

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def the_loop():
    """(what stands in front of the loop over the layers, one step)"""
    with open(os.path.join(ROOT, "README.md")) as f:
        text = f.read()
    code = text[text.index("## A cache in 8 bits"):].split("```python\n")[1].split("```")[0]
    at = code.index("for layer in")
    return code[:at], code[at:]


def test_the_readme_loop_keeps_the_newest_tokens():
    setup, step = the_loop()
    n_layers, rows, heads, kv_heads, head_size, capacity, keep, recent, tokens = 2, 3, 4, 2, 128, 96, 64, 20, 6
    g = torch.Generator("cuda").manual_seed(1)
    new = lambda *d: torch.randn(d, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    length, emitted = (torch.tensor([40, 64, 33], dtype=torch.int32, device="cuda") for _ in range(2))
    tree = np.asarray([0, 0, 1, 2, 3], dtype=np.int32)
    path = torch.tensor([[0, 1, 3, 5]] * rows, dtype=torch.int32, device="cuda")
    scope = dict(torch=torch, binding=binding, n_layers=n_layers, rows=rows, heads=heads, kv_heads=kv_heads, head_size=head_size, capacity=capacity, max_tokens=tokens, keep=keep, recent=recent,
                 length=length, emitted=emitted, tree=tree, path=path, mass=torch.zeros((n_layers, rows, kv_heads, capacity), device="cuda"),
                 out=torch.empty((rows, tokens, heads, head_size), dtype=torch.bfloat16, device="cuda"),
                 staged_k=torch.empty((n_layers, rows, tokens, kv_heads, head_size), dtype=torch.bfloat16, device="cuda"),
                 staged_v=torch.empty((n_layers, rows, tokens, kv_heads, head_size), dtype=torch.bfloat16, device="cuda"))
    exec(setup, scope)
    scope["cache"].vvs_qcache_append(torch.zeros_like(length), new(n_layers, rows, 64, kv_heads, head_size), new(n_layers, rows, 64, kv_heads, head_size), n_tokens=length, n_layers=n_layers)
    for i in range(16):
        scope["qkv"] = new(n_layers, rows, tokens, heads + 2 * kv_heads, head_size)
        scope["positions"] = torch.stack([emitted // 64, emitted // 8 % 8, emitted % 8], dim=-1)[:, None].expand(rows, tokens, 3).contiguous()
        scope["accepted"] = torch.tensor([1 + (i + r) % 4 for r in range(rows)], dtype=torch.int32, device="cuda")
        was, was_emitted = scope["length"].clone(), scope["emitted"].clone()
        exec(step, scope)
        pos = scope["position_of_slot"].cpu().numpy()
        now, out_of = scope["length"].tolist(), scope["emitted"].tolist()
        assert now == torch.minimum(was + scope["accepted"], torch.tensor(keep, device="cuda")).tolist() and out_of == (was_emitted + scope["accepted"]).tolist()
        for r in range(rows):
            for held in pos[:, r, :, :now[r]].reshape(-1, now[r]):
                assert len(set(held.tolist())) == now[r] and held.min() >= 0 and held.max() == out_of[r] - 1
                assert set(range(out_of[r] - recent, out_of[r])) <= set(held.tolist()), "the newest tokens went"
    assert min(now) == keep
