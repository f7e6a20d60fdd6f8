"""An attention call's output beside its inputs: what shares memory with the queries, keys or values is refused by the binding (the queries are read again, for the counted weights, behind the outputs)."""
import pytest
import torch

from paper_2511_13587_amd import binding as vb


def refused(out, parts):
    """parts: [rows, tokens, heads, size] each."""
    cpu = out.get_device()
    found = [(*vb._per_token(x, cpu, x.dtype, tuple(x.shape), "x"), x.shape[2] * x.shape[3]) for x in parts]
    try:
        vb._apart(out.data_ptr(), out.numel(), [(None, 0, 0)] + found, parts[0].shape[0] * parts[0].shape[1], out.element_size())
    except ValueError:
        return True
    return False


def test_outputs_that_share_memory_are_found():
    wide = torch.zeros((2, 5, 8, 64), dtype=torch.bfloat16)
    parts = wide.split([4, 2, 2], dim=2)
    flat = wide.view(-1)
    out = lambda at: flat[at:at + 2 * 5 * 4 * 64].view(2, 5, 4, 64)  # noqa: E731
    assert refused(out(0), parts) and refused(out(64), parts) and refused(out(2560), parts)
    assert not refused(torch.zeros((2, 5, 4, 64), dtype=torch.bfloat16), parts)
    # neighbours in one buffer, in front of the inputs and behind them
    buf = torch.zeros(2 * 2 * 5 * 4 * 64, dtype=torch.bfloat16)
    half = buf.numel() // 2
    lo, hi = buf[:half].view(2, 5, 4, 64), buf[half:].view(2, 5, 4, 64)
    assert not refused(lo, [hi]) and not refused(hi, [lo]) and refused(lo, [lo])
    # a single token's output beside its own queries, keys and values
    one = torch.zeros(12 * 64, dtype=torch.bfloat16)
    parts = one[:8 * 64].view(1, 1, 8, 64).split([4, 2, 2], dim=2)
    assert not refused(one[8 * 64:].view(1, 1, 4, 64), parts) and refused(one[7 * 64:11 * 64].view(1, 1, 4, 64), parts)


@pytest.mark.gpu
def test_attention_into_its_own_inputs_is_refused():
    cache = vb.QCache(1, 2, 4, 2, 64, 64, 8, vb.VVS_BF16)
    n = torch.zeros(2, dtype=torch.int32, device="cuda")
    qkv = torch.zeros((2, 8, 8, 64), dtype=torch.bfloat16, device="cuda")
    wide = qkv.split([4, 2, 2], dim=2)
    q, k, v = (x.contiguous() for x in wide)
    mass, block = torch.zeros((2, 2, 64), device="cuda"), torch.zeros((2, 2, 8), device="cuda")
    inside = qkv.view(-1)[:q.numel()].view(q.shape)
    for args, kw in (((*wide, inside), {}), ((q, k, v, q), dict(n_counted=8, mass=mass)), ((q, k, v, q), dict(block_mass=block)), ((q, q[:, :, :2].clone(), wide[2], inside), {})):
        with pytest.raises(ValueError):
            cache.vvs_qcache_attention(n, *args, **kw)
    cache.vvs_qcache_attention(n, *wide, torch.empty_like(q), n_counted=8, mass=mass, block_mass=block)
    torch.cuda.synchronize()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,heads,kv_heads,size,tokens,capacity", [("bf16", 4, 4, 64, 1, 64), ("bf16", 8, 2, 128, 9, 1300), ("bf16", 4, 2, 64, 30, 64), ("bf16", 8, 1, 64, 40, 640),
                                                                       ("bf16", 8, 1, 128, 40, 1300), ("fp32", 4, 2, 64, 33, 1300)])
def test_attention_over_its_queries_in_place(dtype, heads, kv_heads, size, tokens, capacity):
    """Where no weights are counted the output may be the queries themselves: the same bits as into a buffer of its own, in every form."""
    dt = torch.float32 if dtype == "fp32" else torch.bfloat16
    g = torch.Generator("cuda").manual_seed(tokens)
    new = lambda *d: torch.randn(d, generator=g, device="cuda").to(dt)  # noqa: E731
    cache = vb.QCache(1, 2, heads, kv_heads, size, capacity, tokens, vb.VVS_FP32 if dtype == "fp32" else vb.VVS_BF16)
    n = torch.zeros(2, dtype=torch.int32, device="cuda")
    cache.vvs_qcache_append(n, new(1, 2, capacity, kv_heads, size), new(1, 2, capacity, kv_heads, size))
    q, k, v = new(2, tokens, heads, size), new(2, tokens, kv_heads, size), new(2, tokens, kv_heads, size)
    out = torch.empty_like(q)
    cache.vvs_qcache_attention(n + capacity - 3, q, k, v, out)
    cache.vvs_qcache_attention(n + capacity - 3, q, k, v, q)
    assert torch.equal(q, out)
