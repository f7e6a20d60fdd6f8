"""Products and rows in 8 bits at the largest numbers of rows and columns that a call takes, and calls that are captured before any has run."""
import pytest
import torch

import qlinear_common as qc
from test_gpu_qlinear import TYPES, _normal, check_gate, check_product

pytestmark = pytest.mark.gpu


def _of_a_few(rows, width):
    """QRows of `rows` rows in which the last 61 repeat the first ones' values: (rows, held values of the 61, where they are)"""
    from paper_2511_13587_amd import binding as vb
    r = vb.QRows(rows, width)
    some = vb.QRows(61, width)
    x = qc.put(some, _normal((61, width), 3))
    at = torch.arange(rows, device="cuda") % 61
    r.values.view(torch.uint8).copy_(some.values.view(torch.uint8)[at])
    r.powers.copy_(some.powers[at])
    return r, x


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("products", [0, 1])
def test_a_million_rows(dtype, products):
    from paper_2511_13587_amd import binding as vb
    rows, width, out = 1 << 20, 140, 9
    w = (_normal((width, out), 1) * width ** -0.5).bfloat16()
    lin = vb.QLinear(width, out, rows, vb.VVS_BF16, products=products)
    lin.vvs_qlinear_load(w.cuda())
    r, x = _of_a_few(rows, width)
    y = torch.full((rows, out), 3.0, dtype=TYPES[dtype], device="cuda")
    lin.vvs_qlinear_apply(r, y)
    check_product(y[:61], x, qc.held(w.t())[0].t(), TYPES[dtype], fast=dtype == "bf16" and products == 0)
    assert torch.equal(y, y[:61][torch.arange(rows, device="cuda") % 61])
    with pytest.raises(vb.VvsError):
        vb.QLinear(width, out, rows + 1, vb.VVS_BF16)


def test_a_million_rows_with_a_gate():
    from paper_2511_13587_amd import binding as vb
    rows, width, out = 1 << 20, 140, 130
    ws = [(_normal((width, out), 1 + i) * width ** -0.5).bfloat16() for i in (0, 1)]
    lin = vb.QLinear(width, out, rows, vb.VVS_BF16, gated=True)
    lin.vvs_qlinear_load(*[w.cuda() for w in ws])
    r, x = _of_a_few(rows, width)
    y = vb.QRows(rows, out)
    lin.vvs_qlinear_gate(r, y)
    check_gate(y.first(61), x, [qc.held(w.t())[0].t() for w in ws], fast=True)
    at = torch.arange(rows, device="cuda") % 61
    assert torch.equal(y.values.view(torch.uint8), y.values.view(torch.uint8)[:61][at]) and torch.equal(y.powers, y.powers[:61][at])


@pytest.mark.parametrize("rows", [1, 14, 40, 70, 130])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_sixteen_million_columns(rows, dtype):
    """2 GB of weights in 8 bits; the first and last columns, and some around multiples of 2^20, beside their products."""
    from paper_2511_13587_amd import binding as vb
    width, out = 20, 1 << 24
    w = torch.empty((width, out), dtype=torch.bfloat16, device="cuda").normal_(0.0, 0.2, generator=torch.Generator("cuda").manual_seed(1))
    lin = vb.QLinear(width, out, rows, vb.VVS_BF16)
    lin.vvs_qlinear_load(w)
    r = vb.QRows(rows, width)
    x = qc.put(r, _normal((rows, width), 2))
    y = torch.full((rows, out), 3.0, dtype=TYPES[dtype], device="cuda")
    lin.vvs_qlinear_apply(r, y)
    cols = torch.cat([torch.arange(max(0, m - 70), min(out, m + 70)) for m in range(0, out + 1, 1 << 20)]).cuda()
    check_product(y[:, cols], x, qc.held(w[:, cols].cpu().t())[0].t(), TYPES[dtype], fast=rows > 64 and dtype == "bf16")
    back = torch.empty_like(w)
    lin.vvs_qlinear_read(back)
    assert torch.equal(back[:, cols].cpu().double(), qc.held(w[:, cols].cpu().t())[0].t())


@pytest.mark.parametrize("rows,width,out,gated", [(9, 8400, 500, False), (30, 5200, 4000, False), (300, 5200, 4200, False), (1700, 300, 4100, False), (70, 4100, 16600, False), (300, 1300, 3500, True), (129, 1281, 13640, True)])
def test_a_map_whose_first_call_is_captured(rows, width, out, gated):
    """Load and product recorded before any call of the map has run; replayed several times beside eager calls of another map of the same weights."""
    from paper_2511_13587_amd import binding as vb
    ws = [(_normal((width, out), 5 + i) * width ** -0.5).bfloat16().cuda() for i in range(2 if gated else 1)]
    r = vb.QRows(rows, width)
    qc.put(r, _normal((rows, width), 6))
    maps = [vb.QLinear(width, out, rows, vb.VVS_BF16, gated=gated) for _ in (0, 1)]
    ys = [vb.QRows(rows, out) if gated else torch.empty((rows, out), dtype=torch.bfloat16, device="cuda") for _ in (0, 1)]

    def call(i):
        maps[i].vvs_qlinear_load(*ws)
        maps[i].vvs_qlinear_gate(r, ys[i]) if gated else maps[i].vvs_qlinear_apply(r, ys[i])

    def bits(y):
        return torch.cat([y.values.view(torch.uint8).flatten(), y.powers.flatten()]) if gated else y

    torch.cuda.synchronize()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        with torch.cuda.graph(graph, stream=stream):
            call(0)
    torch.cuda.synchronize()
    for _ in range(4):
        for w in ws:
            w.neg_()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            graph.replay()
        stream.synchronize()
        call(1)
        torch.cuda.synchronize()
        assert torch.equal(bits(ys[0]), bits(ys[1]))
