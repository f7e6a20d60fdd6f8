"""How products of rows and weights in 8 bits are summed: whole, or by the matrix instructions for e4m3, in every tile that makes them, against plain statements in 64 bits."""
import pytest
import torch

import qlinear_common as qc
from qlinear_variants import VARIANTS
from test_gpu_qlinear import TYPES, _normal, check_gate, product_error

pytestmark = pytest.mark.gpu


def _within(y, want, err, half):
    off, bound = (y.double() - want).abs(), err + half * (want.abs() + err)
    worst = (off - bound).max().item()
    assert worst <= 0, worst


@pytest.mark.parametrize("rows,width,out,gated,products,dtype,fast,tile,shares", VARIANTS)
def test_every_tile(rows, width, out, gated, products, dtype, fast, tile, shares):
    from paper_2511_13587_amd import binding as vb
    ws = [(_normal((width, out), 7 + i) * width ** -0.5).bfloat16() for i in range(2 if gated else 1)]
    lin = vb.QLinear(width, out, rows, vb.VVS_BF16, gated=bool(gated), products=products)
    lin.vvs_qlinear_load(*[w.cuda() for w in ws])
    r = vb.QRows(rows, width)
    x = qc.put(r, _normal((rows, width), rows))
    if gated:
        y = vb.QRows(rows, out)
        lin.vvs_qlinear_gate(r, y)
        check_gate(y, x, [qc.held(w.t())[0].t().contiguous() for w in ws], fast=bool(fast))
        return
    y = torch.full((rows, out), 3.0, dtype=TYPES[dtype], device="cuda")
    lin.vvs_qlinear_apply(r, y)
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    w = qc.held(ws[0].t())[0].t().contiguous()
    want = x @ w
    _within(y.cpu(), want, product_error(x, w, bool(fast)), half)


@pytest.mark.parametrize("rows", [5, 65, 129, 433, 1001])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("out", [300, 14250])
def test_whole_products_keep_small_elements_beside_large_ones(rows, dtype, out):
    """Two large products that cancel and a small one beside them, 2^-18 of theirs: in fp32 (24 bits) all of it is exact, in every tile.  The matrix instructions for e4m3 lose the small one."""
    from paper_2511_13587_amd import binding as vb
    width = 700
    x, w = torch.zeros((rows, width)), torch.zeros((width, out))
    x[:, 0], x[:, 1], x[:, 2] = 1.0, -1.0, 1.0
    w[0], w[1] = 448.0, 448.0
    w[2] = 2.0 ** -9 * (1 + torch.arange(out) % 7).float()                     # subnormal numbers of a block whose largest is 448
    lin = vb.QLinear(width, out, rows, vb.VVS_FP32, products=vb.VVS_PRODUCTS_WHOLE)
    lin.vvs_qlinear_load(w.cuda())
    r = vb.QRows(rows, width)
    qc.put(r, x)
    y = torch.zeros((rows, out), dtype=TYPES[dtype], device="cuda")
    lin.vvs_qlinear_apply(r, y)
    assert torch.equal(y.float().cpu(), w[2].expand(rows, out))


@pytest.mark.parametrize("rows", [5, 65, 129, 433])
@pytest.mark.parametrize("out", [200, 14250])
def test_whole_products_of_a_gate_keep_small_elements_beside_large_ones(rows, out):
    """The same in front of a gate.  Up products of 2^-9 (1 .. 7), gate products of 256: silu(256) = 256 in fp32, so that every hidden unit is a number of three bits, and a block holds it exactly."""
    from paper_2511_13587_amd import binding as vb
    width = 700
    x, gate, up = torch.zeros((rows, width)), torch.zeros((width, out)), torch.zeros((width, out))
    x[:, 0], x[:, 1], x[:, 2], x[:, 3] = 1.0, -1.0, 1.0, 1.0
    gate[0] = gate[1] = up[0] = up[1] = 448.0
    gate[3] = 256.0
    up[2] = 2.0 ** -9 * (1 + torch.arange(out) % 7).float()
    lin = vb.QLinear(width, out, rows, vb.VVS_FP32, gated=True, products=vb.VVS_PRODUCTS_WHOLE)
    lin.vvs_qlinear_load(gate.cuda(), up.cuda())
    r, y = vb.QRows(rows, width), vb.QRows(rows, out)
    qc.put(r, x)
    lin.vvs_qlinear_gate(r, y)
    qc.check_layout(y)
    assert torch.equal(qc.values_of(y), (256.0 * up[2].double()).expand(rows, out))


@pytest.mark.parametrize("rows", [65, 129, 433])
@pytest.mark.parametrize("products", [1, 2])
def test_sums_that_cancel(rows, products):
    """A channel a thousand times its neighbours and rows whose large halves cancel: the error goes by the magnitudes that are summed, which is what the header says of either choice."""
    from paper_2511_13587_amd import binding as vb
    width, out = 1280, 640
    x = _normal((rows, width), 1, 0.3)
    x[:, 3] *= 1000
    x[:, 640:] = -x[:, :640]
    w = _normal((width, out), 2, 0.3) * width ** -0.5
    w[640:] = w[:640] * (1 + 0.03 * _normal((640, out), 3, 0))
    lin = vb.QLinear(width, out, rows, vb.VVS_FP32, products=products)
    lin.vvs_qlinear_load(w.cuda())
    r = vb.QRows(rows, width)
    xh = qc.put(r, x)
    wh = qc.held(w.t())[0].t().contiguous()
    for dtype, half in ((torch.float32, 2.0 ** -24), (torch.bfloat16, 2.0 ** -8)):
        y = torch.zeros((rows, out), dtype=dtype, device="cuda")
        lin.vvs_qlinear_apply(r, y)
        _within(y.cpu(), xh @ wh, product_error(xh, wh, products == vb.VVS_PRODUCTS_E4M3), half)
