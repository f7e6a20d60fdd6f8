"""What a gated product leaves behind the width of its rows: 0, whatever goes in."""
import pytest
import torch

import qlinear_common as qc
from test_gpu_qlinear import _normal, check_gate

pytestmark = pytest.mark.gpu


# few rows by one and two tiles of 16, tiles of 32, 64 and 128 rows; whole and e4m3 products
@pytest.mark.parametrize("rows,width,out,products", [(5, 300, 200, 0), (30, 2100, 3000, 0), (40, 300, 200, 0), (60, 2100, 5601, 0), (100, 300, 200, 0), (500, 300, 200, 0), (500, 300, 200, 1), (129, 700, 13640 - 7, 0),
                                                     (129, 700, 13640 - 7, 1), (70, 300, 1, 0), (17, 128, 129, 0)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_rows_that_are_not_finite_are_zero_behind_their_width(rows, width, out, products, bad):
    """One element of two rows is not finite, the first and the last: their hidden units are NaN, what lies behind them is 0, and the other rows are as they would be."""
    from paper_2511_13587_amd import binding as vb
    ws = [_normal((width, out), i) * width ** -0.5 for i in (1, 2)]
    lin = vb.QLinear(width, out, rows, vb.VVS_FP32, gated=True, products=products)
    lin.vvs_qlinear_load(*[w.cuda() for w in ws])
    x = _normal((rows, width), 3, 0.3)
    x[0, 7], x[rows - 1, width - 1] = bad, bad
    r, y = vb.QRows(rows, width), vb.QRows(rows, out)
    vb.vvs_qrows_round(x.cuda(), r)
    y.values.view(torch.uint8).fill_(0x55)
    y.powers.fill_(200)
    lin.vvs_qlinear_gate(r, y)
    qc.check_layout(y)
    nan = torch.isnan(qc.values_of(y))
    assert nan[[0, rows - 1]].all()
    if rows > 2:
        assert not nan[1:rows - 1].any()
        # the rows between, beside their definition
        between = vb.QRows(rows - 2, out)
        between.values.copy_(y.values[1:rows - 1])
        between.powers.copy_(y.powers[1:rows - 1])
        check_gate(between, qc.values_of(r)[1:rows - 1], [qc.held(w.t())[0].t().contiguous() for w in ws], fast=rows > 64 and products == 0)


@pytest.mark.parametrize("rows", [5, 40, 500])
def test_the_next_product_takes_such_rows(rows):
    """gate, then a product with as many rows as came out: only the row that was not finite is NaN."""
    from paper_2511_13587_amd import binding as vb
    width, hidden, out = 300, 200, 96
    gate = vb.QLinear(width, hidden, rows, vb.VVS_FP32, gated=True)
    gate.vvs_qlinear_load(*[(_normal((width, hidden), i) * width ** -0.5).cuda() for i in (1, 2)])
    down = vb.QLinear(hidden, out, rows, vb.VVS_FP32)
    down.vvs_qlinear_load((_normal((hidden, out), 4) * hidden ** -0.5).cuda())
    x = _normal((rows, width), 3, 0.3)
    x[2, 7] = float("nan")
    r, h, y = vb.QRows(rows, width), vb.QRows(rows, hidden), torch.zeros((rows, out), device="cuda")
    vb.vvs_qrows_round(x.cuda(), r)
    gate.vvs_qlinear_gate(r, h)
    down.vvs_qlinear_apply(h, y)
    want = torch.zeros((rows, out), dtype=torch.bool)
    want[2] = True
    assert torch.equal(torch.isnan(y).cpu(), want)
