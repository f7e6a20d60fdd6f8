"""Products of rows and weights in 8 bits against plain statements in 64 bits."""
import pytest
import torch

import qlinear_common as qc

pytestmark = pytest.mark.gpu
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def _vvs(vb, dtype):
    return vb.VVS_FP32 if dtype == torch.float32 else vb.VVS_BF16


def _normal(dims, seed, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(dims, generator=g) * torch.exp2(torch.randn(dims[-1:], generator=g) * spread)


def _linear(vb, rows, width, out, dtype=torch.bfloat16, gated=False, seed=0):
    """(linear, rows, held x, held weights in float64)"""
    ws = [(_normal((width, out), seed + 1 + i) * width ** -0.5).to(dtype) for i in range(2 if gated else 1)]
    lin = vb.QLinear(width, out, rows, _vvs(vb, dtype), gated=gated)
    lin.vvs_qlinear_load(*[w.cuda() for w in ws])
    r = vb.QRows(rows, width)
    x = qc.put(r, _normal((rows, width), seed))
    return lin, r, x, [qc.held(w.t())[0].t() for w in ws]


def product_error(x, w, fast=False):
    """How far x @ w may be off (float64 x, w as held).  e4m3 numbers are exact in bf16, as are their products in fp32; 32 products go into an fp32 sum by a matrix instruction of at most 8 roundings in a row, partial
    sums of eight waves are added: K / 4 + 16 roundings of at most the sum of magnitudes.
    fast: matrix instructions on the e4m3 numbers themselves add up to 8 neighbouring products aligned to the largest, each cut off 2^13 below it: 7 * 2^-13 of their magnitudes."""
    return ((x.shape[1] / 4 + 16) * 2.0 ** -24 + (7 * 2.0 ** -13 if fast else 0)) * (x.abs() @ w.abs())


def check_product(y, x, w, dtype, fast=False):
    want = x @ w
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    err = product_error(x, w, fast)
    bound = err + half * (want.abs() + err)
    off = y.double().cpu() - want
    worst = (off.abs() - bound).max().item()
    assert worst <= 0, worst
    if off.numel() >= 1000:      # many roundings, even over a step: half / 3^0.5 in the 2-norm at most; what e4m3 products lose is cut off evenly as well, hundreds of groups of them: below 2^-13 of the whole
        assert off.norm() <= want.norm() * (half * 0.6 + (2.0 ** -13 if fast else (x.shape[1] / 32 + 16) * 2.0 ** -24))


def check_gate(out, x, w, fast=False):
    g, u = x @ w[0], x @ w[1]
    a = g * torch.sigmoid(g)
    eg, eu = product_error(x, w[0], fast), product_error(x, w[1], fast)
    # |d silu| <= 1.1; exponential, sum, division, product: 8 roundings at most
    err = 1.1 * eg * (u.abs() + eu) + (a.abs() + 1.1 * eg) * eu + 8 * 2.0 ** -24 * (a * u).abs()
    qc.check_rounded(out, a * u, err)
    # beside the rounded definition: an element known to eps of itself is sent over a border, to the next step, with probability 2 eps / 2^-4 at most.  eps is below 2^-13 for elements of a usual
    # size (0.4 %) and grows for those that are small beside their terms: 8 % are below a tenth of the usual size, 1 % below a hundredth
    want = qc.held(a * u)[0]
    assert (qc.values_of(out) != want).sum().item() <= 0.03 * want.numel() + 1


@pytest.mark.parametrize("width,out", [(1, 1), (128, 64), (129, 65), (344, 128), (1000, 77), (1280, 3840), (515, 300)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("gated", [False, True])
def test_weights_are_held_by_column(width, out, dtype, gated):
    from paper_2511_13587_amd import binding as vb
    ws = [_normal((width, out), 5 + i, 3.0).to(TYPES[dtype]) for i in range(2 if gated else 1)]
    lin = vb.QLinear(width, out, 1, _vvs(vb, TYPES[dtype]), gated=gated)
    lin.vvs_qlinear_load(*[w.cuda() for w in ws])
    got = [torch.full((width, out), 9.0, dtype=TYPES[dtype], device="cuda") for _ in ws]
    lin.vvs_qlinear_read(*got)
    for w, y in zip(ws, got):
        assert torch.equal(y.cpu().double(), qc.held(w.t())[0].t())


@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 31, 33, 64, 65, 100, 129, 257])
@pytest.mark.parametrize("width,out", [(344, 128), (1000, 77), (128, 1), (1, 300)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_product_at_odd_sizes(rows, width, out, dtype):
    from paper_2511_13587_amd import binding as vb
    lin, r, x, (w,) = _linear(vb, rows, width, out, seed=rows)
    y = torch.full((rows, out), 3.0, dtype=TYPES[dtype], device="cuda")
    lin.vvs_qlinear_apply(r, y)
    check_product(y, x, w, TYPES[dtype], fast=rows > 64 and dtype == "bf16")


# every kernel and tile of the product (which calls take which stands at plan_qlinear_product): one and two columns tiles for 16 rows, one, two and four for 32, a contraction in halves, tiles of 32 x 128,
# 64 x 128, 64 x 256, 128 x 256; odd sizes, numbers of blocks that are no multiple of 4, more than the 64 whose powers a tile holds at once
@pytest.mark.parametrize("rows,width,out", [(8, 4096, 512), (16, 1000, 4300), (28, 640, 300), (28, 11008, 256), (31, 8300, 100), (48, 768, 2048), (64, 129, 130), (200, 640, 640), (129, 9000, 500), (432, 1280, 1280),
                                            (65, 8500, 4200), (432, 1280, 3840), (257, 8449, 2700), (1000, 640, 3840), (1001, 8400, 3900), (4100, 300, 4100), (4099, 8321, 4097)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_product(rows, width, out, dtype):
    from paper_2511_13587_amd import binding as vb
    lin, r, x, (w,) = _linear(vb, rows, width, out, seed=rows)
    y = torch.full((rows, out), 3.0, dtype=TYPES[dtype], device="cuda")
    lin.vvs_qlinear_apply(r, y)
    check_product(y, x, w, TYPES[dtype], fast=rows > 64 and dtype == "bf16")


@pytest.mark.parametrize("rows", [1, 14, 16, 17, 33, 65, 130, 300])
@pytest.mark.parametrize("width,out", [(128, 32), (344, 129), (1000, 77), (100, 1)])
def test_gate_at_odd_sizes(rows, width, out):
    from paper_2511_13587_amd import binding as vb
    lin, r, x, w = _linear(vb, rows, width, out, gated=True, seed=rows)
    y = vb.QRows(rows, out)
    lin.vvs_qlinear_gate(r, y)
    check_gate(y, x, w, fast=rows > 64)


# further rows, columns and lengths at which another kernel takes over: tiles of 16 x 16 and 16 x 32 for more than one row tile, 32 x 32 whole and in two and three parts, 32 x 64, tiles for few rows of many columns
@pytest.mark.parametrize("rows,width,out", [(17, 500, 300), (64, 700, 400), (60, 2100, 2050), (100, 1000, 1290), (28, 5200, 2100), (17, 5121, 4096), (28, 10300, 5000), (5, 10241, 4801), (100, 4200, 2000), (60, 4100, 4090), (30, 4096, 9000), (100, 2200, 4100),
                                            (200, 5200, 4100), (33, 300, 33000), (64, 1030, 40001), (300, 400, 16390), (600, 390, 16400)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_product_where_another_kernel_takes_over(rows, width, out, dtype):
    from paper_2511_13587_amd import binding as vb
    lin, r, x, (w,) = _linear(vb, rows, width, out, seed=rows)
    y = torch.full((rows, out), 3.0, dtype=TYPES[dtype], device="cuda")
    lin.vvs_qlinear_apply(r, y)
    check_product(y, x, w, TYPES[dtype], fast=rows > 64 and dtype == "bf16")


# tiles whose workgroups cut the contraction into shares: two and four, shares that begin inside a word of four powers, with one block more than another, with more blocks than their powers lie in LDS at a time
@pytest.mark.parametrize("rows,width,out", [(200, 5200, 4100), (130, 3201, 3000), (432, 2100, 2048), (300, 5200, 4200), (432, 2100, 4200), (200, 1100, 4200), (432, 4200, 8200), (40, 3200, 16390), (61, 3330, 16300), (64, 900, 16300),
                                            (300, 17000, 2100), (600, 8500, 5000), (1000, 1030, 2300), (900, 1153, 1290)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_product_in_shares(rows, width, out, dtype):
    from paper_2511_13587_amd import binding as vb
    lin, r, x, (w,) = _linear(vb, rows, width, out, seed=rows)
    y = torch.full((rows, out), 3.0, dtype=TYPES[dtype], device="cuda")
    lin.vvs_qlinear_apply(r, y)
    check_product(y, x, w, TYPES[dtype], fast=rows > 64 and dtype == "bf16")


@pytest.mark.parametrize("rows,width,out", [(17, 900, 900), (48, 1100, 1030), (33, 640, 2100), (60, 2100, 5600), (100, 2100, 2050), (130, 2049, 1000), (40, 200, 100), (300, 256, 300), (280, 2100, 600), (440, 400, 11000)])
def test_gate_where_another_kernel_takes_over(rows, width, out):
    from paper_2511_13587_amd import binding as vb
    lin, r, x, w = _linear(vb, rows, width, out, gated=True, seed=rows)
    y = vb.QRows(rows, out)
    lin.vvs_qlinear_gate(r, y)
    check_gate(y, x, w, fast=rows > 64)


@pytest.mark.parametrize("rows,width,out", [(14, 4096, 1024), (16, 8300, 150), (28, 1280, 3456), (32, 8449, 129), (48, 768, 2048), (64, 8400, 1000), (432, 1280, 3456), (300, 9000, 500), (700, 512, 1100),
                                            (4100, 640, 1500), (4099, 8321, 1600)])
def test_gate(rows, width, out):
    from paper_2511_13587_amd import binding as vb
    lin, r, x, w = _linear(vb, rows, width, out, gated=True, seed=rows)
    y = vb.QRows(rows, out)
    lin.vvs_qlinear_gate(r, y)
    check_gate(y, x, w, fast=rows > 64)
