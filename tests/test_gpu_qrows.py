"""Rows in 8 bits: rounding, norm with the residual's addition, reading back, against plain statements in 64 bits."""
import pytest
import torch

import qlinear_common as qc

pytestmark = pytest.mark.gpu
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def _inputs(rows, width, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, width), generator=g) * torch.exp2(torch.randn((width,), generator=g) * 2)
    return x.to(dtype)


@pytest.mark.parametrize("rows,width", [(1, 1), (3, 7), (2, 8), (5, 127), (4, 128), (7, 129), (10, 344), (3, 513), (33, 1000), (2, 4096), (1, 65536)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_rounding_and_reading(rows, width, dtype):
    from paper_2511_13587_amd import binding as vb
    x = _inputs(rows, width, TYPES[dtype], rows * 1000 + width)
    r = vb.QRows(rows, width)
    vb.vvs_qrows_round(x.cuda(), r)
    want, e = qc.held(x)
    qc.check_layout(r)
    assert torch.equal(r.powers.cpu()[:, :e.shape[1]].long() - 127, e)
    assert torch.equal(qc.values_of(r), want)
    for t in TYPES.values():
        out = torch.full((rows, width), 7.0, dtype=t, device="cuda")
        vb.vvs_qrows_read(r, out)
        assert torch.equal(out.cpu().double(), want)


def test_rounding_of_special_values():
    """Borders of the power of two, ties, zeros, the smallest and largest numbers, what is not finite: beside finite elements it does not touch their power."""
    from paper_2511_13587_amd import binding as vb
    x = torch.zeros((12, 256))
    x[0, :3] = torch.tensor([448.0, 1.0, -0.5])                        # E = 0 exactly
    x[1, :2] = torch.tensor([448.0000305, 1.0])                        # one step above: E = 1
    x[2, :6] = torch.tensor([256.0, 17.0, 19.0, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10])   # ties to even; subnormal numbers
    x[3, 5], x[3, 6], x[3, 7], x[3, 8] = float("inf"), float("-inf"), float("nan"), 3.0
    x[4, 0], x[4, 200] = 3.4028234663852886e38, -3.4e38
    x[5, 0], x[5, 1] = 1e-45, 1e-38                                    # below what E >= -110 reaches, and near it
    x[6, 127], x[6, 128] = 1000.0, 1e-3                                # neighbours of two blocks
    x[7] = float("nan")
    x[8] = -0.0
    x[9] = torch.arange(256) * 1.75
    x[10] = 2.0 ** torch.arange(-128, 128).float()
    x[11] = -447.9999
    r = vb.QRows(12, 256)
    vb.vvs_qrows_round(x.cuda(), r)
    want, e = qc.held(x)
    assert torch.equal(r.powers.cpu()[:, :2].long() - 127, e)
    got = qc.values_of(r)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got, 0.0), torch.nan_to_num(want, 0.0))
    out = torch.zeros((12, 256), device="cuda")
    vb.vvs_qrows_read(r, out)
    # as a float32: the largest float32 is held as 2^128, which is an infinity there
    assert got[4, 0] == 2.0 ** 128 and out[4, 0] == float("inf")
    assert torch.equal(torch.nan_to_num(out.cpu(), 0.0), torch.nan_to_num(want.float(), 0.0)) and torch.equal(torch.isnan(out.cpu()), torch.isnan(want))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("width,lead,stride", [(128, 0, 384), (200, 1, 513), (64, 8, 640), (255, 3, 256), (40, 5, 41)])
def test_strides_and_unaligned_rows(dtype, width, lead, stride):
    """Parts of wider tensors, pointers off 16 bytes, odd strides; what lies beside the part and behind the last row stays as it was."""
    from paper_2511_13587_amd import binding as vb
    rows = 9
    flat = _inputs(1, rows * stride + lead + 8, TYPES[dtype], width).cuda().view(-1)
    x = flat[lead:].as_strided((rows, width), (stride, 1))
    big = vb.QRows(rows + 2, width)
    big.values.view(torch.uint8).fill_(0x55)
    big.powers.fill_(99)
    r = big.first(rows)
    vb.vvs_qrows_round(x, r)
    want, e = qc.held(x.cpu())
    assert torch.equal(qc.values_of(r), want)
    assert (big.values.view(torch.uint8)[rows:] == 0x55).all() and (big.powers[rows:] == 99).all()
    around = torch.full((rows * stride + lead + 8,), 3.0, dtype=TYPES[dtype], device="cuda")
    out = around[lead:].as_strided((rows, width), (stride, 1))
    vb.vvs_qrows_read(r, out)
    assert torch.equal(out.cpu().double(), want)
    mine = torch.zeros(around.shape, dtype=torch.bool, device="cuda")
    mine[lead:].as_strided((rows, width), (stride, 1)).fill_(True)
    assert (around[~mine] == 3.0).all()


def _norm_check(vb, x, delta, gain, eps, in_place=False, x_out=True):
    rows, width = x.shape
    r = vb.QRows(rows, width)
    xd = x.cuda()
    dd = None if delta is None else delta.cuda()
    out = xd if in_place else torch.full_like(xd, 5.0) if x_out else None
    vb.vvs_qrows_norm(xd, gain.cuda(), eps, r, delta=dd, x_out=out)
    kept = x if delta is None else (x.float() + delta.float()).to(x.dtype)
    if out is not None:
        assert torch.equal(out.cpu(), kept)
    if not in_place:
        assert torch.equal(xd.cpu(), x)
    k = kept.double()
    y = k / torch.sqrt((k * k).mean(dim=1, keepdim=True) + eps) * gain.double()
    # the sum of squares in fp32: fewer than 100 roundings on the way of any term, half of which the square root leaves; then root, division, two products
    qc.check_rounded(r, y, y.abs() * 64 * 2.0 ** -24)


@pytest.mark.parametrize("rows,width", [(1, 1), (2, 8), (10, 128), (3, 129), (5, 512), (4, 513), (7, 1280), (3, 2048), (2, 2049), (33, 4096), (2, 5000), (3, 11008), (1, 20000), (1, 65536)])
@pytest.mark.parametrize("residual,delta", [("fp32", "bf16"), ("bf16", "bf16"), ("fp32", None), ("bf16", "fp32")])
def test_norm(rows, width, residual, delta):
    from paper_2511_13587_amd import binding as vb
    x = _inputs(rows, width, TYPES[residual], width + rows)
    d = None if delta is None else _inputs(rows, width, TYPES[delta], width + rows + 1)
    gain = (1 + 0.3 * torch.randn(width, generator=torch.Generator().manual_seed(1))).to(TYPES[residual if delta else "bf16"])
    _norm_check(vb, x, d, gain, 1e-5)


def test_norm_in_place_without_output_and_of_zeros():
    from paper_2511_13587_amd import binding as vb
    x, d, gain = _inputs(6, 700, torch.float32, 1), _inputs(6, 700, torch.float32, 2), torch.ones(700)
    _norm_check(vb, x, d, gain, 1e-6, in_place=True)
    _norm_check(vb, x, d, gain, 1e-6, x_out=False)
    _norm_check(vb, x.bfloat16(), d, gain, 0.0, in_place=True)
    _norm_check(vb, torch.zeros_like(x), None, gain, 1e-6)
    _norm_check(vb, x * 1e-20, None, gain, 1e-5)
    _norm_check(vb, x * 1e15, None, gain, 1e-5)


def test_norm_of_a_nan_stays_in_its_row():
    from paper_2511_13587_amd import binding as vb
    x, gain = _inputs(4, 300, torch.float32, 3), torch.ones(300)
    x[2, 17] = float("nan")
    r = vb.QRows(4, 300)
    vb.vvs_qrows_norm(x.cuda(), gain.cuda(), 1e-5, r)
    got = qc.values_of(r)
    assert torch.isnan(got[2]).all() and torch.isfinite(got[[0, 1, 3]]).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_norm_of_strided_rows(dtype):
    from paper_2511_13587_amd import binding as vb
    rows, width = 5, 301
    base = _inputs(rows, 1024, TYPES[dtype], 11).cuda()
    x, d, out = base[:, 1:1 + width], base[:, 400:400 + width], torch.zeros((rows, 777), dtype=TYPES[dtype], device="cuda")[:, 3:3 + width]
    gain = torch.rand(width + 1)[1:]
    r = vb.QRows(rows, width)
    vb.vvs_qrows_norm(x, gain.cuda(), 1e-5, r, delta=d, x_out=out)
    kept = (x.float() + d.float()).to(TYPES[dtype]).cpu()
    assert torch.equal(out.cpu(), kept)
    k = kept.double()
    qc.check_rounded(r, k / torch.sqrt((k * k).mean(dim=1, keepdim=True) + 1e-5) * gain.double(), 64 * 2.0 ** -24 * (k.abs() + 1))
