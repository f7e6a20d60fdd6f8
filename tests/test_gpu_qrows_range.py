"""The norm into 8 bits of rows whose squares fp32 does not hold, against its statement in 64 bits."""
import pytest
import torch

import qlinear_common as qc

pytestmark = pytest.mark.gpu
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def _rows(rows, width, scale, seed):
    x = torch.randn((rows, width), generator=torch.Generator().manual_seed(seed), dtype=torch.float64)
    return (x.clamp(-3, 3) * scale).float()


def _check(vb, x, delta, gain, eps):
    rows, width = x.shape
    r, out = vb.QRows(rows, width), torch.full_like(x, 5.0).cuda()
    vb.vvs_qrows_norm(x.cuda(), gain.cuda(), eps, r, delta=None if delta is None else delta.cuda(), x_out=out)
    kept = x if delta is None else (x.float() + delta.float()).to(x.dtype)
    assert torch.equal(out.cpu(), kept)
    k = kept.double()
    # (eps as the call takes it, in fp32)
    y = k / torch.sqrt((k * k).mean(dim=1, keepdim=True) + torch.tensor(eps, dtype=torch.float32).double()) * gain.double()
    # as for rows of usual size: fewer than 100 roundings on the way of a square, half of which the root leaves; root, two products
    qc.check_rounded(r, y, y.abs() * 64 * 2.0 ** -24)


# a wave, several, 2 to 8 times 8 elements per thread
@pytest.mark.parametrize("rows,width", [(3, 8), (5, 300), (4, 513), (2, 5000), (2, 11008), (2, 20000), (1, 65536)])
@pytest.mark.parametrize("scale", [1e-10, 1e-13, 1e-18, 1e-20, 1e-23, 1e-25, 1e-30, 1e-37, 1e-41, 1e17, 1e19, 1e25, 1e37])
@pytest.mark.parametrize("eps", [0.0, 1e-45, 1e-40, 1e-20])
def test_rows_of_any_size(rows, width, scale, eps):
    from paper_2511_13587_amd import binding as vb
    gain = 1 + 0.3 * torch.randn(width, generator=torch.Generator().manual_seed(1))
    _check(vb, _rows(rows, width, scale, width), None, gain, eps)


@pytest.mark.parametrize("residual,delta", [("fp32", "bf16"), ("bf16", "bf16"), ("bf16", "fp32")])
@pytest.mark.parametrize("scale", [1e-22, 1e-30, 1e20, 1e37])
def test_with_an_addition(residual, delta, scale):
    from paper_2511_13587_amd import binding as vb
    x, d = _rows(6, 700, scale, 1).to(TYPES[residual]), _rows(6, 700, scale, 2).to(TYPES[delta])
    _check(vb, x, d, torch.ones(700), 0.0)
    _check(vb, x, d, torch.ones(700).bfloat16(), 1e-5)


def test_rows_of_every_size_beside_each_other():
    """Each row by itself: tiny, usual and huge ones, one that holds both, one of zeros but for an element."""
    from paper_2511_13587_amd import binding as vb
    x = torch.cat([_rows(1, 1000, s, i) for i, s in enumerate((1e-44, 1e-30, 1.0, 1e-12, 1e30, 1e-22, 1e38))])
    x[3, ::7] = 1e25
    x = torch.cat([x, torch.zeros((2, 1000))])
    x[7, 900], x[8, 5] = 1e-45, -3e38
    _check(vb, x, None, torch.ones(1000), 0.0)


def test_what_is_not_finite_stays_what_it_was():
    """NaN: the whole row; an infinity: that element (infinity times 0), and 0 for the others, which are divided by an infinite mean."""
    from paper_2511_13587_amd import binding as vb
    for width in (40, 300, 5000):
        x = _rows(5, width, 1e-25, 3)
        x[1, 17], x[2, 8], x[3, width - 1] = float("nan"), float("inf"), float("-inf")
        r = vb.QRows(5, width)
        vb.vvs_qrows_norm(x.cuda(), torch.ones(width).cuda(), 0.0, r)
        got = qc.values_of(r)
        assert torch.isnan(got[1]).all() and torch.isfinite(got[[0, 4]]).all() and (got[[0, 4]] != 0).any(dim=1).all()
        for row, at in ((2, 8), (3, width - 1)):
            want = torch.zeros(width, dtype=torch.bool)
            want[at] = True
            assert torch.equal(torch.isnan(got[row]), want) and (got[row][~want] == 0).all()
        qc.check_layout(r)


def test_rows_of_zeros():
    """eps 0: NaN, as the header says; any other: zeros."""
    from paper_2511_13587_amd import binding as vb
    r = vb.QRows(3, 300)
    for eps in (0.0, 1e-45, 1e-30, 1e-5):
        vb.vvs_qrows_norm(torch.zeros((3, 300), device="cuda"), torch.ones(300, device="cuda"), eps, r)
        got = qc.values_of(r)
        assert torch.isnan(got).all() if eps == 0 else (got == 0).all()
