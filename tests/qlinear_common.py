"""Plain statements in 64 bits of what rows and weights in 8 bits hold and of the operators on them."""
import torch

BLOCK, LEAST, TOP = 128, -110, 448.0


def blocks_of(width):
    return -(-width // BLOCK)


def power_of(x):
    """E of every block: x float64 [rows, width] -> int64 [rows, blocks]."""
    rows, width = x.shape
    x = torch.nn.functional.pad(x, (0, -width % BLOCK)).view(rows, -1, BLOCK)
    top = torch.where(torch.isfinite(x), x.abs(), 0.0).amax(dim=2)
    e = torch.full(top.shape, LEAST, dtype=torch.int64)
    while True:
        more = top > TOP * torch.exp2(e.double())
        if not more.any():
            return e
        e = torch.where(more, e + 1, e)


def nearest_e4m3(x):
    """Nearest e4m3 number, ties to even, of float64 values of at most 448; what is not finite becomes NaN."""
    a = x.abs()
    _, e = torch.frexp(torch.where((a > 0) & torch.isfinite(a), a, 1.0))      # a = m 2^e, m in [0.5, 1)
    step = torch.exp2(torch.clamp(e.double() - 1, min=-6.0) - 3.0)
    return torch.where(torch.isfinite(x), torch.round(x / step) * step, torch.nan)


def held(x, e=None):
    """Values that rows in 8 bits stand for, and E: x [rows, width] of any float type."""
    x = x.double()
    rows, width = x.shape
    e = power_of(x) if e is None else e
    unit = torch.exp2(e.double()).repeat_interleave(BLOCK, dim=1)[:, :width]
    return nearest_e4m3(x / unit) * unit, e


def values_of(rows):
    """float64 values that a binding.QRows stands for."""
    e = rows.powers.cpu()[:, :blocks_of(rows.width)].to(torch.int64) - 127
    return rows.values.cpu().double()[:, :rows.width] * torch.exp2(e.double()).repeat_interleave(BLOCK, dim=1)[:, :rows.width]


def put(rows, x):
    """Fills a binding.QRows with the held values of x, without the library; returns them in float64."""
    y, e = held(x)
    n, width = x.shape
    unit = torch.exp2(e.double()).repeat_interleave(BLOCK, dim=1)[:, :width]
    padded = torch.zeros(rows.values.shape, dtype=torch.float32)
    padded[:, :width] = (y / unit).float()
    rows.values.copy_(padded.to(torch.float8_e4m3fn))
    powers = torch.zeros(rows.powers.shape, dtype=torch.uint8)
    powers[:, :blocks_of(width)] = (e + 127).to(torch.uint8)
    rows.powers.copy_(powers)
    return y


def check_layout(rows):
    """What lies behind the width and behind the last block is 0."""
    assert (rows.values.cpu().view(torch.uint8)[:, rows.width:] & 0x7F == 0).all()
    assert (rows.powers.cpu()[:, blocks_of(rows.width):] == 0).all()


def check_rounded(rows, y, err):
    """rows hold y (float64), which was known to `err` (absolute, of the same shape) when it was rounded: the power of two is that of a largest element within its error, an element is off by half a
    step at most - 2^-4 of itself, or of the smallest normal number 2^(E - 6) - and its error."""
    check_layout(rows)
    e = rows.powers.cpu()[:, :blocks_of(rows.width)].to(torch.int64) - 127
    low, high = power_of((y.abs() - err).clamp(min=0)), power_of(y.abs() + err)
    assert ((e >= low) & (e <= high)).all()
    unit = torch.exp2(e.double()).repeat_interleave(BLOCK, dim=1)[:, :rows.width]
    off = (values_of(rows) - y).abs()
    bound = torch.maximum((y.abs() + err) * 2.0 ** -4, unit * 2.0 ** -10) + err
    worst = (off - bound).max().item()
    assert worst <= 0, worst
