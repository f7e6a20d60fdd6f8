"""The operators of a decoder layer in 8 bits, each beside its plain form: what it computes in elementary torch operations.

A program whose projections are held in 8 bits calls four operators per layer, around the attention:

  norm    vvs_qrows_norm: the residual takes the last product in, is normalised, and goes to the next product as rows in 8 bits.
  round   vvs_qrows_round: rows that come from elsewhere (the attention's output) are rounded to 8 bits.
  linear  vvs_qlinear_apply: rows in 8 bits times weights in 8 bits.
  gate    vvs_qlinear_gate: silu(rows times gate weights) * (rows times up weights), again rows in 8 bits: what the down product takes.
  read    vvs_qrows_read (inside norm, round and gate here): rows in 8 bits as the numbers they stand for.

What is held in 8 bits.  A row is cut into blocks of 128 elements.  A block has one power of two, 2^E, and its elements are e4m3 numbers
times 2^E; E is the smallest with max |x| <= 448 * 2^E, at least -110.  Weights [in, out] are held likewise, every column in blocks of 128
along `in`.  Rows lie as [rows, width rounded up to 128] e4m3 bytes, 0 behind the width, and [rows, blocks rounded up to 4] bytes E + 127, 0 behind the last block."""
import math
import random

import torch

own = False

BLOCK = 128
TOP = 448.0        # largest e4m3 number
LEAST = -110       # smallest E
EPS = 1e-5
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ------------------------------------------------------------------------------------------------ the cases
def _norm(name, rows, width, residual="fp32", delta="bf16"):
    return {"name": name, "path": "norm", "rows": rows, "width": width, "residual": residual, "delta": delta}


def _round(name, rows, width, part=False, dtype="bf16"):
    return {"name": name, "path": "round", "rows": rows, "width": width, "part": part, "dtype": dtype}


def _linear(name, rows, width, out, dtype="bf16"):
    return {"name": name, "path": "linear", "rows": rows, "width": width, "out": out, "dtype": dtype}


def _gate(name, rows, width, out):
    return {"name": name, "path": "gate", "rows": rows, "width": width, "out": out}


def listed():
    return [
        # the fp32 reference shape, one prompt as a conditional / unconditional pair, chain of 4: the smallest call there is
        _norm("norm_tiny_fp32_x2", 10, 128, delta="fp32"),
        # the benchmark's workload: 26-node tree, 8 prompts, the residual stream in fp32 as the contexts keep it
        _norm("norm_xl_tree26_x16", 432, 1280),
        # prompts of the 7B shape, a residual stream in bf16
        _norm("norm_7b_prompt", 8192, 4096, residual="bf16"),
        # the attention's output of the benchmark's step, in front of its projection
        _round("round_xl_tree26_x16", 432, 1280),
        # one of the three parts of a prompt's projection, rows of another length than the part, an odd number of them
        _round("round_7b_part", 8191, 4096, part=True),
        # the reference shape's hidden units, 2.7 blocks of them, back to its width: the smallest product there is
        _linear("linear_tiny_down_fp32_x2", 10, 344, 128, dtype="fp32"),
        # q, k and v of the benchmark's step in one product
        _linear("linear_xl_qkv_tree26_x16", 432, 1280, 3840),
        # the 7B shape with a chain of 6 for two prompts: reading the weights is everything
        _linear("linear_7b_down_chain6_x4", 28, 11008, 4096, dtype="fp32"),
        # q, k and v of prompts of the 7B shape
        _linear("linear_7b_qkv_prompt", 8192, 4096, 12288),
        # the small model as it is served: chain of 5 for four prompts
        _gate("gate_b_chain5_x8", 48, 768, 2048),
        # one image of the 7B shape for one user, a chain of 6: conditional and unconditional row
        _gate("gate_7b_chain6_x2", 14, 4096, 11008),
        # prompts of the 7B shape, an odd number of tokens in all
        _gate("gate_7b_prompt", 4093, 4096, 11008),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def _size(rng):
    """A width: one of the model shapes', or any number."""
    return rng.choice([128, 344, 768, 1280, 2048, 3456, 4096, 11008]) if rng.random() < 0.5 else _log_int(rng, 16, 12288)


def draw(rng):
    most = {}
    for c in listed():
        most[c["path"]] = max(most.get(c["path"], 0.0), _seconds(c))
    while True:
        path = rng.choices(["norm", "round", "linear", "gate"], [3, 2, 5, 4])[0]
        rows, width = _log_int(rng, 1, 8192), _size(rng)
        if path == "norm":
            c = _norm("", rows, width, rng.choice(["fp32", "fp32", "bf16"]), rng.choice(["bf16", "bf16", "fp32", "none"]))
        elif path == "round":
            c = _round("", rows, width, rng.random() < 0.5, rng.choice(["bf16", "bf16", "fp32"]))
        elif path == "linear":
            c = _linear("", rows, width, _size(rng), rng.choice(["bf16", "bf16", "fp32"]))
        else:
            c = _gate("", rows, width, _size(rng))
        if _seconds(c) <= most[path]:
            del c["name"]
            return c


# ------------------------------------------------------------------------------------------------ sizes
def _wide(dtype):
    return {"fp32": 4, "bf16": 2, "none": 0}[dtype]


def _blocks(width):
    return -(-width // BLOCK)


def work(case):
    path, rows, width = case["path"], case["rows"], case["width"]
    held = rows * (width + _blocks(width))                        # bytes of the rows in 8 bits
    if path == "norm":
        values = rows * width
        return {"bytes": values * (2 * _wide(case["residual"]) + _wide(case["delta"]) + 2) + 4 * width + held, "flops": 6 * values}
    if path == "round":
        return {"bytes": rows * width * (_wide(case["dtype"]) + 2) + held, "flops": 2 * rows * width}
    out = case["out"]
    if path == "linear":
        return {"bytes": held + out * (width + _blocks(width)) + _wide(case["dtype"]) * rows * out, "flops": 2 * rows * width * out}
    return {"bytes": held + 2 * out * (width + _blocks(width)) + rows * (out + _blocks(out) + 2 * out), "flops": 4 * rows * width * out + 6 * rows * out}


def _seconds(case):
    w = work(case)
    return max(w["bytes"] / 8e12, w["flops"] / 5e15)


# ------------------------------------------------------------------------------------------------ inputs
class _Maker:
    def __init__(self, seed):
        self.g = torch.Generator("cuda")
        self.g.manual_seed(int(seed))

    def normal(self, dims, dtype=torch.float32, std=1.0):
        return torch.empty(dims, dtype=dtype, device="cuda").normal_(0.0, std, generator=self.g)

    def spread(self, width, strength=0.6):
        """A factor per dimension: a few are several times as large as the others."""
        return torch.exp2(self.normal((width,)).mul_(strength))


def _exponent(top):
    """Smallest E with top <= 448 * 2^E, at least LEAST."""
    m, e = torch.frexp(top)
    return (e - 9 + (m > 0.875)).clamp_(min=LEAST).to(torch.int32)


def _as_held(x):
    """[rows, width] -> e4m3 numbers [rows, width up to 128] and bytes E + 127 [rows, blocks up to 4]: how rows in 8 bits lie."""
    rows, width = x.shape
    blocks = _blocks(width)
    x = torch.nn.functional.pad(x.float(), (0, blocks * BLOCK - width)).view(rows, blocks, BLOCK)
    e = _exponent(x.abs().amax(dim=2))
    x8 = torch.ldexp(x, -e[:, :, None]).to(torch.float8_e4m3fn).view(rows, blocks * BLOCK)
    return x8, torch.nn.functional.pad((e + 127).to(torch.uint8), (0, -blocks % 4))


def _held_values(x8, powers, width):
    """e4m3 numbers and bytes E + 127 -> fp32 values [rows, width]."""
    rows, padded = x8.shape
    e = powers[:, :padded // BLOCK].to(torch.int32) - 127
    return torch.ldexp(x8.float().view(rows, -1, BLOCK), e[:, :, None]).view(rows, padded)[:, :width]


def prepare(case, seed):
    mk, path, rows, width = _Maker(seed), case["path"], case["rows"], case["width"]
    st = {"case": dict(case)}
    if own:
        from paper_2511_13587_amd import binding as vb
    if path == "norm":
        residual = TYPES[case["residual"]]
        # a residual stream has dimensions that are many times as large as the others
        st["x"] = (mk.normal((rows, width)) * mk.spread(width, 1.0)).to(residual)
        st["delta"] = None if case["delta"] == "none" else mk.normal((rows, width), std=0.3).to(TYPES[case["delta"]])
        st["gain"] = 1.0 + mk.normal((width,), std=0.2)
        st["x_out"], st["y"] = torch.empty_like(st["x"]), torch.empty((rows, width), dtype=torch.bfloat16, device="cuda")
        if own:
            st["rows8"] = vb.QRows(rows, width)
        return st
    if path == "round":
        dtype = TYPES[case["dtype"]]
        wide = mk.normal((rows, 3, width), dtype) if case["part"] else mk.normal((rows, 1, width), dtype)
        st["x"] = wide.mul_(mk.spread(width).to(dtype))[:, wide.shape[1] // 2]
        st["y"] = torch.empty((rows, width), dtype=torch.bfloat16, device="cuda")
        if own:
            st["rows8"] = vb.QRows(rows, width)
        return st
    # rows as a norm leaves them, weights as trained ones are spread: columns of different size
    x = mk.normal((rows, width)) * mk.spread(width)
    out, gated = case["out"], path == "gate"
    weights = [mk.normal((width, out), torch.bfloat16, width ** -0.5).mul_(mk.spread(out, 0.4).to(torch.bfloat16)) for _ in range(2 if gated else 1)]
    x8, powers = _as_held(x)
    held = [_as_held(w.t()) for w in weights]                     # [out, width]: a column's blocks lie along its row here
    if own:
        st["rows8"] = vb.QRows(rows, width)
        st["rows8"].values.copy_(x8)
        st["rows8"].powers.copy_(powers)
        # what is loaded is rounded already: both sides have the same weights, also where ldexp of a tie is one rounding off a power of two
        st["linear"] = vb.QLinear(width, out, rows, vb.VVS_FP32, gated=gated)
        st["linear"].vvs_qlinear_load(*[_held_values(*w, width).t().contiguous() for w in held])
        if gated:
            st["out8"] = vb.QRows(rows, out)
    else:
        st["x8"], st["xe"] = x8, powers
        st["w"] = held
    st["y"] = torch.empty((rows, out), dtype=torch.bfloat16 if gated else TYPES[case["dtype"]], device="cuda")
    return st


# ------------------------------------------------------------------------------------------------ one pass
def run(st):
    return {"norm": _run_norm, "round": _run_round, "linear": _run_linear, "gate": _run_gate}[st["case"]["path"]](st)


def _rounded(x):
    """fp32 values [rows, width] -> the values that they are held as, in bf16 (which has them all)."""
    x8, powers = _as_held(x)
    return _held_values(x8, powers, x.shape[1]).to(torch.bfloat16)


def _run_norm(st):
    if own:
        from paper_2511_13587_amd import binding as vb
        vb.vvs_qrows_norm(st["x"], st["gain"], EPS, st["rows8"], delta=st["delta"], x_out=st["x_out"])
        vb.vvs_qrows_read(st["rows8"], st["y"])
        return {"x": st["x_out"], "y": st["y"]}
    x = st["x"].float()
    if st["delta"] is not None:
        x = x + st["delta"].float()
    kept = x.to(st["x"].dtype)                                    # what is normalised is what the residual stream keeps
    x = kept.float()
    y = x * torch.rsqrt((x * x).mean(dim=1, keepdim=True) + EPS) * st["gain"]
    return {"x": kept, "y": _rounded(y)}


def _run_round(st):
    if own:
        from paper_2511_13587_amd import binding as vb
        vb.vvs_qrows_round(st["x"], st["rows8"])
        vb.vvs_qrows_read(st["rows8"], st["y"])
        return {"y": st["y"]}
    return {"y": _rounded(st["x"].float())}


def _product(st, which):
    width = st["case"]["width"]
    return torch.matmul(_held_values(st["x8"], st["xe"], width), _held_values(*st["w"][which], width).t())


def _run_linear(st):
    if own:
        st["linear"].vvs_qlinear_apply(st["rows8"], st["y"])
        return {"y": st["y"]}
    return {"y": _product(st, 0).to(st["y"].dtype)}


def _run_gate(st):
    if own:
        from paper_2511_13587_amd import binding as vb
        st["linear"].vvs_qlinear_gate(st["rows8"], st["out8"])
        vb.vvs_qrows_read(st["out8"], st["y"])
        return {"y": st["y"]}
    g, u = _product(st, 0), _product(st, 1)
    return {"y": _rounded(g / (1.0 + torch.exp(-g)) * u)}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def _nearest(x):
    """float64 values [rows, width] -> what rows in 8 bits hold of them: per block the least power of two, then steps of 2^-9 of it below 2^-6 and of 1/8 of a
    number's own power of two above, ties to even."""
    y = torch.empty_like(x)
    for at in range(0, x.shape[1], BLOCK):
        part = x[:, at:at + BLOCK]
        top = part.abs().amax(dim=1, keepdim=True)
        e = torch.ceil(torch.log2(torch.where(top > 0, top, 1.0) / TOP))
        e = torch.where(torch.exp2(e - 1) * TOP >= top, e - 1, e)
        e = torch.where(torch.exp2(e) * TOP < top, e + 1, e)
        unit = torch.exp2(torch.where(top > 0, e.clamp(min=float(LEAST)), float(LEAST)))
        a = part.abs() / unit
        power = torch.floor(torch.log2(torch.where(a > 0, a, 1.0)))
        power = torch.where(torch.exp2(power) > a, power - 1, power)
        step = torch.exp2(power.clamp(min=-6.0) - 3.0)
        y[:, at:at + BLOCK] = torch.round(part / unit / step) * step * unit
    return y


def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    path = case["path"]
    if path == "round":
        return {"y": _nearest(st["x"].double())}
    if path == "norm":
        x = st["x"].double()
        if st["delta"] is not None:
            x = (x + st["delta"].double()).to(st["x"].dtype).double()       # the residual stream is rounded to its type, then normalised
        mean = torch.linalg.vector_norm(x, dim=1, keepdim=True) ** 2 / case["width"]
        return {"x": x, "y": _nearest(x / torch.sqrt(mean + EPS) * st["gain"].double())}

    def product(w8, we):
        # block by block: whole products of e4m3 numbers, times both powers of two
        y = torch.zeros((case["rows"], case["out"]), dtype=torch.float64, device="cuda")
        for b in range(_blocks(case["width"])):
            at = slice(b * BLOCK, (b + 1) * BLOCK)
            part = st["x8"][:, at].double() @ w8[:, at].double().t().contiguous()
            y += part * torch.exp2(st["xe"][:, b].double() - 127.0)[:, None] * torch.exp2(we[:, b].double() - 127.0)
        return y

    if path == "linear":
        return {"y": product(*st["w"][0])}
    g, u = product(*st["w"][0]), product(*st["w"][1])
    return {"y": _nearest(g * torch.sigmoid(g) * u)}
