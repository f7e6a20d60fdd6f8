"""The operators of the 8-bit key/value cache, each beside its plain form: what it computes in elementary torch operations.

A decoding program that keeps its keys and values in 8 bits calls four operators per layer, and a fifth now and then:

  rope    vvs_rope_apply: queries and keys are rotated by positions on several axes (frame, row, column).
  attend  vvs_qcache_attention: the block's queries look at the cached slots of their row and at the block's own keys (chain or tree);
          softmax weights of the first queries are added up per slot.
  append  vvs_qcache_append: the block's keys and values, or those of the accepted path, are rounded into the cache.
  evict   vvs_qcache_evict: every head keeps its slots of largest accumulated weight; the others make room.
  read    vvs_qcache_read (inside append and evict here): cached values as the numbers they stand for.

What is held in 8 bits.  A row's keys (and values) of one head are cut into blocks of 32 slots.  A block has one power of two,
2^E, and its elements are e4m3 numbers times 2^E.  E is the smallest with max |x| <= 448 * 2^E over what was written into the
block, at least -110; a block that is written into again keeps the larger E, and what it holds is rounded to it."""
import math
import random

import numpy as np
import torch

own = False

BLOCK = 32
TOP = 448.0        # largest e4m3 number
LEAST = -110       # smallest E
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
PROFILE = (4, 6, 6, 4, 3, 3)     # nodes per depth of the benchmark's 26-node tree


# ------------------------------------------------------------------------------------------------ the cases
def _attend(name, rows, heads, kv_heads, size, cached, tokens, tree=False, counted=0, ragged=False, padded=False, dtype="bf16"):
    return {"name": name, "path": "attend", "rows": rows, "heads": heads, "kv_heads": kv_heads, "size": size, "cached": cached, "tokens": tokens,
            "tree": tree, "counted": counted, "ragged": ragged, "padded": padded, "dtype": dtype}


def _append(name, layers, rows, kv_heads, size, cached, tokens, picked, dtype="bf16"):
    return {"name": name, "path": "append", "layers": layers, "rows": rows, "kv_heads": kv_heads, "size": size, "cached": cached, "tokens": tokens,
            "picked": picked, "dtype": dtype}


def _evict(name, layers, rows, kv_heads, size, cached, keep, recent, ragged=False, dtype="bf16"):
    return {"name": name, "path": "evict", "layers": layers, "rows": rows, "kv_heads": kv_heads, "size": size, "cached": cached, "keep": keep,
            "recent": recent, "ragged": ragged, "dtype": dtype}


def _rope(name, rows, tokens, heads, kv_heads, size, axes, shared, halves, inverse=False, dtype="bf16"):
    return {"name": name, "path": "rope", "rows": rows, "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "size": size, "axes": axes,
            "shared": shared, "halves": halves, "inverse": inverse, "dtype": dtype}


def listed():
    return [
        # the fp32 reference shape, one prompt as a conditional / unconditional pair, chain of 4: the smallest call there is
        _attend("attend_tiny_fp32_x2", 2, 4, 4, 32, 33, 5, dtype="fp32"),
        # the small bf16 model as it is served: chain of 5, half way through a 16 x 16 image
        _attend("attend_b_chain5_x8", 8, 12, 12, 64, 129, 6),
        # the benchmark's workload: 26-node tree, 8 prompts, ragged lengths, the pending token's weights are counted
        _attend("attend_xl_tree26_x16", 16, 20, 20, 64, 408, 27, tree=True, counted=1, ragged=True),
        # the 7B shape with a tree for three prompts
        _attend("attend_7b_tree20_x6", 6, 32, 32, 128, 364, 21, tree=True, ragged=True),
        # one token per row over a long cache, four query heads to a key head: where reading the cache is everything
        _attend("attend_long_token_x16", 16, 32, 8, 128, 32768, 1, counted=1, ragged=True),
        # a chunk of a long prompt behind what is cached already, rows of different lengths, all weights counted
        _attend("attend_chunk512_x4", 4, 32, 8, 128, 2048, 512, counted=512, padded=True),
        # the accepted paths of the benchmark's step: up to 7 of 27 tokens, all 36 layers in one call
        _append("append_xl_path_36_layers", 36, 16, 20, 64, 408, 27, 7),
        # a chunk of a prompt in one layer of the 7B shape, its first block begun already
        _append("append_7b_chunk_x4", 1, 4, 32, 128, 70, 512, 512),
        # the benchmark's model at the end of its image: all layers cut from 696 slots to 256
        _evict("evict_xl_36_layers", 36, 16, 20, 64, 696, 256, 64),
        # one layer of a long cache cut to a quarter
        _evict("evict_long_x16", 1, 16, 8, 128, 32768, 8192, 256, ragged=True),
        # the benchmark's tree as part of a video: frame, row, column, every axis with frequencies of its own
        _rope("rope_xl_tree26_x16", 16, 27, 20, 20, 64, 3, False, False),
        # a long prompt with images and frames in it: one series of frequencies cut into three axes, halves rotate against each other
        _rope("rope_prompt_x4", 4, 8192, 32, 8, 128, 3, True, True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def draw(rng):
    most = {}
    for c in listed():
        most[c["path"]] = max(most.get(c["path"], 0.0), _seconds(c))
    while True:
        path = rng.choices(["attend", "append", "evict", "rope"], [5, 2, 2, 2])[0]
        heads, kv_heads, size = rng.choice([(12, 12, 64), (20, 20, 64), (32, 32, 128), (32, 8, 128), (16, 2, 128), (8, 1, 64), (20, 5, 64)])
        dtype = "bf16"
        if rng.random() < 0.2:
            dtype = "fp32"
            heads, kv_heads, size = rng.choice([(4, 4, 32), (8, 2, 32), (12, 12, 64), (16, 4, 64), (8, 8, 128)])
        rows = _log_int(rng, 1, 64)
        if path == "attend":
            tokens = rng.choice([1, _log_int(rng, 2, 64), _log_int(rng, 2, 64), _log_int(rng, 65, 512)])
            c = _attend("", rows, heads, kv_heads, size, _log_int(rng, 1, 32768), tokens, tree=8 < tokens <= 64 and rng.random() < 0.6,
                        counted=rng.choice([0, 1, tokens]), ragged=rng.random() < 0.5, padded=rng.random() < 0.3, dtype=dtype)
        elif path == "append":
            tokens = _log_int(rng, 1, 512)
            picked = tokens if tokens > 64 or rng.random() < 0.4 else rng.randint(1, tokens)
            c = _append("", rng.choice([1, 12, 36]), rows, kv_heads, size, _log_int(rng, 1, 4096), tokens, picked, dtype=dtype)
        elif path == "evict":
            cached = _log_int(rng, 48, 32768)
            keep = 32 * _log_int(rng, 1, cached // 32)
            c = _evict("", rng.choice([1, 12, 36]), rows, kv_heads, size, cached, keep, rng.randint(0, keep // 2), ragged=rng.random() < 0.5, dtype=dtype)
        else:
            c = _rope("", rows, _log_int(rng, 1, 8192), heads, kv_heads, size, rng.randint(1, 4), rng.random() < 0.5, rng.random() < 0.5,
                      inverse=rng.random() < 0.3, dtype=dtype)
        if _seconds(c) <= most[path] and _held(c) <= 1 << 30:
            del c["name"]
            return c


def _held(c):
    """Elements of keys (and of values) that a case holds: bounds the memory of the plain forms."""
    if c["path"] == "rope":
        return c["rows"] * c["tokens"] * c["heads"] * c["size"]
    return c.get("layers", 1) * c["rows"] * c["kv_heads"] * c["size"] * _capacity(c)


# ------------------------------------------------------------------------------------------------ sizes
def _lengths(case):
    """Cached slots of each row.  Ragged: spread below the case's number, odd ones among them."""
    n, rows = case["cached"], case["rows"]
    return [max(1, n - (r * 37 + 5) % max(2, n // 3)) if case.get("ragged") else n for r in range(rows)]


def _counts(case):
    """Block tokens of each row."""
    n, rows = case["tokens"], case["rows"]
    return [max(1, n - r * (n // 4)) if case.get("padded") else n for r in range(rows)]


def _taken(case):
    """Tokens that an append takes of each row: paths of different lengths, chunks whole."""
    n, rows = case["picked"], case["rows"]
    return [n if n == case["tokens"] else 1 + (r * 5 + n) % n for r in range(rows)]


def _capacity(case):
    return -(-(case["cached"] + case.get("tokens", 0)) // BLOCK) * BLOCK


def _pairs(case):
    """Rotated pairs of each axis: an axis each for frame, row, column and one more, the last ones equal, the first with what is left."""
    half, axes = case["size"] // 2, case["axes"]
    last = half // (axes + 1) if axes > 1 else 0
    return [half - last * (axes - 1)] + [last] * (axes - 1)


def _wide(case):
    return 4 if case["dtype"] == "fp32" else 2


def work(case):
    path, e = case["path"], _wide(case)
    if path == "rope":
        values = case["rows"] * case["tokens"] * (case["heads"] + case["kv_heads"]) * case["size"]
        return {"bytes": 2 * e * values + 4 * case["rows"] * case["tokens"] * case["axes"], "flops": 3 * values}
    per = case["kv_heads"] * case["size"]
    if path == "attend":
        lens, counts = _lengths(case), _counts(case)
        bytes_ = flops = 0
        for n, t in zip(lens, counts):
            bytes_ += 2 * n * per + 2 * e * t * (per + case["heads"] * case["size"])
            if case["counted"]:
                bytes_ += 8 * n * case["kv_heads"]
            seen = t * n + (t * (t + 1) // 2 if not case["tree"] else 4 * t)
            flops += 4 * case["heads"] * case["size"] * seen
        return {"bytes": bytes_, "flops": flops}
    layers = case["layers"]
    if path == "append":
        n = layers * sum(_taken(case))
        old = layers * case["rows"] * (case["cached"] % BLOCK)
        return {"bytes": 2 * per * (n * (e + e) + old * (1 + e)), "flops": 4 * per * n}
    kept = layers * sum(min(n, case["keep"]) for n in _lengths(case))
    return {"bytes": 2 * per * kept * (1 + e) + 8 * case["kv_heads"] * (layers * sum(_lengths(case)) + kept), "flops": 2 * per * kept}


def _seconds(case):
    w = work(case)
    return max(w["bytes"] / 8e12, w["flops"] / 2.5e15)


# ------------------------------------------------------------------------------------------------ inputs
class _Maker:
    def __init__(self, seed):
        self.g = torch.Generator("cuda")
        self.g.manual_seed(int(seed))

    def normal(self, dims, dtype=torch.float32, std=1.0):
        return torch.empty(dims, dtype=dtype, device="cuda").normal_(0.0, std, generator=self.g)

    def uniform(self, dims):
        return torch.rand(dims, generator=self.g, device="cuda")

    def spread(self, heads, size):
        """Keys and values in earnest: a few dimensions of every head are several times as large as the others."""
        return torch.exp2(self.normal((heads, size)).mul_(0.8))


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _parents(n):
    """Parent array of an n-node tree with the benchmark's profile of nodes per depth."""
    ends = [round(n * c / sum(PROFILE)) for c in np.cumsum(PROFILE)]
    levels = [list(range(a + 1, b + 1)) for a, b in zip([0] + ends[:-1], ends) if b > a]
    parent, above = [], [0]
    for nodes in levels:
        parent += [above[i * len(above) // len(nodes)] for i in range(len(nodes))]
        above = nodes
    return np.asarray(parent, dtype=np.int32)


def _seen(parent, n):
    """[n, n]: token i sees token j of its block (itself and its ancestors; parent None: all tokens before it)."""
    if parent is None:
        return torch.ones((n, n), dtype=torch.bool, device="cuda").tril()
    see = np.eye(n, dtype=bool)
    for j in range(1, n):
        see[j] |= see[parent[j - 1]]
    return torch.from_numpy(see).cuda()


def _history(mk, case, layers, slots):
    """What the cache was filled with: keys and values [layers, rows, slots, kv heads, size]."""
    dims = (layers, case["rows"], slots, case["kv_heads"], case["size"])
    dtype = TYPES[case["dtype"]]
    k = mk.normal(dims, dtype).mul_(mk.spread(case["kv_heads"], case["size"]).to(dtype))
    return k, mk.normal(dims, dtype).mul_(mk.spread(case["kv_heads"], case["size"]).to(dtype))


def _as_held(x):
    """[layers, rows, slots, heads, size] -> e4m3 numbers [layers, rows, heads, slots, size] and E [layers, rows, heads, blocks]."""
    layers, rows, slots, heads, size = x.shape
    x = x.float().view(layers, rows, slots // BLOCK, BLOCK, heads, size)
    e = _exponent(x.abs().amax(dim=(3, 5)))
    x = torch.ldexp(x, -e.view(layers, rows, -1, 1, heads, 1)).to(torch.float8_e4m3fn)
    return x.view(layers, rows, slots, heads, size).transpose(2, 3).contiguous(), e.transpose(2, 3).contiguous()


def _exponent(top):
    """Smallest E with top <= 448 * 2^E, at least LEAST."""
    m, e = torch.frexp(top)
    return (e - 9 + (m > 0.875)).clamp_(min=LEAST).to(torch.int32)


def prepare(case, seed):
    mk, path, dtype = _Maker(seed), case["path"], TYPES[case["dtype"]]
    rows, size, kv_heads = case["rows"], case["size"], case["kv_heads"]
    st = {"case": dict(case), "dtype": dtype}
    rng = random.Random(int(seed))
    if path == "rope":
        tokens, heads = case["tokens"], case["heads"]
        st["q"], st["k"] = mk.normal((rows, tokens, heads, size), dtype), mk.normal((rows, tokens, kv_heads, size), dtype)
        # frames far into a film, rows and columns of an image, and a text position that has gone far
        reach = torch.tensor([100000, 32, 32, 4096][:case["axes"]] if case["axes"] > 1 else [131072], device="cuda")
        st["pos"] = (mk.uniform((rows, tokens, case["axes"])) * reach).to(torch.int32)
        base = 10000.0
        pairs = _pairs(case)
        # radians per position of each pair, and the axis it follows
        st["axis"] = torch.tensor([a for a, n in enumerate(pairs) for _ in range(n)], device="cuda")
        rate = [i / (size // 2) for i in range(size // 2)] if case["shared"] else [i / n for n in pairs for i in range(n)]
        st["rate"] = torch.tensor([base ** -r for r in rate], dtype=torch.float64, device="cuda")
        st["q_out"], st["k_out"] = torch.empty_like(st["q"]), torch.empty_like(st["k"])
        if own:
            from paper_2511_13587_amd import binding as vb
            st["rope"] = vb.Rope(size, pairs, base, vb.VVS_FP32 if dtype == torch.float32 else vb.VVS_BF16, shared=case["shared"], halves=case["halves"])
        return st
    lens = _lengths(case)
    rng.shuffle(lens)
    st["len"] = _ints(lens)
    capacity, layers = _capacity(case), case.get("layers", 1)
    heads = case.get("heads", kv_heads)
    k, v = _history(mk, case, layers, capacity)
    if path == "append":
        # the block that the append begins in holds only what is below the length
        past = (torch.arange(capacity, device="cuda") >= case["cached"]).view(1, 1, -1, 1, 1)
        k, v = k.masked_fill(past, 0.0), v.masked_fill(past, 0.0)
    if own:
        from paper_2511_13587_amd import binding as vb
        st["cache"] = vb.QCache(layers, rows, heads, kv_heads, size, capacity, case.get("tokens", 1), vb.VVS_FP32 if dtype == torch.float32 else vb.VVS_BF16)
        st["cache"].vvs_qcache_append(_ints([0] * rows), k, v, n_tokens=_ints([case["cached"]] * rows) if path == "append" else None, n_layers=layers)
    else:
        (st["k8"], st["ke"]), (st["v8"], st["ve"]) = _as_held(k), _as_held(v)
    del k, v
    if path == "attend":
        tokens = case["tokens"]
        counts = _counts(case)
        rng.shuffle(counts)
        st["n"] = _ints(counts) if case["padded"] else None
        st["parent"] = _parents(tokens - 1) if case["tree"] else None
        st["see"] = _seen(st["parent"], tokens)
        # the queries of a row lie beside its keys and values, as one projection writes them
        st["qkv"] = mk.normal((rows, tokens, heads + 2 * kv_heads, size), dtype)
        st["out"] = torch.zeros((rows, tokens, heads, size), dtype=dtype, device="cuda")
        st["lse"] = torch.zeros((rows, tokens, heads), device="cuda")
        st["mass"] = mk.uniform((rows, kv_heads, capacity)) if case["counted"] else None
        st["block_mass"] = torch.zeros((rows, kv_heads, tokens), device="cuda") if case["counted"] else None
    elif path == "append":
        st["k"] = mk.normal((layers, rows, case["tokens"], kv_heads, size), dtype, 1.5)
        st["v"] = mk.normal((layers, rows, case["tokens"], kv_heads, size), dtype, 1.5)
        taken = _taken(case)
        rng.shuffle(taken)
        st["n"] = _ints(taken)
        st["pick"] = None
        if case["picked"] < case["tokens"]:
            st["pick"] = _ints([[0] + sorted(rng.sample(range(1, case["tokens"]), case["picked"] - 1)) for _ in range(rows)])
        # what is looked at afterwards: the blocks that were written into
        st["window"] = BLOCK * -(-(case["cached"] % BLOCK + case["picked"]) // BLOCK)
        st["first"] = st["len"] // BLOCK * BLOCK
        st["after"] = st["len"] + st["n"]
        out = (layers, rows, st["window"], kv_heads, size)
        st["k_out"], st["v_out"] = torch.zeros(out, dtype=dtype, device="cuda"), torch.zeros(out, dtype=dtype, device="cuda")
    else:
        # accumulated weights fall off steeply; some slots were never looked at
        dims = (layers, rows, kv_heads, capacity)
        mass = torch.exp(2.0 * mk.normal(dims)) * (mk.uniform(dims) > 0.05)
        st["mass"], st["mass_out"] = mass, torch.zeros_like(mass)
        # an earlier eviction has mixed the order of the slots
        pos = torch.arange(capacity, dtype=torch.int32, device="cuda")
        turn = capacity // 3
        st["pos"] = torch.cat([pos[turn:2 * turn], pos[:turn], pos[2 * turn:]]).expand(dims).contiguous()
        st["pos_out"] = torch.zeros_like(st["pos"])
        st["after"] = st["len"].clamp(max=case["keep"])
        out = (layers, rows, case["keep"], kv_heads, size)
        st["k_out"], st["v_out"] = torch.zeros(out, dtype=dtype, device="cuda"), torch.zeros(out, dtype=dtype, device="cuda")
    return st


# ------------------------------------------------------------------------------------------------ one pass
def run(st):
    path = st["case"]["path"]
    return {"attend": _run_attend, "append": _run_append, "evict": _run_evict, "rope": _run_rope}[path](st)


def _run_rope(st):
    c = st["case"]
    if own:
        st["rope"].vvs_rope_apply(st["pos"], st["q"], st["k"], st["q_out"], st["k_out"], inverse=c["inverse"])
        return {"q": st["q_out"], "k": st["k_out"]}
    # angles of far positions are taken in 64 bits
    angle = st["pos"][:, :, st["axis"]].double() * st["rate"]
    cos, sin = torch.cos(angle).float()[:, :, None], torch.sin(angle).float()[:, :, None]
    if c["inverse"]:
        sin = -sin
    got = {}
    for name in ("q", "k"):
        x = st[name].float()
        half = c["size"] // 2
        a, b = (x[..., :half], x[..., half:]) if c["halves"] else (x[..., 0::2], x[..., 1::2])
        y = (a * cos - b * sin, a * sin + b * cos)
        got[name] = (torch.cat(y, dim=-1) if c["halves"] else torch.stack(y, dim=-1).flatten(-2)).to(st["dtype"])
    return got


def _held_values(x8, e):
    """e4m3 numbers [..., slots, size] and E [..., blocks] -> fp32 values."""
    x = x8.float()
    return torch.ldexp(x.unflatten(-2, (-1, BLOCK)), e[..., None, None]).flatten(-3, -2)


def _run_attend(st):
    c = st["case"]
    heads, kv_heads, size, tokens, rows = c["heads"], c["kv_heads"], c["size"], c["tokens"], c["rows"]
    q, k, v = st["qkv"].split([heads, kv_heads, kv_heads], dim=2)
    if own:
        st["cache"].vvs_qcache_attention(st["len"], q, k, v, st["out"], n_tokens=st["n"], parent=st["parent"], lse=st["lse"], n_counted=c["counted"],
                                         mass=st["mass"], block_mass=st["block_mass"])
        return {"out": st["out"], "lse": st["lse"], "mass": st["mass"], "block_mass": st["block_mass"]}
    group = heads // kv_heads
    most = int(c["cached"])
    # [rows, kv heads, group * tokens, size]
    q = q.float().view(rows, tokens, kv_heads, group, size).permute(0, 2, 3, 1, 4).reshape(rows, kv_heads, group * tokens, size)
    k = torch.cat([_held_values(st["k8"][0], st["ke"][0])[:, :, :most], k.float().transpose(1, 2)], dim=2)
    v = torch.cat([_held_values(st["v8"][0], st["ve"][0])[:, :, :most], v.float().transpose(1, 2)], dim=2)
    score = torch.matmul(q, k.transpose(2, 3)) * (1.0 / math.sqrt(size))
    cached = (torch.arange(most, device="cuda") < st["len"][:, None]).view(rows, 1, most).expand(rows, tokens, most)
    real = torch.ones((rows, tokens), dtype=torch.bool, device="cuda") if st["n"] is None else torch.arange(tokens, device="cuda") < st["n"][:, None]
    see = torch.cat([cached, st["see"].expand(rows, tokens, tokens) & real[:, None, :]], dim=2)
    score = score.view(rows, kv_heads, group, tokens, most + tokens).masked_fill(~see[:, None, None], -math.inf)
    top = score.amax(dim=-1, keepdim=True)
    top = torch.where(real[:, None, None, :, None], top, 0.0)
    weight = torch.exp(score - top)
    total = weight.sum(dim=-1, keepdim=True)
    weight = torch.where(real[:, None, None, :, None], weight / total, 0.0)
    out = torch.matmul(weight.view(rows, kv_heads, group * tokens, most + tokens), v)
    out = out.view(rows, kv_heads, group, tokens, size).permute(0, 3, 1, 2, 4).reshape(rows, tokens, heads, size).to(st["dtype"])
    lse = torch.where(real[:, None, None, :], (top + torch.log(total))[..., 0], 0.0).permute(0, 3, 1, 2).reshape(rows, tokens, heads)
    if not c["counted"]:
        return {"out": out, "lse": lse, "mass": None, "block_mass": None}
    each = weight[:, :, :, :c["counted"]].sum(dim=(2, 3))
    st["mass"][:, :, :most] += each[:, :, :most]
    return {"out": out, "lse": lse, "mass": st["mass"], "block_mass": each[:, :, most:]}


def _run_append(st):
    c = st["case"]
    if own:
        cache, layers = st["cache"], c["layers"]
        cache.vvs_qcache_append(st["len"], st["k"], st["v"], n_tokens=st["n"], select=st["pick"], n_layers=layers)
        cache.vvs_qcache_read(st["after"], st["k_out"], st["v_out"], first=st["first"], n_layers=layers)
        return {"k": st["k_out"], "v": st["v_out"]}
    layers, rows, width = c["layers"], c["rows"], st["window"]
    slot = st["first"][:, None] + torch.arange(width, device="cuda")            # [rows, width]
    old, new = slot < st["len"][:, None], (slot >= st["len"][:, None]) & (slot < st["after"][:, None])
    token = (slot - st["len"][:, None]).clamp_(0, c["picked"] - 1)
    if st["pick"] is not None:
        token = torch.gather(st["pick"], 1, token)
    row = torch.arange(rows, device="cuda")[:, None]
    got = {}
    for name in ("k", "v"):
        x8, e = st[name + "8"], st[name + "e"]
        at = slot.clamp(max=x8.shape[3] - 1)
        block = st["first"] // BLOCK
        was_e = e[:, row[:, 0], :, block.long()].permute(1, 0, 2)             # [layers, rows, heads]: E of the first block
        was = x8.view(torch.uint8)[:, row, :, at].view(torch.float8_e4m3fn).float().permute(2, 0, 1, 3, 4)
        was = torch.ldexp(was, was_e[:, :, None, :, None])
        fresh = st[name][:, row, token].float()
        fresh = torch.where(new[None, :, :, None, None], fresh, 0.0)
        blocks = (layers, rows, width // BLOCK, BLOCK, c["kv_heads"], c["size"])
        need = _exponent(fresh.view(blocks).abs().amax(dim=(3, 5)))             # [layers, rows, blocks, heads]
        begun = (st["len"] % BLOCK > 0).view(1, rows, 1)
        need[:, :, 0] = torch.where(begun, torch.maximum(need[:, :, 0], was_e), need[:, :, 0])
        both = torch.where(old[None, :, :, None, None], was, fresh).view(blocks)
        need = need.view(layers, rows, -1, 1, c["kv_heads"], 1)
        held = torch.ldexp(torch.ldexp(both, -need).to(torch.float8_e4m3fn).float(), need)
        got[name] = held.view(layers, rows, width, c["kv_heads"], c["size"]).to(st["dtype"])
    return got


def _run_evict(st):
    c = st["case"]
    keep, layers, rows, heads = c["keep"], c["layers"], c["rows"], c["kv_heads"]
    if own:
        cache = st["cache"]
        cache.vvs_qcache_evict(st["len"], keep, c["recent"], st["mass"], st["mass_out"], st["pos"], st["pos_out"], n_layers=layers)
        cache.vvs_qcache_read(st["after"], st["k_out"], st["v_out"], n_layers=layers)
        return {"k": st["k_out"], "v": st["v_out"], "mass": st["mass_out"], "pos": st["pos_out"]}
    mass, pos, length = st["mass"], st["pos"], st["len"].view(1, rows, 1, 1)
    capacity = mass.shape[3]
    slot = torch.arange(capacity, device="cuda").expand_as(mass)
    valid = slot < length
    newest = torch.where(valid, pos, -1).amax(dim=3, keepdim=True)
    key = torch.where(pos > newest - c["recent"], math.inf, mass)
    key = torch.where(valid, key, -math.inf)
    order = torch.sort(key, dim=3, descending=True, stable=True).indices
    kept = torch.zeros_like(valid).scatter_(3, order[..., :keep], True) & valid
    hole, source = ~kept & (slot < keep) & valid, kept & (slot >= keep)
    queue = torch.sort(torch.where(source, slot, capacity), dim=3).values[..., :keep]
    nth = (hole.cumsum(dim=3) - 1).clamp_(min=0)[..., :keep]
    origin = torch.where(hole[..., :keep], torch.gather(queue, 3, nth), slot[..., :keep])   # [layers, rows, heads, keep]
    left = (slot < length.clamp(max=keep))[..., :keep]
    got = {}
    for name in ("k", "v"):
        x8, e = st[name + "8"], st[name + "e"]
        from_e = torch.gather(e, 3, (origin // BLOCK).clamp(max=e.shape[3] - 1))
        to_e = torch.where(left, from_e, LEAST).unflatten(3, (-1, BLOCK)).amax(dim=4)
        # a block that nothing moves into stays as it is
        to_e = torch.where(hole[..., :keep].unflatten(3, (-1, BLOCK)).any(dim=4), to_e, e[..., :keep // BLOCK])
        x = torch.gather(x8.view(torch.uint8), 3, origin.clamp(max=capacity - 1)[..., None].expand(-1, -1, -1, -1, c["size"])).view(torch.float8_e4m3fn).float()
        x = torch.ldexp(x, (from_e - to_e.repeat_interleave(BLOCK, dim=3))[..., None]).to(torch.float8_e4m3fn)
        st[name + "8"][:, :, :, :keep] = x
        st[name + "e"][..., :keep // BLOCK] = to_e
        x = torch.where(left[..., None], _held_values(x, to_e), 0.0)
        got[name] = x.transpose(2, 3).to(st["dtype"])
    went = torch.where(left, torch.gather(mass, 3, origin.clamp(max=capacity - 1)), 0.0)
    got["mass"] = torch.cat([went, torch.zeros_like(mass[..., keep:])], dim=3)
    went = torch.where(left, torch.gather(pos, 3, origin.clamp(max=capacity - 1)), 0)
    got["pos"] = torch.cat([went, torch.zeros_like(pos[..., keep:])], dim=3)
    return got


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def _round_e4m3(x):
    """Nearest e4m3 number, ties to even, of float64 values of at most 448: steps of 2^-9 below 2^-6, of 1/8 of the power of two above."""
    a = x.abs()
    power = torch.floor(torch.log2(torch.where(a > 0, a, 1.0)))
    power = torch.where(torch.exp2(power) > a, power - 1, power)
    step = torch.exp2(torch.clamp(power, min=-6.0) - 3.0)
    return torch.round(x / step) * step


def _least_power(top):
    e = torch.ceil(torch.log2(torch.where(top > 0, top, 1.0) / TOP))
    e = torch.where(torch.exp2(e - 1) * TOP >= top, e - 1, e)
    e = torch.where(torch.exp2(e) * TOP < top, e + 1, e)
    return torch.where(top > 0, torch.clamp(e, min=float(LEAST)), float(LEAST))


def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    path = case["path"]
    if path == "rope":
        rate = st["rate"][None, None]
        theta = torch.stack([st["pos"][:, :, a].double() for a in st["axis"].tolist()], dim=2) * rate
        turn = torch.polar(torch.ones_like(theta), -theta if case["inverse"] else theta)[:, :, None]
        got = {}
        for name in ("q", "k"):
            x = st[name].double()
            if case["halves"]:
                x = x.unflatten(-1, (2, -1)).transpose(-1, -2)
            else:
                x = x.unflatten(-1, (-1, 2))
            y = torch.view_as_real(torch.view_as_complex(x.contiguous()) * turn)
            got[name] = y.transpose(-1, -2).flatten(-2) if case["halves"] else y.flatten(-2)
        return got
    lens = st["len"].tolist()
    if path == "attend":
        heads, kv_heads, size, tokens = case["heads"], case["kv_heads"], case["size"], case["tokens"]
        out = torch.zeros(st["out"].shape, dtype=torch.float64, device="cuda")
        lse = torch.zeros(st["lse"].shape, dtype=torch.float64, device="cuda")
        counted = case["counted"] > 0
        mass = st["mass"].double() if counted else None
        block_mass = torch.zeros(st["block_mass"].shape, dtype=torch.float64, device="cuda") if counted else None
        group = heads // kv_heads
        for r, n in enumerate(lens):
            t = tokens if st["n"] is None else int(st["n"][r])
            for h in range(kv_heads):
                old = [st[x + "8"][0, r, h, :n].double() * torch.exp2(st[x + "e"][0, r, h].double()).repeat_interleave(BLOCK)[:n, None] for x in "kv"]
                keys = torch.cat([old[0], st["qkv"][r, :t, heads + h].double()])
                vals = torch.cat([old[1], st["qkv"][r, :t, heads + kv_heads + h].double()])
                ask = st["qkv"][r, :t, h * group:(h + 1) * group].double().transpose(0, 1).reshape(group * t, size)
                s = ask @ keys.T / size ** 0.5
                s[:, n:] += torch.where(st["see"][:t, :t], 0.0, -math.inf).double().repeat(group, 1)
                lse[r, :t, h * group:(h + 1) * group] = torch.logsumexp(s, dim=1).view(group, t).T
                p = torch.softmax(s, dim=1)
                out[r, :t, h * group:(h + 1) * group] = (p @ vals).view(group, t, size).transpose(0, 1)
                if counted:
                    w = p.view(group, t, n + t)[:, :case["counted"]].sum(dim=(0, 1))
                    mass[r, h, :n] += w[:n]
                    block_mass[r, h, :t] = w[n:]
        return {"out": out, "lse": lse, "mass": mass, "block_mass": block_mass}
    layers, rows, kv_heads = case["layers"], case["rows"], case["kv_heads"]
    if path == "append":
        got = {}
        for name in ("k", "v"):
            y = torch.zeros(st["k_out"].shape, dtype=torch.float64, device="cuda")
            for r, n in enumerate(lens):
                b, count = n // BLOCK, int(st["n"][r])
                tokens = st["pick"][r, :count].long() if st["pick"] is not None else torch.arange(count, device="cuda")
                x = st[name][:, r, tokens].double()                            # [layers, count, heads, size]
                prior = st[name + "8"][:, r, :, b * BLOCK:n].double().transpose(1, 2)
                prior_e = st[name + "e"][:, r, :, b].double()
                prior = prior * torch.exp2(prior_e)[:, None, :, None]
                whole = torch.cat([prior, x], dim=1)
                for j in range(0, whole.shape[1], BLOCK):
                    part = whole[:, j:j + BLOCK]
                    written = x[:, :BLOCK - (n % BLOCK)] if j == 0 else part
                    e = _least_power(written.abs().amax(dim=(1, 3)))
                    if j == 0 and n % BLOCK:
                        e = torch.maximum(e, prior_e)
                    unit = torch.exp2(e)[:, None, :, None]
                    y[:, r, j:j + part.shape[1]] = _round_e4m3(part / unit) * unit
            got[name] = y
        return got
    keep, recent = case["keep"], case["recent"]
    capacity = st["mass"].shape[3]
    mass, pos = st["mass"].double().cpu().numpy(), st["pos"].cpu().numpy()
    origin = np.zeros((layers, rows, kv_heads, keep), dtype=np.int64)
    mass_out, pos_out = np.zeros_like(mass), np.zeros_like(pos)
    for l in range(layers):
        for r, n in enumerate(lens):
            left = min(n, keep)
            for h in range(kv_heads):
                m, p = mass[l, r, h, :n].copy(), pos[l, r, h, :n]
                if n > keep:
                    m[p > p.max() - recent] = np.inf
                    chosen = np.zeros(n, dtype=bool)
                    chosen[np.lexsort((np.arange(n), -m))[:keep]] = True
                    o = np.arange(keep)
                    o[~chosen[:keep]] = keep + np.flatnonzero(chosen[keep:])
                else:
                    o = np.arange(n)
                origin[l, r, h, :left] = o
                mass_out[l, r, h, :left], pos_out[l, r, h, :left] = mass[l, r, h, o], pos[l, r, h, o]
    origin = torch.from_numpy(origin).cuda()
    got = {"mass": torch.from_numpy(mass_out), "pos": torch.from_numpy(pos_out)}
    for name in ("k", "v"):
        y = torch.zeros((layers, rows, keep, kv_heads, case["size"]), dtype=torch.float64, device="cuda")
        for r, n in enumerate(lens):
            left = min(n, keep)
            o = origin[:, r, :, :left]
            e = torch.gather(st[name + "e"][:, r], 2, o // BLOCK).double()
            x = torch.gather(st[name + "8"][:, r].view(torch.uint8), 2, o[..., None].expand(-1, -1, -1, case["size"])).view(torch.float8_e4m3fn).double()
            x = x * torch.exp2(e)[..., None]
            moved = o != torch.arange(left, device="cuda")
            for j in range(0, left, BLOCK):
                top = e[:, :, j:j + BLOCK].amax(dim=2)
                top = torch.where(moved[:, :, j:j + BLOCK].any(dim=2), top, st[name + "e"][:, r, :, j // BLOCK].double())
                unit = torch.exp2(top)[..., None, None]
                part = x[:, :, j:j + BLOCK]
                y[:, r, j:j + part.shape[2]] = (_round_e4m3(part / unit) * unit).transpose(1, 2)
        got[name] = y
    return got
