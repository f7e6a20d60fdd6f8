"""Rows and weights in 8 bits as a program uses them: a whole decoder layer beside the 8-bit cache and the rotary operator, captured graphs, other streams, shared workspaces, special values."""
import pytest
import torch

import qlinear_common as qc
from test_gpu_qlinear import _linear, _normal, check_gate, check_product, product_error

pytestmark = pytest.mark.gpu


class Layer:
    """A decoder layer whose projections are in 8 bits."""

    def __init__(self, vb, d, heads, size, hidden, rows, tokens, seed):
        self.vb, self.heads, self.size, self.tokens, self.rows = vb, heads, size, tokens, rows
        m, e = rows * tokens, heads * size
        self.gains = [(1 + 0.2 * _normal((d,), seed + i, 0)).cuda() for i in range(2)]
        shapes = {"qkv": (d, 3 * e), "o": (e, d), "up": (d, hidden), "gate": (d, hidden), "down": (hidden, d)}
        self.w = {k: (_normal(s, seed + 7 * len(k) + s[1], 0.5) * s[0] ** -0.5).bfloat16() for k, s in shapes.items()}
        maps = {"qkv": vb.QLinear(d, 3 * e, m, vb.VVS_BF16), "o": vb.QLinear(e, d, m, vb.VVS_BF16), "gate": vb.QLinear(d, hidden, m, vb.VVS_BF16, gated=True), "down": vb.QLinear(hidden, d, m, vb.VVS_BF16)}
        maps["qkv"].vvs_qlinear_load(self.w["qkv"].cuda())
        maps["o"].vvs_qlinear_load(self.w["o"].cuda())
        maps["gate"].vvs_qlinear_load(self.w["gate"].cuda(), self.w["up"].cuda())
        maps["down"].vvs_qlinear_load(self.w["down"].cuda())
        self.maps = maps
        self.cache = vb.QCache(1, rows, heads, heads, size, 64, tokens, vb.VVS_BF16)
        self.rope = vb.Rope(size, [size // 4, size // 4], 10000.0, vb.VVS_BF16)
        self.length = torch.zeros(rows, dtype=torch.int32, device="cuda")
        self.pos = torch.arange(m * 2, dtype=torch.int32, device="cuda").view(m, 2) % 17
        self.h8, self.a8, self.g8 = vb.QRows(m, d), vb.QRows(m, e), vb.QRows(m, hidden)
        self.qkv = torch.empty((m, 3, heads, size), dtype=torch.bfloat16, device="cuda")
        self.att = torch.empty((rows, tokens, heads, size), dtype=torch.bfloat16, device="cuda")
        self.o, self.out = (torch.empty((m, d), device="cuda") for _ in range(2))
        self.x1, self.x2 = (torch.empty((m, d), device="cuda") for _ in range(2))

    def run(self, x):
        """x float32 [rows * tokens, d] -> residual stream in front of the last addition, and what is added to it."""
        vb, m = self.vb, self.rows * self.tokens
        vb.vvs_qrows_norm(x, self.gains[0], 1e-5, self.h8, x_out=self.x1)
        self.maps["qkv"].vvs_qlinear_apply(self.h8, self.qkv.view(m, -1))
        q, k, v = self.qkv[:, 0], self.qkv[:, 1], self.qkv[:, 2]
        self.rope.vvs_rope_apply(self.pos, q, k, q, k)
        four = (self.rows, self.tokens, self.heads, self.size)
        self.cache.vvs_qcache_attention(self.length, q.view(four), k.view(four), v.view(four), self.att)
        vb.vvs_qrows_round(self.att.view(m, -1), self.a8)
        self.maps["o"].vvs_qlinear_apply(self.a8, self.o)
        vb.vvs_qrows_norm(self.x1, self.gains[1], 1e-5, self.h8, delta=self.o, x_out=self.x2)
        self.maps["gate"].vvs_qlinear_gate(self.h8, self.g8)
        self.maps["down"].vvs_qlinear_apply(self.g8, self.out)
        return self.x2, self.out


@pytest.mark.parametrize("rows,tokens", [(2, 5), (4, 12), (6, 27)])
def test_a_layer_stage_by_stage(rows, tokens):
    """Every stage beside its statement in 64 bits on what the stage in front of it left."""
    from paper_2511_13587_amd import binding as vb
    d, heads, size, hidden, m = 384, 6, 64, 1000, rows * tokens
    layer = Layer(vb, d, heads, size, hidden, rows, tokens, 3)
    w = {k: qc.held(v.t())[0].t() for k, v in layer.w.items()}
    x = _normal((m, d), 1)
    held = {}

    def norm(gain, x):
        x = x.double()
        return x / torch.sqrt((x * x).mean(dim=1, keepdim=True) + 1e-5) * gain.cpu().double()

    # the rows are overwritten within the layer: its calls one by one
    vb.vvs_qrows_norm(x.cuda(), layer.gains[0], 1e-5, layer.h8, x_out=layer.x1)
    y = norm(layer.gains[0], x)
    qc.check_rounded(layer.h8, y, y.abs() * 64 * 2.0 ** -24)
    held["h"] = qc.values_of(layer.h8)
    layer.maps["qkv"].vvs_qlinear_apply(layer.h8, layer.qkv.view(m, -1))
    check_product(layer.qkv.view(m, -1), held["h"], w["qkv"], torch.bfloat16, fast=m > 64)
    x2, out = layer.run(x.cuda())
    att = layer.att.cpu().double().view(m, -1)
    assert torch.isfinite(att).all()
    held["a"], _ = qc.held(att)
    assert torch.equal(qc.values_of(layer.a8), held["a"])
    check_product(layer.o, held["a"], w["o"], torch.float32)
    kept = (layer.x1.cpu() + layer.o.cpu())
    assert torch.equal(layer.x1.cpu(), x) and torch.equal(x2.cpu(), kept)
    y = norm(layer.gains[1], kept)
    qc.check_rounded(layer.h8, y, y.abs() * 64 * 2.0 ** -24)
    held["h"] = qc.values_of(layer.h8)
    check_gate(layer.g8, held["h"], [w["gate"], w["up"]], fast=m > 64)
    check_product(out, qc.values_of(layer.g8), w["down"], torch.float32)


@pytest.mark.parametrize("rows,tokens", [(2, 5), (4, 12), (6, 27)])
def test_a_captured_layer_gives_the_eager_bits(rows, tokens):
    """A graph of the layer, replayed with other inputs, eager work and synchronizations between."""
    from paper_2511_13587_amd import binding as vb
    layer = Layer(vb, 384, 6, 64, 1000, rows, tokens, 5)
    m = rows * tokens
    inputs = [_normal((m, 384), 20 + i).cuda() for i in range(6)]
    want = []
    for x in inputs:
        x2, out = layer.run(x)
        want.append((x2.clone(), out.clone()))
    x = torch.empty_like(inputs[0])
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        x.copy_(inputs[0])
        layer.run(x)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            x2, out = layer.run(x)
    torch.cuda.synchronize()
    for i in (1, 0, 2, 3, 3, 4, 5, 0):
        x.copy_(inputs[i])
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            graph.replay()
        stream.synchronize()
        assert torch.equal(x2, want[i][0]) and torch.equal(out, want[i][1])
        ex2, eout = layer.run(inputs[(i + 1) % 6])
        torch.cuda.synchronize()
        assert torch.equal(eout, want[(i + 1) % 6][1]) and torch.equal(ex2, want[(i + 1) % 6][0])


# a contraction in halves; columns of one tile; a gated block joined by the last of eight workgroups; tiles
CALLS = [(28, 8300, 300, False), (28, 640, 300, False), (14, 1280, 700, True), (30, 1280, 700, True), (60, 700, 500, True), (200, 1280, 3000, False), (300, 640, 700, True)]


def test_maps_share_a_workspace_on_a_stream():
    """Calls of several maps one after another leave the counters as they found them: three rounds with the same bits, those of maps with workspaces of their own."""
    from paper_2511_13587_amd import binding as vb
    most = max(vb.vvs_qlinear_query_sizes(vb.VvsQLinearConfig(k, n, m, int(g), vb.VVS_BF16))[1] for m, k, n, g in CALLS)
    ws = torch.empty(most, dtype=torch.uint8, device="cuda")
    maps = []
    for i, (m, k, n, g) in enumerate(CALLS):
        w = [(_normal((k, n), 50 + i + j) * k ** -0.5).bfloat16().cuda() for j in range(2 if g else 1)]
        r = vb.QRows(m, k)
        qc.put(r, _normal((m, k), 60 + i))
        both = [vb.QLinear(k, n, m, vb.VVS_BF16, gated=g), vb.QLinear(k, n, m, vb.VVS_BF16, gated=g, workspace=ws)]
        for lin in both:
            lin.vvs_qlinear_load(*w)
        maps.append((r, both, m, n, g))

    def call(lin, r, m, n, g):
        if g:
            y = vb.QRows(m, n)
            lin.vvs_qlinear_gate(r, y)
            return torch.cat([y.values.view(torch.uint8).flatten(), y.powers.flatten()])
        y = torch.empty((m, n), device="cuda")
        lin.vvs_qlinear_apply(r, y)
        return y

    own = [call(both[0], r, m, n, g) for r, both, m, n, g in maps]
    for _ in range(3):
        got = [call(both[1], r, m, n, g) for r, both, m, n, g in maps]
        for a, b in zip(own, got):
            assert torch.equal(a, b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [call(both[1], r, m, n, g) for r, both, m, n, g in maps]
    torch.cuda.synchronize()
    for a, b in zip(own, got):
        assert torch.equal(a, b)
    with pytest.raises(ValueError):
        vb.QLinear(1280, 700, 30, vb.VVS_BF16, gated=True, workspace=ws[:1000])


def test_maps_of_different_sizes_share_a_workspace():
    """The sums of one map (a contraction in halves, 64 rows of hidden units) do not lie where the counters of a much wider one are."""
    from paper_2511_13587_amd import binding as vb
    calls = [(28, 5200, 2100, False), (14, 300, 20000, True), (20, 5200, 4000, False), (48, 300, 900, True), (32, 300, 20000, True)]
    ws = torch.empty(max(vb.vvs_qlinear_query_sizes(vb.VvsQLinearConfig(k, n, m, int(g), vb.VVS_BF16))[1] for m, k, n, g in calls), dtype=torch.uint8, device="cuda")
    maps = []
    for i, (m, k, n, g) in enumerate(calls):
        w = [(_normal((k, n), 70 + i + j) * k ** -0.5).bfloat16().cuda() for j in range(2 if g else 1)]
        r = vb.QRows(m, k)
        qc.put(r, _normal((m, k), 80 + i))
        both = [vb.QLinear(k, n, m, vb.VVS_BF16, gated=g), vb.QLinear(k, n, m, vb.VVS_BF16, gated=g, workspace=ws)]
        outs = []
        for lin in both:
            lin.vvs_qlinear_load(*w)
            outs.append(vb.QRows(m, n) if g else torch.empty((m, n), device="cuda"))
        maps.append((r, both, outs, g))
    for _ in range(3):
        for r, both, outs, g in maps:
            for lin, y in zip(both, outs):
                for t in (y.values, y.powers) if g else (y,):
                    t.view(torch.uint8).fill_(255)
                lin.vvs_qlinear_gate(r, y) if g else lin.vvs_qlinear_apply(r, y)
        for _, _, (a, b), g in maps:
            if g:
                assert torch.equal(a.values.view(torch.uint8), b.values.view(torch.uint8)) and torch.equal(a.powers, b.powers)
            else:
                assert torch.equal(a, b) and torch.isfinite(a).all()


def test_two_maps_with_workspaces_of_their_own_run_at_once():
    """On two streams, again and again: the same bits."""
    from paper_2511_13587_amd import binding as vb
    pairs = []
    for i, (m, k, n, g) in enumerate([(28, 8300, 300, False), (14, 1280, 700, True)]):
        lin, r, _, _ = _linear(vb, m, k, n, gated=g, seed=70 + i)
        pairs.append((lin, r, vb.QRows(m, n) if g else torch.empty((m, n), device="cuda")))

    def both(streams):
        for _ in range(20):
            for (lin, r, y), s in zip(pairs, streams):
                with torch.cuda.stream(s):
                    lin.vvs_qlinear_gate(r, y) if isinstance(y, vb.QRows) else lin.vvs_qlinear_apply(r, y)
        torch.cuda.synchronize()
        return pairs[0][2].clone(), pairs[1][2].values.view(torch.uint8).clone(), pairs[1][2].powers.clone()

    here = torch.cuda.current_stream()
    torch.cuda.synchronize()
    want = both([here, here])
    got = both([torch.cuda.Stream(), torch.cuda.Stream()])
    assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("rows,most", [(3, 9), (17, 40), (33, 40), (70, 90), (300, 320)])
def test_rows_behind_the_last_one_stay(rows, most):
    from paper_2511_13587_amd import binding as vb
    for gated in (False, True):
        lin, r, x, w = _linear(vb, most, 500, 300, gated=gated, seed=rows)
        part = r.first(rows)
        if gated:
            y = vb.QRows(most, 300)
            y.values.view(torch.uint8).fill_(0x33)
            y.powers.fill_(77)
            lin.vvs_qlinear_gate(part, y.first(rows))
            check_gate(y.first(rows), x[:rows], w, fast=rows > 64)
            assert (y.values.view(torch.uint8)[rows:] == 0x33).all() and (y.powers[rows:] == 77).all()
        else:
            for dtype, stride, lead in ((torch.float32, 300, 0), (torch.bfloat16, 301, 1), (torch.bfloat16, 512, 8), (torch.float32, 333, 2)):
                flat = torch.full((most * stride + lead + 8,), 5.0, dtype=dtype, device="cuda")
                y = flat[lead:].as_strided((rows, 300), (stride, 1))
                lin.vvs_qlinear_apply(part, y)
                check_product(y, x[:rows], w[0], dtype, fast=rows > 64 and dtype == torch.bfloat16)
                mine = torch.zeros(flat.shape, dtype=torch.bool, device="cuda")
                mine[lead:].as_strided((rows, 300), (stride, 1)).fill_(True)
                assert (flat[~mine] == 5.0).all()


# outputs that are part of a wider tensor, at multiples of 16 bytes, of 4 elements, of one: the same bits as beside each other, and nothing written around them
@pytest.mark.parametrize("rows,width,out", [(9, 700, 300), (50, 3300, 17000), (70, 1000, 700), (200, 3300, 1000), (300, 2100, 4160), (330, 5300, 4200), (700, 300, 2300), (1100, 640, 3900)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_outputs_inside_a_wider_tensor(rows, width, out, dtype):
    from paper_2511_13587_amd import binding as vb
    lin, r, _, _ = _linear(vb, rows, width, out, seed=rows)
    want = torch.full((rows, out), 3.0, dtype=dtype, device="cuda")
    lin.vvs_qlinear_apply(r, want)
    for at, wider in ((0, 64), (8, 72 + -out % 8), (4, 12 + -out % 4), (1, 3), (3, 5 - out % 2)):
        whole = torch.full((rows + 3, out + at + wider), 3.0, dtype=dtype, device="cuda")
        lin.vvs_qlinear_apply(r, whole[1:rows + 1, at:at + out])
        assert torch.equal(whole[1:rows + 1, at:at + out], want)
        whole[1:rows + 1, at:at + out] = 3.0
        assert (whole == 3.0).all()


@pytest.mark.parametrize("rows,width,out", [(5, 300, 200), (70, 300, 200), (70, 300, 40000)])
def test_rows_further_apart_than_four_billion_elements(rows, width, out):
    """Offsets behind 2^32 elements, of what is rounded, normalised and written."""
    from paper_2511_13587_amd import binding as vb
    stride = 2 ** 32 // (rows - 1) // 8 * 8 + 8 * 4096
    lin, r, x, _ = _linear(vb, rows, width, out, seed=rows)
    want = torch.empty((rows, out), dtype=torch.bfloat16, device="cuda")
    lin.vvs_qlinear_apply(r, want)
    far = torch.empty((rows - 1) * stride + max(out, width), dtype=torch.bfloat16, device="cuda")
    y = far.as_strided((rows, out), (stride, 1))
    lin.vvs_qlinear_apply(r, y)
    assert torch.equal(y, want)
    near, at_far = vb.QRows(rows, width), vb.QRows(rows, width)
    x = _normal((rows, width), 5).bfloat16().cuda()
    far_x = far.as_strided((rows, width), (stride, 1))
    far_x.copy_(x)
    vb.vvs_qrows_round(x, near)
    vb.vvs_qrows_round(far_x, at_far)
    assert torch.equal(near.values.view(torch.uint8), at_far.values.view(torch.uint8)) and torch.equal(near.powers, at_far.powers)
    gain = torch.ones(width, device="cuda")
    x2 = torch.empty_like(x)
    vb.vvs_qrows_norm(x, gain, 1e-5, near, delta=x, x_out=x2)
    vb.vvs_qrows_norm(far_x, gain, 1e-5, at_far, delta=x, x_out=far_x)
    assert torch.equal(near.values.view(torch.uint8), at_far.values.view(torch.uint8)) and torch.equal(far_x, x2)
    vb.vvs_qrows_read(near, x2)
    vb.vvs_qrows_read(at_far, far_x)
    assert torch.equal(far_x, x2)


@pytest.mark.parametrize("rows", [5, 100])
def test_weights_of_more_than_four_billion_bytes(rows):
    """65536 x 70000 in 8 bits: 4.6 GB.  The first and last columns beside their products in 64 bits; sums of 65536 products of e4m3 numbers in fp32, of at most 512 blocks in turn behind sums of 32 in the matrix cores:
    an error of 2^-24 sqrt(65536 / 32) = 2.7e-6 in the 2-norm at most where roundings are independent."""
    from paper_2511_13587_amd import binding as vb
    width, out, part = 65536, 70000, 96
    w = torch.empty((width, out), dtype=torch.bfloat16, device="cuda").normal_(0.0, width ** -0.5, generator=torch.Generator("cuda").manual_seed(1))
    lin = vb.QLinear(width, out, rows, vb.VVS_BF16)
    lin.vvs_qlinear_load(w)
    lin.vvs_qlinear_read(w)
    r, x = vb.QRows(rows, width), torch.empty((rows, width), device="cuda")
    vb.vvs_qrows_round(_normal((rows, width), 2, 0).cuda(), r)
    vb.vvs_qrows_read(r, x)
    y = torch.empty((rows, out), device="cuda")
    lin.vvs_qlinear_apply(r, y)
    for cut in (slice(0, part), slice(out - part, out)):
        want = x.cpu().double() @ w[:, cut].cpu().double()
        assert ((y[:, cut].cpu().double() - want).norm() / want.norm()).item() < 2.7e-6


@pytest.mark.parametrize("rows", [5, 40, 100, 500])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_what_is_not_finite_stays_in_its_row_and_column(rows, dtype):
    from paper_2511_13587_amd import binding as vb
    width, out = 300, 260
    w = _normal((width, out), 1)
    w[7, 100], w[250, 3] = float("inf"), float("nan")
    lin = vb.QLinear(width, out, rows, vb.VVS_FP32)
    lin.vvs_qlinear_load(w.cuda())
    x = _normal((rows, width), 2)
    x[4, 299] = float("-inf")
    r = vb.QRows(rows, width)
    vb.vvs_qrows_round(x.cuda(), r)
    y = torch.zeros((rows, out), dtype=dtype, device="cuda")
    lin.vvs_qlinear_apply(r, y)
    nan = torch.isnan(y).cpu()
    want = torch.zeros((rows, out), dtype=torch.bool)
    want[4] = True
    want[:, [3, 100]] = True
    assert torch.equal(nan, want)
    assert torch.isfinite(y.cpu()[~want]).all()


@pytest.mark.parametrize("rows", [5, 40, 500])
def test_what_is_not_finite_in_a_gate(rows):
    """One NaN in the gate's weights: that hidden unit is NaN in every row, the others of its block are rounded as if it were not there."""
    from paper_2511_13587_amd import binding as vb
    width, out = 256, 200
    ws = [_normal((width, out), i) * width ** -0.5 for i in (1, 2)]
    lin = vb.QLinear(width, out, rows, vb.VVS_FP32, gated=True)
    held = [qc.held(w.t())[0].t() for w in ws]
    ws[0][9, 150] = float("nan")
    lin.vvs_qlinear_load(*[w.cuda() for w in ws])
    r = vb.QRows(rows, width)
    x = qc.put(r, _normal((rows, width), 3, 0.3))
    y = vb.QRows(rows, out)
    lin.vvs_qlinear_gate(r, y)
    nan = torch.isnan(qc.values_of(y))
    assert nan[:, 150].all() and not nan[:, torch.arange(out) != 150].any()
    # beside the same map without that unit
    held[0][:, 150] = 0.0
    y.values.view(torch.uint8)[:, 150] = 0
    check_gate(y, x, held, fast=rows > 64)


@pytest.mark.parametrize("rows", [5, 40, 100, 500])
def test_rows_and_weights_of_very_different_size(rows):
    """Powers of two far apart, whose products are ordinary numbers; a row and a column of zeros."""
    from paper_2511_13587_amd import binding as vb
    width, out = 700, 300
    x = _normal((rows, width), 1) * 2.0 ** 90
    x[:, 128:256] *= 2.0 ** -30
    x[2] = 0
    w = _normal((width, out), 2) * 2.0 ** -92
    w[128:256] *= 2.0 ** 28
    w[:, 11] = 0
    lin = vb.QLinear(width, out, rows, vb.VVS_FP32)
    lin.vvs_qlinear_load(w.cuda())
    r = vb.QRows(rows, width)
    xh = qc.put(r, x)
    wh = qc.held(w.t())[0].t()
    for dtype in (torch.float32, torch.bfloat16):
        y = torch.full((rows, out), 9.0, dtype=dtype, device="cuda")
        lin.vvs_qlinear_apply(r, y)
        check_product(y, xh, wh, dtype, fast=rows > 64 and dtype == torch.bfloat16)
        assert (y[2] == 0).all() and (y[:, 11] == 0).all()


def test_products_of_large_and_small_sums():
    """Sums whose terms cancel: e4m3 products are exact in fp32, what few rows and fp32 outputs lose is fp32's."""
    from paper_2511_13587_amd import binding as vb
    width, out = 1024, 64
    x = torch.ones((20, width))
    x[:, 512:] = -1
    w = torch.full((width, out), 448.0)
    w[3, :] = 2.0 ** -9 * 448                     # a small number beside large ones of its block
    lin = vb.QLinear(width, out, 20, vb.VVS_FP32)
    lin.vvs_qlinear_load(w.cuda())
    r = vb.QRows(20, width)
    xh = qc.put(r, x)
    wh = qc.held(w.t())[0].t()
    y = torch.zeros((20, out), device="cuda")
    lin.vvs_qlinear_apply(r, y)
    assert torch.equal(y.cpu().double(), xh @ wh)
    assert (product_error(xh, wh) > 0).all()
