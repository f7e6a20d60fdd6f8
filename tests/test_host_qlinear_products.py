"""How a linear map's products are summed: which kernel a call takes by its config (tests/host_qlinear_products.cpp), and what is refused."""
import os
import shutil
import subprocess

import pytest

from qlinear_variants import TILES, VARIANTS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_calls_take_the_kernel_of_their_config(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime.h"):
        pytest.skip("needs g++ and the HIP headers")
    exe, csrc = str(tmp_path / "host_qlinear_products"), os.path.join(ROOT, "paper_2511_13587_amd", "csrc")
    cmd = [gxx, "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I", csrc, "-O1", "-w",
           os.path.join(csrc, "vvs_qlinear_host.cpp"), os.path.join(ROOT, "tests", "host_qlinear_products.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-3000:]
    args = []
    for rows, width, out, gated, products, dtype, fast, tile, shares in VARIANTS:
        args += [rows, width, out, gated, products, 1 if dtype == "bf16" else 0, fast, TILES.index(tile), shares]
    r = subprocess.run([exe, *map(str, args)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and f"ok, {len(VARIANTS)} launches" in r.stdout, (r.stdout, r.stderr)


def test_every_tile_is_among_them():
    """With e4m3 instructions and without, with and without a gate: each tile in each number of shares that a call takes."""
    have = {(gated, fast, tile, shares) for _, _, _, gated, _, _, fast, tile, shares in VARIANTS}
    want = {(0, 1, t, s) for t, s in (("128x256", 1), ("64x256", 1), ("64x128", 1), ("64x128", 2), ("64x128", 4), ("32x128", 1), ("32x128", 2), ("32x128", 4))}
    want |= {(0, 0, t, s) for t, s in (("128x256", 1), ("64x256", 1), ("64x128", 1), ("64x128", 2), ("32x128", 1), ("32x128", 2), ("32x128", 4))}
    want |= {(1, f, t, 1) for f in (0, 1) for t in ("128x256", "64x256")} | {(1, 0, "32x256", 1)}
    assert want <= have


def test_config_of_the_binding():
    from paper_2511_13587_amd import binding as vb
    from paper_2511_13587_amd import synth
    for products in (vb.VVS_PRODUCTS_AUTO, vb.VVS_PRODUCTS_WHOLE, vb.VVS_PRODUCTS_E4M3):
        assert vb.vvs_qlinear_query_sizes(vb.VvsQLinearConfig(300, 200, 70, 0, vb.VVS_BF16, products)) == vb.vvs_qlinear_query_sizes(vb.VvsQLinearConfig(300, 200, 70, 0, vb.VVS_BF16))
    for products in (-1, 3):
        with pytest.raises(vb.VvsError) as e:
            vb.QLinear(300, 200, 70, vb.VVS_BF16, products=products)
        assert e.value.status == vb.VVS_EINVAL and "products" in str(e.value)
    sizes = [vb.vvs_query_sizes(vb.make_config(synth.XL_TREE, weight_kind=k)) for k in (vb.VVS_WEIGHTS_E4M3, vb.VVS_WEIGHTS_E4M3_WHOLE)]
    assert sizes[0] == sizes[1]
    for kw in (dict(weight_kind=3, draft_input=1), dict(weight_kind=4)):
        with pytest.raises(vb.VvsError) as e:
            vb.vvs_query_sizes(vb.make_config(synth.XL_TREE, **kw))
        assert e.value.status == vb.VVS_EINVAL
