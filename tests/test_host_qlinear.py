"""Host side of the rows and weights in 8 bits under the sanitizers on the CPU (tests/host_qlinear.cpp), and the binding's checks that need no GPU."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_host_side_is_clean_under_sanitizers(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime.h"):
        pytest.skip("needs g++ and the HIP headers")
    exe, csrc = str(tmp_path / "host_qlinear"), os.path.join(ROOT, "paper_2511_13587_amd", "csrc")
    cmd = [gxx, "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I", csrc,
           "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-static-libasan", "-g", "-O1", "-w", "-pthread",
           os.path.join(csrc, "vvs_qlinear_host.cpp"), os.path.join(ROOT, "tests", "host_qlinear.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    if r.returncode != 0 and "san" in r.stderr.lower() and "cannot find" in r.stderr.lower():
        pytest.skip("the sanitizer runtime is not installed")
    assert r.returncode == 0, r.stderr[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="verify_asan_link_order=0:detect_leaks=1", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300, env=env)
    assert r.returncode == 0 and "host qlinear ok" in r.stdout, (r.stdout[-2000:], r.stderr[-3000:])


def test_binding_refuses_what_the_library_refuses():
    from paper_2511_13587_amd import binding as vb
    for args, status in (((0, 4, 1), vb.VVS_EINVAL), ((4, 0, 1), vb.VVS_EINVAL), ((4, 4, 0), vb.VVS_EINVAL), ((65537, 4, 1), vb.VVS_ESIZE), ((4, 4, 1 << 21), vb.VVS_ESIZE)):
        with pytest.raises(vb.VvsError) as e:
            vb.QLinear(*args, vb.VVS_BF16)
        assert e.value.status == status and "qlinear" in str(e.value)
    for n, width, status in ((0, 8, vb.VVS_EINVAL), (8, 0, vb.VVS_EINVAL), (8, 70000, vb.VVS_ESIZE)):
        with pytest.raises(vb.VvsError) as e:
            vb.QRows(n, width)
        assert e.value.status == status and "qrows" in str(e.value)


def test_sizes():
    from paper_2511_13587_amd import binding as vb
    assert vb.vvs_qrows_sizes(4096, 3) == (3 * 4096, 3 * 32)
    assert vb.vvs_qrows_sizes(1, 1) == (128, 4)
    weights, ws = vb.vvs_qlinear_query_sizes(vb.VvsQLinearConfig(4096, 11008, 64, 1, vb.VVS_BF16))
    assert 2 * 4096 * 11008 <= weights <= 2 * 4096 * 11008 * 1.01 and ws < 2 << 20      # half of bf16


def test_contexts_with_weights_in_8_bits():
    """Half of the layers' bytes; refused where it does not go."""
    from paper_2511_13587_amd import binding as vb
    from paper_2511_13587_amd import synth
    _, _, same = vb.vvs_query_sizes(vb.make_config(synth.SEVEN_B))
    _, _, held8 = vb.vvs_query_sizes(vb.make_config(synth.SEVEN_B, weight_kind=vb.VVS_WEIGHTS_E4M3))
    layers = 32 * (4 * 4096 ** 2 + 3 * 4096 * 11008)
    assert layers * 0.98 <= same - held8 <= layers
    for shape, kw, status in ((synth.XL_TREE, dict(weight_kind=2), vb.VVS_EINVAL), (synth.XL_TREE, dict(weight_kind=-1), vb.VVS_EINVAL), (synth.XL_TREE, dict(weight_kind=1, draft_input=1), vb.VVS_EINVAL),
                              (synth.TINY.replace(d_model=72, n_heads=2), dict(weight_kind=1), vb.VVS_ESIZE), (synth.TINY.replace(d_model=72, n_heads=2), dict(), vb.VVS_OK),
                              (synth.TINY.replace(d_ff=65544), dict(weight_kind=1), vb.VVS_ESIZE), (synth.TINY, dict(weight_kind=1, cache_kind=1), vb.VVS_OK)):
        try:
            vb.vvs_query_sizes(vb.make_config(shape, **kw))
            got = vb.VVS_OK
        except vb.VvsError as e:
            got = e.status
        assert got == status, (shape.name, kw)


def test_rows_of_matrices():
    """What the binding takes as rows of a matrix: parts of wider ones, any leading dimensions; not what lies otherwise."""
    import torch
    from paper_2511_13587_amd import binding as vb
    wide = torch.zeros((4, 3, 40))
    cpu = wide.get_device()
    at = wide.data_ptr()
    for t, rows, width, want in ((wide, 12, 40, (at, 40)), (wide[:, :, 8:24], 12, 16, (at + 32, 40)), (wide[:, 1], 4, 40, (at + 160, 120)), (wide[:1, :1, :7], 1, 7, (at, 7)), (wide[0, 0], 1, 40, (at, 40)),
                                 (wide[:, :1, 3:4], 4, 1, (at + 12, 120))):
        assert vb._matrix(t, rows, width, cpu, "x")[:2] == want
    for t, rows, width in ((wide[:, :, ::2], 12, 20), (wide[:, ::2], 8, 40), (wide.transpose(0, 1), 12, 40), (wide[:, :2], 8, 40), (wide[:, :1].expand(4, 3, 40), 12, 40), (wide, 11, 40), (wide, 12, 39),
                           (wide.half(), 12, 40), (wide.double(), 12, 40), (wide[0, 0, 0], 1, 1), (wide.view(-1), 12, 40)):
        with pytest.raises(ValueError):
            vb._matrix(t, rows, width, cpu, "x")
    with pytest.raises(ValueError):
        vb._matrix(wide, 12, 40, 0, "x")


def test_parts_of_rows():
    import torch
    from paper_2511_13587_amd import binding as vb
    r = vb.QRows(5, 200, device="cpu")
    assert r.values.shape == (5, 256) and r.values.dtype == torch.float8_e4m3fn and r.powers.shape == (5, 4)
    p = r.first(3)
    assert (p.n_rows, p.width, p.values.data_ptr(), p.powers.data_ptr()) == (3, 200, r.values.data_ptr(), r.powers.data_ptr())
    for n in (0, 6, -1):
        with pytest.raises(ValueError):
            r.first(n)
