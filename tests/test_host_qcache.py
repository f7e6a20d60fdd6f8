"""Host side of the 8-bit key/value cache and the rotary operator under the sanitizers on the CPU (tests/host_qcache.cpp), and the binding's checks that need no GPU."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_host_side_is_clean_under_sanitizers(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime.h"):
        pytest.skip("needs g++ and the HIP headers")
    exe, csrc = str(tmp_path / "host_qcache"), os.path.join(ROOT, "paper_2511_13587_amd", "csrc")
    cmd = [gxx, "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I", csrc, "-I", os.path.join(ROOT, "tests"),
           "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-static-libasan", "-g", "-O1", "-w", "-pthread",
           os.path.join(csrc, "vvs_host.cpp"), os.path.join(csrc, "vvs_qcache_host.cpp"), os.path.join(ROOT, "tests", "host_qcache.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    if r.returncode != 0 and "san" in r.stderr.lower() and "cannot find" in r.stderr.lower():
        pytest.skip("the sanitizer runtime is not installed")
    assert r.returncode == 0, r.stderr[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="verify_asan_link_order=0:detect_leaks=1", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300, env=env)
    assert r.returncode == 0 and "host qcache ok" in r.stdout, (r.stdout[-2000:], r.stderr[-3000:])


def test_binding_refuses_what_the_library_refuses():
    from paper_2511_13587_amd import binding as vb
    with pytest.raises(vb.VvsError) as e:
        vb.QCache(1, 1, 4, 3, 64, 64, 1, vb.VVS_BF16)
    assert e.value.status == vb.VVS_EINVAL and "n_kv_heads" in str(e.value)
    with pytest.raises(vb.VvsError) as e:
        vb.QCache(1, 1, 4, 2, 96, 64, 1, vb.VVS_BF16)
    assert e.value.status == vb.VVS_ESIZE
    for size, pairs, status in ((64, [33], vb.VVS_EINVAL), (64, [], vb.VVS_ESIZE), (64, [4] * 5, vb.VVS_ESIZE), (60, [4], vb.VVS_ESIZE)):
        with pytest.raises(vb.VvsError) as e:
            vb.Rope(size, pairs, 10000.0, vb.VVS_BF16)
        assert e.value.status == status
    rope = vb.Rope(64, [16, 16], 10000.0, vb.VVS_BF16)
    rope.close()
    rope.close()


def test_cache_takes_half_of_bf16_and_a_quarter_of_fp32():
    from paper_2511_13587_amd import binding as vb
    cfg = vb.VvsQCacheConfig(36, 16, 20, 20, 64, 696, 27, vb.VVS_BF16)
    cache, _ = vb.vvs_qcache_query_sizes(cfg)
    slots = 36 * 16 * 20 * 704
    assert slots * 2 * 64 <= cache <= slots * 2 * 64 * 1.01


def test_per_token_strides():
    import torch
    from paper_2511_13587_amd import binding as vb
    wide = torch.zeros((2, 3, 8, 64), dtype=torch.bfloat16)
    cpu = wide.get_device()
    ok = [(wide[:, :, 2:4], (2, 3, 2, 64), 512), (wide, (2, 3, 8, 64), 512), (wide[:, :1, :2], (2, 1, 2, 64), 1536), (wide[:1, :1, :2], (1, 1, 2, 64), 128),
          (wide[:, :, :1], (2, 3, 1, 64), 512)]
    for t, shape, stride in ok:
        assert vb._per_token(t, cpu, torch.bfloat16, shape, "x") == (t.data_ptr(), stride)
    for t in (wide[:, :, ::2], wide[:, ::2], wide[:, :, :, ::2], wide.transpose(1, 2), wide[:, :2], wide[:, :1].expand(2, 3, 8, 64)):
        with pytest.raises(ValueError):
            vb._per_token(t, cpu, torch.bfloat16, tuple(t.shape), "x")


def test_context_with_the_cache_in_8_bits_takes_half_of_it():
    from paper_2511_13587_amd import binding as vb
    from paper_2511_13587_amd import synth
    same, _, _ = vb.vvs_query_sizes(vb.make_config(synth.SEVEN_B))
    held8, _, _ = vb.vvs_query_sizes(vb.make_config(synth.SEVEN_B, cache_kind=vb.VVS_CACHE_E4M3))
    assert 0.5 * same <= held8 <= 0.54 * same                 # weights and positions are 8 bytes per slot of 256
    for shape, kw, status in ((synth.XL_TREE, dict(cache_kind=-1), vb.VVS_EINVAL), (synth.XL_TREE, dict(cache_kind=1, draft_input=1), vb.VVS_EINVAL),
                              (synth.TINY.replace(n_heads=8), dict(cache_kind=1), vb.VVS_ESIZE), (synth.TINY.replace(n_heads=8), dict(), vb.VVS_OK)):
        cfg = vb.make_config(shape, **kw)
        try:
            vb.vvs_query_sizes(cfg)
            got = vb.VVS_OK
        except vb.VvsError as e:
            got = e.status
        assert got == status
