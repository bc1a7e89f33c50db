"""Rows between the projection and the attention as they are built: reservations and refusals under AddressSanitizer and
UndefinedBehaviorSanitizer (host pass only; no device call is made), and what the compiler makes of the kernels."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_rows_host_paths_under_asan_and_ubsan(tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("no hipcc here")
    exe = str(tmp_path / "tl_rows_sanitize")
    csrc = os.path.join(ROOT, "paper_2508_17219_amd", "csrc")
    srcs = [os.path.join(csrc, s) for s in ("pool.hip", "prefix_tree.hip", "rows.hip")]
    cmd = [hipcc, "-O1", "-g", "-std=c++17", "--offload-arch=gfx950",
           "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=undefined",
           "-I", os.path.join(ROOT, "include"), "-I", csrc,
           os.path.join(ROOT, "tests", "host_sanitize", "rows_driver.cpp")] + srcs + ["-o", exe]
    build = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert build.returncode == 0, build.stdout[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    run = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=env, timeout=300)
    assert run.returncode == 0, run.stdout[-3000:]
    assert "all statuses as expected" in run.stdout and "runtime error" not in run.stdout, run.stdout[-3000:]


def test_rows_kernels_keep_everything_in_registers():
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("no hipcc here")
    csrc = os.path.join(ROOT, "paper_2508_17219_amd", "csrc")
    cmd = [hipcc, "-O3", "-std=c++17", "--offload-arch=gfx950", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-I", os.path.join(ROOT, "include"),
           "-I", csrc, "--cuda-device-only", "-c", os.path.join(csrc, "rows.hip"), "-o", os.devnull, "-Rpass-analysis=kernel-resource-usage"]
    text = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, check=True).stdout
    kernels = re.findall(r"Function Name: (\S+).*?VGPRs: (\d+).*?ScratchSize \[bytes/lane\]: (\d+)", text, re.S)
    assert len(kernels) == 30, kernels        # dense and to the pool: 2 types x 2 orders x 3 ways by the cache; moves: 2 x 3
    for name, registers, scratch in kernels:
        assert int(scratch) == 0 and int(registers) <= 64, (name, registers, scratch)        # 64: eight waves to a SIMD


def test_every_head_is_dealt_to_one_wave_and_every_launch_takes_tokens(tmp_path):
    """The dealing that the library launches by and the kernel finds its place by, over head counts up to the most that a call may have."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("no hipcc here")
    exe = str(tmp_path / "tl_rows_deal")
    cmd = [hipcc, "-O1", "-g", "-std=c++17", "--offload-arch=gfx950", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=undefined",
           "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2508_17219_amd", "csrc"),
           os.path.join(ROOT, "tests", "host_sanitize", "deal_driver.cpp"), "-o", exe]
    build = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert build.returncode == 0, build.stdout[-3000:]
    run = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=100)
    assert run.returncode == 0, run.stdout[-3000:]
    assert "every head dealt once" in run.stdout and "runtime error" not in run.stdout, run.stdout[-3000:]


def test_host_memory_that_runs_out_registers_nothing(tmp_path):
    """tl_pool_adopt, tl_pool_reserve_batch, tl_pool_put, tl_pool_evict_lru and the prefix tree where an allocation fails: TL_ENOMEM, no exception, the pool as it was."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("no hipcc here")
    exe = str(tmp_path / "tl_memory")
    csrc = os.path.join(ROOT, "paper_2508_17219_amd", "csrc")
    cmd = [hipcc, "-O1", "-g", "-std=c++17", "--offload-arch=gfx950", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=undefined", "-I", os.path.join(ROOT, "include"), "-I", csrc,
           os.path.join(ROOT, "tests", "host_sanitize", "memory_driver.cpp"), os.path.join(csrc, "pool.hip"), os.path.join(csrc, "prefix_tree.hip"), "-o", exe]
    build = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert build.returncode == 0, build.stdout[-3000:]
    run = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=100)
    assert run.returncode == 0, run.stdout[-3000:]
    assert "nothing registered" in run.stdout, run.stdout[-3000:]
