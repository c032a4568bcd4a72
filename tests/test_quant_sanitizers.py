"""The host side of the operators of quantised inference (argument checks and launch plans) built with g++ under
AddressSanitizer and UndefinedBehaviorSanitizer, the launchers replaced by stand-ins that check what reaches them
(tests/host_sanitize/quant_driver.cpp).  CPU only."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HERE = os.path.join(ROOT, "tests", "host_sanitize")
CSRC = os.path.join(ROOT, "paper_2609_24519_amd", "csrc")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


def test_quantised_inference_host_side(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None or not os.path.exists(os.path.join(ROCM, "include", "hip", "hip_runtime.h")):
        pytest.skip("needs g++ and the HIP headers")
    exe = str(tmp_path / "quant_driver")
    cmd = [gxx, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROCM, "include"), "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           os.path.join(CSRC, "awe_tables.cpp"), os.path.join(CSRC, "awe_api.cpp"), os.path.join(CSRC, "awe_quant_api.cpp"),
           os.path.join(HERE, "launch_stubs.cpp"), os.path.join(HERE, "quant_driver.cpp"),
           "-L", os.path.join(ROCM, "lib"), "-lamdhip64", "-Wl,-rpath," + os.path.join(ROCM, "lib"), "-lpthread", "-o", exe]
    b = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=600)
    if b.returncode != 0 and ("asan" in b.stdout or "ubsan" in b.stdout):
        pytest.skip("sanitizer runtime not available: " + b.stdout[-300:])
    assert b.returncode == 0, b.stdout[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=600, env=env)
    assert r.returncode == 0, r.stdout[-3000:]
    last = r.stdout.strip().splitlines()[-1].split()
    assert last[0] == "calls" and int(last[3]) > 1000 and last[-2:] == ["failures", "0"], last
