"""CPU build with AddressSanitizer and UndefinedBehaviorSanitizer of the
feed-forward block's C-ABI layer (cci_block_api.cpp linked against launcher
stand-ins, so no GPU is involved)."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
SAN = ["-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer", "-g", "-O1"]


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir("/opt/rocm/include"), reason="needs g++ and HIP headers")
def test_block_host_layer_under_sanitizers(tmp_path):
    exe = str(tmp_path / "block_driver")
    src = [os.path.join(ROOT, "paper_1910_11971_amd", "csrc", "cci_block_api.cpp"),
           os.path.join(HERE, "sanitize", "block_stubs.cpp"), os.path.join(HERE, "sanitize", "block_driver.cpp")]
    r = subprocess.run(["g++", *SAN, "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I", "/opt/rocm/include", "-I",
                        os.path.join(ROOT, "include"), *src, "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib",
                        "-o", exe], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, timeout=600, env=env)
    assert r.returncode == 0 and "block driver ok" in r.stdout, r.stdout + r.stderr
