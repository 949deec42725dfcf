"""The gated recurrence's, layer norm's and dropout's host code under AddressSanitizer and
UndefinedBehaviorSanitizer, on the CPU, by tests/asan/abi_host_block_driver.c: as
test_abi_asan.py for the other entry points.  (The sanitizers are on the host side only; no
GPU code is instrumented and nothing is launched.)"""
import os
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from conftest import ROOT
from test_abi_asan import CLANG, CSRC, INC, SAN_HOST, _have_toolchain


@pytest.mark.skipif(not _have_toolchain(), reason="hipcc / ROCm clang not installed")
def test_host_code_is_clean_under_asan_and_ubsan(tmp_path):
    srcs = sorted(f for f in os.listdir(CSRC) if f.endswith(".hip"))

    def compile_one(f):
        cmd = ["hipcc", "-c", "-O1", "-g", "-std=c++17", "--offload-arch=gfx950",
               "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"] + SAN_HOST + \
              ["-I", INC, os.path.join(CSRC, f), "-o", str(tmp_path / (f + ".o"))]
        return subprocess.run(cmd, capture_output=True, text=True)

    with ThreadPoolExecutor(max_workers=min(8, len(srcs))) as ex:
        for res in ex.map(compile_one, srcs):
            assert res.returncode == 0, res.stderr[-2000:]
    drv_o, exe = str(tmp_path / "driver.o"), str(tmp_path / "driver")
    subprocess.run([CLANG, "-O1", "-g", "-fsanitize=address,undefined", "-fno-omit-frame-pointer", "-I", INC,
                    "-c", os.path.join(ROOT, "tests", "asan", "abi_host_block_driver.c"), "-o", drv_o], check=True)
    subprocess.run([CLANG + "++", "--hip-link", "--offload-arch=gfx950", "-fsanitize=address,undefined", "-o", exe, drv_o]
                   + [str(tmp_path / (f + ".o")) for f in srcs]
                   + ["-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib"], check=True)
    env = dict(os.environ, UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1", ASAN_OPTIONS="detect_leaks=1")
    res = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=120)
    assert res.returncode == 0, res.stdout + res.stderr[-3000:]
    assert "runtime error" not in res.stderr and "AddressSanitizer" not in res.stderr, res.stderr[-3000:]
    assert "validation done" in res.stdout
