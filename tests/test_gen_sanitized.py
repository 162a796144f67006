"""The host C++ of the generation tables built with AddressSanitizer and
UndefinedBehaviorSanitizer (host code only, g++), running the CPU tests of
generation in a child process.  The sanitized library links the host sources,
compiled here, with the HIP objects that the regular build left in _build
(their device code is not instrumented and never runs here)."""
import os
import shutil
import subprocess
import sys

import pytest

from tests.test_planner_sanitized import HIP_OBJECTS, HOST_SOURCES, PKG, ROOT, _runtime


def test_generation_tables_under_asan_and_ubsan(tmp_path):
    hip_objs = [os.path.join(PKG, "_build", o) for o in HIP_OBJECTS + ("gen.hip.o", "step.hip.o")]
    if shutil.which("g++") is None or not all(os.path.exists(o) for o in hip_objs):
        pytest.skip("needs g++ and the regular build's HIP objects")
    asan, ubsan = _runtime("libasan.so"), _runtime("libubsan.so")
    if not asan or not ubsan:
        pytest.skip("sanitizer runtimes not found")
    san = ["-fsanitize=address,undefined", "-fno-sanitize-recover=all"]
    objs = []
    for src in HOST_SOURCES + ("gen_plan.cpp",):
        objs.append(str(tmp_path / (src + ".o")))
        subprocess.run(["g++", "-O1", "-g", "-fno-omit-frame-pointer", "-std=c++17", "-fPIC"] + san +
                       ["-I", os.path.join(ROOT, "include"), "-I", os.path.join(PKG, "csrc"), "-c",
                        os.path.join(PKG, "csrc", src), "-o", objs[-1]], check=True)
    lib = str(tmp_path / "libharts_san.so")
    subprocess.run(["g++", "-shared"] + san + objs + hip_objs +
                   ["-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib", "-o", lib], check=True)
    env = dict(os.environ, HARTS_LIB=lib, LD_PRELOAD=f"{asan}:{ubsan}", ASAN_OPTIONS="detect_leaks=0:abort_on_error=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    code = ("import sys, pytest\n"
            "sys.exit(pytest.main(['-q', '-x', '-p', 'no:cacheprovider', 'tests/test_gen_tables.py']))\n")
    res = subprocess.run([sys.executable, "-c", code], cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    out = res.stdout + res.stderr
    assert res.returncode == 0, out[-3000:]
    assert "AddressSanitizer" not in out and "runtime error" not in out and " passed" in out
