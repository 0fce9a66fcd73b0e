"""The extents that the scaled operators take, on the CPU: the C ABI's host
code built by g++ with its launchers replaced by stubs that count."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2602_04870_amd", "csrc")
SAN = ["-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all"]


def test_extents_on_both_sides_of_each_limit(tmp_path):
    """What the header takes is launched, and one tile or block more is
    refused, also where the limit is no multiple of the other extent."""
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    body = ['#include "scaled_launch.hpp"', "int g_launches = 0;", "namespace mhl {"]
    for header in ("launch.hpp", "scaled_launch.hpp"):
        text = open(os.path.join(CSRC, header)).read()
        for name, params in re.findall(r"^hipError_t\s+(\w+)\(([^;{]*)\);", text, flags=re.M):
            body.append(f"hipError_t {name}({params}) {{ ++g_launches; return hipSuccess; }}")
    stubs = tmp_path / "stubs.cpp"
    stubs.write_text("\n".join(body + ["}"]) + "\n")
    exe = str(tmp_path / "scaled_limits_check")
    cmd = [gxx, "-std=c++17", *SAN, "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
           f"-I{ROOT}/include", f"-I{CSRC}", "-Wno-unused-result", "-Wno-unused-value",
           "-Wno-attributes", os.path.join(CSRC, "api.cpp"), os.path.join(CSRC, "api_scaled.cpp"),
           str(stubs), os.path.join(ROOT, "tests", "scaled_limits_check.cpp"), "-L/opt/rocm/lib",
           "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib", "-o", exe]
    res = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert res.returncode == 0, res.stderr[-4000:]
    env = {k: v for k, v in os.environ.items() if k != "MHLMOE_DEBUG"}
    res = subprocess.run([exe], capture_output=True, text=True, timeout=300,
                         env=dict(env, ASAN_OPTIONS="detect_leaks=0",
                                  UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1"))
    out = res.stdout + res.stderr
    assert res.returncode == 0 and "done 0 failures" in res.stdout, out[-4000:]
    assert "runtime error" not in out, out[-4000:]
    taken, refused = map(int, re.search(r"(\d+) taken, (\d+) refused", res.stdout).groups())
    assert taken > 100 and refused > 50
