"""The 8-bit cache's host layer under AddressSanitizer and UndefinedBehaviorSanitizer,
and its header as C and as C++ (no GPU)."""
import os
import shutil
import subprocess

import pytest

from test_sanitizers import HIPCC, ROOT, SAN, build_and_run

CSRC = os.path.join(ROOT, "paper_2405_11143_amd", "csrc")
INCLUDE = os.path.join(ROOT, "include")


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc is not installed")
def test_fp8_host_layer_under_sanitizer(tmp_path):
    exe = str(tmp_path / "fp8_api_sanitize")
    # each sanitizer flag applies to the host pass alone; no device code runs
    cmd = [HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17",
           "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=all", "-I", INCLUDE, "-I", CSRC,
           os.path.join(CSRC, "pda_api.hip"), os.path.join(CSRC, "pda_fp8_api.hip"),
           "-x", "hip", os.path.join(SAN, "fp8_api_sanitize.cpp"), "-o", exe]
    build_and_run(cmd, exe, {"ASAN_OPTIONS": "detect_leaks=0"})


@pytest.mark.skipif(shutil.which("gcc") is None, reason="gcc is not installed")
@pytest.mark.parametrize("compiler,std", [("gcc", "c11"), ("g++", "c++17")])
def test_header_stands_alone(tmp_path, compiler, std):
    src = tmp_path / ("x.c" if compiler == "gcc" else "x.cpp")
    src.write_text('#include "pda_fp8.h"\nint main(void) { pda_rotary r; pda_rotary_scaling s; (void)r; (void)s; return '
                   'PDA_ROTARY_RAMP == 4 ? 0 : 1; }\n')
    subprocess.run([compiler, f"-std={std}", "-Wall", "-Wextra", "-Werror", "-D__HIP_PLATFORM_AMD__", "-I", INCLUDE,
                    "-I", "/opt/rocm/include", "-fsyntax-only", str(src)], check=True)
