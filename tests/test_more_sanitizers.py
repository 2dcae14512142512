"""The host layers of the head norms, the windowed attention and the block tables under
AddressSanitizer and UndefinedBehaviorSanitizer, with the list of blocks that a window's rows see
against a search token by token; and their headers as C and as C++ (no GPU)."""
import os
import shutil
import subprocess

import pytest

from test_sanitizers import HIPCC, ROOT, SAN, build_and_run

CSRC = os.path.join(ROOT, "paper_2405_11143_amd", "csrc")
INCLUDE = os.path.join(ROOT, "include")


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc is not installed")
def test_host_layers_under_sanitizer(tmp_path):
    exe = str(tmp_path / "more_api_sanitize")
    # each sanitizer flag applies to the host pass alone; no device code runs
    cmd = [HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17",
           "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=all", "-I", INCLUDE, "-I", CSRC,
           *(os.path.join(CSRC, f) for f in ("pda_api.hip", "pda_norm_rotary_api.hip", "pda_window_api.hip", "pda_blocks_api.hip")),
           "-x", "hip", os.path.join(SAN, "more_api_sanitize.cpp"), "-o", exe]
    build_and_run(cmd, exe, {"ASAN_OPTIONS": "detect_leaks=0"})


@pytest.mark.skipif(shutil.which("gcc") is None, reason="gcc is not installed")
@pytest.mark.parametrize("header", ["pda_norm_rotary.h", "pda_window.h", "pda_blocks.h"])
@pytest.mark.parametrize("compiler,std", [("gcc", "c11"), ("g++", "c++17")])
def test_header_stands_alone(tmp_path, compiler, std, header):
    src = tmp_path / ("x.c" if compiler == "gcc" else "x.cpp")
    src.write_text(f'#include "{header}"\nint main(void) {{ return PDA_OK; }}\n')
    subprocess.run([compiler, f"-std={std}", "-Wall", "-Wextra", "-Werror", "-D__HIP_PLATFORM_AMD__", "-I", INCLUDE,
                    "-I", "/opt/rocm/include", "-fsyntax-only", str(src)], check=True)
