"""What pda_decode_fp8 hands to its kernels, for seeded random descriptors up to the
largest, with launchers that check it against the plan's workspace (no GPU)."""
import os

import pytest

from test_fp8_sanitizers import CSRC, INCLUDE
from test_sanitizers import HIPCC, SAN, build_and_run


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc is not installed")
def test_launch_arguments_under_sanitizer(tmp_path):
    exe = str(tmp_path / "fp8_carving_sanitize")
    # each sanitizer flag applies to the host pass alone; no device code runs
    cmd = [HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17",
           "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=all", "-I", INCLUDE, "-I", CSRC,
           os.path.join(CSRC, "pda_api.hip"), os.path.join(CSRC, "pda_fp8_api.hip"),
           "-x", "hip", os.path.join(SAN, "fp8_carving_sanitize.cpp"), "-o", exe]
    build_and_run(cmd, exe, {"ASAN_OPTIONS": "detect_leaks=0"})
