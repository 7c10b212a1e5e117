"""Positions of the divisions over 4-bit codes fit 32 bits (tests/host_fp4_guards.cpp), also where a tile or a request is made to count for more: kernels and host share
the constants."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2401_11181_amd", "csrc")
HIP_INCLUDE = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include")
CONSTANTS = {"kFp4TileStages": "tetri_attn.hip", "kFp4RequestSteps": "tetri_decode_fp4.hip", "kPrefillFp4TileSteps": "tetri_prefill_fp4.hip"}


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir(os.path.join(HIP_INCLUDE, "hip")), reason="needs g++ and the HIP headers")
@pytest.mark.parametrize("value", [None, 5000])
def test_positions_fit(tmp_path, value):
    for name in ("tetri_fp4_host.cpp", "tetri_rope_host.cpp", "tetri_host.cpp", "tetri_plan.cpp", "tetri_plan.h", "tetri_internal.h"):
        shutil.copy(os.path.join(CSRC, name), tmp_path)
    if value is not None:
        text = (tmp_path / "tetri_internal.h").read_text()
        for name in CONSTANTS:
            text, n = re.subn(r"(constexpr int32_t %s = )\d+;" % name, r"\g<1>%d;" % value, text)
            assert n == 1, name
        (tmp_path / "tetri_internal.h").write_text(text)
    exe = str(tmp_path / "guards")
    subprocess.run(["g++", "-std=c++17", "-g", "-O1", "-D__HIP_PLATFORM_AMD__=1", "-I", HIP_INCLUDE, "-I", os.path.join(ROOT, "include"), "-I", str(tmp_path),
                    os.path.join(ROOT, "tests", "host_fp4_guards.cpp")] +
                   [str(tmp_path / name) for name in ("tetri_fp4_host.cpp", "tetri_rope_host.cpp", "tetri_host.cpp", "tetri_plan.cpp")] + ["-o", exe], check=True)
    res = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0 and "guards: ok" in res.stdout, res.stdout + res.stderr


@pytest.mark.parametrize("name", sorted(CONSTANTS))
def test_kernels_count_with_them(name):
    with open(os.path.join(CSRC, CONSTANTS[name])) as f:
        assert name in f.read()
