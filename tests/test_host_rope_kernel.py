"""The kernel of the norm and rotation on the CPU, lane by lane (tests/rope_on_cpu.cpp): arrays of a chunk's q and k, and its outputs, that end with their last real row are
not touched behind it, whatever the rows of the call; nor are those of calls with given positions."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
CLANG = os.path.join(ROCM, "llvm", "bin", "clang++")

pytestmark = pytest.mark.skipif(not os.path.exists(CLANG) or not os.path.isdir(os.path.join(ROCM, "include", "hip")),
                                reason="needs clang++ and the HIP headers")


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    where = tmp_path_factory.mktemp("rope")
    csrc = os.path.join(ROOT, "paper_2401_11181_amd", "csrc")
    # (beside the stand-in for attn_common.h, which is looked for beside the file that includes it)
    shutil.copy(os.path.join(csrc, "tetri_rope.hip"), where)
    shutil.copy(os.path.join(ROOT, "tests", "rope_on_cpu.h"), where / "attn_common.h")
    exe = str(where / "rope_on_cpu")
    subprocess.run([CLANG, "-x", "c++", "-std=c++17", "-O1", "-w", "-D__HIP_PLATFORM_AMD__=1", "-I", str(where), "-I", os.path.join(ROCM, "include"), "-I",
                    os.path.join(ROOT, "include"), "-I", csrc, os.path.join(ROOT, "tests", "rope_on_cpu.cpp"), "-o", exe, "-lm"], check=True)
    return exe


# heads, kv heads, head_dim, rows of the call, segments (0: given positions), rows of a segment, wavefronts of a row at most, pairs, adjacent
CASES = [(4, 2, 128, 9, 0, 0, 1, 64, 0), (6, 2, 64, 5, 0, 0, 3, 16, 1),
         (4, 2, 128, 12, 1, 12, 1, 64, 0),                                  # a chunk without padding
         (4, 2, 128, 12, 1, 5, 1, 64, 0), (4, 2, 128, 64, 3, 2, 2, 32, 1), (3, 1, 64, 130, 70, 1, 1, 32, 0), (20, 4, 64, 9, 2, 4, 8, 32, 0),
         (1, 1, 64, 5, 1, 1, 1, 8, 0), (8, 8, 128, 7, 2, 0, 4, 64, 0)]      # ... and one of padding alone


@pytest.mark.parametrize("case", CASES, ids=str)
def test_nothing_behind_the_last_row_is_touched(driver, case):
    res = subprocess.run([driver, *map(str, case)], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0 and res.stdout.strip() == "ok", res.stdout + res.stderr
