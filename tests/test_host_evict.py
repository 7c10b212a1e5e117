"""The host layer of the eviction calls without a GPU: what is refused launches nothing, workspaces hold what the launches are given
(tests/host_evict.cpp, with a recording HIP runtime)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIP_INCLUDE = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include")

pytestmark = pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir(os.path.join(HIP_INCLUDE, "hip")),
                                reason="needs g++ and the HIP headers")


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("host") / "host_evict")
    csrc = os.path.join(ROOT, "paper_2401_11181_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-g", "-O1", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    "-static-libasan", "-static-libubsan", "-Wall", "-D__HIP_PLATFORM_AMD__=1", "-I", HIP_INCLUDE,
                    "-I", os.path.join(ROOT, "include"), "-I", csrc, os.path.join(ROOT, "tests", "host_evict.cpp")] +
                   [os.path.join(csrc, name) for name in ("tetri_evict_host.cpp", "tetri_host.cpp", "tetri_plan.cpp")] + ["-o", exe], check=True)
    return exe


@pytest.mark.parametrize("check", ["refusals", "workspaces", "arguments"])
def test_host_layer(driver, check):
    res = subprocess.run([driver, check], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0 and check + ": ok" in res.stdout, res.stdout + res.stderr


def test_kernels_of_the_gpu_tests(driver):
    """The shapes of tests/test_gpu_evict_instances.py go to the kernels that they are meant for."""
    res = subprocess.run([driver, "instances"], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0 and "instances: ok" in res.stdout, res.stdout + res.stderr
