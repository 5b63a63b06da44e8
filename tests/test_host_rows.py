"""Rows of a badly divided batch on the host (tests/host_plan): each is one request's.  No GPU and no HIP runtime are involved."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CXX = "/opt/rocm/llvm/bin/clang++"

pytestmark = pytest.mark.skipif(not os.path.exists(CXX), reason="ROCm clang++ not installed")


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("rows") / "rows")
    src = os.path.join(ROOT, "tests", "host_plan")
    r = subprocess.run([CXX, "-std=c++20", "-O1", "-g", f"-I{src}", f"-I{ROOT}/paper_2609_24197_amd/csrc",
                        os.path.join(src, "rows_driver.cpp"), "-o", out], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-4000:]
    return out


@pytest.mark.parametrize("seed", range(4))
def test_rows_of_several_ranges_are_the_first_requests(driver, seed):
    r = subprocess.run([driver, str(seed)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, (r.returncode, r.stderr[-2000:])
