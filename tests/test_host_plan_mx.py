"""The chunk attention's plan over the 4-bit cache, run on the host thread by thread (tests/host_plan): units, split tiles
and columns stay inside the workspace and hold every key of every tile of rows once.  No GPU and no HIP runtime are
involved."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CXX = "/opt/rocm/llvm/bin/clang++"

pytestmark = pytest.mark.skipif(not os.path.exists(CXX), reason="ROCm clang++ not installed")


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("plan") / "plan")
    src = os.path.join(ROOT, "tests", "host_plan")
    r = subprocess.run([CXX, "-std=c++20", "-O1", "-g", f"-I{src}", f"-I{ROOT}/paper_2609_24197_amd/csrc",
                        os.path.join(src, "mx_driver.cpp"), "-o", out], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-4000:]
    return out


@pytest.mark.parametrize("mode", ["valid", "malformed", "longest"])
def test_plans(driver, mode):
    r = subprocess.run([driver, mode], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, (r.returncode, r.stderr[-2000:])
    columns, lanes = map(int, re.search(r"(\d+) plans in columns, (\d+) of lanes", r.stdout).groups())
    assert columns >= 3 and (lanes >= 50 or mode == "longest")
