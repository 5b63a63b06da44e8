"""The 4-bit cache's layout on the host: what the kernels step from page to page by, at sizes past 32 bits."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CXX = "/opt/rocm/llvm/bin/clang++"

pytestmark = pytest.mark.skipif(not os.path.exists(CXX), reason="ROCm clang++ not installed")


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("layout") / "layout")
    src = os.path.join(ROOT, "tests", "host_plan")
    r = subprocess.run([CXX, "-std=c++20", "-O1", f"-I{src}", f"-I{ROOT}/paper_2609_24197_amd/csrc",
                        os.path.join(src, "mx_layout_driver.cpp"), "-o", out], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-4000:]
    return out


@pytest.mark.parametrize("ps,D,Hkv", [(16, 64, 1), (16, 128, 8), (1 << 20, 128, 64), (1 << 23, 128, 8), (1 << 24, 128, 8),
                                      (1 << 25, 64, 64), (1 << 24, 128, 4096)])
def test_bytes_of_pages(driver, ps, D, Hkv):
    head = ps * D * 17 // 32                 # 4 bits a channel and a byte for 32 of them
    got = subprocess.run([driver, str(ps), str(D), str(Hkv)], capture_output=True, text=True, timeout=60, check=True).stdout
    assert list(map(int, got.split())) == [head, head * Hkv]
