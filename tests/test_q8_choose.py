"""The choice of kernel for products in 8-bit integers and its launch, checked
without a GPU (built with g++)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_every_product_that_fits_the_card_has_a_launch(tmp_path):
    exe = tmp_path / "q8_choose_check"
    subprocess.run(["g++", "-std=c++17", "-O1", "-I" + os.path.join(ROOT, "paper_2305_06942_amd", "csrc"),
                    os.path.join(ROOT, "tests", "q8_choose_check.cpp"), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "bad=0" in r.stdout
