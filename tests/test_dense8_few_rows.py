"""CPU-only: products of few rows with a large weight, which memory bounds, take the kernel made for them."""
import os
import shutil
import subprocess

import pytest

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plans") / "dense8_plans")
    source = os.path.join(os.path.dirname(os.path.abspath(__file__)), "emu", "dense8_plans.cpp")
    subprocess.run(["g++", "-O1", "-std=c++17", "-o", exe, source], check=True, timeout=300)
    return lambda sizes: subprocess.run([exe, *(str(v) for size in sizes for v in size)], capture_output=True, text=True, check=True, timeout=300).stdout.split()


@pytest.mark.parametrize("wide", [0, 1])
def test_one_to_sixteen_rows_and_a_weight_of_over_100_mb(kernels, wide):
    sizes = [(m, n, k, wide) for m in (1, 2, 5, 16) for n, k in ((16384, 16384), (9216, 16384), (16384, 9216), (14000, 14000), (32768, 4096), (20000, 6000), (12000, 12000))]
    # the weight may as well be a
    turned = [(n, m, k, wide) for m, n, k, _ in sizes]
    assert set(kernels(sizes)) == {"rows1"}
    assert all(k.startswith("rows") for k in kernels(turned))
