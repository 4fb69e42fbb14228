"""CPU-only: how products in 8 bits are cut into tiles and slices, and gradients to be clipped into chunks and launches."""
import os
import shutil
import subprocess

import pytest

import dense8_reference as R

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plans") / "dense8_plans")
    source = os.path.join(os.path.dirname(os.path.abspath(__file__)), "emu", "dense8_plans.cpp")
    subprocess.run(["g++", "-O1", "-std=c++17", "-fsanitize=address,undefined", "-o", exe, source], check=True, timeout=300)

    def run(*args):
        out = subprocess.run([exe, *map(str, args)], capture_output=True, text=True, timeout=300)
        assert out.returncode == 0, out.stdout + out.stderr
        return out.stdout

    return run


def test_plans_cover_what_they_should(plans):
    assert plans().startswith("OK")


@pytest.mark.parametrize("wide,kernels", [(0, {"rows1", "rows2", "rows4", "128", "128sliced", "128deep", "128deepsliced", "256", "256sliced"}),
                                          (1, {"rows1", "rows2", "rows4", "128", "128sliced"})])
def test_the_products_sizes_reach_every_kernel(plans, wide, kernels):
    reached = plans(*[v for size in R.PRODUCT_SIZES for v in (*size, wide)]).split()
    assert len(reached) == len(R.PRODUCT_SIZES) and set(reached) == kernels
    # slices are another launch, not another kernel
    every = plans(*[v for size in R.PRODUCT_KINDS for v in (*size, wide)]).split()
    assert {k.replace("sliced", "") for k in every} == {k.replace("sliced", "") for k in kernels}
