"""CPU-only: how the library cuts the operators of group normalisation and of 8-bit checkpoints into workgroups."""
import os
import shutil
import subprocess

import pytest

import norm_sizes as N
import test_gpu_checkpoint

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
EMU = os.path.join(os.path.dirname(os.path.abspath(__file__)), "emu")


def built(tmp_path_factory, name):
    exe = str(tmp_path_factory.mktemp(name) / name)
    subprocess.run(["g++", "-O1", "-std=c++17", "-fsanitize=address,undefined", "-o", exe, os.path.join(EMU, name + ".cpp")], check=True,
                   timeout=300)
    return exe


def run(exe, *args):
    out = subprocess.run([exe, *map(str, args)], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stdout + out.stderr
    return out.stdout


@pytest.fixture(scope="module")
def fc(tmp_path_factory):
    return built(tmp_path_factory, "fc_plan_check")


def test_weight_plans_cover_rows_and_weights(fc):
    assert run(fc).startswith("OK")


def test_the_weight_gradients_sizes_reach_every_tile(fc):
    """Each tile for each number of terms (types of dy), with its rows split over workgroups and not."""
    small = next(m for m in test_gpu_checkpoint.test_weight_gradient.pytestmark if "rows" in m.args[0]).args[1]
    for tile, sizes in (("64x64", small), ("64x128", N.WEIGHT_64x128), ("128x256", N.WEIGHT_128x256)):
        for terms in (1, 2, 3):
            plans = [line.split() for line in run(fc, *[v for s in sizes for v in (*s, terms)]).splitlines()]
            split = {int(slices) > 1 for name, slices in plans if name == tile}
            assert len(plans) == len(sizes) and split == {False, True}, (tile, terms, plans)


@pytest.fixture(scope="module")
def slabs(tmp_path_factory):
    return built(tmp_path_factory, "norm_library_plans")


def test_slabs_of_the_library_cover_the_picture_and_fit(slabs):
    assert run(slabs).startswith("OK")


@pytest.mark.parametrize("kind,steps", [(0, (1, 2, 4, 6, 8, 12, 16)), (1, (1, 2, 4, 6, 8, 12, 16)), (2, (1, 2, 4, 6, 8))],
                         ids=["forward", "forward_kept", "backward"])
@pytest.mark.parametrize("size", [4, 2])
def test_the_maps_reach_every_resident_kernel(slabs, kind, steps, size):
    """Every number of pixels of a thread that a kernel is built for, workgroups of every size, few and many of them."""
    plans = [[int(v) for v in line.split()] for line in run(slabs, *[v for s in N.RESIDENT for v in (*s, size, kind)]).splitlines()]
    assert len(plans) == len(N.RESIDENT)
    plans = [p for p in plans if p[0]]
    assert {next(r for r in steps if regs <= r) for regs, _, _ in plans} == set(steps)
    assert {threads for _, threads, _ in plans} == {256, 512, 1024}
    assert {0 if count < 256 else 1 if count < 1024 else 2 for _, _, count in plans} == {0, 1, 2}
    # 512 threads also with the most pixels each
    assert max(regs for regs, threads, _ in plans if threads == 512) > steps[-2]
