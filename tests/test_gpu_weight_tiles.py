"""The weight gradient from a checkpoint on its larger tiles of dw: values, edges and what is not finite."""
import numpy as np
import pytest
import torch

import norm_reference as R
import norm_sizes as N

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
CODES = [torch.int8, torch.float8_e4m3fn]
SIZES = N.WEIGHT_64x128 + N.WEIGHT_128x256


def inputs(lib, rows, cols, out, dtype, code, seed, wide=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((rows, cols), device="cuda", generator=gen)
    x *= torch.exp2(torch.randint(-6, 7, (rows, 1), device="cuda", generator=gen).float())  # a scale of their own to rows
    x[:, 32:64] *= 64  # and to neighbouring blocks
    dy = (torch.randn((rows, out + wide), device="cuda", generator=gen) * 0.1).to(dtype)[:, wide:]
    return lib.checkpoint_pack(x, code), dy


def values(kept):
    """The definition, in 64 bits."""
    scale = torch.exp2(kept.scales.double() - 127).repeat_interleave(32, 1)[:, :kept.shape[1]]
    return kept.codes.float().double() * scale


def check(kept, dy, dw, db):
    x, d = values(kept), dy.double()
    rows = x.shape[0]
    # products are exact, or rounded once for terms of fp32; an accumulator is rounded at most once a product and the slices'
    # sums join in a few more additions
    k = (rows + 64) * R.EPS32
    assert bool(((dw.double() - d.t().contiguous() @ x).abs() <= k * (d.abs().t().contiguous() @ x.abs()) + 1e-38).all())
    assert bool(((db.double() - d.sum(0)).abs() <= k * d.abs().sum(0) + 1e-38).all())
    if rows >= 64:  # in the mean far less: random signs
        want = d.t().contiguous() @ x
        assert float((dw.double() - want).norm()) <= 2e-6 * float(want.norm())


@pytest.mark.parametrize("rows,cols,out", SIZES)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_weight_gradient(lib, rows, cols, out, dtype):
    for i, code in enumerate(CODES):
        kept, dy = inputs(lib, rows, cols, out, dtype, code, rows + i, wide=i)
        # nothing behind the last row or column is written
        room = torch.full((out * cols + 64,), 7.0, device="cuda")
        bias = torch.full((out + 64,), 7.0, device="cuda")
        dw, db = lib.checkpoint_fc_backward_weight(kept, dy, dw=room[:out * cols].view(out, cols), db=bias[:out])
        check(kept, dy, dw, db)
        assert bool((room[out * cols:] == 7).all()) and bool((bias[out:] == 7).all())


@pytest.mark.parametrize("rows,cols,out", [(70, 777, 2501), (3000, 513, 259), (97, 4097, 2049), (40000, 1030, 515)])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("code", CODES, ids=str)
def test_what_is_not_finite(lib, rows, cols, out, dtype, code):
    """An infinity or a NaN of dy reaches its own row of dw, a block that is not finite its own columns, and nothing else."""
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.rand((rows, cols), device="cuda", generator=gen) + 0.5
    dy = torch.randn((rows, out), device="cuda", generator=gen).to(dtype)
    clean, clean_b = lib.checkpoint_fc_backward_weight(lib.checkpoint_pack(x, code), dy)
    dy[0, 1], dy[rows - 1, out - 1] = float("-inf"), float("nan")
    x[rows - 2, cols - 1] = float("nan")
    dw, db = lib.checkpoint_fc_backward_weight(lib.checkpoint_pack(x, code), dy)
    last = (cols - 1) // 32 * 32  # the block
    assert bool((dw[1, :last] == float("-inf")).all()) and bool(torch.isnan(dw[out - 1]).all()) and bool(torch.isnan(dw[:, last:]).all())
    assert float(db[1]) == float("-inf") and bool(torch.isnan(db[out - 1]))
    rest = [i for i in range(out) if i not in (1, out - 1)]
    assert torch.equal(dw[rest, :last], clean[rest, :last]) and torch.equal(db[rest], clean_b[rest])


@pytest.mark.parametrize("rows,cols,out", [(300, 4098, 2051), (40000, 1030, 515)])
def test_captured_and_replayed(lib, rows, cols, out):
    kept, dy = inputs(lib, rows, cols, out, torch.float32, torch.int8, 4)
    lib.checkpoint_fc_backward_weight(kept, dy)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dw, db = lib.checkpoint_fc_backward_weight(kept, dy)
    for seed in range(3):
        other, d = inputs(lib, rows, cols, out, torch.float32, torch.int8, 40 + seed)
        kept.codes.copy_(other.codes)
        kept.scales.copy_(other.scales)
        dy.copy_(d)
        graph.replay()
        torch.cuda.synchronize()
        want, want_b = lib.checkpoint_fc_backward_weight(other, d)
        assert torch.equal(dw, want) and torch.equal(db, want_b)
