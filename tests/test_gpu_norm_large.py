"""Group normalisation at the largest sizes that it takes: launches as large as a grid, sums past 31 bits of elements."""
import numpy as np
import pytest
import torch

import norm_reference as R

pytestmark = pytest.mark.gpu


def test_as_many_workgroups_as_a_grid_holds(lib):
    """4095 pictures of one pixel and 2^20 - 1 channels, dx in place of dy: value by value, so the launch that writes dx has
    4095 * 4096 workgroups of 256 threads, and the parameter gradients' 2^17 more are past the 2^32 threads of a grid."""
    n, c = 4095, (1 << 20) - 1
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn((n, 1, c), device="cuda", dtype=torch.bfloat16, generator=gen)
    dy = torch.randn((n, 1, c), device="cuda", dtype=torch.bfloat16, generator=gen)
    mean = torch.randn((n, 1), device="cuda", generator=gen) * 0.1
    rstd = torch.rand((n, 1), device="cuda", generator=gen) + 0.5
    sums = torch.zeros((4, c), device="cuda", dtype=torch.float64)  # dbeta, dgamma, and of their terms' magnitudes
    ends = {}
    for i in range(0, n, 105):
        d = dy[i:i + 105, 0].double()
        hat = (x[i:i + 105, 0].double() - mean[i:i + 105].double()) * rstd[i:i + 105].double()
        sums += torch.stack([d.sum(0), (d * hat).sum(0), d.abs().sum(0), (d * hat).abs().sum(0)])
        for k in (0, 104):
            if i + k in (0, n - 1):
                a, b = d[k].mean(), (d[k] * hat[k]).mean()
                off_a, off_b = R.DEPTH * R.EPS32 * d[k].abs().mean(), (R.DEPTH + 3) * R.EPS32 * (d[k] * hat[k]).abs().mean()
                r = rstd[i + k].double()
                want = r * (d[k] - a - hat[k] * b)
                # four roundings of the terms and the one to bfloat16
                off = r * (off_a + hat[k].abs() * off_b + 4 * R.EPS32 * (d[k].abs() + a.abs() + 2 * (hat[k] * b).abs()))
                ends[i + k] = (want, off + want.abs() * R.HALF_STEP[torch.bfloat16] * 1.01)
        del d, hat
    dx, dgamma, dbeta = lib.group_norm_backward(x, dy, mean, rstd, None, None, out=dy)
    assert dx.data_ptr() == dy.data_ptr()
    assert bool(((dbeta.double() - sums[0]).abs() <= R.DEPTH * R.EPS32 * sums[2]).all())
    assert bool(((dgamma.double() - sums[1]).abs() <= (R.DEPTH + 3) * R.EPS32 * sums[3]).all())
    assert sorted(ends) == [0, n - 1]
    for i, (want, off) in ends.items():
        assert bool(((dx[i, 0].double() - want).abs() <= off).all())
    del x, dy, dx, sums, ends
    torch.cuda.empty_cache()
