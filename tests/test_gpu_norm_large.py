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


@pytest.mark.parametrize("code", [None, torch.int8, torch.float8_e4m3fn], ids=str)
def test_gradient_sums_past_31_bits_of_elements(lib, code):
    """Two pictures of 2^25 + 3 pixels.  dy and x rise along the pixels and from picture to picture, so that a chunk left out
    or taken twice moves a sum by some 2^-11 of its terms.  A term passes at most 1311 additions of a thread, 25 rows,
    64 chunks of a thread and five more: under 2048."""
    n, hw, c, groups = 2, (1 << 25) + 3, 40, 4
    gen = torch.Generator(device="cuda").manual_seed(9)
    ramp = torch.linspace(0, 1, hw, device="cuda")[None, :, None] + torch.tensor([0.0, 0.5], device="cuda")[:, None, None]
    x = torch.randn((n, hw, c), device="cuda", generator=gen).add_(ramp, alpha=2.0)
    dy = torch.randn((n, hw, c), device="cuda", generator=gen).add_(ramp + 1.0)
    gamma = torch.randn(c, device="cuda", generator=gen) * 0.2 + 1
    _, mean, rstd, kept = lib.group_norm_forward(x, gamma, None, groups, 1e-5, "none", checkpoint=code)
    wide_m, wide_r = (t.double().repeat_interleave(c // groups, 1)[:, None] for t in (mean, rstd))
    sums = torch.zeros((n, 4, c), device="cuda", dtype=torch.float64)  # of dy, of dy hat, and of their magnitudes

    def hats(a, b):
        part = x[:, a:b] if kept is None else lib.checkpoint_unpack(
            lib.Checkpoint(kept.codes[:, a:b].contiguous(), kept.scales[:, a:b].contiguous()))
        return (part.double() - wide_m) * wide_r

    step = 1 << 21
    for a in range(0, hw, step):
        d, hat = dy[:, a:a + step].double(), hats(a, min(hw, a + step))
        sums += torch.stack([d.sum(1), (d * hat).sum(1), d.abs().sum(1), (d * hat).abs().sum(1)], 1)
        del d, hat
    # the first, the last and some pixels between, before dx takes the place of dy
    spots = [(0, 500), (hw // 2, hw // 2 + 500), (hw - 500, hw)]
    some = [(dy[:, a:b].double(), hats(a, b)) for a, b in spots]
    dx, dgamma, dbeta = lib.group_norm_backward(x if kept is None else kept, dy, mean, rstd, gamma, None, "none", out=dy)
    k = 2048 * R.EPS32
    total = sums.sum(0)
    assert bool(((dbeta.double() - total[0]).abs() <= k * total[2]).all())
    assert bool(((dgamma.double() - total[1]).abs() <= (k + 3 * R.EPS32) * total[3]).all())
    g = gamma.double()

    def group_mean(t):
        return (t.view(n, groups, -1).sum(2) / (hw * (c // groups))).repeat_interleave(c // groups, 1)[:, None]

    a, b = group_mean(g * sums[:, 0]), group_mean(g * sums[:, 1])
    off_a, off_b = k * group_mean(g.abs() * sums[:, 2]), (k + 3 * R.EPS32) * group_mean(g.abs() * sums[:, 3])
    for (lo, hi), (d, hat) in zip(spots, some):
        want = wide_r * (g * d - a - hat * b)
        off = wide_r * (off_a + hat.abs() * off_b + 4 * R.EPS32 * ((g * d).abs() + a.abs() + 2 * (hat * b).abs()))
        assert bool(((dx[:, lo:hi].double() - want).abs() <= off + want.abs() * R.HALF_STEP[torch.float32] * 1.01).all())
    del x, dy, dx, kept, some
    torch.cuda.empty_cache()


@pytest.mark.parametrize("size", [(2, 300, 64, 4), (2, 5000, 64, 4), (1, 9000, 300, 2)], ids=str)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_the_largest_and_smallest_values_that_sums_hold(lib, size, dtype):
    """Squares that add up to 2^125 to 2^126 in a group, values that add up to 2^126, and values next to nothing beside eps."""
    n, hw, c, groups = size
    count = hw * c // groups
    gen = torch.Generator(device="cuda").manual_seed(hw)
    sign = torch.randint(0, 2, (n, hw, c), device="cuda", generator=gen).double() * 2 - 1
    spread = 2.0 ** 62.5 / count ** 0.5 * sign * (1 + 0.1 * torch.rand((n, hw, c), device="cuda", generator=gen))
    level = 2.0 ** 126 / count * torch.ones_like(spread)
    tiny = 2.0 ** -100 * sign
    for v, eps in ((spread, 1e-5), (level, 1e-5), (tiny, 1e-5), (tiny, 1e-37)):
        x = v.to(dtype)
        y, mean, rstd, kept = lib.group_norm_forward(x, None, None, groups, eps, "none", checkpoint=torch.int8)
        xd = x.double().view(n, hw, groups, c // groups)
        m = xd.mean((1, 3))
        r = (((xd - m[:, None, :, None]) ** 2).mean((1, 3)) + eps) ** -0.5
        tol_m = R.DEPTH * R.EPS32 * xd.abs().mean((1, 3)) + 1e-38
        if v is level:  # all values alike: the deviations are the mean's own rounding
            assert bool(((mean.double() - m).abs() <= tol_m).all()) and bool(torch.isfinite(y).all())
            continue
        tol_r = R.DEPTH * R.EPS32 + (tol_m * r) ** 2
        assert bool(((mean.double() - m).abs() <= tol_m).all()) and bool(((rstd.double() - r).abs() <= tol_r * r).all())
        want = (xd - m[:, None, :, None]) * r[:, None, :, None]
        off = tol_m[:, None, :, None] * r[:, None, :, None] + want.abs() * (tol_r[:, None, :, None] + 3 * R.EPS32)
        off = off + want.abs() * R.HALF_STEP[dtype] * 1.01 + R.TINY[dtype]
        assert bool(((y.double().view(xd.shape) - want).abs() <= off).all())
        back = lib.checkpoint_unpack(kept, torch.float32)
        most = torch.nn.functional.pad(x.float().abs(), (0, -c % 32)).view(n, hw, -1, 32).amax(3).repeat_interleave(32, 2)[..., :c]
        assert bool(((back - x.float()).abs() <= most / 127).all())


@pytest.mark.parametrize("size", [(2, 300, 64, 4), (2, 5000, 64, 4), (1, 9000, 300, 2), (3, 9000, 256, 256)], ids=str)
def test_a_mean_whose_square_no_float_holds(lib, size):
    """Only squares of deviations count: values of 2^64.5 with deviations of 2^54, whose squares add up to 2^126 at most."""
    n, hw, c, groups = size
    gen = torch.Generator(device="cuda").manual_seed(hw)
    x = (2.0 ** 64.5 + 2.0 ** 54 / (hw * c // groups / 2.0 ** 17 + 1) ** 0.5
         * torch.randn((n, hw, c), device="cuda", generator=gen, dtype=torch.float64)).float()
    xd = x.double().view(n, hw, groups, c // groups)
    m = xd.mean((1, 3))
    r = (((xd - m[:, None, :, None]) ** 2).mean((1, 3)) + 1e-5) ** -0.5
    y, mean, rstd, _ = lib.group_norm_forward(x, None, None, groups)
    tol_m = R.DEPTH * R.EPS32 * xd.abs().mean((1, 3))
    tol_r = R.DEPTH * R.EPS32 + (tol_m * r) ** 2
    assert bool(((mean.double() - m).abs() <= tol_m).all()) and bool(((rstd.double() - r).abs() <= tol_r * r).all())
    want = (xd - m[:, None, :, None]) * r[:, None, :, None]
    off = tol_m[:, None, :, None] * r[:, None, :, None] + want.abs() * (tol_r[:, None, :, None] + 4 * R.EPS32) + R.EPS32
    assert bool(((y.double().view(xd.shape) - want).abs() <= off).all())
