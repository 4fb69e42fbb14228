"""Group normalisation of maps whose groups fit a workgroup, at sizes that reach every kernel of it, against 64 bits (on the
GPU, as some of these are a minibatch's)."""
import pytest
import torch

import norm_reference as R
import norm_sizes as N

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]


def wide(stat, c):
    return stat.repeat_interleave(c // stat.shape[1], 1)[:, None]


def group_mean(t, groups):
    n, hw, c = t.shape
    return t.reshape(n, hw, groups, c // groups).mean((1, 3))


def sigmoid(z):
    return 1.0 / (1.0 + torch.exp(-z))


def rounding(v, dtype):
    return v.abs() * R.HALF_STEP[dtype] * 1.01 + R.TINY[dtype]


def values(kept):
    """What a checkpoint stands for."""
    return kept.codes.float().double() * torch.exp2(kept.scales.double() - 127).repeat_interleave(32, -1)[..., :kept.shape[-1]]


def check_forward(x, gamma, beta, groups, act, got):
    """Tolerances as norm_reference derives them."""
    y, mean, rstd = got
    c, k, e = x.shape[2], R.DEPTH * R.EPS32, R.EPS32
    xd, g, b = x.double(), gamma.double(), beta.double()
    m = group_mean(xd, groups)
    r = (group_mean((xd - wide(m, c)) ** 2, groups) + 1e-5) ** -0.5
    tol_m = k * group_mean(xd.abs(), groups) + 1e-38
    tol_r = k + (tol_m * r) ** 2
    assert bool(((mean.double() - m).abs() <= tol_m).all()), "mean"
    assert bool(((rstd.double() - r).abs() <= tol_r * r).all()), "rstd"
    t = (xd - wide(m, c)) * wide(r, c) * g
    z = t + b
    tol = wide(tol_m, c) * wide(r, c) * g.abs() + t.abs() * (wide(tol_r, c) + 3 * e) + (z.abs() + b.abs()) * e
    want = z.clamp(min=0) if act == "relu" else z * sigmoid(z) if act == "silu" else z
    if act == "silu":
        tol = 1.1 * tol + want.abs() * (z.abs() + 8) * 2 * e
    assert bool(((y.double() - want).abs() <= tol + rounding(want, x.dtype)).all()), "y"


def check_backward(xd, dy, mean, rstd, gamma, beta, act, got):
    dx, dgamma, dbeta = got
    c, groups, k, e = xd.shape[2], mean.shape[1], R.DEPTH * R.EPS32, R.EPS32
    d, g, b, r = dy.double(), gamma.double(), beta.double(), wide(rstd.double(), xd.shape[2])
    hat = (xd - wide(mean.double(), c)) * r
    z = hat * g + b
    s = sigmoid(z)
    dz = d * ((z > 0).double() if act == "relu" else s * (1 + z * (1 - s)) if act == "silu" else 1.0)
    off = 4 * e * dz.abs()
    if act == "silu":
        off = off + d.abs() * (0.5 * 4 * e * ((hat * g).abs() + b.abs()) + (z.abs() + 8) * 4 * e)

    def gm(t):
        return wide(group_mean(t, groups), c)

    gz, ah, ag, og = g * dz, hat.abs(), (g * dz).abs(), g.abs() * off
    want = r * (gz - gm(gz) - hat * gm(gz * hat))
    tol = r * (og + gm(og + k * ag) + ah * gm(og * ah + k * ag * ah) + 4 * e * (ag + gm(ag) + 2 * ah * gm(ag * ah)))
    assert bool(((dx.double() - want).abs() <= tol + rounding(want, dy.dtype)).all()), "dx"
    # pictures add at most 5 additions of a thread and 7 of the workgroup, which DEPTH holds too
    assert bool(((dgamma.double() - (dz * hat).sum((0, 1))).abs() <= (off * ah + (k + 3 * e) * dz.abs() * ah).sum((0, 1)) + 1e-38).all())
    assert bool(((dbeta.double() - dz.sum((0, 1))).abs() <= (off + k * dz.abs()).sum((0, 1)) + 1e-38).all())


@pytest.mark.parametrize("size", N.RESIDENT, ids=str)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_forward_and_backward(lib, size, dtype):
    n, hw, c, groups = size
    gen = torch.Generator(device="cuda").manual_seed(n + hw + c)
    gamma = torch.randn(c, device="cuda", generator=gen) * 0.3 + 1
    beta = torch.randn(c, device="cuda", generator=gen) * 0.3
    x = (torch.randn((n, hw, c), device="cuda", generator=gen) * (gamma.abs() + 0.2) + beta).to(dtype)
    dy = torch.randn((n, hw, c), device="cuda", generator=gen).to(dtype)
    for act, code in (("relu", None), ("silu", torch.int8), ("relu", torch.float8_e4m3fn)):
        y, mean, rstd, kept = lib.group_norm_forward(x, gamma, beta, groups, 1e-5, act, checkpoint=code)
        check_forward(x, gamma, beta, groups, act, (y, mean, rstd))
        if kept is not None:
            alone = lib.checkpoint_pack(x, code)
            assert torch.equal(kept.codes.view(torch.uint8), alone.codes.view(torch.uint8)) and torch.equal(kept.scales, alone.scales)
        source, xd = (x, x.double()) if kept is None else (kept, values(kept))
        check_backward(xd, dy, mean, rstd, gamma, beta, act, lib.group_norm_backward(source, dy, mean, rstd, gamma, beta, act))
        # in place, from the same registers
        x2, d2 = x.clone(), dy.clone()
        assert torch.equal(lib.group_norm_forward(x2, gamma, beta, groups, 1e-5, act, out=x2)[0],
                           lib.group_norm_forward(x, gamma, beta, groups, 1e-5, act)[0])
        assert torch.equal(lib.group_norm_backward(source, d2, mean, rstd, gamma, beta, act, out=d2)[0],
                           lib.group_norm_backward(source, dy, mean, rstd, gamma, beta, act)[0])
