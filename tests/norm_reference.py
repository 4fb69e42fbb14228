"""Plain 64-bit group normalisation and 8-bit coding for the tests, and how far the library's results may be from them.

EPS32 is half a step of float32 relative to the value.  A sum over a group goes through at most DEPTH additions on the way of
any one term (a thread's own, the rows of a workgroup, chunks, channels), so it is off by at most DEPTH * EPS32 times the sum of
the terms' magnitudes."""
import numpy as np
import torch

EPS32 = 2.0 ** -24
DEPTH = 96
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}  # half a step of the smallest numbers


def rounding(v, dtype):
    return np.abs(v) * HALF_STEP[dtype] * 1.01 + TINY[dtype]


def per_channel(stat, c):
    """[n][groups] as [n][1][c]"""
    return np.repeat(stat, c // stat.shape[1], axis=1)[:, None, :]


def forward(x, gamma, beta, groups, eps, act):
    n, hw, c = x.shape
    g = x.reshape(n, hw, groups, c // groups)
    mean = g.mean(axis=(1, 3))
    rstd = 1.0 / np.sqrt(((g - mean[:, None, :, None]) ** 2).mean(axis=(1, 3)) + eps)
    z = (x - per_channel(mean, c)) * per_channel(rstd, c) * gamma + beta
    return activation(z, act), mean, rstd, z


def sigmoid(z):
    return 1.0 / (1.0 + np.exp(-np.clip(z, -700, 700)))


def activation(z, act):
    return np.where(z > 0, z, 0.0) if act == "relu" else z * sigmoid(z) if act == "silu" else z


def slope(z, act):
    s = sigmoid(z)
    return (z > 0).astype(np.float64) if act == "relu" else s * (1.0 + z * (1.0 - s)) if act == "silu" else np.ones_like(z)


def backward(x, dy, mean, rstd, gamma, beta, act):
    n, hw, c = x.shape
    groups = mean.shape[1]
    hat = (x - per_channel(mean, c)) * per_channel(rstd, c)
    dz = dy * slope(hat * gamma + beta, act)
    g = gamma * dz

    def group_mean(t):
        return per_channel(t.reshape(n, hw, groups, c // groups).mean(axis=(1, 3)), c)

    dx = per_channel(rstd, c) * (g - group_mean(g) - hat * group_mean(g * hat))
    return dx, (dz * hat).sum(axis=(0, 1)), dz.sum(axis=(0, 1))


def statistics_tolerance(x, groups, rstd):
    """(of mean, relative of rstd).  The variance is a sum of squares about a mean that is off by `mean`: the first counts with
    DEPTH, the second adds (mean / deviation)^2; half of the relative error of the variance is that of rstd."""
    n, hw, c = x.shape
    size = np.abs(x).reshape(n, hw, groups, c // groups).mean(axis=(1, 3))
    mean = DEPTH * EPS32 * size + 1e-38
    return mean, DEPTH * EPS32 + (mean * rstd) ** 2


def forward_tolerance(x, y, z, gamma, beta, mean, rstd, dtype, act):
    c = x.shape[2]
    tol_mean, tol_rstd = statistics_tolerance(x, mean.shape[1], rstd)
    r = per_channel(rstd, c) * np.abs(gamma)
    t = np.abs(x - per_channel(mean, c)) * r
    # the subtraction, the factor and the fma round once each
    tol_z = per_channel(tol_mean, c) * r + t * (per_channel(tol_rstd, c) + 3 * EPS32) + (np.abs(z) + np.abs(beta)) * EPS32
    if act == "silu":  # slope at most 1.1; the exponential's argument is rounded, its result and the reciprocal by an ulp each
        tol_z = 1.1 * tol_z + np.abs(y) * (np.abs(z) + 8) * 2 * EPS32
    return tol_z + rounding(y, dtype)


def backward_tolerance(x, dy, mean, rstd, gamma, beta, act, dx, dtype):
    """(dx, dgamma, dbeta): mean and rstd are inputs here, so only roundings count."""
    n, hw, c = x.shape
    groups = mean.shape[1]
    r = per_channel(rstd, c)
    hat = np.abs((x - per_channel(mean, c)) * r)
    z = (x - per_channel(mean, c)) * r * gamma + beta
    dz = np.abs(dy * slope(z, act))
    off = 4 * EPS32 * dz
    if act == "silu":  # z is off by 4 roundings of its terms, the slope's own slope is at most 0.5
        off = off + np.abs(dy) * (0.5 * 4 * EPS32 * (hat * np.abs(gamma) + np.abs(beta)) + (np.abs(z) + 8) * 4 * EPS32)
    g, off_g = np.abs(gamma) * dz, np.abs(gamma) * off

    def group_mean(t):
        return per_channel(t.reshape(n, hw, groups, c // groups).mean(axis=(1, 3)), c)

    k = DEPTH * EPS32
    tol = r * (off_g + group_mean(off_g + k * g) + hat * group_mean(off_g * hat + k * g * hat)
               + 4 * EPS32 * (g + group_mean(g) + 2 * hat * group_mean(g * hat)))
    return (tol + rounding(dx, dtype), (off * hat + (k + 3 * EPS32) * dz * hat).sum(axis=(0, 1)) + 1e-38,
            (off + k * dz).sum(axis=(0, 1)) + 1e-38)


# ---- 8 bits ----
def e4m3(v):
    """v rounded to four significant bits down to 2^-6, to steps of 2^-9 below, ties to even."""
    _, e = np.frexp(v)
    step = np.exp2(np.maximum(e - 1, -6) - 3.0)
    return np.round(v / step) * step


def code(x, kind):
    """(codes as numbers, scale codes) of x [rows][cols]"""
    rows, cols = x.shape
    nb = -(-cols // 32)
    full = np.zeros((rows, nb * 32))
    full[:, :cols] = x
    full = full.reshape(rows, nb, 32)
    bad = ~np.isfinite(full).all(axis=2)
    most = np.where(bad, 1.0, np.abs(np.where(np.isfinite(full), full, 0.0)).max(axis=2))
    top = 127.0 if kind == torch.int8 else 448.0
    with np.errstate(divide="ignore"):
        e = np.maximum(np.ceil(np.log2(most / top)), -126.0)
    # the logarithm rounds: settle its neighbours by the definition
    e = np.where(most > top * np.exp2(e), e + 1, e)
    e = np.where((e > -126) & (most <= top * np.exp2(e - 1)), e - 1, e)
    v = np.where(bad[..., None], 0.0, full) / np.exp2(e)[..., None]
    codes = np.round(v) if kind == torch.int8 else e4m3(v)
    return codes.reshape(rows, -1)[:, :cols], np.where(bad, 255, e + 127).astype(np.uint8)


def decode(codes, scales):
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127.0))
    return codes * np.repeat(s, 32, axis=1)[:, :codes.shape[1]]
