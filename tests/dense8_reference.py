"""64-bit references of the 8-bit operands, their products, root-mean-square normalisation and gradient clipping, and what their
float32 arithmetic may be off by."""
import numpy as np
import torch

EPS32 = 2.0 ** -24  # half a step of float32
BLOCK = 128
# Products (m, n, k) that reach every kernel: one row and up, odd sizes, k under, at and over a block; tiles of 128 and 256, the sum whole or
# in slices, of any number of turns of the stages and left-over steps
PRODUCT_SIZES = [
    (1, 1, 1), (1, 16, 128), (1, 1000, 2304), (2, 17, 129), (15, 3, 64), (16, 130, 1152), (17, 33, 1025), (32, 48, 256), (33, 100, 1280),
    (63, 65, 127), (64, 16, 4096), (65, 7, 1000), (129, 515, 1001), (128, 128, 128), (200, 130, 5000), (300, 1000, 260), (1000, 65, 640),
    (65, 4096, 130), (257, 4149, 131), (259, 4129, 67), (770, 1250, 1188), (1485, 41, 3733), (41, 41, 37486), (4399, 40, 951), (4204, 40, 1039),
    (4026, 40, 1188), (3935, 40, 1282), (40, 41, 42430), (41, 41, 41627), (642, 776, 4320), (609, 618, 7298), (656, 516, 10255), (16390, 1030, 129),
    (4000, 4090, 257), (3900, 4096, 1100), (1700, 2340, 5300)]
# and those for every pair of codes and kinds of blocks
PRODUCT_KINDS = [(5, 40, 700), (20, 40, 300), (129, 515, 300), (300, 1000, 260), (257, 4149, 131), (4204, 40, 1039), (40, 41, 42430), (4000, 4090, 200)]
TOP = {torch.float8_e4m3fn: 448.0, torch.float8_e5m2: 57344.0}
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
# half the distance of neighbours among the smallest numbers
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}


def f64(t):
    return t.detach().double().cpu().numpy()


def rounding(v, dtype):
    return np.abs(v) * HALF[dtype] * 1.01 + TINY[dtype]


def round8(v, code):
    """v to the nearest code as a number, ties to even."""
    low, bits = (-6, 3.0) if code == torch.float8_e4m3fn else (-14, 2.0)
    _, e = np.frexp(v)
    step = np.exp2(np.maximum(e - 1, low) - bits)
    return np.round(v / step) * step


def pack(x, code, square=False):
    """(codes as numbers [rows][whole blocks], scales [blocks][rows up to a multiple of 4, or blocks of rows]) of x [rows][cols]"""
    rows, cols = x.shape
    tall = BLOCK if square else 1
    full = np.zeros((-(-rows // tall) * tall, -(-cols // BLOCK) * BLOCK))
    full[:rows, :cols] = x
    blocks = full.reshape(full.shape[0] // tall, tall, -1, BLOCK)
    bad = ~np.isfinite(blocks).all(axis=(1, 3))
    most = np.abs(np.where(np.isfinite(blocks), blocks, 0.0)).max(axis=(1, 3))
    most = np.where(bad, 1.0, most)
    top = TOP[code]
    with np.errstate(divide="ignore"):
        e = np.maximum(np.ceil(np.log2(most / top)), -126.0)
    # the logarithm rounds: settle its neighbours by the definition
    e = np.where(most > top * np.exp2(e), e + 1, e)
    e = np.where((e > -126) & (most <= top * np.exp2(e - 1)), e - 1, e)
    v = np.where(bad[:, None, :, None], 0.0, blocks) / np.exp2(e)[:, None, :, None]
    scales = np.where(bad, 255, e + 127).astype(np.uint8).T
    if not square:
        scales = np.pad(scales, ((0, 0), (0, -rows % 4)))
    return round8(v, code).reshape(full.shape)[:rows], scales


def values(codes, scales, cols, square=False):
    rows = codes.shape[0]
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127.0)).T
    s = np.repeat(s, BLOCK if square else 1, axis=0)[:rows]
    return (codes * np.repeat(s, BLOCK, axis=1))[:, :cols]


def product_tolerance(a, b, y, dtype):
    """Products are exact.  To float32 sums are float32: on the way to a result are at most 64 additions inside an instruction,
    one for each instruction, and 40 for waves and slices; each may leave off a step.  To 16 bits eight products at a time are
    added with 13 bits under the largest: seven of them may each lose as much."""
    k = a.shape[1]
    size = np.nan_to_num(np.abs(a)) @ np.nan_to_num(np.abs(b)).T
    own = (104 + k / 64) * 2 * EPS32 + (0.0 if dtype == torch.float32 else 7 * 2.0 ** -13)
    return own * size + rounding(np.abs(y) + own * size, dtype) + 2.0 ** -126


def rms_norm(x, residual, gamma, eps, dtype):
    """(y, s, rstd) with s rounded to the type."""
    s = x
    if residual is not None:
        with np.errstate(over="ignore"):
            s = f64(torch.from_numpy(x + residual).to(dtype))
    rstd = 1.0 / np.sqrt((s * s).mean(axis=1) + eps)
    return s * rstd[:, None] * (1.0 if gamma is None else gamma), s, rstd


# Additions one after another on the way to a row's sum: a lane's share of the row (64 where it is in registers, 2^20 / 1024 at
# most), then 20 across lanes and waves
def row_depth(cols):
    return 84 + cols / 1024


def rstd_tolerance(cols):
    """Relative: half of the sum's, the division by the columns, the addition of eps, the root and the reciprocal."""
    return (row_depth(cols) / 2 + 4) * EPS32


def norm_tolerance(y, cols):
    return np.abs(y) * (rstd_tolerance(cols) + 2 * EPS32)


def rms_norm_backward(s, dy, rstd, gamma, dsum):
    h = s * rstd[:, None]
    g = dy * (1.0 if gamma is None else gamma)
    dx = rstd[:, None] * (g - h * (g * h).mean(axis=1, keepdims=True))
    return dx + (0.0 if dsum is None else dsum), (dy * h).sum(axis=0)


def backward_tolerance(s, dy, rstd, gamma, dsum, dx, dtype):
    rows, cols = s.shape
    h = np.abs(s * rstd[:, None])
    g = np.abs(dy * (1.0 if gamma is None else gamma))
    mean = (g * h).mean(axis=1, keepdims=True)
    tol = rstd[:, None] * (2 * g + h * mean * (row_depth(cols) + 6)) * EPS32
    tol = tol + 2 * EPS32 * (rstd[:, None] * (g + h * mean) + (0.0 if dsum is None else np.abs(dsum)))
    # rows one after another in a team, then teams and workgroups
    depth = rows / 512 + 100
    return tol + rounding(dx, dtype), (depth + 2) * EPS32 * np.abs(dy * h).sum(axis=0) + 2.0 ** -126
