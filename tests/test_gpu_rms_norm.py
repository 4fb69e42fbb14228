"""Root-mean-square normalisation against 64 bits: every register plan, rows that none holds, strides, in place, 8-bit results."""
import numpy as np
import pytest
import torch

import dense8_reference as R
from dense8_reference import f64

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2
EPS = 1e-5
# every plan of rms_plan, at its edge and off it
COLS = [1, 2, 7, 8, 127, 128, 129, 256, 300, 384, 385, 512, 777, 1024, 2048, 2049, 4096, 5000, 8192, 12345, 16384, 20000, 32768, 40001, 65536, 65537, 70000]


def rows_for(cols):
    return max(3, min(700, 300000 // cols)) | 1


def data(rows, cols, dtype, seed=0):
    gen = torch.Generator().manual_seed(rows * 131 + cols + seed)
    make = lambda scale: (torch.randn((rows, cols), generator=gen) * scale).to(dtype)  # noqa: E731
    size = torch.exp2(torch.randint(-6, 6, (rows, 1), generator=gen).float())
    return make(size), make(size), make(0.1), make(0.1), 1 + 0.3 * torch.randn(cols, generator=gen)


def within(got, want, tol):
    off = np.abs(f64(got) - want)
    assert (off <= tol).all(), (off / tol).max()


def check_forward(got, x, residual, gamma, dtype):
    y, s, rstd = got
    want, sum64, rstd64 = R.rms_norm(f64(x), None if residual is None else f64(residual), None if gamma is None else f64(gamma), EPS, dtype)
    cols = x.shape[-1]
    assert np.array_equal(f64(s), sum64)
    within(rstd, rstd64, rstd64 * R.rstd_tolerance(cols))
    if y is not None:
        within(y, want, R.norm_tolerance(want, cols) + R.rounding(want, dtype))
    return want, sum64, rstd64


def check_backward(got, s, dy, rstd, gamma, dsum, dtype):
    args = [None if t is None else f64(t) for t in (s, dy, rstd, gamma, dsum)]
    dx, dgamma = R.rms_norm_backward(*args)
    tol_dx, tol_gamma = R.backward_tolerance(*args, dx, dtype)
    within(got[0], dx, tol_dx)
    within(got[1], dgamma, tol_gamma)


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("joined", [False, True], ids=["alone", "residual"])
def test_forward_and_backward(lib, cols, dtype, joined):
    x, residual, dy, dsum, gamma = (t.cuda() for t in data(rows_for(cols), cols, dtype))
    residual, dsum = (residual, dsum) if joined else (None, None)
    y, s, rstd = lib.rms_norm_forward(x, gamma, residual, EPS)
    assert (s is x) == (not joined)
    check_forward((y, s, rstd), x, residual, gamma, dtype)
    check_backward(lib.rms_norm_backward(s, dy, rstd, gamma, dsum), s, dy, rstd, gamma, dsum, dtype)


@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 63, 513, 2049, 40000])
@pytest.mark.parametrize("cols", [24, 200, 700])
def test_numbers_of_rows(lib, rows, cols):
    x, residual, dy, dsum, gamma = (t.cuda() for t in data(rows, cols, torch.bfloat16))
    got = lib.rms_norm_forward(x, gamma, residual, EPS)
    check_forward(got, x, residual, gamma, torch.bfloat16)
    check_backward(lib.rms_norm_backward(got[1], dy, got[2], gamma, dsum), got[1], dy, got[2], gamma, dsum, torch.bfloat16)


@pytest.mark.parametrize("cols", [1, 5, 128, 130, 384, 500, 1000, 2048, 4096, 9999, 16384, 30000, 65536, 70001])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("code", [E4M3, E5M2], ids=str)
def test_blocks(lib, cols, dtype, code):
    """As an operand: scales that hold the block and no larger ones, values off by half a code step at most."""
    rows = rows_for(cols)
    x, residual, _, _, gamma = (t.cuda() for t in data(rows, cols, dtype))
    blocks, s, rstd = lib.rms_norm_forward(x, gamma, residual, EPS, blocks=code)
    want, _, _ = check_forward((None, s, rstd), x, residual, gamma, dtype)
    tol = R.norm_tolerance(want, cols)
    codes, scales = f64(blocks.codes.float()), blocks.scales.cpu().numpy()
    assert blocks.shape == (rows, cols) and not blocks.square
    assert (codes[:, cols:] == 0).all() and (scales[:, rows:] == 0).all()
    e = scales[:, :rows].T.astype(np.float64) - 127
    full = np.zeros(codes.shape)
    full[:, :cols] = np.abs(want)
    most = full.reshape(rows, -1, 128).max(axis=2)
    loose = R.rstd_tolerance(cols) + 4 * R.EPS32
    top = R.TOP[code]
    assert (most <= top * np.exp2(e) * (1 + loose)).all()
    assert ((most >= top * np.exp2(e - 1) * (1 - loose)) | (e == -126)).all()
    half, small = (2.0 ** -4, 2.0 ** -10) if code == E4M3 else (2.0 ** -3, 2.0 ** -17)
    step = np.repeat(np.exp2(e), 128, axis=1)[:, :cols]
    within(lib.block8_unpack(blocks), want, np.maximum(np.abs(want) * half, step * small) + tol * (1 + half))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("cols", [100, 1000, 40000])
def test_strides_shapes_and_places(lib, dtype, cols):
    rows = 6
    x, residual, dy, dsum, gamma = (t.cuda() for t in data(rows, cols, dtype))
    y, s, rstd = lib.rms_norm_forward(x, gamma, residual, EPS)
    dx, dgamma = lib.rms_norm_backward(s, dy, rstd, gamma, dsum)

    def wide(t, at):
        room = torch.full((rows, cols + 21), 7.0, dtype=dtype, device="cuda")
        room[:, at:at + cols] = t
        return room[:, at:at + cols]

    a = lib.rms_norm_forward(wide(x, 1), gamma, wide(residual, 2), EPS, out=wide(x, 3), out_sum=wide(x, 5))
    assert all(torch.equal(p, q) for p, q in zip(a, (y, s, rstd)))
    b = lib.rms_norm_backward(wide(s, 1), wide(dy, 9), rstd, gamma, wide(dsum, 4), out=wide(x, 7))
    assert torch.equal(b[0], dx) and torch.equal(b[1], dgamma)
    # [..][cols] of any shape
    c = lib.rms_norm_forward(x.view(2, 3, cols), gamma, residual.view(2, 3, cols), EPS)
    assert c[0].shape == (2, 3, cols) and torch.equal(c[0].view(rows, cols), y)
    # in place: y for x and the sum for the residual, the other way round, the sum for x
    for out, out_sum in ((0, 1), (1, 0), (None, 0), (None, 1), (0, None), (1, None)):
        places = [x.clone(), residual.clone()]
        got = lib.rms_norm_forward(places[0], gamma, places[1], EPS, out=None if out is None else places[out],
                                   out_sum=None if out_sum is None else places[out_sum])
        assert all(torch.equal(p, q) for p, q in zip(got, (y, s, rstd))), (out, out_sum)
    alone = lib.rms_norm_forward(x, gamma, eps=EPS)[0]
    place = x.clone()
    assert torch.equal(lib.rms_norm_forward(place, gamma, eps=EPS, out=place)[0], alone)
    for k in range(3):
        places = [s.clone(), dy.clone(), dsum.clone()]
        got = lib.rms_norm_backward(places[0], places[1], rstd, gamma, places[2], out=places[k])
        assert torch.equal(got[0], dx) and torch.equal(got[1], dgamma), k


@pytest.mark.parametrize("cols", [40, 40000])
def test_without_gamma(lib, cols):
    x, residual, dy, _, _ = (t.cuda() for t in data(9, cols, torch.float32))
    got = lib.rms_norm_forward(x, None, residual, EPS)
    check_forward(got, x, residual, None, torch.float32)
    check_backward(lib.rms_norm_backward(got[1], dy, got[2], None), got[1], dy, got[2], None, None, torch.float32)


@pytest.mark.parametrize("cols", [40, 600, 5000, 70000])
def test_rows_of_zeros_infinities_and_nans(lib, cols):
    """A row of zeros is zeros; a bad row does not touch its neighbours."""
    x, _, dy, _, gamma = (t.cuda() for t in data(5, cols, torch.float32))
    clean = lib.rms_norm_forward(x, gamma, eps=EPS)
    bad = x.clone()
    bad[1], bad[2, cols // 2], bad[3, 0] = 0, float("inf"), float("nan")
    y, _, rstd = lib.rms_norm_forward(bad, gamma, eps=EPS)
    assert torch.equal(y[[0, 4]], clean[0][[0, 4]]) and (y[1] == 0).all()
    assert abs(rstd[1].item() - EPS ** -0.5) < 1e-4 * EPS ** -0.5
    assert y[2, cols // 2].isnan() and y[3].isnan().all() and rstd[2] == 0 and rstd[3].isnan()
    blocks = lib.rms_norm_forward(bad, gamma, eps=EPS, blocks=E4M3)[0]
    got = lib.block8_unpack(blocks)
    block = cols // 2 // 128 * 128
    assert got[2, block:block + 128].isnan().all() and got[3].isnan().all() and not got[[0, 1, 4]].isnan().any()


def test_gradients_against_differences(lib):
    """Of sum(w y) + sum(v s), along random directions, in 64 bits of the reference, which the kernels are held to elsewhere; and the
    kernel's own gradient along the same directions."""
    rows, cols, step = 3, 50, 1e-5
    x, residual, dy, dsum, gamma = (t.double() for t in data(rows, cols, torch.float32))
    gen = torch.Generator().manual_seed(5)
    dirs = [torch.randn(t.shape, generator=gen).double() for t in (x, residual, gamma)]

    def loss(h):
        a, b, g = (t + h * d for t, d in zip((x, residual, gamma), dirs))
        s = a + b
        y = s / torch.sqrt((s * s).mean(1, keepdim=True) + EPS) * g
        return ((dy * y).sum() + (dsum * s).sum()).item()

    slope = (loss(step) - loss(-step)) / (2 * step)
    x, residual, dy, dsum, gamma = (t.float().cuda() for t in (x, residual, dy, dsum, gamma))
    _, s, rstd = lib.rms_norm_forward(x, gamma, residual, EPS)
    dx, dgamma = lib.rms_norm_backward(s, dy, rstd, gamma, dsum)
    along = (dx.double().cpu() * (dirs[0] + dirs[1])).sum().item() + (dgamma.double().cpu() * dirs[2]).sum().item()
    scale = (dx.double().cpu().abs() * (dirs[0] + dirs[1]).abs()).sum().item() + (dgamma.double().cpu().abs() * dirs[2].abs()).sum().item()
    assert abs(along - slope) < 1e-5 * scale  # float32 roundings, and the difference's own step^2


def test_no_rows(lib):
    x, rstd, gamma = torch.zeros((0, 9), device="cuda"), torch.zeros(0, device="cuda"), torch.ones(9, device="cuda")
    y, s, r = lib.rms_norm_forward(x, gamma, x)
    assert y.shape == s.shape == (0, 9) and r.shape == (0,)
    assert lib.rms_norm_forward(x, gamma, blocks=E4M3)[0].shape == (0, 9)
    dx, dgamma = lib.rms_norm_backward(x, x, rstd, gamma)
    assert dx.shape == (0, 9) and torch.equal(dgamma, torch.zeros(9, device="cuda"))


def test_captured_and_replayed(lib):
    sets = [[t.cuda() for t in data(rows, cols, torch.bfloat16)] for rows, cols in ((700, 384), (40, 4096), (3, 70000))]

    def run():
        out = []
        for x, residual, dy, dsum, gamma in sets:
            y, s, rstd = lib.rms_norm_forward(x, gamma, residual, EPS)
            blocks = lib.rms_norm_forward(x, gamma, residual, EPS, blocks=E4M3)[0]
            out += [y, s, rstd, lib.block8_unpack(blocks), *lib.rms_norm_backward(s, dy, rstd, gamma, dsum)]
        return out

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = run()
    for turn in range(4):
        for x, residual, dy, dsum, gamma in sets:
            for t in (x, dy, gamma):
                t.mul_(-1.25)
        graph.replay()
        eager = run()
        torch.cuda.synchronize()
        assert all(torch.equal(c, e) for c, e in zip(captured, eager)), turn


def test_on_another_stream(lib):
    x, residual, dy, dsum, gamma = (t.cuda() for t in data(100, 700, torch.bfloat16))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    y, s, rstd = lib.rms_norm_forward(x, gamma, residual, EPS, stream=side)
    dx, dgamma = lib.rms_norm_backward(s, dy, rstd, gamma, dsum, stream=side)
    side.synchronize()
    here = lib.rms_norm_forward(x, gamma, residual, EPS)
    assert all(torch.equal(p, q) for p, q in zip((y, s, rstd), here))
    assert all(torch.equal(p, q) for p, q in zip((dx, dgamma), lib.rms_norm_backward(s, dy, rstd, gamma, dsum)))


@pytest.mark.parametrize("cols", [1, 8, 129, 384, 777, 1024, 2049, 8192, 20000, 65536, 70001])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_squares_past_float32(lib, cols, dtype):
    """Rows of numbers from 2^55 to just under 2^128, among ordinary ones."""
    gen = torch.Generator().manual_seed(cols)
    x = (torch.rand((37, cols), generator=gen) + 0.5) * torch.where(torch.rand((37, cols), generator=gen) < 0.5, -1.0, 1.0)
    x = (x * torch.exp2(torch.tensor([0.0, 55, 60, 63, 64, 65, 100, 126, 127] * 5)[:37, None] * 0.999)).to(dtype)
    assert x.isfinite().all()
    gamma = torch.rand(cols, generator=gen) + 0.5
    want, _, _ = check_forward(lib.rms_norm_forward(x.cuda(), gamma.cuda(), None, EPS), x, None, gamma, dtype)
    y = lib.block8_unpack(lib.rms_norm_forward(x.cuda(), gamma.cuda(), None, EPS, blocks=torch.float8_e4m3fn)[0])
    # eight steps of a code to each power of two
    within(y, want, np.abs(want) * 2.0 ** -4 + R.norm_tolerance(want, cols) * 2 + np.abs(want).max(1, keepdims=True) * 2.0 ** -17)
