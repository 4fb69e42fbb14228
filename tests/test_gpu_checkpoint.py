"""8-bit activation checkpoints: codes, scales and values exactly as the definition has them, and the dense weight gradient that
multiplies with them."""
import numpy as np
import pytest
import torch

import norm_reference as R

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
CODES = [torch.int8, torch.float8_e4m3fn]


def f64(t):
    return t.detach().double().cpu().numpy()


def numbers(kept):
    return f64(kept.codes.float())


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 31), (1, 32), (3, 33), (7, 37), (130, 64), (5, 100), (2, 9216), (3, 1037), (2001, 48), (9, 4096)])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("code", CODES, ids=str)
def test_pack_and_unpack(lib, rows, cols, dtype, code):
    gen = torch.Generator().manual_seed(rows + cols)
    x = (torch.randn((rows, cols), generator=gen) * torch.exp2(torch.randint(-9, 9, (rows, 1), generator=gen).float())).to(dtype)
    x[torch.rand((rows, cols), generator=gen) < 0.3] = 0
    want, scales = R.code(f64(x), code)
    kept = lib.checkpoint_pack(x.cuda(), code)
    assert np.array_equal(numbers(kept), want) and np.array_equal(kept.scales.cpu().numpy(), scales)
    values = R.decode(want, scales)
    # the nearest code is at most half a step away: half of 2^e for int8, 2^-4 of the value or half of 2^(e - 9) for e4m3
    step = np.repeat(np.exp2(scales - 127.0), 32, axis=1)[:, :cols]
    assert np.all(np.abs(values - f64(x)) <= (0.5 * step if code == torch.int8 else np.maximum(np.abs(f64(x)) / 16, step * 2.0 ** -10)))
    for out in TYPES:
        got = lib.checkpoint_unpack(kept, out)
        assert torch.equal(got.cpu(), torch.from_numpy(values).to(out)), out


@pytest.mark.parametrize("code", CODES, ids=str)
@pytest.mark.parametrize("cols", [64, 45])
def test_extremes(lib, code, cols):
    """Powers of two, ties, the largest and smallest numbers, zeros of either sign."""
    top = 127.0 if code == torch.int8 else 448.0
    rows = []
    for e in (-149, -140, -130, -127, -126, -120, -60, 0, 60, 120):
        for most in (1.0, 1.75, 1.984375, 1.9843751, 1.9999999, top / 64, np.nextafter(np.float32(top / 64), np.float32(9))):
            row = np.linspace(-1, 1, cols).astype(np.float64) * most
            row[0] = most
            row[5], row[6] = 0.0, -0.0
            rows.append(np.ldexp(row, e))
    rows.append(np.full(cols, np.finfo(np.float32).max))
    rows.append(np.zeros(cols))
    half = np.arange(cols) % 60 + 0.5
    half[0] = top  # scale 1: halves are ties
    half[32] = top
    rows.append(half)
    with np.errstate(over="ignore"):
        x = np.array(rows).astype(np.float32)
    x[~np.isfinite(x)] = np.finfo(np.float32).max
    want, scales = R.code(x.astype(np.float64), code)
    kept = lib.checkpoint_pack(torch.from_numpy(x).cuda(), code)
    assert np.array_equal(kept.scales.cpu().numpy(), scales)
    assert np.array_equal(numbers(kept), want)
    got = lib.checkpoint_unpack(kept, torch.float32)
    with np.errstate(over="ignore"):
        assert np.array_equal(got.cpu().numpy(), R.decode(want, scales).astype(np.float32))


@pytest.mark.parametrize("code", CODES, ids=str)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_a_block_that_is_not_finite(lib, code, dtype):
    for cols in (96, 70):
        x = torch.randn((4, cols)).to(dtype)
        clean = lib.checkpoint_unpack(lib.checkpoint_pack(x.cuda(), code), dtype)
        for i, bad in enumerate([float("nan"), float("inf"), float("-inf")]):
            x[i + 1, 32 + 5 * i] = bad
        kept = lib.checkpoint_pack(x.cuda(), code)
        got = lib.checkpoint_unpack(kept, dtype)
        assert bool((kept.scales[1:, 1] == 255).all()) and int((kept.scales == 255).sum()) == 3
        assert bool(torch.isnan(got[1:, 32:64]).all())
        got[1:, 32:64] = clean[1:, 32:64]
        assert torch.equal(got, clean)


def test_every_code_and_every_scale_reads_back(lib):
    """Checkpoints that other programs wrote may hold any byte: all 256 codes under all 256 scales."""
    for code in CODES:
        raw = torch.arange(256, dtype=torch.uint8).view(1, 256).repeat(256, 1)
        codes = raw.view(code)
        scales = torch.arange(256, dtype=torch.uint8).view(256, 1).repeat(1, 8)
        got = lib.checkpoint_unpack(lib.Checkpoint(codes.cuda(), scales.cuda())).cpu().numpy()
        s = np.where(np.arange(256) == 255, np.nan, np.exp2(np.arange(256) - 127.0))[:, None]
        with np.errstate(over="ignore"):
            want = (codes.float().numpy().astype(np.float64) * s).astype(np.float32)
        assert np.array_equal(got, want, equal_nan=True)


def test_slices(lib):
    for dtype in TYPES:
        wide = torch.randn((50, 100), device="cuda").to(dtype)
        for a, b in [(0, 64), (8, 72), (3, 60)]:
            kept = lib.checkpoint_pack(wide[:, a:b], torch.int8)
            alone = lib.checkpoint_pack(wide[:, a:b].contiguous(), torch.int8)
            assert torch.equal(kept.codes, alone.codes) and torch.equal(kept.scales, alone.scales)
            room = torch.full((50, 100), 3.0, dtype=dtype, device="cuda")
            lib.checkpoint_unpack(kept, dtype, out=room[:, a:b])
            assert torch.equal(room[:, a:b].contiguous(), lib.checkpoint_unpack(kept, dtype))
            assert bool((room[:, :a] == 3).all()) and bool((room[:, b:] == 3).all())


def test_nothing_to_do(lib):
    kept = lib.checkpoint_pack(torch.empty((0, 40), device="cuda"))
    assert kept.shape == (0, 40) and lib.checkpoint_unpack(kept).shape == (0, 40)
    dw, db = lib.checkpoint_fc_backward_weight(kept, torch.empty((0, 3), device="cuda"))
    assert dw.shape == (3, 40) and bool((dw == 0).all()) and bool((db == 0).all())


# ---- weight gradient ----
def weight_case(rows, cols, out, dtype, code, seed, ld=0):
    gen = torch.Generator().manual_seed(seed)
    x = torch.relu(torch.randn((rows, cols), generator=gen) + 0.2)
    dy = (torch.randn((rows, out + ld), generator=gen) * 0.1).to(dtype)[:, ld:]
    codes, scales = R.code(f64(x), code)
    return codes, scales, dy


def check_weight(lib, rows, cols, out, dtype, code, seed, ld=0):
    codes, scales, dy = weight_case(rows, cols, out, dtype, code, seed, ld)
    kept = lib.Checkpoint(torch.from_numpy(codes).to(torch.float32).to(code).cuda(), torch.from_numpy(scales).cuda())
    room = torch.full((rows, out + ld), float("nan"), dtype=dtype, device="cuda")
    room[:, ld:] = dy.cuda()
    dw, db = lib.checkpoint_fc_backward_weight(kept, room[:, ld:])
    x, d = R.decode(codes, scales), f64(dy)
    want, sums = d.T @ x, d.sum(0)
    # products are exact, or rounded once for terms of fp32; sums of `rows` terms: an accumulator is rounded at most once a
    # product and the slices' sums join in a few more additions
    k = (rows + 64) * R.EPS32
    tol, tol_b = k * (np.abs(d).T @ np.abs(x)) + 1e-38, k * np.abs(d).sum(0) + 1e-38
    assert np.all(np.abs(f64(dw) - want) <= tol), float(np.max(np.abs(f64(dw) - want) / tol))
    assert np.all(np.abs(f64(db) - sums) <= tol_b)
    # in the mean far less: random signs
    if rows >= 64:
        assert np.linalg.norm(f64(dw) - want) <= 2e-6 * np.linalg.norm(want)


@pytest.mark.parametrize("rows,cols,out", [(1, 1, 1), (1, 32, 8), (2, 37, 5), (16, 256, 10), (31, 64, 64), (33, 100, 130), (64, 128, 128),
                                           (128, 200, 136), (100, 9216, 16), (257, 48, 300), (1000, 64, 96), (5000, 72, 40),
                                           (20000, 33, 17), (4097, 256, 256), (3, 1000, 1000)])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_weight_gradient(lib, rows, cols, out, dtype):
    for i, code in enumerate(CODES):
        check_weight(lib, rows, cols, out, dtype, code, rows + i)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_weight_gradient_of_a_slice(lib, dtype):
    for ld in (1, 8):
        check_weight(lib, 200, 96, 48, dtype, torch.int8, 3, ld)


def test_weight_gradient_range(lib):
    """Rows of very different sizes, and numbers near both ends of float32."""
    rows, cols, out = 40, 64, 32
    gen = torch.Generator().manual_seed(8)
    x = torch.randn((rows, cols), generator=gen)
    for scale in (1e-36, 1e30):
        dy = (torch.randn((rows, out), generator=gen) * scale).cuda()
        kept = lib.checkpoint_pack(x.cuda(), torch.int8)
        dw, db = lib.checkpoint_fc_backward_weight(kept, dy)
        values = f64(lib.checkpoint_unpack(kept))
        want, size = f64(dy).T @ values, np.abs(f64(dy)).T @ np.abs(values)
        assert np.all(np.abs(f64(dw) - want) <= (rows + 64) * R.EPS32 * size + 2.0 ** -126)
        assert np.all(np.abs(f64(db) - f64(dy).sum(0)) <= (rows + 64) * R.EPS32 * np.abs(f64(dy)).sum(0) + 2.0 ** -126)


def test_weight_gradient_shows_what_is_not_finite(lib):
    rows, cols, out = 70, 96, 40
    x = torch.rand((rows, cols)) + 0.5
    dy = torch.randn((rows, out))
    kept = lib.checkpoint_pack(x.cuda())
    clean, clean_b = lib.checkpoint_fc_backward_weight(kept, dy.cuda())
    dy[9, 4], dy[50, 30] = float("inf"), float("nan")
    dw, db = lib.checkpoint_fc_backward_weight(kept, dy.cuda())
    assert bool(torch.isinf(dw[4]).all()) and bool(torch.isnan(dw[30]).all())
    assert bool(torch.isinf(db[4])) and bool(torch.isnan(db[30]))
    rest = [i for i in range(out) if i not in (4, 30)]
    assert torch.equal(dw[rest], clean[rest]) and torch.equal(db[rest], clean_b[rest])
    x[3, 40] = float("inf")  # the block's columns
    dw, _ = lib.checkpoint_fc_backward_weight(lib.checkpoint_pack(x.cuda()), dy.cuda())
    assert bool(torch.isnan(dw[:, 32:64]).all()) and torch.equal(dw[rest][:, :32], clean[rest][:, :32])
    assert torch.equal(dw[rest][:, 64:], clean[rest][:, 64:])


def test_weight_gradient_of_a_tiny_dy(lib):
    """Under 2^-126 down to nothing: what a float32 has under 2^-133 is left off, bfloat16 and float16 lose nothing."""
    rows, cols, out = 48, 64, 32
    gen = torch.Generator().manual_seed(12)
    x = (torch.randn((rows, cols), generator=gen) * 2.0 ** 40).cuda()
    kept = lib.checkpoint_pack(x, torch.int8)
    values = f64(lib.checkpoint_unpack(kept))
    for dtype, scale, lost in ((torch.float32, 2.0 ** -128, 2.0 ** -133), (torch.bfloat16, 2.0 ** -128, 0.0), (torch.float16, 2.0 ** -20, 0.0)):
        dy = (torch.randn((rows, out), generator=gen).double() * scale).to(dtype).cuda()
        dw, _ = lib.checkpoint_fc_backward_weight(kept, dy)
        want, size = f64(dy).T @ values, np.abs(f64(dy)).T @ np.abs(values)
        assert np.all(np.abs(f64(dw) - want) <= (rows + 64) * R.EPS32 * size + lost * np.abs(values).sum(0))
        assert np.linalg.norm(want) > 0


@pytest.mark.parametrize("code", CODES, ids=str)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,cols,out", [(70, 96, 40), (300, 1030, 257)])
def test_weight_gradient_of_what_is_not_finite(lib, code, dtype, rows, cols, out):
    """An infinity or a NaN of dy reaches its own row of dw, a block that is not finite its own columns, and nothing else."""
    gen = torch.Generator().manual_seed(rows)
    x, dy = torch.rand((rows, cols), generator=gen) + 0.5, torch.randn((rows, out), generator=gen).to(dtype)
    clean, clean_b = lib.checkpoint_fc_backward_weight(lib.checkpoint_pack(x.cuda(), code), dy.cuda())
    dy[0, 1], dy[rows - 1, out - 1] = float("-inf"), float("nan")
    x[rows - 2, cols - 1] = float("nan")
    dw, db = lib.checkpoint_fc_backward_weight(lib.checkpoint_pack(x.cuda(), code), dy.cuda())
    last = (cols - 1) // 32 * 32  # the block
    assert bool((dw[1, :last] == float("-inf")).all()) and bool(torch.isnan(dw[out - 1]).all()) and bool(torch.isnan(dw[:, last:]).all())
    assert float(db[1]) == float("-inf") and bool(torch.isnan(db[out - 1]))
    rest = [i for i in range(out) if i not in (1, out - 1)]
    assert torch.equal(dw[rest, :last], clean[rest, :last]) and torch.equal(db[rest], clean_b[rest])


def test_more_codes_than_32_bits_count(lib):
    """The last rows of the longest checkpoint: only they have a gradient."""
    rows, cols, out, tail = 1 << 22, 1030, 5, 40
    gen = torch.Generator().manual_seed(6)
    x = torch.randn((tail, cols), generator=gen)
    some = lib.checkpoint_pack(x.cuda(), torch.int8)
    codes = torch.ones((rows, cols), dtype=torch.int8, device="cuda")
    scales = torch.full((rows, some.scales.shape[1]), 127, dtype=torch.uint8, device="cuda")
    codes[-tail:], scales[-tail:] = some.codes, some.scales
    kept = lib.Checkpoint(codes, scales)
    dy = torch.zeros((rows, out), device="cuda")
    dy[-tail:] = torch.randn((tail, out), generator=gen).cuda()
    dw, db = lib.checkpoint_fc_backward_weight(kept, dy)
    values, d = f64(lib.checkpoint_unpack(some)), f64(dy[-tail:])
    k = (tail + 64) * R.EPS32
    assert np.all(np.abs(f64(dw) - d.T @ values) <= k * (np.abs(d).T @ np.abs(values)))
    assert np.all(np.abs(f64(db) - d.sum(0)) <= k * np.abs(d).sum(0))
    back = lib.checkpoint_unpack(kept, torch.bfloat16)
    assert torch.equal(back[-tail:], lib.checkpoint_unpack(some, torch.bfloat16)) and bool((back[:tail] == 1).all())
    again = lib.checkpoint_pack(back, torch.int8)
    same = lib.checkpoint_pack(back[-tail:], torch.int8)
    assert torch.equal(again.codes[-tail:], same.codes) and torch.equal(again.scales[-tail:], same.scales)


def test_on_given_buffers_captured_and_on_another_stream(lib):
    gen = torch.Generator().manual_seed(2)
    x, dy = torch.randn((3000, 64), generator=gen).cuda(), torch.randn((3000, 48), generator=gen).cuda()
    dw, db = torch.empty((48, 64), device="cuda"), torch.empty(48, device="cuda")

    def step(stream=None, **to):
        return lib.checkpoint_fc_backward_weight(lib.checkpoint_pack(x, stream=stream), dy, stream=stream, **to)

    want = step()
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    other = step(st)
    torch.cuda.synchronize()
    assert torch.equal(other[0], want[0]) and torch.equal(other[1], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(dw=dw, db=db)
    for seed in range(3):
        x.copy_(torch.randn((3000, 64), generator=gen))
        dw.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        want = step()
        assert torch.equal(dw, want[0]) and torch.equal(db, want[1])
