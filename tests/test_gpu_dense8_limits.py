"""Dense layers in 8 bits, normalisation and clipping where places in a tensor pass 32 bits, and launches 2^32 threads.

Inputs repeat a few rows over and over, so that every result is held against that of its row's first time."""
import numpy as np
import pytest
import torch

import dense8_reference as R
from dense8_reference import EPS32, f64

pytestmark = pytest.mark.gpu

E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2


@pytest.fixture(autouse=True)
def memory():
    yield
    torch.cuda.empty_cache()


def need(gib):
    if torch.cuda.get_device_properties(0).total_memory < gib * 2**30:
        pytest.skip(f"needs {gib} GiB of device memory")


def repeats(x, times, every):
    """Whether x is `times` times its first `every` rows, bit for bit."""
    kind = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[x.element_size()]
    x = x.view(kind).view(times, every, *x.shape[1:])
    return all(torch.equal(x[i], x[0]) for i in range(1, times))


def matrix(rows, cols, dtype, seed):
    return torch.randn((rows, cols), generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_results_past_2_to_the_31(lib, dtype):
    need(32)
    times, every, n, k = 70, 1000, 33000, 130
    x, w = matrix(every, k, torch.float32, 1), matrix(n, k, torch.float32, 2)
    a, b = lib.block8_pack(x.repeat(times, 1)), lib.block8_pack(w, E5M2, True)
    y = lib.block8_product(a, b, dtype)
    assert y.numel() > 2**31 and repeats(y, times, every)
    va, vb = f64(lib.block8_unpack(a))[:40], f64(lib.block8_unpack(b))
    want = va @ vb.T
    assert (np.abs(f64(y[:40]) - want) <= R.product_tolerance(va, vb, want, dtype)).all()


@pytest.mark.parametrize("square", [False, True], ids=["rows", "square"])
def test_operands_past_2_to_the_31(lib, square):
    need(64)
    times, every, cols = 1100, 1024, 2000
    x = matrix(every, cols, torch.bfloat16, 3)
    by_rows, by_columns = lib.block8_pack(x.repeat(times, 1), E4M3, square, "both")
    assert by_rows.codes.numel() > 2**31 and by_columns.codes.numel() > 2**31
    small, turned = lib.block8_pack(x, E4M3, square, "both")
    per = every // 128 if square else every
    assert repeats(by_rows.codes, times, every) and torch.equal(by_rows.codes[:every].view(torch.uint8), small.codes.view(torch.uint8))
    assert torch.equal(by_rows.scales.view(-1, times, per), small.scales[:, None].expand(-1, times, per))
    assert torch.equal(by_columns.codes.view(torch.uint8).view(cols, times, every), turned.codes.view(torch.uint8)[:, None].expand(cols, times, every))
    assert torch.equal(by_columns.scales.view(times, every // 128, -1), turned.scales[None].expand(times, -1, -1))
    back = lib.block8_unpack(by_rows, torch.bfloat16)
    assert repeats(back, times, every) and torch.equal(back[:every], lib.block8_unpack(small, torch.bfloat16))
    del back
    back = lib.block8_unpack(by_columns, torch.bfloat16)
    assert torch.equal(back.view(cols, times, every), lib.block8_unpack(turned, torch.bfloat16)[:, None].expand(cols, times, every))
    del back
    for n in (20, 300):
        w = lib.block8_pack(matrix(n, cols, torch.float32, n), E4M3, True)
        for dtype in (torch.float32, torch.bfloat16):
            y = lib.block8_product(by_rows, w, dtype)
            va, vb = f64(lib.block8_unpack(small)), f64(lib.block8_unpack(w))
            want = va @ vb.T
            assert repeats(y, times, every), (n, dtype)
            assert (np.abs(f64(y[:every]) - want) <= R.product_tolerance(va, vb, want, dtype)).all(), (n, dtype)
            # the other way round they are b
            y = lib.block8_product(w, by_rows, dtype)
            assert torch.equal(y.view(n, times, every), y[:, None, :every].expand(n, times, every)), (n, dtype)
            assert (np.abs(f64(y[:, :every].T) - want) <= R.product_tolerance(va, vb, want, dtype)).all(), (n, dtype)


# 256 and 1024 threads to a row: as many rows as there may be, and as many as make 2^32 threads
@pytest.mark.parametrize("times,every,cols", [(2**14, 2**10, 2056), (2**13, 2**9, 16392)], ids=str)
def test_rms_norm_of_many_rows(lib, times, every, cols):
    need(200)
    small = matrix(every, cols, torch.bfloat16, cols)
    gamma = matrix(1, cols, torch.float32, 4)[0]
    y, _, rstd = lib.rms_norm_forward(small, gamma)
    x = small.repeat(times, 1)
    got, _, r = lib.rms_norm_forward(x, gamma, out=x)
    assert got is x and repeats(x, times, every) and torch.equal(x[:every], y) and torch.equal(r.view(times, every), rstd.expand(times, every))
    dx, dgamma = lib.rms_norm_backward(small, small, rstd, gamma)
    x.view(times, every, cols).copy_(small)
    got, many = lib.rms_norm_backward(x, x, r, gamma, out=x)
    assert got is x and repeats(x, times, every) and torch.equal(x[:every], dx)
    # the terms are those of `every` rows, added up in another order: a share of 2^15 rows one by one, 512 shares by eights and 64
    s = f64(small)
    sums = (s * s * f64(rstd)[:, None]).sum(0) * times  # all of one sign
    assert (np.abs(f64(many) - sums) <= (times * every / 512 + 80) * EPS32 * sums).all()


def test_clipping_past_2_to_the_31(lib):
    need(32)
    sizes, values = [5, 2**31 + 8195, 0, 2**20 + 1], [0.5, 0.25, 1.0, 0.75]
    grads = [torch.full((n,), v, dtype=t, device="cuda") for n, v, t in zip(sizes, values, [torch.float32, torch.bfloat16, torch.float32, torch.float16])]
    want = np.sqrt(sum(n * v * v for n, v in zip(sizes, values)))
    norm = lib.gradient_norm(grads)
    assert abs(norm.item() - want) <= 1.01 * EPS32 * want
    out = [torch.empty_like(g) for g in grads]
    for result in (out, None):  # a quarter of each value is of its type
        assert lib.clip_gradients(grads, want / 4, out=result) == norm
        for g, v in zip(out if result else grads, values):
            assert g.numel() == 0 or (g[0] == g).all() and abs(g[0].item() - v / 4) <= 4 * EPS32 * v
