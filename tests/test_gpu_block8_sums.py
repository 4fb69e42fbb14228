"""Products in 8 bits with 16-bit results whose sums are float32 throughout."""
import numpy as np
import pytest
import torch

import dense8_reference as R
from dense8_reference import EPS32, f64

pytestmark = pytest.mark.gpu

E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2
SIXTEEN = [torch.bfloat16, torch.float16]


def pairs(m, n, k):
    """Operands of neighbours a, -a and b, b with |a b| = 2^16 among products of a few units, and their exact product: every eight of a sum has
    terms 2^13 times smaller than its largest, and all sums, in any order, are whole numbers under 2^24."""
    gen = torch.Generator().manual_seed(m + n + k)
    x, w = (torch.randint(1, 4, (r, k), generator=gen).float() for r in (m, n))
    for at in (0, 4):
        x[:, at:k - 1:8], x[:, at + 1:k:8] = 256, -256
        w[:, at:k - 1:8] = w[:, at + 1:k:8] = 256
    return x, w, x.double() @ w.double().t()


@pytest.mark.parametrize("m,n,k", R.PRODUCT_SIZES)
@pytest.mark.parametrize("dtype", SIXTEEN, ids=str)
def test_full_sums(lib, m, n, k, dtype):
    """The float32 result, rounded once: within float32's part of the tolerance and half a step."""
    gen = torch.Generator(device="cuda").manual_seed(m + n + k)
    x, w = (torch.randn((r, k), generator=gen, device="cuda") for r in (m, n))
    a, b = lib.block8_pack(x, E4M3 if m % 2 else E5M2, bool(n % 2)), lib.block8_pack(w, E5M2 if n % 2 else E4M3, bool(m % 2))
    y = lib.block8_product(a, b, dtype, full_sums=True)
    assert y.dtype == dtype and torch.equal(y, lib.block8_product(a, b, torch.float32).to(dtype))
    va, vb = f64(lib.block8_unpack(a)), f64(lib.block8_unpack(b))
    want = va @ vb.T
    own = (104 + k / 64) * 2 * EPS32 * (np.abs(va) @ np.abs(vb).T)
    assert (np.abs(f64(y) - want) <= own + R.rounding(np.abs(want) + own, dtype)).all()


@pytest.mark.parametrize("m,n,k", [(3, 40, 700), (20, 40, 300), (64, 100, 960), (129, 515, 300), (300, 1000, 260), (257, 4149, 131), (1024, 1000, 250),
                                   (642, 776, 1000), (4000, 4090, 200)])
@pytest.mark.parametrize("dtype", SIXTEEN, ids=str)
def test_large_products_that_cancel(lib, m, n, k, dtype):
    x, w, y = pairs(m, n, k)
    a, b = lib.block8_pack(x.cuda(), E4M3), lib.block8_pack(w.cuda(), E5M2, True)
    assert torch.equal(lib.block8_product(a, b, torch.float32).cpu().double(), y)
    assert torch.equal(lib.block8_product(a, b, dtype, full_sums=True).cpu(), y.to(dtype))
    # without, each eight may lose seven times 2^-13 of its 2^16
    off = np.abs(f64(lib.block8_product(a, b, dtype)) - y.numpy())
    assert (off <= -(-k // 8) * 56 + R.rounding(y.numpy() + -(-k // 8) * 56, dtype)).all()


def test_strides_streams_and_replays(lib):
    x, w, y = pairs(200, 130, 900)
    a, b = lib.block8_pack(x.cuda()), lib.block8_pack(w.cuda(), square=True)
    want = y.to(torch.bfloat16).cuda()
    room = torch.full((202, 150), 7.0, dtype=torch.bfloat16, device="cuda")
    out = room[1:-1, 3:133]
    assert lib.block8_product(a, b, out=out, full_sums=True) is out and torch.equal(out, want)
    out.fill_(7.0)
    assert (room == 7).all()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    there = lib.block8_product(a, b, stream=side, full_sums=True)
    side.synchronize()
    assert torch.equal(there, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = lib.block8_product(a, b, full_sums=True)
    for _ in range(3):
        captured.fill_(7.0)
        graph.replay()
        assert torch.equal(captured, want) and torch.equal(lib.block8_product(a, b, full_sums=True), want)


def test_nothing_to_add(lib):
    a, b = lib.block8_pack(torch.zeros((0, 70), device="cuda"), along="columns"), lib.block8_pack(torch.zeros((0, 9), device="cuda"), along="columns")
    assert torch.equal(lib.block8_product(a, b, full_sums=True), torch.zeros((70, 9), dtype=torch.bfloat16, device="cuda"))


@pytest.mark.parametrize("m,n,k", [(1, 16, 128), (1, 1000, 960), (2, 17, 129), (9, 20, 300), (16, 130, 1000), (5, 5000, 512), (16, 4200, 700)])
@pytest.mark.parametrize("dtype", SIXTEEN, ids=str)
def test_few_rows_have_full_sums_anyway(lib, m, n, k, dtype):
    """Where memory is what counts nothing is won by fewer bits."""
    x, w, y = pairs(m, n, k)
    a, b = lib.block8_pack(x.cuda(), E5M2), lib.block8_pack(w.cuda(), E4M3, True)
    assert torch.equal(lib.block8_product(a, b, dtype).cpu(), y.to(dtype))
