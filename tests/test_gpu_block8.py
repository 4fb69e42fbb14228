"""Operands in 8-bit floating point: codes, scales and values exactly as the definition has them, and their products."""
import numpy as np
import pytest
import torch

import dense8_reference as R
from dense8_reference import f64

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2
CODES = [E4M3, E5M2]


def matrix(rows, cols, dtype=torch.float32, seed=0, spread=9):
    gen = torch.Generator().manual_seed(1000 * rows + cols + seed)
    x = torch.randn((rows, cols), generator=gen) * torch.exp2(torch.randint(-spread, spread, (rows, 1), generator=gen).float())
    x[torch.rand((rows, cols), generator=gen) < 0.2] = 0
    return x.to(dtype)


def same(blocks, want):
    codes, scales = want
    return (np.array_equal(f64(blocks.codes.float()), codes) and np.array_equal(blocks.scales.cpu().numpy(), scales))


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 128), (3, 129), (5, 7), (127, 255), (128, 128), (130, 64), (257, 300), (2, 1000), (1001, 3), (385, 512)])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("code", CODES, ids=str)
@pytest.mark.parametrize("square", [False, True], ids=["rows", "square"])
def test_pack_and_unpack(lib, rows, cols, dtype, code, square):
    x = matrix(rows, cols, dtype, spread=9 if dtype != torch.float16 else 5)
    want, turned = R.pack(f64(x), code, square), R.pack(f64(x).T, code, square)
    by_rows, by_columns = lib.block8_pack(x.cuda(), code, square, "both")
    assert same(by_rows, want) and same(by_columns, turned)
    assert by_rows.shape == (rows, cols) and by_columns.shape == (cols, rows)
    assert same(lib.block8_pack(x.cuda(), code, square), want) and same(lib.block8_pack(x.cuda(), code, square, "columns"), turned)
    if square:
        assert np.array_equal(R.values(*want, cols, True), R.values(*turned, rows, True).T)
    exact = R.values(*want, cols, square)
    for out in TYPES:
        assert torch.equal(lib.block8_unpack(by_rows, out).cpu(), torch.from_numpy(exact).to(out)), out
    assert torch.equal(lib.block8_unpack(by_columns).cpu().double(), torch.from_numpy(R.values(*turned, rows, square)))


@pytest.mark.parametrize("code", CODES, ids=str)
@pytest.mark.parametrize("square", [False, True], ids=["rows", "square"])
def test_extremes(lib, code, square):
    """Largest values on either side of a power of two's reach, ties, the largest and smallest numbers."""
    top = R.TOP[code]
    rows = []
    for e in (-149, -140, -127, -126, -118, -117, -60, 0, 100):
        for most in (1.0, 1.75, np.nextafter(np.float32(1.75), np.float32(9)), 1.9999999):
            row = np.linspace(-1, 1, 200) * most
            row[0], row[5], row[6] = most, 0.0, -0.0
            rows.append(np.ldexp(row, e))
    rows.append(np.full(200, np.finfo(np.float32).max))
    rows.append(np.zeros(200))
    ties = (np.arange(200) % 13 + 16.5) / 32
    ties[0] = ties[128] = top
    rows.append(ties)
    x = torch.from_numpy(np.array(rows)).float()
    if square:  # a row of its own to each block
        x = torch.cat([torch.nn.functional.pad(r[None], (0, 0, 0, 127)) for r in x])
    by_rows, by_columns = lib.block8_pack(x.cuda(), code, square, "both")
    assert same(by_rows, R.pack(f64(x), code, square)) and same(by_columns, R.pack(f64(x).T, code, square))


@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("square", [False, True], ids=["rows", "square"])
def test_infinities_and_nans_mark_their_block(lib, bad, square):
    x = matrix(260, 300)
    x[129, 130] = bad
    by_rows, by_columns = lib.block8_pack(x.cuda(), E4M3, square, "both")
    assert same(by_rows, R.pack(f64(x), E4M3, square)) and same(by_columns, R.pack(f64(x).T, E4M3, square))
    got = lib.block8_unpack(by_rows).cpu().isnan()
    want = torch.zeros_like(got)
    want[(128 if square else 129):(256 if square else 130), 128:256] = True
    assert torch.equal(got, want)
    # and a product has them where that block counts
    y = lib.block8_product(by_rows, lib.block8_pack(matrix(70, 300).cuda())).cpu().isnan()
    assert torch.equal(y, want.any(1)[:, None].expand(260, 70))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("code", CODES, ids=str)
@pytest.mark.parametrize("square", [False, True], ids=["rows", "square"])
def test_every_16_bit_number_packs_as_its_float32_does(lib, dtype, code, square):
    """Sorted, so that blocks are of neighbours, and shuffled with the largest ones left out of most blocks."""
    numbers = torch.arange(-2**15, 2**15, dtype=torch.int32).to(torch.int16)
    order = torch.randperm(2**16, generator=torch.Generator().manual_seed(5))
    for x in (numbers, numbers[order], numbers[torch.argsort(numbers.view(dtype).float().abs() // 1 + order % 7)]):
        x = x.view(dtype).view(512, 128)
        for got, want in zip(lib.block8_pack(x.cuda(), code, square, "both"), lib.block8_pack(x.cuda().float(), code, square, "both")):
            assert torch.equal(got.codes.view(torch.uint8), want.codes.view(torch.uint8)) and torch.equal(got.scales, want.scales)
    # and the float32's are the definition's
    by_rows, by_columns = lib.block8_pack(x.cuda().float(), code, square, "both")
    assert same(by_rows, R.pack(f64(x), code, square)) and same(by_columns, R.pack(f64(x).T, code, square))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_strided_and_unaligned(lib, dtype):
    wide = matrix(70, 333, dtype, spread=4).cuda()
    for x in (wide[:, 5:205], wide[3:, 1:], wide.view(7, 10, 333)[..., :129]):
        flat = f64(x.reshape(-1, x.shape[-1]))
        by_rows, by_columns = lib.block8_pack(x, E4M3, along="both")
        assert same(by_rows, R.pack(flat, E4M3)) and same(by_columns, R.pack(flat.T, E4M3))
    out = torch.full((70, 333), 7.0, dtype=dtype, device="cuda")
    blocks = lib.block8_pack(wide[:, 5:205], E5M2)
    lib.block8_unpack(blocks, dtype, out=out[:, 9:209])
    assert torch.equal(out[:, 9:209], lib.block8_unpack(blocks, dtype)) and (out[:, :9] == 7).all() and (out[:, 209:] == 7).all()


def product_case(lib, m, n, k, dtype, ca, cb, sa, sb, seed=0):
    x, w = matrix(m, k, seed=seed, spread=3).cuda(), matrix(n, k, seed=seed + 1, spread=3).cuda()
    a, b = lib.block8_pack(x, ca, sa), lib.block8_pack(w, cb, sb)
    va, vb = f64(lib.block8_unpack(a)), f64(lib.block8_unpack(b))
    return a, b, va, vb


def close(y, va, vb, dtype):
    want = va @ vb.T
    off, tol = np.abs(f64(y) - want), R.product_tolerance(va, vb, want, dtype)
    assert y.dtype == dtype and (off <= tol).all(), (off / tol).max()


@pytest.mark.parametrize("m,n,k", R.PRODUCT_SIZES)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_product(lib, m, n, k, dtype):
    which = m + n + k
    ca, cb, sa, sb = CODES[which % 2], CODES[which // 2 % 2], bool(which // 4 % 2), bool(which // 8 % 2)
    a, b, va, vb = product_case(lib, m, n, k, dtype, ca, cb, sa, sb)
    close(lib.block8_product(a, b, dtype), va, vb, dtype)


@pytest.mark.parametrize("m,n,k", R.PRODUCT_SIZES + [(70, 66, 20000), (3, 5, 40000)])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_products_of_small_whole_numbers_are_exact(lib, m, n, k, dtype):
    """Sums that no arithmetic rounds: every value of the operands counts once, whatever the kernel."""
    gen = torch.Generator().manual_seed(m + n + k)
    x, w = (torch.randint(-4, 5, (r, k), generator=gen).float() for r in (m, n))
    y = (x.double() @ w.double().t()) / 4
    for code, square in ((E4M3, False), (E5M2, True)):
        a, b = lib.block8_pack(x.cuda() / 2, code, square), lib.block8_pack(w.cuda() / 2, E4M3, not square)
        assert torch.equal(lib.block8_product(a, b, dtype).cpu(), y.to(dtype)), (code, square)


@pytest.mark.parametrize("m,n,k", R.PRODUCT_KINDS)
@pytest.mark.parametrize("ca", CODES, ids=str)
@pytest.mark.parametrize("cb", CODES, ids=str)
@pytest.mark.parametrize("sa", [False, True], ids=["rows", "square"])
@pytest.mark.parametrize("sb", [False, True], ids=["rows", "square"])
def test_product_of_all_kinds(lib, m, n, k, ca, cb, sa, sb):
    a, b, va, vb = product_case(lib, m, n, k, torch.float32, ca, cb, sa, sb)
    for dtype in (torch.float32, torch.bfloat16):
        close(lib.block8_product(a, b, dtype), va, vb, dtype)


@pytest.mark.parametrize("m,n", [(3, 21), (129, 515), (300, 1000), (581, 2154), (4000, 4090)])
def test_every_code_under_many_scales(lib, m, n):
    """Operands of any bytes, not of packing alone."""
    k = 384
    gen = torch.Generator().manual_seed(m)
    for code, worst in ((E4M3, 127), (E5M2, 124)):
        def operand(rows):
            codes = torch.randint(0, 256, (rows, k), generator=gen, dtype=torch.uint8)
            codes[(codes & 127) >= worst] = 5  # no NaN and no infinity
            scales = torch.randint(100, 155, (3, -(-rows // 4) * 4), generator=gen, dtype=torch.uint8)
            blocks = lib.Blocks8(codes.view(code).cuda(), scales.cuda(), k)
            return blocks, R.values(f64(codes.view(code).float()), scales.numpy()[:, :rows], k)
        (a, va), (b, vb) = operand(m), operand(n)
        for dtype in (torch.float32, torch.bfloat16):
            close(lib.block8_product(a, b, dtype), va, vb, dtype)
        assert np.array_equal(f64(lib.block8_unpack(a)), va.astype(np.float32).astype(np.float64))


@pytest.mark.parametrize("m,n,k", [(9, 20, 300), (129, 515, 1001), (300, 1000, 260), (257, 4149, 131), (4204, 40, 1039), (642, 776, 4320), (4000, 4090, 128)])
def test_product_writes_its_result_and_nothing_else(lib, m, n, k):
    a, b, va, vb = product_case(lib, m, n, k, torch.bfloat16, E4M3, E4M3, False, True)
    room = torch.full((m + 2, n + 11), 7.0, dtype=torch.bfloat16, device="cuda")
    out = room[1:-1, 3:n + 3]
    assert lib.block8_product(a, b, out=out) is out
    assert torch.equal(out, lib.block8_product(a, b))  # bit for bit, each time
    out.fill_(7.0)
    assert (room == 7).all()


def test_empty(lib):
    x = torch.zeros((0, 5), device="cuda")
    by_rows, by_columns = lib.block8_pack(x, along="both")
    assert by_rows.shape == (0, 5) and by_columns.shape == (5, 0)
    w = lib.block8_pack(matrix(3, 5).cuda())
    assert lib.block8_product(by_rows, w).shape == (0, 3) and lib.block8_product(w, by_rows).shape == (3, 0)
    # the weight gradient of no rows
    dy = lib.block8_pack(torch.zeros((0, 70), device="cuda"), along="columns")
    assert torch.equal(lib.block8_product(dy, by_columns, torch.float32), torch.zeros((70, 5), device="cuda"))
    assert lib.block8_unpack(by_rows).shape == (0, 5)


def test_a_layer_and_its_gradients(lib):
    """Forward, data gradient and weight gradient of a dense layer against 64 bits of the packed operands, and against the layer itself
    by what packing moved."""
    rows, cols, out = 300, 260, 200
    x, w, dy = matrix(rows, cols, torch.bfloat16, 1, 1).cuda(), matrix(out, cols, seed=2, spread=1).cuda(), matrix(rows, out, torch.bfloat16, 3, 1).cuda()
    (qx, qx_t), (qw, qw_t), (qd, qd_t) = (lib.block8_pack(x, E4M3, along="both"), lib.block8_pack(w, E4M3, True, "both"),
                                          lib.block8_pack(dy, E5M2, along="both"))
    v = {id(q): f64(lib.block8_unpack(q)) for q in (qx, qx_t, qw, qw_t, qd, qd_t)}
    assert np.array_equal(v[id(qw)], v[id(qw_t)].T)
    for a, b, ta, tb in ((qx, qw, f64(x), f64(w)), (qd, qw_t, f64(dy), f64(w).T), (qd_t, qx_t, f64(dy).T, f64(x).T)):
        y = lib.block8_product(a, b, torch.float32)
        close(y, v[id(a)], v[id(b)], torch.float32)
        moved_a, moved_b = np.abs(v[id(a)] - ta), np.abs(v[id(b)] - tb)  # by packing
        tol = moved_a @ np.abs(tb).T + np.abs(ta) @ moved_b.T + moved_a @ moved_b.T
        assert (np.abs(f64(y) - ta @ tb.T) <= tol + R.product_tolerance(v[id(a)], v[id(b)], f64(y), torch.float32)).all()


def test_captured_and_replayed(lib):
    """Packing and products of every kind in one graph over static buffers, replayed with other inputs, eager work between."""
    sizes = [(3, 200, 300), (642, 776, 4320), (4000, 4090, 130)]
    xs = [matrix(m, k).cuda() for m, n, k in sizes]
    ws = [matrix(n, k).cuda() for m, n, k in sizes]

    def run():
        return [lib.block8_product(lib.block8_pack(x), lib.block8_pack(w, E5M2, True)) for x, w in zip(xs, ws)]

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = run()
    for turn in range(4):
        for t in xs + ws:
            t.mul_(-1.5)
        graph.replay()
        eager = run()
        torch.cuda.synchronize()
        assert all(torch.equal(c, e) for c, e in zip(captured, eager)), turn


def test_on_another_stream(lib):
    side = torch.cuda.Stream()
    x, w = matrix(130, 2600).cuda(), matrix(140, 2600).cuda()
    torch.cuda.synchronize()
    a, b = lib.block8_pack(x, stream=side), lib.block8_pack(w, stream=side)
    y = lib.block8_product(a, b, stream=side)
    v = lib.block8_unpack(a, stream=side)
    side.synchronize()
    assert torch.equal(y, lib.block8_product(a, b)) and torch.equal(v, lib.block8_unpack(lib.block8_pack(x)))
