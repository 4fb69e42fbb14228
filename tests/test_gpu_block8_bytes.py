"""Products in 8 bits of operands that hold any bytes: every scale, and what is not a number, in every kernel and every type of result."""
import pytest
import torch

import dense8_reference as R

pytestmark = pytest.mark.gpu

E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2
KINDS = [(torch.float32, False), (torch.bfloat16, False), (torch.bfloat16, True), (torch.float16, False), (torch.float16, True)]
FEW = [(9, 20, 300), (3, 40, 1500), (64, 4100, 400), (129, 515, 300), (300, 1000, 260), (33, 2100, 300)]  # rows of 16, 32 and 64
TILES = [(257, 4149, 131), (4204, 40, 1039), (40, 41, 42430), (642, 776, 4320), (1024, 1000, 1188), (4000, 4090, 200)]
PAIRS = [(E4M3, E5M2, False, True), (E5M2, E4M3, True, False), (E4M3, E4M3, True, True), (E5M2, E5M2, False, False)]


def codes(gen, rows, k, code, most=4.0):
    """Any codes of numbers up to `most`; zeros behind the columns."""
    c = torch.randint(0, 256, (rows, -(-k // 128) * 128), generator=gen, dtype=torch.uint8)
    c[(c & 127) > torch.tensor(most).to(code).view(torch.uint8)] &= 0x93
    c[:, k:] = 0
    return c.view(code)


def scales(gen, rows, square, at):
    """A byte for every block, 0 to 2 from that block's `at`, in bounds."""
    of_rows = -(-rows // 128) if square else -(-rows // 4) * 4
    return (at[:, None] + torch.randint(0, 3, (len(at), of_rows), generator=gen)).clamp(0, 254).to(torch.uint8)


def operand(lib, gen, rows, k, code, square, at):
    q = lib.Blocks8(codes(gen, rows, k, code).cuda(), scales(gen, rows, square, at).cuda(), k, square)
    each = torch.exp2(q.scales.double() - 127).t().repeat_interleave(128 if square else 1, 0)[:rows].repeat_interleave(128, 1)
    return q, (q.codes.double() * each)[:, :k]


def times(a, b):
    return a @ b.t().contiguous()


def tolerance(a, b, y, dtype, full):
    """What tests of products allow, in torch: see dense8_reference."""
    own = (104 + a.shape[1] / 64) * 2 * R.EPS32 + (0.0 if dtype == torch.float32 or full else 7 * 2.0 ** -13)
    size = own * times(a.abs(), b.abs())
    return size + (y.abs() + size) * R.HALF[dtype] * 1.01 + R.TINY[dtype] + 2.0 ** -126


@pytest.mark.parametrize("m,n,k", FEW + TILES)
@pytest.mark.parametrize("ca,cb,sa,sb", PAIRS)
def test_every_scale(lib, m, n, k, ca, cb, sa, sb):
    """Blocks from the smallest scales to the largest, against blocks whose scales bring the products near 1.  With float32 sums values are
    taken in bf16, so that scales end where every code under them is a number of bf16's."""
    gen = torch.Generator().manual_seed(m + n + k)
    few, blocks = (m, n, k) in FEW, -(-k // 128)
    for turn in range(3):
        low = torch.randint(0, 127, (blocks,), generator=gen)
        for any_scale, at in ((True, low), (False, low.clamp(min=17))):
            a, va = operand(lib, gen, m, k, ca, sa, at)
            b, vb = operand(lib, gen, n, k, cb, sb, 252 - at)
            for x, y, vx, vy in ((a, b, va, vb), (b, a, vb, va)):
                want = times(vx, vy)
                for dtype, full in KINDS:
                    if any_scale and (few or dtype == torch.float32 or full):
                        continue
                    got = lib.block8_product(x, y, dtype, full_sums=full)
                    off = (got.double() - want).abs()
                    assert (off <= tolerance(vx, vy, want, dtype, full)).all(), (turn, any_scale, dtype, full)


@pytest.mark.parametrize("m,n,k", FEW + TILES)
@pytest.mark.parametrize("ca,cb,sa,sb", PAIRS)
def test_small_values_of_float32_sums(lib, m, n, k, ca, cb, sa, sb):
    """Values under 2^-126 may be taken as the nearest multiple of 2^-133, and no others are: half of that, times the other operand."""
    few = (m, n, k) in FEW
    gen = torch.Generator().manual_seed(m + n + k)
    blocks = -(-k // 128)
    for least in (0, 10 if E5M2 in (ca, cb) else 3):
        a, va = operand(lib, gen, m, k, ca, sa, torch.full((blocks,), least))
        b, vb = operand(lib, gen, n, k, cb, sb, torch.full((blocks,), 236))
        want = times(va, vb)
        near = (torch.round(va * 2.0 ** 133) / 2.0 ** 133 - va).abs()
        assert (near > 0).any() == (least == 0) and (near <= 2.0 ** -134).all()
        lost = times(near, vb.abs())
        for dtype, full in KINDS:
            off = (lib.block8_product(a, b, dtype, full_sums=full).double() - want).abs()
            tol = tolerance(va, vb, want, dtype, full)
            assert (off <= (tol + lost * (1 + R.HALF[dtype]) if few or dtype == torch.float32 or full else tol)).all(), (least, dtype, full)


def mark(q, row, block):
    """That block as packing leaves one with an infinity or a NaN in it."""
    q.scales[block, row // 128 if q.square else row] = 255
    first, last = (row // 128 * 128, row // 128 * 128 + 128) if q.square else (row, row + 1)
    q.codes.view(torch.uint8)[first:last, 128 * block:128 * block + 128] = 0


@pytest.mark.parametrize("m,n,k", FEW + TILES)
@pytest.mark.parametrize("ca,cb,sa,sb", PAIRS)
def test_blocks_that_are_not_numbers(lib, m, n, k, ca, cb, sa, sb):
    gen = torch.Generator().manual_seed(m + n + k)
    blocks = -(-k // 128)
    for turn, which in enumerate(((True, False), (False, True), (True, True))):
        a, _ = operand(lib, gen, m, k, ca, sa, torch.full((blocks,), 126))
        b, _ = operand(lib, gen, n, k, cb, sb, torch.full((blocks,), 126))
        for q, rows, marked in ((a, m, which[0]), (b, n, which[1])):
            if marked:
                for row, block in ((rows - 1, blocks - 1), (rows // 3, blocks // 2), (0, 0))[:turn + 1]:
                    mark(q, row, block)
        bad = lib.block8_unpack(a).isnan().any(1)[:, None] | lib.block8_unpack(b).isnan().any(1)[None]
        assert bad.any()
        for dtype, full in KINDS:
            assert torch.equal(lib.block8_product(a, b, dtype, full_sums=full).isnan(), bad), (turn, dtype, full)


@pytest.mark.parametrize("m,n,k", FEW + TILES)
@pytest.mark.parametrize("ca,cb,sa,sb", PAIRS)
def test_codes_that_are_not_numbers(lib, m, n, k, ca, cb, sa, sb):
    """NaNs of both codes, infinities of E5M2, alone and against zeros and each other."""
    gen = torch.Generator().manual_seed(m + n + k)
    blocks = -(-k // 128)
    a, _ = operand(lib, gen, m, k, ca, sa, torch.full((blocks,), 110))
    b, _ = operand(lib, gen, n, k, cb, sb, torch.full((blocks,), 110))
    for q, rows, code in ((a, m, ca), (b, n, cb)):
        byte = q.codes.view(torch.uint8)
        byte[rows // 2, k // 2] = 0x7f
        byte[rows - 1, k - 1] = 0xff
        if code == E5M2:
            byte[rows // 3, k // 3], byte[rows // 4, 0], byte[rows // 5, k - 1] = 0x7c, 0xfc, 0x7d
        byte[0, k // 3] = 0
    va, vb = (lib.block8_unpack(q).double() for q in (a, b))
    # as a sum of products has them: a NaN, an infinity times 0 and infinities of both signs make NaN
    want = times(va, vb)
    for dtype, full in KINDS:
        got = lib.block8_product(a, b, dtype, full_sums=full)
        assert torch.equal(got.isnan(), want.isnan()), (dtype, full)
        assert torch.equal(got[want.isinf()].double(), want[want.isinf()]), (dtype, full)
        assert got[want.isfinite()].isfinite().all(), (dtype, full)
