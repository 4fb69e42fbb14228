"""CPU-only: the kinds of sums that a product in 8 bits takes."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def B():
    from paper_1412_2302_amd import binding
    return binding


def test_types_with_full_sums(B):
    def query(m, n, k, type):
        ws = C.c_size_t()
        return B._lib.alexnet_block8_product_query(m, n, k, type, ws), ws.value

    for m, n, k in ((1, 16, 128), (300, 260, 50000), (642, 776, 4320), (609, 618, 7298), (4000, 4090, 300)):
        full = query(m, n, k, 0)
        assert full[0] == B.OK
        for type in (0, 1, 2):  # the slices are those of the float32 result
            assert query(m, n, k, type + B._SUMS_FP32) == full
    for bad in (3, 19, 15, 32, 33, 48, -1, -16, -17, 1 << 30):
        assert query(5, 6, 7, bad)[0] == B.EINVAL and "type" in B.last_error()
    operand = B.Blocks8Arg(1 << 36, 1 << 37, 1, 0)
    for bad in (3, 19, 32, -16):
        assert B._lib.alexnet_block8_product(operand, operand, 5, 6, 7, 1 << 38, 6, bad, None, 0, None) == B.EINVAL
    # refusals of the sizes that a result's own type has
    assert B._lib.alexnet_block8_product(operand, operand, 5, 6, 7, (1 << 38) + 1, 6, 1 + B._SUMS_FP32, None, 0, None) == B.EALIGN
    assert B._lib.alexnet_block8_product(operand, operand, 5, 6, 7, (1 << 36), 6, 1 + B._SUMS_FP32, None, 0, None) == B.EINVAL
    assert "overlap" in B.last_error()
