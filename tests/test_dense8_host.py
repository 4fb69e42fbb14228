"""CPU-only: what products in 8 bits, root-mean-square normalisation and gradient clipping refuse before any GPU work."""
import ctypes as C
import itertools

import numpy as np
import pytest
import torch

import dense8_reference as R

E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2


@pytest.fixture(scope="module")
def B():
    from paper_1412_2302_amd import binding
    return binding


# every buffer at an address of its own, far apart
NAMES = ["x", "residual", "sum", "y", "dy", "dsum", "dx", "gamma", "dgamma", "rstd", "work", "codes", "scales", "codes2", "scales2", "norm", "g0", "g1", "o0", "o1"]
AT = {name: (i + 1) << 36 for i, name in enumerate(NAMES)}
WORK = 1 << 34


def pack(B, rows=300, cols=260, ld=None, type=0, code=1, code2=1, square=0, square2=0, one=True, two=True, **at):
    p = {**AT, **at}
    return B._lib.alexnet_block8_pack(p["x"], cols if ld is None else ld, type, rows, cols, B.Blocks8Arg(p["codes"], p["scales"], code, square) if one else None,
                                      B.Blocks8Arg(p["codes2"], p["scales2"], code2, square2) if two else None, None)


def unpack(B, rows=300, cols=260, ld=None, type=0, code=1, square=0, **at):
    p = {**AT, **at}
    return B._lib.alexnet_block8_unpack(B.Blocks8Arg(p["codes"], p["scales"], code, square), rows, cols, p["x"], cols if ld is None else ld, type, None)


def product(B, m=300, n=260, k=50000,  # a long sum: slices, and scratch for them
            ld=None, type=1, code=1, code2=2, square=0, square2=1, size=WORK, **at):
    p = {**AT, **at}
    return B._lib.alexnet_block8_product(B.Blocks8Arg(p["codes"], p["scales"], code, square), B.Blocks8Arg(p["codes2"], p["scales2"], code2, square2),
                                         m, n, k, p["y"], n if ld is None else ld, type, p["work"], size, None)


def forward(B, rows=300, cols=260, type=0, eps=1e-5, ld_x=None, ld_residual=None, ld_sum=None, ld_y=None, blocks=None, **at):
    p = {**AT, **at}
    lds = [cols if v is None else v for v in (ld_x, ld_residual, ld_sum, ld_y)]
    return B._lib.alexnet_rms_norm_forward(p["x"], lds[0], p["residual"], lds[1], type, rows, cols, eps, p["gamma"], p["sum"], lds[2],
                                           None if blocks else p["y"], lds[3], blocks, p["rstd"], None)


def backward(B, rows=300, cols=260, type=0, ld_sum=None, ld_dy=None, ld_dsum=None, ld_dx=None, size=WORK, **at):
    p = {**AT, **at}
    lds = [cols if v is None else v for v in (ld_sum, ld_dy, ld_dsum, ld_dx)]
    return B._lib.alexnet_rms_norm_backward(p["sum"], lds[0], p["dy"], lds[1], p["dsum"], lds[2], type, rows, cols, p["rstd"], p["gamma"], p["dx"],
                                            lds[3], p["dgamma"], p["work"], size, None)


def clip(B, sizes=(100, 9000), types=(0, 1), max_norm=1.0, outs=True, size=WORK, count=None, just_norm=False, **at):
    p = {**AT, **at}
    n = len(sizes)
    grads, results = (C.c_void_p * n)(p["g0"], p["g1"]), (C.c_void_p * n)(p["o0"], p["o1"]) if outs else None
    s, t = (C.c_int64 * n)(*sizes), (C.c_int32 * n)(*types)
    count = n if count is None else count
    if just_norm:
        return B._lib.alexnet_gradient_norm(count, grads, s, t, p["norm"], p["work"], size, None)
    return B._lib.alexnet_clip_gradients(count, grads, results, s, t, max_norm, p["norm"], p["work"], size, None)


def test_types_and_sizes(B):
    ws = C.c_size_t()
    for call in (pack, unpack, product, forward, backward):
        assert call(B, type=3) == call(B, type=-1) == B.EINVAL and "type" in B.last_error()
    assert pack(B, rows=-1) == pack(B, cols=-1) == pack(B, rows=1 << 29) == pack(B, cols=1 << 29) == pack(B, rows=1 << 20, cols=1 << 20) == B.ESHAPE
    assert unpack(B, rows=-1) == unpack(B, rows=1 << 29, cols=1) == B.ESHAPE
    for bad in (dict(m=-1), dict(n=-1), dict(k=-1), dict(m=1 << 29), dict(k=(1 << 22) + 1), dict(m=1 << 20, n=(1 << 12) + 1), dict(m=1 << 27, n=1, k=1024)):
        assert product(B, **bad) == B.ESHAPE, bad
        q = {**dict(m=300, n=260, k=5000), **bad}
        assert B._lib.alexnet_block8_product_query(q["m"], q["n"], q["k"], 1, ws) == B.ESHAPE
    for call in (forward, backward):
        assert call(B, rows=-1) == call(B, cols=0) == call(B, rows=(1 << 24) + 1) == call(B, cols=(1 << 20) + 1) == B.ESHAPE
    assert B._lib.alexnet_rms_norm_query(3, 0, 0, ws) == B.ESHAPE and B._lib.alexnet_rms_norm_query(3, 4, 5, ws) == B.EINVAL
    for eps in (0.0, -1.0, float("nan")):
        assert forward(B, eps=eps) == B.EINVAL and "eps" in B.last_error()
    assert clip(B, types=(0, 3)) == clip(B, types=(-1, 0)) == B.EINVAL
    assert clip(B, sizes=(1, -1)) == clip(B, sizes=(1 << 40, 1)) == clip(B, count=-1) == clip(B, count=(1 << 20) + 1) == B.ESHAPE
    assert clip(B, max_norm=-1.0) == clip(B, max_norm=float("nan")) == B.EINVAL and "max_norm" in B.last_error()


def test_null_pointers_strides_and_alignment(B):
    ws = C.c_size_t()
    for call, names in ((pack, ["x", "codes", "scales", "codes2", "scales2"]), (unpack, ["x", "codes", "scales"]),
                        (product, ["y", "codes", "scales", "codes2", "scales2"]), (forward, ["x", "y"]), (backward, ["sum", "dy", "rstd", "dx"]),
                        (clip, ["g0", "g1", "o0", "o1"])):
        for name in names:
            assert call(B, **{name: None}) == B.EINVAL, (call, name)
    assert forward(B, residual=None) == forward(B, sum=None) == B.EINVAL and "residual" in B.last_error()
    assert B._lib.alexnet_rms_norm_forward(256, 9, None, 0, 0, 3, 9, 1e-5, None, None, 0, None, 0, None, None, None) == B.EINVAL
    assert B._lib.alexnet_rms_norm_forward(256, 9, None, 0, 0, 3, 9, 1e-5, None, None, 0, 1 << 30, 9, B.Blocks8Arg(1 << 31, 1 << 32, 1, 0), None, None) == B.EINVAL
    assert forward(B, blocks=B.Blocks8Arg(AT["codes"], AT["scales"], 1, 1)) == B.EINVAL and "square" in B.last_error()
    assert pack(B, one=False, two=False) == B.EINVAL
    assert pack(B, code=2) == pack(B, square=1) == B.EINVAL and "different" in B.last_error()
    for code in (0, 3, -1):
        assert pack(B, code=code, code2=code) == unpack(B, code=code) == product(B, code=code) == product(B, code2=code) == B.EINVAL
    assert unpack(B, square=2) == product(B, square2=-1) == B.EINVAL
    assert pack(B, ld=259) == unpack(B, ld=259) == product(B, ld=259) == pack(B, ld=-260) == product(B, ld=1 << 41) == B.ESHAPE
    for name in ("ld_x", "ld_residual", "ld_sum", "ld_y"):
        assert forward(B, **{name: 259}) == forward(B, **{name: 1 << 41}) == B.ESHAPE
    for name in ("ld_sum", "ld_dy", "ld_dsum", "ld_dx"):
        assert backward(B, **{name: 259}) == B.ESHAPE
    for call, names in ((pack, ["x"]), (unpack, ["x"]), (forward, ["x", "residual", "sum", "y", "gamma", "rstd"]),
                        (backward, ["sum", "dy", "dsum", "dx", "gamma", "dgamma", "rstd", "work"]), (clip, ["g0", "o0", "norm", "work"])):
        for name in names:
            assert call(B, **{name: AT[name] + 2}) == B.EALIGN, (call, name)
    assert product(B, y=AT["y"] + 1) == product(B, work=AT["work"] + 128) == B.EALIGN
    for call in (pack, unpack, product):
        assert call(B, codes=AT["codes"] + 8) == call(B, scales=AT["scales"] + 2) == B.EALIGN
    assert clip(B, g1=AT["g1"] + 1, types=(0, 2)) == B.EALIGN
    # scratch
    assert B._lib.alexnet_block8_product_query(300, 260, 50000, 1, ws) == B.OK and ws.value > 0
    assert product(B, size=ws.value - 1) == product(B, work=None) == B.ENOMEM and "workspace" in B.last_error()
    assert B._lib.alexnet_rms_norm_query(300, 260, 0, ws) == B.OK and ws.value > 0
    assert backward(B, size=ws.value - 1) == backward(B, work=None) == B.ENOMEM
    sizes = (C.c_int64 * 2)(100, 9000)
    assert B._lib.alexnet_clip_query(2, sizes, ws) == B.OK and ws.value > 0
    assert clip(B, size=ws.value - 1) == clip(B, work=None) == clip(B, size=ws.value - 1, just_norm=True) == B.ENOMEM
    assert clip(B, just_norm=True, norm=None) == B.EINVAL
    assert B._lib.alexnet_clip_query(2, None, ws) == B._lib.alexnet_clip_query(2, sizes, None) == B._lib.alexnet_block8_product_query(1, 1, 1, 0, None) == B.EINVAL
    assert B._lib.alexnet_clip_query(-1, sizes, ws) == B.ESHAPE


def test_sizes_of_nothing(B):
    ws = C.c_size_t()
    q = B._lib.alexnet_block8_product_query
    assert q(0, 5, 7, 0, ws) == q(5, 0, 7, 0, ws) == q(300, 300, 0, 0, ws) == q(0, 0, 0, 0, ws) == B.OK and ws.value == 0
    assert B._lib.alexnet_rms_norm_query(0, 5, 0, ws) == B.OK and ws.value == 0
    assert B._lib.alexnet_clip_query(0, None, ws) == B.OK
    # nothing is read then
    assert pack(B, rows=0, x=None, codes=None) == unpack(B, cols=0, x=None) == product(B, m=0, codes=None) == forward(B, rows=0, x=None) == B.OK
    assert backward(B, rows=0, sum=None, dgamma=None) == B.OK


CALLS = {  # what a call reads and writes
    "pack": (pack, ["x"], ["codes", "scales", "codes2", "scales2"]),
    "unpack": (unpack, ["codes", "scales"], ["x"]),
    "product": (product, ["codes", "scales", "codes2", "scales2"], ["y", "work"]),
    "forward": (forward, ["x", "residual", "gamma"], ["y", "sum", "rstd"]),
    "backward": (backward, ["sum", "dy", "dsum", "rstd", "gamma"], ["dx", "dgamma", "work"]),
    "clip": (clip, ["g0", "g1"], ["o0", "o1", "norm", "work"]),
}
IN_PLACE = {("y", "x"), ("y", "residual"), ("sum", "x"), ("sum", "residual"), ("dx", "sum"), ("dx", "dy"), ("dx", "dsum"), ("o0", "g0"), ("o1", "g1")}


@pytest.mark.parametrize("kind", CALLS)
def test_overlaps(B, kind):
    call, reads, writes = CALLS[kind]
    for a, b in [*itertools.product(writes, reads), *itertools.combinations(writes, 2)]:
        for off in (0, 256):  # at the same address, and some way inside
            if off == 0 and (a, b) in IN_PLACE:
                continue
            if off and (b == "norm" or (kind, b) in (("product", "scales2"), ("clip", "work"))):  # ends before that
                continue
            assert call(B, **{a: AT[b] + off}) == B.EINVAL and "overlap" in B.last_error(), (a, b, off)


def test_overlaps_of_blocks(B):
    for a, b in (("codes", "x"), ("scales", "residual"), ("codes", "gamma"), ("scales", "codes"), ("codes", "sum"), ("scales", "rstd")):
        at = {**AT, a: AT[b]}
        assert forward(B, blocks=B.Blocks8Arg(at["codes"], at["scales"], 1, 0)) == B.EINVAL and "overlap" in B.last_error(), (a, b)
    # another stride is another place
    assert forward(B, y=AT["x"], ld_y=300) == backward(B, dx=AT["dy"], ld_dx=300) == B.EINVAL


def test_one_tensor_twice(B):
    assert clip(B, outs=False, g1=AT["g0"]) == clip(B, outs=False, g1=AT["g0"] + 396) == B.EINVAL and "overlap" in B.last_error()
    assert clip(B, o1=AT["g0"]) == clip(B, o0=AT["g0"], g1=AT["g0"]) == B.EINVAL


def test_blocks8_of_the_wrong_sizes(B):
    codes, scales = torch.zeros((5, 256), dtype=torch.uint8).view(E4M3), torch.zeros((2, 8), dtype=torch.uint8)
    made = B.Blocks8(codes, scales, 200)
    assert made.shape == (5, 200) and not made.square
    assert B.Blocks8(codes, torch.zeros((2, 1), dtype=torch.uint8), 129, square=True).square
    for bad in (lambda: B.Blocks8(codes[:, :0], scales[:0], -5), lambda: B.Blocks8(codes, scales, 128), lambda: B.Blocks8(codes, scales, 257), lambda: B.Blocks8(codes, scales, 200, square=True),
                lambda: B.Blocks8(codes.view(torch.uint8), scales, 200), lambda: B.Blocks8(codes, scales.int(), 200),
                lambda: B.Blocks8(codes[:4], scales, 200), lambda: B.Blocks8(codes, scales[:, :5], 200), lambda: B.Blocks8(codes.view(5, 2, 128), scales, 200),
                lambda: B.Blocks8(torch.zeros((256, 5), dtype=torch.uint8).t().view(E4M3), scales, 200)):
        with pytest.raises(ValueError, match="Blocks8"):
            bad()


def test_arguments_of_the_wrong_kind(B):
    x = torch.zeros(4, 40)
    blocks = B.Blocks8(torch.zeros((4, 128), dtype=torch.uint8).view(E4M3), torch.zeros((1, 4), dtype=torch.uint8), 40)
    for call in (lambda: B.block8_pack(None), lambda: B.rms_norm_forward([1.0], None), lambda: B.rms_norm_backward(x.numpy(), x, None, None),
                 lambda: B.gradient_norm([1.0]), lambda: B.clip_gradients([None], 1.0)):
        with pytest.raises(TypeError, match="expected .*torch.Tensor"):
            call()
    for call in (lambda: B.block8_unpack(x), lambda: B.block8_product(x, blocks), lambda: B.block8_product(None, x)):
        with pytest.raises(TypeError, match="expected Blocks8"):
            call()
    for call in (lambda: B.block8_pack(x), lambda: B.rms_norm_forward(x, None), lambda: B.rms_norm_backward(x, x, x, None), lambda: B.gradient_norm([x]),
                 lambda: B.block8_unpack(blocks), lambda: B.block8_product(blocks, blocks)):
        with pytest.raises(ValueError, match="device tensor|on one device"):
            call()
    with pytest.raises(ValueError, match="no gradients"):
        B.gradient_norm([])


def test_the_reference_against_brute_force():
    """Codes as the nearest of all 256, scales as the smallest that hold the block."""
    gen = np.random.default_rng(3)
    for code, worst in ((E4M3, 127), (E5M2, 124)):
        every = torch.arange(256, dtype=torch.uint8)
        every = every[(every & 127) < worst].view(code).double().numpy()
        for square in (False, True):
            x = gen.standard_normal((130, 140)) * np.exp2(gen.integers(-12, 12, (130, 1)))
            x[3, 5] = 0
            codes, scales = R.pack(x, code, square)
            for i, j in gen.integers(0, 130, (60, 2)):
                block = x[i // 128 * 128:i // 128 * 128 + 128] if square else x[i:i + 1]
                block = np.abs(block[:, j // 128 * 128:j // 128 * 128 + 128]).max()
                e = int(scales[j // 128, i // 128 if square else i]) - 127
                assert block <= R.TOP[code] * 2.0 ** e and block > R.TOP[code] * 2.0 ** (e - 1)
                near = np.abs(every * 2.0 ** e - x[i, j])
                assert abs(codes[i, j] * 2.0 ** e - x[i, j]) == near.min()
            assert (R.values(codes, scales if square else scales[:, :130], 140, square) == codes[:, :140] * np.exp2(
                np.repeat(np.repeat(scales.astype(float), 128, 0)[:140] - 127, 128 if square else 1, 1)[:, :130].T)).all()
