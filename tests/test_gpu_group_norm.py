"""Group normalisation with an activation against 64-bit formulas: sizes from a single value to groups wider than a workgroup,
odd channel counts, slices of wider tensors, both sources of the backward pass."""
import numpy as np
import pytest
import torch

import norm_reference as R

pytestmark = pytest.mark.gpu

# pictures, pixels, channels, groups
SIZES = [
    (1, 1, 4, 1), (1, 1, 1, 1), (2, 1, 7, 7), (3, 5, 6, 2), (2, 49, 24, 3), (1, 300, 96, 32), (4, 63, 40, 8), (2, 1030, 64, 16),
    (1, 17, 2050, 2), (2, 9, 4100, 1), (1, 5000, 3, 1), (5, 169, 384, 32), (3, 1, 4096, 32), (2, 3025, 48, 16), (70, 4, 64, 32),
    (1, 20011, 8, 2), (2, 33, 37, 37), (1, 3001, 1500, 3), (1, 2000, 1025, 5), (2, 1500, 1100, 275), (1, 9000, 300, 2),
]
TYPES = [torch.float32, torch.bfloat16, torch.float16]
CODES = [None, torch.int8, torch.float8_e4m3fn]


def make(n, hw, c, dtype, seed, wide=0):
    gen = torch.Generator().manual_seed(seed)
    scale, shift = torch.rand(c + wide, generator=gen) * 2 + 0.2, torch.randn(c + wide, generator=gen)
    x = ((torch.randn((n, hw, c + wide), generator=gen) * scale + shift).to(dtype)).cuda()[..., wide:]
    dy = torch.randn((n, hw, c), generator=gen).to(dtype).cuda()
    gamma, beta = (torch.randn(c, generator=gen) * 0.3 + 1).cuda(), (torch.randn(c, generator=gen) * 0.3).cuda()
    return x, dy, gamma, beta


def f64(t):
    return t.detach().double().cpu().numpy()


def near(got, want, tol, what):
    off = np.abs(f64(got) - want)
    assert np.all(off <= tol), (what, float(np.max(off / tol)), float(off.max()))


def check_forward(x, gamma, beta, groups, eps, act, got):
    y, mean, rstd = got
    n, c, dtype = x.shape[0], x.shape[-1], x.dtype
    xf = f64(x).reshape(n, -1, c)
    g = np.ones(c) if gamma is None else f64(gamma)
    b = np.zeros(c) if beta is None else f64(beta)
    want, m, r, z = R.forward(xf, g, b, groups, eps, act)
    tol_m, tol_r = R.statistics_tolerance(xf, groups, r)
    near(mean, m, tol_m, "mean")
    near(rstd, r, tol_r * r, "rstd")
    near(y.reshape(n, -1, c), want, R.forward_tolerance(xf, want, z, g, b, m, r, dtype, act), "y")


def check_backward(xf, dy, mean, rstd, gamma, beta, act, got):
    dx, dgamma, dbeta = got
    n, c = dy.shape[0], dy.shape[-1]
    g = np.ones(c) if gamma is None else f64(gamma)
    b = np.zeros(c) if beta is None else f64(beta)
    d, m, r = f64(dy).reshape(n, -1, c), f64(mean), f64(rstd)
    want, want_g, want_b = R.backward(xf, d, m, r, g, b, act)
    tol, tol_g, tol_b = R.backward_tolerance(xf, d, m, r, g, b, act, want, dy.dtype)
    near(dx.reshape(n, -1, c), want, tol, "dx")
    near(dgamma, want_g, tol_g, "dgamma")
    near(dbeta, want_b, tol_b, "dbeta")


def kept_values(lib, kept):
    """The values that a checkpoint stands for, from its codes alone."""
    c = kept.shape[-1]
    return R.decode(f64(kept.codes.float()).reshape(-1, c), kept.scales.cpu().numpy().reshape(-1, kept.scales.shape[-1]))


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_forward_and_backward(lib, size, dtype):
    n, hw, c, groups = size
    for i, (act, code) in enumerate([("none", None), ("relu", torch.int8), ("silu", torch.float8_e4m3fn), ("relu", None), ("silu", torch.int8)]):
        x, dy, gamma, beta = make(n, hw, c, dtype, 100 * i + c)
        y, mean, rstd, kept = lib.group_norm_forward(x, gamma, beta, groups, 1e-5, act, checkpoint=code)
        check_forward(x, gamma, beta, groups, 1e-5, act, (y, mean, rstd))
        assert (kept is None) == (code is None)
        xf = f64(x).reshape(n, hw, c)
        if kept is not None:
            codes, scales = R.code(xf.reshape(-1, c), code)
            assert np.array_equal(f64(kept.codes.float()).reshape(-1, c), codes)
            assert np.array_equal(kept.scales.cpu().numpy().reshape(scales.shape), scales)
            xf = kept_values(lib, kept).reshape(n, hw, c)
        got = lib.group_norm_backward(x if kept is None else kept, dy, mean, rstd, gamma, beta, act)
        check_backward(xf, dy, mean, rstd, gamma, beta, act, got)


@pytest.mark.parametrize("size", [(2, 3000, 300, 300), (1, 60000, 128, 128), (1, 60000, 128, 8), (3, 9000, 256, 256), (2, 4000, 64, 2)], ids=str)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_groups_and_chunks_of_every_number(lib, size, dtype):
    """Few pairs of a picture are joined where they are used, many by a launch of their own."""
    n, hw, c, groups = size
    x, dy, gamma, beta = make(n, hw, c, dtype, 77)
    y, mean, rstd, _ = lib.group_norm_forward(x, gamma, beta, groups, 1e-5, "silu")
    check_forward(x, gamma, beta, groups, 1e-5, "silu", (y, mean, rstd))
    check_backward(f64(x), dy, mean, rstd, gamma, beta, "silu", lib.group_norm_backward(x, dy, mean, rstd, gamma, beta, "silu"))
    x += 300  # a mean far from zero
    y, mean, rstd, _ = lib.group_norm_forward(x, gamma, beta, groups, 1e-5, "none")
    check_forward(x, gamma, beta, groups, 1e-5, "none", (y, mean, rstd))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("wide", [1, 8, 32])
def test_slices_of_wider_tensors_leave_the_rest_alone(lib, dtype, wide):
    n, hw, c, groups = 3, 70, 48, 8
    x, dy, gamma, beta = make(n, hw, c, dtype, 5, wide)
    room = torch.full((n, hw, c + 2 * wide), 7.0, dtype=dtype, device="cuda")
    y, mean, rstd, _ = lib.group_norm_forward(x, gamma, beta, groups, 1e-3, "relu", out=room[..., wide:wide + c])
    check_forward(x, gamma, beta, groups, 1e-3, "relu", (y, mean, rstd))
    assert bool((room[..., :wide] == 7).all()) and bool((room[..., wide + c:] == 7).all())
    room = torch.full((n, hw, c + 2 * wide), 7.0, dtype=dtype, device="cuda")
    got = lib.group_norm_backward(x, dy, mean, rstd, gamma, beta, "relu", out=room[..., wide:wide + c])
    check_backward(f64(x), dy, mean, rstd, gamma, beta, "relu", got)
    assert bool((room[..., :wide] == 7).all()) and bool((room[..., wide + c:] == 7).all())
    # the gradient's own stride
    d2 = torch.randn((n, hw, c + wide), device="cuda").to(dtype)[..., wide:]
    check_backward(f64(x), d2, mean, rstd, gamma, beta, "silu", lib.group_norm_backward(x, d2, mean, rstd, gamma, beta, "silu"))


@pytest.mark.parametrize("size", [(2, 49, 24, 3), (1, 5000, 64, 4), (2, 9, 4100, 1)], ids=str)
def test_in_place(lib, size):
    n, hw, c, groups = size
    x, dy, gamma, beta = make(n, hw, c, torch.float32, 9)
    y, mean, rstd, kept = lib.group_norm_forward(x, gamma, beta, groups, 1e-5, "silu", checkpoint=torch.int8)
    dx, dgamma, dbeta = lib.group_norm_backward(kept, dy, mean, rstd, gamma, beta, "silu")
    x2, dy2 = x.clone(), dy.clone()
    y2, mean2, rstd2, kept2 = lib.group_norm_forward(x2, gamma, beta, groups, 1e-5, "silu", checkpoint=torch.int8, out=x2)
    assert y2.data_ptr() == x2.data_ptr()
    out = lib.group_norm_backward(kept2, dy2, mean2, rstd2, gamma, beta, "silu", out=dy2)
    for a, b in [(y, y2), (mean, mean2), (rstd, rstd2), (kept.codes, kept2.codes), (kept.scales, kept2.scales), (dx, out[0]),
                 (dgamma, out[1]), (dbeta, out[2])]:
        assert torch.equal(a, b)


@pytest.mark.parametrize("size", [(1, 4000, 74, 2), (2, 6000, 37, 1), (1, 2000, 1025, 5), (2, 60, 37, 37), (3, 40, 3, 1)], ids=str)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_in_place_where_rows_are_no_whole_vectors(lib, size, dtype):
    """No thread may read what another has already overwritten; dx may also take the place of x."""
    n, hw, c, groups = size
    x, dy, gamma, beta = make(n, hw, c, dtype, 10)
    want = lib.group_norm_forward(x, gamma, beta, groups, 1e-5, "relu")
    x2 = x.clone()
    got = lib.group_norm_forward(x2, gamma, beta, groups, 1e-5, "relu", out=x2)
    check_forward(x, gamma, beta, groups, 1e-5, "relu", got[:3])
    for over in ("dy", "x"):
        x2, dy2 = x.clone(), dy.clone()
        got = lib.group_norm_backward(x2, dy2, want[1], want[2], gamma, beta, "relu", out=dy2 if over == "dy" else x2)
        check_backward(f64(x).reshape(n, hw, c), dy, want[1], want[2], gamma, beta, "relu", got)
        assert torch.equal(dy2, dy) if over == "x" else torch.equal(x2, x)


@pytest.mark.parametrize("hw", [50, 5000])
def test_what_overlaps_is_refused(lib, hw):
    x, dy, gamma, beta = make(2, hw, 24, torch.float32, 12)
    y, mean, rstd, _ = lib.group_norm_forward(x, gamma, beta, 3)
    room = torch.zeros((2, hw, 60), device="cuda")
    inside = room[..., 10:34]
    inside.copy_(x)
    for a in (11, 33, 0):
        with pytest.raises(Exception, match="overlaps"):
            lib.group_norm_forward(inside, gamma, beta, 3, out=room[..., a:a + 24])
    got = lib.group_norm_forward(inside, gamma, beta, 3, out=room[..., 34:58])[0]
    assert torch.equal(got.contiguous(), y) and torch.equal(inside.contiguous(), x)
    with pytest.raises(Exception, match="overlaps"):
        lib.group_norm_backward(x, inside, mean, rstd, gamma, beta, out=room[..., 12:36])


def test_more_values_than_31_bits_count(lib):
    n, hw, c, groups = 2, (1 << 25) + 3, 40, 4
    x = torch.randn((n, hw, c), device="cuda", dtype=torch.bfloat16)
    x[1] += 2.0
    gamma, beta = torch.randn(c, device="cuda"), torch.randn(c, device="cuda")
    y, mean, rstd, kept = lib.group_norm_forward(x, gamma, beta, groups, 1e-5, "silu", checkpoint=torch.int8)
    last = x[1].view(hw, groups, c // groups)
    for g in range(groups):
        part = last[:, g].double()
        m, r = float(part.mean()), float(1 / torch.sqrt(part.var(unbiased=False) + 1e-5))
        size = float(part.abs().mean())
        # a chunk of the picture is no longer than a thousand groups of four pixels a thread
        off = 2048 * R.EPS32 * size
        assert abs(float(mean[1, g]) - m) <= off and abs(float(rstd[1, g]) / r - 1) <= 2048 * R.EPS32 + (off * r) ** 2
    end = x[1, -1000:].contiguous()
    codes = lib.checkpoint_pack(end, torch.int8)
    assert torch.equal(kept.codes[1, -1000:], codes.codes) and torch.equal(kept.scales[1, -1000:], codes.scales)
    wide = (mean[1].repeat_interleave(c // groups), rstd[1].repeat_interleave(c // groups))
    z = (end.double() - wide[0].double()) * wide[1].double() * gamma.double() + beta.double()
    want = z * torch.sigmoid(z)
    off = 16 * R.EPS32 * (1 + z.abs()) * (1 + want.abs() + (end.double() * wide[1] * gamma).abs() + (wide[0] * wide[1] * gamma).abs())
    assert bool(((y[1, -1000:].double() - want).abs() <= off + want.abs() * R.HALF_STEP[torch.bfloat16] * 1.01).all())
    dy = y  # any gradient will do; in place
    tail = dy[1, -1000:].clone().double()
    dx, dgamma, dbeta = lib.group_norm_backward(kept, dy, mean, rstd, gamma, beta, "none", out=dy)
    values = lib.checkpoint_unpack(codes).double()
    hat = (values - wide[0].double()) * wide[1].double()
    # the means over the group are what every pixel of a channel has in common
    rest = wide[1].double() * gamma.double() * tail - dx[1, -1000:].double()
    rest = rest.view(1000, groups, c // groups)
    for g in range(groups):
        a = torch.stack([torch.ones(10000, device="cuda", dtype=torch.float64), hat.view(1000, groups, -1)[:, g].reshape(-1)], 1)
        t = rest[:, g].reshape(-1, 1)
        fit = torch.linalg.lstsq(a.cpu(), t.cpu()).solution
        # what is left is the rounding of dx to bfloat16
        left = (t.cpu() - a.cpu() @ fit).abs()
        assert float(left.max()) <= float(dx[1, -1000:].double().abs().max()) * R.HALF_STEP[torch.bfloat16] * 2
    assert bool(torch.isfinite(dgamma).all()) and bool(torch.isfinite(dbeta).all())


def test_without_gamma_and_beta_and_on_maps(lib):
    x, dy, _, _ = make(2, 30, 20, torch.float32, 11)
    x4, dy4 = x.view(2, 5, 6, 20), dy.view(2, 5, 6, 20)
    y, mean, rstd, _ = lib.group_norm_forward(x4, None, None, 4)
    assert y.shape == x4.shape
    check_forward(x, None, None, 4, 1e-5, "none", (y, mean, rstd))
    dx, dgamma, dbeta = lib.group_norm_backward(x4, dy4, mean, rstd, None, None)
    assert dx.shape == x4.shape
    check_backward(f64(x), dy, mean, rstd, None, None, "none", (dx, dgamma, dbeta))


def test_empty_batches_and_maps(lib):
    gamma = torch.ones(6, device="cuda")
    for shape in [(0, 5, 6), (3, 0, 6)]:
        x = torch.empty(shape, device="cuda")
        y, mean, rstd, kept = lib.group_norm_forward(x, gamma, gamma, 2, 0.25, checkpoint=torch.int8)
        assert y.shape == x.shape and kept.shape == x.shape
        assert bool((mean == 0).all()) and bool((rstd == 2).all())
        dx, dgamma, dbeta = lib.group_norm_backward(kept, x, mean, rstd, gamma, gamma)
        assert dx.shape == x.shape and bool((dgamma == 0).all()) and bool((dbeta == 0).all())


def test_far_from_zero(lib):
    """A mean a thousand deviations off: the squares are summed about the mean, so the variance keeps its digits."""
    x, dy, gamma, beta = make(2, 500, 64, torch.float32, 13)
    x = (x + 1000.0).contiguous()
    y, mean, rstd, _ = lib.group_norm_forward(x, gamma, beta, 16, 1e-5, "none")
    check_forward(x, gamma, beta, 16, 1e-5, "none", (y, mean, rstd))
    x[:, 0] = 1e7  # the first pixel far from all others
    y, mean, rstd, _ = lib.group_norm_forward(x, gamma, beta, 16, 1e-5, "none")
    check_forward(x, gamma, beta, 16, 1e-5, "none", (y, mean, rstd))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("hw", [40, 4000])
def test_what_is_not_finite_stays_in_its_group_and_shows(lib, bad, hw):
    x, dy, gamma, beta = make(3, hw, 64, torch.float32, 17)
    good = lib.group_norm_forward(x, gamma, beta, 8, 1e-5, "relu", checkpoint=torch.int8)
    clean = lib.group_norm_backward(x, dy, good[1], good[2], gamma, beta, "relu")
    x = x.clone()
    x[1, 7, 13] = bad  # picture 1, group 1
    y, mean, rstd, kept = lib.group_norm_forward(x, gamma, beta, 8, 1e-5, "relu", checkpoint=torch.int8)
    hit = torch.zeros((3, 8), dtype=torch.bool, device="cuda")
    hit[1, 1] = True
    wide = hit.repeat_interleave(8, 1)[:, None].expand_as(y)
    assert bool(torch.isnan(y[wide]).all()) and torch.equal(y[~wide], good[0][~wide])
    assert torch.equal(mean[~hit], good[1][~hit]) and torch.equal(rstd[~hit], good[2][~hit])
    assert int((kept.scales == 255).sum()) == 1 and int(kept.scales[1, 7, 0]) == 255
    dx, dgamma, dbeta = lib.group_norm_backward(x, dy, mean, rstd, gamma, beta, "relu")
    assert bool(torch.isnan(dx[wide]).all()) and torch.equal(dx[~wide], clean[0][~wide])


def test_gates_next_to_the_border(lib):
    """beta is set so that z of many values is zero to within a few ulps: each gate falls as its exact value says."""
    n, hw, c, groups = 2, 600, 32, 8
    gen = torch.Generator().manual_seed(3)
    x = (torch.randint(-4, 5, (n, hw, c), generator=gen).float() * 0.3).cuda()
    dy = torch.ones_like(x)
    gamma = (torch.rand(c, generator=gen) + 0.5).cuda()
    _, mean, rstd, _ = lib.group_norm_forward(x, gamma, None, groups)
    wide = c // groups
    at = -((0.6 - mean[0].double().repeat_interleave(wide)) * rstd[0].double().repeat_interleave(wide) * gamma.double())
    beta = at.float()
    m, r = mean.double().repeat_interleave(wide, 1)[:, None], rstd.double().repeat_interleave(wide, 1)[:, None]
    z = (x.double() - m) * r * gamma.double() + beta.double()
    assert int((z.abs() < 1e-6).sum()) > 500
    _, _, dbeta = lib.group_norm_backward(x, dy, mean, rstd, gamma, beta, "relu")
    assert torch.equal(dbeta, (z > 0).sum((0, 1)).float())


def test_gradients_are_the_forward_pass_own(lib):
    """Differences of the forward pass along random directions: sum(dy * y) changes by the gradients' products.  Steps of
    2^-7 leave a third-order term of about 1e-4 of the slope and a rounding of some 1e-5."""
    n, hw, c, groups = 2, 50, 24, 4
    x, dy, gamma, beta = make(n, hw, c, torch.float32, 21)
    for act in ("none", "silu"):
        _, mean, rstd, _ = lib.group_norm_forward(x, gamma, beta, groups, 1e-5, act)
        dx, dgamma, dbeta = lib.group_norm_backward(x, dy, mean, rstd, gamma, beta, act)
        gen = torch.Generator().manual_seed(4)
        vx, vg, vb = [torch.randn(t.shape, generator=gen).cuda() for t in (x, gamma, beta)]
        h = 2.0 ** -7

        def loss(s):
            y = lib.group_norm_forward(x + s * h * vx, gamma + s * h * vg, beta + s * h * vb, groups, 1e-5, act)[0]
            return float((y.double() * dy.double()).sum())

        slope = (loss(1) - loss(-1)) / (2 * h)
        want = float((dx.double() * vx).sum() + (dgamma.double() * vg).sum() + (dbeta.double() * vb).sum())
        size = float((dx.double() * vx).norm() + (dgamma.double() * vg).norm() + (dbeta.double() * vb).norm())
        assert abs(slope - want) <= 2e-3 * size, (act, slope, want, size)


def test_same_bits_every_time(lib):
    x, dy, gamma, beta = make(6, 1500, 96, torch.bfloat16, 23)
    first = None
    for _ in range(3):
        y, mean, rstd, kept = lib.group_norm_forward(x, gamma, beta, 32, 1e-5, "silu", checkpoint=torch.float8_e4m3fn)
        now = (y, mean, rstd, kept.codes.view(torch.uint8), kept.scales, *lib.group_norm_backward(kept, dy, mean, rstd, gamma, beta, "silu"))
        first = first or now
        assert all(torch.equal(a, b) for a, b in zip(first, now))


def test_captured_and_replayed(lib):
    """A graph of forward and backward over static buffers, replayed with other inputs, eager work between the replays."""
    n, hw, c, groups = 3, 400, 64, 16
    x, dy, gamma, beta = make(n, hw, c, torch.float32, 31)

    def step():
        y, mean, rstd, kept = lib.group_norm_forward(x, gamma, beta, groups, 1e-5, "silu", checkpoint=torch.int8)
        return (y, mean, rstd, *lib.group_norm_backward(kept, dy, mean, rstd, gamma, beta, "silu"))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for seed in range(3):
        nx, ndy, _, _ = make(n, hw, c, torch.float32, 40 + seed)
        x.copy_(nx)
        dy.copy_(ndy)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, step()):
            assert torch.equal(a, b)


def test_two_streams_at_once(lib):
    """Calls on two streams share nothing: each gives what it gives alone."""
    a, b = make(8, 3000, 64, torch.float32, 51), make(2, 700, 96, torch.bfloat16, 52)
    want = [lib.group_norm_forward(v[0], v[2], v[3], 32, 1e-5, "relu") for v in (a, b)]
    grads = [lib.group_norm_backward(v[0], v[1], w[1], w[2], v[2], v[3], "relu") for v, w in zip((a, b), want)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for _ in range(4):
        for v, st in zip((a, b), streams):
            y, mean, rstd, _ = lib.group_norm_forward(v[0], v[2], v[3], 32, 1e-5, "relu", stream=st)
            got.append((y, mean, rstd, *lib.group_norm_backward(v[0], v[1], mean, rstd, v[2], v[3], "relu", stream=st)))
    torch.cuda.synchronize()
    for i, g in enumerate(got):
        for t, w in zip(g, (*want[i % 2][:3], *grads[i % 2])):
            assert torch.equal(t, w)
