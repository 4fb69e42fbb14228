"""The norm of many gradients and their clipping against 64 bits."""
import numpy as np
import pytest
import torch

from dense8_reference import EPS32, f64, rounding

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]


def gradients(sizes, seed=0):
    """Tensors of the three types in turn."""
    gen = torch.Generator().manual_seed(seed + len(sizes))
    return [(torch.randn(n, generator=gen) * 2.0 ** (k % 7 - 3)).to(TYPES[(k + seed) % 3]).cuda() for k, n in enumerate(sizes)]


def norm64(grads):
    return np.sqrt(sum((f64(g) ** 2).sum() for g in grads))


def check(got, want, factor):
    for g, w in zip(got, want):
        v = f64(w) * factor
        assert g.dtype == w.dtype and (np.abs(f64(g) - v) <= 3 * EPS32 * np.abs(v) + rounding(v, g.dtype)).all()


SIZES = [[1], [0], [5, 0, 3], [8191], [8192], [8193], [7, 100000, 1, 33, 8192 * 3 + 5], [1000003], [3] * 97, [2049] * 300, [0] * 96 + [9], [20000000, 3]]


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s)}")
@pytest.mark.parametrize("seed", [0, 1, 2])
def test_norm_and_clipping(lib, sizes, seed):
    grads = gradients(sizes, seed)
    want = norm64(grads)
    norm = lib.gradient_norm(grads)
    # the sums are float64: one rounding of the norm
    assert norm.shape == () and abs(norm.item() - want) <= want * 1.01 * EPS32
    for limit in (0.25, 1.5, 0.0):
        max_norm = float(limit * want)
        factor = min(1.0, max_norm / want) if want else 1.0
        out = [torch.full_like(g, 7.0) for g in grads]
        before = [g.clone() for g in grads]
        assert lib.clip_gradients(grads, max_norm, out=out) == norm
        assert all(torch.equal(a, b) for a, b in zip(grads, before))
        check(out, grads, factor)
        if factor == 1.0:
            assert all(torch.equal(a, b) for a, b in zip(out, grads))
        inside = [g.clone() for g in grads]
        assert lib.clip_gradients(inside, max_norm) == norm
        assert all(torch.equal(a, b) for a, b in zip(inside, out))
        mixed = [g.clone() if k % 2 else torch.zeros_like(g) for k, g in enumerate(grads)]  # every second one in its place
        assert lib.clip_gradients([m if k % 2 else g for k, (m, g) in enumerate(zip(mixed, grads))], max_norm, out=mixed) == norm
        assert all(torch.equal(a, b) for a, b in zip(mixed, out))


def test_many_values_at_any_alignment(lib):
    """Results past the cache, not aligned to more than their elements, with neighbours that stay as they are."""
    gen = torch.Generator(device="cuda").manual_seed(8)
    whole = [torch.randn(n, generator=gen, device="cuda").to(t) for n, t in ((30000001, torch.float32), (9000013, torch.bfloat16), (8195, torch.float16))]
    grads = [w[1 + k:-1] for k, w in enumerate(whole)]
    rooms = [torch.full_like(w, 7.0) for w in whole]
    out = [r[3 - k:][:len(g)] for k, (r, g) in enumerate(zip(rooms, grads))]
    grads = [g[:len(o)] for g, o in zip(grads, out)]
    want = norm64(grads)
    assert abs(lib.clip_gradients(grads, float(want) / 3, out=out).item() - want) <= 1.01 * EPS32 * want
    check(out, grads, float(np.float32(want / 3)) / want)
    for k, (r, o) in enumerate(zip(rooms, out)):
        assert (r[:3 - k] == 7).all() and (r[3 - k + len(o):] == 7).all()


def test_far_from_one(lib):
    """Squares past float32's range, on either side."""
    for size in (1e30, 1e-30, 1e-44):
        g = [torch.full((5000,), size, device="cuda"), torch.full((7,), -size, device="cuda")]
        want = norm64(g)
        assert abs(lib.gradient_norm(g).item() - want) <= want * 1.01 * EPS32 + 2.0 ** -150
        out = [torch.empty_like(t) for t in g]
        lib.clip_gradients(g, float(want / 2), out=out)
        check(out, g, float(np.float32(want / 2)) / want)
    largest = [torch.full((100,), torch.finfo(torch.float32).max, device="cuda")]
    assert lib.clip_gradients(largest, 1.0).item() == float("inf")  # past float32, but finite in the sum: scaled all the same
    check(largest, [torch.full((100,), torch.finfo(torch.float32).max)], 1.0 / (10 * float(np.finfo(np.float32).max)))


@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
def test_infinities_and_nans_change_nothing(lib, bad):
    grads = gradients([100, 20000, 5])
    grads[1][12345] = bad
    before = [g.clone() for g in grads]
    norm = lib.clip_gradients(grads, 1.0)
    assert norm.isnan() if bad != bad else norm == float("inf")
    assert all(torch.equal(a.nan_to_num(), b.nan_to_num()) for a, b in zip(grads, before))
    assert lib.gradient_norm(grads).isfinite() == False  # noqa: E712


def test_zeros_and_no_limit(lib):
    grads = [torch.zeros(9, device="cuda"), torch.zeros((0, 3), device="cuda")]
    assert lib.clip_gradients(grads, 0.0) == 0 and (grads[0] == 0).all()
    grads = gradients([1000, 10])
    before = [g.clone() for g in grads]
    lib.clip_gradients(grads, float("inf"))
    assert all(torch.equal(a, b) for a, b in zip(grads, before))


def test_unaligned_and_any_shape(lib):
    room = torch.randn(50001, device="cuda").half()
    grads = [room[1:20002].view(3, -1), room[20003:50000]]
    want = norm64(grads)
    assert abs(lib.gradient_norm(grads).item() - want) <= want * 1.01 * EPS32
    before = room.clone()
    lib.clip_gradients(grads, float(want / 3))
    check([room], [torch.cat([before[:1] * 3, before[1:20002], before[20002:20003] * 3, before[20003:50000], before[50000:] * 3])], 1 / 3)


def test_the_same_gradient_twice_counts_twice(lib):
    g = torch.randn(1000, device="cuda")
    want = norm64([g, g])
    assert abs(lib.gradient_norm([g, g]).item() - want) <= want * 1.01 * EPS32
    out = [torch.empty_like(g), torch.empty_like(g)]
    lib.clip_gradients([g, g], 1.0, out=out)
    check(out, [g, g], 1 / want)
    with pytest.raises(lib.AlexNetError, match="overlaps"):
        lib.clip_gradients([g, g], 1.0)


def test_captured_and_replayed(lib):
    grads = gradients([5, 100000, 77] + [300] * 120)
    static = [g.clone() for g in grads]

    def run():
        for s, g in zip(static, grads):
            s.copy_(g)
        out = [torch.empty_like(g) for g in grads]
        return [lib.gradient_norm(grads), lib.clip_gradients(grads, 20.0, out=out), *out, lib.clip_gradients(static, 20.0)]

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = run()
        captured += static
    for turn in range(4):
        for g in grads:
            g.mul_(0.05 if turn == 2 else -1.5)
        graph.replay()
        torch.cuda.synchronize()
        kept = [c.clone() for c in captured]
        eager = run() + static
        torch.cuda.synchronize()
        assert all(torch.equal(c, e) for c, e in zip(kept, eager)), turn


def test_on_another_stream(lib):
    grads = gradients([100, 70000])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    norm = lib.gradient_norm(grads, stream=side)
    out = [torch.empty_like(g) for g in grads]
    again = lib.clip_gradients(grads, 1.0, out=out, stream=side)
    side.synchronize()
    assert norm == again == lib.gradient_norm(grads)
    lib.clip_gradients(grads, 1.0)
    assert all(torch.equal(a, b) for a, b in zip(grads, out))
