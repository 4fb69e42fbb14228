"""Clipping at the ends of float32: norms past its range, infinities, NaNs."""
import numpy as np
import pytest
import torch

from dense8_reference import EPS32, HALF, f64

pytestmark = pytest.mark.gpu


def norm64(g):
    return np.sqrt((f64(g) ** 2).sum())


@pytest.mark.parametrize("places", ["there", "elsewhere"])
@pytest.mark.parametrize("count", [3, 200])
def test_a_norm_past_float32_of_finite_gradients(lib, places, count):
    """Returned as an infinity; what was scaled has the norm that was asked for, to the rounding of its values."""
    gen = torch.Generator().manual_seed(count)
    types = [torch.float32, torch.bfloat16, torch.float32]
    grads = [((torch.rand(50 + i, generator=gen) + 0.5) * 1e38).to(types[i % 3]).cuda() for i in range(count)]
    want = np.sqrt(sum((f64(g) / 1e38) ** 2 @ np.ones(g.numel()) for g in grads)) * 1e38
    assert np.isfinite(want) and want > np.finfo(np.float32).max and lib.gradient_norm(grads) == float("inf")
    before, out = [f64(g) for g in grads], [torch.empty_like(g) for g in grads] if places == "elsewhere" else None
    assert lib.clip_gradients(grads, 2.0, out=out) == float("inf")
    for g, b in zip(out or grads, before):
        assert (np.abs(f64(g) - b * (2.0 / want)) <= np.abs(b) * (2.0 / want) * (HALF[g.dtype] + 3 * EPS32)).all()
    assert abs(lib.gradient_norm(out or grads).item() - 2.0) <= 2.0 * (HALF[torch.bfloat16] + 3 * EPS32)


@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("size", [1e-3, 1e38])
def test_an_infinity_or_a_nan_among_the_gradients(lib, bad, dtype, size):
    """The same norm as above may come with it, but then nothing is scaled, here or elsewhere."""
    grads = [torch.full((9000,), size, device="cuda"), torch.ones(100, dtype=dtype, device="cuda")]
    grads[1][77] = bad
    before, out = [g.clone() for g in grads], [torch.zeros_like(g) for g in grads]
    for places in (out, None):
        norm = lib.clip_gradients(grads, 1e-4, out=places)
        assert norm.isnan() if bad != bad else norm == float("inf")
        for g, b in zip(places or grads, before):
            assert torch.equal(g.nan_to_num(nan=123.0), b.nan_to_num(nan=123.0))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=str)
def test_the_roundings_of_a_result(lib, dtype):
    """From float64 to float32 and from there to the type, under the factor that the norm makes."""
    g = torch.randn(400000, generator=torch.Generator().manual_seed(3)).to(dtype)
    max_norm = float(np.float32(300.7))
    out = torch.empty_like(g, device="cuda")
    lib.clip_gradients([g.cuda()], max_norm, out=[out])
    want = (g.double() * (max_norm / norm64(g))).float().to(dtype)
    # the order of the sum moves the factor by some of float64's steps, 2^-29 of float32's: hardly a result falls the other way
    assert (out.cpu() != want).sum() <= 2
