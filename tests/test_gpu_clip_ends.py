"""Clipping at the ends of float32: norms past its range, infinities, NaNs."""
import numpy as np
import pytest
import torch

from dense8_reference import EPS32, HALF, f64

pytestmark = pytest.mark.gpu


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
