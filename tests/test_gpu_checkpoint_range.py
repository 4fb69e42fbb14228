"""What the weight gradient reads from a checkpoint: every code under every scale, value by value."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

SCALES = 247  # 448 * 2^(246 - 127) is the largest finite e4m3 value of a power-of-two scale


@pytest.mark.parametrize("code", [torch.int8, torch.float8_e4m3fn], ids=str)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("out", [SCALES, 4099])  # tiles of 64 x 64 and of 128 x 256
def test_every_code_and_scale_is_multiplied_as_its_value(lib, code, dtype, out):
    """dy is one in a place of its own per row: a row of dw is a row of values.  Those are exact in bfloat16 but for e4m3 under
    2^-126, which are rounded to its multiples of 2^-133: by 2^-134 at most."""
    raw = torch.arange(256, dtype=torch.uint8).view(1, 256).repeat(SCALES, 9 if out > SCALES else 1)
    if code == torch.float8_e4m3fn:
        raw[(raw & 127) == 127] = 0  # not a number
    scales = torch.arange(SCALES, dtype=torch.uint8).view(SCALES, 1).repeat(1, raw.shape[1] // 32)
    want = raw.view(code).float().numpy().astype(np.float64) * np.exp2(np.arange(SCALES) - 127.0)[:, None]
    dy = torch.zeros((SCALES, out))
    dy[torch.arange(SCALES), out - 1 - torch.arange(SCALES)] = 1
    dw, db = lib.checkpoint_fc_backward_weight(lib.Checkpoint(raw.view(code).cuda(), scales.cuda()), dy.to(dtype).cuda())
    got = dw.flip(0)[:SCALES].double().cpu().numpy()
    assert torch.equal(db.cpu(), dy.sum(0)) and bool((dw.flip(0)[SCALES:] == 0).all())
    if code == torch.int8:
        assert np.array_equal(got, want)
    else:
        assert np.array_equal(got[3:], want[3:])
        assert np.all(np.abs(got - want) <= 2.0 ** -134) and np.array_equal(got[:3], np.round(want[:3] * 2.0 ** 133) / 2.0 ** 133)
