"""Training with 8-bit checkpoints in the place of what they were made from: where a rectifier's gates move, and dense layers
whose inputs are dropped after the forward pass."""
import pytest
import torch

import norm_reference as R
import synthetic_inputs as S

pytestmark = pytest.mark.gpu

CODES = [torch.int8, torch.float8_e4m3fn]
FP32_PRODUCT = 2.0 ** -20  # of the dense layers' sums of up to 256 float32 products, relative to the sum of their magnitudes


def wide(stat, c):
    return stat.double().repeat_interleave(c // stat.shape[1], 1)[:, None]


@pytest.mark.parametrize("size", [(4, 169, 384, 32), (2, 3025, 96, 32)], ids=str)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("code", CODES, ids=str)
def test_gates_of_a_rectifier_behind_a_checkpoint(lib, size, dtype, code):
    """The backward pass gates by the unpacked values.  A gate differs from the forward pass's where x and its unpacked value lie
    on either side of the border, so where |z| is at most r |gamma| times their distance: at most half a step, which is a 127th of
    the block's largest value (int8), or a 16th of the value, near zero 2^-17 of the block's largest (e4m3)."""
    n, hw, c, groups = size
    gen = torch.Generator(device="cuda").manual_seed(c)
    x = (torch.randn((n, hw, c), device="cuda", generator=gen) + torch.randn(c, device="cuda", generator=gen) * 0.5).to(dtype)
    gamma, beta = torch.randn(c, device="cuda", generator=gen) * 0.2 + 1, torch.randn(c, device="cuda", generator=gen) * 0.2
    y, mean, rstd, kept = lib.group_norm_forward(x, gamma, beta, groups, 1e-5, "relu", checkpoint=code)
    _, _, open_kept = lib.group_norm_backward(kept, torch.ones_like(x), mean, rstd, gamma, beta, "relu")
    _, _, open_x = lib.group_norm_backward(x, torch.ones_like(x), mean, rstd, gamma, beta, "relu")
    back = lib.checkpoint_unpack(kept, torch.float32).double()
    slope = wide(rstd, c) * gamma.double()
    z, z_kept = ((v - wide(mean, c)) * slope + beta.double() for v in (x.double(), back))
    assert torch.equal(open_x.double(), (z > 0).double().sum((0, 1))) and torch.equal(open_kept.double(), (z_kept > 0).double().sum((0, 1)))
    most = torch.nn.functional.pad(x.double().abs(), (0, -c % 32)).view(n, hw, -1, 32).amax(3).repeat_interleave(32, 2)[..., :c]
    step = most / 127 if code == torch.int8 else torch.maximum(x.double().abs() / 16, most * 2.0 ** -17)
    moved = (z > 0) != (z_kept > 0)
    assert bool((z[moved].abs() <= (slope.abs() * step)[moved] * (1 + 1e-12) + 1e-14).all())
    print(f"{code} {dtype}: {float(moved.double().mean()):.2%} of the gates move")


@pytest.mark.parametrize("code", CODES, ids=str)
@pytest.mark.parametrize("batch", [1, 7, 64])
def test_dense_layers_whose_inputs_are_dropped(lib, batch, code):
    """Between the passes only checkpoints stay.  The data gradient comes from fc_backward, which is given the unpacked input and
    leaves a weight gradient too: the same as the one from the checkpoint, to the rounding of sums."""
    net = lib.AlexNet(S.MINI, batch)
    gen = torch.Generator(device="cuda").manual_seed(batch)

    def normal(*shape, std=1.0):
        return torch.randn(shape, device="cuda", generator=gen) * std

    flat = normal(batch, 128)
    w6, b6, w7, b7, w8, b8 = (normal(*s, std=0.1) for s in ((256, 128), (256,), (256, 256), (256,), (10, 256), (10,)))
    labels = torch.randint(0, 10, (batch,), device="cuda", generator=gen, dtype=torch.int32)
    h, kept = flat, []
    for layer, w, b in ((6, w6, b6), (7, w7, b7), (8, w8, b8)):
        kept.append(lib.checkpoint_pack(h, code))
        h = net.fc_forward(layer, h, w, b, relu=layer < 8)
    dz, _ = net.softmax_xent(h, labels)
    del h, flat
    for layer, w in ((8, w8), (7, w7), (6, w6)):
        k = kept[layer - 6]
        x = lib.checkpoint_unpack(k)
        dw, db = lib.checkpoint_fc_backward_weight(k, dz)
        dx, dw_too, db_too = net.fc_backward(layer, x, w, dz)
        d, xd = dz.double(), x.double()
        k1 = (batch + 64) * R.EPS32  # an accumulator is rounded at most once a product
        for gradient, bias, off in ((dw, db, k1), (dw_too, db_too, FP32_PRODUCT)):
            assert bool(((gradient.double() - d.t().contiguous() @ xd).abs() <= off * (d.abs().t().contiguous() @ xd.abs()) + 1e-38).all())
            assert bool(((bias.double() - d.sum(0)).abs() <= off * d.abs().sum(0) + 1e-38).all())
        assert bool(((dx.double() - d @ w.double()).abs() <= FP32_PRODUCT * (d.abs() @ w.double().abs()) + 1e-38).all())
        dz = dx * (x > 0)
    net.close()
