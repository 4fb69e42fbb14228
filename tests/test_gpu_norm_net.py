"""Group normalisation and 8-bit checkpoints in a training step with the library's dense layers and loss, as a net would use them:
maps -> normalisation and activation (keeps its input in 8 bits) -> dense layer -> rectifier (kept in 8 bits) -> dense layer -> loss,
and back from what was kept."""
import numpy as np
import pytest
import torch

import norm_reference as R
import synthetic_inputs as S
from test_gpu_group_norm import check_backward, check_forward, f64, kept_values

pytestmark = pytest.mark.gpu

FP32_PRODUCT = 2.0 ** -20  # of sums of up to 256 float32 products, relative to the sum of their magnitudes


def near(got, want, tol, what):
    off = np.abs(f64(got) - want)
    assert np.all(off <= tol), (what, float(np.max(off / tol)))


@pytest.mark.parametrize("code", [torch.int8, torch.float8_e4m3fn], ids=str)
@pytest.mark.parametrize("batch", [1, 7, 64])
def test_a_training_step(lib, batch, code):
    net = lib.AlexNet(S.MINI, batch)
    gen = torch.Generator().manual_seed(batch)

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=gen) * std).cuda()

    c, groups = 32, 8
    x = normal(batch, 2, 2, c) + 0.3  # the last stage's maps, 128 features of a picture
    gamma, beta = 1 + normal(c, std=0.2), normal(c, std=0.2)
    w6, b6, w7, b7, w8, b8 = (normal(*s, std=d) for s, d in (((256, 128), 0.1), ((256,), 0.1), ((256, 256), 0.1), ((256,), 0.1),
                                                              ((10, 256), 0.1), ((10,), 0.1)))
    labels = torch.randint(0, 10, (batch,), generator=gen, dtype=torch.int32)

    # forward: of every layer's input only 8 bits stay
    y, mean, rstd, kept_x = lib.group_norm_forward(x, gamma, beta, groups, 1e-5, "silu", checkpoint=code)
    flat = y.view(batch, 128)
    kept6 = lib.checkpoint_pack(flat, code)
    h6 = net.fc_forward(6, flat, w6, b6, relu=True)
    kept7 = lib.checkpoint_pack(h6, code)
    h7 = net.fc_forward(7, h6, w7, b7, relu=True)
    kept8 = lib.checkpoint_pack(h7, code)
    dz, _ = net.softmax_xent(net.fc_forward(8, h7, w8, b8), labels)

    # and back
    dw8, db8 = lib.checkpoint_fc_backward_weight(kept8, dz)
    d7 = net.fc_backward(8, h7, w8, dz)[0] * (h7 > 0)
    dw7, db7 = lib.checkpoint_fc_backward_weight(kept7, d7)
    d6 = net.fc_backward(7, h6, w7, d7)[0] * (h6 > 0)
    dw6, db6 = lib.checkpoint_fc_backward_weight(kept6, d6)
    dflat = net.fc_backward(6, flat, w6, d6)[0]
    dx, dgamma, dbeta = lib.group_norm_backward(kept_x, dflat.view(x.shape), mean, rstd, gamma, beta, "silu")

    # each operator for its own inputs
    check_forward(x.reshape(batch, 4, c), gamma, beta, groups, 1e-5, "silu", (y, mean, rstd))
    check_backward(kept_values(lib, kept_x).reshape(batch, 4, c), dflat.view(batch, 4, c), mean, rstd, gamma, beta, "silu",
                   (dx, dgamma, dbeta))
    # and the weights' gradients for the whole step in 64 bits: a kept value is off by a 16th of itself (e4m3) or, with its
    # block's largest value, by a 127th of that (int8) at most; sums in float32 add FP32_PRODUCT a layer
    h, grads = [f64(flat)], []
    for w, b in ((w6, b6), (w7, b7)):
        h.append(np.maximum(h[-1] @ f64(w).T + f64(b), 0))
    logits = h[-1] @ f64(w8).T + f64(b8)
    p = np.exp(logits - logits.max(1, keepdims=True))
    d = p / p.sum(1, keepdims=True)
    d[np.arange(batch), labels.numpy()] -= 1
    d /= batch
    gates = [None, f64(h6) > 0, f64(h7) > 0]
    for got_w, got_b, a, w, gate in ((dw8, db8, h[2], w8, gates[2]), (dw7, db7, h[1], w7, gates[1]), (dw6, db6, h[0], w6, None)):
        rows, cols = a.shape
        most = np.abs(a).reshape(rows, -1, 32).max(2).repeat(32, 1)
        off = most / 127 if code == torch.int8 else np.maximum(np.abs(a) / 16, most * 2.0 ** -17)
        size = np.abs(d).max() + 0 * np.abs(d)
        near(got_w, d.T @ a, np.abs(d).T @ off + 64 * FP32_PRODUCT * (size.T @ most), "dw")
        near(got_b, d.sum(0), 64 * FP32_PRODUCT * size.sum(0), "db")
        d = d @ f64(w) * (1 if gate is None else gate)
    net.close()
