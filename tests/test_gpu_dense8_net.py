"""A run of the operators together, as a residual net of dense layers uses them: normalisation with the residual, products in 8 bits,
their gradients, clipping of all gradients at once, beside group normalisation's checkpoint and the dense weight gradient from one."""
import numpy as np
import pytest
import torch

import dense8_reference as R
from dense8_reference import f64

pytestmark = pytest.mark.gpu

E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2
EPS = 1e-5


def forward(lib, x, params):
    """Residual blocks: h += w(norm(h)).  Returns the last sum's normalisation and what the backward pass wants."""
    kept, h, branch = [], x, None
    for gamma, w in params:
        y, s, rstd = lib.rms_norm_forward(h, gamma, residual=branch, eps=EPS)
        (q, q_t), (w8, w8_t) = lib.block8_pack(y, E4M3, along="both"), lib.block8_pack(w, E4M3, True, "both")
        kept.append((s, rstd, gamma, q_t, w8_t))
        h, branch = s, lib.block8_product(q, w8, x.dtype)
    return lib.rms_norm_forward(h, None, residual=branch, eps=EPS), kept


def backward(lib, top, kept, dy):
    """Gradients of every gamma and w, and of x."""
    _, s, rstd = top
    grads = []
    dh, _ = lib.rms_norm_backward(s, dy, rstd, None)  # of the sum: of the stream and of the last branch alike
    for s, rstd, gamma, q_t, w8_t in reversed(kept):
        d, d_t = lib.block8_pack(dh, E5M2, along="both")
        dw = lib.block8_product(d_t, q_t, torch.float32)
        dy = lib.block8_product(d, w8_t, dh.dtype)
        dh, dgamma = lib.rms_norm_backward(s, dy, rstd, gamma, dsum=dh)
        grads += [dw, dgamma]
    return dh, grads[::-1]


def inputs(rows, cols, depth, dtype, seed=0):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, cols), generator=gen).to(dtype).cuda()
    params = [((1 + 0.1 * torch.randn(cols, generator=gen)).cuda(), (torch.randn((cols, cols), generator=gen) / cols ** 0.5).cuda()) for _ in range(depth)]
    return x, params, (torch.randn((rows, cols), generator=gen) / rows).to(dtype).cuda()


def plain(x, params, dy):
    """The same net in 64 bits without any rounding, and its gradients."""
    x = x.double().cpu().requires_grad_()
    params = [(g.double().cpu().requires_grad_(), w.double().cpu().requires_grad_()) for g, w in params]
    h, branch = x, None
    norm = lambda s: s / torch.sqrt((s * s).mean(1, keepdim=True) + EPS)  # noqa: E731
    for g, w in params:
        h = h if branch is None else h + branch
        branch = (norm(h) * g) @ w.t()
    y = norm(h + branch)
    y.backward(dy.double().cpu())
    return y.detach(), x.grad, [p.grad for pair in params for p in pair]


@pytest.mark.parametrize("rows,cols", [(200, 256), (37, 300), (700, 130)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_a_training_step(lib, rows, cols, dtype):
    """Against the net without rounding.  A code is off by half a step at most, 2^-4 of a value (E5M2 2^-3) where values are spread
    evenly 0.29 of a step, so a product's relative error (2-norm) is near 0.29 * (2^-3 + 2^-3) * 2^-0.5 from its two operands, 0.04 at most;
    of gradients, with E5M2 on one side, 0.06 at most; three layers' errors add up to under three times one's."""
    x, params, dy = inputs(rows, cols, 3, dtype)
    top, kept = forward(lib, x, params)
    dx, grads = backward(lib, top, kept, dy)
    want_y, want_dx, want = plain(x, params, dy)

    def rel(a, b):
        return ((a.double().cpu() - b).norm() / b.norm()).item()

    assert rel(top[0], want_y) < 3 * 0.04
    assert rel(dx, want_dx) < 3 * 0.06 + 3 * 0.04
    for got, w in zip(grads, [g for pair in zip(want[0::2], want[1::2]) for g in pair]):
        assert rel(got, w) < 3 * 0.06 + 3 * 0.04
    # and the update's side: all gradients together
    norm = lib.gradient_norm(grads)
    exact = np.sqrt(sum((f64(g) ** 2).sum() for g in grads))
    assert abs(norm.item() - exact) <= 1.01 * R.EPS32 * exact
    clipped = [torch.empty_like(g) for g in grads]
    lib.clip_gradients(grads, exact / 3, out=clipped)
    assert abs(lib.gradient_norm(clipped).item() * 3 / exact - 1) < 8 * R.EPS32


def test_the_whole_step_captured_and_replayed(lib):
    """One graph of forward, backward and clipping; other inputs, eager work and another graph of the same operators between replays."""
    x, params, dy = inputs(150, 384, 2, torch.bfloat16, 5)

    def run():
        top, kept = forward(lib, x, params)
        dx, grads = backward(lib, top, kept, dy)
        norm = lib.clip_gradients(grads, 0.01)
        return [top[0], dx, norm, *grads]

    run()
    torch.cuda.synchronize()
    graphs, results = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            results.append(run())
        graphs.append(graph)
    for turn in range(4):
        x.mul_(-1.1)
        dy.mul_(1.3)
        for graph in graphs[::1 if turn % 2 else -1]:
            graph.replay()
        eager = run()
        torch.cuda.synchronize()
        for result in results:
            assert all(torch.equal(a, b) for a, b in zip(result, eager)), turn


def test_two_steps_at_once_on_two_streams(lib):
    """Calls share nothing: two nets on two streams, none waiting for the other."""
    sets = [inputs(300, 256, 2, torch.bfloat16, seed) for seed in (1, 2)]

    def run(s):
        x, params, dy = s
        top, kept = forward(lib, x, params)
        dx, grads = backward(lib, top, kept, dy)
        return [top[0], dx, lib.clip_gradients(grads, 0.01), *grads]

    want = [run(s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(5):
        got = []
        for s, stream in zip(sets, streams):
            with torch.cuda.stream(stream):
                got.append(run(s))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, w in zip(got, want) for a, b in zip(g, w))


def test_weight_gradient_from_the_normalisations_codes(lib):
    """Blocks of 128 are blocks of 32 that share a scale: the codes that the forward pass left serve the weight gradient that takes a
    checkpoint, without packing the input along its columns."""
    rows, cols, out = 300, 256, 100
    x, _, _ = inputs(rows, cols, 0, torch.bfloat16)
    dy = (torch.randn((rows, out), generator=torch.Generator().manual_seed(3)) / rows).to(torch.bfloat16).cuda()
    blocks, _, _ = lib.rms_norm_forward(x, None, eps=EPS, blocks=E4M3)
    kept = lib.Checkpoint(blocks.codes, blocks.scales[:, :rows].t().repeat_interleave(4, 1).contiguous())
    dw, db = lib.checkpoint_fc_backward_weight(kept, dy)
    v = f64(lib.block8_unpack(blocks))
    want = f64(dy).T @ v
    assert (np.abs(f64(dw) - want) <= 400 * R.EPS32 * (np.abs(f64(dy)).T @ np.abs(v)) + 1e-38).all()
    assert np.allclose(f64(db), f64(dy).sum(0), rtol=0, atol=400 * R.EPS32 * np.abs(f64(dy)).sum())
