"""CPU-only: what group normalisation and the 8-bit checkpoints refuse, before any GPU work, and the tests' own references
against brute force."""
import ctypes as C
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

import norm_reference as R


@pytest.fixture(scope="module")
def B():
    from paper_1412_2302_amd import binding
    return binding


def cfg(B, **kw):
    v = dict(n=2, hw=9, c=8, groups=2, type=0, act=0, eps=1e-5)
    v.update(kw)
    return B.GroupNormCfg(*[v[k] for k in ("n", "hw", "c", "groups", "type", "act", "eps")])


@pytest.mark.parametrize("change,code", [
    (dict(type=3), "EINVAL"), (dict(type=-1), "EINVAL"), (dict(act=3), "EINVAL"), (dict(act=-1), "EINVAL"), (dict(eps=0.0), "EINVAL"),
    (dict(eps=-1.0), "EINVAL"), (dict(eps=float("nan")), "EINVAL"), (dict(eps=float("inf")), "EINVAL"), (dict(n=-1), "ESHAPE"),
    (dict(hw=-1), "ESHAPE"), (dict(c=0), "ESHAPE"), (dict(groups=0), "ESHAPE"), (dict(groups=3), "ESHAPE"),
    (dict(c=(1 << 20) + 8), "ESHAPE"), (dict(hw=(1 << 28) + 1), "ESHAPE"), (dict(n=1 << 21, groups=2), "ESHAPE"),
    (dict(n=1 << 20, c=1 << 13, groups=1), "ESHAPE")])
def test_configurations_that_are_refused(B, change, code):
    ws, ws2 = C.c_size_t(), C.c_size_t()
    c = cfg(B, **change)
    for rc in (B._lib.alexnet_group_norm_query(c, 0, ws, ws2),
               B._lib.alexnet_group_norm_forward(c, 256, 1 << 20, None, None, 512, 1 << 20, None, None, None, 1024, 1 << 40, None),
               B._lib.alexnet_group_norm_backward(c, 256, 1 << 20, None, 512, 1 << 20, 256, 256, None, None, 512, 1 << 20, None, None,
                                                  1024, 1 << 40, None)):
        assert rc == getattr(B, code) and "group_norm" in B.last_error()


def test_arguments_that_are_refused(B):
    ws, ws2 = C.c_size_t(), C.c_size_t()
    q = B._lib.alexnet_group_norm_query
    assert q(None, 0, ws, ws2) == q(cfg(B), 0, None, ws2) == q(cfg(B), 0, ws, None) == B.EINVAL
    # maps that no workgroup holds: both passes need scratch
    c = cfg(B, n=3, hw=100000)
    assert q(c, 0, ws, ws2) == B.OK
    need, need_b = ws.value, ws2.value
    assert need > 0 and need_b > 0
    kept = B.CheckpointArg(256, 512, 0)

    def forward(x=256, ld_x=8, gamma=None, beta=None, y=512, ld_y=8, mean=None, rstd=None, keep=None, work=1024, size=1 << 40, conf=c):
        return B._lib.alexnet_group_norm_forward(conf, x, ld_x, gamma, beta, y, ld_y, mean, rstd, keep, work, size, None)

    def backward(x=256, ld_x=8, kept=None, dy=512, ld_dy=8, mean=256, rstd=256, dx=512, ld_dx=8, dgamma=None, work=1024, size=1 << 40, conf=c):
        return B._lib.alexnet_group_norm_backward(conf, x, ld_x, kept, dy, ld_dy, mean, rstd, None, None, dx, ld_dx, dgamma, None, work,
                                                  size, None)

    assert forward(x=None) == forward(y=None) == B.EINVAL
    assert forward(ld_x=7) == forward(ld_y=7) == forward(ld_x=-8) == B.ESHAPE
    assert forward(x=257) == forward(y=514) == forward(gamma=3) == forward(beta=2) == forward(mean=1) == forward(rstd=2) == B.EALIGN
    assert forward(x=257, conf=cfg(B, type=1)) == B.EALIGN
    assert forward(keep=B.CheckpointArg(None, 512, 0)) == forward(keep=B.CheckpointArg(256, None, 0)) == B.EINVAL
    assert forward(keep=B.CheckpointArg(256, 512, 2)) == forward(keep=B.CheckpointArg(256, 512, -1)) == B.EINVAL
    assert forward(size=need - 1) == forward(work=None) == B.ENOMEM and "workspace" in B.last_error()
    assert forward(work=1028) == backward(work=1028) == B.EALIGN
    assert backward(size=need_b - 1) == backward(work=None) == B.ENOMEM
    # one picture whose groups fit a workgroup: none
    assert q(cfg(B, n=1), 1, ws, ws2) == B.OK and ws.value == 0 and ws2.value == 0
    assert backward(x=None) == backward(kept=kept) == backward(dy=None) == backward(mean=None) == backward(rstd=None) == B.EINVAL
    assert backward(dx=None) == B.EINVAL
    assert backward(ld_x=7) == backward(ld_dy=7) == backward(ld_dx=7) == backward(x=None, kept=kept, ld_dy=7) == B.ESHAPE
    assert backward(x=258) == backward(dy=513) == backward(dx=514) == backward(mean=2) == backward(dgamma=6) == B.EALIGN
    assert backward(x=None, kept=B.CheckpointArg(256, 512, 7)) == B.EINVAL


def test_results_that_overlap_an_input_are_refused(B):
    """In place means the same pixels; another place has no byte of the input's."""
    n, hw, c, ld = 2, 9, 8, 24
    conf = cfg(B, n=n, hw=hw, c=c)
    reach = ((n * hw - 1) * ld + c) * 4
    x = 1 << 20

    def forward(y, ld_y=ld):
        return B._lib.alexnet_group_norm_forward(conf, x, ld, None, None, y, ld_y, None, None, None, None, 0, None)

    def backward(dx, dy, ld_dx=ld, x=x):
        ws = 1 << 30  # scratch of two pictures
        return B._lib.alexnet_group_norm_backward(conf, x, ld, None, dy, ld, 256, 256, None, None, dx, ld_dx, None, None, ws, 1 << 20,
                                                  None)

    for y, ld_y in [(x + 4, ld), (x - 4, ld), (x + 28, ld), (x - 28, ld), (x + ld * 4, ld), (x + 68, ld), (x, ld + 1), (x, c),
                    (x + reach - 4, ld), (x + reach - 4, c), (x - reach + 4, ld)]:
        assert forward(y, ld_y) == B.EINVAL and "overlaps" in B.last_error(), (y - x, ld_y)
        assert backward(y, 1 << 25, ld_y) == B.EINVAL and "overlaps" in B.last_error()
        assert backward(y, x, ld_y, 1 << 25) == B.EINVAL and "overlaps" in B.last_error()


def test_checkpoint_arguments_that_are_refused(B):
    k = B.CheckpointArg(256, 512, 0)
    pack, unpack, fc = B._lib.alexnet_checkpoint_pack, B._lib.alexnet_checkpoint_unpack, B._lib.alexnet_checkpoint_fc_backward_weight
    assert pack(None, 8, 0, 4, 8, k, None) == pack(256, 8, 3, 4, 8, k, None) == pack(256, 8, 0, 4, 8, None, None) == B.EINVAL
    assert pack(256, 7, 0, 4, 8, k, None) == pack(256, 8, 0, -1, 8, k, None) == pack(256, 8, 0, 4, 0, k, None) == B.ESHAPE
    assert pack(258, 8, 0, 4, 8, k, None) == pack(257, 8, 1, 4, 8, k, None) == B.EALIGN
    assert pack(256, 8, 0, 1 << 30, 1 << 20, k, None) == B.ESHAPE
    assert pack(256, 8, 0, 4, 8, B.CheckpointArg(256, 512, 2), None) == B.EINVAL
    assert unpack(k, 4, 8, None, 8, 0, None) == unpack(None, 4, 8, 256, 8, 0, None) == unpack(k, 4, 8, 256, 8, 9, None) == B.EINVAL
    assert unpack(k, 4, 8, 256, 7, 0, None) == unpack(k, 4, (1 << 20) + 1, 256, 1 << 21, 0, None) == B.ESHAPE
    assert unpack(k, 4, 8, 254, 8, 0, None) == B.EALIGN
    ws = C.c_size_t()
    q = B._lib.alexnet_checkpoint_fc_query
    assert q(4, 8, 8, 5, ws) == q(4, 8, 8, 0, None) == B.EINVAL
    assert q(-1, 8, 8, 0, ws) == q(4, 0, 8, 0, ws) == q(4, 8, 0, 0, ws) == q(4, 1 << 21, 8, 0, ws) == B.ESHAPE
    assert q(5000, 256, 64, 0, ws) == B.OK
    assert q(1 << 22, 1 << 17, 1 << 16, 0, ws) == B.ESHAPE and "launch" in B.last_error()  # 1024 slices of 2^17 tiles and more
    big = 1 << 40

    def weight(x=k, dy=256, ld=8, kind=0, rows=4, cols=8, out=8, dw=512, db=None, work=1024, size=big):
        return fc(x, dy, ld, kind, rows, cols, out, dw, db, work, size, None)

    assert weight(x=None) == weight(dy=None) == weight(dw=None) == weight(kind=7) == weight(x=B.CheckpointArg(256, 512, 5)) == B.EINVAL
    assert weight(ld=7) == weight(rows=-1) == weight(cols=0) == weight(out=0) == B.ESHAPE
    assert weight(dy=258) == weight(dw=514) == weight(db=513) == B.EALIGN
    rows = 100000
    assert q(rows, 64, 64, 0, ws) == B.OK
    if ws.value:
        assert weight(rows=rows, cols=64, out=64, ld=64, size=ws.value - 1) == B.ENOMEM
        assert weight(rows=rows, cols=64, out=64, ld=64, work=None) == B.ENOMEM
        assert weight(rows=rows, cols=64, out=64, ld=64, work=1028) == B.EALIGN


def test_the_binding_refuses_tensors_of_the_wrong_kind(B):
    x = torch.zeros(2, 9, 8)
    with pytest.raises(ValueError, match="device tensor"):
        B.group_norm_forward(x, None, None, 2)
    with pytest.raises(TypeError):
        B.checkpoint_pack([1.0])
    with pytest.raises(ValueError, match="scales"):
        B.Checkpoint(torch.zeros(4, 40, dtype=torch.int8), torch.zeros(4, 1, dtype=torch.uint8))
    with pytest.raises(ValueError, match="int8 or float8"):
        B.Checkpoint(torch.zeros(4, 40), torch.zeros(4, 2, dtype=torch.uint8))
    with pytest.raises(ValueError, match="belong"):
        B.Checkpoint(torch.empty(1, 1 << 31, dtype=torch.int8, device="meta"), torch.empty(1, 1 << 26, dtype=torch.uint8, device="meta"))
    with pytest.raises(ValueError, match="contiguous"):
        B.Checkpoint(torch.zeros(40, 4, dtype=torch.int8).t(), torch.zeros(4, 2, dtype=torch.uint8))
    with pytest.raises(ValueError, match="device tensor"):
        B.checkpoint_unpack(B.Checkpoint(torch.zeros(4, 40, dtype=torch.int8), torch.zeros(4, 2, dtype=torch.uint8)))
    with pytest.raises(ValueError, match="activation"):
        B._group_norm_cfg(1, 4, 8, 2, 0, "tanh", 1e-5, False)


def test_the_reference_codes_by_brute_force():
    """norm_reference.code against a search over all codes and scales."""
    gen = np.random.default_rng(1)
    grid8 = np.arange(256, dtype=np.uint8)
    tables = {torch.int8: np.arange(-127, 128).astype(np.float64),
              torch.float8_e4m3fn: torch.from_numpy(grid8).view(torch.float8_e4m3fn).float().numpy().astype(np.float64)}
    for kind, table in tables.items():
        table = np.unique(table[np.isfinite(table)])
        for spread in (1e-3, 1.0, 300.0):
            x = (gen.normal(size=(3, 40)) * spread * np.exp(gen.normal(size=(3, 40)))).astype(np.float32).astype(np.float64)
            codes, scales = R.code(x, kind)
            for r in range(3):
                for b in range(2):
                    part, cols = x[r, 32 * b:32 * b + 32], codes[r, 32 * b:32 * b + 32]
                    s = 2.0 ** (float(scales[r, b]) - 127)
                    assert np.abs(part).max() <= table[-1] * s and np.abs(part).max() > table[-1] * s / 2
                    best = np.abs(part[:, None] / s - table).min(axis=1)
                    assert np.array_equal(np.abs(part / s - cols), best) and np.isin(cols, table).all()


def test_the_reference_gradients_by_differences():
    gen = np.random.default_rng(2)
    x, dy = gen.normal(size=(2, 5, 6)), gen.normal(size=(2, 5, 6))
    gamma, beta = gen.normal(size=6) + 1, gen.normal(size=6)
    for act in ("none", "relu", "silu"):
        _, mean, rstd, _ = R.forward(x, gamma, beta, 2, 1e-3, act)
        dx, dgamma, dbeta = R.backward(x, dy, mean, rstd, gamma, beta, act)

        def loss(x, g, b):
            return (R.forward(x, g, b, 2, 1e-3, act)[0] * dy).sum()

        h = 1e-6
        for at in np.ndindex(x.shape):
            e = np.zeros_like(x)
            e[at] = h
            assert abs((loss(x + e, gamma, beta) - loss(x - e, gamma, beta)) / (2 * h) - dx[at]) < 1e-7
        for i in range(6):
            e = np.eye(6)[i] * h
            assert abs((loss(x, gamma + e, beta) - loss(x, gamma - e, beta)) / (2 * h) - dgamma[i]) < 1e-7
            assert abs((loss(x, gamma, beta + e) - loss(x, gamma, beta - e)) / (2 * h) - dbeta[i]) < 1e-7


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_slabs_cover_the_picture_and_fit(tmp_path):
    exe = str(tmp_path / "norm_plan_check")
    src = os.path.join(os.path.dirname(os.path.abspath(__file__)), "emu", "norm_plan_check.cpp")
    subprocess.run(["g++", "-O1", "-std=c++17", "-fsanitize=address,undefined", "-o", exe, src], check=True, timeout=300)
    out = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and out.stdout.startswith("OK"), out.stdout + out.stderr
