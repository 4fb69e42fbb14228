"""Timed workloads of group normalisation with an activation and of 8-bit activation checkpoints.

Activations are channel-last, [pictures][pixels][channels].  A case is one pass of one of these kinds:

  forward   y = act(group_norm(x)) with the statistics, as inference and the forward half of training call it
  backward  dx, dgamma, dbeta from x, dy and the statistics
  step      forward that leaves an 8-bit checkpoint of x, then the backward pass that reads it in place of x
  store     an activation put into 8 bits (one power-of-two scale per 32 channels of a pixel) and brought back
  weight    a dense layer's weight and bias gradient from the checkpoint of its input: dw = dy^T x, db = sum of dy

Sizes are those of the convolution maps and dense layers in synthetic_inputs.py, and pictures of 227 x 227.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
CODES = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
EPS = 1e-5
BLOCK = 32


def listed():
    return [
        # serving one picture: a single map of 13 x 13, so launches and latency are what it costs
        dict(name="forward_b1_13x13x256_fp32", kind="forward", n=1, hw=169, c=256, groups=32, act="relu", type="fp32", wide=0),
        # the widest activations of a large minibatch, 16 bits
        dict(name="forward_b256_27x27x256_bf16", kind="forward", n=256, hw=729, c=256, groups=32, act="silu", type="bf16", wide=0),
        # two whole pictures: groups of 206,116 values, far more than one workgroup holds
        dict(name="forward_b2_227x227x64_fp32", kind="forward", n=2, hw=51529, c=64, groups=16, act="relu", type="fp32", wide=0),
        # a small net's first map, minibatch of 16
        dict(name="backward_b16_29x29x16_fp32", kind="backward", n=16, hw=841, c=16, groups=4, act="relu", type="fp32", wide=0),
        # the largest backward pass: minibatch of 256
        dict(name="backward_b256_27x27x256_fp32", kind="backward", n=256, hw=729, c=256, groups=32, act="relu", type="fp32", wide=0),
        # first map of the large net, three channels to a group: no group fills a vector
        dict(name="step_b128_55x55x96_fp32_int8", kind="step", n=128, hw=3025, c=96, groups=32, act="silu", type="fp32", code="int8"),
        # last, ragged minibatch of an epoch, 16 bits
        dict(name="step_b37_13x13x384_bf16_e4m3", kind="step", n=37, hw=169, c=384, groups=32, act="silu", type="bf16", code="e4m3"),
        # what a training run of 128 pictures keeps of its second layer
        dict(name="store_93312x256_fp32_int8", kind="store", rows=93312, cols=256, type="fp32", code="int8"),
        # odd sizes: the last block of every row is short and no row starts on a vector
        dict(name="store_8325x37_fp16_e4m3", kind="store", rows=8325, cols=37, type="fp16", code="e4m3"),
        # a small net's last dense layer
        dict(name="weight_16x256x10_fp32_int8", kind="weight", rows=16, cols=256, out=10, type="fp32", code="int8"),
        # the large net's first dense layer, minibatch of 256: the gradient itself is most of the traffic
        dict(name="weight_256x9216x4096_fp32_int8", kind="weight", rows=256, cols=9216, out=4096, type="fp32", code="int8"),
        # a 1 x 1 layer over the pixels of 256 maps: a long sum into a small gradient
        dict(name="weight_43264x384x384_bf16_e4m3", kind="weight", rows=43264, cols=384, out=384, type="bf16", code="e4m3"),
    ]


MAX_VALUES = 128 * 3025 * 96  # of an activation, and of the dense layers' operands together
MAX_PRODUCTS = 256 * 9216 * 4096


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _map(rng):
    """Pictures, pixels, channels and groups of one activation: groups of at least 16 values, since the gradient of a
    normalised pair is the rounding of two equal numbers."""
    while True:
        n, hw = _log_int(rng, 1, 256), rng.choice([_log_int(rng, 1, 60) ** 2, _log_int(rng, 1, 51529)])
        groups = rng.choice([1, 2, 3, 4, 7, 8, 16, 32, 32, 32])
        c = groups * _log_int(rng, 1, max(1, 1024 // groups))
        if n * hw * c <= MAX_VALUES and hw * (c // groups) >= 16:
            return dict(n=n, hw=hw, c=c, groups=groups)


def draw(rng):
    kind = rng.choice(["forward", "backward", "step", "store", "weight"])
    kind_of = rng.choice(["fp32", "fp32", "bf16", "fp16"])
    code = rng.choice(["int8", "e4m3"])
    if kind in ("forward", "backward"):
        wide = rng.choice([0, 0, 0, 8, 32])  # channels beside those of this operator in the same tensor
        return dict(kind=kind, **_map(rng), act=rng.choice(["none", "relu", "relu", "silu"]), type=kind_of, wide=wide)
    if kind == "step":
        # no relu: a gate hangs on the last bit of the forward pass's statistics
        return dict(kind=kind, **_map(rng), act=rng.choice(["none", "silu"]), type=kind_of, code=code)
    while True:
        rows = _log_int(rng, 1, 200000)
        cols = rng.choice([_log_int(rng, 1, 9216), 8 * _log_int(rng, 1, 1152)])
        if kind == "store" and rows * cols <= MAX_VALUES:
            return dict(kind=kind, rows=rows, cols=cols, type=kind_of, code=code)
        out = rng.choice([_log_int(rng, 1, 4096), 8 * _log_int(rng, 1, 512)])
        if kind == "weight" and rows * cols * out <= MAX_PRODUCTS and rows * (cols + out) <= MAX_VALUES:
            return dict(kind=kind, rows=rows, cols=cols, out=out, type=kind_of, code=code)


# ------------------------------------------------------------------ inputs ---
def _activation(gen, lead, c, dtype):
    """What a convolution leaves: channels of different scales and offsets."""
    scale = torch.rand(c, generator=gen, device="cuda") * 1.5 + 0.5
    shift = torch.randn(c, generator=gen, device="cuda") * 0.5
    return (torch.randn((*lead, c), generator=gen, device="cuda") * scale + shift).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = TYPES[case["type"]]
    if case["kind"] == "store":
        return {"case": case, "x": _activation(gen, (case["rows"],), case["cols"], dtype)}
    if case["kind"] == "weight":
        x = torch.relu(_activation(gen, (case["rows"],), case["cols"], torch.float32))  # the layer's input, behind a relu
        codes, exponent = _put(x, case["code"])
        dy = (torch.randn((case["rows"], case["out"]), generator=gen, device="cuda") / case["rows"]).to(dtype)
        return {"case": case, "codes": codes, "scales": (exponent + 127).to(torch.uint8), "dy": dy}
    n, hw, c, wide = case["n"], case["hw"], case["c"], case.get("wide", 0)
    x = _activation(gen, (n, hw), c + wide, dtype)[..., wide:]
    gamma = 1.0 + 0.2 * torch.randn(c, generator=gen, device="cuda")
    beta = 0.2 * torch.randn(c, generator=gen, device="cuda")
    state = {"case": case, "x": x, "gamma": gamma, "beta": beta}
    if case["kind"] != "forward":
        state["dy"] = (torch.randn((n, hw, c), generator=gen, device="cuda") * 0.1).to(dtype)
    if case["kind"] == "backward":
        state["mean"], state["rstd"] = _statistics(x.float(), case["groups"])
    return state


# -------------------------------------------------------------- plain forms ---
def _put(x, code):
    """Codes and exponents of x [rows][cols]: per 32 columns the smallest power of two that holds the largest value."""
    rows, cols = x.shape
    blocks = torch.nn.functional.pad(x.float(), (0, -cols % BLOCK)).view(rows, -1, BLOCK)
    part, power = torch.frexp(blocks.abs().amax(2))
    largest, bits = (127 / 128, 7) if code == "int8" else (448 / 512, 9)
    exponent = (power - bits + (part > largest).to(power.dtype)).clamp(min=-126)
    scaled = blocks * torch.exp2(-exponent.float())[..., None]
    scaled = torch.round(scaled) if code == "int8" else scaled
    return scaled.view(rows, -1)[:, :cols].contiguous().to(CODES[code]), exponent


def _values(codes, exponent):
    rows, cols = codes.shape
    scale = torch.exp2(exponent.float()).repeat_interleave(BLOCK, 1)[:, :cols]
    return codes.float() * scale


def _statistics(x, groups):
    n, hw, c = x.shape
    x = x.reshape(n, hw, groups, c // groups)
    mean = x.mean((1, 3))
    var = (x - mean[:, None, :, None]).square().mean((1, 3))
    return mean, torch.rsqrt(var + EPS)


def _over(stat, c):
    """[n][groups] as [n][1][c]."""
    return stat.repeat_interleave(c // stat.shape[1], 1)[:, None]


def _forward(x, gamma, beta, groups, act):
    mean, rstd = _statistics(x, groups)
    c = x.shape[2]
    z = (x - _over(mean, c)) * _over(rstd, c) * gamma + beta
    if act == "relu":
        z = torch.clamp(z, min=0.0)
    elif act == "silu":
        z = z / (1.0 + torch.exp(-z))
    return z, mean, rstd


def _backward(x, dy, mean, rstd, gamma, beta, act):
    n, hw, c = x.shape
    groups = mean.shape[1]
    hat = (x - _over(mean, c)) * _over(rstd, c)
    dz = dy
    if act == "relu":  # a gate is a border: in 64 bits
        z = (x.double() - _over(mean, c)) * _over(rstd, c).double() * gamma.double() + beta
        dz = torch.where(z > 0, dy, torch.zeros_like(dy))
    elif act == "silu":
        z = hat * gamma + beta
        s = 1.0 / (1.0 + torch.exp(-z))
        dz = dy * (s * (1.0 + z * (1.0 - s)))
    dbeta, dgamma = dz.sum((0, 1)), (dz * hat).sum((0, 1))
    g = dz * gamma
    a = g.view(n, hw, groups, -1).mean((1, 3))
    b = (g * hat).view(n, hw, groups, -1).mean((1, 3))
    return _over(rstd, c) * (g - _over(a, c) - hat * _over(b, c)), dgamma, dbeta


def _run_plain(state):
    case = state["case"]
    if case["kind"] == "weight":
        dy, x = state["dy"].float(), _values(state["codes"], state["scales"].int() - 127)
        return {"dw": dy.t() @ x, "db": dy.sum(0)}
    x = state["x"]
    if case["kind"] == "store":
        return {"values": _values(*_put(x, case["code"])).to(x.dtype)}
    gamma, beta, act = state["gamma"], state["beta"], case["act"]
    if case["kind"] == "backward":
        dx, dgamma, dbeta = _backward(x.float(), state["dy"].float(), state["mean"], state["rstd"], gamma, beta, act)
        return {"dx": dx.to(x.dtype), "dgamma": dgamma, "dbeta": dbeta}
    y, mean, rstd = _forward(x.float(), gamma, beta, case["groups"], act)
    out = {"y": y.to(x.dtype), "mean": mean, "rstd": rstd}
    if case["kind"] == "step":
        kept = _values(*_put(x.reshape(-1, case["c"]), case["code"])).view(x.shape)
        dx, dgamma, dbeta = _backward(kept, state["dy"].float(), mean, rstd, gamma, beta, act)
        out.update(dx=dx.to(x.dtype), dgamma=dgamma, dbeta=dbeta)
    return out


# --------------------------------------------------------------------- run ---
def _run_own(state):
    from paper_1412_2302_amd import binding as B

    case = state["case"]
    if case["kind"] == "weight":
        dw, db = B.checkpoint_fc_backward_weight(B.Checkpoint(state["codes"], state["scales"]), state["dy"])
        return {"dw": dw, "db": db}
    x = state["x"]
    if case["kind"] == "store":
        return {"values": B.checkpoint_unpack(B.checkpoint_pack(x, CODES[case["code"]]), x.dtype)}
    gamma, beta, act = state["gamma"], state["beta"], case["act"]
    if case["kind"] == "backward":
        dx, dgamma, dbeta = B.group_norm_backward(x, state["dy"], state["mean"], state["rstd"], gamma, beta, act)
        return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    keep = CODES[case["code"]] if case["kind"] == "step" else None
    y, mean, rstd, kept = B.group_norm_forward(x, gamma, beta, case["groups"], EPS, act, checkpoint=keep)
    out = {"y": y, "mean": mean, "rstd": rstd}
    if case["kind"] == "step":
        dx, dgamma, dbeta = B.group_norm_backward(kept, state["dy"], mean, rstd, gamma, beta, act)
        out.update(dx=dx, dgamma=dgamma, dbeta=dbeta)
    return out


def run(state):
    return _run_own(state) if own else _run_plain(state)


# -------------------------------------------------------------------- work ---
def work(case):
    """Inputs and outputs once; one multiply-add per term of a product, about ten operations per normalised value."""
    size = {"fp32": 4, "bf16": 2, "fp16": 2}[case["type"]]
    if case["kind"] == "weight":
        rows, cols, out = case["rows"], case["cols"], case["out"]
        kept = rows * (cols + math.ceil(cols / BLOCK))
        return {"bytes": float(kept + rows * out * size + 4 * out * (cols + 1)), "flops": 2.0 * rows * cols * out}
    if case["kind"] == "store":  # written and read back in 8 bits
        values, scales = case["rows"] * case["cols"], case["rows"] * math.ceil(case["cols"] / BLOCK)
        return {"bytes": float(values * (2 * size + 2) + 2 * scales), "flops": 4.0 * values}
    n, hw, c, groups = case["n"], case["hw"], case["c"], case["groups"]
    values, statistics = n * hw * c, 8 * n * groups
    if case["kind"] == "forward":
        return {"bytes": float(2 * values * size + 8 * c + statistics), "flops": 10.0 * values}
    if case["kind"] == "backward":
        return {"bytes": float(3 * values * size + 16 * c + statistics), "flops": 16.0 * values}
    kept = n * hw * (c + math.ceil(c / BLOCK))
    return {"bytes": float(4 * values * size + 2 * kept + 24 * c + 2 * statistics), "flops": 30.0 * values}


# ------------------------------------------------------------------- exact ---
def _round64(v, code):
    if code == "int8":
        return torch.round(v)
    # four significant bits down to 2^-6, steps of 2^-9 below
    step = torch.exp2(torch.clamp(torch.floor(torch.log2(v.abs().clamp(min=1e-300))), min=-6.0) - 3.0)
    return torch.round(v / step) * step


def _kept64(x, code):
    rows, cols = x.shape
    top = 127.0 if code == "int8" else 448.0
    full = torch.zeros((rows, math.ceil(cols / BLOCK) * BLOCK), dtype=torch.float64, device=x.device)
    full[:, :cols] = x
    full = full.reshape(rows, -1, BLOCK)
    most = full.abs().max(dim=2, keepdim=True).values
    scale = torch.exp2(torch.clamp(torch.ceil(torch.log2(most / top)), min=-126.0))
    return (_round64(full / scale, code) * scale).reshape(rows, -1)[:, :cols]


def exact(case, seed):
    state = prepare(case, seed)
    if case["kind"] == "weight":
        exponent = state["scales"].double() - 127.0
        block = torch.arange(case["cols"], device="cuda") // BLOCK
        x = state["codes"].double() * torch.exp2(exponent)[:, block]
        dy = state["dy"].double()
        return {"dw": torch.matmul(dy.t().contiguous(), x), "db": dy.sum(0)}
    x = state["x"].double()
    if case["kind"] == "store":
        return {"values": _kept64(x, case["code"])}
    n, hw, c = x.shape
    groups, gamma, beta = case["groups"], state["gamma"].double(), state["beta"].double()
    group = torch.arange(c, device="cuda") // (c // groups)
    count = hw * (c // groups)

    def per_group(t):  # sums over a group's pixels and channels, as [n][groups]
        return torch.zeros((n, groups), dtype=torch.float64, device="cuda").index_add_(1, group, t.sum(1))

    out = {}
    if case["kind"] == "backward":
        mean, rstd = state["mean"].double(), state["rstd"].double()
    else:
        mean = per_group(x) / count
        rstd = (per_group((x - mean[:, group].unsqueeze(1)) ** 2) / count + EPS) ** -0.5
        z = (x - mean[:, group].unsqueeze(1)) * rstd[:, group].unsqueeze(1) * gamma + beta
        y = {"none": lambda: z, "relu": lambda: z * (z > 0), "silu": lambda: z * torch.sigmoid(z)}[case["act"]]()
        out = {"y": y, "mean": mean, "rstd": rstd}
    if case["kind"] == "forward":
        return out
    if case["kind"] == "step":
        x = _kept64(x.reshape(-1, c), case["code"]).reshape(n, hw, c)
    hat = (x - mean[:, group].unsqueeze(1)) * rstd[:, group].unsqueeze(1)
    z = hat * gamma + beta
    sig = torch.sigmoid(z)
    slope = {"none": lambda: torch.ones_like(z), "relu": lambda: (z > 0).double(),
             "silu": lambda: sig + z * sig * (1.0 - sig)}[case["act"]]()
    dz = state["dy"].double() * slope
    first, second = per_group(dz * gamma) / count, per_group(dz * gamma * hat) / count
    dx = rstd[:, group].unsqueeze(1) * (dz * gamma - first[:, group].unsqueeze(1) - hat * second[:, group].unsqueeze(1))
    return {**out, "dx": dx, "dgamma": (dz * hat).sum((0, 1)), "dbeta": dz.sum((0, 1))}
