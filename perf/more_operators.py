"""Timed workloads of root-mean-square normalisation, of dense products in 8-bit floating point and of gradient clipping.

A case is one pass of one of these kinds:

  norm     s = x + residual, y = s / sqrt(mean(s^2) + eps) * gamma of every row, as inference calls it
  norm8    the same with y in 8 bits, ready for a product; returned are the values that the codes stand for
  step     norm, then its backward pass: the gradient of x (and residual) from dy and the gradient of s, and that of gamma
  product  y = a b^T of two operands that are in 8 bits already: rows of codes, one power-of-two scale per 128 of them, or,
           of a weight, per 128 x 128
  layer    one training pass of a dense layer: x, w and dy put into 8 bits along both of their sides, y = x w^T, dx = dy w,
           dw = dy^T x
  clip     gradients scaled to a norm over all of them together, if theirs is larger

Sizes are those of the convolution maps, dense layers and parameter tensors in synthetic_inputs.py, and generic ones.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
CODES = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
LARGEST = {"e4m3": (448 / 512, 9, 448.0), "e5m2": (57344 / 65536, 16, 57344.0)}  # fraction, power, number
EPS = 1e-5
BLOCK = 128

# weights and biases, layer by layer
NETS = {
    "small": [2352, 16, 6400, 32, 13824, 48, 10368, 48, 6912, 32, 32768, 256, 65536, 256, 2560, 10],
    "large": [34848, 96, 307200, 256, 884736, 384, 663552, 384, 442368, 256, 37748736, 4096, 16777216, 4096, 4096000, 1000],
}


def listed():
    return [
        # serving one picture: the features of one dense layer, so launches and latency are what it costs
        dict(name="norm_1x4096_bf16", kind="norm", rows=1, cols=4096, residual=True, wide=0, type="bf16"),
        # 256 maps of 13 x 13 in front of a 1 x 1 layer in 8 bits
        dict(name="norm8_43264x384_bf16_e4m3", kind="norm8", rows=43264, cols=384, residual=True, wide=0, type="bf16", code="e4m3"),
        # 128 maps of 27 x 27 in training, without a residual
        dict(name="step_93312x256_fp32", kind="step", rows=93312, cols=256, residual=False, wide=0, type="fp32"),
        # a wide residual stream in training
        dict(name="step_16384x4096_bf16", kind="step", rows=16384, cols=4096, residual=True, wide=0, type="bf16"),
        # serving one picture through the first dense layer: the weights are all that moves
        dict(name="product_1x9216x4096_bf16", kind="product", rows=1, cols=9216, out=4096, square=True, type="bf16", code="e4m3", other="e4m3"),
        # a minibatch of 64 through the second
        dict(name="product_64x4096x4096_bf16", kind="product", rows=64, cols=4096, out=4096, square=True, type="bf16", code="e4m3", other="e4m3"),
        # odd sizes, mixed codes, results in full
        dict(name="product_129x1001x515_fp32", kind="product", rows=129, cols=1001, out=515, square=False, type="fp32", code="e5m2", other="e4m3"),
        # the largest product: a long minibatch of wide rows
        dict(name="product_16384x4096x4096_bf16", kind="product", rows=16384, cols=4096, out=4096, square=True, type="bf16", code="e4m3", other="e4m3"),
        # training the first dense layer with 256 pictures: few rows, a large weight
        dict(name="layer_256x9216x4096_bf16", kind="layer", rows=256, cols=9216, out=4096, type="bf16", code="e4m3", other="e5m2"),
        # training a 1 x 1 layer over the pixels of 256 maps: many rows, a small weight
        dict(name="layer_43264x384x384_bf16", kind="layer", rows=43264, cols=384, out=384, type="bf16", code="e4m3", other="e4m3"),
        # all gradients of a small net, under the limit: nothing has to shrink
        dict(name="clip_small_16_fp32", kind="clip", sizes=",".join(map(str, NETS["small"])), type="fp32", limit=2.0),
        # all gradients of the large net, over the limit
        dict(name="clip_large_16_fp32", kind="clip", sizes=",".join(map(str, NETS["large"])), type="fp32", limit=0.5),
    ]


MAX_VALUES = 16384 * 4096  # of an activation
MAX_OPERAND = 128 << 20  # of an operand or result of a product
MAX_PRODUCTS = 16384 * 4096 * 4096


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "norm8", "step", "product", "product", "layer", "clip"])
    kind_of = rng.choice(["fp32", "bf16", "bf16", "fp16"])
    code, other = rng.choice(["e4m3", "e4m3", "e5m2"]), rng.choice(["e4m3", "e4m3", "e5m2"])
    if kind == "clip":
        count = _log_int(rng, 1, 60)
        while True:
            sizes = [_log_int(rng, 1, 37748736) for _ in range(count)]
            if sum(sizes) <= sum(NETS["large"]):
                return dict(kind=kind, sizes=",".join(map(str, sizes)), type=kind_of, limit=rng.choice([0.1, 0.5, 2.0]))
    if kind in ("norm", "norm8", "step"):
        while True:
            rows, cols = _log_int(rng, 1, 93312), rng.choice([_log_int(rng, 2, 16384), 8 * _log_int(rng, 1, 2048)])
            if rows * cols <= MAX_VALUES:
                break
        case = dict(kind=kind, rows=rows, cols=cols, residual=rng.random() < 0.6, wide=rng.choice([0, 0, 0, 8, 37]), type=kind_of)
        return dict(case, code=code) if kind == "norm8" else case
    while True:
        rows = _log_int(rng, 1, 43264)
        cols, out = (rng.choice([_log_int(rng, 1, 9216), 16 * _log_int(rng, 1, 576)]) for _ in range(2))
        products = rows * cols * out * (3 if kind == "layer" else 1)
        if products <= MAX_PRODUCTS and max(rows * cols, rows * out, cols * out) <= MAX_OPERAND:
            case = dict(kind=kind, rows=rows, cols=cols, out=out, type=kind_of, code=code, other=other)
            return dict(case, square=rng.random() < 0.5) if kind == "product" else case


# ------------------------------------------------------------------ inputs ---
def _features(gen, rows, cols, dtype):
    """Rows of different size, columns of different size."""
    scale = torch.rand(cols, generator=gen, device="cuda") * 1.5 + 0.25
    size = torch.exp2(torch.randn((rows, 1), generator=gen, device="cuda"))
    return (torch.randn((rows, cols), generator=gen, device="cuda") * scale * size).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype, kind = TYPES[case["type"]], case["kind"]
    if kind == "clip":
        sizes = [int(n) for n in case["sizes"].split(",")]
        # layers of different size
        grads = [(torch.randn(n, generator=gen, device="cuda") * 2.0 ** -(4 + k % 5)).to(dtype) for k, n in enumerate(sizes)]
        expected = math.sqrt(sum(n * 4.0 ** -(4 + k % 5) for k, n in enumerate(sizes)))
        return {"case": case, "grads": grads, "max_norm": case["limit"] * expected, "out": [torch.empty_like(g) for g in grads]}
    rows, cols = case["rows"], case["cols"]
    if kind == "product":
        a = _put(_features(gen, rows, cols, torch.float32), case["code"], 1)
        w = torch.randn((case["out"], cols), generator=gen, device="cuda") / math.sqrt(cols)
        b = _put(w, case["other"], BLOCK if case["square"] else 1)
        return {"case": case, "a": a, "b": b}
    if kind == "layer":
        w = torch.randn((case["out"], cols), generator=gen, device="cuda") / math.sqrt(cols)
        dy = (torch.randn((rows, case["out"]), generator=gen, device="cuda") / math.sqrt(rows)).to(dtype)
        return {"case": case, "x": _features(gen, rows, cols, dtype), "w": w, "dy": dy}
    wide = case["wide"]
    state = {"case": case, "x": _features(gen, rows, cols + wide, dtype)[:, wide:], "residual": None, "dsum": None,
             "gamma": 1.0 + 0.2 * torch.randn(cols, generator=gen, device="cuda")}
    if case["residual"]:
        state["residual"] = _features(gen, rows, cols, dtype)
    if kind == "step":
        state["dy"] = (torch.randn((rows, cols), generator=gen, device="cuda") * 0.1).to(dtype)
        if case["residual"]:
            state["dsum"] = (torch.randn((rows, cols), generator=gen, device="cuda") * 0.1).to(dtype)
    return state


# -------------------------------------------------------------- plain forms ---
def _put(x, code, tall):
    """Codes and scales of x [rows][cols]: for `tall` rows by 128 columns the smallest power of two under which the largest
    value has a code.  Codes come as [rows][whole blocks of 128], zeros behind the columns; scales (exponent + 127) as [blocks
    of columns][blocks of rows], those of single rows up to a multiple of four."""
    rows, cols = x.shape
    full = torch.nn.functional.pad(x.float(), (0, -cols % BLOCK, 0, -rows % tall))
    blocks = full.view(full.shape[0] // tall, tall, -1, BLOCK)
    part, power = torch.frexp(blocks.abs().amax((1, 3)))
    fraction, bits, _ = LARGEST[code]
    exponent = (power - bits + (part > fraction).to(power.dtype)).clamp(min=-126)
    codes = (blocks * torch.exp2(-exponent.float())[:, None, :, None]).view(full.shape)[:rows].contiguous().to(CODES[code])
    scales = (exponent.t() + 127).to(torch.uint8)
    return codes, torch.nn.functional.pad(scales, (0, -rows % 4 if tall == 1 else 0)).contiguous()


def _values(codes, scales, tall, cols):
    rows = codes.shape[0]
    scale = torch.exp2(scales.t().float() - 127.0).repeat_interleave(tall, 0)[:rows]
    return (codes.float().view(rows, -1, BLOCK) * scale[:, :, None]).view(rows, -1)[:, :cols]


def _through(x, code, tall):
    return _values(*_put(x, code, tall), tall, x.shape[1])


def _norm(x, residual, gamma):
    s = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    s32 = s.float()
    rstd = torch.rsqrt(s32.square().mean(1) + EPS)
    return s32 * rstd[:, None] * gamma, s, rstd


def _norm_backward(s, dy, rstd, gamma, dsum):
    hat, dy = s.float() * rstd[:, None], dy.float()
    g = dy * gamma
    ds = rstd[:, None] * (g - hat * (g * hat).mean(1, keepdim=True))
    return (ds if dsum is None else ds + dsum.float()).to(s.dtype), (dy * hat).sum(0)


def _run_plain(state):
    case = state["case"]
    kind, dtype = case["kind"], TYPES[case["type"]]
    if kind == "clip":
        norm = torch.sqrt(sum(g.double().square().sum() for g in state["grads"]))
        factor = torch.clamp(state["max_norm"] / norm, max=1.0).float()
        return {"norm": norm.float(), "clipped": [(g.float() * factor).to(dtype) for g in state["grads"]]}
    if kind == "product":
        a, b = (_values(*state[k], t, case["cols"]) for k, t in (("a", 1), ("b", BLOCK if case["square"] else 1)))
        return {"y": (a @ b.t()).to(dtype)}
    if kind == "layer":
        x, w, dy, code, other = state["x"].float(), state["w"], state["dy"].float(), case["code"], case["other"]
        weight = _through(w, code, BLOCK)
        y = _through(x, code, 1) @ weight.t()
        dx = _through(dy, other, 1) @ weight
        dw = _through(dy.t().contiguous(), other, 1) @ _through(x.t().contiguous(), code, 1).t()
        return {"y": y.to(dtype), "dx": dx.to(dtype), "dw": dw}
    y, s, rstd = _norm(state["x"], state["residual"], state["gamma"])
    if kind == "norm8":
        return {"y": _through(y, case["code"], 1).to(torch.bfloat16), "sum": s, "rstd": rstd}
    out = {"y": y.to(dtype), "sum": s, "rstd": rstd}
    if kind == "step":
        out["dx"], out["dgamma"] = _norm_backward(s, state["dy"], rstd, state["gamma"], state["dsum"])
    return out


# --------------------------------------------------------------------- run ---
def _run_own(state):
    from paper_1412_2302_amd import binding as B

    case = state["case"]
    kind, dtype = case["kind"], TYPES[case["type"]]
    if kind == "clip":
        norm = B.clip_gradients(state["grads"], state["max_norm"], out=state["out"])
        return {"norm": norm, "clipped": state["out"]}
    if kind == "product":
        a = B.Blocks8(*state["a"], case["cols"])
        b = B.Blocks8(*state["b"], case["cols"], square=case["square"])
        return {"y": B.block8_product(a, b, dtype)}
    if kind == "layer":
        code, other = CODES[case["code"]], CODES[case["other"]]
        x, x_t = B.block8_pack(state["x"], code, along="both")
        w, w_t = B.block8_pack(state["w"], code, square=True, along="both")
        dy, dy_t = B.block8_pack(state["dy"], other, along="both")
        return {"y": B.block8_product(x, w, dtype), "dx": B.block8_product(dy, w_t, dtype),
                "dw": B.block8_product(dy_t, x_t, torch.float32)}
    code = CODES[case["code"]] if kind == "norm8" else None
    y, s, rstd = B.rms_norm_forward(state["x"], state["gamma"], residual=state["residual"], eps=EPS, blocks=code)
    if kind == "norm8":
        return {"y": B.block8_unpack(y, torch.bfloat16), "sum": s, "rstd": rstd}
    out = {"y": y, "sum": s, "rstd": rstd}
    if kind == "step":
        out["dx"], out["dgamma"] = B.rms_norm_backward(s, state["dy"], rstd, state["gamma"], dsum=state["dsum"])
    return out


def run(state):
    return _run_own(state) if own else _run_plain(state)


# -------------------------------------------------------------------- work ---
def work(case):
    """Inputs and outputs once; one multiply-add per term of a product, about ten operations per normalised value.  The codes
    of a layer's operands count neither written nor read: that is the way taken, not the work."""
    size, kind = {"fp32": 4, "bf16": 2, "fp16": 2}[case["type"]], case["kind"]
    if kind == "clip":
        n = sum(int(n) for n in case["sizes"].split(","))
        return {"bytes": 2.0 * n * size, "flops": 3.0 * n}
    rows, cols = case["rows"], case["cols"]
    if kind == "product":
        codes = (rows + case["out"]) * cols * (1.0 + 1.0 / BLOCK)
        return {"bytes": codes + rows * case["out"] * size, "flops": 2.0 * rows * cols * case["out"]}
    if kind == "layer":
        out = case["out"]
        return {"bytes": 2.0 * size * rows * (cols + out) + 8.0 * cols * out, "flops": 6.0 * rows * cols * out}
    values, streams = rows * cols, 2 if case["residual"] else 0  # the residual, and the sum where it is not x
    small = 4.0 * (rows + cols)
    if kind == "norm8":  # codes written, read back, values written
        return {"bytes": values * (size * (1 + streams) + 4.0) + small, "flops": 10.0 * values}
    forward = values * size * (2.0 + streams) + small
    if kind == "norm":
        return {"bytes": forward, "flops": 7.0 * values}
    return {"bytes": forward + values * size * (3.0 + (1 if case["residual"] else 0)) + 2 * small, "flops": 18.0 * values}


# ------------------------------------------------------------------- exact ---
def _round64(v, code):
    """To four significant bits down to 2^-6 (e4m3), to three down to 2^-14 (e5m2), fixed steps below."""
    low, bits = (-6.0, 3.0) if code == "e4m3" else (-14.0, 2.0)
    step = torch.exp2(torch.clamp(torch.floor(torch.log2(v.abs().clamp(min=1e-300))), min=low) - bits)
    return torch.round(v / step) * step


def _kept64(x, code, tall):
    rows, cols = x.shape
    down, across = math.ceil(rows / tall), math.ceil(cols / BLOCK)
    most = torch.zeros((down, across), dtype=torch.float64, device=x.device)
    row, col = torch.arange(rows, device=x.device) // tall, torch.arange(cols, device=x.device) // BLOCK
    wide = torch.zeros((rows, across), dtype=torch.float64, device=x.device)
    wide.scatter_reduce_(1, col.expand(rows, cols), x.abs(), "amax")
    most.scatter_reduce_(0, row[:, None].expand(rows, across), wide, "amax")
    scale = torch.exp2(torch.clamp(torch.ceil(torch.log2(most / LARGEST[code][2])), min=-126.0))
    each = scale[row][:, col]
    return _round64(x / each, code) * each


def _meant64(codes, scales, tall, cols):
    rows = codes.shape[0]
    row, col = torch.arange(rows, device=codes.device) // tall, torch.arange(cols, device=codes.device) // BLOCK
    return codes[:, :cols].double() * torch.exp2(scales.double() - 127.0)[col][:, row].t()


def exact(case, seed):
    state, kind = prepare(case, seed), case["kind"]
    if kind == "clip":
        grads = [g.double() for g in state["grads"]]
        norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(g) for g in grads]))
        factor = torch.where(norm > state["max_norm"], state["max_norm"] / norm, torch.ones_like(norm))
        return {"norm": norm, "clipped": [g * factor for g in grads]}
    if kind == "product":
        a = _meant64(*state["a"], 1, case["cols"])
        b = _meant64(*state["b"], BLOCK if case["square"] else 1, case["cols"])
        return {"y": torch.matmul(a, b.t().contiguous())}
    if kind == "layer":
        x, w, dy, code, other = state["x"].double(), state["w"].double(), state["dy"].double(), case["code"], case["other"]
        w8 = _kept64(w, code, BLOCK)
        y = torch.matmul(_kept64(x, code, 1), w8.t().contiguous())
        dx = torch.matmul(_kept64(dy, other, 1), w8)
        dw = torch.matmul(_kept64(dy.t().contiguous(), other, 1), _kept64(x.t().contiguous(), code, 1).t().contiguous())
        return {"y": y, "dx": dx, "dw": dw}
    gamma, cols = state["gamma"].double(), case["cols"]
    s = state["x"].double()
    if state["residual"] is not None:
        s = (s + state["residual"].double()).to(state["x"].dtype).double()  # what follows is of the sum that is handed on
    rstd = ((s * s).sum(1) / cols + EPS) ** -0.5
    hat = s * rstd.unsqueeze(1)
    y = hat * gamma
    out = {"y": _kept64(y, case["code"], 1) if kind == "norm8" else y, "sum": s, "rstd": rstd}
    if kind == "step":
        dy = state["dy"].double()
        mean = (dy * gamma * hat).sum(1) / cols
        dx = rstd.unsqueeze(1) * (dy * gamma - hat * mean.unsqueeze(1))
        out["dx"] = dx if state["dsum"] is None else dx + state["dsum"].double()
        out["dgamma"] = (dy * hat).sum(0)
    return out
