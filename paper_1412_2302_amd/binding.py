"""Thin ctypes binding of libalexnet_hip.so (include/alexnet.h).

Argument marshalling only: every step of the training path runs inside the
HIP library.  PyTorch is used to own device memory and streams.  Importing
this module fails loudly when the library has not been built
(python -m paper_1412_2302_amd.build); there is no CPU fallback.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
from typing import Dict, Optional, Tuple

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libalexnet_hip.so")
if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_1412_2302_amd.build`")
_lib = C.CDLL(LIB_PATH)

OK, EINVAL, ESHAPE, EALIGN, ELABEL, EHIP, ENOTIMPL, ENOMEM = 0, -1, -2, -3, -4, -5, -6, -7

T_INPUT, T_CONV_ACT, T_LRN, T_POOL, T_ARGMAX, T_FC_ACT, T_CROP_X, T_CROP_Y, T_FLIP, T_DLOGITS, T_CONV_DACT = range(11)
_INT_KINDS = {T_ARGMAX, T_CROP_X, T_CROP_Y, T_FLIP}


class ConvCfg(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("cout", "k", "stride", "pad", "groups", "lrn", "pool")]


class Config(C.Structure):
    _fields_ = [
        ("batch", C.c_int32), ("in_c", C.c_int32), ("crop_h", C.c_int32), ("crop_w", C.c_int32),
        ("raw_h", C.c_int32), ("raw_w", C.c_int32),
        ("conv", ConvCfg * 5), ("fc", C.c_int32 * 3),
        ("lrn_n", C.c_int32), ("lrn_k", C.c_float), ("lrn_alpha", C.c_float), ("lrn_beta", C.c_float),
        ("dropout_p", C.c_float), ("lr", C.c_float), ("momentum", C.c_float), ("weight_decay", C.c_float),
        ("precision", C.c_int32), ("flags", C.c_int32), ("seed", C.c_uint64),
    ]


_vp, _i32, _u64, _sz = C.c_void_p, C.c_int32, C.c_uint64, C.c_size_t
_SIGS = {
    "alexnet_query": [C.POINTER(Config), C.POINTER(_sz), C.POINTER(_sz)],
    "alexnet_create": [C.POINTER(Config), _vp, _vp, _vp, _sz, _vp, C.POINTER(_vp)],
    "alexnet_preprocess": [_vp, _vp, _vp, _u64, _i32, _vp],
    "alexnet_set_input": [_vp, _vp, _i32, _vp],
    "alexnet_train_step": [_vp, _i32, _vp, _u64, _vp, _vp],
    "alexnet_forward_backward": [_vp, _i32, _vp, _u64, _vp, _vp],
    "alexnet_apply_update": [_vp, _vp],
    "alexnet_forward": [_vp, _vp, _vp, _vp],
    "alexnet_average_replicas": [_vp, _vp, _vp],
    "alexnet_average_gradients_update": [_vp, _vp, _vp],
    "alexnet_preprocess_center": [_vp, _vp, _vp, _i32, _vp],
    "alexnet_loader_create": [_vp, _vp, _vp, _vp, C.c_int64, _i32, _vp, _vp, _vp, _vp, _vp, C.POINTER(_vp)],
    "alexnet_loader_stage": [_vp, _u64, _vp, _vp, _vp, C.POINTER(_vp)],
    "alexnet_loader_done": [_vp, _u64, _vp],
    "alexnet_loader_destroy": [_vp],
    "alexnet_validate": [_vp, _i32, _vp, C.POINTER(_i32), _i32, _vp, _vp],
    "alexnet_set_params": [_vp, _vp, _vp],
    "alexnet_get_params": [_vp, _vp, _vp],
    "alexnet_set_momentum": [_vp, _vp, _vp],
    "alexnet_get_momentum": [_vp, _vp, _vp],
    "alexnet_get_grads": [_vp, _vp, _vp],
    "alexnet_tensor_elems": [_vp, _i32, _i32, C.POINTER(_sz)],
    "alexnet_get_tensor": [_vp, _i32, _i32, _vp, _vp],
    "alexnet_check": [_vp, _vp],
    "alexnet_conv_forward": [_vp, _i32, _vp, _vp, _vp, _i32, _vp, _vp],
    "alexnet_conv_backward_data": [_vp, _i32, _vp, _vp, _vp, _vp],
    "alexnet_conv_backward_weight": [_vp, _i32, _vp, _vp, _vp, _vp, _vp],
    "alexnet_nchw_to_nhwc": [_vp, _vp, _i32, _i32, _i32, _i32, _vp],
    "alexnet_nhwc_to_nchw": [_vp, _vp, _i32, _i32, _i32, _i32, _vp],
    "alexnet_pack_conv_weight": [_vp, _i32, _vp, _vp, _vp, _vp],
    "alexnet_unpack_conv_weight": [_vp, _i32, _vp, _vp, _vp],
    "alexnet_conv_forward_nhwc": [_vp, _i32, _vp, _vp, _vp, _i32, _vp, _vp],
    "alexnet_conv_backward_data_nhwc": [_vp, _i32, _vp, _vp, _vp, _vp, _vp],
    "alexnet_conv_backward_weight_nhwc": [_vp, _i32, _vp, _vp, _vp, _vp, _vp],
}


class ProfEntry(C.Structure):
    _fields_ = [("name", C.c_char * 48), ("calls", C.c_int32), ("total_ms", C.c_float),
                ("flops", C.c_double), ("bytes", C.c_double)]


_SIGS.update({
    "alexnet_lrn_forward": [_vp, _i32, _vp, _vp, _vp],
    "alexnet_lrn_backward": [_vp, _i32, _vp, _vp, _i32, _vp, _vp],
    "alexnet_pool_forward": [_vp, _i32, _vp, _vp, _vp, _vp],
    "alexnet_pool_backward": [_vp, _i32, _vp, _vp, _i32, _vp, _vp],
    "alexnet_lrn_pool_forward": [_vp, _i32, _vp, _vp, _vp, _vp],
    "alexnet_pool_lrn_backward": [_vp, _i32, _vp, _vp, _i32, _vp, _vp, _vp],
    "alexnet_fc_forward": [_vp, _i32, _vp, _vp, _vp, _i32, _vp, _vp],
    "alexnet_fc_backward": [_vp, _i32, _vp, _vp, _vp, _vp, _vp, _vp, _vp],
    "alexnet_softmax_xent": [_vp, _vp, _vp, _vp, _vp, _vp],
    "alexnet_softmax_xent_static": [_vp, _vp, _i32, _i32, _vp, _vp, _vp, _vp],
})


class CheckpointArg(C.Structure):
    _fields_ = [("d_codes", C.c_void_p), ("d_scales", C.c_void_p), ("code", C.c_int32)]


class GroupNormCfg(C.Structure):
    _fields_ = [("n", C.c_int32), ("hw", C.c_int32), ("c", C.c_int32), ("groups", C.c_int32),
                ("type", C.c_int32), ("act", C.c_int32), ("eps", C.c_float)]


_i64, _kp, _gp = C.c_int64, C.POINTER(CheckpointArg), C.POINTER(GroupNormCfg)
_SIGS.update({
    "alexnet_group_norm_query": [_gp, _i32, C.POINTER(_sz), C.POINTER(_sz)],
    "alexnet_group_norm_forward": [_gp, _vp, _i64, _vp, _vp, _vp, _i64, _vp, _vp, _kp, _vp, _sz, _vp],
    "alexnet_group_norm_backward": [_gp, _vp, _i64, _kp, _vp, _i64, _vp, _vp, _vp, _vp, _vp, _i64, _vp, _vp, _vp, _sz,
                                    _vp],
    "alexnet_checkpoint_pack": [_vp, _i64, _i32, _i64, _i32, _kp, _vp],
    "alexnet_checkpoint_unpack": [_kp, _i64, _i32, _vp, _i64, _i32, _vp],
    "alexnet_checkpoint_fc_query": [_i64, _i32, _i32, _i32, C.POINTER(_sz)],
    "alexnet_checkpoint_fc_backward_weight": [_kp, _vp, _i64, _i32, _i64, _i32, _i32, _vp, _vp, _vp, _sz, _vp],
})
_SIGS["alexnet_profile_begin"] = []
_SIGS["alexnet_profile_end"] = [C.POINTER(ProfEntry), _i32, C.POINTER(_i32)]
for _name, _args in _SIGS.items():
    _f = getattr(_lib, _name)
    _f.argtypes = _args
    _f.restype = C.c_int
_lib.alexnet_destroy.argtypes = [_vp]
_lib.alexnet_destroy.restype = None
_lib.alexnet_last_error.restype = C.c_char_p
_lib.alexnet_version.restype = C.c_char_p
EXPORTS = sorted(list(_SIGS) + ["alexnet_destroy", "alexnet_last_error", "alexnet_version"])


class AlexNetError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"libalexnet_hip error {code}: {msg}")
        self.code = code


def last_error() -> str:
    return (_lib.alexnet_last_error() or b"").decode()


def version() -> str:
    return _lib.alexnet_version().decode()


def profile_begin():
    _check(_lib.alexnet_profile_begin())


def profile_end(cap: int = 256):
    """Returns [{name, calls, total_ms, flops, bytes}] for the kernels launched since profile_begin."""
    buf = (ProfEntry * cap)()
    n = _i32()
    _check(_lib.alexnet_profile_end(buf, cap, C.byref(n)))
    return [dict(name=buf[i].name.decode(), calls=buf[i].calls, total_ms=buf[i].total_ms, flops=buf[i].flops,
                 bytes=buf[i].bytes) for i in range(min(n.value, cap))]


def _check(rc: int):
    if rc != OK:
        raise AlexNetError(rc, last_error())


FLAG_DIRECT_CONV = 1


def make_config(workload: dict, batch: int, seed: int = 0, precision: int = 0, flags: int = 0) -> Config:
    cfg = Config()
    cfg.batch = batch
    cfg.in_c = workload["in_c"]
    cfg.crop_h = cfg.crop_w = workload["crop"]
    cfg.raw_h = cfg.raw_w = workload["raw"]
    for i, (co, k, st, pd, g, l, p) in enumerate(workload["conv"]):
        cfg.conv[i] = ConvCfg(co, k, st, pd, g, l, p)
    for j, f in enumerate(workload["fc"]):
        cfg.fc[j] = f
    n, k, a, b = workload["lrn"]
    cfg.lrn_n, cfg.lrn_k, cfg.lrn_alpha, cfg.lrn_beta = n, k, a, b
    cfg.dropout_p, cfg.lr = workload["dropout_p"], workload["lr"]
    cfg.momentum, cfg.weight_decay = workload["momentum"], workload["weight_decay"]
    cfg.precision, cfg.flags, cfg.seed = precision, flags, seed
    return cfg


def query(cfg: Config) -> Tuple[int, int]:
    n, w = _sz(), _sz()
    _check(_lib.alexnet_query(C.byref(cfg), C.byref(n), C.byref(w)))
    return n.value, w.value


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else _vp(t.data_ptr())


def _need(t, dtype, numel: int, what: str) -> torch.Tensor:
    """The library takes bare device pointers: a tensor of the wrong kind, place or size would be read past its
    end on the GPU, so it is refused here."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{what}: expected a torch.Tensor, got {type(t).__name__}")
    if not t.is_cuda:
        raise ValueError(f"{what}: expected a device tensor, got one on {t.device}")
    if t.dtype != dtype:
        raise ValueError(f"{what}: expected {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{what}: expected a contiguous tensor")
    if t.numel() < numel:
        raise ValueError(f"{what}: expected at least {numel} elements, got {t.numel()}")
    return t


def _stream(stream: Optional[torch.cuda.Stream]):
    s = stream if stream is not None else torch.cuda.current_stream()
    return _vp(s.cuda_stream)


def _dev(a, dtype=None) -> torch.Tensor:
    if isinstance(a, torch.Tensor):
        t = a.to("cuda")
    else:
        t = torch.from_numpy(np.ascontiguousarray(a)).to("cuda")
    if dtype is not None:
        t = t.to(dtype)
    return t.contiguous()


class AlexNet:
    """One replica: owns parameter, momentum and workspace tensors on cuda:0."""

    def __init__(self, workload: dict, batch: int, seed: int = 0, precision: int = 0, flags: int = 0):
        if not torch.cuda.is_available():
            raise RuntimeError("libalexnet_hip needs a GPU; there is no CPU path")
        self.workload, self.batch = workload, batch
        self.cfg = make_config(workload, batch, seed, precision, flags)
        self.n_params, self.ws_bytes = query(self.cfg)
        dev = torch.device("cuda", 0)
        self.params = torch.zeros(self.n_params, dtype=torch.float32, device=dev)
        self.momentum = torch.zeros(self.n_params, dtype=torch.float32, device=dev)
        self.workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=dev)
        self.loss = torch.zeros(1, dtype=torch.float32, device=dev)
        h = _vp()
        _check(_lib.alexnet_create(C.byref(self.cfg), _ptr(self.params), _ptr(self.momentum), _ptr(self.workspace),
                                   self.ws_bytes, _stream(None), C.byref(h)))
        self._h = h
        self.shapes = self._param_shapes()

    def close(self):
        if getattr(self, "_h", None) and _lib is not None:  # _lib is gone at interpreter shutdown
            _lib.alexnet_destroy(self._h)
            self._h = None

    def __del__(self):
        self.close()

    # ---- bookkeeping of the canonical flat vector (marshalling only) ----
    def _param_shapes(self) -> Dict[str, Tuple[int, ...]]:
        wl = self.workload
        c, h = wl["in_c"], wl["crop"]
        ws, bs = {}, {}
        for i, (co, k, st, pd, g, l, p) in enumerate(wl["conv"]):
            ws[f"conv{i+1}.w"] = (co, c // g, k, k)
            bs[f"conv{i+1}.b"] = (co,)
            h = (h + 2 * pd - k) // st + 1
            if p:
                h = (h - 3) // 2 + 1
            c = co
        fin = c * h * h
        for j, fo in enumerate(wl["fc"]):
            ws[f"fc{6+j}.w"] = (fo, fin)
            bs[f"fc{6+j}.b"] = (fo,)
            fin = fo
        ws.update(bs)
        total = sum(int(np.prod(s)) for s in ws.values())
        assert total == self.n_params, (total, self.n_params)
        return ws

    def flatten(self, d: Dict[str, np.ndarray]) -> np.ndarray:
        return np.concatenate([np.asarray(d[k], np.float32).ravel() for k in self.shapes])

    def unflatten(self, flat: np.ndarray) -> Dict[str, np.ndarray]:
        out, o = {}, 0
        for k, s in self.shapes.items():
            n = int(np.prod(s))
            out[k] = flat[o:o + n].reshape(s)
            o += n
        return out

    # ---- parameters ----
    def _set(self, fn, d):
        flat = _dev(self.flatten(d) if isinstance(d, dict) else d, torch.float32)
        assert flat.numel() == self.n_params
        _check(fn(self._h, _ptr(flat), _stream(None)))
        torch.cuda.current_stream().synchronize()

    def _get(self, fn) -> Dict[str, np.ndarray]:
        flat = torch.empty(self.n_params, dtype=torch.float32, device="cuda")
        _check(fn(self._h, _ptr(flat), _stream(None)))
        return self.unflatten(flat.cpu().numpy())

    def set_params(self, d): self._set(_lib.alexnet_set_params, d)
    def set_momentum(self, d): self._set(_lib.alexnet_set_momentum, d)
    def get_params(self): return self._get(_lib.alexnet_get_params)
    def get_momentum(self): return self._get(_lib.alexnet_get_momentum)
    def get_grads(self): return self._get(_lib.alexnet_get_grads)

    # ---- the hot path ----
    def _raw_elems(self) -> int:
        return self.workload["in_c"] * self.workload["raw"] * self.workload["raw"]

    def _input_elems(self) -> int:
        return self.batch * self.workload["in_c"] * self.workload["crop"] * self.workload["crop"]

    def preprocess(self, raw_u8: torch.Tensor, mean: torch.Tensor, step: int, slot: int, stream=None):
        _need(raw_u8, torch.uint8, self.batch * self._raw_elems(), "preprocess: stored pictures")
        _need(mean, torch.float32, self._raw_elems(), "preprocess: mean image")
        _check(_lib.alexnet_preprocess(self._h, _ptr(raw_u8), _ptr(mean), step, slot, _stream(stream)))

    def preprocess_center(self, raw_u8: torch.Tensor, mean: torch.Tensor, slot: int, stream=None):
        _need(raw_u8, torch.uint8, self.batch * self._raw_elems(), "preprocess_center: stored pictures")
        _need(mean, torch.float32, self._raw_elems(), "preprocess_center: mean image")
        _check(_lib.alexnet_preprocess_center(self._h, _ptr(raw_u8), _ptr(mean), slot, _stream(stream)))

    def validate(self, labels: torch.Tensor, ks, counts: torch.Tensor, slot: int = 0, stream=None):
        """counts (int32, device, one per k) += pictures of input slot `slot` whose label is in the top k."""
        _need(labels, torch.int32, self.batch, "validate: labels")
        _need(counts, torch.int32, len(ks), "validate: counts")
        arr = (_i32 * len(ks))(*ks)
        _check(_lib.alexnet_validate(self._h, slot, _ptr(labels), arr, len(ks), _ptr(counts), _stream(stream)))

    def set_input(self, x_nchw: torch.Tensor, slot: int = 0, stream=None):
        _need(x_nchw, torch.float32, self._input_elems(), "set_input: input")
        _check(_lib.alexnet_set_input(self._h, _ptr(x_nchw), slot, _stream(stream)))

    def train_step(self, labels: torch.Tensor, step: int, slot: int = 0, stream=None) -> torch.Tensor:
        _need(labels, torch.int32, self.batch, "train_step: labels")
        _check(_lib.alexnet_train_step(self._h, slot, _ptr(labels), step, _ptr(self.loss), _stream(stream)))
        return self.loss

    def forward_backward(self, labels: torch.Tensor, step: int, slot: int = 0, stream=None) -> torch.Tensor:
        _need(labels, torch.int32, self.batch, "forward_backward: labels")
        _check(_lib.alexnet_forward_backward(self._h, slot, _ptr(labels), step, _ptr(self.loss), _stream(stream)))
        return self.loss

    def apply_update(self, stream=None):
        _check(_lib.alexnet_apply_update(self._h, _stream(stream)))

    def forward(self, x_nchw: torch.Tensor, stream=None) -> torch.Tensor:
        _need(x_nchw, torch.float32, self._input_elems(), "forward: input")
        probs = torch.empty(self.batch, self.workload["fc"][-1], dtype=torch.float32, device="cuda")
        _check(_lib.alexnet_forward(self._h, _ptr(x_nchw), _ptr(probs), _stream(stream)))
        return probs

    def check(self, stream=None):
        _check(_lib.alexnet_check(self._h, _stream(stream)))

    def tensor(self, kind: int, layer: int) -> np.ndarray:
        n = _sz()
        _check(_lib.alexnet_tensor_elems(self._h, kind, layer, C.byref(n)))
        out = torch.empty(n.value, dtype=torch.int32 if kind in _INT_KINDS else torch.float32, device="cuda")
        _check(_lib.alexnet_get_tensor(self._h, kind, layer, _ptr(out), _stream(None)))
        return out.cpu().numpy()

    # ---- single operators on canonical tensors ----
    def conv_forward(self, layer, x, w, b, relu=False):
        xs, wt = _dev(x, torch.float32), _dev(w, torch.float32)
        bt = None if b is None else _dev(b, torch.float32)
        n = _sz()
        _check(_lib.alexnet_tensor_elems(self._h, T_CONV_ACT, layer, C.byref(n)))
        y = torch.empty(n.value, dtype=torch.float32, device="cuda")
        _check(_lib.alexnet_conv_forward(self._h, layer, _ptr(xs), _ptr(wt), _ptr(bt), int(relu), _ptr(y), _stream(None)))
        return y

    def conv_backward_data(self, layer, dy, w, x_shape):
        dyt, wt = _dev(dy, torch.float32), _dev(w, torch.float32)
        dx = torch.empty(int(np.prod(x_shape)), dtype=torch.float32, device="cuda")
        _check(_lib.alexnet_conv_backward_data(self._h, layer, _ptr(dyt), _ptr(wt), _ptr(dx), _stream(None)))
        return dx.view(*x_shape)

    def conv_backward_weight(self, layer, x, dy, w_shape):
        xs, dyt = _dev(x, torch.float32), _dev(dy, torch.float32)
        dw = torch.empty(int(np.prod(w_shape)), dtype=torch.float32, device="cuda")
        db = torch.empty(w_shape[0], dtype=torch.float32, device="cuda")
        _check(_lib.alexnet_conv_backward_weight(self._h, layer, _ptr(xs), _ptr(dyt), _ptr(dw), _ptr(db), _stream(None)))
        return dw.view(*w_shape), db

    # channel-last variants: no conversion kernels in the call
    def pack_conv_weight(self, layer, w_oihw: torch.Tensor):
        wf, wb = torch.empty_like(w_oihw).view(-1), torch.empty_like(w_oihw).view(-1)
        _check(_lib.alexnet_pack_conv_weight(self._h, layer, _ptr(w_oihw), _ptr(wf), _ptr(wb), _stream(None)))
        return wf, wb

    def unpack_conv_weight(self, layer, wf: torch.Tensor, w_shape):
        w = torch.empty(int(np.prod(w_shape)), dtype=torch.float32, device="cuda")
        _check(_lib.alexnet_unpack_conv_weight(self._h, layer, _ptr(wf), _ptr(w), _stream(None)))
        return w.view(*w_shape)

    def _conv_elems(self, layer: int) -> Tuple[int, int, int, int]:
        """Elements of a convolution stage's input, output, weights and bias (the geometry rule of the library:
        out = (in + 2 pad - k) / stride + 1, 3x3 stride-2 pooling behind the stages that pool)."""
        if not 1 <= layer <= len(self.workload["conv"]):
            raise ValueError(f"layer must be 1..{len(self.workload['conv'])}")
        c, h = self.workload["in_c"], self.workload["crop"]
        for i, (cout, k, stride, pad, groups, _lrn, pool) in enumerate(self.workload["conv"], start=1):
            ho = (h + 2 * pad - k) // stride + 1
            if i == layer:
                return self.batch * h * h * c, self.batch * ho * ho * cout, cout * (c // groups) * k * k, cout
            c, h = cout, ((ho - 3) // 2 + 1 if pool else ho)
        raise AssertionError

    def conv_forward_nhwc(self, layer, x, wf, b, relu, y, stream=None):
        nx, ny, nw, nb = self._conv_elems(layer)
        _need(x, torch.float32, nx, "conv_forward_nhwc: x")
        _need(wf, torch.float32, nw, "conv_forward_nhwc: wf")
        _need(y, torch.float32, ny, "conv_forward_nhwc: y")
        if b is not None:
            _need(b, torch.float32, nb, "conv_forward_nhwc: bias")
        _check(_lib.alexnet_conv_forward_nhwc(self._h, layer, _ptr(x), _ptr(wf), _ptr(b), int(relu), _ptr(y), _stream(stream)))

    def conv_backward_data_nhwc(self, layer, dy, wb, dx, wf=None, stream=None):
        nx, ny, nw, _ = self._conv_elems(layer)
        _need(dy, torch.float32, ny, "conv_backward_data_nhwc: dy")
        _need(wb, torch.float32, nw, "conv_backward_data_nhwc: wb")
        _need(dx, torch.float32, nx, "conv_backward_data_nhwc: dx")
        if wf is not None:
            _need(wf, torch.float32, nw, "conv_backward_data_nhwc: wf")
        _check(_lib.alexnet_conv_backward_data_nhwc(self._h, layer, _ptr(dy), _ptr(wf), _ptr(wb), _ptr(dx), _stream(stream)))

    def conv_backward_weight_nhwc(self, layer, x, dy, dwf, db, stream=None):
        nx, ny, nw, nb = self._conv_elems(layer)
        _need(x, torch.float32, nx, "conv_backward_weight_nhwc: x")
        _need(dy, torch.float32, ny, "conv_backward_weight_nhwc: dy")
        _need(dwf, torch.float32, nw, "conv_backward_weight_nhwc: dwf")
        if db is not None:
            _need(db, torch.float32, nb, "conv_backward_weight_nhwc: db")
        _check(_lib.alexnet_conv_backward_weight_nhwc(self._h, layer, _ptr(x), _ptr(dy), _ptr(dwf), _ptr(db), _stream(stream)))


    # ---- bandwidth-bound operators and dense layers alone (canonical tensors) ----
    def lrn_forward(self, layer, a):
        at = _dev(a, torch.float32)
        b = torch.empty_like(at)
        _check(_lib.alexnet_lrn_forward(self._h, layer, _ptr(at), _ptr(b), _stream(None)))
        return b

    def lrn_backward(self, layer, a, db, relu_gate=False):
        at, dbt = _dev(a, torch.float32), _dev(db, torch.float32)
        da = torch.empty_like(at)
        _check(_lib.alexnet_lrn_backward(self._h, layer, _ptr(at), _ptr(dbt), int(relu_gate), _ptr(da), _stream(None)))
        return da

    def pool_forward(self, layer, x):
        xt = _dev(x, torch.float32)
        n, c, h, w = xt.shape
        ho, wo = (h - 3) // 2 + 1, (w - 3) // 2 + 1
        y = torch.empty(n, c, ho, wo, dtype=torch.float32, device="cuda")
        arg = torch.empty(n, c, ho, wo, dtype=torch.int32, device="cuda")
        _check(_lib.alexnet_pool_forward(self._h, layer, _ptr(xt), _ptr(y), _ptr(arg), _stream(None)))
        return y, arg

    def pool_backward(self, layer, x, dy, relu_gate=False):
        xt, dyt = _dev(x, torch.float32), _dev(dy, torch.float32)
        dx = torch.empty_like(xt)
        _check(_lib.alexnet_pool_backward(self._h, layer, _ptr(xt), _ptr(dyt), int(relu_gate), _ptr(dx), _stream(None)))
        return dx

    def lrn_pool_forward(self, layer, a):
        """The fused normalisation + pool kernel of a training step, alone: pooled values and winning taps."""
        at = _dev(a, torch.float32)
        n, c, h, w = at.shape
        ho, wo = (h - 3) // 2 + 1, (w - 3) // 2 + 1
        y = torch.empty(n, c, ho, wo, dtype=torch.float32, device="cuda")
        arg = torch.empty(n, c, ho, wo, dtype=torch.int32, device="cuda")
        _check(_lib.alexnet_lrn_pool_forward(self._h, layer, _ptr(at), _ptr(y), _ptr(arg), _stream(None)))
        return y, arg

    def pool_lrn_backward(self, layer, a, dy, relu_gate=True):
        """The fused pool adjoint + normalisation adjoint + gate + bias sums kernel, alone: (da, db)."""
        at, dyt = _dev(a, torch.float32), _dev(dy, torch.float32)
        da = torch.empty_like(at)
        db = torch.empty(at.shape[1], dtype=torch.float32, device="cuda")
        _check(_lib.alexnet_pool_lrn_backward(self._h, layer, _ptr(at), _ptr(dyt), int(relu_gate), _ptr(da), _ptr(db),
                                              _stream(None)))
        return da, db

    def fc_forward(self, layer, x, w, b, relu=False):
        xt, wt, bt = _dev(x, torch.float32), _dev(w, torch.float32), _dev(b, torch.float32)
        y = torch.empty(xt.shape[0], wt.shape[0], dtype=torch.float32, device="cuda")
        _check(_lib.alexnet_fc_forward(self._h, layer, _ptr(xt), _ptr(wt), _ptr(bt), int(relu), _ptr(y), _stream(None)))
        return y

    def fc_backward(self, layer, x, w, dy):
        xt, wt, dyt = _dev(x, torch.float32), _dev(w, torch.float32), _dev(dy, torch.float32)
        dx, dw = torch.empty_like(xt), torch.empty_like(wt)
        db = torch.empty(wt.shape[0], dtype=torch.float32, device="cuda")
        _check(_lib.alexnet_fc_backward(self._h, layer, _ptr(xt), _ptr(wt), _ptr(dyt), _ptr(dx), _ptr(dw), _ptr(db),
                                        _stream(None)))
        return dx, dw, db

    def softmax_xent(self, logits, labels):
        zt, lt = _dev(logits, torch.float32), _dev(labels, torch.int32)
        dz = torch.empty_like(zt)
        loss = torch.empty(1, dtype=torch.float32, device="cuda")
        _check(_lib.alexnet_softmax_xent(self._h, _ptr(zt), _ptr(lt), _ptr(dz), _ptr(loss), _stream(None)))
        return dz, loss


def average_replicas(a: AlexNet, b: AlexNet, stream=None):
    _check(_lib.alexnet_average_replicas(a._h, b._h, _stream(stream)))


class Loader:
    """Section 2.1's loading thread: `images` (uint8 [count][C][RH][RW]) and `labels` (int32 [count]) are CPU
    tensors standing for the disk; staging memory (pinned host + device) is allocated here with torch."""

    def __init__(self, net: AlexNet, images: torch.Tensor, labels: torch.Tensor, depth: int = 2, copy_stream=None):
        """copy_stream: the stream of the host-to-device copies (best the side stream later given to stage());
        None lets the library create one."""
        want = (net.workload["in_c"], net.workload["raw"], net.workload["raw"])
        if images.dtype != torch.uint8 or images.is_cuda or images.dim() != 4 or tuple(images.shape[1:]) != want:
            raise ValueError(f"Loader: images must be a CPU uint8 tensor [count]{list(want)}, got "
                             f"{images.dtype} {list(images.shape)} on {images.device}")
        if labels.dtype != torch.int32 or labels.is_cuda or labels.numel() != images.shape[0]:
            raise ValueError("Loader: labels must be a CPU int32 tensor with one entry per picture")
        if depth < 1 or images.shape[0] < 1:
            raise ValueError("Loader: need at least one staging set and one picture")
        self.net, self.images, self.labels = net, images.contiguous(), labels.contiguous()
        per = net.batch * int(np.prod(images.shape[1:]))
        self.pinned_raw = torch.empty(depth * per, dtype=torch.uint8, pin_memory=True)
        self.pinned_labels = torch.empty(depth * net.batch, dtype=torch.int32, pin_memory=True)
        self.d_raw = torch.empty(depth * per, dtype=torch.uint8, device="cuda")
        self.d_labels = torch.empty(depth * net.batch, dtype=torch.int32, device="cuda")
        h = _vp()
        _check(_lib.alexnet_loader_create(net._h, C.byref(net.cfg), self.images.data_ptr(), self.labels.data_ptr(),
                                          self.images.shape[0], depth, self.pinned_raw.data_ptr(),
                                          self.pinned_labels.data_ptr(), self.d_raw.data_ptr(),
                                          self.d_labels.data_ptr(),
                                          None if copy_stream is None else _stream(copy_stream), C.byref(h)))
        self._h = h
        self._copy_stream = copy_stream  # keep the torch stream alive as long as the loader

    def stage(self, k: int, mean: torch.Tensor, side_stream, compute_stream) -> torch.Tensor:
        """Returns the labels of minibatch k (a view of the loader's device buffer)."""
        _need(mean, torch.float32, self.net._raw_elems(), "Loader.stage: mean image")
        p = _vp()
        _check(_lib.alexnet_loader_stage(self._h, k, _ptr(mean), _stream(side_stream), _stream(compute_stream),
                                         C.byref(p)))
        off = (p.value - self.d_labels.data_ptr()) // 4
        return self.d_labels[off:off + self.net.batch]

    def done(self, k: int, compute_stream):
        _check(_lib.alexnet_loader_done(self._h, k, _stream(compute_stream)))

    def close(self):
        if self._h is not None and _lib is not None:
            _lib.alexnet_loader_destroy(self._h)
            self._h = None

    def __del__(self):
        self.close()


def softmax_xent_static(logits: torch.Tensor, labels: torch.Tensor, dz: torch.Tensor, loss: torch.Tensor,
                        bad_label: Optional[torch.Tensor] = None, stream=None):
    """alexnet_softmax_xent_static: no handle, no workspace; every tensor is the caller's."""
    batch, classes = logits.shape
    _need(logits, torch.float32, batch * classes, "softmax_xent_static: logits")
    _need(labels, torch.int32, batch, "softmax_xent_static: labels")
    _need(dz, torch.float32, batch * classes, "softmax_xent_static: dz")
    _need(loss, torch.float32, 1, "softmax_xent_static: loss")
    if bad_label is not None:
        _need(bad_label, torch.int32, 1, "softmax_xent_static: bad_label")
    _check(_lib.alexnet_softmax_xent_static(_ptr(logits), _ptr(labels), batch, classes, _ptr(dz), _ptr(loss),
                                            _ptr(bad_label), _stream(stream)))


def average_gradients_update(a: AlexNet, b: AlexNet, stream=None):
    _check(_lib.alexnet_average_gradients_update(a._h, b._h, _stream(stream)))


def nchw_to_nhwc(x: torch.Tensor) -> torch.Tensor:
    n, c, h, w = x.shape
    y = torch.empty(n, h, w, c, dtype=torch.float32, device="cuda")
    _check(_lib.alexnet_nchw_to_nhwc(_ptr(x.contiguous()), _ptr(y), n, c, h, w, _stream(None)))
    return y


def nhwc_to_nchw(x: torch.Tensor) -> torch.Tensor:
    n, h, w, c = x.shape
    y = torch.empty(n, c, h, w, dtype=torch.float32, device="cuda")
    _check(_lib.alexnet_nhwc_to_nchw(_ptr(x.contiguous()), _ptr(y), n, c, h, w, _stream(None)))
    return y


# ---- group normalisation and 8-bit activation checkpoints ----
# Channel-last tensors [n]...[c] of float32, bfloat16 or float16.  A channel slice of a wider tensor is taken as it is (pixels
# at one stride).  Outputs and scratch are allocated on the stream that the call runs on, so calls share nothing.  A call on another
# `stream` than the current one waits for nothing: whoever passes one orders it behind the work that makes the inputs.  As everywhere
# in this module nothing is recorded for autograd: a gradient is its own call.
ACTIVATIONS = {"none": 0, "relu": 1, "silu": 2}
_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_CODES = {torch.int8: 0, torch.float8_e4m3fn: 1}
CODE_BLOCK = 32  # channels that share a scale


class Checkpoint:
    """An activation in 8 bits: codes (int8 or float8_e4m3fn) of its shape, scales (uint8) [...][ceil(c / 32)];
    value = code * 2^(scale - 127)."""

    __slots__ = ("codes", "scales")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor):
        if codes.dtype not in _CODES or scales.dtype != torch.uint8:
            raise ValueError(f"Checkpoint: codes are int8 or float8_e4m3fn and scales uint8, got {codes.dtype} and {scales.dtype}")
        if (codes.dim() < 2 or not 1 <= codes.shape[-1] < 1 << 31 or codes.shape[:-1] != scales.shape[:-1]
                or scales.shape[-1] != -(-codes.shape[-1] // CODE_BLOCK)):
            raise ValueError(f"Checkpoint: scales {list(scales.shape)} do not belong to codes {list(codes.shape)}")
        if not codes.is_contiguous() or not scales.is_contiguous() or codes.device != scales.device:
            raise ValueError("Checkpoint: codes and scales must be contiguous, on one device")
        self.codes, self.scales = codes, scales

    @staticmethod
    def _empty(shape, dtype: torch.dtype, device) -> "Checkpoint":
        if dtype not in _CODES:
            raise ValueError(f"a checkpoint's codes are int8 or float8_e4m3fn, got {dtype}")
        kept = Checkpoint.__new__(Checkpoint)
        kept.codes = torch.empty(shape, dtype=dtype, device=device)
        kept.scales = torch.empty((*shape[:-1], -(-shape[-1] // CODE_BLOCK)), dtype=torch.uint8, device=device)
        return kept

    @property
    def shape(self):
        return self.codes.shape

    def _arg(self) -> CheckpointArg:
        return CheckpointArg(self.codes.data_ptr(), self.scales.data_ptr(), _CODES[self.codes.dtype])

    @staticmethod
    def _need(kept, what: str):
        if not isinstance(kept, Checkpoint):
            raise TypeError(f"{what}: expected a Checkpoint, got {type(kept).__name__}")
        if not kept.codes.is_cuda:
            raise ValueError(f"{what}: expected a device tensor, got a checkpoint on {kept.codes.device}")


def _rows_stride(t, what: str) -> int:
    """Elements from one pixel to the next of a channel-last tensor whose pixels lie at one stride."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{what}: expected a torch.Tensor, got {type(t).__name__}")
    if not t.is_cuda:
        raise ValueError(f"{what}: expected a device tensor, got one on {t.device}")
    if t.dtype not in _TYPES:
        raise ValueError(f"{what}: expected float32, bfloat16 or float16, got {t.dtype}")
    if t.dim() < 2 or not 1 <= t.shape[-1] < 1 << 31:
        raise ValueError(f"{what}: expected [rows]...[channels], got {list(t.shape)}")
    c = t.shape[-1]
    if t.is_contiguous():
        return c
    ld = reach = None
    for size, stride in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if size == 1:
            continue
        if ld is None:
            ld = stride
        elif stride != reach:
            ld = -1
            break
        reach = stride * size
    ld = c if ld is None else ld
    if (c > 1 and t.stride(-1) != 1) or ld < c:
        raise ValueError(f"{what}: pixels must lie at one stride with their channels side by side, got strides {t.stride()} "
                         f"of {list(t.shape)}")
    return ld


_raw_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


def _here(t: torch.Tensor, stream) -> bool:
    """Whether a call on t runs on the current device and its current stream."""
    return stream is None and t.get_device() == torch.cuda.current_device()


def _there(t: torch.Tensor, stream, inputs, call):
    """call() on t's device, on `stream` if that is given: what it allocates then belongs to that stream's pool, and the
    allocator learns of the tensors that are used on a stream other than their own."""
    if stream is None:
        with torch.cuda.device(t.device):
            return call()
    if stream.device != t.device:
        raise ValueError(f"the stream belongs to {stream.device}, the tensors to {t.device}")
    caller = torch.cuda.current_stream(t.device)
    with torch.cuda.stream(stream):
        result = call()
    if stream != caller:
        outputs = result if isinstance(result, tuple) else (result,)
        for group, user in ((inputs, stream), (outputs, caller)):
            for x in group:
                for part in (x.codes, x.scales) if isinstance(x, Checkpoint) else (x,):
                    if part is not None:
                        part.record_stream(user)
    return result


def _vector(t, n: int, first: torch.Tensor, what: str):
    if t is None:
        return None
    _need(t, torch.float32, n, what)
    if t.numel() != n or t.device != first.device:
        raise ValueError(f"{what}: expected {n} elements on {first.device}, got {t.numel()} on {t.device}")
    return t.data_ptr()


def _result(out, shape, dtype, device, what: str):
    if out is None:
        return torch.empty(shape, dtype=dtype, device=device), shape[-1]
    ld = _rows_stride(out, what)
    if out.shape != shape or out.dtype != dtype or out.device != device:
        raise ValueError(f"{what}: expected {dtype} {list(shape)} on {device}, got {out.dtype} {list(out.shape)} on {out.device}")
    return out, ld


def _scratch(nbytes: int, device):
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None


@functools.lru_cache(maxsize=256)
def _group_norm_cfg(n: int, hw: int, c: int, groups: int, kind: int, act: str, eps: float, keep: bool):
    if act not in ACTIVATIONS:
        raise ValueError(f"activation must be one of {sorted(ACTIVATIONS)}, got {act!r}")
    if max(n, hw, c, groups) >= 1 << 31:
        raise ValueError("group_norm: sizes of 2^31 and more are not supported")
    cfg, forward, backward = GroupNormCfg(n, hw, c, groups, kind, ACTIVATIONS[act], eps), _sz(), _sz()
    _check(_lib.alexnet_group_norm_query(cfg, keep, forward, backward))
    return cfg, forward.value, backward.value


def group_norm_forward(x: torch.Tensor, gamma: Optional[torch.Tensor], beta: Optional[torch.Tensor], groups: int,
                       eps: float = 1e-5, act: str = "none", checkpoint: Optional[torch.dtype] = None,
                       out: Optional[torch.Tensor] = None, stream=None):
    """y = act(group_norm(x) * gamma + beta) of x [n]...[c]: (y, mean [n][groups], rstd [n][groups], kept).  checkpoint: the
    type of the codes (torch.int8, torch.float8_e4m3fn) of an 8-bit copy of x to leave in `kept`, else that is None.  out: where y
    goes (may be x)."""
    ld_x = _rows_stride(x, "group_norm_forward: x")
    if not _here(x, stream):
        return _there(x, stream, (x, gamma, beta, out),
                      lambda: group_norm_forward(x, gamma, beta, groups, eps, act, checkpoint, out))
    shape, device = x.shape, x.device
    n, c = shape[0], shape[-1]
    cfg, ws_bytes, _ = _group_norm_cfg(n, shape[1:-1].numel(), c, groups, _TYPES[x.dtype], act, eps, checkpoint is not None)
    p_gamma, p_beta = _vector(gamma, c, x, "group_norm_forward: gamma"), _vector(beta, c, x, "group_norm_forward: beta")
    y, ld_y = _result(out, shape, x.dtype, device, "group_norm_forward: out")
    mean = torch.empty((n, groups), dtype=torch.float32, device=device)
    rstd = torch.empty_like(mean)
    kept = None if checkpoint is None else Checkpoint._empty(shape, checkpoint, device)
    ws = _scratch(ws_bytes, device)
    _check(_lib.alexnet_group_norm_forward(cfg, x.data_ptr(), ld_x, p_gamma, p_beta, y.data_ptr(), ld_y, mean.data_ptr(),
                                           rstd.data_ptr(), None if kept is None else kept._arg(),
                                           None if ws is None else ws.data_ptr(), ws_bytes, _raw_stream(device.index)))
    return y, mean, rstd, kept


def group_norm_backward(x, dy: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor, gamma: Optional[torch.Tensor],
                        beta: Optional[torch.Tensor], act: str = "none", out: Optional[torch.Tensor] = None, stream=None):
    """(dx, dgamma, dbeta) of group_norm_forward from x, or its Checkpoint, and the forward call's mean and rstd.  out: where dx
    goes (may be dy, or x)."""
    what = "group_norm_backward"
    ld_dy = _rows_stride(dy, "group_norm_backward: dy")
    if not _here(dy, stream):
        return _there(dy, stream, (x, dy, mean, rstd, gamma, beta, out),
                      lambda: group_norm_backward(x, dy, mean, rstd, gamma, beta, act, out))
    shape, device = dy.shape, dy.device
    kept = p_x = None
    ld_x = 0
    if isinstance(x, Checkpoint):
        Checkpoint._need(x, what)
        kept, source = x._arg(), x.codes
    else:
        ld_x, p_x, source = _rows_stride(x, "group_norm_backward: x"), x.data_ptr(), x
    if source.shape != shape or source.device != device or (kept is None and x.dtype != dy.dtype):
        raise ValueError(f"{what}: x {list(source.shape)} and dy {list(shape)} differ in shape, type or device")
    n, c = shape[0], shape[-1]
    if not isinstance(mean, torch.Tensor) or not isinstance(rstd, torch.Tensor):
        raise TypeError(f"{what}: mean and rstd: expected torch.Tensors, got {type(mean).__name__} and {type(rstd).__name__}")
    if mean.dim() != 2 or mean.shape[0] != n or mean.shape[1] < 1:
        raise ValueError(f"{what}: mean: expected [{n}][groups], got {list(mean.shape)}")
    groups = mean.shape[1]
    p_mean, p_rstd = _vector(mean, n * groups, dy, "group_norm_backward: mean"), _vector(rstd, n * groups, dy, "group_norm_backward: rstd")
    p_gamma, p_beta = _vector(gamma, c, dy, "group_norm_backward: gamma"), _vector(beta, c, dy, "group_norm_backward: beta")
    cfg, _, ws_bytes = _group_norm_cfg(n, shape[1:-1].numel(), c, groups, _TYPES[dy.dtype], act, 1e-5, False)
    dx, ld_dx = _result(out, shape, dy.dtype, device, "group_norm_backward: out")
    dgamma = torch.empty(c, dtype=torch.float32, device=device)
    dbeta = torch.empty_like(dgamma)
    ws = _scratch(ws_bytes, device)
    _check(_lib.alexnet_group_norm_backward(cfg, p_x, ld_x, kept, dy.data_ptr(), ld_dy, p_mean, p_rstd, p_gamma, p_beta,
                                            dx.data_ptr(), ld_dx, dgamma.data_ptr(), dbeta.data_ptr(),
                                            None if ws is None else ws.data_ptr(), ws_bytes, _raw_stream(device.index)))
    return dx, dgamma, dbeta


def checkpoint_pack(x: torch.Tensor, dtype: torch.dtype = torch.int8, stream=None) -> Checkpoint:
    """x [rows]...[c] in 8 bits: codes of `dtype` (torch.int8 or torch.float8_e4m3fn), a power-of-two scale per 32 channels."""
    ld = _rows_stride(x, "checkpoint_pack: x")
    if not _here(x, stream):
        return _there(x, stream, (x,), lambda: checkpoint_pack(x, dtype))
    kept = Checkpoint._empty(x.shape, dtype, x.device)
    _check(_lib.alexnet_checkpoint_pack(x.data_ptr(), ld, _TYPES[x.dtype], x.shape[:-1].numel(), x.shape[-1], kept._arg(),
                                        _raw_stream(x.get_device())))
    return kept


def checkpoint_unpack(kept: Checkpoint, dtype: torch.dtype = torch.float32, out: Optional[torch.Tensor] = None,
                      stream=None) -> torch.Tensor:
    """The values of a checkpoint as float32, bfloat16 or float16."""
    Checkpoint._need(kept, "checkpoint_unpack")
    codes = kept.codes
    if dtype not in _TYPES:
        raise ValueError(f"checkpoint_unpack: expected float32, bfloat16 or float16, got {dtype}")
    if not _here(codes, stream):
        return _there(codes, stream, (kept, out), lambda: checkpoint_unpack(kept, dtype, out))
    x, ld = _result(out, codes.shape, dtype, codes.device, "checkpoint_unpack: out")
    _check(_lib.alexnet_checkpoint_unpack(kept._arg(), codes.shape[:-1].numel(), codes.shape[-1], x.data_ptr(), ld,
                                          _TYPES[dtype], _raw_stream(codes.get_device())))
    return x


@functools.lru_cache(maxsize=256)
def _checkpoint_fc_ws(rows: int, cols: int, out: int, kind: int) -> int:
    ws = _sz()
    _check(_lib.alexnet_checkpoint_fc_query(rows, cols, out, kind, C.byref(ws)))
    return ws.value


def checkpoint_fc_backward_weight(kept: Checkpoint, dy: torch.Tensor, dw: Optional[torch.Tensor] = None,
                                  db: Optional[torch.Tensor] = None, stream=None):
    """(dw [out][in], db [out]) in float32 of a dense layer, or of a 1 x 1 convolution over pixels, whose input [rows]...[in]
    was kept as a Checkpoint, from dy [rows]...[out].  dw, db: where they go."""
    what = "checkpoint_fc_backward_weight"
    Checkpoint._need(kept, what)
    codes = kept.codes
    ld = _rows_stride(dy, "checkpoint_fc_backward_weight: dy")
    if not _here(dy, stream):
        return _there(dy, stream, (kept, dy, dw, db), lambda: checkpoint_fc_backward_weight(kept, dy, dw, db))
    device = dy.device
    rows, cols, wide, kind = codes.shape[:-1].numel(), codes.shape[-1], dy.shape[-1], _TYPES[dy.dtype]
    if rows != dy.shape[:-1].numel() or codes.device != device:
        raise ValueError(f"{what}: a checkpoint {list(codes.shape)} on {codes.device} and dy {list(dy.shape)} on {device} differ "
                         "in their rows or device")
    _vector(dw, wide * cols, dy, "checkpoint_fc_backward_weight: dw")
    _vector(db, wide, dy, "checkpoint_fc_backward_weight: db")
    ws_bytes = _checkpoint_fc_ws(rows, cols, wide, kind)
    dw = torch.empty((wide, cols), dtype=torch.float32, device=device) if dw is None else dw
    db = torch.empty(wide, dtype=torch.float32, device=device) if db is None else db
    ws = _scratch(ws_bytes, device)
    _check(_lib.alexnet_checkpoint_fc_backward_weight(kept._arg(), dy.data_ptr(), ld, kind, rows, cols, wide, dw.data_ptr(),
                                                      db.data_ptr(), None if ws is None else ws.data_ptr(), ws_bytes,
                                                      _raw_stream(device.index)))
    return dw, db
