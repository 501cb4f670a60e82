"""ctypes binding of libslicemoe.so: the same entry points as include/slicemoe.h.

Argument marshalling only.  PyTorch supplies device memory (tensors) and streams; every step
of the layer runs in the HIP kernels of the library.  There is no fallback: if the library is
not built, or no GPU is present, calls raise.
"""
from __future__ import annotations

import ctypes
import itertools
import operator
import os
import struct

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libslicemoe.so")

SLICEMOE_OK = 0
SLICEMOE_ERR_INVALID_ARG = 1
SLICEMOE_ERR_UNSUPPORTED = 2
SLICEMOE_ERR_WORKSPACE = 3
SLICEMOE_ERR_HIP = 4
SLICEMOE_F32 = 0
SLICEMOE_BF16 = 1
SLICEMOE_GATE_NONE = 0
SLICEMOE_GATE_CHANNEL = 1
SLICEMOE_GATE_TOKEN = 2
SLICEMOE_FEW_ASSIGNMENTS = 1024
SLICEMOE_FLAG_FORCE_GENERIC = 1
SLICEMOE_FLAG_REQUIRE_MFMA = 2
SLICEMOE_FLAG_SINGLE_STREAM = 4

EXPORTS = [
    "slicemoe_status_string", "slicemoe_uses_mfma", "slicemoe_capacity", "slicemoe_workspace_bytes",
    "slicemoe_dispatch_workspace_bytes", "slicemoe_get_workspace_layout", "slicemoe_packed_bytes",
    "slicemoe_pack_weights", "slicemoe_route", "slicemoe_dispatch", "slicemoe_expert_ffn",
    "slicemoe_combine", "slicemoe_load_stats", "slicemoe_forward",
    "slicemoe_route_train", "slicemoe_forward_train", "slicemoe_backward_workspace_bytes", "slicemoe_backward",
    "slicemoe_backward_uses_mfma", "slicemoe_dispatch_noalloc",
    "slicemoe_add_rmsnorm", "slicemoe_add_rmsnorm_backward_workspace_bytes", "slicemoe_add_rmsnorm_backward",
    "slicemoe_gated_ffn_workspace_bytes", "slicemoe_gated_ffn", "slicemoe_gated_ffn_backward_workspace_bytes",
    "slicemoe_gated_ffn_backward", "slicemoe_gated_ffn_quantized_workspace_bytes", "slicemoe_gated_ffn_quantized",
    "slicemoe_gated_ffn_quantize_weights", "slicemoe_clip_grads_workspace_bytes", "slicemoe_clip_grads",
    "slicemoe_forward_few", "slicemoe_block_norm", "slicemoe_block_norm_backward_workspace_bytes", "slicemoe_block_norm_backward",
    "slicemoe_mx_bytes", "slicemoe_mx_quantize", "slicemoe_mx_dequantize", "slicemoe_mx_product_workspace_bytes", "slicemoe_mx_product",
    "slicemoe_gated_ffn_mx_workspace_bytes", "slicemoe_gated_ffn_mx",
]


class SliceMoEError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: status {status}")


class slicemoe_config(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("d", ctypes.c_int32), ("S", ctypes.c_int32), ("k", ctypes.c_int32),
                ("E", ctypes.c_int32), ("Hr", ctypes.c_int32), ("He", ctypes.c_int32),
                ("capacity_factor", ctypes.c_float), ("dtype", ctypes.c_int32), ("flags", ctypes.c_uint32)]


class slicemoe_weights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("Wr1", "br1", "Wr2", "br2", "W1", "b1", "W2", "b2", "packed")]


class slicemoe_route_train_params(ctypes.Structure):
    _fields_ = [("temperature", ctypes.c_float), ("noise_std", ctypes.c_float), ("dropout_rate", ctypes.c_float),
                ("capacity_alpha", ctypes.c_float)]


class slicemoe_weight_grads(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("Wr1", "br1", "Wr2", "br2", "W1", "b1", "W2", "b2")]


class slicemoe_workspace_layout(ctypes.Structure):
    _fields_ = [(n, ctypes.c_size_t) for n in ("topk_idx", "topk_p", "counts_raw", "counts", "offsets", "perm",
                                               "inv", "y", "stats", "scratch", "packed", "total")]


class slicemoe_norm_config(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("d", ctypes.c_int32), ("eps", ctypes.c_float), ("dtype", ctypes.c_int32)]


class slicemoe_gated_config(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("d", ctypes.c_int32), ("H", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class slicemoe_gated_weights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("Wg", "Wu", "Wd")]


class slicemoe_gated_weight_grads(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("Wg", "Wu", "Wd")]


class slicemoe_gated_weights_quantized(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("Wg", "Wu", "Wg_scale", "Wu_scale", "Wd")]


class slicemoe_grad(ctypes.Structure):
    _fields_ = [("grad", ctypes.c_void_p), ("out", ctypes.c_void_p), ("n", ctypes.c_int64), ("dtype", ctypes.c_int32)]


class slicemoe_block_norm_config(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("d", ctypes.c_int32), ("eps", ctypes.c_float), ("residual_scale", ctypes.c_float),
                ("gate", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class slicemoe_mx_config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("rows", "cols", "bits", "dtype", "transposed")]


class slicemoe_mx_product_config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("T", "K", "N", "bits", "dtype")]


class slicemoe_gated_weights_mx(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("Wg", "Wu", "Wd")]


_lib = None


def lib() -> ctypes.CDLL:
    """Load libslicemoe.so (built in-tree by paper_2510_04286_amd.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built: run `python -m paper_2510_04286_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        cfgp, wp, vp, st = ctypes.POINTER(slicemoe_config), ctypes.POINTER(slicemoe_weights), ctypes.c_void_p, ctypes.c_size_t
        L.slicemoe_status_string.restype = ctypes.c_char_p
        L.slicemoe_status_string.argtypes = [ctypes.c_int]
        L.slicemoe_uses_mfma.restype = ctypes.c_int
        L.slicemoe_uses_mfma.argtypes = [cfgp]
        L.slicemoe_capacity.restype = ctypes.c_int64
        L.slicemoe_capacity.argtypes = [cfgp]
        for f in (L.slicemoe_workspace_bytes, L.slicemoe_dispatch_workspace_bytes, L.slicemoe_packed_bytes):
            f.restype = st
            f.argtypes = [cfgp]
        L.slicemoe_get_workspace_layout.restype = ctypes.c_int
        L.slicemoe_get_workspace_layout.argtypes = [cfgp, ctypes.POINTER(slicemoe_workspace_layout)]
        L.slicemoe_pack_weights.restype = ctypes.c_int
        L.slicemoe_pack_weights.argtypes = [cfgp, wp, vp, st, vp]
        L.slicemoe_route.restype = ctypes.c_int
        L.slicemoe_route.argtypes = [cfgp, vp, wp, vp, vp, vp, st, vp]
        L.slicemoe_dispatch.restype = ctypes.c_int
        L.slicemoe_dispatch.argtypes = [cfgp, vp, vp, vp, vp, vp, vp, vp, st, vp]
        L.slicemoe_expert_ffn.restype = ctypes.c_int
        L.slicemoe_expert_ffn.argtypes = [cfgp, vp, vp, vp, vp, wp, vp, vp, st, vp]
        L.slicemoe_combine.restype = ctypes.c_int
        L.slicemoe_combine.argtypes = [cfgp, vp, vp, vp, vp]
        L.slicemoe_load_stats.restype = ctypes.c_int
        L.slicemoe_load_stats.argtypes = [cfgp, vp, vp, vp, vp]
        L.slicemoe_forward.restype = ctypes.c_int
        L.slicemoe_forward.argtypes = [cfgp, vp, wp, vp, vp, st, vp]
        tpp = ctypes.POINTER(slicemoe_route_train_params)
        L.slicemoe_route_train.restype = ctypes.c_int
        L.slicemoe_route_train.argtypes = [cfgp, vp, wp, tpp, vp, vp, vp, vp, vp, st, vp]
        L.slicemoe_forward_train.restype = ctypes.c_int
        L.slicemoe_forward_train.argtypes = [cfgp, vp, wp, tpp, vp, vp, vp, vp, st, vp]
        L.slicemoe_dispatch_noalloc.restype = ctypes.c_int
        L.slicemoe_dispatch_noalloc.argtypes = [cfgp, vp, vp, vp, vp, vp, vp, vp]
        L.slicemoe_backward_uses_mfma.restype = ctypes.c_int
        L.slicemoe_backward_uses_mfma.argtypes = [cfgp]
        L.slicemoe_backward_workspace_bytes.restype = ctypes.c_size_t
        L.slicemoe_backward_workspace_bytes.argtypes = [cfgp]
        L.slicemoe_backward.restype = ctypes.c_int
        L.slicemoe_backward.argtypes = [cfgp, vp, wp, tpp, vp, vp, vp, st, vp, vp, ctypes.POINTER(slicemoe_weight_grads),
                                        vp, st, vp]
        ncp, gcp = ctypes.POINTER(slicemoe_norm_config), ctypes.POINTER(slicemoe_gated_config)
        gwp, grp = ctypes.POINTER(slicemoe_gated_weights), ctypes.POINTER(slicemoe_grad)
        for f, a in ((L.slicemoe_add_rmsnorm_backward_workspace_bytes, [ncp]), (L.slicemoe_gated_ffn_workspace_bytes, [gcp]),
                     (L.slicemoe_gated_ffn_backward_workspace_bytes, [gcp]), (L.slicemoe_gated_ffn_quantized_workspace_bytes, [gcp]),
                     (L.slicemoe_clip_grads_workspace_bytes, [grp, ctypes.c_int32])):
            f.restype, f.argtypes = st, a
        for f, a in ((L.slicemoe_add_rmsnorm, [ncp, vp, vp, vp, vp, vp, vp, vp, vp]),
                     (L.slicemoe_add_rmsnorm_backward, [ncp, vp, vp, vp, vp, vp, vp, vp, st, vp]),
                     (L.slicemoe_gated_ffn, [gcp, vp, gwp, vp, vp, vp, st, vp]),
                     (L.slicemoe_gated_ffn_backward, [gcp, vp, gwp, vp, vp, vp, ctypes.POINTER(slicemoe_gated_weight_grads), vp, st, vp]),
                     (L.slicemoe_gated_ffn_quantized, [gcp, vp, vp, ctypes.POINTER(slicemoe_gated_weights_quantized), vp, vp, vp, st, vp]),
                     (L.slicemoe_gated_ffn_quantize_weights, [gcp, gwp, vp, vp, vp, vp, vp]),
                     (L.slicemoe_clip_grads, [grp, ctypes.c_int32, ctypes.c_float, vp, vp, st, vp])):
            f.restype, f.argtypes = ctypes.c_int, a
        i32, bnp, mxp, mpp = ctypes.c_int32, ctypes.POINTER(slicemoe_block_norm_config), ctypes.POINTER(slicemoe_mx_config), ctypes.POINTER(slicemoe_mx_product_config)
        for f, a in ((L.slicemoe_block_norm_backward_workspace_bytes, [bnp]), (L.slicemoe_mx_bytes, [mxp]),
                     (L.slicemoe_mx_product_workspace_bytes, [mpp]), (L.slicemoe_gated_ffn_mx_workspace_bytes, [gcp, i32])):
            f.restype, f.argtypes = st, a
        for f, a in ((L.slicemoe_forward_few, [cfgp, vp, wp, vp, vp, vp, vp]),
                     (L.slicemoe_block_norm, [bnp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, vp]),
                     (L.slicemoe_block_norm_backward, [bnp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, st, vp]),
                     (L.slicemoe_mx_quantize, [mxp, vp, vp, vp]), (L.slicemoe_mx_dequantize, [mxp, vp, vp, vp]),
                     (L.slicemoe_mx_product, [mpp, vp, vp, vp, vp, vp, st, vp]),
                     (L.slicemoe_gated_ffn_mx, [gcp, i32, vp, ctypes.POINTER(slicemoe_gated_weights_mx), vp, vp, vp, st, vp])):
            f.restype, f.argtypes = ctypes.c_int, a
        _lib = L
    return _lib


def make_config(T, d, S, k, E, He, dtype="bf16", capacity_factor=0.0, Hr=256, flags=0) -> slicemoe_config:
    return slicemoe_config(T, d, S, k, E, Hr, He, float(capacity_factor),
                           SLICEMOE_BF16 if dtype in ("bf16", SLICEMOE_BF16) else SLICEMOE_F32, flags)


def config_of(shape, flags=0) -> slicemoe_config:
    """slicemoe_config of a workload.SliceMoEShape."""
    return make_config(shape.T, shape.d, shape.S, shape.k, shape.E, shape.He, shape.dtype,
                       shape.capacity_factor, shape.Hr, flags)


# A small batch is bound by this marshalling and the launches (32 tokens of the d=1024 layer: 10 of 24 us), so the checks of a tensor
# are one pass over its attributes, addresses travel as integers, and the stream is asked for as a raw handle.
def _ptr(t, dtype=None, numel=None, name="tensor", dev=None):
    """Device address of a checked tensor; None for None.  dev: the device that it has to be on."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or (not t.is_cuda if dev is None else t.get_device() != dev):
        if isinstance(t, torch.Tensor) and t.is_cuda:
            raise ValueError(f"{name} is on device {t.get_device()}, the current device is {dev}")
        raise TypeError(f"{name} must be a CUDA/HIP tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if numel is not None and t.numel() < numel:
        raise ValueError(f"{name} has {t.numel()} elements, needs {numel}")
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return stream.cuda_stream


def _tdtype(cfg):
    return torch.bfloat16 if cfg.dtype == SLICEMOE_BF16 else torch.float32


def y_dtype(cfg):
    """Element type of the stacked expert outputs y: fp16 with bf16 storage, fp32 with fp32 storage."""
    return torch.float16 if cfg.dtype == SLICEMOE_BF16 else torch.float32


def _weights(cfg, w) -> slicemoe_weights:
    """dict of device tensors (logical layout, optional 'packed' uint8 buffer) -> C struct."""
    dt = _tdtype(cfg)
    E, Hr, He = cfg.E, cfg.Hr, cfg.He
    ds = cfg.d // cfg.S
    get, nW = w.get, E * ds * He
    pk = get("packed")
    return slicemoe_weights(
        _ptr(get("Wr1"), dt, ds * Hr, "Wr1"), _ptr(get("br1"), dt, Hr, "br1"), _ptr(get("Wr2"), dt, Hr * E, "Wr2"),
        _ptr(get("br2"), dt, E, "br2"), _ptr(get("W1"), dt, nW, "W1"), _ptr(get("b1"), dt, E * He, "b1"),
        _ptr(get("W2"), dt, nW, "W2"), _ptr(get("b2"), dt, E * ds, "b2"),
        None if pk is None else _ptr(pk, torch.uint8, (_lib or lib()).slicemoe_packed_bytes(ctypes.byref(cfg)), "packed"))


def _ws(workspace, dev=None):
    if workspace is None:
        return None, 0
    return _ptr(workspace, torch.uint8, None, "workspace", dev), workspace.numel()


def _check(status, what):
    if status != SLICEMOE_OK:
        raise SliceMoEError(status, f"{what}: {lib().slicemoe_status_string(status).decode()}")


# ------------------------------------------------------------------ queries
def slicemoe_status_string(status: int) -> str:
    return lib().slicemoe_status_string(status).decode()


def slicemoe_uses_mfma(cfg) -> int:
    return lib().slicemoe_uses_mfma(ctypes.byref(cfg))


def slicemoe_capacity(cfg) -> int:
    return lib().slicemoe_capacity(ctypes.byref(cfg))


def slicemoe_workspace_bytes(cfg) -> int:
    return lib().slicemoe_workspace_bytes(ctypes.byref(cfg))


def slicemoe_dispatch_workspace_bytes(cfg) -> int:
    return lib().slicemoe_dispatch_workspace_bytes(ctypes.byref(cfg))


def slicemoe_packed_bytes(cfg) -> int:
    return lib().slicemoe_packed_bytes(ctypes.byref(cfg))


def slicemoe_get_workspace_layout(cfg) -> slicemoe_workspace_layout:
    out = slicemoe_workspace_layout()
    _check(lib().slicemoe_get_workspace_layout(ctypes.byref(cfg), ctypes.byref(out)), "slicemoe_get_workspace_layout")
    return out


# ------------------------------------------------------------------ stages
def slicemoe_pack_weights(cfg, w, packed_out, stream=None):
    ws = _weights(cfg, {k: v for k, v in w.items() if k != "packed"})
    _check(lib().slicemoe_pack_weights(ctypes.byref(cfg), ctypes.byref(ws), _ptr(packed_out, torch.uint8, None, "packed_out"),
                                       packed_out.numel(), _stream(stream)), "slicemoe_pack_weights")


def slicemoe_route(cfg, h, w, topk_idx, topk_p, workspace=None, stream=None):
    Ns = cfg.T * cfg.S
    wsp, wsb = _ws(workspace)
    ws = _weights(cfg, w)
    _check(lib().slicemoe_route(ctypes.byref(cfg), _ptr(h, _tdtype(cfg), cfg.T * cfg.d, "h"), ctypes.byref(ws),
                                _ptr(topk_idx, torch.int32, Ns * cfg.k, "topk_idx"),
                                _ptr(topk_p, torch.float32, Ns * cfg.k, "topk_p"), wsp, wsb, _stream(stream)),
           "slicemoe_route")


def slicemoe_dispatch(cfg, topk_idx, counts_raw, counts, offsets, perm, inv, workspace, stream=None):
    Na = cfg.T * cfg.S * cfg.k
    wsp, wsb = _ws(workspace)
    _check(lib().slicemoe_dispatch(ctypes.byref(cfg), _ptr(topk_idx, torch.int32, Na, "topk_idx"),
                                   _ptr(counts_raw, torch.int32, cfg.E, "counts_raw"),
                                   _ptr(counts, torch.int32, cfg.E, "counts"),
                                   _ptr(offsets, torch.int32, cfg.E + 1, "offsets"),
                                   _ptr(perm, torch.int32, Na, "perm"), _ptr(inv, torch.int32, Na, "inv"),
                                   wsp, wsb, _stream(stream)), "slicemoe_dispatch")


def slicemoe_dispatch_noalloc(cfg, topk_idx, counts_raw, counts, offsets, perm, inv, stream=None):
    Na = cfg.T * cfg.S * cfg.k
    _check(lib().slicemoe_dispatch_noalloc(ctypes.byref(cfg), _ptr(topk_idx, torch.int32, Na, "topk_idx"),
                                           _ptr(counts_raw, torch.int32, cfg.E, "counts_raw"),
                                           _ptr(counts, torch.int32, cfg.E, "counts"),
                                           _ptr(offsets, torch.int32, cfg.E + 1, "offsets"),
                                           _ptr(perm, torch.int32, Na, "perm"), _ptr(inv, torch.int32, Na, "inv"),
                                           _stream(stream)), "slicemoe_dispatch_noalloc")


def slicemoe_expert_ffn(cfg, h, topk_p, offsets, perm, w, y, workspace=None, stream=None):
    Na = cfg.T * cfg.S * cfg.k
    wsp, wsb = _ws(workspace)
    ws = _weights(cfg, w)
    _check(lib().slicemoe_expert_ffn(ctypes.byref(cfg), _ptr(h, _tdtype(cfg), cfg.T * cfg.d, "h"),
                                     _ptr(topk_p, torch.float32, Na, "topk_p"),
                                     _ptr(offsets, torch.int32, cfg.E + 1, "offsets"),
                                     _ptr(perm, torch.int32, Na, "perm"), ctypes.byref(ws),
                                     _ptr(y, y_dtype(cfg), Na * (cfg.d // cfg.S), "y"), wsp, wsb, _stream(stream)),
           "slicemoe_expert_ffn")


def slicemoe_combine(cfg, y, inv, h_out, stream=None):
    Na = cfg.T * cfg.S * cfg.k
    _check(lib().slicemoe_combine(ctypes.byref(cfg), _ptr(y, y_dtype(cfg), Na * (cfg.d // cfg.S), "y"),
                                  _ptr(inv, torch.int32, Na, "inv"),
                                  _ptr(h_out, _tdtype(cfg), cfg.T * cfg.d, "h_out"), _stream(stream)),
           "slicemoe_combine")


def slicemoe_load_stats(cfg, counts_raw, counts, stats, stream=None):
    _check(lib().slicemoe_load_stats(ctypes.byref(cfg), _ptr(counts_raw, torch.int32, cfg.E, "counts_raw"),
                                     _ptr(counts, torch.int32, cfg.E, "counts"),
                                     _ptr(stats, torch.float32, 4, "stats"), _stream(stream)), "slicemoe_load_stats")


def slicemoe_forward(cfg, h, w, h_out, workspace, stream=None):
    wsp, wsb = _ws(workspace)
    ws = _weights(cfg, w)
    _check(lib().slicemoe_forward(ctypes.byref(cfg), _ptr(h, _tdtype(cfg), cfg.T * cfg.d, "h"), ctypes.byref(ws),
                                  _ptr(h_out, _tdtype(cfg), cfg.T * cfg.d, "h_out"), wsp, wsb, _stream(stream)),
           "slicemoe_forward")


def slicemoe_forward_few(cfg, h, w, h_out, topk_idx=None, topk_p=None, stream=None):
    """The layer for a few tokens in one launch; on the matrix-core path w needs its 'packed' buffer and nothing else."""
    L, dev, Na = _lib or lib(), _device(), cfg.T * cfg.S * cfg.k
    dt, n = _tdtype(cfg), cfg.T * cfg.d
    need = L.slicemoe_packed_bytes(ctypes.byref(cfg))   # 0: generic
    if need:
        ws = slicemoe_weights(None, None, None, None, None, None, None, None, _ptr(w.get("packed"), torch.uint8, need, "packed", dev))
    else:
        for name, t in w.items():
            _ptr(t, None, None, name, dev)
        ws = _weights(cfg, w)
    st = L.slicemoe_forward_few(ctypes.byref(cfg), _ptr(h, dt, n, "h", dev), ctypes.byref(ws), _ptr(h_out, dt, n, "h_out", dev),
                                _ptr(topk_idx, torch.int32, Na, "topk_idx", dev), _ptr(topk_p, torch.float32, Na, "topk_p", dev), _stream_on(dev, stream))
    if st:
        _check(st, "slicemoe_forward_few")


def _train_args(cfg, temperature, noise_std, dropout_rate, noise, drop_u, capacity_alpha=0.0):
    tp = slicemoe_route_train_params(temperature, noise_std, dropout_rate, capacity_alpha)
    Ns = cfg.T * cfg.S
    npt = None if noise is None else _ptr(noise, torch.float32, Ns * cfg.E, "noise")
    upt = None if drop_u is None else _ptr(drop_u, torch.float32, Ns * cfg.k, "drop_u")
    return tp, npt, upt


def slicemoe_route_train(cfg, h, w, topk_idx, topk_p, temperature=1.0, noise_std=0.0, dropout_rate=0.0, noise=None,
                         drop_u=None, workspace=None, stream=None, capacity_alpha=0.0):
    """capacity_alpha travels in the parameter struct; only slicemoe_backward reads it."""
    Ns = cfg.T * cfg.S
    wsp, wsb = _ws(workspace)
    ws = _weights(cfg, w)
    tp, npt, upt = _train_args(cfg, temperature, noise_std, dropout_rate, noise, drop_u, capacity_alpha)
    _check(lib().slicemoe_route_train(ctypes.byref(cfg), _ptr(h, _tdtype(cfg), cfg.T * cfg.d, "h"), ctypes.byref(ws),
                                      ctypes.byref(tp), npt, upt, _ptr(topk_idx, torch.int32, Ns * cfg.k, "topk_idx"),
                                      _ptr(topk_p, torch.float32, Ns * cfg.k, "topk_p"), wsp, wsb, _stream(stream)),
           "slicemoe_route_train")


def slicemoe_forward_train(cfg, h, w, h_out, workspace, temperature=1.0, noise_std=0.0, dropout_rate=0.0, noise=None,
                           drop_u=None, stream=None, capacity_alpha=0.0):
    """capacity_alpha travels in the parameter struct; only slicemoe_backward reads it."""
    wsp, wsb = _ws(workspace)
    ws = _weights(cfg, w)
    tp, npt, upt = _train_args(cfg, temperature, noise_std, dropout_rate, noise, drop_u, capacity_alpha)
    _check(lib().slicemoe_forward_train(ctypes.byref(cfg), _ptr(h, _tdtype(cfg), cfg.T * cfg.d, "h"), ctypes.byref(ws),
                                        ctypes.byref(tp), npt, upt, _ptr(h_out, _tdtype(cfg), cfg.T * cfg.d, "h_out"),
                                        wsp, wsb, _stream(stream)), "slicemoe_forward_train")


def slicemoe_backward_uses_mfma(cfg) -> int:
    return int(lib().slicemoe_backward_uses_mfma(ctypes.byref(cfg)))


def slicemoe_backward_workspace_bytes(cfg) -> int:
    return int(lib().slicemoe_backward_workspace_bytes(ctypes.byref(cfg)))


def alloc_weight_grads(cfg, device="cuda:0") -> dict:
    """fp32 device tensors in the logical layout of each weight tensor (contents undefined until slicemoe_backward)."""
    ds = cfg.d // cfg.S
    shapes = {"Wr1": (ds, cfg.Hr), "br1": (cfg.Hr,), "Wr2": (cfg.Hr, cfg.E), "br2": (cfg.E,),
              "W1": (cfg.E, ds, cfg.He), "b1": (cfg.E, cfg.He), "W2": (cfg.E, cfg.He, ds), "b2": (cfg.E, ds)}
    return {n: torch.empty(sh, dtype=torch.float32, device=device) for n, sh in shapes.items()}


def slicemoe_backward(cfg, h, w, forward_workspace, d_out, d_h, grads: dict, workspace, train: dict | None = None,
                      stream=None):
    """train: None after slicemoe_forward, else the keyword arguments given to slicemoe_forward_train, and optionally
    capacity_alpha (weight of the capacity loss's gradient; the forward calls do not read it)."""
    fwp, fwb = _ws(forward_workspace)
    wsp, wsb = _ws(workspace)
    ws = _weights(cfg, w)
    tpp, npt, upt = None, None, None
    if train is not None:
        tp, npt, upt = _train_args(cfg, train.get("temperature", 1.0), train.get("noise_std", 0.0),
                                   train.get("dropout_rate", 0.0), train.get("noise"), train.get("drop_u"),
                                   train.get("capacity_alpha", 0.0))
        tpp = ctypes.byref(tp)
    E, Hr, He = cfg.E, cfg.Hr, cfg.He
    ds, f32 = cfg.d // cfg.S, torch.float32
    nW = E * ds * He
    g = slicemoe_weight_grads(
        _ptr(grads["Wr1"], f32, ds * Hr, "grads.Wr1"), _ptr(grads["br1"], f32, Hr, "grads.br1"), _ptr(grads["Wr2"], f32, Hr * E, "grads.Wr2"),
        _ptr(grads["br2"], f32, E, "grads.br2"), _ptr(grads["W1"], f32, nW, "grads.W1"), _ptr(grads["b1"], f32, E * He, "grads.b1"),
        _ptr(grads["W2"], f32, nW, "grads.W2"), _ptr(grads["b2"], f32, E * ds, "grads.b2"))
    _check(lib().slicemoe_backward(ctypes.byref(cfg), _ptr(h, _tdtype(cfg), cfg.T * cfg.d, "h"), ctypes.byref(ws), tpp,
                                   npt, upt, fwp, fwb, _ptr(d_out, _tdtype(cfg), cfg.T * cfg.d, "d_out"),
                                   _ptr(d_h, _tdtype(cfg), cfg.T * cfg.d, "d_h"), ctypes.byref(g), wsp, wsb,
                                   _stream(stream)), "slicemoe_backward")


# ------------------------------------------------------------------ operators around the layer
_DTYPE_CODES = {**dict.fromkeys(("bf16", "bfloat16", torch.bfloat16, SLICEMOE_BF16), SLICEMOE_BF16),
                **dict.fromkeys(("f32", "fp32", "float32", torch.float32, SLICEMOE_F32), SLICEMOE_F32)}


def _dtype_code(dtype):
    try:
        return _DTYPE_CODES[dtype]
    except (KeyError, TypeError):   # (TypeError: nothing that can be a name)
        raise ValueError(f"dtype must be one of 'bf16', 'f32', torch.bfloat16 and torch.float32, got {dtype!r}") from None


def make_norm_config(T, d, eps=1e-5, dtype="bf16") -> slicemoe_norm_config:
    return slicemoe_norm_config(T, d, float(eps), _dtype_code(dtype))


def make_gated_config(T, d, H, dtype="bf16") -> slicemoe_gated_config:
    return slicemoe_gated_config(T, d, H, _dtype_code(dtype))


def _device():
    """The current device.  Kernels go to it, so the tensors and the stream of a call have to be on it: another card's memory need not be
    reachable from here, and a launch that reaches for it all the same takes the process down."""
    try:
        return torch._C._cuda_getDevice()
    except (AttributeError, RuntimeError):   # no GPU: no tensor is on it
        return -2


def _stream_on(dev, stream):
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(dev)
    if stream.device_index != dev:
        raise ValueError(f"stream is of device {stream.device_index}, the current device is {dev}")
    return stream.cuda_stream


def _bytes_ptr(t, numel, name, dev):
    """Address of e4m3 values: a float8_e4m3fn tensor, or its bytes."""
    if t is not None and isinstance(t, torch.Tensor) and t.dtype == torch.uint8:
        return _ptr(t, torch.uint8, numel, name, dev)
    return _ptr(t, torch.float8_e4m3fn, numel, name, dev)


def slicemoe_add_rmsnorm(cfg, x, residual, weight, sum_out, y, y_quantized=None, y_scale=None, stream=None):
    """residual, sum_out and, with y_quantized, y may be None."""
    d, T, dev = cfg.d, cfg.T, _device()
    dt, n = _tdtype(cfg), T * d
    st = (_lib or lib()).slicemoe_add_rmsnorm(
        ctypes.byref(cfg), _ptr(x, dt, n, "x", dev), _ptr(residual, dt, n, "residual", dev), _ptr(weight, dt, d, "weight", dev),
        _ptr(sum_out, dt, n, "sum_out", dev), _ptr(y, dt, n, "y", dev), None if y_quantized is None else _bytes_ptr(y_quantized, n, "y_quantized", dev),
        None if y_scale is None else _ptr(y_scale, torch.float32, T, "y_scale", dev), _stream_on(dev, stream))
    if st:
        _check(st, "slicemoe_add_rmsnorm")


def slicemoe_add_rmsnorm_backward_workspace_bytes(cfg) -> int:
    return lib().slicemoe_add_rmsnorm_backward_workspace_bytes(ctypes.byref(cfg))


def slicemoe_add_rmsnorm_backward(cfg, sum_in, weight, d_y, d_x, d_weight, workspace, d_sum=None, stream=None):
    dt, n, dev = _tdtype(cfg), cfg.T * cfg.d, _device()
    wsp, wsb = _ws(workspace, dev)
    _check(lib().slicemoe_add_rmsnorm_backward(ctypes.byref(cfg), _ptr(sum_in, dt, n, "sum_in", dev), _ptr(weight, dt, cfg.d, "weight", dev),
                                               _ptr(d_y, dt, n, "d_y", dev), _ptr(d_sum, dt, n, "d_sum", dev), _ptr(d_x, dt, n, "d_x", dev),
                                               _ptr(d_weight, torch.float32, cfg.d, "d_weight", dev), wsp, wsb, _stream_on(dev, stream)),
           "slicemoe_add_rmsnorm_backward")


def slicemoe_gated_ffn_workspace_bytes(cfg) -> int:
    return lib().slicemoe_gated_ffn_workspace_bytes(ctypes.byref(cfg))


def slicemoe_gated_ffn_backward_workspace_bytes(cfg) -> int:
    return lib().slicemoe_gated_ffn_backward_workspace_bytes(ctypes.byref(cfg))


def slicemoe_gated_ffn_quantized_workspace_bytes(cfg) -> int:
    return lib().slicemoe_gated_ffn_quantized_workspace_bytes(ctypes.byref(cfg))


def _gated_weights(cfg, w, dev, kind=slicemoe_gated_weights, what="", down=True):
    dt, n = _tdtype(cfg), cfg.d * cfg.H
    return kind(_ptr(w["Wg"], dt, n, what + "Wg", dev), _ptr(w["Wu"], dt, n, what + "Wu", dev), _ptr(w["Wd"], dt, n, what + "Wd", dev) if down else None)


def slicemoe_gated_ffn(cfg, x, w, y, workspace, addend=None, stream=None):
    """w: dict of Wg, Wu [d, H] and Wd [H, d]."""
    dt, n, dev = _tdtype(cfg), cfg.T * cfg.d, _device()
    wsp, wsb = _ws(workspace, dev)
    ws = _gated_weights(cfg, w, dev)
    _check(lib().slicemoe_gated_ffn(ctypes.byref(cfg), _ptr(x, dt, n, "x", dev), ctypes.byref(ws), _ptr(addend, dt, n, "addend", dev),
                                    _ptr(y, dt, n, "y", dev), wsp, wsb, _stream_on(dev, stream)), "slicemoe_gated_ffn")


def slicemoe_gated_ffn_backward(cfg, x, w, d_y, d_x, grads, workspace, addend=None, stream=None):
    """grads: dict of Wg, Wu, Wd in the storage dtype, overwritten."""
    dt, n, dev = _tdtype(cfg), cfg.T * cfg.d, _device()
    wsp, wsb = _ws(workspace, dev)
    ws, g = _gated_weights(cfg, w, dev), _gated_weights(cfg, grads, dev, slicemoe_gated_weight_grads, "grads.")
    _check(lib().slicemoe_gated_ffn_backward(ctypes.byref(cfg), _ptr(x, dt, n, "x", dev), ctypes.byref(ws), _ptr(d_y, dt, n, "d_y", dev),
                                             _ptr(addend, dt, n, "addend", dev), _ptr(d_x, dt, n, "d_x", dev), ctypes.byref(g), wsp, wsb,
                                             _stream_on(dev, stream)), "slicemoe_gated_ffn_backward")


def slicemoe_gated_ffn_quantized(cfg, x_quantized, x_scale, w, y, workspace, addend=None, stream=None):
    """w: dict of Wg, Wu [H, d] e4m3 with Wg_scale, Wu_scale [H], and Wd [H, d] bf16 (see quantize_gated_weights)."""
    n, nw, f32, dev = cfg.T * cfg.d, cfg.d * cfg.H, torch.float32, _device()
    wsp, wsb = _ws(workspace, dev)
    ws = slicemoe_gated_weights_quantized(_bytes_ptr(w["Wg"], nw, "Wg", dev), _bytes_ptr(w["Wu"], nw, "Wu", dev), _ptr(w["Wg_scale"], f32, cfg.H, "Wg_scale", dev),
                                          _ptr(w["Wu_scale"], f32, cfg.H, "Wu_scale", dev), _ptr(w["Wd"], torch.bfloat16, nw, "Wd", dev))
    _check(lib().slicemoe_gated_ffn_quantized(ctypes.byref(cfg), _bytes_ptr(x_quantized, n, "x_quantized", dev), _ptr(x_scale, f32, cfg.T, "x_scale", dev),
                                              ctypes.byref(ws), _ptr(addend, torch.bfloat16, n, "addend", dev),
                                              _ptr(y, torch.bfloat16, n, "y", dev), wsp, wsb, _stream_on(dev, stream)), "slicemoe_gated_ffn_quantized")


def slicemoe_gated_ffn_quantize_weights(cfg, w, Wg, Wg_scale, Wu, Wu_scale, stream=None):
    nw, f32, dev = cfg.d * cfg.H, torch.float32, _device()
    ws = _gated_weights(cfg, w, dev, down=False)
    _check(lib().slicemoe_gated_ffn_quantize_weights(ctypes.byref(cfg), ctypes.byref(ws), _bytes_ptr(Wg, nw, "Wg", dev),
                                                     _ptr(Wg_scale, f32, cfg.H, "Wg_scale", dev), _bytes_ptr(Wu, nw, "Wu", dev),
                                                     _ptr(Wu_scale, f32, cfg.H, "Wu_scale", dev), _stream_on(dev, stream)),
           "slicemoe_gated_ffn_quantize_weights")


def quantize_gated_weights(cfg, w: dict, device=None) -> dict:
    """The weight dict that slicemoe_gated_ffn_quantized takes, from the bf16 one (Wd is shared), on the device of w."""
    device = w["Wg"].device if device is None else device
    q = {n: torch.empty((cfg.H, cfg.d), dtype=torch.float8_e4m3fn, device=device) for n in ("Wg", "Wu")}
    q.update({n: torch.empty(cfg.H, dtype=torch.float32, device=device) for n in ("Wg_scale", "Wu_scale")})
    slicemoe_gated_ffn_quantize_weights(cfg, w, q["Wg"], q["Wg_scale"], q["Wu"], q["Wu_scale"])
    return {**q, "Wd": w["Wd"]}


_GRAD_CODES = {torch.float32: SLICEMOE_F32, torch.bfloat16: SLICEMOE_BF16}
_GRAD_FIELDS = "QQqi4x"   # slicemoe_grad
_dtype_of = operator.attrgetter("dtype")


def _check_list(tensors, name, dev):
    for i, t in enumerate(tensors):
        if t is None:
            raise TypeError(f"{name}[{i}] must be a CUDA/HIP tensor")
        _ptr(t, None, None, f"{name}[{i}]", dev)


def _grad_list(grads, out, dev=None):
    """C array of a list of gradient tensors; out: the list written, the same list for in place, or None to measure only.  (One
    attribute of all tensors at a time: dozens of small tensors are bound by this marshalling, 40 us for 48 of them tensor by tensor, 25 so.)"""
    T = torch.Tensor
    for tensors, name in ((grads, "grads"),) if out is None or out is grads else ((grads, "grads"), (out, "out")):
        try:
            on = set(map(T.get_device, tensors))
            fine = all(map(T.is_contiguous, tensors)) and (-1 not in on if dev is None else on <= {dev})   # (-1: host memory)
        except TypeError:   # not a tensor
            fine = False
        if not fine:
            _check_list(tensors, name, dev)   # raises
    types, sizes, addresses = list(map(_dtype_of, grads)), list(map(T.numel, grads)), list(map(T.data_ptr, grads))
    codes = list(map(_GRAD_CODES.get, types))
    if None in codes:
        raise TypeError(f"grads[{codes.index(None)}] must be a float32 or bfloat16 tensor")
    if out is None:
        written = [0] * len(grads)
    elif out is grads:
        written = addresses
    else:
        if types != list(map(_dtype_of, out)) or sizes != list(map(T.numel, out)):
            raise ValueError("out must have the tensors of grads: as many, of their sizes and types")
        written = list(map(T.data_ptr, out))
    return struct.pack(_GRAD_FIELDS * len(grads), *itertools.chain.from_iterable(zip(addresses, written, sizes, codes)))


def _grad_pointer(packed):
    return ctypes.cast(packed, ctypes.POINTER(slicemoe_grad)) if packed else None


def slicemoe_clip_grads_workspace_bytes(grads) -> int:
    packed = _grad_list(grads, None)
    return lib().slicemoe_clip_grads_workspace_bytes(_grad_pointer(packed), len(grads))


def slicemoe_clip_grads(grads, max_norm, norm, workspace, out=None, stream=None):
    """out: the tensors written (grads itself for in place); None leaves all of them as they are and only measures."""
    dev = _device()
    wsp, wsb = _ws(workspace, dev)
    packed = _grad_list(grads, out, dev)
    _check(lib().slicemoe_clip_grads(_grad_pointer(packed), len(grads), max_norm, _ptr(norm, torch.float32, 1, "norm", dev), wsp, wsb,
                                     _stream_on(dev, stream)), "slicemoe_clip_grads")


_GATE_CODES = {None: SLICEMOE_GATE_NONE, "channel": SLICEMOE_GATE_CHANNEL, "token": SLICEMOE_GATE_TOKEN}


def make_block_norm_config(T, d, eps=1e-5, residual_scale=1.0, gate="channel", dtype="bf16") -> slicemoe_block_norm_config:
    """gate: None, "channel" (one row [d] for all tokens) or "token" (a row for each, [T, d])."""
    if gate not in _GATE_CODES:
        raise ValueError(f"gate must be None, 'channel' or 'token', got {gate!r}")
    return slicemoe_block_norm_config(T, d, float(eps), float(residual_scale), _GATE_CODES[gate], _dtype_code(dtype))


def make_mx_config(rows, cols, bits=4, dtype="bf16", transposed=False) -> slicemoe_mx_config:
    return slicemoe_mx_config(rows, cols, bits, _dtype_code(dtype), int(transposed))


def make_mx_product_config(T, K, N, bits=4, dtype="bf16") -> slicemoe_mx_product_config:
    return slicemoe_mx_product_config(T, K, N, bits, _dtype_code(dtype))


def slicemoe_mx_bytes(cfg) -> int:
    return (_lib or lib()).slicemoe_mx_bytes(ctypes.byref(cfg))


def _mx_ptr(t, rows, cols, bits, name, dev):
    """Address of a packed matrix of microscaled values."""
    return _ptr(t, torch.uint8, -(-rows // 32) * -(-cols // 256) * (1024 * bits + 256), name, dev)


def _gate_numel(cfg):
    return cfg.T * cfg.d if cfg.gate == SLICEMOE_GATE_TOKEN else cfg.d


def slicemoe_block_norm(cfg, x, post_weight, gate, residual, pre_weight, sum_out, y, y_mx=None, y_bits=0, stats=None, stream=None):
    """post_weight, gate (as cfg says), y with y_mx, and pre_weight with both of them, may be None."""
    d, T, dev = cfg.d, cfg.T, _device()
    dt, n = _tdtype(cfg), T * d
    st = (_lib or lib()).slicemoe_block_norm(
        ctypes.byref(cfg), _ptr(x, dt, n, "x", dev), _ptr(post_weight, dt, d, "post_weight", dev), _ptr(gate, dt, _gate_numel(cfg), "gate", dev),
        _ptr(residual, dt, n, "residual", dev), _ptr(pre_weight, dt, d, "pre_weight", dev), _ptr(sum_out, dt, n, "sum_out", dev), _ptr(y, dt, n, "y", dev),
        None if y_mx is None else _mx_ptr(y_mx, T, d, y_bits, "y_mx", dev), y_bits,
        None if stats is None else _ptr(stats, torch.float32, 2 * T, "stats", dev), _stream_on(dev, stream))
    if st:
        _check(st, "slicemoe_block_norm")


def slicemoe_block_norm_backward_workspace_bytes(cfg) -> int:
    return lib().slicemoe_block_norm_backward_workspace_bytes(ctypes.byref(cfg))


def slicemoe_block_norm_backward(cfg, x, post_weight, gate, sum_in, pre_weight, stats, d_y, d_x, d_residual, d_post_weight, d_gate, d_pre_weight,
                                 workspace, d_sum=None, stream=None):
    """d_gate: float32 [d] with a "channel" gate, [T, d] of the storage type with a "token" one; None without; d_post_weight likewise."""
    d, T, dev = cfg.d, cfg.T, _device()
    dt, n, f32 = _tdtype(cfg), T * d, torch.float32
    wsp, wsb = _ws(workspace, dev)
    st = (_lib or lib()).slicemoe_block_norm_backward(
        ctypes.byref(cfg), _ptr(x, dt, n, "x", dev), _ptr(post_weight, dt, d, "post_weight", dev), _ptr(gate, dt, _gate_numel(cfg), "gate", dev),
        _ptr(sum_in, dt, n, "sum_in", dev), _ptr(pre_weight, dt, d, "pre_weight", dev), _ptr(stats, f32, 2 * T, "stats", dev), _ptr(d_y, dt, n, "d_y", dev),
        _ptr(d_sum, dt, n, "d_sum", dev), _ptr(d_x, dt, n, "d_x", dev), _ptr(d_residual, dt, n, "d_residual", dev),
        _ptr(d_post_weight, f32, d, "d_post_weight", dev), _ptr(d_gate, dt if cfg.gate == SLICEMOE_GATE_TOKEN else f32, _gate_numel(cfg), "d_gate", dev),
        _ptr(d_pre_weight, f32, d, "d_pre_weight", dev), wsp, wsb, _stream_on(dev, stream))
    if st:
        _check(st, "slicemoe_block_norm_backward")


def slicemoe_mx_quantize(cfg, x, mx, stream=None):
    """x: [rows, cols], or [cols, rows] with cfg.transposed -> mx, a uint8 buffer of slicemoe_mx_bytes."""
    dev = _device()
    st = (_lib or lib()).slicemoe_mx_quantize(ctypes.byref(cfg), _ptr(x, _tdtype(cfg), cfg.rows * cfg.cols, "x", dev),
                                              _mx_ptr(mx, cfg.rows, cfg.cols, cfg.bits, "mx", dev), _stream_on(dev, stream))
    if st:
        _check(st, "slicemoe_mx_quantize")


def slicemoe_mx_dequantize(cfg, mx, x, stream=None):
    dev = _device()
    _check((_lib or lib()).slicemoe_mx_dequantize(ctypes.byref(cfg), _mx_ptr(mx, cfg.rows, cfg.cols, cfg.bits, "mx", dev),
                                                  _ptr(x, _tdtype(cfg), cfg.rows * cfg.cols, "x", dev), _stream_on(dev, stream)), "slicemoe_mx_dequantize")


def quantize_mx(t, bits=4, transposed=False) -> torch.Tensor:
    """The packed matrix of a 2-d tensor (of its transpose: a weight stored [in, out]), on its device."""
    rows, cols = (t.shape[1], t.shape[0]) if transposed else t.shape
    cfg = make_mx_config(rows, cols, bits, t.dtype, transposed)
    mx = torch.empty(slicemoe_mx_bytes(cfg), dtype=torch.uint8, device=t.device)
    slicemoe_mx_quantize(cfg, t, mx)
    return mx


def slicemoe_mx_product_workspace_bytes(cfg) -> int:
    return lib().slicemoe_mx_product_workspace_bytes(ctypes.byref(cfg))


def slicemoe_mx_product(cfg, x_mx, w_mx, y, workspace=None, addend=None, stream=None):
    dt, n, dev = _tdtype(cfg), cfg.T * cfg.N, _device()
    wsp, wsb = _ws(workspace, dev)
    st = (_lib or lib()).slicemoe_mx_product(ctypes.byref(cfg), _mx_ptr(x_mx, cfg.T, cfg.K, cfg.bits, "x_mx", dev), _mx_ptr(w_mx, cfg.N, cfg.K, 4, "w_mx", dev),
                                             _ptr(addend, dt, n, "addend", dev), _ptr(y, dt, n, "y", dev), wsp, wsb, _stream_on(dev, stream))
    if st:
        _check(st, "slicemoe_mx_product")


def slicemoe_gated_ffn_mx_workspace_bytes(cfg, bits) -> int:
    return lib().slicemoe_gated_ffn_mx_workspace_bytes(ctypes.byref(cfg), bits)


def slicemoe_gated_ffn_mx(cfg, bits, x_mx, w, y, workspace, addend=None, stream=None):
    """w: dict of packed Wg, Wu (H rows of d columns) and Wd (d rows of H columns), see quantize_gated_weights_mx."""
    dt, n, dev, d, H = _tdtype(cfg), cfg.T * cfg.d, _device(), cfg.d, cfg.H
    wsp, wsb = _ws(workspace, dev)
    ws = slicemoe_gated_weights_mx(_mx_ptr(w["Wg"], H, d, 4, "Wg", dev), _mx_ptr(w["Wu"], H, d, 4, "Wu", dev), _mx_ptr(w["Wd"], d, H, 4, "Wd", dev))
    st = (_lib or lib()).slicemoe_gated_ffn_mx(ctypes.byref(cfg), bits, _mx_ptr(x_mx, cfg.T, d, bits, "x_mx", dev), ctypes.byref(ws),
                                               _ptr(addend, dt, n, "addend", dev), _ptr(y, dt, n, "y", dev), wsp, wsb, _stream_on(dev, stream))
    if st:
        _check(st, "slicemoe_gated_ffn_mx")


def quantize_gated_weights_mx(w: dict) -> dict:
    """The weight dict that slicemoe_gated_ffn_mx takes, from Wg, Wu [d, H] and Wd [H, d]."""
    return {n: quantize_mx(w[n], 4, transposed=True) for n in ("Wg", "Wu", "Wd")}


# ------------------------------------------------------------------ plumbing helpers (device memory only)
def to_device(arr, dtype: str, device="cuda:0") -> torch.Tensor:
    """Host fp32 array holding storage-representable values -> device tensor of the storage dtype."""
    t = torch.from_numpy(arr).to(device)
    return t.to(torch.bfloat16) if dtype == "bf16" else t


def weights_to_device(weights: dict, dtype: str, device="cuda:0") -> dict:
    return {n: to_device(a, dtype, device).contiguous() for n, a in weights.items()}


def alloc_workspace(cfg, device="cuda:0") -> torch.Tensor:
    n = slicemoe_workspace_bytes(cfg)
    if n == 0:
        raise SliceMoEError(SLICEMOE_ERR_UNSUPPORTED, "slicemoe_workspace_bytes returned 0 (invalid or unsupported config)")
    return torch.empty(n, dtype=torch.uint8, device=device)


def pack(cfg, w: dict, device="cuda:0") -> dict:
    """Return a copy of the weight dict with the 'packed' buffer added (no-op on generic configs)."""
    n = slicemoe_packed_bytes(cfg)
    out = dict(w)
    if n > 0:
        buf = torch.empty(n, dtype=torch.uint8, device=device)
        slicemoe_pack_weights(cfg, w, buf)
        out["packed"] = buf
    return out


def workspace_views(cfg, workspace: torch.Tensor) -> dict:
    """Typed views of the intermediates slicemoe_forward left in its workspace."""
    L = slicemoe_get_workspace_layout(cfg)
    Na = cfg.T * cfg.S * cfg.k
    ds = cfg.d // cfg.S

    def view(off, n, dt):
        return workspace[off:off + n * torch.empty(0, dtype=dt).element_size()].view(dt)

    return {
        "topk_idx": view(L.topk_idx, Na, torch.int32).view(-1, cfg.k),
        "topk_p": view(L.topk_p, Na, torch.float32).view(-1, cfg.k),
        "counts_raw": view(L.counts_raw, cfg.E, torch.int32),
        "counts": view(L.counts, cfg.E, torch.int32),
        "offsets": view(L.offsets, cfg.E + 1, torch.int32),
        "perm": view(L.perm, Na, torch.int32),
        "inv": view(L.inv, Na, torch.int32),
        "y": view(L.y, Na * ds, y_dtype(cfg)).view(-1, ds),
        "stats": view(L.stats, 4, torch.float32),
    }
