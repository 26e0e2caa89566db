"""Python binding of libcnn (include/cnn.h): argument marshalling only.

Every function here checks that its tensors are contiguous float32 CUDA
(ROCm) tensors (those of the sections on mixtures of experts and on the norm,
8-bit floats and sampling: contiguous, on one GPU, of the types and shapes they
state), passes their device pointers and the current torch stream to
the C entry point of the same name, and raises ``CnnError`` with
``cnn_last_error()`` on a non-OK status.  All computation happens in the HIP
kernels of libcnn; torch provides device memory and the stream.  Importing
this module fails if libcnn.so has not been built.
"""
from __future__ import annotations

import contextlib
import ctypes
import functools
import os
from dataclasses import dataclass
from typing import Dict, List, Optional, Sequence, Tuple

import torch

from . import workloads as _wl

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libcnn.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it with `python __graft_entry__.py` "
                      "(or paper_1511_07376_amd/build.py) before using the GPU path")

lib = ctypes.CDLL(LIB_PATH)

_i = ctypes.c_int
_p = ctypes.c_void_p
_ip = ctypes.POINTER(ctypes.c_int)

CNN_OK, CNN_ERR_INVALID, CNN_ERR_UNSUPPORTED, CNN_ERR_HIP, CNN_ERR_WORKSPACE = 0, -1, -2, -3, -4
CNN_POOL_MAX, CNN_POOL_AVG = 0, 1
CNN_LAYER_CONV, CNN_LAYER_FC, CNN_LAYER_POOL, CNN_LAYER_LRN, CNN_LAYER_RELU = 0, 1, 2, 3, 4
CNN_LAYER_SOFTMAX = 5
CNN_F32, CNN_BF16, CNN_F16, CNN_MX4, CNN_F8 = 0, 1, 2, 3, 4


class cnn_layer_desc(ctypes.Structure):
    _fields_ = [
        ("type", ctypes.c_int32), ("out_channels", ctypes.c_int32),
        ("kernel_h", ctypes.c_int32), ("kernel_w", ctypes.c_int32),
        ("stride_h", ctypes.c_int32), ("stride_w", ctypes.c_int32),
        ("pad_h", ctypes.c_int32), ("pad_w", ctypes.c_int32),
        ("groups", ctypes.c_int32), ("pool_mode", ctypes.c_int32),
        ("ceil_mode", ctypes.c_int32), ("fuse_relu", ctypes.c_int32),
        ("lrn_size", ctypes.c_int32), ("lrn_alpha", ctypes.c_float),
        ("lrn_beta", ctypes.c_float), ("lrn_k", ctypes.c_float),
        ("in_channels", ctypes.c_int32), ("in_features", ctypes.c_int32),
        ("weight", ctypes.c_void_p), ("bias", ctypes.c_void_p), ("pool_index", ctypes.c_void_p),
    ]


lib.cnn_conv2d_out_shape.argtypes = [_i] * 8 + [_ip, _ip]
lib.cnn_pool_out_shape.argtypes = [_i] * 9 + [_ip, _ip]
lib.cnn_conv2d_fwd.argtypes = [_p, _i, _i, _i, _i, _p, _i, _i, _i, _p, _i, _i, _i, _i, _i, _i, _p, _p]
lib.cnn_fc_fwd.argtypes = [_p, _i, _i, _p, _p, _i, _i, _p, _p]
lib.cnn_pool_fwd.argtypes = [_p, _i, _i, _i, _i, _i, _i, _i, _i, _i, _i, _i, _i, _i, _p, _p, _p]
lib.cnn_lrn_fwd.argtypes = [_p, _i, _i, _i, _i, _i, ctypes.c_float, ctypes.c_float, ctypes.c_float,
                            _p, _p]
lib.cnn_relu_fwd.argtypes = [_p, _p, ctypes.c_int64, _p]
lib.cnn_softmax_fwd.argtypes = [_p, _i, _i, _i, _p, _p]
lib.cnn_mx4_quantize.argtypes = [_p, _i, _i, _i, _p, _p, _p]
lib.cnn_mx4_dequantize.argtypes = [_p, _p, _i, _i, _p, _i, _p]
lib.cnn_fc_mx4_fwd.argtypes = [_p, _p, _i, _i, _i, _p, _p, _p, _i, _i, _p, _i, _p, ctypes.c_size_t, _p]
lib.cnn_fc_mx4_workspace_bytes.argtypes = [_i] * 4
lib.cnn_fc_mx4_workspace_bytes.restype = ctypes.c_size_t
lib.cnn_fc_grouped_fwd.argtypes = [_p, _p, _i, _i, _i, _p, _i, _p, _i, _p, _p, _i, _p, _i, _i, _p, _i, _p,
                                   ctypes.c_size_t, _p]
lib.cnn_fc_grouped_workspace_bytes.argtypes = [_i] * 6
lib.cnn_fc_grouped_workspace_bytes.restype = ctypes.c_size_t
lib.cnn_route_workspace_bytes.argtypes = [_i, _i, _i]
lib.cnn_route_workspace_bytes.restype = ctypes.c_size_t
lib.cnn_route_fwd.argtypes = [_p, _i, _i, _i, _i, _i, _p, _p, _p, _p, _p, _p, ctypes.c_size_t, _p]
lib.cnn_combine_fwd.argtypes = [_p, _i, _i, _i, _p, _p, _i, _i, _p, _p]
lib.cnn_f8_quantize.argtypes = [_p, _i, _i, _i, _i, _p, _p, _p]
lib.cnn_f8_dequantize.argtypes = [_p, _p, _i, _i, _i, _p, _i, _p]
lib.cnn_rms_norm_fwd.argtypes = [_p, _p, _i, _i, _i, _p, ctypes.c_float, _p, _p, _i, _p, _p]
lib.cnn_fc_f8_fwd.argtypes = [_p, _p, _i, _i, _p, _p, _p, _i, _i, _p, _i, _p, ctypes.c_size_t, _p]
lib.cnn_fc_f8_workspace_bytes.argtypes = [_i, _i, _i]
lib.cnn_fc_f8_workspace_bytes.restype = ctypes.c_size_t
lib.cnn_sample_fwd.argtypes = [_p, _i, _i, _i, _p, _p, _p, _p, _p, _p, _p, _p, ctypes.c_size_t, _p]
lib.cnn_sample_workspace_bytes.argtypes = [_i, _i, _i]
lib.cnn_sample_workspace_bytes.restype = ctypes.c_size_t


class cnn_netfile_config(ctypes.Structure):
    _fields_ = [("in_channels", ctypes.c_int32), ("in_height", ctypes.c_int32),
                ("in_width", ctypes.c_int32), ("execution_mode", ctypes.c_int32),
                ("auto_tuning", ctypes.c_int32), ("allocated_ram_mib", ctypes.c_int32)]


CNN_EXEC_PARALLEL, CNN_EXEC_GRAPH = 0, 1
_descp = ctypes.POINTER(cnn_layer_desc)
lib.cnn_net_out_shape.argtypes = [_descp, _i, _i, _i, _i, _i, _ip, _ip, _ip]
lib.cnn_net_workspace_bytes.argtypes = [_descp, _i, _i, _i, _i, _i]
lib.cnn_net_workspace_bytes.restype = ctypes.c_size_t
lib.cnn_net_fwd.argtypes = [_descp, _i, _p, _i, _i, _i, _i, _p, _p, ctypes.c_size_t, _p]
lib.cnn_net_fwd_timed.argtypes = [_descp, _i, _p, _i, _i, _i, _i, _p, _p, ctypes.c_size_t,
                                  ctypes.POINTER(ctypes.c_void_p), _p]
lib.cnn_net_fwd_kernel_timed.argtypes = [_descp, _i, _p, _i, _i, _i, _i, _p, _p, ctypes.c_size_t,
                                         ctypes.POINTER(ctypes.c_void_p), ctypes.POINTER(ctypes.c_void_p), _p]
lib.cnn_net_fwd_dump.argtypes = [_descp, _i, _p, _i, _i, _i, _i, _p, _p, ctypes.c_size_t,
                                 ctypes.POINTER(ctypes.c_void_p), _ip, _p]
lib.cnn_net_fwd_noalloc.argtypes = [_descp, _i, _p, _i, _i, _i, _i, _p, _p]
CNN_NOALLOC_SCRATCH_BYTES = 256 << 20
lib.cnn_conv2d_fwd_config.argtypes = lib.cnn_conv2d_fwd.argtypes[:17] + [_i, _p]
lib.cnn_netfile_parse.argtypes = [ctypes.c_char_p, _descp, _i, _ip, ctypes.POINTER(cnn_netfile_config)]
lib.cnn_net_graph_create.argtypes = [_descp, _i, _p, _i, _i, _i, _i, _p, _p, ctypes.c_size_t,
                                     ctypes.POINTER(ctypes.c_void_p)]
lib.cnn_net_graph_launch.argtypes = [_p, _p]
lib.cnn_net_graph_destroy.argtypes = [_p]
lib.cnn_conv2d_num_configs.argtypes = []
lib.cnn_conv2d_config_name.argtypes = [_i]
lib.cnn_conv2d_config_name.restype = ctypes.c_char_p
lib.cnn_fc_fwd_config.argtypes = lib.cnn_fc_fwd.argtypes[:8] + [_i, _p]
lib.cnn_fc_num_configs.argtypes = []
lib.cnn_fc_config_name.argtypes = [_i]
lib.cnn_fc_config_name.restype = ctypes.c_char_p
lib.cnn_set_autotune.argtypes = [_i]
lib.cnn_tuning_export.argtypes = [ctypes.c_char_p, ctypes.c_size_t]
lib.cnn_tuning_export.restype = ctypes.c_size_t
lib.cnn_tuning_import.argtypes = [ctypes.c_char_p]
lib.cnn_tuning_clear.argtypes = []
lib.cnn_last_error.restype = ctypes.c_char_p
lib.cnn_version.restype = ctypes.c_char_p
for _name in ("cnn_conv2d_out_shape", "cnn_pool_out_shape", "cnn_conv2d_fwd", "cnn_fc_fwd",
              "cnn_pool_fwd", "cnn_lrn_fwd", "cnn_relu_fwd", "cnn_softmax_fwd", "cnn_net_out_shape",
              "cnn_mx4_quantize", "cnn_mx4_dequantize", "cnn_fc_mx4_fwd", "cnn_fc_grouped_fwd",
              "cnn_route_fwd", "cnn_combine_fwd",
              "cnn_f8_quantize", "cnn_f8_dequantize", "cnn_rms_norm_fwd", "cnn_fc_f8_fwd", "cnn_sample_fwd",
              "cnn_net_fwd",
              "cnn_net_fwd_timed", "cnn_net_fwd_kernel_timed", "cnn_net_fwd_dump", "cnn_net_fwd_noalloc",
              "cnn_conv2d_fwd_config",
              "cnn_conv2d_num_configs", "cnn_fc_fwd_config", "cnn_fc_num_configs",
              "cnn_set_autotune", "cnn_tuning_import", "cnn_tuning_clear", "cnn_netfile_parse",
              "cnn_net_graph_create", "cnn_net_graph_launch", "cnn_net_graph_destroy"):
    getattr(lib, _name).restype = _i

EXPORTED = ("cnn_conv2d_out_shape", "cnn_pool_out_shape", "cnn_conv2d_fwd", "cnn_fc_fwd",
            "cnn_pool_fwd", "cnn_lrn_fwd", "cnn_relu_fwd", "cnn_softmax_fwd", "cnn_net_out_shape",
            "cnn_mx4_quantize", "cnn_mx4_dequantize", "cnn_fc_mx4_fwd", "cnn_fc_grouped_fwd",
            "cnn_fc_mx4_workspace_bytes", "cnn_fc_grouped_workspace_bytes",
            "cnn_route_workspace_bytes", "cnn_route_fwd", "cnn_combine_fwd",
            "cnn_f8_quantize", "cnn_f8_dequantize", "cnn_rms_norm_fwd", "cnn_fc_f8_fwd",
            "cnn_fc_f8_workspace_bytes", "cnn_sample_fwd", "cnn_sample_workspace_bytes",
            "cnn_net_workspace_bytes", "cnn_net_fwd", "cnn_net_fwd_timed", "cnn_net_fwd_kernel_timed",
            "cnn_net_fwd_dump",
            "cnn_net_fwd_noalloc", "cnn_last_error",
            "cnn_version", "cnn_conv2d_num_configs", "cnn_conv2d_config_name",
            "cnn_conv2d_fwd_config", "cnn_fc_num_configs", "cnn_fc_config_name", "cnn_fc_fwd_config",
            "cnn_set_autotune", "cnn_tuning_export",
            "cnn_tuning_import", "cnn_tuning_clear", "cnn_netfile_parse", "cnn_net_graph_create",
            "cnn_net_graph_launch", "cnn_net_graph_destroy")


class CnnError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"libcnn status {status}: {message}")
        self.status = status


def cnn_last_error() -> str:
    # the message may quote the caller's text (a NetFile line), which need not be UTF-8
    return lib.cnn_last_error().decode(errors="replace")


def cnn_version() -> str:
    return lib.cnn_version().decode()


def _ok(rc: int) -> None:
    if rc != CNN_OK:
        raise CnnError(rc, cnn_last_error())


def _dev(t: Optional[torch.Tensor], name: str, dtype=torch.float32):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise TypeError(f"{name} must be contiguous")
    return t.data_ptr()


def _stream(stream) -> int:
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def _pair(v) -> Tuple[int, int]:
    return (int(v), int(v)) if isinstance(v, int) else (int(v[0]), int(v[1]))


def cnn_conv2d_out_shape(H, W, R, S, stride=1, pad=0) -> Tuple[int, int]:
    sh, sw = _pair(stride)
    ph, pw = _pair(pad)
    P, Q = ctypes.c_int(), ctypes.c_int()
    _ok(lib.cnn_conv2d_out_shape(H, W, R, S, sh, sw, ph, pw, ctypes.byref(P), ctypes.byref(Q)))
    return P.value, Q.value


def cnn_pool_out_shape(H, W, kernel, stride, pad=0, ceil_mode=True) -> Tuple[int, int]:
    kh, kw = _pair(kernel)
    sh, sw = _pair(stride)
    ph, pw = _pair(pad)
    P, Q = ctypes.c_int(), ctypes.c_int()
    _ok(lib.cnn_pool_out_shape(H, W, kh, kw, sh, sw, ph, pw, int(ceil_mode), ctypes.byref(P),
                               ctypes.byref(Q)))
    return P.value, Q.value


def cnn_conv2d_fwd(x, w, bias=None, stride=1, pad=0, groups=1, fuse_relu=False, y=None, stream=None,
                   config=None):
    """x [N][C][H][W], w [K][C/G][R][S], bias [K] -> y [N][K][P][Q] (allocated if None).

    config=None uses the tuned / heuristic tile configuration (cnn_conv2d_fwd);
    an int calls cnn_conv2d_fwd_config with that configuration (-1: heuristic)."""
    N, C, H, W = x.shape
    K, _cg, R, S = w.shape
    sh, sw = _pair(stride)
    ph, pw = _pair(pad)
    if y is None:
        P, Q = cnn_conv2d_out_shape(H, W, R, S, (sh, sw), (ph, pw))
        y = torch.empty((N, K, P, Q), dtype=torch.float32, device=x.device)
    args = (_dev(x, "x"), N, C, H, W, _dev(w, "w"), K, R, S, _dev(bias, "bias"),
            sh, sw, ph, pw, groups, int(fuse_relu), _dev(y, "y"))
    if config is None:
        _ok(lib.cnn_conv2d_fwd(*args, _stream(stream)))
    else:
        _ok(lib.cnn_conv2d_fwd_config(*args, int(config), _stream(stream)))
    return y


def cnn_conv2d_num_configs() -> int:
    return int(lib.cnn_conv2d_num_configs())


def cnn_conv2d_config_name(i: int) -> Optional[str]:
    r = lib.cnn_conv2d_config_name(int(i))
    return None if r is None else r.decode()


def cnn_set_autotune(on: bool) -> None:
    _ok(lib.cnn_set_autotune(int(bool(on))))


def cnn_tuning_export() -> str:
    n = lib.cnn_tuning_export(None, 0)
    buf = ctypes.create_string_buffer(n)
    lib.cnn_tuning_export(buf, n)
    return buf.value.decode()


def cnn_tuning_import(text: str) -> int:
    rc = lib.cnn_tuning_import(text.encode())
    if rc < 0:
        raise CnnError(rc, cnn_last_error())
    return rc


def cnn_tuning_clear() -> None:
    _ok(lib.cnn_tuning_clear())


def cnn_fc_fwd(x, w, bias=None, fuse_relu=False, y=None, stream=None, config=None):
    """x [N][I] (or [N][C][H][W], read flattened), w [O][I] -> y [N][O].

    config=None calls cnn_fc_fwd (the built-in kernel choice); an int calls
    cnn_fc_fwd_config with that configuration (-1: the built-in choice)."""
    N = x.shape[0]
    I = x.numel() // max(N, 1) if N else int(w.shape[1])
    O = w.shape[0]
    if y is None:
        y = torch.empty((N, O), dtype=torch.float32, device=x.device)
    args = (_dev(x, "x"), N, I, _dev(w, "w"), _dev(bias, "bias"), O, int(fuse_relu), _dev(y, "y"))
    if config is None:
        _ok(lib.cnn_fc_fwd(*args, _stream(stream)))
    else:
        _ok(lib.cnn_fc_fwd_config(*args, int(config), _stream(stream)))
    return y


def cnn_fc_num_configs() -> int:
    return int(lib.cnn_fc_num_configs())


def cnn_fc_config_name(i: int) -> Optional[str]:
    r = lib.cnn_fc_config_name(int(i))
    return None if r is None else r.decode()


def cnn_pool_fwd(x, mode="max", kernel=2, stride=2, pad=0, ceil_mode=True, fuse_relu=False,
                 with_index=False, y=None, idx=None, stream=None):
    """Returns y, or (y, idx) for max pooling with with_index."""
    N, C, H, W = x.shape
    kh, kw = _pair(kernel)
    sh, sw = _pair(stride)
    ph, pw = _pair(pad)
    m = {"max": CNN_POOL_MAX, "avg": CNN_POOL_AVG}[mode] if isinstance(mode, str) else int(mode)
    P, Q = cnn_pool_out_shape(H, W, (kh, kw), (sh, sw), (ph, pw), ceil_mode)
    if y is None:
        y = torch.empty((N, C, P, Q), dtype=torch.float32, device=x.device)
    if with_index and idx is None:
        idx = torch.empty((N, C, P, Q), dtype=torch.int32, device=x.device)
    _ok(lib.cnn_pool_fwd(_dev(x, "x"), N, C, H, W, m, kh, kw, sh, sw, ph, pw, int(ceil_mode),
                         int(fuse_relu), _dev(y, "y"), _dev(idx, "idx", torch.int32), _stream(stream)))
    return (y, idx) if idx is not None else y


def cnn_lrn_fwd(x, size=5, alpha=1e-4, beta=0.75, k=1.0, y=None, stream=None):
    N, C, H, W = x.shape
    if y is None:
        y = torch.empty_like(x)
    _ok(lib.cnn_lrn_fwd(_dev(x, "x"), N, C, H, W, size, alpha, beta, k, _dev(y, "y"), _stream(stream)))
    return y


def cnn_relu_fwd(x, y=None, stream=None):
    """y = max(x, 0); pass y=x for in place."""
    if y is None:
        y = torch.empty_like(x)
    if y.numel() != x.numel():
        raise ValueError("relu: x and y differ in size")
    _ok(lib.cnn_relu_fwd(_dev(x, "x"), _dev(y, "y"), x.numel(), _stream(stream)))
    return y


def cnn_softmax_fwd(x, y=None, stream=None):
    """Softmax across dim 1 of an [N][C] or [N][C][H][W] tensor; pass y=x for
    in place."""
    if x.dim() < 2:
        raise ValueError("softmax: x must be [N][C...]")
    if y is None:
        y = torch.empty_like(x)
    if y.numel() != x.numel():
        raise ValueError("softmax: x and y differ in size")
    N, C = x.shape[0], x.shape[1]
    HW = 1
    for d in x.shape[2:]:
        HW *= d
    _ok(lib.cnn_softmax_fwd(_dev(x, "x"), N, C, HW, _dev(y, "y"), _stream(stream)))
    return y


# ---------------------------------------------------------------- experts, 4-bit weights
_WIDE = {torch.float32: CNN_F32, torch.bfloat16: CNN_BF16, torch.float16: CNN_F16}


_INT_MAX = 0x7fffffff


def _on(t, name: str, device: torch.device, dtype=None, shape=None):
    """Device pointer of a contiguous tensor on `device`, of this type and shape where given; None for None."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.device != device:
        raise TypeError(f"{name} must be a tensor on {device}")
    if dtype is not None and t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise TypeError(f"{name} must be contiguous")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
    return t.data_ptr()


def _wide(dtype, name: str) -> int:
    code = _WIDE.get(dtype)
    if code is None:
        raise TypeError(f"{name} must be float32, bfloat16 or float16, got {dtype}")
    return code


def _gpu(t, name: str) -> torch.device:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    if t.numel() > _INT_MAX:
        _too_large(name)
    return t.device


def _too_large(name: str):
    """Sizes are passed as int: none is cut to one that fits."""
    raise CnnError(CNN_ERR_UNSUPPORTED, f"{name}: a size above 2^31-1")


# what a workspace takes is a matter of sizes and types alone
_fc_mx4_workspace = functools.lru_cache(maxsize=4096)(lib.cnn_fc_mx4_workspace_bytes)
_fc_grouped_workspace = functools.lru_cache(maxsize=4096)(lib.cnn_fc_grouped_workspace_bytes)


# the current GPU and stream as numbers, in a tenth of torch.cuda.current_stream()'s time
_current_gpu, _raw_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream


@contextlib.contextmanager
def _there(device, stream):
    """Makes the tensors' GPU and the call's stream current, for its kernels and the tensors it allocates."""
    with torch.cuda.device(device):
        if stream is None:
            yield
            return
        if not isinstance(stream, torch.cuda.Stream):
            handle = int(stream)
            stream = (torch.cuda.ExternalStream(handle, device=device) if handle
                      else torch.cuda.default_stream(device))
        if stream.device != device:
            raise ValueError(f"the stream is of {stream.device}, the tensors are on {device}")
        with torch.cuda.stream(stream):
            yield


def cnn_mx4_quantize(x, q=None, scale=None, stream=None):
    """x [rows][cols] -> (q uint8 [rows][ceil(cols/32)*16], scale uint8 [rows][ceil(cols/32)]): mx4 (CNN_MX4).

    Leading dimensions are kept: x [G][O][I] gives q [G][O][...]."""
    device = _gpu(x, "x")
    if stream is not None or device.index != _current_gpu():
        with _there(device, stream):
            return cnn_mx4_quantize(x, q, scale)
    if x.dim() < 2:
        raise ValueError("mx4_quantize: x must be [rows][cols]")
    lead, cols = tuple(x.shape[:-1]), x.shape[-1]
    rows = 1
    for d in lead:
        rows *= d
    blocks = (cols + 31) // 32
    code = _wide(x.dtype, "x")
    xp = _on(x, "x", device)
    st = _raw_stream(device.index)
    if q is None:
        q = torch.empty(lead + (blocks * 16,), dtype=torch.uint8, device=device)
        qp = q.data_ptr()
    else:
        qp = _on(q, "q", device, torch.uint8, lead + (blocks * 16,))
    if scale is None:
        scale = torch.empty(lead + (blocks,), dtype=torch.uint8, device=device)
        scalep = scale.data_ptr()
    else:
        scalep = _on(scale, "scale", device, torch.uint8, lead + (blocks,))
    _ok(lib.cnn_mx4_quantize(xp, code, rows, cols, qp,
                             scalep, st))
    return q, scale


def cnn_mx4_dequantize(q, scale, cols=None, dtype=None, y=None, stream=None):
    """The values of mx4 rows, [...][cols] (cols: 32 a block if not given), of type dtype (y's, or float32, if not
    given)."""
    device = _gpu(q, "q")
    if stream is not None or device.index != _current_gpu():
        with _there(device, stream):
            return cnn_mx4_dequantize(q, scale, cols, dtype, y)
    blocks = scale.shape[-1]
    cols = 32 * blocks if cols is None else int(cols)
    if not 32 * (blocks - 1) < cols <= 32 * blocks:
        raise ValueError(f"mx4_dequantize: {cols} columns in {blocks} blocks")
    lead = tuple(scale.shape[:-1])
    rows = 1
    for d in lead:
        rows *= d
    qp = _on(q, "q", device, torch.uint8, lead + (blocks * 16,))
    sp = _on(scale, "scale", device, torch.uint8)
    st = _raw_stream(device.index)
    if y is None:
        y = torch.empty(lead + (cols,), dtype=dtype or torch.float32, device=device)
        yp = y.data_ptr()
    else:
        yp = _on(y, "y", device, dtype, lead + (cols,))
    _ok(lib.cnn_mx4_dequantize(qp, sp, rows, cols, yp,
                               _wide(y.dtype, "y"), st))
    return y


def _operand(x, x_scale, device, name: str):
    """(pointer, scale pointer, type, rows, columns as far as the tensors say) of rows that may be mx4."""
    if x_scale is None:
        return _on(x, name, device), None, _wide(x.dtype, name), x.shape[-1]
    blocks = x_scale.shape[-1]
    return (_on(x, name, device, torch.uint8, tuple(x_scale.shape[:-1]) + (blocks * 16,)),
            _on(x_scale, name + "_scale", device, torch.uint8), CNN_MX4, 32 * blocks)


def _columns(x_type: int, x_cols: int, w_type: int, w_cols: int, what: str) -> int:
    """The length of the reduction: that of x, or whole blocks where both are mx4."""
    fits = x_cols == w_cols if (x_type == CNN_MX4) == (w_type == CNN_MX4) else w_cols - 32 < x_cols <= w_cols
    if not fits:
        raise ValueError(f"{what}: x has {x_cols} columns, w {w_cols}")
    return x_cols


def _result_type(x, xs, y_dtype):
    """The type of a product's result: that of wide inputs; of mx4 ones the asked one, float32 if none."""
    if xs is not None:
        return y_dtype or torch.float32
    if y_dtype is not None and y_dtype is not x.dtype:
        raise TypeError(f"y_dtype must be {x.dtype}, the type of x, got {y_dtype}")
    return x.dtype


def cnn_fc_mx4_fwd(x, w, w_scale, bias=None, fuse_relu=False, x_scale=None, y_dtype=None, y=None, stream=None):
    """x [N][I] (or [N][C][H][W], read flattened), w and w_scale mx4 of [O][I] -> y [N][O], of x's type.

    With x_scale x is mx4 too, and y of type y_dtype (float32 if not given)."""
    device = _gpu(x, "x")
    if stream is not None or device.index != _current_gpu():
        with _there(device, stream):
            return cnn_fc_mx4_fwd(x, w, w_scale, bias, fuse_relu, x_scale, y_dtype, y)
    if x_scale is None and x.dim() > 2:
        x = x.flatten(1) if x.is_contiguous() else x
    if x.dim() != 2 or w.dim() != 2 or w_scale.dim() != 2:
        raise ValueError("fc_mx4: x, w and w_scale must have two dimensions")
    xp, xs, xt, xc = _operand(x, x_scale, device, "x")
    wp, ws, wt, wc = _operand(w, w_scale, device, "w")
    cols = _columns(xt, xc, wt, wc, "fc_mx4")
    N, O = x.shape[0], w.shape[0]
    if O > _INT_MAX or cols > _INT_MAX:
        _too_large("fc_mx4")
    bp = _on(bias, "bias", device, torch.float32, (O,))
    dtype = _result_type(x, xs, y_dtype)
    st = _raw_stream(device.index)
    if y is None:
        y = torch.empty((N, O), dtype=dtype, device=device)
        yp = y.data_ptr()
    else:
        yp = _on(y, "y", device, dtype, (N, O))
    need = _fc_mx4_workspace(xt, N, cols, O)
    work = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    _ok(lib.cnn_fc_mx4_fwd(xp, xs, xt, N, cols, wp, ws, bp, O, 1 if fuse_relu else 0,
                           yp, _WIDE.get(dtype, -1),
                           work.data_ptr() if need else None, need, st))
    return y


def cnn_fc_grouped_fwd(x, w, offsets, bias=None, fuse_relu=False, rows=None, w_scale=None, x_scale=None,
                       y_dtype=None, y=None, stream=None):
    """x [N][I], w [G][O][I], offsets int32 [G+1] -> y [M][O], of x's type: row m of y is row rows[m] (int32 [M];
    row m if not given) of x through the weights of the group with offsets[g] <= m < offsets[g+1].

    With w_scale [G][O][blocks] w is mx4; with x_scale x is too, and y of type y_dtype (float32 if not given).
    Rows of y in no group are not written."""
    device = _gpu(x, "x")
    if stream is not None or device.index != _current_gpu():
        with _there(device, stream):
            return cnn_fc_grouped_fwd(x, w, offsets, bias, fuse_relu, rows, w_scale, x_scale, y_dtype, y)
    if x.dim() != 2 or w.dim() != 3:
        raise ValueError("fc_grouped: x must be [N][I], w [G][O][I]")
    xp, xs, xt, xc = _operand(x, x_scale, device, "x")
    wp, ws, wt, wc = _operand(w, w_scale, device, "w")
    cols = _columns(xt, xc, wt, wc, "fc_grouped")
    N, (G, O) = x.shape[0], w.shape[:2]
    M = N if rows is None else rows.numel()
    if max(M, G, O, cols) > _INT_MAX:
        _too_large("fc_grouped")
    bp = _on(bias, "bias", device, torch.float32, (G, O))
    op = _on(offsets, "offsets", device, torch.int32, (G + 1,))
    rp = _on(rows, "rows", device, torch.int32)
    dtype = _result_type(x, xs, y_dtype)
    st = _raw_stream(device.index)
    if y is None:
        y = torch.empty((M, O), dtype=dtype, device=device)
        yp = y.data_ptr()
    else:
        yp = _on(y, "y", device, dtype, (M, O))
    need = _fc_grouped_workspace(xt, cols, M, G, wt, O)
    work = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    _ok(lib.cnn_fc_grouped_fwd(xp, xs, xt, N, cols, rp, M, op, G, wp, ws, wt, bp, O, 1 if fuse_relu else 0,
                               yp, _WIDE.get(dtype, -1),
                               work.data_ptr() if need else None, need, st))
    return y


def cnn_route_fwd(logits, k, renormalize=False, stream=None):
    """logits [T][E] -> (expert int32 [T][k], weight float32 [T][k], rows int32 [T*k], offsets int32 [E+1],
    slot int32 [T][k]): each token's k experts and their weights, and the rows for cnn_fc_grouped_fwd.

    The five are parts of one allocation: it lives as long as any of them (clone what is to be kept alone), and
    autograd takes a write in place to one as a write to all."""
    device = _gpu(logits, "logits")
    if stream is not None or device.index != _current_gpu():
        with _there(device, stream):
            return cnn_route_fwd(logits, k, renormalize)
    if logits.dim() != 2:
        raise ValueError("route: logits must be [T][E]")
    T, E = logits.shape
    k = int(k)
    if max(T, E, abs(k)) > _INT_MAX:
        _too_large("route")
    code = _wide(logits.dtype, "logits")
    lp = _on(logits, "logits", device)
    need = lib.cnn_route_workspace_bytes(T, E, k)
    st = _raw_stream(device.index)
    n = T * k
    if k <= 0 or n > _INT_MAX:
        _ok(lib.cnn_route_fwd(None, code, T, E, k, 0, None, None, None, None, None, None, 0, None))  # says why not
        _too_large("route")
    # one allocation: what is handed out are parts of it
    parts = torch.empty(4 * n + E + 1, dtype=torch.int32, device=device)
    expert, slot, rows, weight, offsets = parts.split_with_sizes((n, n, n, n, E + 1))
    base = parts.data_ptr()
    ws = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    _ok(lib.cnn_route_fwd(lp, code, T, E, k, 1 if renormalize else 0, base, base + 12 * n, base + 8 * n,
                          base + 16 * n, base + 4 * n, ws.data_ptr() if need else None, need, st))
    expert, slot, weight = expert.view(T, k), slot.view(T, k), weight.view(torch.float32).view(T, k)
    return expert, weight, rows, offsets, slot


def cnn_combine_fwd(x, slot, weight, y=None, stream=None):
    """x [M][D], slot int32 [N][k], weight float32 [N][k] -> y [N][D] = sum over j of weight[n][j] * x[slot[n][j]]."""
    device = _gpu(x, "x")
    if stream is not None or device.index != _current_gpu():
        with _there(device, stream):
            return cnn_combine_fwd(x, slot, weight, y)
    if x.dim() != 2 or slot.dim() != 2:
        raise ValueError("combine: x must be [M][D], slot [N][k]")
    (M, D), (N, k) = x.shape, slot.shape
    if max(M, D, N, k) > _INT_MAX:
        _too_large("combine")
    code = _wide(x.dtype, "x")
    xp = _on(x, "x", device)
    sp = _on(slot, "slot", device, torch.int32)
    wp = _on(weight, "weight", device, torch.float32, (N, k))
    st = _raw_stream(device.index)
    if y is None:
        y = torch.empty((N, D), dtype=x.dtype, device=device)
        yp = y.data_ptr()
    else:
        yp = _on(y, "y", device, x.dtype, (N, D))
    _ok(lib.cnn_combine_fwd(xp, code, M, D, sp, wp, N, k, yp, st))
    return y


# ---------------------------------------------------------------- norm, 8-bit floats, sampling
_F8 = torch.float8_e4m3fn

_fc_f8_workspace = functools.lru_cache(maxsize=4096)(lib.cnn_fc_f8_workspace_bytes)
_sample_workspace = functools.lru_cache(maxsize=4096)(lib.cnn_sample_workspace_bytes)


def _f8_shapes(lead, cols: int, block_rows: int, what: str):
    """(rows, shape of the scales) of f8 rows [lead][cols]; blocks of 128 rows: of one matrix."""
    if block_rows not in (1, 128):
        raise ValueError(f"{what}: blocks of {block_rows} rows, not 1 or 128")
    if block_rows == 128 and len(lead) != 1:
        raise ValueError(f"{what}: blocks of 128 rows are those of a matrix [rows][cols]")
    rows = 1
    for d in lead:
        rows *= d
    blocks = (cols + 127) // 128
    return rows, (lead + (blocks,) if block_rows == 1 else ((rows + 127) // 128, blocks))


def cnn_f8_quantize(x, block_rows=1, q=None, scale=None, stream=None):
    """x [rows][cols] -> (q float8_e4m3fn [rows][cols], scale float32 [ceil(rows/block_rows)][ceil(cols/128)]): f8
    (CNN_F8), block_rows 1 for activations or 128 for weights.

    With block_rows 1 leading dimensions are kept: x [G][N][I] gives q [G][N][I] and scale [G][N][blocks]."""
    device = _gpu(x, "x")
    if stream is not None or device.index != _current_gpu():
        with _there(device, stream):
            return cnn_f8_quantize(x, block_rows, q, scale)
    if x.dim() < 2:
        raise ValueError("f8_quantize: x must be [rows][cols]")
    lead, cols = tuple(x.shape[:-1]), x.shape[-1]
    rows, scales = _f8_shapes(lead, cols, block_rows, "f8_quantize")
    if max(rows, cols) > _INT_MAX:
        _too_large("f8_quantize")
    code = _wide(x.dtype, "x")
    xp = _on(x, "x", device)
    st = _raw_stream(device.index)
    if q is None:
        q = torch.empty_like(x, dtype=_F8)  # of the ways to allocate the quickest: 1.5 us, torch.empty 2.6
        qp = q.data_ptr()
    else:
        qp = _on(q, "q", device, _F8, x.shape)
    if scale is None:
        scale = x.new_empty(scales, dtype=torch.float32)
        sp = scale.data_ptr()
    else:
        sp = _on(scale, "scale", device, torch.float32, scales)
    _ok(lib.cnn_f8_quantize(xp, code, rows, cols, block_rows, qp, sp, st))
    return q, scale


def cnn_f8_dequantize(q, scale, block_rows=1, dtype=None, y=None, stream=None):
    """The values of f8 rows, [...][cols], of type dtype (y's, or float32, if not given)."""
    device = _gpu(q, "q")
    if stream is not None or device.index != _current_gpu():
        with _there(device, stream):
            return cnn_f8_dequantize(q, scale, block_rows, dtype, y)
    if q.dim() < 2:
        raise ValueError("f8_dequantize: q must be [rows][cols]")
    lead, cols = tuple(q.shape[:-1]), q.shape[-1]
    rows, scales = _f8_shapes(lead, cols, block_rows, "f8_dequantize")
    if max(rows, cols) > _INT_MAX:
        _too_large("f8_dequantize")
    qp = _on(q, "q", device, _F8)
    sp = _on(scale, "scale", device, torch.float32, scales)
    st = _raw_stream(device.index)
    if y is None:
        y = torch.empty_like(q, dtype=dtype or torch.float32)
        yp = y.data_ptr()
    else:
        yp = _on(y, "y", device, dtype, q.shape)
    _ok(lib.cnn_f8_dequantize(qp, sp, rows, cols, block_rows, yp, _wide(y.dtype, "y"), st))
    return y


def cnn_rms_norm_fwd(x, weight=None, residual=None, eps=1e-6, f8=False, sum=None, y=None, y_scale=None, stream=None):
    """s = x + residual; y = s / sqrt(mean of s^2 over the last dimension + eps) * weight.

    x [...][cols], residual like it or None, weight float32 [cols] or None.  Returns y, of x's type; with f8 (y
    float8_e4m3fn, y_scale float32 [...][ceil(cols/128)]); with a residual s, rounded to x's type, as one more.  y and
    sum may each be x or residual (y not with f8), but not both the same one."""
    device = _gpu(x, "x")
    if stream is not None or device.index != _current_gpu():
        with _there(device, stream):
            return cnn_rms_norm_fwd(x, weight, residual, eps, f8, sum, y, y_scale)
    if x.dim() < 1:
        raise ValueError("rms_norm: x must be [...][cols]")
    shape = x.shape
    cols = shape[-1]
    if cols == 0:
        raise ValueError("rms_norm: rows of no values")
    rows = 1
    for d in shape[:-1]:
        rows *= d
    if max(rows, cols) > _INT_MAX:
        _too_large("rms_norm")
    code = _wide(x.dtype, "x")
    xp = _on(x, "x", device)
    rp = _on(residual, "residual", device, x.dtype, shape)
    wp = _on(weight, "weight", device, torch.float32, (cols,))
    st = _raw_stream(device.index)
    if sum is not None:
        if residual is None:
            raise ValueError("rms_norm: sum goes with a residual")
        sump = _on(sum, "sum", device, x.dtype, shape)
    elif residual is not None:
        sum = torch.empty_like(x)
        sump = sum.data_ptr()
    else:
        sump = None
    if y is None:
        y = torch.empty_like(x, dtype=_F8) if f8 else torch.empty_like(x)
        yp = y.data_ptr()
    else:
        yp = _on(y, "y", device, _F8 if f8 else x.dtype, shape)
    if f8:
        scales = shape[:-1] + ((cols + 127) // 128,)
        if y_scale is None:
            y_scale = x.new_empty(scales, dtype=torch.float32)
            yscalep = y_scale.data_ptr()
        else:
            yscalep = _on(y_scale, "y_scale", device, torch.float32, scales)
    elif y_scale is not None:
        raise ValueError("rms_norm: y_scale goes with f8")
    else:
        yscalep = None
    _ok(lib.cnn_rms_norm_fwd(xp, rp, code, rows, cols, wp, eps, sump, yp, CNN_F8 if f8 else code, yscalep, st))
    if f8:
        return (y, y_scale) if residual is None else (y, y_scale, sum)
    return y if residual is None else (y, sum)


def cnn_fc_f8_fwd(x, x_scale, w, w_scale, bias=None, fuse_relu=False, y_dtype=None, y=None, stream=None):
    """x float8_e4m3fn [N][I] with x_scale [N][ceil(I/128)], w float8_e4m3fn [O][I] with w_scale
    [ceil(O/128)][ceil(I/128)] -> y [N][O], of type y_dtype (y's, or float32, if not given)."""
    device = _gpu(x, "x")
    if stream is not None or device.index != _current_gpu():
        with _there(device, stream):
            return cnn_fc_f8_fwd(x, x_scale, w, w_scale, bias, fuse_relu, y_dtype, y)
    if x.dim() != 2 or w.dim() != 2:
        raise ValueError("fc_f8: x must be [N][I], w [O][I]")
    (N, I), (O, cols) = x.shape, w.shape
    if cols != I:
        raise ValueError(f"fc_f8: x has {I} columns, w {cols}")
    if max(N, I, O) > _INT_MAX:
        _too_large("fc_f8")
    blocks = (I + 127) // 128
    xp = _on(x, "x", device, _F8)
    xs = _on(x_scale, "x_scale", device, torch.float32, (N, blocks))
    wp = _on(w, "w", device, _F8)
    ws = _on(w_scale, "w_scale", device, torch.float32, ((O + 127) // 128, blocks))
    bp = _on(bias, "bias", device, torch.float32, (O,))
    st = _raw_stream(device.index)
    if y is None:
        y = x.new_empty((N, O), dtype=y_dtype or torch.float32)
        yp = y.data_ptr()
    else:
        yp = _on(y, "y", device, y_dtype, (N, O))
    need = _fc_f8_workspace(N, I, O)
    work = x.new_empty(need, dtype=torch.uint8) if need else None
    _ok(lib.cnn_fc_f8_fwd(xp, xs, N, I, wp, ws, bp, O, 1 if fuse_relu else 0, yp, _WIDE.get(y.dtype, -1),
                          work.data_ptr() if need else None, need, st))
    return y


def cnn_sample_fwd(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, stream=None):
    """logits [N][V], u float32 [N] uniform in [0, 1) -> (token int32 [N], prob float32 [N]): a token for each row, and
    its probability among those that the row's top_k (int32 [N]), top_p and min_p (float32 [N]) keep at its temperature
    (float32 [N]); None for a parameter that no row has.  token is -1 where there is nothing to take.

    The two are parts of one allocation: it lives as long as either of them."""
    device = _gpu(logits, "logits")
    if stream is not None or device.index != _current_gpu():
        with _there(device, stream):
            return cnn_sample_fwd(logits, u, temperature, top_k, top_p, min_p)
    if logits.dim() != 2:
        raise ValueError("sample: logits must be [N][V]")
    N, V = logits.shape
    if max(N, V) > _INT_MAX:
        _too_large("sample")
    code = _wide(logits.dtype, "logits")
    if u is None:
        raise TypeError(f"u must be a tensor on {device}")
    row = (N,)
    lp = _on(logits, "logits", device)
    up = _on(u, "u", device, torch.float32, row)
    tp = _on(temperature, "temperature", device, torch.float32, row)
    kp = _on(top_k, "top_k", device, torch.int32, row)
    pp = _on(top_p, "top_p", device, torch.float32, row)
    mp = _on(min_p, "min_p", device, torch.float32, row)
    st = _raw_stream(device.index)
    parts = logits.new_empty((2, N), dtype=torch.int32)
    base = parts.data_ptr()
    need = _sample_workspace(code, N, V)
    work = logits.new_empty(need, dtype=torch.uint8) if need else None
    _ok(lib.cnn_sample_fwd(lp, code, N, V, up, tp, kp, pp, mp, base, base + 4 * N,
                           work.data_ptr() if need else None, need, st))
    token, prob = parts.unbind(0)
    return token, prob.view(torch.float32)


# ---------------------------------------------------------------- NetFile
@dataclass(frozen=True)
class NetFile:
    """A parsed NetFile (cnn_netfile_parse): engine parameters and the layer
    list, as a ``workloads.Net`` whose layers carry the shapes that the
    library's own shape rules give for the declared input."""

    net: "_wl.Net"
    execution_mode: str
    auto_tuning: bool
    allocated_ram_mib: int


def parse_netfile(text: str, name: str = "netfile", input_chw: Optional[Tuple[int, int, int]] = None,
                  weight_std: float = 0.01, bias_std: float = 0.01) -> NetFile:
    """Parses NetFile text.  input_chw overrides (or supplies) the "input"
    statement; weight_std / bias_std only describe synthetic parameters."""
    raw = text.encode()
    n = ctypes.c_int()
    cfg = cnn_netfile_config()
    _ok(lib.cnn_netfile_parse(raw, None, 0, ctypes.byref(n), ctypes.byref(cfg)))
    descs = (cnn_layer_desc * max(n.value, 1))()
    _ok(lib.cnn_netfile_parse(raw, descs, n.value, ctypes.byref(n), ctypes.byref(cfg)))
    chw = input_chw or (cfg.in_channels, cfg.in_height, cfg.in_width)
    if min(chw) <= 0:
        raise ValueError("NetFile: no input shape (an 'input C H W' line or input_chw=)")
    layers = []
    shape = tuple(chw)
    oc, oh, ow = ctypes.c_int(), ctypes.c_int(), ctypes.c_int()
    for i in range(n.value):
        d = descs[i]
        c, h, w = shape
        if d.type == CNN_LAYER_CONV:
            layers.append(_wl.conv(c, d.out_channels, (d.kernel_h, d.kernel_w), (d.stride_h, d.stride_w),
                                   (d.pad_h, d.pad_w), d.groups, bool(d.fuse_relu)))
        elif d.type == CNN_LAYER_FC:
            layers.append(_wl.fc(c * h * w, d.out_channels, bool(d.fuse_relu)))
        elif d.type == CNN_LAYER_POOL:
            layers.append(_wl.pool("max" if d.pool_mode == CNN_POOL_MAX else "avg", (d.kernel_h, d.kernel_w),
                                   (d.stride_h, d.stride_w), (d.pad_h, d.pad_w), bool(d.ceil_mode),
                                   bool(d.fuse_relu)))
        elif d.type == CNN_LAYER_LRN:
            layers.append(_wl.lrn(d.lrn_size, d.lrn_alpha, d.lrn_beta, d.lrn_k))
        elif d.type == CNN_LAYER_RELU:
            layers.append(_wl.relu())
        else:
            layers.append(_wl.softmax())
        # shape after this layer, by the library's rules (also checks in=)
        _ok(lib.cnn_net_out_shape(descs, i + 1, 1, *chw, ctypes.byref(oc), ctypes.byref(oh),
                                  ctypes.byref(ow)))
        shape = (oc.value, oh.value, ow.value)
    net = _wl.Net(name, tuple(chw), tuple(layers), weight_std, bias_std)
    mode = "graph" if cfg.execution_mode == CNN_EXEC_GRAPH else "parallel"
    return NetFile(net, mode, bool(cfg.auto_tuning), cfg.allocated_ram_mib)


def load_netfile(path: str, **kw) -> NetFile:
    with open(path) as f:
        return parse_netfile(f.read(), name=os.path.splitext(os.path.basename(path))[0], **kw)


NETFILE_DIR = os.path.join(HERE, "netfiles")


# ---------------------------------------------------------------- networks
class Network:
    """A layer-descriptor array bound to device-resident parameters.

    Built from a ``workloads.Net`` and its (weight, bias) list; parameters are
    copied to the device once (loading is outside the timed path, as in the
    paper's measurements).  ``pool_index=True`` allocates an int32 index
    output for every max-pooling layer (per batch size, on first use).

    execution_mode (the NetFile parameter): "parallel" enqueues the layers on
    every call (cnn_net_fwd); "graph" runs the first call for a given
    (input, output, batch) eagerly, captures it into a HIP graph
    (cnn_net_graph_create) and replays the graph from then on.  In graph mode
    an output allocated by the call (y=None) is a buffer reused by later
    calls of the same batch size.
    """

    def __init__(self, net, params, device="cuda", pool_index: bool = False,
                 execution_mode: str = "parallel"):
        if execution_mode not in ("parallel", "graph"):
            raise ValueError(f"execution_mode {execution_mode!r}: parallel or graph")
        self.execution_mode = execution_mode
        self._graphs: Dict[tuple, ctypes.c_void_p] = {}
        self._outs: Dict[int, torch.Tensor] = {}
        self.net = net
        self.device = torch.device(device)
        self.weights: List[Tuple[Optional[torch.Tensor], Optional[torch.Tensor]]] = []
        for layer, pr in zip(net.layers, params):
            if layer.has_params:
                self.weights.append((torch.from_numpy(pr[0]).to(self.device).contiguous(),
                                     torch.from_numpy(pr[1]).to(self.device).contiguous()))
            else:
                self.weights.append((None, None))
        self.pool_index = pool_index
        self.indices: List[Optional[torch.Tensor]] = [None] * len(net.layers)
        self.descs = (cnn_layer_desc * len(net.layers))()
        for i, (layer, (w, b)) in enumerate(zip(net.layers, self.weights)):
            d = self.descs[i]
            if layer.kind == "conv":
                d.type = CNN_LAYER_CONV
                d.in_channels = layer.in_channels
                d.out_channels = layer.out_channels
                d.kernel_h, d.kernel_w = layer.kernel
                d.stride_h, d.stride_w = layer.stride
                d.pad_h, d.pad_w = layer.pad
                d.groups = layer.groups
                d.fuse_relu = int(layer.relu)
            elif layer.kind == "fc":
                d.type = CNN_LAYER_FC
                d.out_channels = layer.out_features
                d.in_features = layer.in_features
                d.fuse_relu = int(layer.relu)
            elif layer.kind == "pool":
                d.type = CNN_LAYER_POOL
                d.pool_mode = CNN_POOL_MAX if layer.mode == "max" else CNN_POOL_AVG
                d.kernel_h, d.kernel_w = layer.kernel
                d.stride_h, d.stride_w = layer.stride
                d.pad_h, d.pad_w = layer.pad
                d.ceil_mode = int(layer.ceil)
                d.fuse_relu = int(layer.relu)
            elif layer.kind == "lrn":
                d.type = CNN_LAYER_LRN
                d.lrn_size = layer.size
                d.lrn_alpha, d.lrn_beta, d.lrn_k = layer.alpha, layer.beta, layer.k
            elif layer.kind == "relu":
                d.type = CNN_LAYER_RELU
            elif layer.kind == "softmax":
                d.type = CNN_LAYER_SOFTMAX
            else:
                raise ValueError(f"unknown layer kind {layer.kind}")
            d.weight = w.data_ptr() if w is not None else None
            d.bias = b.data_ptr() if b is not None else None
        self._ws: Optional[torch.Tensor] = None
        self._ws_key = None

    def replica(self) -> "Network":
        """A Network over the same device parameters with its own workspace,
        index buffers and graphs, so that a second pass can run concurrently
        on another stream (two passes never share a workspace)."""
        r = Network.__new__(Network)
        r.execution_mode = self.execution_mode
        r._graphs, r._outs = {}, {}
        r.net, r.device, r.weights = self.net, self.device, self.weights
        r.pool_index = self.pool_index
        r.indices = [None] * len(self.net.layers)
        r.descs = (cnn_layer_desc * len(self.descs))()
        ctypes.memmove(r.descs, self.descs, ctypes.sizeof(self.descs))
        for d in r.descs:
            d.pool_index = None
        r._ws, r._ws_key = None, None
        return r

    def out_shape(self, N: int) -> Tuple[int, int, int, int]:
        C, H, W = self.net.input_chw
        oc, oh, ow = ctypes.c_int(), ctypes.c_int(), ctypes.c_int()
        _ok(lib.cnn_net_out_shape(self.descs, len(self.descs), N, C, H, W, ctypes.byref(oc),
                                  ctypes.byref(oh), ctypes.byref(ow)))
        last = [l for l in self.net.layers if l.kind not in ("relu", "softmax")]
        if last and last[-1].kind == "fc":
            return (N, oc.value)
        return (N, oc.value, oh.value, ow.value)

    def workspace_bytes(self, N: int) -> int:
        C, H, W = self.net.input_chw
        n = lib.cnn_net_workspace_bytes(self.descs, len(self.descs), N, C, H, W)
        if n == 0 and N > 0:
            raise CnnError(CNN_ERR_INVALID, cnn_last_error())
        return int(n)

    @classmethod
    def from_netfile(cls, netfile, params, device="cuda", pool_index: bool = False) -> "Network":
        """A Network for a parsed NetFile (or NetFile text): its execution
        mode, and auto-tuning switched on for the library when it asks so."""
        if isinstance(netfile, str):
            netfile = parse_netfile(netfile)
        if netfile.auto_tuning:
            cnn_set_autotune(True)
        return cls(netfile.net, params, device, pool_index, netfile.execution_mode)

    def close(self) -> None:
        """Destroys the captured graphs."""
        for g in self._graphs.values():
            lib.cnn_net_graph_destroy(g)
        self._graphs.clear()

    def __del__(self):
        try:
            self.close()
        except Exception:  # interpreter shutdown
            pass

    def _prepare(self, N: int):
        key = N
        if self._ws_key != key:
            self.close()  # graphs hold the old workspace and index buffers
            nbytes = self.workspace_bytes(N)
            self._ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=self.device)
            self._ws_key = key
            if self.pool_index:
                self._alloc_indices(N)

    def _alloc_indices(self, N: int):
        C, H, W = self.net.input_chw
        c, h, w = C, H, W
        for i, layer in enumerate(self.net.layers):
            if layer.kind == "conv":
                h, w = cnn_conv2d_out_shape(h, w, *layer.kernel, layer.stride, layer.pad)
                c = layer.out_channels
            elif layer.kind == "pool":
                h, w = cnn_pool_out_shape(h, w, layer.kernel, layer.stride, layer.pad, layer.ceil)
                if layer.mode == "max":
                    self.indices[i] = torch.empty((N, c, h, w), dtype=torch.int32, device=self.device)
                    self.descs[i].pool_index = self.indices[i].data_ptr()
            elif layer.kind == "fc":
                c, h, w = layer.out_features, 1, 1

    def forward(self, x: torch.Tensor, y: Optional[torch.Tensor] = None, stream=None,
                events: Optional[Sequence] = None,
                kernel_events: Optional[Tuple[Sequence, Sequence]] = None) -> torch.Tensor:
        """cnn_net_fwd; cnn_net_fwd_timed with `events` (one torch.cuda.Event
        per layer + 1); cnn_net_fwd_kernel_timed with `kernel_events` = (starts,
        stops), one event of each per layer, every event already recorded once
        (torch creates its events lazily)."""
        N, C, H, W = x.shape
        self._prepare(N)
        if events is not None and kernel_events is not None:
            raise ValueError("events and kernel_events are exclusive")
        graph = self.execution_mode == "graph" and events is None and kernel_events is None
        if y is None:
            if graph:
                if N not in self._outs:
                    self._outs[N] = torch.empty(self.out_shape(N), dtype=torch.float32, device=x.device)
                y = self._outs[N]
            else:
                y = torch.empty(self.out_shape(N), dtype=torch.float32, device=x.device)
        args = (self.descs, len(self.descs), _dev(x, "x"), N, C, H, W, _dev(y, "y"),
                self._ws.data_ptr(), self._ws.numel())
        if graph:
            key = (N, C, H, W, x.data_ptr(), y.data_ptr())
            g = self._graphs.get(key)
            if g is None:
                # eager first pass: validates, and tunes new shapes when auto-tuning is on
                _ok(lib.cnn_net_fwd(*args, _stream(stream)))
                g = ctypes.c_void_p()
                _ok(lib.cnn_net_graph_create(*args, ctypes.byref(g)))
                self._graphs[key] = g
                return y
            _ok(lib.cnn_net_graph_launch(g, _stream(stream)))
            return y
        if kernel_events is not None:
            starts, stops = kernel_events
            if len(starts) != len(self.descs) or len(stops) != len(self.descs):
                raise ValueError("need one start and one stop event per layer")
            arrs = [(ctypes.c_void_p * len(ev))(*[e.cuda_event if hasattr(e, "cuda_event") else int(e) for e in ev])
                    for ev in (starts, stops)]
            _ok(lib.cnn_net_fwd_kernel_timed(*args, arrs[0], arrs[1], _stream(stream)))
        elif events is None:
            _ok(lib.cnn_net_fwd(*args, _stream(stream)))
        else:
            if len(events) != len(self.descs) + 1:
                raise ValueError("need one event per layer plus one")
            arr = (ctypes.c_void_p * len(events))(*[e.cuda_event if hasattr(e, "cuda_event") else int(e)
                                                    for e in events])
            _ok(lib.cnn_net_fwd_timed(*args, arr, _stream(stream)))
        return y

    __call__ = forward

    def forward_noalloc(self, x: torch.Tensor, y: Optional[torch.Tensor] = None, stream=None):
        """cnn_net_fwd_noalloc: the pass with the library's static device
        scratch as its workspace (no workspace tensor is allocated here; y is
        allocated when None)."""
        N, C, H, W = x.shape
        if y is None:
            y = torch.empty(self.out_shape(N), dtype=torch.float32, device=x.device)
        _ok(lib.cnn_net_fwd_noalloc(self.descs, len(self.descs), _dev(x, "x"), N, C, H, W, _dev(y, "y"),
                                    _stream(stream)))
        return y

    def layer_shapes(self, N: int) -> List[Tuple[int, ...]]:
        """Output shape of every layer for a batch of N (the library's shape rules)."""
        C, H, W = self.net.input_chw
        oc, oh, ow = ctypes.c_int(), ctypes.c_int(), ctypes.c_int()
        shapes = []
        flat = False  # after an FC layer (and the ReLU / softmax layers after it): [N][O]
        for i, layer in enumerate(self.net.layers):
            _ok(lib.cnn_net_out_shape(self.descs, i + 1, N, C, H, W, ctypes.byref(oc),
                                      ctypes.byref(oh), ctypes.byref(ow)))
            if layer.kind not in ("relu", "softmax"):
                flat = layer.kind == "fc"
            shapes.append((N, oc.value) if flat else (N, oc.value, oh.value, ow.value))
        return shapes

    def forward_dump(self, x: torch.Tensor, y: Optional[torch.Tensor] = None, stream=None):
        """cnn_net_fwd_dump: one pass that also writes every layer's output.

        Returns (y, outs, written): outs[i] is layer i's output (a tensor of
        its shape) where written[i], else None (a RELU layer executed inside
        its predecessor, whose entry then holds the output after it)."""
        N, C, H, W = x.shape
        self._prepare(N)
        if y is None:
            y = torch.empty(self.out_shape(N), dtype=torch.float32, device=x.device)
        bufs = [torch.empty(s, dtype=torch.float32, device=x.device) for s in self.layer_shapes(N)]
        ptrs = (ctypes.c_void_p * len(bufs))(*[b.data_ptr() for b in bufs])
        written = (ctypes.c_int * len(bufs))()
        _ok(lib.cnn_net_fwd_dump(self.descs, len(self.descs), _dev(x, "x"), N, C, H, W, _dev(y, "y"),
                                 self._ws.data_ptr(), self._ws.numel(), ptrs, written, _stream(stream)))
        flags = [bool(written[i]) for i in range(len(bufs))]
        return y, [b if f else None for b, f in zip(bufs, flags)], flags


def cnn_net_fwd(network: Network, x, y=None, stream=None):
    return network.forward(x, y, stream)
