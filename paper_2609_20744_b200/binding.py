"""Thin ctypes binding over the C ABI declared in include/vdn_vda.h.

Argument marshalling only: every step of the layer runs inside the CUDA library.  torch is used
for device memory and streams.  There is no CPU fallback: if the shared library is missing or a
call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Optional

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("VDN_VDA_LIB") or os.path.join(_HERE, "libvdn_vda.so")   # VDN_VDA_LIB: another build of the library

VDN_OK = 0
STATUS_NAMES = {0: "VDN_OK", 1: "VDN_ERR_INVALID_ARG", 2: "VDN_ERR_UNSUPPORTED", 3: "VDN_ERR_WORKSPACE",
                4: "VDN_ERR_CUDA", 5: "VDN_ERR_ARCH", 6: "VDN_ERR_TIMEOUT", 7: "VDN_ERR_INTERNAL"}
VDN_ERR_INVALID_ARG, VDN_ERR_TIMEOUT, VDN_ERR_INTERNAL = 1, 6, 7
VDN_F32, VDN_BF16 = 0, 1
VDN_FLAG_FORCE_SIMT = 1
VDN_FLAG_ADDITIVE_RULE = 4
VDN_FLAG_SCAN_CHUNKWISE = 8
VDN_FLAG_SCAN_FRAMEWISE = 16
VDN_FLAG_EXACT_STATS = 32
VDN_FLAG_FP32_RESOLVE = 64
VDN_ROTARY_HALF, VDN_ROTARY_INVERSE = 1, 2
VIEW_STATS, VIEW_INV, VIEW_FWD, VIEW_READ, VIEW_INV_SPLIT, VIEW_READ_FWD, VIEW_READ_BWD, VIEW_COMP_M, VIEW_COMP_J = range(9)

EXPORTS = (
    "vdn_vda_create", "vdn_vda_workspace_bytes", "vdn_vda_set_workspace", "vdn_vda_forward", "vdn_vda_forward_ex",
    "vdn_vda_forward_opt", "vdn_vda_workspace_bytes_opt", "vdn_vda_prepare",
    "vdn_vda_token_scan_workspace_bytes", "vdn_vda_token_scan", "vdn_vda_token_step", "vdn_vda_rotate",
    "vdn_vda_quantize", "vdn_vda_scaled_matmul", "vdn_vda_cross_attention_workspace_bytes", "vdn_vda_cross_attention",
    "vdn_vda_staging_bytes", "vdn_vda_staging_bytes_opt", "vdn_vda_set_staging", "vdn_vda_forward_host",
    "vdn_vda_forward_host_opt", "vdn_vda_workspace_view",
    "vdn_vda_last_launch_count", "vdn_vda_profile", "vdn_vda_kernel_times", "vdn_vda_scan_static", "vdn_vda_status",
    "vdn_vda_clear_status", "vdn_vda_set_wait_limit_us", "vdn_vda_selftest_wait_expiry", "vdn_vda_selftest_marker",
    "vdn_vda_last_error", "vdn_vda_destroy",
)


class VdnConfig(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("io_dtype", ctypes.c_int32), ("d", ctypes.c_int32),
                ("rms_eps", ctypes.c_float), ("flags", ctypes.c_uint32), ("device", ctypes.c_int32)]


class VdnOptions(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("chunk", ctypes.c_int32), ("radius", ctypes.c_int32),
                ("anchors", ctypes.c_int32), ("alpha", ctypes.c_void_p), ("s0", ctypes.c_void_p),
                ("gate_elem", ctypes.c_void_p), ("norm_weight", ctypes.c_void_p), ("q_l2_eps", ctypes.c_float),
                ("reserved", ctypes.c_uint32)]


class VdnPrepParams(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("Y", ctypes.c_int32), ("X", ctypes.c_int32),
                ("anchors", ctypes.c_int32), ("l2_eps", ctypes.c_float), ("wk_spatial", ctypes.c_void_p),
                ("wk_temporal", ctypes.c_void_p), ("wv_spatial", ctypes.c_void_p), ("wv_temporal", ctypes.c_void_p)]


class VdnTokenParams(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("heads", ctypes.c_int32), ("key_heads", ctypes.c_int32),
                ("n_seqs", ctypes.c_int32), ("scale", ctypes.c_float), ("l2_eps", ctypes.c_float),
                ("cu_seqlens", ctypes.c_void_p), ("index", ctypes.c_void_p), ("log_alpha", ctypes.c_void_p),
                ("s0", ctypes.c_void_p), ("state", ctypes.c_void_p), ("n_slots", ctypes.c_int64),
                ("q_stride", ctypes.c_int64), ("k_stride", ctypes.c_int64), ("v_stride", ctypes.c_int64),
                ("out_stride", ctypes.c_int64)]


class VdnRotaryParams(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("flags", ctypes.c_uint32), ("pairs", ctypes.c_int32),
                ("key_heads", ctypes.c_int32), ("Y", ctypes.c_int32), ("X", ctypes.c_int32), ("t0", ctypes.c_int32),
                ("norm_eps", ctypes.c_float), ("freq", ctypes.c_void_p), ("axis", ctypes.c_void_p),
                ("positions", ctypes.c_void_p), ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p),
                ("q_stride", ctypes.c_int64), ("k_stride", ctypes.c_int64), ("q_out_stride", ctypes.c_int64),
                ("k_out_stride", ctypes.c_int64)]


class VdnQuantizeParams(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("block_rows", ctypes.c_int32), ("x_stride", ctypes.c_int64),
                ("out_stride", ctypes.c_int64)]


class VdnMatmulParams(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("reserved", ctypes.c_uint32), ("a_scale", ctypes.c_void_p),
                ("w_scale", ctypes.c_void_p), ("bias", ctypes.c_void_p), ("add", ctypes.c_void_p), ("a_stride", ctypes.c_int64),
                ("w_stride", ctypes.c_int64), ("add_stride", ctypes.c_int64), ("out_stride", ctypes.c_int64)]


class VdnCrossParams(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("batch", ctypes.c_int32), ("heads", ctypes.c_int32), ("key_heads", ctypes.c_int32),
                ("scale", ctypes.c_float), ("reserved", ctypes.c_uint32), ("cu_seqlens", ctypes.c_void_p), ("lengths", ctypes.c_void_p),
                ("mask", ctypes.c_void_p), ("lse", ctypes.c_void_p), ("q_stride", ctypes.c_int64), ("k_stride", ctypes.c_int64),
                ("v_stride", ctypes.c_int64), ("out_stride", ctypes.c_int64)]


# the same structs as packed bytes (the header's layout, no padding anywhere): a third of the time of filling a Structure
_TOKEN_PARAMS = struct.Struct("=IiiiffQQQQQqqqqq")
_ROTARY_PARAMS = struct.Struct("=IIiiiiifQQQQQqqqq")
_QUANTIZE_PARAMS = struct.Struct("=Iiqq")
_MATMUL_PARAMS = struct.Struct("=IIQQQQqqqq")
_CROSS_PARAMS = struct.Struct("=IiiifIQQQQqqqq")
SCALE_BLOCK = 128


class VdnError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {msg}")
        self.status = status


_lib = None


def load_library(path: Optional[str] = None) -> ctypes.CDLL:
    """dlopen the CUDA library and declare its signatures.  Raises if it has not been built."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise FileNotFoundError(
            f"{p} not found: build it with `python -m paper_2609_20744_b200.build` (there is no CPU fallback)")
    lib = ctypes.CDLL(p)
    vp, ci, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    shape = [ci, ci, ci, ci, ci]
    lib.vdn_vda_create.argtypes = [ctypes.POINTER(VdnConfig), ctypes.POINTER(vp)]
    lib.vdn_vda_create.restype = ci
    lib.vdn_vda_workspace_bytes.argtypes = [vp, *shape]
    lib.vdn_vda_workspace_bytes.restype = sz
    lib.vdn_vda_set_workspace.argtypes = [vp, vp, sz]
    lib.vdn_vda_set_workspace.restype = ci
    lib.vdn_vda_staging_bytes.argtypes = [vp, *shape]
    lib.vdn_vda_staging_bytes.restype = sz
    lib.vdn_vda_set_staging.argtypes = [vp, vp, sz]
    lib.vdn_vda_set_staging.restype = ci
    fwd_args = [vp, vp, vp, vp, vp, vp, vp, *shape, vp]
    lib.vdn_vda_forward.argtypes = fwd_args
    lib.vdn_vda_forward.restype = ci
    lib.vdn_vda_forward_ex.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, *shape, vp]
    lib.vdn_vda_forward_ex.restype = ci
    lib.vdn_vda_forward_opt.argtypes = [vp, vp, vp, vp, vp, vp, vp, *shape, ctypes.POINTER(VdnOptions), vp]
    lib.vdn_vda_forward_opt.restype = ci
    lib.vdn_vda_workspace_bytes_opt.argtypes = [vp, *shape, ctypes.POINTER(VdnOptions)]
    lib.vdn_vda_workspace_bytes_opt.restype = sz
    lib.vdn_vda_prepare.argtypes = [vp, vp, vp, vp, vp, vp, vp, *shape, ctypes.POINTER(VdnPrepParams), vp]
    lib.vdn_vda_prepare.restype = ci
    tok, i64 = vp, ctypes.c_longlong        # parameter structs: packed bytes, or byref of the Structure
    lib.vdn_vda_token_scan_workspace_bytes.argtypes = [vp, i64, tok]
    lib.vdn_vda_token_scan_workspace_bytes.restype = sz
    lib.vdn_vda_token_scan.argtypes = [vp, vp, vp, vp, vp, vp, i64, tok, vp, sz, vp]
    lib.vdn_vda_token_scan.restype = ci
    lib.vdn_vda_token_step.argtypes = [vp, vp, vp, vp, vp, vp, ci, ci, tok, vp]
    lib.vdn_vda_token_step.restype = ci
    lib.vdn_vda_rotate.argtypes = [vp, vp, vp, vp, vp, *shape, vp, vp]
    lib.vdn_vda_rotate.restype = ci
    lib.vdn_vda_quantize.argtypes = [vp, vp, vp, vp, i64, i64, vp, vp]
    lib.vdn_vda_quantize.restype = ci
    lib.vdn_vda_scaled_matmul.argtypes = [vp, vp, vp, vp, i64, i64, i64, vp, vp]
    lib.vdn_vda_scaled_matmul.restype = ci
    lib.vdn_vda_cross_attention_workspace_bytes.argtypes = [vp, i64, i64, vp]
    lib.vdn_vda_cross_attention_workspace_bytes.restype = sz
    lib.vdn_vda_cross_attention.argtypes = [vp, vp, vp, vp, vp, i64, i64, vp, vp, sz, vp]
    lib.vdn_vda_cross_attention.restype = ci
    lib.vdn_vda_forward_host.argtypes = fwd_args
    lib.vdn_vda_forward_host.restype = ci
    lib.vdn_vda_forward_host_opt.argtypes = [vp, vp, vp, vp, vp, vp, vp, *shape, ctypes.POINTER(VdnOptions), vp]
    lib.vdn_vda_forward_host_opt.restype = ci
    lib.vdn_vda_staging_bytes_opt.argtypes = [vp, *shape, ctypes.POINTER(VdnOptions)]
    lib.vdn_vda_staging_bytes_opt.restype = sz
    lib.vdn_vda_clear_status.argtypes = [vp]
    lib.vdn_vda_clear_status.restype = ci
    lib.vdn_vda_set_wait_limit_us.argtypes = [vp, ctypes.c_ulonglong]
    lib.vdn_vda_set_wait_limit_us.restype = ci
    lib.vdn_vda_selftest_wait_expiry.argtypes = [vp, ctypes.c_ulonglong, vp]
    lib.vdn_vda_selftest_wait_expiry.restype = ci
    lib.vdn_vda_selftest_marker.argtypes = [vp]
    lib.vdn_vda_selftest_marker.restype = ci
    lib.vdn_vda_workspace_view.argtypes = [vp, ci, *shape, ctypes.POINTER(sz), ctypes.POINTER(sz)]
    lib.vdn_vda_workspace_view.restype = ci
    lib.vdn_vda_last_launch_count.argtypes = [vp]
    lib.vdn_vda_last_launch_count.restype = ci
    lib.vdn_vda_profile.argtypes = [vp, ci]
    lib.vdn_vda_profile.restype = ci
    lib.vdn_vda_kernel_times.argtypes = [vp, ci, ctypes.POINTER(ctypes.c_char_p), ctypes.POINTER(ctypes.c_float),
                                         ctypes.POINTER(ci)]
    lib.vdn_vda_kernel_times.restype = ci
    lib.vdn_vda_scan_static.argtypes = [vp, vp, vp, ci, ci, ci, ci, vp, ctypes.c_char_p, sz]
    lib.vdn_vda_scan_static.restype = ci
    lib.vdn_vda_status.argtypes = [vp]
    lib.vdn_vda_status.restype = ci
    lib.vdn_vda_last_error.argtypes = [vp]
    lib.vdn_vda_last_error.restype = ctypes.c_char_p
    lib.vdn_vda_destroy.argtypes = [vp]
    lib.vdn_vda_destroy.restype = ci
    if path is None:
        _lib = lib
    return lib


SCAN_STATIC_MAX_BYTES = 8 << 20


def scan_static(stats, inv, read, stream=None):
    """vdn_vda_scan_static: the fp32 frame scan + gather with its scratch inside the library image.

    For callers that may not allocate device memory.  stats [BH,T,2d,d], inv [BH,T,d,d] and the output
    read [BH,T,d,d] are contiguous float CUDA tensors owned by the caller; nothing is allocated here or
    in the library.  Raises VdnError (VDN_ERR_WORKSPACE) when BH*T*d*d*4 exceeds SCAN_STATIC_MAX_BYTES.
    Calls that may overlap on the GPU share the scratch and must be serialised by the caller.
    """
    import torch
    lib = load_library()
    BH, T, d2, d = stats.shape
    for x in (stats, inv, read):
        if not (x.is_cuda and x.is_contiguous() and x.dtype == torch.float32):
            raise ValueError("scan_static needs contiguous float32 CUDA tensors")
    if d2 != 2 * d or tuple(inv.shape) != (BH, T, d, d) or tuple(read.shape) != (BH, T, d, d):
        raise ValueError("scan_static: shapes must be stats [BH,T,2d,d], inv/read [BH,T,d,d]")
    dev = stats.device.index or 0
    s = stream if stream is not None else torch.cuda.current_stream(dev)
    err = ctypes.create_string_buffer(256)
    st = lib.vdn_vda_scan_static(ctypes.c_void_p(stats.data_ptr()), ctypes.c_void_p(inv.data_ptr()),
                                 ctypes.c_void_p(read.data_ptr()), BH, T, d, dev, ctypes.c_void_p(s.cuda_stream),
                                 err, len(err))
    if st != VDN_OK:
        raise VdnError(st, err.value.decode())
    return read


def _require(name, x, shape, dtype, on_cuda, device_index):
    """One tensor argument against what the C ABI will assume about it (the library sees only a pointer)."""
    if x is None:
        raise ValueError(f"{name} is missing")
    where = "CUDA" if on_cuda else "host"
    if bool(x.is_cuda) != on_cuda:
        raise ValueError(f"{name} must be a {where} tensor")
    if on_cuda and (x.device.index or 0) != device_index:
        raise ValueError(f"{name} is on cuda:{x.device.index}, the handle is bound to cuda:{device_index}")
    if not x.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if x.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {x.dtype}")
    if tuple(x.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(x.shape)}")


def validate_layer_args(io_dtype, d_handle, device_index, q, k, v, beta, gate, out=None, alpha=None, s0=None,
                        gate_elem=None, norm_weight=None, on_cuda=True):
    """Checks every tensor of a forward call before anything reaches the library: dtype, shape, device and
    contiguity.  The kernels and the TMA tensor maps index by the shape that is passed, so a tensor of another dtype
    or a shorter one would be read (and `out` written) past its end.  Raises ValueError; returns (B, T, F, H, d).

    io_dtype is the torch dtype of the handle's q, k, v, out; on_cuda = False checks host tensors instead
    (the host-buffer entry point)."""
    import torch
    if q is None or q.dim() != 5:
        raise ValueError("q must have shape [B, T, F, H, d]")
    B, T, F, H, d = (int(n) for n in q.shape)
    del d_handle                      # a head dimension other than the handle's is the library's to refuse
    f32 = torch.float32
    _require("q", q, (B, T, F, H, d), io_dtype, on_cuda, device_index)
    _require("k", k, (B, T, F, H, d), io_dtype, on_cuda, device_index)
    _require("v", v, (B, T, F, H, d), io_dtype, on_cuda, device_index)
    _require("beta", beta, (B, T, F, H), f32, on_cuda, device_index)
    if gate is None and gate_elem is None:
        raise ValueError("gate may only be left out when gate_elem is given")
    if gate is not None:
        _require("gate", gate, (H,), f32, on_cuda, device_index)
    if out is not None:
        _require("out", out, (B, T, F, H, d), io_dtype, on_cuda, device_index)
    if alpha is not None:
        _require("alpha", alpha, (B, T, H, d), f32, on_cuda, device_index)
    if s0 is not None:
        _require("s0", s0, (B, H, d, d), f32, on_cuda, device_index)
    if gate_elem is not None:
        _require("gate_elem", gate_elem, (B, T, F, H, d), io_dtype, on_cuda, device_index)
    if norm_weight is not None:
        _require("norm_weight", norm_weight, (H, d), f32, on_cuda, device_index)
    return B, T, F, H, d


def _require_rows(name, x, lead, heads, d, dtype, on_cuda, device_index):
    """A tensor [*lead, heads, d] whose tokens may lie apart: the heads of a token dense, one distance between all tokens,
    a multiple of 16 bytes.  Returns that distance in elements."""
    if x is None:
        raise ValueError(f"{name} is missing")
    if tuple(x.shape) != (*lead, heads, d):
        raise ValueError(f"{name} must have shape {(*lead, heads, d)}, got {tuple(x.shape)}")
    if x.is_contiguous():
        _require(name, x, x.shape, dtype, on_cuda, device_index)
        return heads * d
    st = x.stride()
    n, step, ok = 1, None, (d == 1 or st[-1] == 1) and (heads == 1 or st[-2] == d)
    for size, stride in zip(reversed(lead), reversed(st[:-2])):
        if size != 1:
            step = stride if step is None else step
            ok = ok and stride == step * n
        n *= size
    step = heads * d if step is None else step
    if not ok or step < heads * d or (step * x.element_size()) % 16:
        raise ValueError(f"{name}: the heads of a token must be contiguous and its tokens evenly spaced, by a multiple of 16 bytes")
    if bool(x.is_cuda) != on_cuda:
        raise ValueError(f"{name} must be a {'CUDA' if on_cuda else 'host'} tensor")
    if on_cuda and (x.device.index or 0) != device_index:
        raise ValueError(f"{name} is on cuda:{x.device.index}, the handle is bound to cuda:{device_index}")
    if x.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {x.dtype}")
    return step


def _rows(name, x, shape, dtype, on_cuda, device_index):
    """_require_rows for a tensor that in all likelihood is dense and right: one glance, the words only if it is not."""
    if x is not None and x.shape == shape and x.dtype is dtype and x.get_device() == (device_index if on_cuda else -1) \
            and x.is_contiguous():
        return shape[-2] * shape[-1]
    return _require_rows(name, x, shape[:-2], shape[-2], shape[-1], dtype, on_cuda, device_index)


def _dense(name, x, shape, dtype, on_cuda, device_index):
    if x is None or x.shape != shape or x.dtype is not dtype or x.get_device() != (device_index if on_cuda else -1) \
            or not x.is_contiguous():
        _require(name, x, shape, dtype, on_cuda, device_index)


def validate_token_args(io_dtype, d_handle, device_index, q, k, v, beta, out=None, log_alpha=None, on_cuda=True):
    """Checks the token tensors of token_scan / token_step: q, k [..., Hk, d], v, out [..., H, d], beta, log_alpha [..., H].
    Returns (leading shape, H, Hk, strides of q, k, v, out)."""
    if v is None or v.dim() < 3:
        raise ValueError("v must have shape [tokens, heads, d]")
    if q is None or q.dim() != v.dim():
        raise ValueError("q must have as many dimensions as v")
    vs = tuple(v.shape)
    lead, H, Hk, d = vs[:-2], vs[-2], q.shape[-2], vs[-1]
    if d != d_handle:
        raise ValueError(f"v must have head dimension {d_handle}, got {d}")
    if H == 0 or Hk == 0 or H % Hk:
        raise ValueError(f"q must have a number of heads that divides the {H} of v, got {Hk}")
    ks, gates = (*lead, Hk, d), (*lead, H)
    strides = (_rows("q", q, ks, io_dtype, on_cuda, device_index), _rows("k", k, ks, io_dtype, on_cuda, device_index),
               _rows("v", v, vs, io_dtype, on_cuda, device_index),
               H * d if out is None else _rows("out", out, vs, io_dtype, on_cuda, device_index))
    f32 = _float32()
    _dense("beta", beta, gates, f32, on_cuda, device_index)
    if log_alpha is not None:
        _dense("log_alpha", log_alpha, gates, f32, on_cuda, device_index)
    return lead, H, Hk, strides


def _matrix(name, x, shape, dtype, on_cuda, device_index, step_bytes=0):
    """A tensor [..., columns] taken as rows that may lie apart: the elements of a row dense, one distance between all rows, with
    step_bytes a multiple of so many bytes.  Returns that distance in elements."""
    if x is None:
        raise ValueError(f"{name} is missing")
    if bool(x.is_cuda) != on_cuda:
        raise ValueError(f"{name} must be a {'CUDA' if on_cuda else 'host'} tensor")
    if on_cuda and (x.device.index or 0) != device_index:
        raise ValueError(f"{name} is on cuda:{x.device.index}, the handle is bound to cuda:{device_index}")
    if x.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {x.dtype}")
    if tuple(x.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(x.shape)}")
    cols, step, n = shape[-1], None, 1
    ok = cols == 1 or x.stride(-1) == 1
    if not x.is_contiguous():
        for size, stride in zip(reversed(shape[:-1]), reversed(x.stride()[:-1])):
            if size != 1:
                step = stride if step is None else step
                ok = ok and stride == step * n
            n *= size
    # (a single row has no distance: the next multiple that covers it)
    only = all(size == 1 for size in shape[:-1]) or x.numel() == 0
    unit = max(1, step_bytes // x.element_size())
    step = -(-cols // unit) * unit if only else cols if step is None else step
    if not ok or step < cols or (step_bytes and (step * x.element_size()) % step_bytes):
        raise ValueError(f"{name}: the elements of a row must be contiguous and its rows evenly spaced"
                         + (f", by a multiple of {step_bytes} bytes" if step_bytes else ""))
    return step


def _glance(x, shape, dtype, on_cuda, device_index):
    """Whether x is dense and just so, as in all likelihood it is."""
    return x is not None and x.dtype is dtype and x.shape == shape and x.get_device() == (device_index if on_cuda else -1) and x.is_contiguous()


def validate_matmul_args(io_dtype, device_index, a, a_scale, w, w_scale, bias=None, add=None, out=None, on_cuda=True):
    """Checks the tensors of scaled_matmul: a [..., K], w [N, K] (float8_e4m3fn), a_scale [..., blocks], w_scale [.., blocks], bias [N],
    add and out [..., N].  Returns (M, N, K, strides of a, w, add, out)."""
    if a is None or a.dim() < 1 or w is None or w.dim() != 2:
        raise ValueError("a must have shape [..., K] and w [N, K]")
    e4m3, f32 = _e4m3(), _float32()
    sa_, sw_ = a.shape, w.shape
    lead, k, n = tuple(sa_[:-1]), sa_[-1], sw_[0]
    blocks = -(-k // SCALE_BLOCK)
    dense = k % 16 == 0
    sa = k if dense and _glance(a, sa_, e4m3, on_cuda, device_index) else _matrix("a", a, (*lead, k), e4m3, on_cuda, device_index, 16)
    sw = k if dense and _glance(w, (n, k), e4m3, on_cuda, device_index) else _matrix("w", w, (n, k), e4m3, on_cuda, device_index, 16)
    _dense("a_scale", a_scale, (*lead, blocks), f32, on_cuda, device_index)
    _dense("w_scale", w_scale, (-(-n // SCALE_BLOCK), blocks), f32, on_cuda, device_index)
    if bias is not None:
        _dense("bias", bias, (n,), f32, on_cuda, device_index)
    shape = (*lead, n)
    sd = so = n
    if add is None:
        sd = 0
    elif not _glance(add, shape, io_dtype, on_cuda, device_index):
        sd = _matrix("add", add, shape, io_dtype, on_cuda, device_index)
    if out is not None and not _glance(out, shape, io_dtype, on_cuda, device_index):
        so = _matrix("out", out, shape, io_dtype, on_cuda, device_index)
    m = 1
    for x in lead:
        m *= x
    return m, n, k, (sa, sw, sd, so)


def validate_cross_args(io_dtype, d_handle, device_index, q, k, v, cu_seqlens=None, lengths=None, mask=None, out=None, lse=None,
                        on_cuda=True):
    """Checks the tensors of cross_attention: q, out [B, ..., H, d], k, v [B, Lk, Hk, d] or, with cu_seqlens [B + 1], packed [N, Hk, d];
    lengths [B], mask [B, Lk] or [N], lse [B, ..., H].  Returns (B, queries, keys, H, Hk, strides of q, k, v, out)."""
    import torch
    if q is None or q.dim() < 3:
        raise ValueError("q must have shape [batch, ..., heads, d]")
    packed = cu_seqlens is not None
    if k is None or k.dim() != (3 if packed else 4):
        raise ValueError("k must have shape " + ("[keys, key_heads, d] with cu_seqlens" if packed else "[batch, keys, key_heads, d]"))
    qs, ks = tuple(q.shape), tuple(k.shape)
    B, H, d, Hk = qs[0], qs[-2], qs[-1], ks[-2]
    if d != d_handle:
        raise ValueError(f"q must have head dimension {d_handle}, got {d}")
    if H == 0 or Hk == 0 or H % Hk:
        raise ValueError(f"k must have a number of heads that divides the {H} of q, got {Hk}")
    lead = ks[:1] if packed else (B, ks[1])
    ks = (*lead, Hk, d)
    strides = (_rows("q", q, qs, io_dtype, on_cuda, device_index), _rows("k", k, ks, io_dtype, on_cuda, device_index),
               _rows("v", v, ks, io_dtype, on_cuda, device_index),
               H * d if out is None else _rows("out", out, qs, io_dtype, on_cuda, device_index))
    if packed:
        _dense("cu_seqlens", cu_seqlens, (B + 1,), torch.int32, on_cuda, device_index)
        if lengths is not None:
            raise ValueError("lengths belong to keys that are not packed")
    if lengths is not None:
        _dense("lengths", lengths, (B,), torch.int32, on_cuda, device_index)
    if mask is not None:
        _dense("mask", mask, lead, torch.bool, on_cuda, device_index)
    if lse is not None:
        _dense("lse", lse, qs[:-1], torch.float32, on_cuda, device_index)
    n = 1
    for x in qs[1:-2]:
        n *= x
    return B, n, lead[-1], H, Hk, strides


_E4M3 = None


def _e4m3():
    global _E4M3
    if _E4M3 is None:
        import torch
        _E4M3 = torch.float8_e4m3fn
    return _E4M3


def _float32():
    import torch
    return torch.float32


def _ptr(x):
    return x.data_ptr() if x is not None else 0


def _current_raw_stream(torch, device):
    """Handle of the current stream, without the Stream object around it where torch offers that."""
    get = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return get(device) if get is not None else torch.cuda.current_stream(device).cuda_stream


def rotary_tables(sections, theta=10000.0, shared_ladder=False):
    """(freq, axis) of rotate() for pairs that are `sections` = (time, height, width) pairs, one axis behind another (host
    tensors).  Each axis has its own ladder theta^(-i / n) over its n pairs; with shared_ladder pair p of all n pairs has
    theta^(-p / n) whatever its axis."""
    import torch
    if len(sections) != 3 or any(int(n) != n or n < 0 for n in sections) or sum(sections) == 0:
        raise ValueError("sections must be three numbers of pairs, not all zero")
    axis = torch.repeat_interleave(torch.arange(3, dtype=torch.int32), torch.tensor([int(n) for n in sections]))
    if shared_ladder:
        e = torch.arange(len(axis), dtype=torch.float64) / len(axis)
    else:
        e = torch.cat([torch.arange(int(n), dtype=torch.float64) / max(1, int(n)) for n in sections])
    return theta ** -e, axis


class Vda:
    """One handle of the library (vdn_vda_create .. vdn_vda_destroy) plus its torch-owned workspace."""

    def __init__(self, d: int, dtype: str = "bf16", rms_eps: float = 1e-6, flags: int = 0, device: int = 0):
        import torch
        self._torch = torch
        self.lib = load_library()
        self.d = d
        self.dtype = dtype
        self.torch_dtype = torch.float32 if dtype == "f32" else torch.bfloat16
        self.device = device
        self._dev = torch.device("cuda", device)
        cfg = VdnConfig(ctypes.sizeof(VdnConfig), VDN_F32 if dtype == "f32" else VDN_BF16, d, rms_eps, flags, device)
        self.h = ctypes.c_void_p()
        st = self.lib.vdn_vda_create(ctypes.byref(cfg), ctypes.byref(self.h))
        if st != VDN_OK:
            self.h = None
            raise VdnError(st, "vdn_vda_create failed")
        self._ws = None
        self._staging = None

    # -- helpers ------------------------------------------------------------------------------
    def _check(self, st: int):
        if st != VDN_OK:
            raise VdnError(st, self.lib.vdn_vda_last_error(self.h).decode())

    def _stream(self, stream):
        torch = self._torch
        s = stream if stream is not None else torch.cuda.current_stream(self.device)
        return ctypes.c_void_p(s.cuda_stream)

    def workspace_bytes(self, B, T, F, H, chunk=1) -> int:
        if chunk > 1:
            opt = VdnOptions(ctypes.sizeof(VdnOptions), chunk, 0, 0, None, None, None, None)
            return int(self.lib.vdn_vda_workspace_bytes_opt(self.h, B, T, F, H, self.d, ctypes.byref(opt)))
        return int(self.lib.vdn_vda_workspace_bytes(self.h, B, T, F, H, self.d))

    def ensure_workspace(self, B, T, F, H, chunk=1):
        torch = self._torch
        need = self.workspace_bytes(B, T, F, H, chunk)
        if need == 0:
            raise VdnError(1, "invalid shape")
        if self._ws is None or self._ws.numel() < need:
            self._ws = torch.empty(need, dtype=torch.uint8, device=f"cuda:{self.device}")
            self._check(self.lib.vdn_vda_set_workspace(self.h, ctypes.c_void_p(self._ws.data_ptr()), need))
        return self._ws

    def ensure_staging(self, B, T, F, H, opt=None):
        torch = self._torch
        if opt is None:
            need = int(self.lib.vdn_vda_staging_bytes(self.h, B, T, F, H, self.d))
        else:
            need = int(self.lib.vdn_vda_staging_bytes_opt(self.h, B, T, F, H, self.d, ctypes.byref(opt)))
        if need == 0:
            raise VdnError(1, "invalid shape")
        if self._staging is None or self._staging.numel() < need:
            self._staging = torch.empty(need, dtype=torch.uint8, device=f"cuda:{self.device}")
            self._check(self.lib.vdn_vda_set_staging(self.h, ctypes.c_void_p(self._staging.data_ptr()), need))
        return self._staging

    # -- the two entry points -----------------------------------------------------------------
    def forward(self, q, k, v, beta, gate, out=None, stream=None, alpha=None, s0=None,
                chunk=1, radius=0, anchors=False, gate_elem=None, norm_weight=None, q_l2_eps=0.0):
        """vdn_vda_forward on device tensors q,k,v [B,T,F,H,d], beta [B,T,F,H], gate [H].

        With alpha [B,T,H,d] (decay gates) and/or s0 [B,H,d,d] (text state) the call goes to vdn_vda_forward_ex;
        with a chunk window (chunk, radius), boundary anchors, an element-wise gate gate_elem [B,T,F,H,d] (then
        `gate` may be None), a norm weight norm_weight [H,d] or q_l2_eps > 0 (q arrives without its L2
        normalisation; the read-out applies it) it goes to vdn_vda_forward_opt.
        """
        torch = self._torch
        B, T, F, H, d = validate_layer_args(self.torch_dtype, self.d, self.device, q, k, v, beta, gate, out, alpha, s0,
                                            gate_elem, norm_weight)
        if out is None:
            out = torch.empty_like(q)
        self.ensure_workspace(B, T, F, H, chunk)
        p = lambda x: ctypes.c_void_p(x.data_ptr()) if x is not None else None
        a = lambda x: x.data_ptr() if x is not None else None
        if (chunk, radius, bool(anchors)) != (1, 0, False) or gate_elem is not None or norm_weight is not None \
                or gate is None or q_l2_eps:
            opt = VdnOptions(ctypes.sizeof(VdnOptions), chunk, radius, 1 if anchors else 0, a(alpha), a(s0),
                             a(gate_elem), a(norm_weight), float(q_l2_eps), 0)
            st = self.lib.vdn_vda_forward_opt(self.h, p(q), p(k), p(v), p(beta), p(gate), p(out),
                                              B, T, F, H, d, ctypes.byref(opt), self._stream(stream))
        elif alpha is not None or s0 is not None:
            st = self.lib.vdn_vda_forward_ex(self.h, p(q), p(k), p(v), p(beta), p(gate), p(alpha), p(s0), p(out),
                                             B, T, F, H, d, self._stream(stream))
        else:
            st = self.lib.vdn_vda_forward(self.h, p(q), p(k), p(v), p(beta), p(gate), p(out),
                                          B, T, F, H, d, self._stream(stream))
        self._check(st)
        return out

    def prepare(self, q, k, v, filters, Y, X, anchors=False, l2_eps=1e-6, out=None, stream=None):
        """vdn_vda_prepare: projected q, k, v [B,T,F,H,d] -> prepared (q', k', v') (Sec. 2.3).

        filters = dict(wk_spatial [H*d,5,5], wk_temporal [H*d,5], wv_spatial, wv_temporal), float32 CUDA tensors.
        `out` = optional (q_out, k_out, v_out); q_out may be q itself.  q may be None: the queries are then left
        to the read-out (forward(..., q_l2_eps=l2_eps)) and the first element of the result is None.
        """
        torch = self._torch
        if k is None or k.dim() != 5:
            raise ValueError("k must have shape [B, T, F, H, d]")
        B, T, F, H, d = (int(n) for n in k.shape)
        names = ("wk_spatial", "wk_temporal", "wv_spatial", "wv_temporal")
        given = [n for n in names if filters.get(n) is not None]      # spatial filters may be left out (identity)
        for n, x in (("q", q), ("k", k), ("v", v)):
            if x is not None:
                _require(n, x, (B, T, F, H, d), self.torch_dtype, True, self.device)
        for n in given:
            want = (H * d, 5, 5) if n.endswith("spatial") else (H * d, 5)
            _require(n, filters[n], want, torch.float32, True, self.device)
        qo, ko, vo = out if out is not None else (torch.empty_like(q) if q is not None else None,
                                                  torch.empty_like(k), torch.empty_like(v))
        for n, x in (("q_out", qo), ("k_out", ko), ("v_out", vo)):
            if x is not None:
                _require(n, x, (B, T, F, H, d), self.torch_dtype, True, self.device)
        p = lambda x: ctypes.c_void_p(x.data_ptr()) if x is not None else None
        prm = VdnPrepParams(ctypes.sizeof(VdnPrepParams), Y, X, 1 if anchors else 0, l2_eps,
                            *(filters[n].data_ptr() if filters.get(n) is not None else None for n in names))
        self._check(self.lib.vdn_vda_prepare(self.h, p(q), p(k), p(v), p(qo), p(ko), p(vo), B, T, F, H, d,
                                             ctypes.byref(prm), self._stream(stream)))
        return qo, ko, vo

    # -- token-wise rule, rotary positions ----------------------------------------------------
    def _streams(self, stream):
        """(handle of the call's stream, the stream where it is not the current one)."""
        torch = self._torch
        here = _current_raw_stream(torch, self.device)
        if stream is None or stream.cuda_stream == here:
            return here, None
        return stream.cuda_stream, stream

    def _new(self, streams, shape, dtype):
        """Memory made for a call: taken on the call's stream, so that the allocator does not hand it on while the call still
        runs; where that is not the current stream, what the caller gets back is marked as in use there too."""
        torch = self._torch
        if streams[1] is None:
            return torch.empty(shape, dtype=dtype, device=self._dev)
        with torch.cuda.stream(streams[1]):
            x = torch.empty(shape, dtype=dtype, device=self._dev)
        x.record_stream(torch.cuda.current_stream(self.device))
        return x

    def _new_like(self, streams, x):
        """_new for a checked input's shape and type (a microsecond less where that is dense)."""
        if streams[1] is None and x.is_contiguous():
            return self._torch.empty_like(x)
        return self._new(streams, x.shape, x.dtype)

    def _new_beside(self, streams, x, shape, dtype):
        """_new where a checked input lies (a little less to work out)."""
        return x.new_empty(shape, dtype=dtype) if streams[1] is None else self._new(streams, shape, dtype)

    def token_scan(self, q, k, v, beta, log_alpha=None, cu_seqlens=None, s0=None, out=None, state=None, scale=1.0,
                   l2_eps=0.0, stream=None):
        """vdn_vda_token_scan: the gated delta rule over packed sequences.  Returns (out, state).

        q, k [N,Hk,d], v [N,H,d], beta, log_alpha [N,H] (float), cu_seqlens int32 [S+1] (CUDA; None: one sequence of all N
        rows), s0 [S,H,d,d] (float, state before each sequence).  state [S,H,d,d] after each sequence, in s0's orientation
        and that of forward(s0=...); `state` may be s0 itself.  Rows behind the last sequence are not written: a fresh `out`
        holds whatever was there.  Kernels are chosen for the average length: a long sequence among many short ones is faster in a
        call of its own.
        """
        torch, dev = self._torch, self.device
        lead, H, Hk, st = validate_token_args(self.torch_dtype, self.d, dev, q, k, v, beta, out, log_alpha)
        if len(lead) != 1:
            raise ValueError("v must have shape [tokens, heads, d]")
        n, d, S = lead[0], self.d, 1
        if cu_seqlens is not None:
            if cu_seqlens.dim() != 1 or cu_seqlens.numel() < 2:
                raise ValueError("cu_seqlens must have shape [sequences + 1]")
            S = cu_seqlens.numel() - 1
            _dense("cu_seqlens", cu_seqlens, (S + 1,), torch.int32, True, dev)
        shape = (S, H, d, d)
        if s0 is not None:
            _dense("s0", s0, shape, torch.float32, True, dev)
        streams = self._streams(stream)
        if out is None:
            out = self._new_like(streams, v)
        if state is None:
            state = self._new(streams, shape, torch.float32) if s0 is None else self._new_like(streams, s0)
        else:
            _dense("state", state, shape, torch.float32, True, dev)
        prm = _TOKEN_PARAMS.pack(_TOKEN_PARAMS.size, H, Hk, S, scale, l2_eps, _ptr(cu_seqlens), 0, _ptr(log_alpha), _ptr(s0),
                                 state.data_ptr(), 0, *st)
        need = self.lib.vdn_vda_token_scan_workspace_bytes(self.h, n, prm)
        ws = self._new(streams, (need,), torch.uint8) if need else None
        r = self.lib.vdn_vda_token_scan(self.h, q.data_ptr(), k.data_ptr(), v.data_ptr(), beta.data_ptr(), out.data_ptr(), n, prm,
                                        _ptr(ws), need, streams[0])
        if r:
            self._check(r)
        return out, state

    def token_step(self, q, k, v, beta, state, log_alpha=None, index=None, out=None, scale=1.0, l2_eps=0.0, stream=None):
        """vdn_vda_token_step: the same rule for one token or a few of each request; `state` is updated in place.

        q, k [R,Hk,d] or [R,L,Hk,d] for R requests of L tokens, v [.., H,d], beta, log_alpha [.., H]; state [slots,H,d,d]
        (float); index int32 [R] (CUDA): each request's slot, None: request r has slot r.  Requests with an index outside
        the pool are padding: their rows of `out` are not written.
        """
        torch, dev = self._torch, self.device
        lead, H, Hk, st = validate_token_args(self.torch_dtype, self.d, dev, q, k, v, beta, out, log_alpha)
        if len(lead) > 2 or (len(lead) == 2 and lead[1] == 0):
            raise ValueError("v must have shape [requests, heads, d] or [requests, tokens, heads, d]")
        R, per, d = lead[0], lead[1] if len(lead) == 2 else 1, self.d
        if state is None or state.dim() != 4:
            raise ValueError("state must have shape [slots, heads, d, d]")
        slots = state.shape[0]
        _dense("state", state, (slots, H, d, d), torch.float32, True, dev)
        if index is not None:
            _dense("index", index, (R,), torch.int32, True, dev)
        streams = self._streams(stream)
        if out is None:
            out = self._new_like(streams, v)
        prm = _TOKEN_PARAMS.pack(_TOKEN_PARAMS.size, H, Hk, 0, scale, l2_eps, 0, _ptr(index), _ptr(log_alpha), 0, state.data_ptr(),
                                 slots, *st)
        r = self.lib.vdn_vda_token_step(self.h, q.data_ptr(), k.data_ptr(), v.data_ptr(), beta.data_ptr(), out.data_ptr(), R, per,
                                        prm, streams[0])
        if r:
            self._check(r)
        return out

    def rotate(self, q, k, freq, axis, Y=None, X=None, t0=0, positions=None, half=False, inverse=False, q_weight=None,
               k_weight=None, norm_eps=0.0, out=None, stream=None):
        """vdn_vda_rotate: rotary positions on (time, height, width) for q [B,T,F,H,d] and k [B,T,F,Hk,d] (or None).

        freq [pairs] (float64) and axis [pairs] (int32, 0 time / 1 height / 2 width) as CUDA tensors (rotary_tables makes
        them).  Positions are (t0 + t, u // X, u % X) of token u of frame t, F = Y * X, or positions int32 [3, B*T*F].  With
        norm_eps > 0 each head is RMS-normalised first (weights [d], float).  `out` = optional (q_out, k_out); each may be
        its input.  Returns (q', k').
        """
        torch, dev, io = self._torch, self.device, self.torch_dtype
        if q is None or q.dim() != 5:
            raise ValueError("q must have shape [B, T, F, H, d]")
        shape = tuple(q.shape)
        B, T, F, H, d = shape
        qs, ks, Hk = _rows("q", q, shape, io, True, dev), 0, 0
        kshape = None
        if k is not None:
            if k.dim() != 5:
                raise ValueError("k must have shape [B, T, F, Hk, d]")
            Hk = k.shape[3]
            kshape = (B, T, F, Hk, d)
            ks = _rows("k", k, kshape, io, True, dev)
        if freq is None or freq.dim() != 1:
            raise ValueError("freq must have shape [pairs]")
        n = freq.shape[0]
        _dense("freq", freq, (n,), torch.float64, True, dev)
        _dense("axis", axis, (n,), torch.int32, True, dev)
        if positions is not None:
            _dense("positions", positions, (3, B * T * F), torch.int32, True, dev)
        elif Y is None or X is None:
            raise ValueError("either Y and X or positions are needed")
        if q_weight is not None:
            _dense("q_weight", q_weight, (d,), torch.float32, True, dev)
        if k_weight is not None:
            _dense("k_weight", k_weight, (d,), torch.float32, True, dev)
        qo, ko = out if out is not None else (None, None)
        streams = self._streams(stream)
        if qo is None:
            qo, qos = self._new_like(streams, q), H * d
        else:
            qos = _rows("q_out", qo, shape, io, True, dev)
        kos = Hk * d
        if k is None:
            if ko is not None:
                raise ValueError("out has keys, but there are none to rotate")
        elif ko is None:
            ko = self._new_like(streams, k)
        else:
            kos = _rows("k_out", ko, kshape, io, True, dev)
        prm = _ROTARY_PARAMS.pack(_ROTARY_PARAMS.size, (VDN_ROTARY_HALF if half else 0) | (VDN_ROTARY_INVERSE if inverse else 0),
                                  n, Hk, Y or 0, X or 0, t0, norm_eps, freq.data_ptr(), axis.data_ptr(), _ptr(positions),
                                  _ptr(q_weight), _ptr(k_weight), qs, ks, qos, kos)
        r = self.lib.vdn_vda_rotate(self.h, q.data_ptr(), _ptr(k), qo.data_ptr(), _ptr(ko), B, T, F, H, d, prm, streams[0])
        if r:
            self._check(r)
        return qo, ko

    # -- around the layer: 8-bit projections, attention to an encoder's states ------------------
    def quantize(self, x, rows=1, out=None, scale=None, stream=None):
        """vdn_vda_quantize: x [..., K] to (x8 [..., K] float8_e4m3fn, scale), a power of two for each block of 128 channels.

        rows = 1: a block is 128 channels of a row, scale [..., ceil(K/128)] (activations); rows = 128: 128 x 128 of x [N, K],
        scale [ceil(N/128), ceil(K/128)] (weights).  Rows of a fresh x8 begin at multiples of 16 bytes, as scaled_matmul wants them.
        """
        torch, dev = self._torch, self.device
        if rows not in (1, SCALE_BLOCK):
            raise ValueError("rows must be 1 or 128")
        if x is None or x.dim() < 1 or (rows != 1 and x.dim() != 2):
            raise ValueError("x must have shape " + ("[..., K]" if rows == 1 else "[N, K]"))
        shape = x.shape
        k = shape[-1]
        xs = k if _glance(x, shape, self.torch_dtype, True, dev) else _matrix("x", x, tuple(shape), self.torch_dtype, True, dev)
        n = 1
        for s in shape[:-1]:
            n *= s
        blocks = -(-k // SCALE_BLOCK)
        streams = self._streams(stream)
        pitch = -(-k // 16) * 16
        if out is None:
            if pitch == k and streams[1] is None and x.is_contiguous():
                out = torch.empty_like(x, dtype=torch.float8_e4m3fn)
            else:
                out = self._new(streams, (*shape[:-1], pitch), torch.float8_e4m3fn)
                if pitch != k:
                    out = out[..., :k]
        else:
            pitch = _matrix("out", out, tuple(shape), torch.float8_e4m3fn, True, dev, 16)
        want = (*shape[:-1], blocks) if rows == 1 else (-(-n // SCALE_BLOCK), blocks)
        if scale is None:
            scale = self._new_beside(streams, x, want, torch.float32)
        else:
            _dense("scale", scale, want, torch.float32, True, dev)
        prm = _QUANTIZE_PARAMS.pack(_QUANTIZE_PARAMS.size, rows, xs, pitch)
        r = self.lib.vdn_vda_quantize(self.h, x.data_ptr(), out.data_ptr(), scale.data_ptr(), n, k, prm, streams[0])
        if r:
            self._check(r)
        return out, scale

    def scaled_matmul(self, a, a_scale, w, w_scale, bias=None, add=None, out=None, stream=None):
        """vdn_vda_scaled_matmul: a w^T + bias + add of 8-bit operands with a scale for each block of 128; [..., N] in the handle's type.

        a [..., K] and w [N, K] float8_e4m3fn, rows at multiples of 16 bytes (quantize makes them so); a_scale [..., ceil(K/128)],
        w_scale [ceil(N/128), ceil(K/128)], bias [N] (float); add [..., N] in the handle's type, `out` may be `add`.
        """
        m, n, k, st = validate_matmul_args(self.torch_dtype, self.device, a, a_scale, w, w_scale, bias, add, out)
        streams = self._streams(stream)
        if out is None:
            out = self._new_beside(streams, a, (*a.shape[:-1], n), self.torch_dtype) if add is None else self._new_like(streams, add)
        prm = _MATMUL_PARAMS.pack(_MATMUL_PARAMS.size, 0, a_scale.data_ptr(), w_scale.data_ptr(), _ptr(bias), _ptr(add), *st)
        r = self.lib.vdn_vda_scaled_matmul(self.h, a.data_ptr(), w.data_ptr(), out.data_ptr(), m, n, k, prm, streams[0])
        if r:
            self._check(r)
        return out

    def cross_attention(self, q, k, v, cu_seqlens=None, lengths=None, mask=None, scale=None, out=None, lse=False, stream=None):
        """vdn_vda_cross_attention: softmax(scale q k^T) v of q [B, ..., H, d] over an encoder's states k, v [B, Lk, Hk, d].

        lengths int32 [B]: keys of each batch row (None: Lk); or cu_seqlens int32 [B + 1] with k, v packed [N, Hk, d]; mask bool
        [B, Lk] or [N]: False keys do not count, whatever they hold.  scale: None is d ** -0.5.  lse: True, or a float tensor
        [B, ..., H], returns (out, lse), the logarithm of the sum of exponentials (-inf, and out = 0, for a row without keys).
        """
        dev = self.device
        given = lse if hasattr(lse, "data_ptr") else None
        B, n, keys, H, Hk, st = validate_cross_args(self.torch_dtype, self.d, dev, q, k, v, cu_seqlens, lengths, mask, out, given)
        streams = self._streams(stream)
        if out is None:
            out = self._new_like(streams, q)
        if given is None and lse:
            given = self._new_beside(streams, q, q.shape[:-1], self._torch.float32)
        prm = _CROSS_PARAMS.pack(_CROSS_PARAMS.size, B, H, Hk, self.d ** -0.5 if scale is None else scale, 0, _ptr(cu_seqlens),
                                 _ptr(lengths), _ptr(mask), _ptr(given), *st)
        need = self.lib.vdn_vda_cross_attention_workspace_bytes(self.h, n, keys, prm)
        ws = self._new(streams, (need,), self._torch.uint8) if need else None
        r = self.lib.vdn_vda_cross_attention(self.h, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), n, keys, prm,
                                             _ptr(ws), need, streams[0])
        if r:
            self._check(r)
        return out if given is None else (out, given)

    def forward_host(self, q, k, v, beta, gate, out, stream=None, alpha=None, s0=None, chunk=1, radius=0,
                     anchors=False, gate_elem=None, norm_weight=None, q_l2_eps=0.0):
        """vdn_vda_forward_host(_opt) on HOST tensors (pinned recommended); `out` and every optional input are host
        tensors too.  The keyword arguments are those of forward()."""
        B, T, F, H, d = validate_layer_args(self.torch_dtype, self.d, self.device, q, k, v, beta, gate, out, alpha, s0,
                                            gate_elem, norm_weight, on_cuda=False)
        self.ensure_workspace(B, T, F, H, chunk)
        p = lambda x: ctypes.c_void_p(x.data_ptr()) if x is not None else None
        a = lambda x: x.data_ptr() if x is not None else None
        plain = (chunk, radius, bool(anchors)) == (1, 0, False) and gate is not None and not q_l2_eps and \
            all(x is None for x in (alpha, s0, gate_elem, norm_weight))
        opt = VdnOptions(ctypes.sizeof(VdnOptions), chunk, radius, 1 if anchors else 0, a(alpha), a(s0),
                         a(gate_elem), a(norm_weight), float(q_l2_eps), 0)
        self.ensure_staging(B, T, F, H, None if plain else opt)
        if plain:
            st = self.lib.vdn_vda_forward_host(self.h, p(q), p(k), p(v), p(beta), p(gate), p(out),
                                               B, T, F, H, d, self._stream(stream))
        else:
            st = self.lib.vdn_vda_forward_host_opt(self.h, p(q), p(k), p(v), p(beta), p(gate), p(out),
                                                   B, T, F, H, d, ctypes.byref(opt), self._stream(stream))
        self._check(st)
        return out

    # -- inspection ---------------------------------------------------------------------------
    def view(self, which: int, B, T, F, H):
        """A torch view of a workspace intermediate (valid after synchronising the stream)."""
        torch = self._torch
        off, size = ctypes.c_size_t(), ctypes.c_size_t()
        self._check(self.lib.vdn_vda_workspace_view(self.h, which, B, T, F, H, self.d,
                                                    ctypes.byref(off), ctypes.byref(size)))
        raw = self._ws[off.value: off.value + size.value]
        d = self.d
        if which == VIEW_STATS:
            return raw.view(torch.float32).view(B, H, T, 2 * d, d)
        if which == VIEW_INV_SPLIT:
            return raw.view(torch.bfloat16).view(B, H, T, 3, d, d)
        if which in (VIEW_READ_FWD, VIEW_READ_BWD):
            return raw.view(torch.bfloat16).view(B, H, T, d, d)
        if which == VIEW_COMP_M:
            return raw.view(torch.bfloat16).view(B * H, 2, -1, 3, d, d)
        if which == VIEW_COMP_J:
            return raw.view(torch.float32).view(B * H, 2, -1, d, d)
        return raw.view(torch.float32).view(B, H, T, d, d)

    def uses_tensor_cores(self) -> bool:
        """True when this handle runs the tcgen05 kernels (bf16 I/O, d = 128, plain-fp32 path not forced)."""
        off, size = ctypes.c_size_t(), ctypes.c_size_t()
        return self.lib.vdn_vda_workspace_view(self.h, VIEW_INV_SPLIT, 1, 1, 1, 1, self.d,
                                               ctypes.byref(off), ctypes.byref(size)) == VDN_OK

    def profile(self, enable: bool = True):
        """Start (and reset) or stop per-kernel CUDA-event timing of forward calls."""
        self._check(self.lib.vdn_vda_profile(self.h, 1 if enable else 0))

    def kernel_times(self):
        """[(kernel name, mean ms per launch, launches)] since profile(True); waits for the events."""
        n = 8
        names = (ctypes.c_char_p * n)()
        ms = (ctypes.c_float * n)()
        cnt = (ctypes.c_int * n)()
        got = self.lib.vdn_vda_kernel_times(self.h, n, names, ms, cnt)
        return [(names[i].decode(), float(ms[i]), int(cnt[i])) for i in range(got)]

    def launch_count(self) -> int:
        return int(self.lib.vdn_vda_last_launch_count(self.h))

    def status(self) -> int:
        return int(self.lib.vdn_vda_status(self.h))

    def clear_status(self) -> int:
        """Resets the sticky device-side status word; returns what it held."""
        return int(self.lib.vdn_vda_clear_status(self.h))

    def set_wait_limit_us(self, microseconds: int):
        """Longest single wait inside a kernel before its CTA gives up (default 2 s)."""
        self._check(self.lib.vdn_vda_set_wait_limit_us(self.h, int(microseconds)))

    def selftest_wait_expiry(self, limit_us: int = 1000, stream=None):
        """Enqueues the stand-alone kernel whose wait runs out (see vdn_vda_selftest_wait_expiry)."""
        self._check(self.lib.vdn_vda_selftest_wait_expiry(self.h, int(limit_us), self._stream(stream)))

    def selftest_marker(self) -> int:
        return int(self.lib.vdn_vda_selftest_marker(self.h))

    def close(self):
        if getattr(self, "h", None):
            self.lib.vdn_vda_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
