"""ctypes binding of libclt.so (include/clt.h).

Argument marshalling only: every step of the CLT train step runs in the HIP
kernels of the library.  torch is used for device memory and streams.  The
module-level functions carry the C names and take torch tensors; `CLTStep`
bundles a handle with its workspace and output buffers.

Importing this module without a built libclt.so raises: there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libclt.so")

CLT_OK = 0
DTYPE_F32, DTYPE_BF16 = 0, 1
INPUT_NATIVE, INPUT_INT8_ROWSCALE = 0, 1
DECODE_AUTO, DECODE_DENSE, DECODE_GATHER = 0, 1, 2

EXPORTS = ("clt_workspace_bytes", "clt_init", "clt_destroy", "clt_last_error", "clt_forward",
           "clt_loss", "clt_backward", "clt_adam_step", "clt_backward_adam_step", "clt_workspace_view",
           "clt_profile_enable", "clt_profile_num_kernels", "clt_profile_query", "clt_norm_accumulate",
           "clt_normalise", "clt_diag_mfma_loop", "clt_norm_accumulate_static", "clt_rms_norm",
           "clt_rms_norm_backward_workspace_bytes", "clt_rms_norm_backward", "clt_adamw_step", "clt_mx4_bytes",
           "clt_mx4_quantise", "clt_mx4_dequantise", "clt_mx4_product")


class CLTError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"libclt error {code}: {msg}")
        self.code = code


class clt_config(C.Structure):
    _fields_ = [("size", C.c_uint32), ("L", C.c_int32), ("d", C.c_int32), ("F", C.c_int32), ("B", C.c_int32),
                ("dtype", C.c_int32), ("input_format", C.c_int32), ("master_weights", C.c_int32),
                ("decode_mode", C.c_int32), ("log_threshold", C.c_int32), ("activation", C.c_int32), ("topk_k", C.c_int32),
                ("reuse_decoder_norms", C.c_int32),
                ("gather_density_threshold", C.c_float), ("list_backward_density_threshold", C.c_float),
                ("C", C.c_float),
                ("ste_bandwidth", C.c_float), ("beta1", C.c_float), ("beta2", C.c_float), ("adam_eps", C.c_float)]


class clt_tensors(C.Structure):
    _fields_ = [("W_enc", C.c_void_p), ("b_enc", C.c_void_p), ("theta", C.c_void_p),
                ("W_dec", C.c_void_p), ("b_dec", C.c_void_p)]


class clt_adamw_tensor(C.Structure):
    _fields_ = [("p", C.c_void_p), ("g", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p), ("m_scale", C.c_void_p),
                ("v_scale", C.c_void_p), ("master", C.c_void_p), ("n", C.c_int64), ("dtype", C.c_int32),
                ("grad_dtype", C.c_int32), ("state_bits", C.c_int32), ("weight_decay", C.c_float)]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it first (python -c 'import __graft_entry__ as g; g.build()')")
    lib = C.CDLL(LIB_PATH)
    vp, fp = C.c_void_p, C.c_void_p
    lib.clt_workspace_bytes.argtypes = [C.POINTER(clt_config), C.POINTER(C.c_size_t)]
    lib.clt_init.argtypes = [C.POINTER(vp), C.POINTER(clt_config), vp, C.c_size_t]
    lib.clt_destroy.argtypes = [vp]
    lib.clt_last_error.argtypes = [vp]
    lib.clt_last_error.restype = C.c_char_p
    lib.clt_forward.argtypes = [vp, vp] + [vp] * 12
    lib.clt_loss.argtypes = [vp, vp, vp, fp, fp, vp, vp, fp, C.c_float, C.c_float, fp, C.POINTER(C.c_float)]
    lib.clt_backward.argtypes = [vp, vp, vp, fp, fp, vp, vp, vp, C.POINTER(clt_tensors)]
    lib.clt_adam_step.argtypes = [vp, vp, C.c_int64, C.c_float] + [C.POINTER(clt_tensors)] * 5
    lib.clt_backward_adam_step.argtypes = [vp, vp, vp, fp, vp, vp, C.c_int64, C.c_float] + [C.POINTER(clt_tensors)] * 5
    lib.clt_workspace_view.argtypes = [vp, C.c_int, C.POINTER(vp), C.POINTER(C.c_size_t)]
    lib.clt_norm_accumulate.argtypes = [vp, vp, vp, fp, vp]
    lib.clt_normalise.argtypes = [vp, vp, vp, C.c_int64, vp, fp, vp, fp]
    lib.clt_profile_enable.argtypes = [vp, C.c_int]
    lib.clt_profile_num_kernels.argtypes = []
    lib.clt_profile_query.argtypes = [vp, C.c_int, C.POINTER(C.c_char_p), C.POINTER(C.c_double),
                                      C.POINTER(C.c_int64)]
    lib.clt_norm_accumulate_static.argtypes = [vp, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32, vp, fp, vp]
    lib.clt_diag_mfma_loop.argtypes = [vp, C.c_int, C.c_int, vp, C.c_size_t, vp, C.POINTER(C.c_double), C.POINTER(C.c_double)]
    i32, size_p = C.c_int32, C.POINTER(C.c_size_t)
    lib.clt_rms_norm.argtypes = [vp, i32, i32, i32, i32, vp, vp, fp, C.c_float, vp, vp, vp, fp, fp]
    lib.clt_rms_norm_backward_workspace_bytes.argtypes = [i32, i32, i32, size_p]
    lib.clt_rms_norm_backward.argtypes = [vp, i32, i32, i32, i32, vp, fp, fp, vp, vp, vp, fp, vp, C.c_size_t]
    lib.clt_adamw_step.argtypes = [vp, i32, C.POINTER(clt_adamw_tensor), C.c_int64, C.c_double, C.c_double, C.c_double,
                                   C.c_double, C.c_uint64]
    lib.clt_mx4_bytes.argtypes = [i32, i32, i32, size_p, size_p]
    lib.clt_mx4_quantise.argtypes = [vp, i32, i32, i32, i32, i32, i32, vp, fp, vp, vp]
    lib.clt_mx4_dequantise.argtypes = [vp, i32, i32, i32, i32, vp, vp, vp]
    lib.clt_mx4_product.argtypes = [vp, i32, i32, i32, i32, vp, vp, vp, vp, fp, fp, i32, vp]
    for n in EXPORTS:
        if n != "clt_last_error":
            getattr(lib, n).restype = C.c_int
    return lib


_lib = _load()

_TORCH_T = {DTYPE_F32: torch.float32, DTYPE_BF16: torch.bfloat16}


def _check(rc, handle=None):
    if rc != CLT_OK:
        raise CLTError(rc, _lib.clt_last_error(handle).decode())


def _stream(device=None):
    # (by its pointer: making a torch.cuda.Stream object of it takes 2.7 us of a call's 9)
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device() if device is None else device)


def _ptr(t, shape, dtype, name, optional=False):
    """Device pointer of a tensor after checking what the kernels assume."""
    if t is None:
        if optional:
            return None
        raise ValueError(f"{name} is required")
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous device tensor")
    if t.dtype != dtype or tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: expected {tuple(shape)} {dtype}, got {tuple(t.shape)} {t.dtype}")
    return t.data_ptr()


def make_config(L, d, F, B, dtype=DTYPE_BF16, input_format=INPUT_NATIVE, master_weights=False,
                decode_mode=DECODE_DENSE, gather_density_threshold=0.0045, C_=4.0, ste_bandwidth=0.05,
                beta1=0.9, beta2=0.999, adam_eps=1e-8, log_threshold=False, topk=None, reuse_decoder_norms=False,
                list_backward_density_threshold=0.0):
    """topk: None for JumpReLU, else k of the TopK activation.  reuse_decoder_norms: see include/clt.h (the caller
    promises that only clt_backward_adam_step writes W_dec between steps).  list_backward_density_threshold: AUTO
    mode's second threshold, for the backward through the decoder (0 = the same as gather_density_threshold)."""
    return clt_config(C.sizeof(clt_config), L, d, F, B, dtype, input_format, int(master_weights), decode_mode,
                      int(log_threshold), 0 if topk is None else 1, 0 if topk is None else int(topk),
                      int(reuse_decoder_norms), gather_density_threshold, list_backward_density_threshold, C_, ste_bandwidth,
                      beta1, beta2, adam_eps)


def clt_workspace_bytes(cfg: clt_config) -> int:
    n = C.c_size_t(0)
    _check(_lib.clt_workspace_bytes(C.byref(cfg), C.byref(n)))
    return n.value


class Handle:
    """A clt_handle plus the shapes needed to validate tensors on the Python side."""

    def __init__(self, cfg: clt_config, workspace: torch.Tensor):
        self.cfg = cfg
        self.workspace = workspace          # keeps the device memory alive
        h = C.c_void_p()
        _check(_lib.clt_init(C.byref(h), C.byref(cfg), workspace.data_ptr(), workspace.numel()))
        self.h = h
        self.T = _TORCH_T[cfg.dtype]
        self.TX = torch.int8 if cfg.input_format == INPUT_INT8_ROWSCALE else self.T
        L, d, F, B = cfg.L, cfg.d, cfg.F, cfg.B
        P = L * (L + 1) // 2
        self.shapes = {"x": (L, B, d), "y": (L, B, d), "scale": (L, B), "W_enc": (L, d, F), "b_enc": (L, F),
                       "theta": (L, F), "W_dec": (P, F, d), "b_dec": (L, d), "z": (L, B, F), "y_hat": (L, B, d)}

    def close(self):
        if self.h:
            _lib.clt_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def clt_init(cfg: clt_config, workspace: torch.Tensor) -> Handle:
    if workspace.dtype != torch.uint8 or not workspace.is_cuda or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 device tensor")
    return Handle(cfg, workspace)


def clt_norm_accumulate(H: Handle, a, norm_sum, a_scale=None):
    s = H.shapes
    rc = _lib.clt_norm_accumulate(H.h, _stream(), _ptr(a, s["x"], H.TX, "a"),
                                  _ptr(a_scale, s["scale"], torch.float32, "a_scale", True),
                                  _ptr(norm_sum, (H.cfg.L,), torch.float64, "norm_sum"))
    _check(rc, H.h)


def clt_norm_accumulate_static(a, norm_sum, a_scale=None):
    """clt_norm_accumulate without a handle or workspace (the library's own static scratch); a is [L,B,d] float32,
    bfloat16 or int8 (then a_scale [L,B] float32 is required)."""
    if a is None or a.dim() != 3:
        raise ValueError("a must be a [L, B, d] device tensor")
    L, B, d = a.shape
    int8 = a.dtype == torch.int8
    dt = DTYPE_F32 if a.dtype == torch.float32 else DTYPE_BF16
    if a.dtype not in (torch.float32, torch.bfloat16, torch.int8):
        raise ValueError(f"a: unsupported dtype {a.dtype}")
    rc = _lib.clt_norm_accumulate_static(_stream(), L, B, d, dt, INPUT_INT8_ROWSCALE if int8 else INPUT_NATIVE,
                                         _ptr(a, (L, B, d), a.dtype, "a"),
                                         _ptr(a_scale, (L, B), torch.float32, "a_scale", True),
                                         _ptr(norm_sum, (L,), torch.float64, "norm_sum"))
    _check(rc)


def clt_normalise(H: Handle, norm_sum, n_tokens, a_in=None, scale_in=None, a_out=None, scale_out=None):
    s, f32 = H.shapes, torch.float32
    rc = _lib.clt_normalise(H.h, _stream(), _ptr(norm_sum, (H.cfg.L,), torch.float64, "norm_sum"), int(n_tokens),
                            _ptr(a_in, s["x"], H.T, "a_in", True), _ptr(scale_in, s["scale"], f32, "scale_in", True),
                            _ptr(a_out, s["x"], H.T, "a_out", True), _ptr(scale_out, s["scale"], f32, "scale_out", True))
    _check(rc, H.h)


def clt_forward(H: Handle, x, W_enc, b_enc, theta, W_dec, b_dec, z, act_class, y_hat,
                pre=None, l0_per_layer=None, x_scale=None):
    s, f32 = H.shapes, torch.float32
    rc = _lib.clt_forward(
        H.h, _stream(), _ptr(x, s["x"], H.TX, "x"), _ptr(x_scale, s["scale"], f32, "x_scale", True),
        _ptr(W_enc, s["W_enc"], H.T, "W_enc"), _ptr(b_enc, s["b_enc"], f32, "b_enc"),
        _ptr(theta, s["theta"], f32, "theta"), _ptr(W_dec, s["W_dec"], H.T, "W_dec"),
        _ptr(b_dec, s["b_dec"], f32, "b_dec"), _ptr(z, s["z"], H.T, "z"), _ptr(pre, s["z"], H.T, "pre", True),
        _ptr(act_class, s["z"], torch.uint8, "act_class"), _ptr(y_hat, s["y_hat"], f32, "y_hat"),
        _ptr(l0_per_layer, (H.cfg.L,), torch.int32, "l0_per_layer", True))
    _check(rc, H.h)


def clt_loss(H: Handle, y, y_hat, z, lambda0, loss_dev, y_scale=None, to_host=False, lambda1=0.0, pre=None,
             theta=None):
    s, f32 = H.shapes, torch.float32
    host = (C.c_float * 4)() if to_host else None
    dead = lambda1 > 0.0
    rc = _lib.clt_loss(H.h, _stream(), _ptr(y, s["y"], H.TX, "y"), _ptr(y_scale, s["scale"], f32, "y_scale", True),
                       _ptr(y_hat, s["y_hat"], f32, "y_hat"), _ptr(z, s["z"], H.T, "z"),
                       _ptr(pre, s["z"], H.T, "pre", not dead), _ptr(theta, s["theta"], f32, "theta", not dead),
                       float(lambda0), float(lambda1), _ptr(loss_dev, (4,), f32, "loss_dev"), host)
    _check(rc, H.h)
    return tuple(host) if to_host else None


def _tensors(H: Handle, t: dict, name: str, matrix_dtype, matrices_only=False) -> clt_tensors:
    s, f32 = H.shapes, torch.float32
    out = clt_tensors()
    out.W_enc = _ptr(t["W_enc"], s["W_enc"], matrix_dtype, f"{name}.W_enc")
    out.W_dec = _ptr(t["W_dec"], s["W_dec"], matrix_dtype, f"{name}.W_dec")
    if not matrices_only:
        out.b_enc = _ptr(t["b_enc"], s["b_enc"], f32, f"{name}.b_enc")
        out.theta = _ptr(t["theta"], s["theta"], f32, f"{name}.theta")
        out.b_dec = _ptr(t["b_dec"], s["b_dec"], f32, f"{name}.b_dec")
    return out


def clt_backward(H: Handle, x, theta, W_dec, z, act_class, grads: dict, x_scale=None):
    s, f32 = H.shapes, torch.float32
    g = _tensors(H, grads, "grads", H.T)
    rc = _lib.clt_backward(H.h, _stream(), _ptr(x, s["x"], H.TX, "x"),
                           _ptr(x_scale, s["scale"], f32, "x_scale", True), _ptr(theta, s["theta"], f32, "theta"),
                           _ptr(W_dec, s["W_dec"], H.T, "W_dec"), _ptr(z, s["z"], H.T, "z"),
                           _ptr(act_class, s["z"], torch.uint8, "act_class"), C.byref(g))
    _check(rc, H.h)


def clt_adam_step(H: Handle, t: int, lr: float, params: dict, grads: dict, m: dict, v: dict, master: dict = None):
    f32 = torch.float32
    p = _tensors(H, params, "params", H.T)
    g = _tensors(H, grads, "grads", H.T)
    mm = _tensors(H, m, "m", f32)
    vv = _tensors(H, v, "v", f32)
    ms = _tensors(H, master, "master", f32, matrices_only=True) if master is not None else None
    rc = _lib.clt_adam_step(H.h, _stream(), int(t), float(lr), C.byref(p), C.byref(g), C.byref(mm), C.byref(vv),
                            C.byref(ms) if ms is not None else None)
    _check(rc, H.h)


def clt_backward_adam_step(H: Handle, x, z, act_class, t: int, lr: float, params: dict, grads: dict, m: dict, v: dict,
                           master: dict = None, x_scale=None):
    """grads must hold b_enc, theta, b_dec; W_enc / W_dec entries are optional (written when present)."""
    s, f32 = H.shapes, torch.float32
    p = _tensors(H, params, "params", H.T)
    mm = _tensors(H, m, "m", f32)
    vv = _tensors(H, v, "v", f32)
    ms = _tensors(H, master, "master", f32, matrices_only=True) if master is not None else None
    g = clt_tensors()
    g.b_enc = _ptr(grads["b_enc"], s["b_enc"], f32, "grads.b_enc")
    g.theta = _ptr(grads["theta"], s["theta"], f32, "grads.theta")
    g.b_dec = _ptr(grads["b_dec"], s["b_dec"], f32, "grads.b_dec")
    g.W_enc = _ptr(grads.get("W_enc"), s["W_enc"], H.T, "grads.W_enc", True)
    g.W_dec = _ptr(grads.get("W_dec"), s["W_dec"], H.T, "grads.W_dec", True)
    rc = _lib.clt_backward_adam_step(H.h, _stream(), _ptr(x, s["x"], H.TX, "x"),
                                     _ptr(x_scale, s["scale"], f32, "x_scale", True), _ptr(z, s["z"], H.T, "z"),
                                     _ptr(act_class, s["z"], torch.uint8, "act_class"), int(t), float(lr),
                                     C.byref(p), C.byref(g), C.byref(mm), C.byref(vv),
                                     C.byref(ms) if ms is not None else None)
    _check(rc, H.h)


# ---- around the training step: no handle ------------------------------------------------------------------------

def _device_of(t, name):
    """Device index of a call's first tensor.  The kernels run on the current device's current stream: it has to be there."""
    if t is None:
        raise ValueError(f"{name} is required")
    dev = t.get_device()
    if dev < 0:
        raise ValueError(f"{name} must be a contiguous device tensor")
    if dev != torch.cuda.current_device():
        raise ValueError(f"{name} is on cuda:{dev}, the current device is cuda:{torch.cuda.current_device()}")
    return dev


def _arg(t, dev, shape, dtype, name):
    """_ptr for a required tensor of a call on device `dev`."""
    if t is None:
        raise ValueError(f"{name} is required")
    if t.get_device() != dev or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous tensor on cuda:{dev}")
    if t.dtype != dtype or t.shape != shape:
        raise ValueError(f"{name}: expected {tuple(shape)} {dtype}, got {tuple(t.shape)} {t.dtype}")
    return t.data_ptr()


def _may(t, dev, shape, dtype, name):
    return None if t is None else _arg(t, dev, shape, dtype, name)


_TYPES = {torch.float32: DTYPE_F32, torch.bfloat16: DTYPE_BF16}


def _storage(t, name):
    """Type code of a native activation or matrix tensor [L, B, d], which sets the type of the call."""
    if t.dim() != 3 or t.dtype not in _TYPES:
        raise ValueError(f"{name}: expected a 3-dimensional float32 or bfloat16 tensor, got {tuple(t.shape)} {t.dtype}")
    return _TYPES[t.dtype]


def clt_rms_norm(x, weight, eps, y=None, q=None, q_scale=None, residual=None, h=None, rstd=None):
    """RMS norm of residual streams x (+ residual, the sum stored in h) into y and / or int8 codes q with row scales
    q_scale (include/clt.h).  x [L, B, d] float32 or bfloat16, weight [L, d] float32; rstd [L, B] for the backward pass."""
    dev = _device_of(x, "x")
    dt, T, s, f32 = _storage(x, "x"), x.dtype, x.shape, torch.float32
    L, B, d = s
    _check(_lib.clt_rms_norm(
        _stream(dev), L, B, d, dt, _arg(x, dev, s, T, "x"), _may(residual, dev, s, T, "residual"), _arg(weight, dev, (L, d), f32, "weight"), eps,
        _may(h, dev, s, T, "h"), _may(y, dev, s, T, "y"), _may(q, dev, s, torch.int8, "q"), _may(q_scale, dev, (L, B), f32, "q_scale"),
        _may(rstd, dev, (L, B), f32, "rstd")))


def clt_rms_norm_backward_workspace_bytes(L, B, d) -> int:
    n = C.c_size_t(0)
    _check(_lib.clt_rms_norm_backward_workspace_bytes(L, B, d, C.byref(n)))
    return n.value


def _room(t, dev):
    """(pointer, bytes) of an optional workspace."""
    if t is None:
        return None, 0
    if t.dtype != torch.uint8 or t.get_device() != dev or not t.is_contiguous():
        raise ValueError(f"workspace must be a contiguous uint8 tensor on cuda:{dev}")
    return t.data_ptr(), t.numel()


def clt_rms_norm_backward(h, weight, rstd, dy, dx, dweight=None, workspace=None, dh=None):
    """Gradients of clt_rms_norm; dx may be dy or dh.  workspace: uint8, clt_rms_norm_backward_workspace_bytes, with dweight."""
    dev = _device_of(h, "h")
    dt, T, s, f32 = _storage(h, "h"), h.dtype, h.shape, torch.float32
    L, B, d = s
    _check(_lib.clt_rms_norm_backward(
        _stream(dev), L, B, d, dt, _arg(h, dev, s, T, "h"), _arg(weight, dev, (L, d), f32, "weight"), _arg(rstd, dev, (L, B), f32, "rstd"),
        _arg(dy, dev, s, T, "dy"), _may(dh, dev, s, T, "dh"), _arg(dx, dev, s, T, "dx"), _may(dweight, dev, (L, d), f32, "dweight"),
        *_room(workspace, dev)))


ADAMW_BLOCK = 128


class AdamWTensor:
    """One tensor of clt_adamw_step: parameters p, gradient g (each float32 or bfloat16), moments m and v: float32, or uint8
    with the block scales m_scale and v_scale (uint8, one per 128 elements); master: float32 copy of p.  Any shape,
    contiguous; p, g, m, v and master have the same number of elements.  It stands for the tensors' present memory: one that is
    given other memory (a new p.data, a new p.grad) needs a new AdamWTensor."""

    def __init__(self, p, g, m, v, m_scale=None, v_scale=None, master=None, weight_decay=0.0):
        dev = _device_of(p, "p")
        n = p.numel()
        eight = m is not None and m.dtype == torch.uint8
        if p.dtype not in _TYPES or g is None or g.dtype not in _TYPES:
            raise ValueError("p and g must be float32 or bfloat16 tensors")
        if eight != (m_scale is not None) or eight != (v_scale is not None):
            raise ValueError("m_scale and v_scale belong to 8-bit (uint8) moments")
        state = torch.uint8 if eight else torch.float32
        for t, dt, name in ((p, p.dtype, "p"), (g, g.dtype, "g"), (m, state, "m"), (v, state, "v")):
            _arg(t, dev, t.shape if t is not None and t.numel() == n else (n,), dt, name)
        if master is not None:
            _arg(master, dev, master.shape if master.numel() == n else (n,), torch.float32, "master")
        blocks = ((n + ADAMW_BLOCK - 1) // ADAMW_BLOCK,)
        _may(m_scale, dev, blocks, torch.uint8, "m_scale")
        _may(v_scale, dev, blocks, torch.uint8, "v_scale")
        self.device = dev
        self.tensors = (p, g, m, v, m_scale, v_scale, master)
        # kept alive, whatever the tensors are given afterwards: the step works on this memory
        self.storages = tuple(t.untyped_storage() for t in self.tensors if t is not None)
        self.c = clt_adamw_tensor(*(None if t is None else t.data_ptr() for t in self.tensors), n, _TYPES[p.dtype], _TYPES[g.dtype],
                                  8 if eight else 32, float(weight_decay))


def clt_adamw_step(tensors, t, lr, beta1=0.9, beta2=0.999, eps=1e-8, seed=0):
    """One AdamW step over a list of AdamWTensor (include/clt.h)."""
    AdamW(tensors, beta1, beta2, eps, seed).step(t, lr)


class AdamW:
    """AdamW over a list of AdamWTensor that stays the same from step to step (a training loop checks it once)."""

    def __init__(self, tensors, beta1=0.9, beta2=0.999, eps=1e-8, seed=0):
        self.tensors = list(tensors)
        self.device = self.tensors[0].device if self.tensors else None
        if any(t.device != self.device for t in self.tensors):
            raise ValueError("the tensors are on different devices")
        # what a step writes (every tensor but the gradients) overlaps nothing else, such as a weight that is in the list twice
        spans = sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size(), k != 1) for x in self.tensors for k, t in enumerate(x.tensors)
                       if t is not None and t.numel())
        end, end_written = 0, 0      # of all spans so far, of the written ones
        for a, b, written in spans:
            if a < (end if written else end_written):
                raise ValueError("the tensors overlap in memory")
            end, end_written = max(end, b), max(end_written, b if written else 0)
        self._array = (clt_adamw_tensor * max(1, len(self.tensors)))(*(t.c for t in self.tensors))
        self.scalars = (float(beta1), float(beta2), float(eps), int(seed))

    @staticmethod
    def moments(p, bits=32):
        """Zero moments for a parameter: (m, v, m_scale, v_scale) of an AdamWTensor."""
        if bits == 32:
            return torch.zeros_like(p, dtype=torch.float32), torch.zeros_like(p, dtype=torch.float32), None, None
        if bits != 8:
            raise ValueError(f"moments are held in 32 or 8 bits, not {bits}")
        z = lambda *s: torch.zeros(s, dtype=torch.uint8, device=p.device)
        blocks = (p.numel() + ADAMW_BLOCK - 1) // ADAMW_BLOCK
        return z(*p.shape), z(*p.shape), z(blocks), z(blocks)

    def step(self, t, lr):
        if self.device is not None and torch.cuda.current_device() != self.device:
            raise ValueError(f"the tensors are on cuda:{self.device}, the current device is cuda:{torch.cuda.current_device()}")
        _check(_lib.clt_adamw_step(_stream(self.device), len(self.tensors), self._array, t, lr, *self.scalars))


def clt_mx4_bytes(L, rows, K):
    """(bytes of the codes, bytes of the scales) of a packed 4-bit matrix [L][rows][K]."""
    c, s = C.c_size_t(0), C.c_size_t(0)
    _check(_lib.clt_mx4_bytes(L, rows, K, C.byref(c), C.byref(s)))
    return c.value, s.value


def _mx4_shapes(L, rows, K):
    rp, ks = (rows + 63) // 64, (K + 127) // 128
    return (L, 4 * rp, ks, 1024), (L, rp, ks, 256)


def mx4_empty(L, rows, K, device="cuda:0"):
    """Room for a packed 4-bit matrix [L][rows][K]: (codes, scales), uint8."""
    clt_mx4_bytes(L, rows, K)
    codes, scales = _mx4_shapes(L, rows, K)
    return torch.empty(codes, dtype=torch.uint8, device=device), torch.empty(scales, dtype=torch.uint8, device=device)


def _packed(codes, scales, dev, L, rows, K, name):
    c, s = _mx4_shapes(L, rows, K)
    return _arg(codes, dev, c, torch.uint8, name + "codes"), _arg(scales, dev, s, torch.uint8, name + "scales")


def clt_mx4_quantise(a, codes, scales, a_scale=None, transposed=False):
    """Packs a [L, rows, K] (float32, bfloat16, or int8 with a_scale [L, rows]; transposed: [L, K, rows]) into 4 bits."""
    dev = _device_of(a, "a")
    if a.dtype == torch.int8:
        if a.dim() != 3:
            raise ValueError(f"a: expected a 3-dimensional tensor, got {tuple(a.shape)}")
        dt, fmt = DTYPE_BF16, INPUT_INT8_ROWSCALE
    else:
        dt, fmt = _storage(a, "a"), INPUT_NATIVE
    s = a.shape
    L, rows, K = (s[0], s[2], s[1]) if transposed else s
    _check(_lib.clt_mx4_quantise(_stream(dev), L, rows, K, dt, fmt, int(transposed), _arg(a, dev, s, a.dtype, "a"),
                                 _may(a_scale, dev, (L, rows), torch.float32, "a_scale"), *_packed(codes, scales, dev, L, rows, K, "")))


def clt_mx4_dequantise(codes, scales, out):
    """The values of a packed matrix into out [L, rows, K] float32 or bfloat16."""
    dev = _device_of(out, "out")
    dt, s = _storage(out, "out"), out.shape
    L, rows, K = s
    _check(_lib.clt_mx4_dequantise(_stream(dev), L, rows, K, dt, *_packed(codes, scales, dev, L, rows, K, ""), _arg(out, dev, s, out.dtype, "out")))


def clt_mx4_product(a_codes, a_scales, b_codes, b_scales, out, K, bias=None, theta=None):
    """out [L, M, N] = A B^T + bias of packed A [L][M][K] and B [L][N][K], with theta kept where above it, else 0 (a NaN too).
    theta is the threshold itself: of a step with log_threshold it is params["theta"].exp()."""
    dev = _device_of(out, "out")
    dt, s, f32 = _storage(out, "out"), out.shape, torch.float32
    L, M, N = s
    _check(_lib.clt_mx4_product(_stream(dev), L, M, N, K, *_packed(a_codes, a_scales, dev, L, M, K, "a_"), *_packed(b_codes, b_scales, dev, L, N, K, "b_"),
                                _may(bias, dev, (L, N), f32, "bias"), _may(theta, dev, (L, N), f32, "theta"), dt, _arg(out, dev, s, out.dtype, "out")))


_VIEWS = {"norms": (0, torch.float32, lambda c: (c.L, c.F)), "d_yhat": (1, None, lambda c: (c.L, c.B, c.d)),
          "dpre": (2, None, lambda c: (c.L, c.B, c.F)), "G": (3, torch.float32, lambda c: (c.L, c.F)),
          "decode_switch": (4, torch.int32, lambda c: (5,))}


def clt_workspace_view(H: Handle, which: str) -> torch.Tensor:
    """A tensor aliasing one of the workspace regions (norms, d_yhat, dpre, G)."""
    idx, dt, shp = _VIEWS[which]
    dt = dt or H.T
    ptr, nbytes = C.c_void_p(), C.c_size_t()
    _check(_lib.clt_workspace_view(H.h, idx, C.byref(ptr), C.byref(nbytes)), H.h)
    off = ptr.value - H.workspace.data_ptr()
    return H.workspace[off:off + nbytes.value].view(dt).view(shp(H.cfg))


def clt_profile_enable(H: Handle, on: bool):
    _check(_lib.clt_profile_enable(H.h, int(on)), H.h)


def clt_profile_query(H: Handle) -> dict:
    """{kernel name: (total device ms, launches)} since profiling was enabled."""
    out = {}
    for k in range(_lib.clt_profile_num_kernels()):
        name, ms, n = C.c_char_p(), C.c_double(), C.c_int64()
        _check(_lib.clt_profile_query(H.h, k, C.byref(name), C.byref(ms), C.byref(n)), H.h)
        out[name.value.decode()] = (ms.value, n.value)
    return out


DIAG_RANDOM_DATA, DIAG_LDS_READS, DIAG_LDS_WRITES, DIAG_LOADS_L2, DIAG_LOADS_FAR = 1, 2, 4, 8, 16


def clt_diag_mfma_loop(iters: int, mode: int, counters: torch.Tensor, buf: torch.Tensor = None):
    """Enqueues the diagnostic MFMA loop (see include/clt.h for the mode bits); returns (flop of the launch, rate
    of the constant-rate counter in Hz).  counters: int64 device tensor of 4 elements; [0] shader cycles, [1]
    constant-rate ticks of one wavefront.  buf: uint8 device scratch for the modes that load from memory."""
    flop, hz = C.c_double(), C.c_double()
    if buf is not None and (buf.dtype != torch.uint8 or not buf.is_cuda or not buf.is_contiguous()):
        raise ValueError("buf must be a contiguous uint8 device tensor")
    _check(_lib.clt_diag_mfma_loop(_stream(), int(iters), int(mode), buf.data_ptr() if buf is not None else None,
                                   buf.numel() if buf is not None else 0,
                                   _ptr(counters, (4,), torch.int64, "counters"), C.byref(flop), C.byref(hz)))
    return flop.value, hz.value


class CLTStep:
    """A handle with its workspace and the per-step buffers of one configuration."""

    def __init__(self, L, d, F, B, dtype="bf16", int8_inputs=False, master_weights=False, C_=4.0,
                 ste_bandwidth=0.05, beta1=0.9, beta2=0.999, adam_eps=1e-8, device="cuda:0", keep_pre=True,
                 decode_mode=DECODE_DENSE, gather_density_threshold=0.0045, matrix_grads=True, log_threshold=False,
                 topk=None, workspace=None, reuse_decoder_norms=False, list_backward_density_threshold=0.016):
        """workspace: a uint8 device tensor of at least clt_workspace_bytes(config) bytes that the caller
        owns (256-byte aligned); by default one is allocated here."""
        dt = DTYPE_BF16 if dtype == "bf16" else DTYPE_F32
        self.cfg = make_config(L, d, F, B, dt, INPUT_INT8_ROWSCALE if int8_inputs else INPUT_NATIVE,
                               master_weights, decode_mode, gather_density_threshold, C_, ste_bandwidth, beta1,
                               beta2, adam_eps, log_threshold, topk, reuse_decoder_norms,
                               list_backward_density_threshold)
        self.device = torch.device(device)
        ws = workspace
        if ws is None:
            ws = torch.empty(clt_workspace_bytes(self.cfg), dtype=torch.uint8, device=self.device)
        self.H = clt_init(self.cfg, ws)
        self.adam = (beta1, beta2, adam_eps)
        T = self.H.T
        P = L * (L + 1) // 2
        e = lambda *s, dtype=T: torch.empty(s, dtype=dtype, device=self.device)
        self.z = e(L, B, F)
        self.pre = e(L, B, F) if keep_pre else None
        self.act_class = e(L, B, F, dtype=torch.uint8)
        self.y_hat = e(L, B, d, dtype=torch.float32)
        self.l0 = e(L, dtype=torch.int32)
        self.loss_dev = e(4, dtype=torch.float32)
        self.grads = {"b_enc": e(L, F, dtype=torch.float32), "theta": e(L, F, dtype=torch.float32),
                      "b_dec": e(L, d, dtype=torch.float32)}
        if matrix_grads:    # not needed by the fused backward + Adam path
            self.grads["W_enc"] = e(L, d, F)
            self.grads["W_dec"] = e(P, F, d)

    def workspace_fill(self, byte: int):
        """Overwrites the whole workspace (nothing in it is meant to outlive a step)."""
        self.H.workspace.fill_(byte)

    def forward(self, x, params, x_scale=None):
        clt_forward(self.H, x, params["W_enc"], params["b_enc"], params["theta"], params["W_dec"], params["b_dec"],
                    self.z, self.act_class, self.y_hat, self.pre, self.l0, x_scale)

    def loss(self, y, lambda0, y_scale=None, to_host=False, lambda1=0.0, params=None):
        """`params` (for its theta tensor) is needed only when the dead-feature term is on (lambda1 > 0)."""
        theta = params["theta"] if lambda1 > 0.0 else None
        pre = self.pre if lambda1 > 0.0 else None
        return clt_loss(self.H, y, self.y_hat, self.z, lambda0, self.loss_dev, y_scale, to_host, lambda1, pre, theta)

    def backward(self, x, params, x_scale=None):
        clt_backward(self.H, x, params["theta"], params["W_dec"], self.z, self.act_class, self.grads, x_scale)

    def adam_step(self, t, lr, params, m, v, master=None):
        clt_adam_step(self.H, t, lr, params, self.grads, m, v, master)

    def backward_adam_step(self, x, params, m, v, t, lr, master=None, x_scale=None):
        clt_backward_adam_step(self.H, x, self.z, self.act_class, t, lr, params, self.grads, m, v, master, x_scale)

    def adamw(self, params, bits=8, master=None, weight_decay=0.0, seed=0):
        """An AdamW over this step's gradients for train_step: moments of the matrices in 8 or 32 bits, beginning at zero, those
        of the vectors in 32; weight decay and master copies for the matrices.  Needs matrix_grads, and with master_weights a
        master of both matrices."""
        if "W_dec" not in self.grads:
            raise ValueError("adamw needs the matrices' gradients (matrix_grads=True)")
        matrices = ("W_enc", "W_dec")
        if self.cfg.master_weights and any((master or {}).get(k) is None for k in matrices):
            raise ValueError("master_weights: adamw needs the master copies of W_enc and W_dec")
        tensors = []
        for k, g in self.grads.items():
            matrix = k in matrices
            tensors.append(AdamWTensor(params[k], g, *AdamW.moments(params[k], bits if matrix else 32), (master or {}).get(k) if matrix else None,
                                       weight_decay if matrix else 0.0))
        return AdamW(tensors, *self.adam, seed)

    def _check_optimiser(self, optimiser, params):
        """What an AdamW updates from this step's gradients has to be the parameters that the step reads."""
        mine = {g.data_ptr(): params[k].data_ptr() for k, g in self.grads.items()}
        held = [(t.c.g, t.c.p) for t in optimiser.tensors if t.c.g in mine]
        if not held:
            raise ValueError("the optimiser holds none of this step's gradients")
        if any(mine[g] != p for g, p in held):
            raise ValueError("the optimiser holds other parameters than the step is given")

    def train_step(self, x, y, params, m, v, t, lr, lambda0, master=None, x_scale=None, y_scale=None, fused=True,
                   lambda1=0.0, optimiser=None):
        """forward, loss, backward and Adam; `fused` runs Adam inside the weight-gradient GEMMs.  With an optimiser (see adamw) its
        step takes Adam's place: m, v, master and fused are not used, and what it updates from this step's gradients has to be params."""
        if isinstance(optimiser, AdamW):
            self._check_optimiser(optimiser, params)
        self.forward(x, params, x_scale)
        self.loss(y, lambda0, y_scale, False, lambda1, params)
        if optimiser is not None:
            self.backward(x, params, x_scale)
            optimiser.step(t, lr)
        elif fused:
            self.backward_adam_step(x, params, m, v, t, lr, master, x_scale)
        else:
            self.backward(x, params, x_scale)
            self.adam_step(t, lr, params, m, v, master)
