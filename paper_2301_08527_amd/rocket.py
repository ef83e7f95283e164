"""Python binding of librocket_mi355x.so (include/rocket.h), same names as the C ABI.

Argument marshalling only: every step of the transform runs in the HIP
library.  torch supplies device memory and the current stream.  There is no
CPU fallback: importing works without a GPU (kernel sampling is host code),
but the compute calls need the library and a device and fail loudly otherwise.
"""
import ctypes as C
import os

import numpy as np

ROCKET_F_MAX, ROCKET_F_PPV, ROCKET_F_SOFTPPV = 1, 2, 4
ROCKET_F32, ROCKET_BF16, ROCKET_F16 = 0, 1, 2
ROCKET_OK, ROCKET_EINVAL, ROCKET_ENOMEM, ROCKET_EHIP, ROCKET_ESHAPE, ROCKET_EWORKSPACE = 0, -1, -2, -3, -4, -5

_HERE = os.path.dirname(os.path.abspath(__file__))
# the in-tree library; the environment variable ROCKET_LIB names another build of it
LIB_PATH = os.environ.get("ROCKET_LIB") or os.path.join(_HERE, "librocket_mi355x.so")

EXPORTS = [
    "rocket_make_kernels", "rocket_kernels_import", "rocket_kernels_view_get",
    "rocket_kernels_set_params", "rocket_num_features", "rocket_workspace_bytes",
    "rocket_transform", "rocket_transform_noalloc", "rocket_soft_ppv_backward", "rocket_transform_u8", "rocket_soft_ppv_backward_u8",
    "rocket_work_per_series", "rocket_jobs_view_get",
    "rocket_profile_enable", "rocket_profile_read", "rocket_calibrate_fma", "rocket_calibrate_units",
    "rocket_ridge_workspace_bytes", "rocket_ridge_fit", "rocket_ridge_predict", "rocket_infer",
    "rocket_mse_grad", "rocket_sgd_update", "rocket_train_workspace_bytes", "rocket_train_step",
    "rocket_kernels_subset",
    "rocket_layer_norm_workspace_bytes", "rocket_layer_norm", "rocket_layer_norm_backward",
    "rocket_grad_workspace_bytes", "rocket_grad_norm", "rocket_grad_clip", "rocket_sgd_tensors", "rocket_sgd_update_clipped",
    "rocket_infer_normed_workspace_bytes", "rocket_infer_normed", "rocket_train_normed_workspace_bytes",
    "rocket_train_step_normed",
    "rocket_minirocket_kernels", "rocket_minirocket_fit_workspace_bytes", "rocket_minirocket_fit_bias",
    "rocket_minirocket_workspace_bytes", "rocket_minirocket_transform", "rocket_minirocket_transform_u8",
    "rocket_minirocket_jobs_view_get",
    "rocket_free_kernels", "rocket_last_error",
]


class RocketError(RuntimeError):
    def __init__(self, code, message):
        super().__init__("rocket error %d: %s" % (code, message))
        self.code = code


class _View(C.Structure):
    _fields_ = [
        ("K", C.c_int32), ("C", C.c_int32), ("L", C.c_int32),
        ("total_channels", C.c_int64), ("total_weights", C.c_int64),
        ("length", C.POINTER(C.c_int32)), ("dilation", C.POINTER(C.c_int32)),
        ("padding", C.POINTER(C.c_int32)), ("n_ch", C.POINTER(C.c_int32)),
        ("bias", C.POINTER(C.c_float)),
        ("ch_off", C.POINTER(C.c_int64)), ("w_off", C.POINTER(C.c_int64)),
        ("channels", C.POINTER(C.c_int32)), ("weights", C.POINTER(C.c_float)),
    ]


_lib = None


def load_library():
    """Loads the in-tree library; builds it first only if it is absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        from . import build as _build
        _build.build()
    lib = C.CDLL(LIB_PATH)
    vp, i32, u32, u64, f32 = C.c_void_p, C.c_int32, C.c_uint32, C.c_uint64, C.c_float
    lib.rocket_make_kernels.argtypes = [u64, i32, i32, i32, C.POINTER(vp)]
    lib.rocket_kernels_import.argtypes = [i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, C.POINTER(vp)]
    lib.rocket_kernels_view_get.argtypes = [vp, C.POINTER(_View)]
    lib.rocket_kernels_set_params.argtypes = [vp, vp, vp]
    lib.rocket_num_features.argtypes = [u32]
    lib.rocket_num_features.restype = i32
    lib.rocket_workspace_bytes.argtypes = [vp, i32, u32, C.c_int]
    lib.rocket_workspace_bytes.restype = C.c_size_t
    lib.rocket_transform.argtypes = [vp, vp, i32, u32, f32, f32, vp, vp, C.c_size_t, vp]
    lib.rocket_transform_noalloc.argtypes = [vp, vp, i32, u32, f32, f32, vp, vp]
    lib.rocket_soft_ppv_backward.argtypes = [vp, vp, i32, u32, vp, f32, f32, C.c_int, vp, vp, vp, C.c_size_t, vp]
    lib.rocket_transform_u8.argtypes = lib.rocket_transform.argtypes
    lib.rocket_soft_ppv_backward_u8.argtypes = lib.rocket_soft_ppv_backward.argtypes
    lib.rocket_jobs_view_get.argtypes = [vp, C.POINTER(i32)] + [C.POINTER(C.POINTER(i32))] * 4 + [C.POINTER(i32)]
    lib.rocket_work_per_series.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(C.c_double)]
    lib.rocket_profile_enable.argtypes = [vp, C.c_int]
    lib.rocket_profile_read.argtypes = [vp, C.POINTER(i32), C.POINTER(C.c_double)]
    lib.rocket_calibrate_fma.argtypes = [C.POINTER(C.c_double), vp]
    lib.rocket_calibrate_units.argtypes = [C.POINTER(C.c_double), i32, vp]
    lib.rocket_ridge_workspace_bytes.argtypes = [i32, i32]
    lib.rocket_ridge_workspace_bytes.restype = C.c_size_t
    lib.rocket_ridge_fit.argtypes = [vp, vp, i32, i32, C.c_double, vp, vp, vp, C.c_size_t, vp]
    lib.rocket_ridge_predict.argtypes = [vp, i32, i32, vp, vp, vp, vp]
    lib.rocket_infer.argtypes = [vp, vp, C.c_int, i32, u32, f32, f32, vp, vp, vp, vp, vp, C.c_size_t, vp]
    lib.rocket_mse_grad.argtypes = [vp, vp, vp, i32, i32, vp, vp, vp]
    lib.rocket_sgd_update.argtypes = [vp, vp, vp, f32, C.c_int, vp]
    lib.rocket_train_workspace_bytes.argtypes = [vp, i32, u32]
    lib.rocket_train_workspace_bytes.restype = C.c_size_t
    lib.rocket_train_step.argtypes = [vp, vp, C.c_int, i32, u32, f32, f32, vp, vp, vp, f32, C.c_int, vp, vp,
                                      C.c_size_t, vp]
    lib.rocket_kernels_subset.argtypes = [vp, vp, i32, C.POINTER(vp)]
    f64, sz = C.c_double, C.c_size_t
    lib.rocket_layer_norm_workspace_bytes.argtypes = [i32, i32, i32, C.c_int]
    lib.rocket_layer_norm_workspace_bytes.restype = sz
    lib.rocket_layer_norm.argtypes = [vp, i32, i32, i32, i32, vp, vp, f32, vp, vp, vp, vp, sz, vp]
    lib.rocket_layer_norm_backward.argtypes = [vp, vp, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.rocket_grad_workspace_bytes.argtypes = [vp, i32]
    lib.rocket_grad_workspace_bytes.restype = sz
    lib.rocket_grad_norm.argtypes = [vp, i32, f64, vp, vp, sz, vp]
    lib.rocket_grad_clip.argtypes = [vp, vp, i32, f64, vp, vp, sz, vp]
    lib.rocket_sgd_tensors.argtypes = [vp, vp, vp, i32, f64, vp, vp]
    lib.rocket_sgd_update_clipped.argtypes = [vp, vp, vp, f32, C.c_int, vp, vp]
    for name in ("rocket_infer_normed_workspace_bytes", "rocket_train_normed_workspace_bytes"):
        getattr(lib, name).argtypes = [vp, i32, u32]
        getattr(lib, name).restype = sz
    lib.rocket_infer_normed.argtypes = [vp, vp, C.c_int, i32, u32, f32, f32, vp, vp, f32, vp, vp, vp, vp, vp, sz, vp]
    lib.rocket_train_step_normed.argtypes = [vp, vp, C.c_int, i32, u32, f32, f32, vp, vp, f32, vp, vp, vp, f32, C.c_int, f64,
                                             vp, vp, vp, sz, vp]
    lib.rocket_minirocket_kernels.argtypes = [u64, i32, i32, i32, C.POINTER(vp)]
    lib.rocket_minirocket_fit_workspace_bytes.argtypes = [vp, i32]
    lib.rocket_minirocket_fit_workspace_bytes.restype = C.c_size_t
    lib.rocket_minirocket_fit_bias.argtypes = [vp, vp, i32, u64, vp, C.c_size_t, vp]
    lib.rocket_minirocket_workspace_bytes.argtypes = [vp, i32]
    lib.rocket_minirocket_workspace_bytes.restype = C.c_size_t
    lib.rocket_minirocket_transform.argtypes = [vp, vp, i32, vp, vp, C.c_size_t, vp]
    lib.rocket_minirocket_transform_u8.argtypes = [vp, vp, i32, vp, vp, C.c_size_t, vp]
    lib.rocket_minirocket_jobs_view_get.argtypes = [vp, C.POINTER(i32), C.POINTER(C.POINTER(i32))]
    lib.rocket_free_kernels.argtypes = [vp]
    lib.rocket_free_kernels.restype = None
    lib.rocket_last_error.restype = C.c_char_p
    _lib = lib
    return lib


def rocket_last_error():
    return load_library().rocket_last_error().decode()


def _check(rc):
    if rc != ROCKET_OK:
        raise RocketError(rc, rocket_last_error())


def rocket_num_features(mask):
    return int(load_library().rocket_num_features(mask))


class Kernels:
    """Owns a rocket_kernels handle."""

    def __init__(self, handle):
        self._h = C.c_void_p(handle)
        # the sizes never change; keeping them here lets the compute wrappers check their
        # arguments without asking the library for a view (which, after a training update,
        # would wait for the device and download the parameters)
        v = _View()
        _check(load_library().rocket_kernels_view_get(self._h, C.byref(v)))
        self.K, self.C, self.L = int(v.K), int(v.C), int(v.L)
        self.total_channels, self.total_weights = int(v.total_channels), int(v.total_weights)

    @property
    def handle(self):
        if not self._h:
            raise RocketError(ROCKET_EINVAL, "kernels already freed")
        return self._h

    def free(self):
        if self._h:
            load_library().rocket_free_kernels(self._h)
            self._h = C.c_void_p(None)

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass


def rocket_make_kernels(seed, K, C_, L):
    out = C.c_void_p()
    _check(load_library().rocket_make_kernels(seed, K, C_, L, C.byref(out)))
    return Kernels(out.value)


def _np(a, dt):
    return np.ascontiguousarray(a, dtype=dt)


def rocket_kernels_import(K, C_, L, length, dilation, padding, bias, n_ch, channels, weights):
    arrs = [_np(length, np.int32), _np(dilation, np.int32), _np(padding, np.int32), _np(bias, np.float32),
            _np(n_ch, np.int32), _np(channels, np.int32), _np(weights, np.float32)]
    out = C.c_void_p()
    _check(load_library().rocket_kernels_import(K, C_, L, *[a.ctypes.data for a in arrs], C.byref(out)))
    return Kernels(out.value)


def rocket_kernels_view_get(kernels):
    """Copies of the handle's arrays, keyed like the C struct."""
    v = _View()
    _check(load_library().rocket_kernels_view_get(kernels.handle, C.byref(v)))
    K = v.K

    def arr(ptr, n, dt):
        return np.ctypeslib.as_array(ptr, shape=(n,)).astype(dt, copy=True) if n else np.zeros(0, dt)

    return {
        "K": K, "C": v.C, "L": v.L,
        "length": arr(v.length, K, np.int32), "dilation": arr(v.dilation, K, np.int32),
        "padding": arr(v.padding, K, np.int32), "n_ch": arr(v.n_ch, K, np.int32),
        "bias": arr(v.bias, K, np.float32),
        "ch_off": arr(v.ch_off, K + 1, np.int64), "w_off": arr(v.w_off, K + 1, np.int64),
        "channels": arr(v.channels, v.total_channels, np.int32),
        "weights": arr(v.weights, v.total_weights, np.float32),
    }


def rocket_kernels_set_params(kernels, weights=None, bias=None):
    w = None if weights is None else _np(weights, np.float32)
    b = None if bias is None else _np(bias, np.float32)
    _check(load_library().rocket_kernels_set_params(
        kernels.handle, None if w is None else w.ctypes.data, None if b is None else b.ctypes.data))


def rocket_workspace_bytes(kernels, B, feature_mask, backward=False):
    return int(load_library().rocket_workspace_bytes(kernels.handle, B, feature_mask, int(bool(backward))))


def rocket_jobs_view_get(kernels):
    """dict of int32 arrays (copies): kernel, row0, row1, flags of every job, in launch order."""
    n, stride = C.c_int32(), C.c_int32()
    ptrs = [C.POINTER(C.c_int32)() for _ in range(4)]
    _check(load_library().rocket_jobs_view_get(kernels.handle, C.byref(n), *[C.byref(p) for p in ptrs], C.byref(stride)))
    step = stride.value // 4
    out = {}
    for name, p in zip(("kernel", "row0", "row1", "flags"), ptrs):
        out[name] = np.ctypeslib.as_array(p, shape=(n.value * step,))[::step].copy()
    return out


def rocket_work_per_series(kernels):
    fma, outs = C.c_double(), C.c_double()
    _check(load_library().rocket_work_per_series(kernels.handle, C.byref(fma), C.byref(outs)))
    return fma.value, outs.value


def rocket_profile_enable(kernels, enable=True):
    _check(load_library().rocket_profile_enable(kernels.handle, int(bool(enable))))


def rocket_profile_read(kernels):
    """(launches, total milliseconds) of the dominant kernel since the last read."""
    n, ms = C.c_int32(), C.c_double()
    _check(load_library().rocket_profile_read(kernels.handle, C.byref(n), C.byref(ms)))
    return n.value, ms.value


def _torch():
    import torch
    if not torch.cuda.is_available():
        raise RocketError(ROCKET_EHIP, "no GPU visible: the transform has no CPU path")
    return torch


def _stream_ptr(torch, stream):
    s = torch.cuda.current_stream() if stream is None else stream
    return C.c_void_p(s.cuda_stream)


def _workspace(torch, kernels, B, mask, backward, workspace, device):
    need = rocket_workspace_bytes(kernels, B, mask, backward)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
    return workspace, need


def rocket_transform(kernels, x, feature_mask, lam=10.0, shift=-3.0, out=None, workspace=None, stream=None,
                     _dtype="float32", _entry="rocket_transform"):
    """x: float32 CUDA tensor (B, C, L), contiguous.  Returns out (B, F*K)."""
    torch = _torch()
    if not (x.is_cuda and x.dtype == getattr(torch, _dtype) and x.is_contiguous() and x.dim() == 3):
        raise RocketError(ROCKET_EINVAL, "x must be a contiguous %s CUDA tensor of shape (B, C, L)" % _dtype)
    v = kernels
    B = x.shape[0]
    if x.shape[1] != v.C or x.shape[2] != v.L:
        raise RocketError(ROCKET_ESHAPE, "x is (B, %d, %d) but the kernels were made for (%d, %d)"
                          % (x.shape[1], x.shape[2], v.C, v.L))
    F = rocket_num_features(feature_mask)
    if out is None:
        out = torch.empty((B, max(F, 1) * v.K), dtype=torch.float32, device=x.device)
    workspace, _ = _workspace(torch, kernels, B, feature_mask, False, workspace, x.device)
    _check(getattr(load_library(), _entry)(
        kernels.handle, x.data_ptr(), B, feature_mask, lam, shift, out.data_ptr(),
        workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream_ptr(torch, stream)))
    return out


def rocket_transform_noalloc(kernels, x, feature_mask, out, lam=10.0, shift=-3.0, stream=None):
    """rocket_transform into `out` (float32 CUDA, (B, F*K)) with the library's resident workspace:
    nothing is allocated, here or in the library."""
    torch = _torch()
    if not (x.is_cuda and x.dtype == torch.float32 and x.is_contiguous() and x.dim() == 3):
        raise RocketError(ROCKET_EINVAL, "x must be a contiguous float32 CUDA tensor of shape (B, C, L)")
    B = x.shape[0]
    if x.shape[1] != kernels.C or x.shape[2] != kernels.L:
        raise RocketError(ROCKET_ESHAPE, "x does not match the kernels' (C, L)")
    F = rocket_num_features(feature_mask)
    if not (out.is_cuda and out.dtype == torch.float32 and out.is_contiguous() and tuple(out.shape) == (B, F * kernels.K)):
        raise RocketError(ROCKET_EINVAL, "out must be a contiguous float32 CUDA tensor of shape (B, F*K)")
    _check(load_library().rocket_transform_noalloc(kernels.handle, x.data_ptr(), B, feature_mask, lam, shift,
                                                   out.data_ptr(), _stream_ptr(torch, stream)))
    return out


def rocket_transform_u8(kernels, x_u8, feature_mask, lam=10.0, shift=-3.0, out=None, workspace=None, stream=None):
    """x_u8: uint8 CUDA tensor (B, C, L), contiguous; rows are z-normalised inside the call."""
    return rocket_transform(kernels, x_u8, feature_mask, lam, shift, out, workspace, stream,
                            _dtype="uint8", _entry="rocket_transform_u8")


def rocket_soft_ppv_backward(kernels, x, feature_mask, grad_out, lam=10.0, shift=-3.0, include_max=False,
                             grad_w=None, grad_b=None, workspace=None, stream=None,
                             _dtype="float32", _entry="rocket_soft_ppv_backward"):
    """Returns (grad_w [total_weights], grad_b [K]) as float32 CUDA tensors."""
    torch = _torch()
    for t, name, dt in ((x, "x", _dtype), (grad_out, "grad_out", "float32")):
        if not (t.is_cuda and t.dtype == getattr(torch, dt) and t.is_contiguous()):
            raise RocketError(ROCKET_EINVAL, "%s must be a contiguous %s CUDA tensor" % (name, dt))
    v = kernels
    B = x.shape[0]
    if x.dim() != 3 or x.shape[1] != v.C or x.shape[2] != v.L:
        raise RocketError(ROCKET_ESHAPE, "x does not match the kernels' (C, L)")
    F = rocket_num_features(feature_mask)
    if tuple(grad_out.shape) != (B, F * v.K):
        raise RocketError(ROCKET_ESHAPE, "grad_out must be (B, F*K)")
    if grad_w is None:
        grad_w = torch.empty(v.total_weights, dtype=torch.float32, device=x.device)
    if grad_b is None:
        grad_b = torch.empty(v.K, dtype=torch.float32, device=x.device)
    workspace, _ = _workspace(torch, kernels, B, feature_mask, True, workspace, x.device)
    _check(getattr(load_library(), _entry)(
        kernels.handle, x.data_ptr(), B, feature_mask, grad_out.data_ptr(), lam, shift, int(bool(include_max)),
        grad_w.data_ptr(), grad_b.data_ptr(), workspace.data_ptr(),
        workspace.numel() * workspace.element_size(), _stream_ptr(torch, stream)))
    return grad_w, grad_b


def rocket_soft_ppv_backward_u8(kernels, x_u8, feature_mask, grad_out, lam=10.0, shift=-3.0, include_max=False,
                                grad_w=None, grad_b=None, workspace=None, stream=None):
    """The backward pass on uint8 samples, z-normalised inside the call."""
    return rocket_soft_ppv_backward(kernels, x_u8, feature_mask, grad_out, lam, shift, include_max,
                                    grad_w, grad_b, workspace, stream,
                                    _dtype="uint8", _entry="rocket_soft_ppv_backward_u8")


def rocket_calibrate_fma(stream=None):
    """Measured plain-FMA rate of the current device in TFLOP/s."""
    torch = _torch()
    v = C.c_double()
    _check(load_library().rocket_calibrate_fma(C.byref(v), _stream_ptr(torch, stream)))
    return v.value


CAL_NAMES = ("load_b32_l1_GBps", "load_b32_l2_GBps", "load_b128_l1_GBps", "load_b128_l2_GBps",
             "load_b128_to_lds_GBps", "lds_read_b32_GBps", "mfma_f32_4x4x1_TFLOPs", "mfma_valu_serial_ratio",
             "conv_strip_valu_TFLOPs", "conv_strip_mfma_toeplitz_TFLOPs")


def rocket_calibrate_units(stream=None):
    """Measured rates of the load, LDS and matrix units of the current device, keyed by CAL_NAMES."""
    torch = _torch()
    v = (C.c_double * len(CAL_NAMES))()
    _check(load_library().rocket_calibrate_units(v, len(CAL_NAMES), _stream_ptr(torch, stream)))
    return dict(zip(CAL_NAMES, list(v)))


def rocket_ridge_workspace_bytes(n, p):
    return int(load_library().rocket_ridge_workspace_bytes(n, p))


def rocket_ridge_fit(features, targets, alpha, workspace=None, stream=None):
    """features: float32 CUDA (n, p); targets: float32 CUDA (n).  Returns (coef [p], intercept [1]) float64 CUDA."""
    torch = _torch()
    if not (features.is_cuda and features.dtype == torch.float32 and features.is_contiguous() and features.dim() == 2):
        raise RocketError(ROCKET_EINVAL, "features must be a contiguous float32 CUDA tensor (n, p)")
    n, p = features.shape
    if not (targets.is_cuda and targets.dtype == torch.float32 and targets.is_contiguous() and tuple(targets.shape) == (n,)):
        raise RocketError(ROCKET_EINVAL, "targets must be a contiguous float32 CUDA tensor (n,)")
    coef = torch.empty(p, dtype=torch.float64, device=features.device)
    intercept = torch.empty(1, dtype=torch.float64, device=features.device)
    if workspace is None:
        workspace = torch.empty(rocket_ridge_workspace_bytes(n, p), dtype=torch.uint8, device=features.device)
    _check(load_library().rocket_ridge_fit(features.data_ptr(), targets.data_ptr(), n, p, float(alpha), coef.data_ptr(),
                                           intercept.data_ptr(), workspace.data_ptr(),
                                           workspace.numel(), _stream_ptr(torch, stream)))
    return coef, intercept


def rocket_ridge_predict(features, coef, intercept, stream=None):
    """Returns float64 CUDA predictions (m,) for float32 CUDA features (m, p)."""
    torch = _torch()
    if not (features.is_cuda and features.dtype == torch.float32 and features.is_contiguous() and features.dim() == 2):
        raise RocketError(ROCKET_EINVAL, "features must be a contiguous float32 CUDA tensor (m, p)")
    m, p = features.shape
    if not (coef.is_cuda and coef.dtype == torch.float64 and coef.numel() == p and intercept.dtype == torch.float64):
        raise RocketError(ROCKET_EINVAL, "coef must be float64 CUDA of length p, intercept float64")
    pred = torch.empty(m, dtype=torch.float64, device=features.device)
    _check(load_library().rocket_ridge_predict(features.data_ptr(), m, p, coef.data_ptr(), intercept.data_ptr(),
                                               pred.data_ptr(), _stream_ptr(torch, stream)))
    return pred


def rocket_infer(kernels, x, feature_mask, coef, intercept, lam=10.0, shift=-3.0, features=None, workspace=None,
                 stream=None):
    """x: float32 or uint8 CUDA tensor (B, C, L).  Returns (pred float64 (B,), features float32 (B, F*K))."""
    torch = _torch()
    if not (x.is_cuda and x.dtype in (torch.float32, torch.uint8) and x.is_contiguous() and x.dim() == 3):
        raise RocketError(ROCKET_EINVAL, "x must be a contiguous float32 or uint8 CUDA tensor of shape (B, C, L)")
    v = kernels
    B = x.shape[0]
    if x.shape[1] != v.C or x.shape[2] != v.L:
        raise RocketError(ROCKET_ESHAPE, "x does not match the kernels' (C, L)")
    p = rocket_num_features(feature_mask) * v.K
    if not (coef.is_cuda and coef.dtype == torch.float64 and coef.numel() == p and coef.is_contiguous()
            and intercept.is_cuda and intercept.dtype == torch.float64 and intercept.numel() == 1):
        raise RocketError(ROCKET_EINVAL, "coef must be float64 CUDA of length F*K, intercept float64 CUDA of length 1")
    if features is None:
        features = torch.empty((B, max(p, 1)), dtype=torch.float32, device=x.device)
    pred = torch.empty(B, dtype=torch.float64, device=x.device)
    workspace, _ = _workspace(torch, kernels, B, feature_mask, False, workspace, x.device)
    _check(load_library().rocket_infer(
        kernels.handle, x.data_ptr(), int(x.dtype == torch.uint8), B, feature_mask, lam, shift,
        coef.data_ptr(), intercept.data_ptr(), features.data_ptr(), pred.data_ptr(),
        workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream_ptr(torch, stream)))
    return pred, features


def rocket_mse_grad(pred, targets, coef, grad_out=None, stream=None):
    """pred float64 (B,), targets float32 (B,), coef float64 (p,), all CUDA.
    Returns (grad_out float32 (B, p), loss float64 (1,))."""
    torch = _torch()
    B, p = pred.numel(), coef.numel()
    if not (pred.is_cuda and pred.dtype == torch.float64 and targets.is_cuda and targets.dtype == torch.float32
            and targets.numel() == B and coef.is_cuda and coef.dtype == torch.float64
            and pred.is_contiguous() and targets.is_contiguous() and coef.is_contiguous()):
        raise RocketError(ROCKET_EINVAL, "pred float64 (B,), targets float32 (B,), coef float64 (p,) CUDA tensors expected")
    if grad_out is None:
        grad_out = torch.empty((B, p), dtype=torch.float32, device=pred.device)
    loss = torch.empty(1, dtype=torch.float64, device=pred.device)
    _check(load_library().rocket_mse_grad(pred.data_ptr(), targets.data_ptr(), coef.data_ptr(), B, p,
                                          grad_out.data_ptr(), loss.data_ptr(), _stream_ptr(torch, stream)))
    return grad_out, loss


def rocket_sgd_update(kernels, grad_w, grad_b, lr, recentre=False, stream=None):
    torch = _torch()
    v = kernels
    for t, n, name in ((grad_w, v.total_weights, "grad_w"), (grad_b, v.K, "grad_b")):
        if not (t.is_cuda and t.dtype == torch.float32 and t.is_contiguous() and t.numel() == n):
            raise RocketError(ROCKET_EINVAL, "%s must be a contiguous float32 CUDA tensor of %d elements" % (name, n))
    _check(load_library().rocket_sgd_update(kernels.handle, grad_w.data_ptr(), grad_b.data_ptr(), lr,
                                            int(bool(recentre)), _stream_ptr(torch, stream)))


def rocket_train_workspace_bytes(kernels, B, feature_mask):
    return int(load_library().rocket_train_workspace_bytes(kernels.handle, B, feature_mask))


def rocket_train_step(kernels, x, feature_mask, coef, intercept, targets, lr, lam=10.0, shift=-3.0, recentre=False,
                      workspace=None, stream=None):
    """One gradient-descent step on the kernels' weights and biases.  Returns the loss before
    the update as a float64 CUDA tensor of one element."""
    torch = _torch()
    if not (x.is_cuda and x.dtype in (torch.float32, torch.uint8) and x.is_contiguous() and x.dim() == 3):
        raise RocketError(ROCKET_EINVAL, "x must be a contiguous float32 or uint8 CUDA tensor of shape (B, C, L)")
    v = kernels
    B = x.shape[0]
    if x.shape[1] != v.C or x.shape[2] != v.L:
        raise RocketError(ROCKET_ESHAPE, "x does not match the kernels' (C, L)")
    p = rocket_num_features(feature_mask) * v.K
    if not (coef.is_cuda and coef.dtype == torch.float64 and coef.numel() == p and coef.is_contiguous()
            and intercept.is_cuda and intercept.dtype == torch.float64 and intercept.numel() == 1
            and targets.is_cuda and targets.dtype == torch.float32 and targets.numel() == B
            and targets.is_contiguous()):
        raise RocketError(ROCKET_EINVAL, "coef float64 (F*K,), intercept float64 (1,), targets float32 (B,) CUDA expected")
    if workspace is None:
        workspace = torch.empty(rocket_train_workspace_bytes(kernels, B, feature_mask), dtype=torch.uint8,
                                device=x.device)
    loss = torch.empty(1, dtype=torch.float64, device=x.device)
    _check(load_library().rocket_train_step(
        kernels.handle, x.data_ptr(), int(x.dtype == torch.uint8), B, feature_mask, lam, shift,
        coef.data_ptr(), intercept.data_ptr(), targets.data_ptr(), lr, int(bool(recentre)), loss.data_ptr(),
        workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream_ptr(torch, stream)))
    return loss


# ------------------------------------------------------------------ layer norm, many tensors

_TYPE_CODES = {}


def _type_code(torch, dtype):
    if not _TYPE_CODES:
        _TYPE_CODES.update({torch.float32: ROCKET_F32, torch.bfloat16: ROCKET_BF16, torch.float16: ROCKET_F16})
    return _TYPE_CODES.get(dtype)


def _here(torch):
    """The current device."""
    try:
        return torch.cuda.current_device()
    except (RuntimeError, AssertionError) as e:
        raise RocketError(ROCKET_EHIP, "no GPU visible: these calls have no CPU path") from e


def _lists(here, *lists):
    """Refuses lists on another device than the current one."""
    for v in lists:
        if v is not None and v.index != here:
            raise RocketError(ROCKET_EINVAL, "tensors on cuda:%d: the current device is cuda:%d" % (v.index, here))


def _queue(torch, stream, here):
    """The hipStream_t of a call on device `here`.  (torch.cuda.current_stream makes an object first: 2.6 us of a call's 10.)"""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(here)
    if stream.device.index != here:
        raise RocketError(ROCKET_EINVAL, "a stream of %s: the current device is cuda:%d" % (stream.device, here))
    return stream.cuda_stream


def _empty(torch, shape, dtype, stream):
    """Memory of the current device that belongs to the stream it will be used on."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device="cuda")
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device="cuda")


def _scratch(torch, need, workspace, stream, here):
    """(address, bytes) of the workspace, and the tensor to keep until the call was made."""
    if workspace is None:
        if need == 0:
            return None, 0, None
        workspace = _empty(torch, need, torch.uint8, stream)
    elif not (workspace.get_device() == here and workspace.is_contiguous()):
        raise RocketError(ROCKET_EWORKSPACE, "workspace must be a contiguous CUDA tensor on the current device")
    return workspace.data_ptr(), workspace.nbytes, workspace


def _fits(t, like, dtype, name, here):
    """An output or input that has to have a shape, a type and the current device."""
    if not (t.get_device() == here and t.dtype is dtype and t.is_contiguous() and t.shape == like):
        raise RocketError(ROCKET_EINVAL, "%s must be a contiguous %s tensor of shape %s on the current device, cuda:%d"
                          % (name, dtype, tuple(like), here))


def _ptr(t):
    return None if t is None else t.data_ptr()


def _int32(value, name):
    """A size that the library takes in 32 bits; ctypes would drop the upper bits of a larger one and say nothing."""
    if not -2 ** 31 <= value < 2 ** 31:
        raise RocketError(ROCKET_ESHAPE, "%s = %d does not fit 32 bits" % (name, value))
    return value


def _norm_sizes(torch, x, planes, here):
    code = _type_code(torch, x.dtype)
    if not (code is not None and x.get_device() == here and x.is_contiguous() and x.dim() == 2):
        raise RocketError(ROCKET_EINVAL, "x must be a contiguous float32, bfloat16 or float16 tensor (rows, planes * n) on the current "
                          "device, cuda:%d" % here)
    rows, wide = x.shape
    if planes < 1 or rows < 1 or wide < 1 or wide % planes:
        raise RocketError(ROCKET_ESHAPE, "x (%d, %d) is not rows of %d planes" % (rows, wide, planes))
    _int32(planes, "planes")
    return code, _int32(rows, "rows"), _int32(wide // planes, "n")


def rocket_layer_norm_workspace_bytes(rows, planes, n, backward=True):
    return int(load_library().rocket_layer_norm_workspace_bytes(_int32(rows, "rows"), _int32(planes, "planes"), _int32(n, "n"),
                                                                int(bool(backward))))


def rocket_layer_norm(x, weight=None, bias=None, eps=1e-5, planes=1, y=None, mean=None, rstd=None, workspace=None, stream=None):
    """x: (rows, planes * n), float32, bfloat16 or float16; weight, bias: float32 (planes * n,).  Every plane of a row is
    normalised by itself.  Returns y (x's type); mean and rstd, float32 (rows, planes), are written for the backward pass
    where both are given."""
    import torch
    here = _here(torch)
    code, rows, n = _norm_sizes(torch, x, planes, here)
    if weight is not None:
        _fits(weight, (planes * n,), torch.float32, "weight", here)
    if bias is not None:
        _fits(bias, (planes * n,), torch.float32, "bias", here)
    if mean is not None:
        _fits(mean, (rows, planes), torch.float32, "mean", here)
    if rstd is not None:
        _fits(rstd, (rows, planes), torch.float32, "rstd", here)
    if y is not None:
        _fits(y, x.shape, x.dtype, "y", here)
    queue = _queue(torch, stream, here)
    if y is None:
        y = _empty(torch, x.shape, x.dtype, stream)
    ws, size, keep = _scratch(torch, rocket_layer_norm_workspace_bytes(rows, planes, n, False), workspace, stream, here)
    _check(load_library().rocket_layer_norm(x.data_ptr(), code, rows, planes, n, _ptr(weight), _ptr(bias), eps, y.data_ptr(),
                                            _ptr(mean), _ptr(rstd), ws, size, queue))
    return y


def rocket_layer_norm_backward(x, grad_y, mean, rstd, weight=None, planes=1, grad_x=None, grad_weight=None, grad_bias=None,
                               workspace=None, stream=None, param_grads=True):
    """Returns (grad_x of x's type, grad_weight, grad_bias float32 (planes * n,)).  grad_x may be grad_y.  param_grads=False
    leaves out what grad_weight and grad_bias are not given for (None is returned for it): a norm that is not trained."""
    import torch
    here = _here(torch)
    code, rows, n = _norm_sizes(torch, x, planes, here)
    _fits(grad_y, x.shape, x.dtype, "grad_y", here)
    _fits(mean, (rows, planes), torch.float32, "mean", here)
    _fits(rstd, (rows, planes), torch.float32, "rstd", here)
    if weight is not None:
        _fits(weight, (planes * n,), torch.float32, "weight", here)
    if grad_x is not None:
        _fits(grad_x, x.shape, x.dtype, "grad_x", here)
    if grad_weight is not None:
        _fits(grad_weight, (planes * n,), torch.float32, "grad_weight", here)
    if grad_bias is not None:
        _fits(grad_bias, (planes * n,), torch.float32, "grad_bias", here)
    queue = _queue(torch, stream, here)
    if grad_x is None:
        grad_x = _empty(torch, x.shape, x.dtype, stream)
    if grad_weight is None and param_grads:
        grad_weight = _empty(torch, (planes * n,), torch.float32, stream)
    if grad_bias is None and param_grads:
        grad_bias = _empty(torch, (planes * n,), torch.float32, stream)
    need = 0 if workspace is not None else rocket_layer_norm_workspace_bytes(rows, planes, n, True)
    ws, size, keep = _scratch(torch, need, workspace, stream, here)
    _check(load_library().rocket_layer_norm_backward(
        x.data_ptr(), grad_y.data_ptr(), code, rows, planes, n, _ptr(weight), mean.data_ptr(), rstd.data_ptr(), grad_x.data_ptr(),
        _ptr(grad_weight), _ptr(grad_bias), ws, size, queue))
    return grad_x, grad_weight, grad_bias


class Tensors:
    """A list of CUDA tensors as the library reads it (rocket_tensor records).  It keeps the tensors alive and holds the
    addresses they have when it is made: make a new one after a tensor's memory was replaced."""

    def __init__(self, tensors):
        import torch
        self.tensors = list(tensors)
        if not self.tensors:
            raise RocketError(ROCKET_EINVAL, "a list holds one tensor at least")
        ts, index = self.tensors, self.tensors[0].get_device()
        _type_code(torch, torch.float32)
        codes = [_TYPE_CODES.get(t.dtype) for t in ts]
        usable = [t.is_cuda and t.is_contiguous() and t.get_device() == index for t in ts]
        if None in codes or False in usable:
            i = next(i for i, (c, u) in enumerate(zip(codes, usable)) if c is None or not u)
            raise RocketError(ROCKET_EINVAL, "tensor %d must be a contiguous float32, bfloat16 or float16 CUDA tensor on one device" % i)
        self._records = np.empty((len(ts), 3), np.int64)      # address, count, type (and the reserved half)
        self._records[:, 0] = [t.data_ptr() for t in ts]
        self._records[:, 1] = [t.numel() for t in ts]
        self._records[:, 2] = codes
        self.index = index
        self.address = self._records.ctypes.data

    def __len__(self):
        return len(self.tensors)


def rocket_tensors(tensors):
    """The list that rocket_grad_norm, rocket_grad_clip and rocket_sgd_tensors take: made once where a program keeps its
    tensors (they also take a plain list, and then make it at every call)."""
    return tensors if isinstance(tensors, Tensors) else Tensors(tensors)


def rocket_grad_workspace_bytes(grads):
    grads = rocket_tensors(grads)
    return int(load_library().rocket_grad_workspace_bytes(grads.address, len(grads)))


def _norm_out(torch, norm, stream, here):
    if norm is None:
        return _empty(torch, 2, torch.float64, stream)
    _fits(norm, (2,), torch.float64, "norm", here)
    return norm


def rocket_grad_norm(grads, max_norm=float("inf"), norm=None, workspace=None, stream=None):
    """Returns norm, float64 (2,): the norm over all values of all gradients, and the coefficient min(1, max_norm / norm)."""
    import torch
    grads, here = rocket_tensors(grads), _here(torch)
    _lists(here, grads)
    queue = _queue(torch, stream, here)
    norm = _norm_out(torch, norm, stream, here)
    need = 0 if workspace is not None else rocket_grad_workspace_bytes(grads)
    ws, size, keep = _scratch(torch, need, workspace, stream, here)
    _check(load_library().rocket_grad_norm(grads.address, len(grads), max_norm, norm.data_ptr(), ws, size, queue))
    return norm


def _same_length(a, b):
    if len(a) != len(b):
        raise RocketError(ROCKET_ESHAPE, "lists of %d and %d tensors" % (len(a), len(b)))


def rocket_grad_clip(grads, max_norm, out=None, norm=None, workspace=None, stream=None):
    """Scales the gradients (in place, or into `out`) so that their norm is at most max_norm.  Returns norm as
    rocket_grad_norm does."""
    import torch
    grads, here = rocket_tensors(grads), _here(torch)
    if out is not None:
        out = rocket_tensors(out)
        _same_length(grads, out)
    _lists(here, grads, out)
    queue = _queue(torch, stream, here)
    norm = _norm_out(torch, norm, stream, here)
    need = 0 if workspace is not None else rocket_grad_workspace_bytes(grads)
    ws, size, keep = _scratch(torch, need, workspace, stream, here)
    _check(load_library().rocket_grad_clip(grads.address, None if out is None else out.address, len(grads), max_norm,
                                           norm.data_ptr(), ws, size, queue))
    return norm


def rocket_sgd_tensors(params, grads, lr, norm=None, out=None, stream=None):
    """params (or `out`) = params - lr * norm[1] * grads; norm as rocket_grad_norm returns it, or None: not clipped."""
    import torch
    params, grads, here = rocket_tensors(params), rocket_tensors(grads), _here(torch)
    _same_length(params, grads)
    if out is not None:
        out = rocket_tensors(out)
        _same_length(params, out)
    _lists(here, params, grads, out)
    if norm is not None:
        _fits(norm, (2,), torch.float64, "norm", here)
    queue = _queue(torch, stream, here)
    _check(load_library().rocket_sgd_tensors(params.address, grads.address, None if out is None else out.address, len(params), lr,
                                             _ptr(norm), queue))


def rocket_sgd_update_clipped(kernels, grad_w, grad_b, lr, norm, recentre=False, stream=None):
    """rocket_sgd_update with lr * norm[1]; norm as rocket_grad_norm returns it."""
    import torch
    here = _here(torch)
    _fits(grad_w, (kernels.total_weights,), torch.float32, "grad_w", here)
    _fits(grad_b, (kernels.K,), torch.float32, "grad_b", here)
    _fits(norm, (2,), torch.float64, "norm", here)
    queue = _queue(torch, stream, here)
    _check(load_library().rocket_sgd_update_clipped(kernels.handle, grad_w.data_ptr(), grad_b.data_ptr(), lr, int(bool(recentre)),
                                                    norm.data_ptr(), queue))


def _normed_inputs(torch, kernels, x, feature_mask, norm_weight, norm_bias, coef, intercept, here):
    if not (x.get_device() == here and x.dtype in (torch.float32, torch.uint8) and x.is_contiguous() and x.dim() == 3):
        raise RocketError(ROCKET_EINVAL, "x must be a contiguous float32 or uint8 tensor of shape (B, C, L) on the current device, cuda:%d" % here)
    if x.shape[1] != kernels.C or x.shape[2] != kernels.L:
        raise RocketError(ROCKET_ESHAPE, "x does not match the kernels' (C, L)")
    p = rocket_num_features(feature_mask) * kernels.K
    for t, name in ((norm_weight, "norm_weight"), (norm_bias, "norm_bias")):
        if t is not None:
            _fits(t, (p,), torch.float32, name, here)
    _fits(coef, (p,), torch.float64, "coef", here)
    _fits(intercept, (1,), torch.float64, "intercept", here)
    return _int32(x.shape[0], "B"), p


def rocket_infer_normed(kernels, x, feature_mask, norm_weight, norm_bias, coef, intercept, eps=1e-5, lam=10.0, shift=-3.0,
                        features=None, workspace=None, stream=None):
    """rocket_infer with a layer norm of every feature plane before the head.  norm_weight, norm_bias: float32 (F*K,) or
    None.  Returns (pred float64 (B,), the normalised features float32 (B, F*K))."""
    import torch
    here = _here(torch)
    B, p = _normed_inputs(torch, kernels, x, feature_mask, norm_weight, norm_bias, coef, intercept, here)
    if features is not None:
        _fits(features, (B, p), torch.float32, "features", here)
    queue = _queue(torch, stream, here)
    if features is None:
        features = _empty(torch, (B, p), torch.float32, stream)
    pred = _empty(torch, B, torch.float64, stream)
    need = int(load_library().rocket_infer_normed_workspace_bytes(kernels.handle, B, feature_mask))
    ws, size, keep = _scratch(torch, need, workspace, stream, here)
    _check(load_library().rocket_infer_normed(
        kernels.handle, x.data_ptr(), int(x.dtype == torch.uint8), B, feature_mask, lam, shift, _ptr(norm_weight), _ptr(norm_bias), eps,
        coef.data_ptr(), intercept.data_ptr(), features.data_ptr(), pred.data_ptr(), ws, size, queue))
    return pred, features


def rocket_infer_normed_workspace_bytes(kernels, B, feature_mask):
    return int(load_library().rocket_infer_normed_workspace_bytes(kernels.handle, _int32(B, "B"), feature_mask))


def rocket_train_normed_workspace_bytes(kernels, B, feature_mask):
    return int(load_library().rocket_train_normed_workspace_bytes(kernels.handle, _int32(B, "B"), feature_mask))


def rocket_train_step_normed(kernels, x, feature_mask, norm_weight, norm_bias, coef, intercept, targets, lr, max_norm=float("inf"),
                             eps=1e-5, lam=10.0, shift=-3.0, recentre=False, norm=None, workspace=None, stream=None):
    """One clipped gradient-descent step on the kernels and, in place, on norm_weight and norm_bias (float32 (F*K,)).
    Returns (loss before the update, float64 (1,), norm as rocket_grad_norm returns it)."""
    import torch
    here = _here(torch)
    B, p = _normed_inputs(torch, kernels, x, feature_mask, norm_weight, norm_bias, coef, intercept, here)
    if norm_weight is None or norm_bias is None:
        raise RocketError(ROCKET_EINVAL, "norm_weight and norm_bias are trained: both are needed")
    _fits(targets, (B,), torch.float32, "targets", here)
    queue = _queue(torch, stream, here)
    norm = _norm_out(torch, norm, stream, here)
    loss = _empty(torch, 1, torch.float64, stream)
    need = rocket_train_normed_workspace_bytes(kernels, B, feature_mask)
    ws, size, keep = _scratch(torch, need, workspace, stream, here)
    _check(load_library().rocket_train_step_normed(
        kernels.handle, x.data_ptr(), int(x.dtype == torch.uint8), B, feature_mask, lam, shift, norm_weight.data_ptr(),
        norm_bias.data_ptr(), eps, coef.data_ptr(), intercept.data_ptr(), targets.data_ptr(), lr, int(bool(recentre)), max_norm,
        loss.data_ptr(), norm.data_ptr(), ws, size, queue))
    return loss, norm


def rocket_kernels_subset(kernels, index):
    idx = np.ascontiguousarray(index, dtype=np.int32)
    out = C.c_void_p()
    _check(load_library().rocket_kernels_subset(kernels.handle, idx.ctypes.data_as(C.c_void_p), len(idx),
                                                C.byref(out)))
    return Kernels(out.value)


def rocket_minirocket_kernels(seed, groups, C_, L):
    out = C.c_void_p()
    _check(load_library().rocket_minirocket_kernels(seed, groups, C_, L, C.byref(out)))
    return Kernels(out.value)


def rocket_minirocket_fit_workspace_bytes(kernels, B):
    return int(load_library().rocket_minirocket_fit_workspace_bytes(kernels.handle, B))


def rocket_minirocket_fit_bias(kernels, x, seed, workspace=None, stream=None):
    """x: float32 CUDA tensor (B, C, L) of training series; sets the kernels' biases from it."""
    torch = _torch()
    if not (x.is_cuda and x.dtype == torch.float32 and x.is_contiguous() and x.dim() == 3):
        raise RocketError(ROCKET_EINVAL, "x must be a contiguous float32 CUDA tensor of shape (B, C, L)")
    if x.shape[1] != kernels.C or x.shape[2] != kernels.L:
        raise RocketError(ROCKET_ESHAPE, "x does not match the kernels' (C, L)")
    B = x.shape[0]
    if workspace is None:
        workspace = torch.empty(rocket_minirocket_fit_workspace_bytes(kernels, B), dtype=torch.uint8, device=x.device)
    _check(load_library().rocket_minirocket_fit_bias(kernels.handle, x.data_ptr(), B, seed, workspace.data_ptr(),
                                                     workspace.numel() * workspace.element_size(),
                                                     _stream_ptr(torch, stream)))


def rocket_minirocket_workspace_bytes(kernels, B):
    return int(load_library().rocket_minirocket_workspace_bytes(kernels.handle, B))


def rocket_minirocket_jobs_view_get(kernels):
    """(count, 8) int32 array (a copy): group, mode, first, count, col0, width, rows, 0 of every work item."""
    n = C.c_int32()
    p = C.POINTER(C.c_int32)()
    _check(load_library().rocket_minirocket_jobs_view_get(kernels.handle, C.byref(n), C.byref(p)))
    return np.ctypeslib.as_array(p, shape=(n.value, 8)).copy()


def rocket_minirocket_transform(kernels, x, out=None, workspace=None, stream=None, _dtype="float32",
                                _entry="rocket_minirocket_transform"):
    """x: float32 CUDA tensor (B, C, L); returns the (B, K) float32 PPV features of a MINIROCKET-style handle."""
    torch = _torch()
    if not (x.is_cuda and x.dtype == getattr(torch, _dtype) and x.is_contiguous() and x.dim() == 3):
        raise RocketError(ROCKET_EINVAL, "x must be a contiguous %s CUDA tensor of shape (B, C, L)" % _dtype)
    if x.shape[1] != kernels.C or x.shape[2] != kernels.L:
        raise RocketError(ROCKET_ESHAPE, "x does not match the kernels' (C, L)")
    B = x.shape[0]
    if out is None:
        out = torch.empty((B, kernels.K), dtype=torch.float32, device=x.device)
    if workspace is None:
        workspace = torch.empty(max(256, rocket_minirocket_workspace_bytes(kernels, B)), dtype=torch.uint8, device=x.device)
    _check(getattr(load_library(), _entry)(kernels.handle, x.data_ptr(), B, out.data_ptr(), workspace.data_ptr(),
                                           workspace.numel() * workspace.element_size(), _stream_ptr(torch, stream)))
    return out


def rocket_minirocket_transform_u8(kernels, x_u8, out=None, workspace=None, stream=None):
    """x_u8: uint8 CUDA tensor (B, C, L), contiguous; rows are z-normalised inside the call."""
    return rocket_minirocket_transform(kernels, x_u8, out, workspace, stream, _dtype="uint8",
                                       _entry="rocket_minirocket_transform_u8")


def rocket_free_kernels(kernels):
    kernels.free()
