"""Thin ctypes binding of libcert_b200.so (argument marshalling only).

Every step of the path runs in the library's CUDA kernels.  PyTorch is used
for device memory and streams.  There is no CPU fallback: if the library is
missing or cannot be loaded, import of this module raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
# CERT_LIB selects another build of the same library (the checking build of build.py), for tests
LIB_PATH = os.environ.get("CERT_LIB") or os.path.join(_HERE, "libcert_b200.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build it with `python -m paper_2507_20055_b200.build` "
        "(nvcc, sm_100a); there is no CPU fallback")

_lib = ctypes.CDLL(LIB_PATH)

CERT_OK = 0
CONTRACTION_AUTO, CONTRACTION_FFMA, CONTRACTION_TC3XTF32, CONTRACTION_TC3XFP16 = 0, 1, 2, 3

EXPORTS = [
    "cert_net_create", "cert_net_create_residual", "cert_deeppoly_bounds", "cert_backsub_bounds", "cert_deeppoly_bounds_host",
    "cert_backsub_bounds_host",
    "cert_net_destroy",
    "cert_net_num_neurons", "cert_net_num_relu_neurons", "cert_net_branch_codes",
    "cert_net_last_status", "cert_net_selftest_bounded_wait", "cert_net_set_contraction", "cert_net_last_launch_count",
    "cert_net_backstep_flops", "cert_status_string", "cert_net_set_profiling", "cert_net_profile",
    "cert_net_last_contraction_paths", "cert_first_layer_bounds_noalloc", "cert_net_set_conv_patches",
    "cert_net_enable_reusecert", "cert_reusecert_bounds", "cert_reusecert_bounds_host",
    "cert_net_check_guards", "cert_net_auto_contraction", "cert_net_fp16_coefficient_bound",
    "cert_peak_microbench", "cert_built_with_checked_stores", "cert_net_selftest_checked_store",
    "cert_xent_create", "cert_xent_run", "cert_xent_last_status", "cert_xent_check_guards", "cert_xent_destroy",
    "cert_clip_create", "cert_clip_run", "cert_clip_last_status", "cert_clip_check_guards", "cert_clip_destroy",
    "cert_int4_create", "cert_int4_matvec", "cert_int4_dequantize", "cert_int4_quantize", "cert_int4_last_status",
    "cert_int4_check_guards", "cert_int4_destroy",
]
CLASS_NAMES = ["input", "relax", "relu_step", "affine", "conv", "concretize"]


class cert_layer_desc_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in
                ("kind", "relu_after", "in_features", "out_features",
                 "c_in", "h_in", "w_in", "c_out", "kh", "kw", "stride", "pad")] + \
               [("weight", ctypes.c_void_p), ("bias", ctypes.c_void_p)]


_vp, _i, _f, _ll = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_longlong


class cert_xent_args_t(ctypes.Structure):
    _fields_ = [("rows", _i), ("target_is_64", _i), ("reduction", _i), ("grad_scale", _f), ("ignore_index", _ll),
                ("x", _vp), ("ldx", _ll), ("weight", _vp), ("ldw", _ll), ("bias", _vp), ("target", _vp),
                ("loss", _vp), ("row_losses", _vp), ("dx", _vp), ("lddx", _ll), ("dweight", _vp), ("lddw", _ll),
                ("dbias", _vp)]


class cert_tensor_t(ctypes.Structure):
    _fields_ = [("data", _vp), ("elements", _ll), ("type", _i)]


_lib.cert_net_create.argtypes = [ctypes.POINTER(cert_layer_desc_t), _i, _i, _f, _f, ctypes.POINTER(_vp)]
_lib.cert_net_create.restype = _i
_lib.cert_net_create_residual.argtypes = [ctypes.POINTER(cert_layer_desc_t), _i, _vp, _i, _f, _f, ctypes.POINTER(_vp)]
_lib.cert_net_create_residual.restype = _i
_lib.cert_deeppoly_bounds.argtypes = [_vp, _vp, _f, _i, _vp, _vp, _vp]
_lib.cert_deeppoly_bounds.restype = _i
_lib.cert_backsub_bounds.argtypes = [_vp, _vp, _f, _i, _vp, _vp, _vp, _vp]
_lib.cert_backsub_bounds.restype = _i
_lib.cert_backsub_bounds_host.argtypes = [_vp, _vp, _f, _i, _vp, _vp, _vp, _vp]
_lib.cert_backsub_bounds_host.restype = _i
_lib.cert_deeppoly_bounds_host.argtypes = [_vp, _vp, _f, _i, _vp, _vp, _vp]
_lib.cert_deeppoly_bounds_host.restype = _i
_lib.cert_net_destroy.argtypes = [_vp]
_lib.cert_net_destroy.restype = _i
_lib.cert_net_num_neurons.argtypes = [_vp]
_lib.cert_net_num_neurons.restype = _i
_lib.cert_net_num_relu_neurons.argtypes = [_vp]
_lib.cert_net_num_relu_neurons.restype = _i
_lib.cert_net_branch_codes.argtypes = [_vp, _vp, _vp]
_lib.cert_net_branch_codes.restype = _i
_lib.cert_net_last_status.argtypes = [_vp, _vp]
_lib.cert_net_last_status.restype = _i
_lib.cert_net_selftest_bounded_wait.argtypes = [_vp, _vp]
_lib.cert_net_selftest_bounded_wait.restype = _i
_lib.cert_net_set_contraction.argtypes = [_vp, _i]
_lib.cert_net_set_contraction.restype = _i
_lib.cert_net_last_launch_count.argtypes = [_vp]
_lib.cert_net_last_launch_count.restype = _i
_lib.cert_net_backstep_flops.argtypes = [_vp, _i]
_lib.cert_net_backstep_flops.restype = ctypes.c_double
_lib.cert_net_last_contraction_paths.argtypes = [_vp]
_lib.cert_net_last_contraction_paths.restype = _i
_lib.cert_net_enable_reusecert.argtypes = [_vp]
_lib.cert_net_enable_reusecert.restype = _i
_lib.cert_reusecert_bounds.argtypes = [_vp, _vp, _f, _i, _vp, _vp, _vp]
_lib.cert_reusecert_bounds.restype = _i
_lib.cert_reusecert_bounds_host.argtypes = [_vp, _vp, _f, _i, _vp, _vp, _vp]
_lib.cert_reusecert_bounds_host.restype = _i
_lib.cert_net_set_conv_patches.argtypes = [_vp, _i]
_lib.cert_net_set_conv_patches.restype = _i
_lib.cert_net_set_profiling.argtypes = [_vp, _i]
_lib.cert_net_set_profiling.restype = _i
_lib.cert_net_profile.argtypes = [_vp, _vp, _vp]
_lib.cert_net_profile.restype = _i
_lib.cert_first_layer_bounds_noalloc.argtypes = [_vp, _vp, _i, _i, _vp, _f, _f, _f, _i, _vp, _vp, _vp]
_lib.cert_first_layer_bounds_noalloc.restype = _i
_lib.cert_net_check_guards.argtypes = [_vp, _vp]
_lib.cert_net_check_guards.restype = _i
_lib.cert_net_auto_contraction.argtypes = [_vp]
_lib.cert_net_auto_contraction.restype = _i
_lib.cert_net_fp16_coefficient_bound.argtypes = [_vp, _i]
_lib.cert_net_fp16_coefficient_bound.restype = ctypes.c_float
_lib.cert_built_with_checked_stores.argtypes = []
_lib.cert_built_with_checked_stores.restype = _i
_lib.cert_net_selftest_checked_store.argtypes = [_vp, _vp]
_lib.cert_net_selftest_checked_store.restype = _i
_lib.cert_peak_microbench.argtypes = [_i, ctypes.c_double, _vp, _vp, _vp, _vp]
_lib.cert_peak_microbench.restype = _i
_lib.cert_xent_create.argtypes = [_i, _i, _i, _i, _i, ctypes.POINTER(_vp)]
_lib.cert_xent_run.argtypes = [_vp, ctypes.POINTER(cert_xent_args_t), _vp]
_lib.cert_xent_last_status.argtypes = [_vp, _vp]
_lib.cert_xent_check_guards.argtypes = [_vp, _vp]
_lib.cert_xent_destroy.argtypes = [_vp]
_lib.cert_clip_create.argtypes = [ctypes.POINTER(cert_tensor_t), _i, ctypes.POINTER(_vp), ctypes.POINTER(_vp)]
_lib.cert_clip_run.argtypes = [_vp, _f, _vp, _vp]
_lib.cert_clip_last_status.argtypes = [_vp, _vp]
_lib.cert_clip_check_guards.argtypes = [_vp, _vp]
_lib.cert_clip_destroy.argtypes = [_vp]
_lib.cert_int4_create.argtypes = [_vp, _vp, _vp, _i, _i, _i, _i, _vp, ctypes.POINTER(_vp)]
_lib.cert_int4_matvec.argtypes = [_vp, _vp, _ll, _i, _vp, _i, _vp, _ll, _vp]
_lib.cert_int4_dequantize.argtypes = [_vp, _vp, _vp]
_lib.cert_int4_quantize.argtypes = [_vp, _ll, _i, _i, _i, _i, _vp, _vp, _vp, _vp]
_lib.cert_int4_last_status.argtypes = [_vp, _vp]
_lib.cert_int4_check_guards.argtypes = [_vp, _vp]
_lib.cert_int4_destroy.argtypes = [_vp]
for _name in EXPORTS:
    if _name.startswith(("cert_xent_", "cert_clip_", "cert_int4_")):
        getattr(_lib, _name).restype = _i
_lib.cert_status_string.argtypes = [_i]
_lib.cert_status_string.restype = ctypes.c_char_p


class CertError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {_lib.cert_status_string(code).decode()} (status {code})")


def _check(code: int, where: str):
    if code != CERT_OK:
        raise CertError(code, where)


def marshal_layers(layers: Sequence):
    """ctypes array of cert_layer_desc_t from objects with kind/weight/bias/relu_after(/stride/pad/in_shape)."""
    arr = (cert_layer_desc_t * len(layers))()
    keep = []
    for i, l in enumerate(layers):
        w = np.ascontiguousarray(l.weight, dtype=np.float32)
        b = np.ascontiguousarray(l.bias, dtype=np.float32)
        keep += [w, b]
        d = arr[i]
        d.relu_after = int(bool(l.relu_after))
        d.weight, d.bias = w.ctypes.data, b.ctypes.data
        if l.kind == "fc":
            d.kind = 0
            d.out_features, d.in_features = w.shape
        elif l.kind == "conv":
            d.kind = 1
            d.c_out, d.c_in, d.kh, d.kw = w.shape
            _, d.h_in, d.w_in = l.in_shape
            d.stride, d.pad = int(l.stride), int(l.pad)
        else:
            raise ValueError(f"unknown layer kind {l.kind!r}")
    return arr, keep


def _check_tensor(name, t, shape, device=None):
    """The kernels take raw pointers: a wrong dtype, layout, shape or device would be an out-of-bounds access."""
    import torch
    if not (t.is_cuda and t.dtype == torch.float32 and t.is_contiguous()):
        raise ValueError(f"{name}: a contiguous float32 CUDA tensor is required")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    if device is not None and t.device != device:
        raise ValueError(f"{name}: on {t.device}, expected {device}")


class CertNet:
    """Owns a cert_net_t handle; the three calls of the C ABI plus the helpers."""

    def __init__(self, layers: Sequence, max_batch: int, clip_lo: float = 0.0, clip_hi: float = 1.0,
                 skip_from=None):
        """skip_from: residual connections, one entry per layer (-1 = none): cert_net_create_residual."""
        arr, keep = marshal_layers(layers)
        h = _vp()
        if skip_from is None:
            _check(_lib.cert_net_create(arr, len(layers), int(max_batch), float(clip_lo), float(clip_hi),
                                        ctypes.byref(h)), "cert_net_create")
        else:
            assert len(skip_from) == len(layers)
            skips = (ctypes.c_int * len(layers))(*[int(x) for x in skip_from])
            _check(_lib.cert_net_create_residual(arr, len(layers), ctypes.cast(skips, _vp), int(max_batch),
                                                 float(clip_lo), float(clip_hi), ctypes.byref(h)),
                   "cert_net_create_residual")
        self._h = h
        self.max_batch = int(max_batch)
        self.n0 = int(layers[0].n_in)
        self.n_total = int(_lib.cert_net_num_neurons(h))
        self.n_relu = int(_lib.cert_net_num_relu_neurons(h))
        self.n_layers = len(layers)

    # -- raw-pointer form (what the C ABI takes) --
    def deeppoly_bounds_ptr(self, centers_ptr: int, eps: float, batch: int, lb_ptr: int, ub_ptr: int,
                            stream_ptr: int = 0):
        _check(_lib.cert_deeppoly_bounds(self._h, centers_ptr, float(eps), int(batch), lb_ptr, ub_ptr,
                                         stream_ptr), "cert_deeppoly_bounds")

    # -- torch tensors on the device --
    def deeppoly_bounds(self, centers, eps: float, lb_out=None, ub_out=None, stream=None):
        import torch
        batch = centers.shape[0]
        _check_tensor("centers", centers, (batch, self.n0))
        if lb_out is None:
            lb_out = torch.empty((batch, self.n_total), dtype=torch.float32, device=centers.device)
        if ub_out is None:
            ub_out = torch.empty((batch, self.n_total), dtype=torch.float32, device=centers.device)
        _check_tensor("lb_out", lb_out, (batch, self.n_total), centers.device)
        _check_tensor("ub_out", ub_out, (batch, self.n_total), centers.device)
        st = stream if stream is not None else torch.cuda.current_stream(centers.device)
        self.deeppoly_bounds_ptr(centers.data_ptr(), eps, batch, lb_out.data_ptr(), ub_out.data_ptr(),
                                 st.cuda_stream)
        return lb_out, ub_out

    def backsub_bounds(self, centers, eps: float, backsteps=None, lb_out=None, ub_out=None, stream=None):
        """cert_backsub_bounds: backsteps = one traversal depth per affine layer (negative: to the input)."""
        import torch
        batch = centers.shape[0]
        _check_tensor("centers", centers, (batch, self.n0))
        if lb_out is None:
            lb_out = torch.empty((batch, self.n_total), dtype=torch.float32, device=centers.device)
        if ub_out is None:
            ub_out = torch.empty((batch, self.n_total), dtype=torch.float32, device=centers.device)
        _check_tensor("lb_out", lb_out, (batch, self.n_total), centers.device)
        _check_tensor("ub_out", ub_out, (batch, self.n_total), centers.device)
        st = stream if stream is not None else torch.cuda.current_stream(centers.device)
        steps = None
        if backsteps is not None:
            assert len(backsteps) == self.n_layers
            steps = (ctypes.c_int * self.n_layers)(*[int(x) for x in backsteps])
        _check(_lib.cert_backsub_bounds(self._h, centers.data_ptr(), float(eps), int(batch),
                                        ctypes.addressof(steps) if steps is not None else None,
                                        lb_out.data_ptr(), ub_out.data_ptr(), st.cuda_stream), "cert_backsub_bounds")
        return lb_out, ub_out

    def enable_reusecert(self):
        _check(_lib.cert_net_enable_reusecert(self._h), "cert_net_enable_reusecert")

    def reusecert_bounds(self, centers, eps: float, lb_out=None, ub_out=None, stream=None):
        """cert_reusecert_bounds (enable_reusecert() first)."""
        import torch
        batch = centers.shape[0]
        _check_tensor("centers", centers, (batch, self.n0))
        if lb_out is None:
            lb_out = torch.empty((batch, self.n_total), dtype=torch.float32, device=centers.device)
        if ub_out is None:
            ub_out = torch.empty((batch, self.n_total), dtype=torch.float32, device=centers.device)
        _check_tensor("lb_out", lb_out, (batch, self.n_total), centers.device)
        _check_tensor("ub_out", ub_out, (batch, self.n_total), centers.device)
        st = stream if stream is not None else torch.cuda.current_stream(centers.device)
        _check(_lib.cert_reusecert_bounds(self._h, centers.data_ptr(), float(eps), int(batch), lb_out.data_ptr(),
                                          ub_out.data_ptr(), st.cuda_stream), "cert_reusecert_bounds")
        return lb_out, ub_out

    def reusecert_bounds_host(self, centers: np.ndarray, eps: float, lb: np.ndarray, ub: np.ndarray,
                              stream_ptr: int = 0):
        centers = np.ascontiguousarray(centers, dtype=np.float32)
        _check(_lib.cert_reusecert_bounds_host(self._h, centers.ctypes.data, float(eps), centers.shape[0],
                                               lb.ctypes.data, ub.ctypes.data, stream_ptr),
               "cert_reusecert_bounds_host")
        return lb, ub

    def deeppoly_p_bounds(self, centers, eps: float, p: int, **kw):
        return self.backsub_bounds(centers, eps, [int(p)] * self.n_layers, **kw)

    def ibp_bounds(self, centers, eps: float, **kw):
        return self.backsub_bounds(centers, eps, [0] * self.n_layers, **kw)

    def crown_ibp_bounds(self, centers, eps: float, **kw):
        return self.backsub_bounds(centers, eps, [0] * (self.n_layers - 1) + [-1], **kw)

    # -- host numpy arrays (copies inside the library) --
    def deeppoly_bounds_host(self, centers: np.ndarray, eps: float, lb: Optional[np.ndarray] = None,
                             ub: Optional[np.ndarray] = None, stream_ptr: int = 0, backsteps=None):
        centers = np.ascontiguousarray(centers, dtype=np.float32)
        batch = centers.shape[0]
        if lb is None:
            lb = np.empty((batch, self.n_total), dtype=np.float32)
        if ub is None:
            ub = np.empty((batch, self.n_total), dtype=np.float32)
        steps = None
        if backsteps is not None:
            assert len(backsteps) == self.n_layers
            steps = (ctypes.c_int * self.n_layers)(*[int(x) for x in backsteps])
        _check(_lib.cert_backsub_bounds_host(self._h, centers.ctypes.data, float(eps), batch,
                                             ctypes.addressof(steps) if steps is not None else None,
                                             lb.ctypes.data, ub.ctypes.data, stream_ptr),
               "cert_backsub_bounds_host")
        return lb, ub

    def set_profiling(self, on: bool):
        _check(_lib.cert_net_set_profiling(self._h, int(bool(on))), "cert_net_set_profiling")

    def profile(self):
        """dict class name -> (ms, launches) of the most recent call (profiling must be on)."""
        ms = (ctypes.c_float * len(CLASS_NAMES))()
        cnt = (ctypes.c_int * len(CLASS_NAMES))()
        _check(_lib.cert_net_profile(self._h, ctypes.addressof(ms), ctypes.addressof(cnt)), "cert_net_profile")
        return {n: (float(ms[i]), int(cnt[i])) for i, n in enumerate(CLASS_NAMES)}

    def branch_codes(self, batch: int, stream=None):
        import torch
        if self.n_relu == 0:
            return torch.empty((batch, 0), dtype=torch.uint8, device="cuda")
        codes = torch.empty((batch, self.n_relu), dtype=torch.uint8, device="cuda")
        st = stream if stream is not None else torch.cuda.current_stream()
        _check(_lib.cert_net_branch_codes(self._h, codes.data_ptr(), st.cuda_stream), "cert_net_branch_codes")
        return codes

    def last_status(self, stream_ptr: int = 0) -> int:
        return int(_lib.cert_net_last_status(self._h, stream_ptr))

    def selftest_bounded_wait(self, stream_ptr: int = 0):
        """Enqueues a kernel whose (short) bounded wait runs out; last_status() then reports CERT_ERR_TIMEOUT."""
        _check(_lib.cert_net_selftest_bounded_wait(self._h, stream_ptr), "cert_net_selftest_bounded_wait")

    def set_contraction(self, mode: int):
        _check(_lib.cert_net_set_contraction(self._h, int(mode)), "cert_net_set_contraction")

    def set_conv_patches(self, on: bool):
        _check(_lib.cert_net_set_conv_patches(self._h, int(bool(on))), "cert_net_set_conv_patches")

    def selftest_checked_store(self, stream_ptr: int = 0):
        """Checking build only: one store just past a buffer, which is refused; last_status() then reports 8."""
        _check(_lib.cert_net_selftest_checked_store(self._h, stream_ptr), "cert_net_selftest_checked_store")

    def check_guards(self, stream_ptr: int = 0) -> int:
        """0 = every guard word around the net's device buffers is intact, i + 1 = allocation i was overrun."""
        return int(_lib.cert_net_check_guards(self._h, stream_ptr))

    def auto_contraction(self) -> int:
        return int(_lib.cert_net_auto_contraction(self._h))

    def fp16_coefficient_bound(self, layer: int = -1) -> float:
        return float(_lib.cert_net_fp16_coefficient_bound(self._h, int(layer)))

    def last_contraction_paths(self) -> int:
        return int(_lib.cert_net_last_contraction_paths(self._h))

    def last_launch_count(self) -> int:
        return int(_lib.cert_net_last_launch_count(self._h))

    def backstep_flops(self, batch: int) -> float:
        return float(_lib.cert_net_backstep_flops(self._h, int(batch)))

    def destroy(self):
        if getattr(self, "_h", None):
            _check(_lib.cert_net_destroy(self._h), "cert_net_destroy")
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def first_layer_bounds_noalloc(weight, bias, centers, eps, clip_lo, clip_hi, lb_out, ub_out, stream=None):
    """Interval bounds of one FC layer without any allocation inside the library.

    All tensors are the caller's torch CUDA tensors (float32, contiguous): weight [out, in],
    bias [out], centers [batch, in], lb_out / ub_out [batch, out].  For embedders that may not
    allocate device memory; see cert_first_layer_bounds_noalloc in cert.h for the limit and the
    rules on sharing.  Raises CertError on a bad argument or a batch beyond the built-in limit.
    """
    import torch
    out_features, in_features = weight.shape
    batch = centers.shape[0]
    for name, t, shape in (("weight", weight, (out_features, in_features)), ("bias", bias, (out_features,)),
                           ("centers", centers, (batch, in_features)), ("lb_out", lb_out, (batch, out_features)),
                           ("ub_out", ub_out, (batch, out_features))):
        _check_tensor(name, t, shape, weight.device)
    st = stream if stream is not None else torch.cuda.current_stream(weight.device)
    _check(_lib.cert_first_layer_bounds_noalloc(weight.data_ptr(), bias.data_ptr(), out_features, in_features,
                                                centers.data_ptr(), float(eps), float(clip_lo), float(clip_hi),
                                                centers.shape[0], lb_out.data_ptr(), ub_out.data_ptr(),
                                                st.cuda_stream), "cert_first_layer_bounds_noalloc")


def peak_microbench(kind: int, target_ms: float = 5.0, stream_ptr: int = 0):
    """cert_peak_microbench: (TFLOP/s, SM MHz seen by the kernel, ms) for kind 0 = tcgen05 f16, 1 = tcgen05 tf32,
    2 = fp32 FMA units; kind 3 = bulk copies from L2 into shared memory, first value in TB/s over all SMs."""
    out = (ctypes.c_double * 3)()
    base = ctypes.addressof(out)
    _check(_lib.cert_peak_microbench(int(kind), float(target_ms), base, base + 8, base + 16, stream_ptr),
           "cert_peak_microbench")
    return float(out[0]), float(out[1]), float(out[2])


# ---- operators next to the certifiers: training the networks, and running them as they are stored ----

TYPE_F32, TYPE_BF16, TYPE_F16 = 0, 1, 2


def _type_code(dtype):
    import torch
    codes = {torch.float32: TYPE_F32, torch.bfloat16: TYPE_BF16, torch.float16: TYPE_F16}
    if dtype not in codes:
        raise ValueError(f"type {dtype}: float32, bfloat16 or float16 is required")
    return codes[dtype]


def _int32(name, value):
    """A size as the C ABI takes it: ctypes would cut off what an int does not hold."""
    value = int(value)
    if not -2 ** 31 <= value < 2 ** 31:
        raise ValueError(f"{name}: {value} does not fit an int")
    return value


def _check_rows(name, t, shape, dtype, device):
    """A matrix whose rows may be any distance apart, the elements of a row next to each other."""
    if t.dtype is dtype and t.shape == shape and t.is_contiguous() and t.device == device:
        return
    if t.device != device or t.dtype != dtype:
        raise ValueError(f"{name}: a {dtype} tensor on {device} is required, got {t.dtype} on {t.device}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.dim() == 2 and t.shape[1] > 1 and t.stride(1) != 1 or t.dim() == 1 and t.shape[0] > 1 and t.stride(0) != 1:
        raise ValueError(f"{name}: the elements of a row have to lie next to each other")
    if t.dim() == 2 and t.shape[0] > 1 and t.stride(0) < t.shape[1]:
        raise ValueError(f"{name}: rows overlap (stride {t.stride(0)}, {t.shape[1]} elements)")


def _ld(t):
    """Elements from one row to the next; a matrix of one row may report anything."""
    rows, width = t.shape
    return t.stride(0) if rows > 1 else width


def _cuda_device(device):
    import torch
    d = torch.device("cuda") if device is None else torch.device(device)
    return torch.device("cuda", torch.cuda.current_device()) if d.type == "cuda" and d.index is None else d


def _empty(shape, dtype, device, stream, like=None):
    """Memory for an output: of the stream that will write it, so that it is not handed out again under the kernels.
    like: a contiguous tensor of this shape, type and device, if there is one (half the host's time)."""
    import torch
    if stream is not None:
        with torch.cuda.stream(stream):
            return torch.empty(shape, dtype=dtype, device=device)
    if like is not None and like.is_contiguous():
        return torch.empty_like(like)
    return torch.empty(*shape, dtype=dtype, device=device) if shape else torch.empty(shape, dtype=dtype, device=device)


def _call(device, function, *args):
    """The library's answer with `device` current: a handle belongs to one device, whose default stream is 0 like every other's."""
    global _current_device
    if _current_device is None:
        import torch
        _current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    if _current_device() == device.index:
        return function(*args)
    import torch
    with torch.cuda.device(device):
        return function(*args)


_current_device = None


def _stream_ptr(stream, device):
    """The stream's handle.  (The current stream's is looked up without making a Stream object, a third of a small call.)"""
    if stream is not None:
        if stream.device != device:
            raise ValueError(f"stream: of {stream.device}, the operator is on {device}")
        return stream.cuda_stream
    global _current_raw_stream
    if _current_raw_stream is None:
        import torch
        _current_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
            (lambda index: torch.cuda.current_stream(index).cuda_stream)
    return _current_raw_stream(device.index)


_current_raw_stream = None


class LinearCrossEntropy:
    """Softmax cross entropy of a linear layer over many classes and its gradient, without keeping the logits
    (cert_xent_*; formulas, ignored rows, masked classes and types in cert.h).

    Owns the workspace for up to max_rows rows; two calls on one object must not overlap on the device.
    """

    def __init__(self, max_rows: int, features: int, classes: int, dtype=None, grad: bool = True, device=None):
        import torch
        self.dtype = torch.float32 if dtype is None else dtype
        self.device = _cuda_device(device)
        self.max_rows, self.features, self.classes = _int32("max_rows", max_rows), _int32("features", features), _int32("classes", classes)
        self.grad = bool(grad)
        h = _vp()
        with torch.cuda.device(self.device):
            _check(_lib.cert_xent_create(self.max_rows, self.features, self.classes, _type_code(self.dtype), int(self.grad),
                                         ctypes.byref(h)), "cert_xent_create")
        self._h = h
        self._number = torch.empty((), dtype=torch.float32, device=self.device)
        self._weight_shape, self._bias_shape = torch.Size((self.classes, self.features)), torch.Size((self.classes,))

    def _args(self, x, weight, target, bias, ignore_index, reduction, grad_scale):
        """The checked inputs as cert_xent_args_t, outputs not set."""
        import torch
        rows, device, dtype = x.shape[0], self.device, self.dtype
        _check_rows("x", x, (rows, self.features), dtype, device)
        _check_rows("weight", weight, self._weight_shape, dtype, device)
        if target.dtype is not torch.int64 and target.dtype is not torch.int32:
            raise ValueError(f"target: int64 or int32 is required, got {target.dtype}")
        _check_rows("target", target, (rows,), target.dtype, device)
        if bias is not None:
            _check_rows("bias", bias, self._bias_shape, dtype, device)
        if reduction != "mean" and reduction != "sum":
            raise ValueError(f"reduction {reduction!r}: 'mean' or 'sum' is required")
        return cert_xent_args_t(_int32("rows", rows), target.dtype is torch.int64, reduction == "sum", grad_scale, ignore_index,
                                x.data_ptr(), _ld(x), weight.data_ptr(), _ld(weight),
                                None if bias is None else bias.data_ptr(), target.data_ptr())

    def loss(self, x, weight, target, bias=None, ignore_index: int = -100, reduction: str = "mean", stream=None):
        """(loss, losses of the rows), float32."""
        import torch
        q = self._args(x, weight, target, bias, ignore_index, reduction, 1.0)
        out = _empty((x.shape[0] + 1,), torch.float32, self.device, stream)
        q.loss = out.data_ptr()
        q.row_losses = q.loss + 4
        _check(_call(self.device, _lib.cert_xent_run, self._h, ctypes.byref(q), _stream_ptr(stream, self.device)), "cert_xent_run")
        return out[0], out[1:]

    def loss_and_grad(self, x, weight, target, bias=None, ignore_index: int = -100, reduction: str = "mean",
                      grad_scale: float = 1.0, dx=None, dweight=None, dbias=None, row_losses=None, stream=None):
        """(loss, dx, dweight, dbias); dbias is None without a bias.  Outputs may be given."""
        import torch
        q = self._args(x, weight, target, bias, ignore_index, reduction, grad_scale)
        device, dtype = self.device, self.dtype
        loss = _empty((), torch.float32, device, stream, self._number)
        q.loss = loss.data_ptr()
        if dx is None:
            dx = _empty((x.shape[0], self.features), dtype, device, stream, x)
        else:
            _check_rows("dx", dx, x.shape, dtype, device)
        if dweight is None:
            dweight = _empty(self._weight_shape, dtype, device, stream, weight)
        else:
            _check_rows("dweight", dweight, self._weight_shape, dtype, device)
        q.dx, q.lddx, q.dweight, q.lddw = dx.data_ptr(), _ld(dx), dweight.data_ptr(), _ld(dweight)
        if bias is not None:
            if dbias is None:
                dbias = _empty(self._bias_shape, dtype, device, stream, bias)
            else:
                _check_rows("dbias", dbias, self._bias_shape, dtype, device)
            q.dbias = dbias.data_ptr()
        elif dbias is not None:
            raise ValueError("dbias: there is no bias")
        if row_losses is not None:
            _check_rows("row_losses", row_losses, (x.shape[0],), torch.float32, device)
            q.row_losses = row_losses.data_ptr()
        _check(_call(self.device, _lib.cert_xent_run, self._h, ctypes.byref(q), _stream_ptr(stream, device)), "cert_xent_run")
        return loss, dx, dweight, dbias

    def last_status(self, stream=None) -> int:
        """0, or what went wrong in an earlier call on this object (1: a target outside the classes); clears it."""
        return int(_call(self.device, _lib.cert_xent_last_status, self._h, _stream_ptr(stream, self.device)))

    def check_guards(self, stream=None) -> int:
        return int(_call(self.device, _lib.cert_xent_check_guards, self._h, _stream_ptr(stream, self.device)))

    def destroy(self):
        if getattr(self, "_h", None):
            _check(_call(self.device, _lib.cert_xent_destroy, self._h), "cert_xent_destroy")
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


class GradClipper:
    """The 2-norm over a list of tensors and the tensors scaled so that it is at most max_norm (cert_clip_*).

    grads: contiguous CUDA tensors of float32, bfloat16 or float16, mixed as they come.  out: where the scaled ones go
    (same shapes and types; None: in place).  The list is laid out on the device once, here; clip() reads what the tensors
    hold when it runs.  The object keeps both lists and their memory, so tensors have to stay the gradients' buffers: if backward
    makes new ones (after zero_grad(set_to_none=True)), the old ones would be clipped.  A torch.nn.Parameter in the list
    stands for its .grad, whichever that is when clip() runs (none: nothing to clip); a new one is laid out then, which allocates
    and waits for the device, so kept buffers (set_to_none=False) are the quick way and the one for CUDA graphs.
    """

    def __init__(self, grads: Sequence, out: Optional[Sequence] = None, device=None):
        import torch
        self._given, self._to = list(grads), None if out is None else list(out)
        self._h = None
        self._follow = [i for i, t in enumerate(self._given) if isinstance(t, torch.nn.Parameter)]
        self.device = _cuda_device(self._given[0].device if device is None and self._given else device)
        if self._to is not None and len(self._to) != len(self._given):
            raise ValueError(f"out: {len(self._to)} tensors for {len(self._given)}")
        self._lay_out(self._current())
        self._number = torch.empty((), dtype=torch.float32, device=self.device)

    _follow = ()

    def _current(self):
        now = list(self._given)
        for i in self._follow:
            now[i] = now[i].grad
        return now

    def _lay_out(self, grads):
        """The list of these gradients (None: no gradient) on the device, in place of the one that was there."""
        import torch
        out = grads if self._to is None else self._to
        arr = (cert_tensor_t * max(1, len(grads)))()
        to = (_vp * max(1, len(grads)))()
        for i, (t, o) in enumerate(zip(grads, out)):
            if t is None:
                continue
            if not t.is_cuda or t.device != self.device or not t.is_contiguous():
                raise ValueError(f"grads[{i}]: a contiguous tensor on {self.device} is required")
            if o.device != self.device or not o.is_contiguous() or o.dtype != t.dtype or o.shape != t.shape:
                raise ValueError(f"out[{i}]: a contiguous {t.dtype} tensor of shape {tuple(t.shape)} on {self.device} is required")
            arr[i].data, arr[i].elements, arr[i].type = t.data_ptr() or None, t.numel(), _type_code(t.dtype)
            to[i] = o.data_ptr() or None
        h = _vp()
        with torch.cuda.device(self.device):
            _check(_lib.cert_clip_create(arr, len(grads), to, ctypes.byref(h)), "cert_clip_create")
        self.destroy()
        self._h, self.grads, self.out = h, grads, out
        self._at = [t is not None and t.data_ptr() for t in grads]
        self._memory = [t.untyped_storage() for t in (*grads, *out) if t is not None]       # whatever becomes of the tensors

    def clip(self, max_norm: float, norm_out=None, stream=None):
        """Scales the tensors into `out` and returns their norm before scaling (float32, on the device)."""
        import torch
        if self._follow:
            now = self._current()
            if any(a is not b or a is not None and a.data_ptr() != at for a, b, at in zip(now, self.grads, self._at)):
                self._lay_out(now)
        if norm_out is None:
            norm_out = _empty((), torch.float32, self.device, stream, self._number)
        elif norm_out.device != self.device or norm_out.dtype != torch.float32 or norm_out.numel() != 1:
            raise ValueError("norm_out: one float32 number on the tensors' device is required")
        _check(_call(self.device, _lib.cert_clip_run, self._h, float(max_norm), norm_out.data_ptr(), _stream_ptr(stream, self.device)), "cert_clip_run")
        return norm_out

    def last_status(self, stream=None) -> int:
        return int(_call(self.device, _lib.cert_clip_last_status, self._h, _stream_ptr(stream, self.device)))

    def check_guards(self, stream=None) -> int:
        return int(_call(self.device, _lib.cert_clip_check_guards, self._h, _stream_ptr(stream, self.device)))

    def destroy(self):
        if getattr(self, "_h", None):
            _check(_call(self.device, _lib.cert_clip_destroy, self._h), "cert_clip_destroy")
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def int4_quantize(weight, group: int = 64, zeros: bool = False, stream=None):
    """(codes, scales, zero points or None) of a weight matrix, in the layout Int4Weight takes (cert_int4_quantize)."""
    import torch
    if weight.dim() != 2:
        raise ValueError("weight: a matrix is required")
    _check_rows("weight", weight, weight.shape, weight.dtype, weight.device)
    n, k, group = _int32("rows", weight.shape[0]), _int32("columns", weight.shape[1]), _int32("group", group)
    groups = -(-k // group) if group > 0 else 0
    codes = _empty((n, (k + 1) // 2), torch.uint8, weight.device, stream)
    scales = _empty((n, groups), weight.dtype, weight.device, stream)
    zp = _empty((n, groups), torch.uint8, weight.device, stream) if zeros else None
    with torch.cuda.device(weight.device):
        _check(_lib.cert_int4_quantize(weight.data_ptr(), _ld(weight), n, k, group, _type_code(weight.dtype), codes.data_ptr(),
                                       scales.data_ptr(), zp.data_ptr() if zeros else None, _stream_ptr(stream, weight.device)),
               "cert_int4_quantize")
    return codes, scales, zp


class Int4Weight:
    """A layer's weights in 4 bits with a scale (and zero point) per group, laid out once for the product (cert_int4_*).

    codes: uint8 [out, ceil(in / 2)], even columns in the low four bits; scales [out, ceil(in / group)] in the type of x;
    zeros: uint8, shaped as scales, or None for 8 everywhere.
    """

    def __init__(self, codes, scales, in_features: int, group: int, zeros=None, stream=None):
        import torch
        self.dtype, self.device = scales.dtype, scales.device
        self.in_features, self.group = _int32("in_features", in_features), _int32("group", group)
        if codes.dim() != 2 or self.group < 1:
            raise ValueError("codes: a matrix, and a positive group, are required")
        self.out_features = _int32("out_features", codes.shape[0])
        groups = -(-self.in_features // self.group)
        for name, t, shape, dtype in (("codes", codes, (self.out_features, (self.in_features + 1) // 2), torch.uint8),
                                      ("scales", scales, (self.out_features, groups), self.dtype),
                                      ("zeros", zeros, (self.out_features, groups), torch.uint8)):
            if t is None and name == "zeros":
                continue
            _check_rows(name, t, shape, dtype, self.device)
            if not t.is_contiguous():
                raise ValueError(f"{name}: a contiguous tensor is required")
        h = _vp()
        with torch.cuda.device(self.device):
            _check(_lib.cert_int4_create(codes.data_ptr(), scales.data_ptr(), zeros.data_ptr() if zeros is not None else None,
                                         self.out_features, self.in_features, self.group, _type_code(self.dtype),
                                         _stream_ptr(stream, self.device), ctypes.byref(h)), "cert_int4_create")
        self._h = h

    @classmethod
    def quantize(cls, weight, group: int = 64, zeros: bool = False, stream=None):
        codes, scales, zp = int4_quantize(weight, group, zeros, stream)
        return cls(codes, scales, weight.shape[1], group, zp, stream)

    def matvec(self, x, bias=None, relu: bool = False, out=None, stream=None):
        """x W^T (+ bias, then ReLU) for the rows of x."""
        import torch
        rows = x.shape[0]
        _check_rows("x", x, (rows, self.in_features), self.dtype, self.device)
        if bias is not None:
            _check_rows("bias", bias, (self.out_features,), self.dtype, self.device)
        if out is None:
            out = _empty((rows, self.out_features), self.dtype, self.device, stream)
        else:
            _check_rows("out", out, (rows, self.out_features), self.dtype, self.device)
        _check(_call(self.device, _lib.cert_int4_matvec, self._h, x.data_ptr(), _ld(x), _int32("rows", rows), bias.data_ptr() if bias is not None else None,
                                     int(bool(relu)), out.data_ptr(), _ld(out), _stream_ptr(stream, self.device)),
               "cert_int4_matvec")
        return out

    def dequantize(self, stream=None):
        """The weights as float32: what a CertNet of the stored network is made from."""
        import torch
        w = _empty((self.out_features, self.in_features), torch.float32, self.device, stream)
        _check(_call(self.device, _lib.cert_int4_dequantize, self._h, w.data_ptr(), _stream_ptr(stream, self.device)), "cert_int4_dequantize")
        return w

    def last_status(self, stream=None) -> int:
        return int(_call(self.device, _lib.cert_int4_last_status, self._h, _stream_ptr(stream, self.device)))

    def check_guards(self, stream=None) -> int:
        return int(_call(self.device, _lib.cert_int4_check_guards, self._h, _stream_ptr(stream, self.device)))

    def destroy(self):
        if getattr(self, "_h", None):
            _check(_call(self.device, _lib.cert_int4_destroy, self._h), "cert_int4_destroy")
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


# C-ABI names, as plain functions
cert_net_create = _lib.cert_net_create
cert_deeppoly_bounds = _lib.cert_deeppoly_bounds
cert_backsub_bounds = _lib.cert_backsub_bounds
cert_deeppoly_bounds_host = _lib.cert_deeppoly_bounds_host
cert_net_destroy = _lib.cert_net_destroy
lib = _lib
