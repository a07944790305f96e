"""Python binding of libff (ctypes).  Argument marshalling only.

Every computation runs in libff's CUDA kernels; PyTorch supplies device
memory (tensors whose data pointers are passed through) and streams.  There
is no fallback: if libff.so is missing or the GPU cannot run it, calls raise.

Names follow the C ABI in include/ff.h:
``Layer`` (ff_layer_*), ``overlay_label``, ``predict``, ``adaptive_negatives``,
``Net`` (ff_net_*), ``Head`` (ff_head_*), ``Pff`` (ff_pff_*), ``po_train_step_raw``/
``po_train_step_act``/``po_predict`` (ff_po_*), ``forward_noalloc``; the
layer operators ``group_norm_act`` and its backward pass, ``dropout``,
``fp8_quantize`` and ``fp8_matmul`` (ff_group_norm_*, ff_dropout, ff_fp8_*),
``rms_norm``, ``rms_norm_fp8`` and ``label_logprobs`` with their backward
passes, ``clip_grad_norm``, ``fp4_quantize``, ``fp4_dequantize`` and
``fp4_matmul`` (ff_rms_norm*, ff_label_logprobs*, ff_clip_grad_norm, ff_fp4_*).
"""

from __future__ import annotations

import array
import ctypes
import functools
import inspect
import os
import warnings
from ctypes import POINTER, c_double, c_float, c_int, c_longlong, c_ulonglong, c_void_p

import numpy as np
import torch

FF_FP32, FF_BF16 = 0, 1
_STATUS = {
    0: "FF_OK", 1: "FF_ERR_INVALID_ARG", 2: "FF_ERR_CUDA", 3: "FF_ERR_OOM",
    4: "FF_ERR_TIMEOUT", 5: "FF_ERR_NONFINITE", 6: "FF_ERR_UNSUPPORTED", 7: "FF_ERR_DEVICE_CHECK",
}
# FF_LIB_VARIANT=checked loads the build with device-side checks (build.py).
LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)),
                        "libff_checked.so" if os.environ.get("FF_LIB_VARIANT") == "checked" else "libff.so")


class FFError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {_STATUS.get(status, status)}")


class LayerConfig(ctypes.Structure):
    _fields_ = [
        ("in_features", c_int), ("out_features", c_int), ("has_bias", c_int),
        ("theta", c_float), ("lr", c_float), ("beta1", c_float), ("beta2", c_float), ("eps", c_float),
        ("prec", c_int), ("init_seed", c_ulonglong), ("max_rows", c_int), ("keep_grad", c_int),
    ]


class HeadConfig(ctypes.Structure):
    _fields_ = [
        ("n_features", c_int), ("lr", c_float), ("beta1", c_float), ("beta2", c_float), ("eps", c_float),
        ("max_rows", c_int),
    ]


class PffConfig(ctypes.Structure):
    _fields_ = [
        ("n_pairs", c_int), ("batch_pairs", c_int), ("epochs_per_chapter", c_int), ("chapters", c_int),
        ("mode", c_int), ("nodes", c_int), ("cooldown_start", c_float),
    ]


_lib = None


def lib():
    """Loads libff.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                "libff.so is not built; run `python -c 'import __graft_entry__ as g; g.build()'`")
        L = ctypes.CDLL(LIB_PATH)
        L.ff_status_string.restype = ctypes.c_char_p
        L.ff_status_string.argtypes = [c_int]
        L.ff_row_stride.restype = c_int
        L.ff_row_stride.argtypes = [c_int]
        L.ff_kernel_launches.restype = ctypes.c_ulonglong
        L.ff_kernel_launches.argtypes = []
        sig = {
            "ff_layer_create": [POINTER(LayerConfig), c_void_p, POINTER(c_void_p)],
            "ff_layer_destroy": [c_void_p],
            "ff_overlay_label": [c_void_p, c_void_p, c_int, c_int, c_void_p, c_void_p, c_int, c_void_p],
            "ff_layer_forward": [c_void_p, c_void_p, c_void_p, c_void_p, c_int, c_void_p, c_void_p, c_void_p,
                                 c_void_p],
            "ff_layer_train_step": [c_void_p, c_void_p, c_void_p, c_void_p, c_int, c_void_p, c_void_p, c_void_p,
                                    c_void_p, c_void_p],
            "ff_predict": [c_void_p, c_int, c_void_p, c_int, c_void_p, c_void_p, c_void_p],
            "ff_adaptive_negatives": [c_void_p, c_int, c_void_p, c_void_p, c_int, c_void_p, c_void_p, c_void_p],
            "ff_layer_get_state": [c_void_p] + [c_void_p] * 6 + [POINTER(c_longlong)],
            "ff_layer_set_state": [c_void_p] + [c_void_p] * 6 + [c_longlong],
            "ff_layer_get_grad": [c_void_p, c_void_p, c_void_p],
            "ff_layer_get_grad_operand": [c_void_p, c_void_p, c_int],
            "ff_layer_check": [c_void_p],
            "ff_layer_set_fused_local_grad": [c_void_p, c_int],
            "ff_layer_get_stats": [c_void_p, c_void_p],
            "ff_layer_selftest_wait": [c_void_p, ctypes.c_uint, c_void_p],
            "ff_net_create": [c_void_p, c_int, c_int, c_int, POINTER(c_void_p)],
            "ff_net_destroy": [c_void_p],
            "ff_net_train_step": [c_void_p, c_void_p, c_void_p, c_int, c_void_p, c_void_p],
            "ff_net_train_step_images": [c_void_p, c_void_p, c_void_p, c_int, c_void_p, c_void_p],
            "ff_net_sync": [c_void_p, c_void_p],
            "ff_net_train_epoch": [c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_void_p, c_void_p],
            "ff_net_epoch_trace": [c_void_p, c_int, c_void_p, c_longlong],
            "ff_net_create_po": [c_void_p, c_void_p, c_int, c_int, c_int, POINTER(c_void_p)],
            "ff_net_po_train_step": [c_void_p, c_void_p, c_void_p, c_int, c_void_p, c_void_p],
            "ff_forward_noalloc": [c_void_p, c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_void_p, c_void_p,
                                   c_void_p, c_void_p, c_void_p],
            "ff_head_create": [POINTER(HeadConfig), POINTER(c_void_p)],
            "ff_head_destroy": [c_void_p],
            "ff_head_train_step": [c_void_p, c_void_p, c_int, c_void_p, c_void_p, c_int, c_void_p, c_void_p],
            "ff_head_train_epoch": [c_void_p, c_void_p, c_int, c_void_p, c_void_p, c_int, c_int, c_void_p, c_void_p],
            "ff_head_predict": [c_void_p, c_void_p, c_int, c_void_p, c_int, c_void_p, c_void_p, c_void_p],
            "ff_head_get_state": [c_void_p] + [c_void_p] * 6 + [POINTER(c_longlong)],
            "ff_head_set_state": [c_void_p] + [c_void_p] * 6 + [c_longlong],
            "ff_head_get_grad": [c_void_p, c_void_p, c_void_p],
            "ff_head_check": [c_void_p],
            "ff_po_train_step": [c_void_p, c_void_p, c_void_p, c_int, c_void_p, c_void_p, c_int, c_void_p, c_void_p,
                                 c_void_p, c_void_p],
            "ff_po_predict": [c_void_p, c_int, c_void_p, c_void_p, c_int, c_void_p, c_void_p, c_void_p],
            "ff_pff_create": [c_void_p, c_int, POINTER(PffConfig), POINTER(c_void_p)],
            "ff_pff_destroy": [c_void_p],
            "ff_pff_wait": [c_void_p, ctypes.c_uint],
            "ff_net_wait": [c_void_p, ctypes.c_uint],
            "ff_pff_run": [c_void_p, c_void_p, c_void_p, c_int, c_int, c_void_p, c_void_p],
            "ff_group_norm_act": [c_void_p, c_longlong, c_int, c_int, c_int, c_int, c_void_p, c_void_p, c_float, c_int,
                                  c_int, c_void_p, c_longlong, c_void_p, c_void_p, c_void_p, c_longlong, c_void_p],
            "ff_group_norm_act_backward": [c_void_p, c_longlong, c_void_p, c_longlong, c_int, c_int, c_int, c_int,
                                           c_void_p, c_void_p, c_void_p, c_void_p, c_int, c_int, c_void_p, c_longlong,
                                           c_void_p, c_void_p, c_void_p, c_longlong, c_void_p],
            "ff_dropout": [c_void_p, c_longlong, c_longlong, c_longlong, c_double, c_ulonglong, c_ulonglong, c_void_p,
                           c_void_p, c_longlong, c_int, c_void_p, c_longlong, c_void_p],
            "ff_fp8_stride": [c_int],
            "ff_fp8_quantize": [c_void_p, c_longlong, c_int, c_int, c_int, c_int, c_void_p, c_void_p, c_void_p, c_void_p,
                                c_void_p],
            "ff_fp8_matmul": [c_void_p, c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_int, c_void_p, c_int, c_int,
                              c_void_p, c_longlong, c_void_p, c_void_p],
            "ff_fp8_check": [c_void_p],
            "ff_fp8_selftest_wait": [ctypes.c_uint, c_void_p],
            "ff_rms_norm": [c_void_p, c_longlong, c_void_p, c_longlong, c_int, c_int, c_void_p, c_float, c_int, c_void_p,
                            c_longlong, c_void_p, c_longlong, c_void_p, c_void_p, c_void_p, c_void_p],
            "ff_rms_norm_backward": [c_void_p, c_longlong, c_void_p, c_longlong, c_int, c_int, c_void_p, c_void_p,
                                     c_void_p, c_longlong, c_int, c_void_p, c_longlong, c_void_p, c_void_p, c_longlong,
                                     c_void_p],
            "ff_label_logprobs": [c_void_p, c_longlong, c_int, c_int, c_int, c_void_p, c_void_p, c_void_p, c_int, c_void_p,
                                  c_void_p, c_void_p, c_void_p],
            "ff_label_logprobs_backward": [c_void_p, c_longlong, c_int, c_int, c_int, c_void_p, c_void_p, c_void_p,
                                           c_void_p, c_void_p, c_void_p, c_longlong, c_void_p],
            "ff_clip_grad_norm": [c_void_p, c_void_p, c_void_p, c_void_p, c_int, c_float, c_void_p, c_void_p, c_longlong,
                                  c_void_p],
            "ff_fp4_stride": [c_int],
            "ff_fp4_quantize": [c_void_p, c_longlong, c_int, c_int, c_int, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p],
            "ff_fp4_dequantize": [c_void_p, c_void_p, c_int, c_int, c_int, c_void_p, c_longlong, c_void_p],
            "ff_fp4_matmul": [c_void_p, c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_void_p, c_int, c_int, c_void_p,
                              c_longlong, c_void_p, c_void_p],
        }
        for name, args in sig.items():
            f = getattr(L, name)
            f.restype = c_int
            f.argtypes = args
        L.ff_group_norm_workspace.restype = c_longlong
        L.ff_group_norm_workspace.argtypes = [c_int] * 6
        L.ff_dropout_words.restype = c_longlong
        L.ff_dropout_words.argtypes = [c_longlong, c_longlong]
        L.ff_rms_norm_workspace.restype = c_longlong
        L.ff_rms_norm_workspace.argtypes = [c_int, c_int]
        L.ff_clip_grad_norm_workspace.restype = c_longlong
        L.ff_clip_grad_norm_workspace.argtypes = [c_int]
        L.ff_fp4_scale_bytes.restype = c_longlong
        L.ff_fp4_scale_bytes.argtypes = [c_int, c_int]
        _lib = L
    return _lib


def _check(status: int, what: str):
    if status != 0:
        raise FFError(status, what)


def row_stride(features: int) -> int:
    return lib().ff_row_stride(int(features))


def kernel_launches() -> int:
    """ff_kernel_launches: libff's kernel launches in this process so far."""
    return int(lib().ff_kernel_launches())


def _stream(stream) -> int:
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def _ptr(t, dtype=None, what="tensor", need_cuda=True):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{what} must be a torch.Tensor")
    if need_cuda and not t.is_cuda:
        raise ValueError(f"{what} must be a CUDA tensor")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{what} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    return t.data_ptr()


def _on(stream, device, *used):
    """The stream of an operator call, and what allocates its buffers.  On a
    stream that is not the current one they come from that stream's own pool,
    since the current one's may hand out memory that its queued kernels still
    use; and they count as used on the current one, where the caller goes on
    with them.  `used`: the caller's tensors, which count as used on the call's
    stream (so freeing one after the call is safe).  What the stream has to
    wait for before the call stays the caller's business."""
    current = torch._C._cuda_getCurrentRawStream(device.index)
    if stream is None:
        return current, torch.empty
    ptr = _stream(stream)
    if ptr == current:
        return current, torch.empty
    if isinstance(stream, torch.cuda.Stream):
        other = stream
    else:
        other = torch.cuda.ExternalStream(ptr, device) if ptr else torch.cuda.default_stream(device)
    here = torch.cuda.current_stream(device)
    for t in used:
        if isinstance(t, torch.Tensor) and t.is_cuda:
            t.record_stream(other)

    def empty(shape, dtype, device):
        with torch.cuda.stream(other):
            t = torch.empty(shape, dtype=dtype, device=device)
        t.record_stream(here)
        return t

    return ptr, empty


def act_dtype(prec: str):
    return torch.bfloat16 if prec == "bf16" else torch.float32


class Layer:
    """One FF layer (``ff_layer``): parameters, Adam moments and workspace on the GPU."""

    def __init__(self, in_features: int, out_features: int, prec: str = "bf16", theta: float = 2.0,
                 lr: float = 0.03, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
                 has_bias: bool = True, init_seed: int = 0, max_rows: int = 0, keep_grad: bool = False,
                 stream=None):
        if prec not in ("bf16", "fp32"):
            raise ValueError("prec must be 'bf16' or 'fp32'")
        self.in_features, self.out_features, self.prec = int(in_features), int(out_features), prec
        self.dtype = act_dtype(prec)
        self.cfg = LayerConfig(self.in_features, self.out_features, int(bool(has_bias)), theta, lr, beta1, beta2,
                               eps, FF_BF16 if prec == "bf16" else FF_FP32, int(init_seed), int(max_rows),
                               int(bool(keep_grad)))
        h = c_void_p()
        _check(lib().ff_layer_create(ctypes.byref(self.cfg), c_void_p(_stream(stream)), ctypes.byref(h)),
               "ff_layer_create")
        self._h = h

    @property
    def handle(self):
        return self._h

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            _check(lib().ff_layer_destroy(self._h), "ff_layer_destroy")
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # buffers in the layer's activation format
    def new_activation(self, rows: int, features: int | None = None, device="cuda"):
        f = self.out_features if features is None else features
        return torch.zeros(rows, row_stride(f), dtype=self.dtype, device=device)

    def _x_args(self, x, labels, row_scale):
        if labels is not None:
            xp = _ptr(x, torch.float32, "x (raw input)")
            if x.shape[-1] != self.in_features:
                raise ValueError("raw x must have in_features columns")
            return xp, _ptr(labels, torch.int32, "labels"), None
        xp = _ptr(x, self.dtype, "x (activation)")
        if x.shape[-1] != row_stride(self.in_features):
            raise ValueError("activation x must have ff_row_stride(in_features) columns")
        return xp, None, _ptr(row_scale, torch.float32, "row_scale")

    def train_step(self, x, labels=None, row_scale=None, B=None, h_out=None, next_scale=None, goodness=None,
                   loss=None, stream=None):
        """ff_layer_train_step: rows 0..B-1 positive, B..2B-1 negative."""
        if B is None:
            B = x.shape[0] // 2
        xp, lp, sp = self._x_args(x, labels, row_scale)
        _check(lib().ff_layer_train_step(
            self._h, xp, lp, sp, int(B), _ptr(h_out, self.dtype, "h_out"),
            _ptr(next_scale, torch.float32, "next_scale"), _ptr(goodness, torch.float32, "goodness"),
            _ptr(loss, torch.float32, "loss"), c_void_p(_stream(stream))), "ff_layer_train_step")

    def forward(self, x, labels=None, row_scale=None, rows=None, h_out=None, next_scale=None, goodness=None,
                stream=None):
        """ff_layer_forward (L_i(x)) without an update."""
        if rows is None:
            rows = x.shape[0]
        xp, lp, sp = self._x_args(x, labels, row_scale)
        _check(lib().ff_layer_forward(
            self._h, xp, lp, sp, int(rows), _ptr(h_out, self.dtype, "h_out"),
            _ptr(next_scale, torch.float32, "next_scale"), _ptr(goodness, torch.float32, "goodness"),
            c_void_p(_stream(stream))), "ff_layer_forward")

    def get_state(self):
        N, K = self.out_features, self.in_features
        W = np.empty((N, K), np.float32); mW = np.empty_like(W); vW = np.empty_like(W)
        b = np.empty(N, np.float32); mb = np.empty_like(b); vb = np.empty_like(b)
        step = c_longlong()
        _check(lib().ff_layer_get_state(self._h, W.ctypes.data, b.ctypes.data, mW.ctypes.data, vW.ctypes.data,
                                        mb.ctypes.data, vb.ctypes.data, ctypes.byref(step)), "ff_layer_get_state")
        return dict(W=W, b=b, mW=mW, vW=vW, mb=mb, vb=vb, t=step.value)

    def set_state(self, W=None, b=None, mW=None, vW=None, mb=None, vb=None, t=0):
        N, K = self.out_features, self.in_features

        def host(a, shape):
            if a is None:
                return None, None
            a = np.ascontiguousarray(np.asarray(a, dtype=np.float32))
            if a.shape != shape:
                raise ValueError(f"expected shape {shape}, got {a.shape}")
            return a, a.ctypes.data
        keep = [host(W, (N, K)), host(b, (N,)), host(mW, (N, K)), host(vW, (N, K)), host(mb, (N,)), host(vb, (N,))]
        _check(lib().ff_layer_set_state(self._h, *[k[1] for k in keep], int(t)), "ff_layer_set_state")

    def get_grad(self):
        N, K = self.out_features, self.in_features
        dW = np.empty((N, K), np.float32); db = np.empty(N, np.float32)
        _check(lib().ff_layer_get_grad(self._h, dW.ctypes.data, db.ctypes.data), "ff_layer_get_grad")
        return dW, db

    def get_grad_operand(self, rows: int):
        """ff_layer_get_grad_operand: the last step's weight-gradient operand
        G = diag(s) dZ [rows, ff_row_stride(out_features)] as float64 (from
        bf16 or fp32; exact)."""
        ld = row_stride(self.out_features)
        if self.prec == "bf16":
            raw = np.empty((rows, ld), np.uint16)
            _check(lib().ff_layer_get_grad_operand(self._h, raw.ctypes.data, int(rows)), "ff_layer_get_grad_operand")
            return (raw.astype(np.uint32) << 16).view(np.float32).astype(np.float64)
        out = np.empty((rows, ld), np.float32)
        _check(lib().ff_layer_get_grad_operand(self._h, out.ctypes.data, int(rows)), "ff_layer_get_grad_operand")
        return out.astype(np.float64)

    def stats(self):
        """ff_layer_get_stats: (mean positive goodness, mean negative goodness,
        active-ReLU fraction) of the last train step."""
        out = np.zeros(3, np.float32)
        _check(lib().ff_layer_get_stats(self._h, out.ctypes.data), "ff_layer_get_stats")
        return tuple(float(v) for v in out)

    def check(self):
        _check(lib().ff_layer_check(self._h), "ff_layer_check")

    def set_fused_local_grad(self, enable: bool):
        """ff_layer_set_fused_local_grad: bf16 train steps form the local step in
        the forward GEMM's epilogue (True) or in a separate kernel (False, the
        default); bitwise the same results."""
        _check(lib().ff_layer_set_fused_local_grad(self._h, 1 if enable else 0), "ff_layer_set_fused_local_grad")

    def selftest_wait(self, timeout_us: int, stream=None):
        """ff_layer_selftest_wait: a bounded wait that is made to run out."""
        _check(lib().ff_layer_selftest_wait(self._h, int(timeout_us), c_void_p(_stream(stream))),
               "ff_layer_selftest_wait")


def overlay_label(x, labels, prec="bf16", out=None, row_scale=None, stream=None):
    """ff_overlay_label: returns the overlaid activation buffer."""
    rows, F = x.shape
    px = _ptr(x, torch.float32, "x")
    on, empty = _on(stream, x.device, x, labels, out, row_scale)
    if out is None:
        out = empty((rows, row_stride(F)), dtype=act_dtype(prec), device=x.device)
    _check(lib().ff_overlay_label(px, _ptr(labels, torch.int32, "labels"), rows, F,
                                  _ptr(out, act_dtype(prec), "out"), _ptr(row_scale, torch.float32, "row_scale"),
                                  FF_BF16 if prec == "bf16" else FF_FP32, c_void_p(on)),
           "ff_overlay_label")
    return out


def predict(layers, x, pred=None, goodness=None, stream=None):
    """ff_predict: goodness prediction over the 10 label overlays.  Returns (pred, goodness)."""
    n = x.shape[0]
    px = _ptr(x, torch.float32, "x")
    on, empty = _on(stream, x.device, x, pred, goodness)
    if pred is None:
        pred = empty((n,), dtype=torch.int32, device=x.device)
    arr = (c_void_p * len(layers))(*[l.handle.value for l in layers])
    _check(lib().ff_predict(arr, len(layers), px, n, _ptr(pred, torch.int32, "pred"),
                            _ptr(goodness, torch.float32, "goodness"), c_void_p(on)), "ff_predict")
    return pred, goodness


def adaptive_negatives(layers, x, labels, neg=None, goodness=None, stream=None):
    """ff_adaptive_negatives: AdaptiveNEG negative labels (§5), each sample's
    strongest wrong label under goodness prediction.  Returns (neg, goodness)."""
    n = x.shape[0]
    if labels.shape[0] != n:
        raise ValueError("labels must have one entry per row of x")
    px = _ptr(x, torch.float32, "x")
    on, empty = _on(stream, x.device, x, labels, neg, goodness)
    if neg is None:
        neg = empty((n,), dtype=torch.int32, device=x.device)
    arr = (c_void_p * len(layers))(*[l.handle.value for l in layers])
    _check(lib().ff_adaptive_negatives(arr, len(layers), px,
                                       _ptr(labels, torch.int32, "labels"), n, _ptr(neg, torch.int32, "neg"),
                                       _ptr(goodness, torch.float32, "goodness"), c_void_p(on)),
           "ff_adaptive_negatives")
    return neg, goodness


class Net:
    """ff_net: the layers of a net trained concurrently, one CUDA stream per layer."""

    def __init__(self, layers, max_B: int, depth: int = 2):
        self.layers = list(layers)
        arr = (c_void_p * len(self.layers))(*[l.handle.value for l in self.layers])
        h = c_void_p()
        _check(lib().ff_net_create(arr, len(self.layers), int(max_B), int(depth), ctypes.byref(h)), "ff_net_create")
        self._h = h

    def train_step(self, x, labels, B=None, loss=None, stream=None):
        if B is None:
            B = x.shape[0] // 2
        _check(lib().ff_net_train_step(self._h, _ptr(x, torch.float32, "x"), _ptr(labels, torch.int32, "labels"),
                                       int(B), _ptr(loss, torch.float32, "loss"), c_void_p(_stream(stream))),
               "ff_net_train_step")

    def train_step_images(self, x, labels, loss=None, stream=None):
        """ff_net_train_step_images: x [B, in] holds one image per pair, labels
        [2B] the true labels then the wrong ones."""
        B = x.shape[0]
        if labels.shape[0] != 2 * B:
            raise ValueError("labels must hold 2 * x.shape[0] entries (true labels, then wrong labels)")
        _check(lib().ff_net_train_step_images(self._h, _ptr(x, torch.float32, "x"),
                                              _ptr(labels, torch.int32, "labels"), int(B),
                                              _ptr(loss, torch.float32, "loss"), c_void_p(_stream(stream))),
               "ff_net_train_step_images")

    def train_epoch(self, x, labels, n_pairs: int, B: int, images_per_pair_row: int = 2, loss=None, stream=None):
        """ff_net_train_epoch: n_pairs pairs in batches of B pairs through the
        net in one persistent kernel (the tail batch stepwise); x holds
        images_per_pair_row rows per pair (2: stacked pair batches, 1: one
        image per pair), labels [2 * n_pairs] (per batch the true labels, then
        the wrong ones)."""
        if x.shape[0] != images_per_pair_row * n_pairs or labels.shape[0] != 2 * n_pairs:
            raise ValueError("x must have images_per_pair_row * n_pairs rows and labels 2 * n_pairs entries")
        _check(lib().ff_net_train_epoch(self._h, _ptr(x, torch.float32, "x"), _ptr(labels, torch.int32, "labels"),
                                        int(n_pairs), int(B), int(images_per_pair_row),
                                        _ptr(loss, torch.float32, "loss"), c_void_p(_stream(stream))),
               "ff_net_train_epoch")

    def epoch_trace(self, enable=None):
        """ff_net_epoch_trace: with enable=True/False switches per-task tracing
        of later train_epoch calls; returns the last traced epoch as
        (gemm [G, 6], stream [S, 6]) uint64 arrays (see include/ff.h), or None."""
        L = lib()
        L.ff_net_epoch_trace.restype = c_longlong
        if enable is not None:
            L.ff_net_epoch_trace(self._h, 1 if enable else 0, None, 0)
            return None
        cap = 2 + 6 * (1 << 22)
        buf = np.zeros(cap, np.uint64)
        n = L.ff_net_epoch_trace(self._h, -1, buf.ctypes.data, cap)
        if n < 2:
            return None
        g, st = int(buf[0]), int(buf[1])
        rec = buf[2:n].reshape(-1, 6)
        return rec[:g], rec[g:g + st]

    def sync(self, stream=None):
        _check(lib().ff_net_sync(self._h, c_void_p(_stream(stream))), "ff_net_sync")

    def wait(self, timeout_ms: int):
        """ff_net_wait: host-side wait with a deadline (raises FFError FF_ERR_TIMEOUT)."""
        _check(lib().ff_net_wait(self._h, int(timeout_ms)), "ff_net_wait")

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            lib().ff_net_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def forward_noalloc(x, row_scale, W_bf16, in_features, out_features, h_out, bias=None, goodness=None,
                    next_scale=None, device_status=None, stream=None):
    """ff_forward_noalloc: the bf16 forward pass from caller buffers only (no
    device allocation inside the library); see include/ff.h."""
    rows = x.shape[0]
    _check(lib().ff_forward_noalloc(
        _ptr(x, torch.bfloat16, "x"), _ptr(row_scale, torch.float32, "row_scale"),
        _ptr(W_bf16, torch.bfloat16, "W_bf16"), _ptr(bias, torch.float32, "bias"), int(rows), int(in_features),
        int(out_features), _ptr(h_out, torch.bfloat16, "h_out"), _ptr(goodness, torch.float32, "goodness"),
        _ptr(next_scale, torch.float32, "next_scale"), _ptr(device_status, torch.int32, "device_status"),
        c_void_p(_stream(stream))), "ff_forward_noalloc")


def _layer_array(layers):
    return (c_void_p * len(layers))(*[l.handle.value for l in layers])


class Head:
    """The softmax prediction head (``ff_head``) over layers 2..L of a net."""

    N_CLASSES = 10

    def __init__(self, n_features: int, lr: float = 1e-4, beta1: float = 0.9, beta2: float = 0.999,
                 eps: float = 1e-8, max_rows: int = 0):
        self.n_features = int(n_features)
        self.cfg = HeadConfig(self.n_features, lr, beta1, beta2, eps, int(max_rows))
        h = c_void_p()
        _check(lib().ff_head_create(ctypes.byref(self.cfg), ctypes.byref(h)), "ff_head_create")
        self._h = h

    @staticmethod
    def features_of(layers) -> int:
        """n_features for a layer chain: out_features of layers 2..L (of layer 1 when L == 1)."""
        return sum(l.out_features for l in (layers[1:] if len(layers) > 1 else layers))

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            _check(lib().ff_head_destroy(self._h), "ff_head_destroy")
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def train_step(self, layers, x, labels, loss=None, stream=None):
        n = x.shape[0]
        if labels.shape[0] != n:
            raise ValueError("labels must have one entry per row of x")
        _check(lib().ff_head_train_step(self._h, _layer_array(layers), len(layers), _ptr(x, torch.float32, "x"),
                                        _ptr(labels, torch.int32, "labels"), n, _ptr(loss, torch.float32, "loss"),
                                        c_void_p(_stream(stream))), "ff_head_train_step")

    def train_epoch(self, layers, x, labels, B, loss=None, stream=None):
        """ff_head_train_epoch: ceil(n / B) train steps on consecutive rows, the
        features of many steps formed by one forward pass."""
        n = x.shape[0]
        if labels.shape[0] != n:
            raise ValueError("labels must have one entry per row of x")
        _check(lib().ff_head_train_epoch(self._h, _layer_array(layers), len(layers), _ptr(x, torch.float32, "x"),
                                         _ptr(labels, torch.int32, "labels"), n, int(B),
                                         _ptr(loss, torch.float32, "loss"), c_void_p(_stream(stream))),
               "ff_head_train_epoch")

    def predict(self, layers, x, pred=None, logits=None, stream=None):
        """Returns (pred, logits)."""
        n = x.shape[0]
        px = _ptr(x, torch.float32, "x")
        on, empty = _on(stream, x.device, x, pred, logits)
        if pred is None:
            pred = empty((n,), dtype=torch.int32, device=x.device)
        _check(lib().ff_head_predict(self._h, _layer_array(layers), len(layers), px, n,
                                     _ptr(pred, torch.int32, "pred"), _ptr(logits, torch.float32, "logits"),
                                     c_void_p(on)), "ff_head_predict")
        return pred, logits

    def get_state(self):
        C, F = self.N_CLASSES, self.n_features
        V = np.empty((C, F), np.float32); mV = np.empty_like(V); vV = np.empty_like(V)
        c = np.empty(C, np.float32); mc = np.empty_like(c); vc = np.empty_like(c)
        step = c_longlong()
        _check(lib().ff_head_get_state(self._h, V.ctypes.data, c.ctypes.data, mV.ctypes.data, vV.ctypes.data,
                                       mc.ctypes.data, vc.ctypes.data, ctypes.byref(step)), "ff_head_get_state")
        return dict(V=V, c=c, mV=mV, vV=vV, mc=mc, vc=vc, t=step.value)

    def set_state(self, V=None, c=None, mV=None, vV=None, mc=None, vc=None, t=0):
        C, F = self.N_CLASSES, self.n_features

        def host(a, shape):
            if a is None:
                return None, None
            a = np.ascontiguousarray(np.asarray(a, dtype=np.float32))
            if a.shape != shape:
                raise ValueError(f"expected shape {shape}, got {a.shape}")
            return a, a.ctypes.data
        keep = [host(V, (C, F)), host(c, (C,)), host(mV, (C, F)), host(vV, (C, F)), host(mc, (C,)), host(vc, (C,))]
        _check(lib().ff_head_set_state(self._h, *[k[1] for k in keep], int(t)), "ff_head_set_state")

    def get_grad(self):
        dV = np.empty((self.N_CLASSES, self.n_features), np.float32); dc = np.empty(self.N_CLASSES, np.float32)
        _check(lib().ff_head_get_grad(self._h, dV.ctypes.data, dc.ctypes.data), "ff_head_get_grad")
        return dV, dc

    def check(self):
        _check(lib().ff_head_check(self._h), "ff_head_check")


class Pff:
    """The chapter schedule (``ff_pff``) of a layer chain: Single-Layer PFF
    (one stream per layer) or All-Layers PFF (``nodes`` streams taking the
    chapters in turn)."""

    def __init__(self, layers, n_pairs: int, batch_pairs: int, epochs_per_chapter: int, chapters: int,
                 mode: str = "single_layer", nodes: int = 1, cooldown_start: float = 1.0):
        if mode not in ("single_layer", "all_layers"):
            raise ValueError("mode must be 'single_layer' or 'all_layers'")
        self.layers = list(layers)
        self.cfg = PffConfig(int(n_pairs), int(batch_pairs), int(epochs_per_chapter), int(chapters),
                             0 if mode == "single_layer" else 1, int(nodes), float(cooldown_start))
        h = c_void_p()
        _check(lib().ff_pff_create(_layer_array(self.layers), len(self.layers), ctypes.byref(self.cfg),
                                   ctypes.byref(h)), "ff_pff_create")
        self._h = h

    @property
    def batches(self) -> int:
        return (self.cfg.n_pairs + self.cfg.batch_pairs - 1) // self.cfg.batch_pairs

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            _check(lib().ff_pff_destroy(self._h), "ff_pff_destroy")
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def wait(self, timeout_ms: int):
        """ff_pff_wait: host-side wait with a deadline (raises FFError FF_ERR_TIMEOUT)."""
        _check(lib().ff_pff_wait(self._h, int(timeout_ms)), "ff_pff_wait")

    def run(self, x, labels, first: int, count: int, loss=None, stream=None):
        """Enqueues chapters first .. first+count-1; labels [count, 2P] int32."""
        _check(lib().ff_pff_run(self._h, _ptr(x, torch.float32, "x"), _ptr(labels, torch.int32, "labels"),
                                int(first), int(count), _ptr(loss, torch.float32, "loss"),
                                c_void_p(_stream(stream))), "ff_pff_run")


def _po_step(layer, block, x, labels, raw, row_scale, h_out, next_scale, loss, stream):
    n = x.shape[0]
    if labels.shape[0] != n:
        raise ValueError("labels must have one entry per row of x")
    xp = _ptr(x, torch.float32 if raw else layer.dtype, "x")
    _check(lib().ff_po_train_step(layer.handle, block._h, xp, int(bool(raw)),
                                  _ptr(row_scale, torch.float32, "row_scale"), _ptr(labels, torch.int32, "labels"), n,
                                  _ptr(h_out, layer.dtype, "h_out"), _ptr(next_scale, torch.float32, "next_scale"),
                                  _ptr(loss, torch.float32, "loss"), c_void_p(_stream(stream))), "ff_po_train_step")


def po_train_step_raw(layer, block, x, labels, h_out=None, next_scale=None, loss=None, stream=None):
    """ff_po_train_step on raw float32 input rows (the first layer, with the
    neutral label): one Performance-Optimized step of ``layer`` and its
    softmax ``block`` (a Head with n_features == layer.out_features)."""
    _po_step(layer, block, x, labels, True, None, h_out, next_scale, loss, stream)


def po_train_step_act(layer, block, x, labels, row_scale=None, h_out=None, next_scale=None, loss=None, stream=None):
    """ff_po_train_step on an activation buffer of the layer (a hidden layer)."""
    _po_step(layer, block, x, labels, False, row_scale, h_out, next_scale, loss, stream)


def po_predict(layers, block, x, pred=None, logits=None, stream=None):
    """ff_po_predict: the last layer's block's prediction.  Returns (pred, logits)."""
    n = x.shape[0]
    px = _ptr(x, torch.float32, "x")
    on, empty = _on(stream, x.device, x, pred, logits)
    if pred is None:
        pred = empty((n,), dtype=torch.int32, device=x.device)
    _check(lib().ff_po_predict(_layer_array(layers), len(layers), block._h, px, n,
                               _ptr(pred, torch.int32, "pred"), _ptr(logits, torch.float32, "logits"),
                               c_void_p(on)), "ff_po_predict")
    return pred, logits



def save_checkpoint(path, layers, heads=()):
    """Writes every layer's and head's full state (parameters, Adam moments
    and step) to one .npz file, with the shapes needed to check a restore."""
    arrays = {}
    for k, l in enumerate(layers):
        st = l.get_state()
        for name, v in st.items():
            arrays[f"layer{k}.{name}"] = np.asarray(v)
        arrays[f"layer{k}.shape"] = np.array([l.in_features, l.out_features])
    for k, h in enumerate(heads):
        st = h.get_state()
        for name, v in st.items():
            arrays[f"head{k}.{name}"] = np.asarray(v)
    np.savez(path, n_layers=np.array(len(layers)), n_heads=np.array(len(heads)), **arrays)


def load_checkpoint(path, layers, heads=()):
    """Restores states written by save_checkpoint into layers (and heads) of
    the same shapes; raises ValueError on a mismatch."""
    with np.load(path) as z:
        if int(z["n_layers"]) != len(layers) or int(z["n_heads"]) != len(heads):
            raise ValueError("checkpoint holds a different number of layers or heads")
        for k, l in enumerate(layers):
            if tuple(z[f"layer{k}.shape"]) != (l.in_features, l.out_features):
                raise ValueError(f"layer {k}: checkpoint shape {tuple(z[f'layer{k}.shape'])}")
            l.set_state(**{n: z[f"layer{k}.{n}"] for n in ("W", "b", "mW", "vW", "mb", "vb")},
                        t=int(z[f"layer{k}.t"]))
        for k, h in enumerate(heads):
            h.set_state(**{n: z[f"head{k}.{n}"] for n in ("V", "c", "mV", "vV", "mc", "vc")},
                        t=int(z[f"head{k}.t"]))


class PoNet(Net):
    """A Performance-Optimized net on one CUDA stream per layer
    (ff_net_create_po): layer k with its softmax block blocks[k]."""

    def __init__(self, layers, blocks, max_rows: int, depth: int = 2):
        self.layers, self.blocks = list(layers), list(blocks)
        h = c_void_p()
        _check(lib().ff_net_create_po(_layer_array(self.layers),
                                      (c_void_p * len(self.blocks))(*[b._h.value for b in self.blocks]),
                                      len(self.layers), int(max_rows), int(depth), ctypes.byref(h)),
               "ff_net_create_po")
        self._h = h

    def train_step(self, x, labels, loss=None, stream=None):
        n = x.shape[0]
        if labels.shape[0] != n:
            raise ValueError("labels must have one entry per row of x")
        _check(lib().ff_net_po_train_step(self._h, _ptr(x, torch.float32, "x"), _ptr(labels, torch.int32, "labels"),
                                          n, _ptr(loss, torch.float32, "loss"), c_void_p(_stream(stream))),
               "ff_net_po_train_step")


# ------------------------------------------------------------ layer operators
_PREC = {torch.bfloat16: FF_BF16, torch.float32: FF_FP32}
_ACT = {"none": 0, "relu": 1, "silu": 2}
_INT_MAX = 0x7FFFFFFF


def _on_device_of_first(f):
    """Runs an operator with its first argument's device current (the kernels launch on the current device)."""

    first = next(iter(inspect.signature(f).parameters))

    @functools.wraps(f)
    def call(*args, **kwargs):
        x = args[0] if args else kwargs.get(first)
        try:
            index = x.get_device()
        except AttributeError:
            kind = {"a": "Fp8Matrix" if f.__name__.startswith("fp8") else "Fp4Matrix", "m": "Fp4Matrix"}
            raise TypeError(f"{first} must be a {kind.get(first, 'torch.Tensor')}") from None
        if index < 0:
            raise ValueError(f"{first} must be a CUDA tensor")
        if index == torch._C._cuda_getDevice():
            return f(*args, **kwargs)
        with torch.cuda.device(index):
            return f(*args, **kwargs)

    return call


def _prec(x, what):
    prec = _PREC.get(x.dtype)
    if prec is None:
        raise TypeError(f"{what} must be torch.bfloat16 or torch.float32, got {x.dtype}")
    return prec


def _row_stride_of(x, what):
    """Row stride of x seen as a matrix [rows, last dimension]; raises where its rows are not evenly spaced."""
    if x.is_contiguous():
        return x.shape[-1]
    shape, stride = x.shape, x.stride()
    if x.numel() == 0:
        return shape[-1]
    if stride[-1] != 1 and shape[-1] != 1:
        raise ValueError(f"{what}: the last dimension must be contiguous")
    ld, span = None, 1
    for size, step in zip(reversed(shape[:-1]), reversed(stride[:-1])):
        if size == 1:
            continue
        if ld is None:
            ld = step
        elif step != ld * span:
            raise ValueError(f"{what}: the rows must be evenly spaced")
        span *= size
    ld = shape[-1] if ld is None else ld
    if ld < shape[-1]:
        raise ValueError(f"{what}: rows overlap (row stride {ld} < {shape[-1]})")
    return ld


def _unrecorded(name, depth=4):
    """Says that a call whose inputs require a gradient is not recorded, where autograd is on: the operators work on the
    tensors' memory and return plain results.  depth: frames up to the user's call."""
    if torch.is_grad_enabled():
        warnings.warn(f"{name} is not recorded by autograd: its result has no gradient (the gradient is a call of its "
                      f"own; use torch.no_grad() or detach() where that is meant)", stacklevel=depth)


# Calls write buffers that they are given behind autograd's back: this lets it
# refuse a later backward pass that would read a tensor's values from before.
_written = torch.autograd.graph.increment_version


def _vector(t, size, what, device):
    if t is None:
        return None
    if not (isinstance(t, torch.Tensor) and t.dtype is torch.float32 and t.device == device and t.numel() == size
            and t.is_contiguous()):
        _ptr(t, torch.float32, what)  # says what is wrong with the tensor itself
        if t.numel() != size:
            raise ValueError(f"{what} must have {size} values")
        _same_device(t, device, what)
    return t.data_ptr()


def _same_device(t, device, what):
    if t.device != device:
        raise ValueError(f"{what} must be on {device}")


def _like(t, x, what):
    """Checks an optional buffer that must match x in shape, type and device; returns its row stride."""
    if not isinstance(t, torch.Tensor) or t.shape != x.shape or t.dtype != x.dtype or t.device != x.device:
        raise ValueError(f"{what} must match the input's shape, type and device")
    return _row_stride_of(t, what)


@functools.lru_cache(maxsize=4096)
def _norm_sizes(shape, groups, act, prec, backward):
    """n, positions, channels, groups, ff_activation and workspace bytes of a norm over [n, ..., channels]."""
    if len(shape) < 2:
        raise ValueError("x must be [n, channels] or [n, ..., channels]")
    if act not in _ACT:
        raise ValueError(f"act must be one of {sorted(_ACT)}")
    n, C, spatial, groups = shape[0], shape[-1], 1, int(groups)
    if groups < 1 or C < 1 or C % groups:
        raise ValueError("groups must divide the channels")
    for d in shape[1:-1]:
        spatial *= d
    if max(n, spatial, C) > _INT_MAX:
        raise ValueError("n, positions and channels must each fit 32 bits")
    return n, spatial, C, groups, _ACT[act], lib().ff_group_norm_workspace(n, spatial, C, groups, prec, backward)


@_on_device_of_first
def group_norm_act(x, gamma, beta, groups: int, act: str = "silu", eps: float = 1e-5, out=None, mean=None, rstd=None,
                   stream=None):
    """ff_group_norm_act: y = act(gamma * (x - mean) * rstd + beta) over channel
    groups, channels last.  x [n, channels] or [n, ..., channels] (bf16 or
    fp32, evenly spaced rows); gamma, beta fp32 [channels] or None.  Returns
    (y, mean, rstd), mean and rstd fp32 [n, groups]; out may be x.  Not
    recorded by autograd: its gradient is group_norm_act_backward."""
    prec, dev = _prec(x, "x"), x.device
    n, spatial, C, groups, kind, need = _norm_sizes(x.shape, groups, act, prec, 0)
    on, empty = _on(stream, dev, x, gamma, beta, out, mean, rstd)
    ldx = _row_stride_of(x, "x")
    given = [t for t in (out, mean, rstd) if t is not None]
    if out is None:
        out, ldy = empty(x.shape, dtype=x.dtype, device=dev), C
    else:
        ldy = _like(out, x, "out")
    if mean is None:
        mean = empty((n, groups), dtype=torch.float32, device=dev)
        pm = mean.data_ptr()
    else:
        pm = _vector(mean, n * groups, "mean", dev)
    if rstd is None:
        rstd = empty((n, groups), dtype=torch.float32, device=dev)
        pr = rstd.data_ptr()
    else:
        pr = _vector(rstd, n * groups, "rstd", dev)
    ws = empty((need,), dtype=torch.uint8, device=dev) if need > 0 else None
    _check(lib().ff_group_norm_act(
        x.data_ptr(), ldx, n, spatial, C, groups, _vector(gamma, C, "gamma", dev), _vector(beta, C, "beta", dev),
        eps, kind, prec, out.data_ptr(), ldy, pm, pr, None if ws is None else ws.data_ptr(), need, on),
        "ff_group_norm_act")
    if given:
        _written(given)
    if x.requires_grad or (gamma is not None and gamma.requires_grad) or (beta is not None and beta.requires_grad):
        _unrecorded("group_norm_act")
    return out, mean, rstd


@_on_device_of_first
def group_norm_act_backward(dy, x, mean, rstd, gamma, beta, groups: int, act: str = "silu", out=None, stream=None):
    """ff_group_norm_act_backward: the gradient of group_norm_act at (x, gamma,
    beta), with the mean and rstd it returned.  Returns (dx, dgamma, dbeta);
    out may be dy or x."""
    prec, dev = _prec(x, "x"), x.device
    n, spatial, C, groups, kind, need = _norm_sizes(x.shape, groups, act, prec, 1)
    on, empty = _on(stream, dev, dy, x, mean, rstd, gamma, beta, out)
    ldx, lddy = _row_stride_of(x, "x"), _like(dy, x, "dy")
    given = out
    if out is None:
        out, lddx = empty(x.shape, dtype=x.dtype, device=dev), C
    else:
        lddx = _like(out, x, "out")
    dgamma = empty((C,), dtype=torch.float32, device=dev)
    dbeta = empty((C,), dtype=torch.float32, device=dev)
    if mean is None or rstd is None:
        raise ValueError("mean and rstd of the forward pass are needed")
    ws = empty((need,), dtype=torch.uint8, device=dev) if need > 0 else None
    _check(lib().ff_group_norm_act_backward(
        dy.data_ptr(), lddy, x.data_ptr(), ldx, n, spatial, C, groups, _vector(mean, n * groups, "mean", dev),
        _vector(rstd, n * groups, "rstd", dev), _vector(gamma, C, "gamma", dev), _vector(beta, C, "beta", dev),
        kind, prec, out.data_ptr(), lddx, dgamma.data_ptr(), dbeta.data_ptr(),
        None if ws is None else ws.data_ptr(), need, on), "ff_group_norm_act_backward")
    if given is not None:
        _written(given)
    return out, dgamma, dbeta


def dropout_words(rows: int, cols: int) -> int:
    """ff_dropout_words: generator words that a mask of rows x cols takes."""
    return int(lib().ff_dropout_words(int(rows), int(cols)))


@_on_device_of_first
def dropout(x, p: float, seed: int, offset=0, residual=None, out=None, stream=None):
    """ff_dropout: residual + keep * x / (1 - p) with the mask drawn from the
    counter-based generator at (seed, offset), never stored; its gradient is
    the same call on dy without a residual.  x [..., cols] (bf16 or fp32,
    evenly spaced rows).  offset: an int, or a one-element int64 CUDA tensor
    that is read when the kernel runs (for CUDA graphs).  out may be x or the
    residual.  Not recorded by autograd."""
    prec = _prec(x, "x")
    if x.dim() < 1:
        raise ValueError("x must have at least one dimension")
    dev = x.device
    on, empty = _on(stream, dev, x, offset, residual, out)
    cols = x.shape[-1]
    rows = x.numel() // cols if cols else 0
    ldx = _row_stride_of(x, "x")
    ldr = _like(residual, x, "residual") if residual is not None else 0
    given = out
    if out is None:
        out, ldy = empty(x.shape, dtype=x.dtype, device=dev), cols
    else:
        ldy = _like(out, x, "out")
    odev, host = None, 0
    if isinstance(offset, torch.Tensor):
        if offset.numel() != 1:
            raise ValueError("offset must have one element")
        _same_device(offset, dev, "offset")
        odev = _ptr(offset, torch.int64, "offset")
    else:
        host = int(offset) & 0xFFFFFFFFFFFFFFFF
    _check(lib().ff_dropout(x.data_ptr(), ldx, rows, cols, p, int(seed) & 0xFFFFFFFFFFFFFFFF, host, odev,
                            None if residual is None else residual.data_ptr(), ldr, prec, out.data_ptr(), ldy,
                            on), "ff_dropout")
    if given is not None:
        _written(given)
    if x.requires_grad or (residual is not None and residual.requires_grad):
        _unrecorded("dropout")
    return out


class Fp8Matrix:
    """An 8-bit matrix [rows, k]: e4m3 values q [rows, ff_fp8_stride(k)] and
    fp32 scales, [ceil(k / 128), rows] or, tile=True, [ceil(k / 128),
    ceil(rows / 128)] (see ff_fp8_blocks in include/ff.h)."""

    __slots__ = ("q", "scale", "rows", "k", "tile")

    def __init__(self, q, scale, rows: int, k: int, tile: bool = False):
        self.q, self.scale, self.rows, self.k, self.tile = q, scale, rows, k, tile
        if k < 1 or q.shape != (rows, (k + 15) & ~15) or q.element_size() != 1 or not q.is_contiguous() or not q.is_cuda:
            raise ValueError("q must be a contiguous one-byte CUDA tensor [rows, ff_fp8_stride(k)]")
        if (scale.shape != ((k + 127) // 128, (rows + 127) // 128 if tile else rows) or scale.dtype != torch.float32
                or not scale.is_contiguous() or scale.device != q.device):
            raise ValueError("scale must be contiguous fp32 [ceil(k / 128), rows or row blocks] beside q")

    def get_device(self):
        """The CUDA device's index, as of a tensor."""
        return self.q.get_device()

    @property
    def blocks(self):
        """ff_fp8_blocks of the matrix."""
        return 1 if self.tile else 0


def _fp8_new(empty, rows, k, tile, dev):
    m = object.__new__(Fp8Matrix)
    m.q = empty((rows, (k + 15) & ~15), dtype=torch.float8_e4m3fn, device=dev)
    m.scale = empty(((k + 127) // 128, (rows + 127) // 128 if tile else rows), dtype=torch.float32, device=dev)
    m.rows, m.k, m.tile = rows, k, tile
    return m


@_on_device_of_first
def _fp8_quantize(x, tile, straight, transposed, stream):
    prec = _prec(x, "x")
    if x.dim() != 2 or x.shape[1] < 1:
        raise ValueError("x must be [rows, k] with k >= 1")
    dev = x.device
    on, empty = _on(stream, dev, x)
    rows, k = x.shape
    if max(rows, k) > _INT_MAX:
        raise ValueError("rows and k must each fit 32 bits")
    if transposed and rows < 1:
        raise ValueError("the transpose needs at least one row")
    ldx = _row_stride_of(x, "x")
    a = _fp8_new(empty, rows, k, tile, dev) if straight else None
    t = _fp8_new(empty, k, rows, tile, dev) if transposed else None
    _check(lib().ff_fp8_quantize(x.data_ptr(), ldx, rows, k, prec, 1 if tile else 0,
                                 a.q.data_ptr() if a else None, a.scale.data_ptr() if a else None,
                                 t.q.data_ptr() if t else None, t.scale.data_ptr() if t else None, on),
           "ff_fp8_quantize")
    if x.requires_grad:
        _unrecorded("fp8_quantize", depth=5)
    return a, t


def fp8_quantize(x, tile: bool = False, transpose: bool = False, stream=None):
    """ff_fp8_quantize: x [rows, k] (bf16 or fp32, evenly spaced rows) as an
    Fp8Matrix in row blocks or 128 x 128 tiles; transpose=True gives x's
    transpose instead.  Not recorded by autograd."""
    return _fp8_quantize(x, tile, not transpose, transpose, stream)[1 if transpose else 0]


def fp8_quantize_both(x, tile: bool = False, stream=None):
    """ff_fp8_quantize, both ways round from one read of x: (x, x's transpose)."""
    return _fp8_quantize(x, tile, True, True, stream)


@_on_device_of_first
def fp8_matmul(a, b, bias=None, relu: bool = False, out=None, out_dtype=torch.bfloat16, status=None, stream=None):
    """ff_fp8_matmul: act(a b^T + bias) of two Fp8Matrix (a in row blocks).
    Returns [a.rows, b.rows] in out_dtype (torch.bfloat16 or torch.float32) or
    out's type; bias fp32 [b.rows].  Not recorded by autograd: the gradients
    are products of their own (see ff_fp8_matmul in include/ff.h).  status: a
    one-element int32 CUDA tensor that is OR-ed with 1 if a kernel wait timed
    out; without one, fp8_check reports it."""
    if not isinstance(a, Fp8Matrix) or not isinstance(b, Fp8Matrix):
        raise TypeError("a and b must be Fp8Matrix")
    if a.k != b.k:
        raise ValueError("a and b must have the same k")
    if a.tile:
        raise ValueError("a must be quantized in row blocks")
    dev = a.q.device
    _same_device(b.q, dev, "b")
    on, empty = _on(stream, dev, a.q, a.scale, b.q, b.scale, bias, out, status)
    m, n = a.rows, b.rows
    given = out
    if out is None:
        prec = _PREC.get(out_dtype)
        if prec is None:
            raise TypeError("out_dtype must be torch.bfloat16 or torch.float32")
        out, ldc = empty((m, n), dtype=out_dtype, device=dev), n
    else:
        if out.shape != (m, n):
            raise ValueError("out must be [a.rows, b.rows]")
        _same_device(out, dev, "out")
        prec, ldc = _prec(out, "out"), _row_stride_of(out, "out")
    if status is not None:
        _same_device(status, dev, "status")
    _check(lib().ff_fp8_matmul(a.q.data_ptr(), a.scale.data_ptr(), b.q.data_ptr(), b.scale.data_ptr(), b.blocks, m,
                               n, a.k, _vector(bias, n, "bias", dev), 1 if relu else 0, prec, out.data_ptr(), ldc,
                               _ptr(status, torch.int32, "status"), on), "ff_fp8_matmul")
    if given is not None:
        _written(given)
    if bias is not None and bias.requires_grad:
        _unrecorded("fp8_matmul")
    return out


def fp8_check(stream=None):
    """ff_fp8_check: waits for the stream and raises if a wait of an fp8_matmul
    that was given no status timed out on the current device (its result is
    not valid)."""
    _check(lib().ff_fp8_check(c_void_p(_stream(stream))), "ff_fp8_check")


def fp8_selftest_wait(timeout_us: int, stream=None):
    """ff_fp8_selftest_wait: a bounded wait that is made to run out, for fp8_check to report."""
    _check(lib().ff_fp8_selftest_wait(int(timeout_us), c_void_p(_stream(stream))), "ff_fp8_selftest_wait")


# ------------------------------------------------- RMS norm, log-probabilities, clipping
# (These calls take a few us of host time in all, so buffers come from the
# shortest way there is to one on the current device: size, stride, type.)
try:
    _new_cuda = torch._C._dynamo.guards._empty_strided_cuda
except AttributeError:
    def _new_cuda(size, stride, dtype):
        return torch.empty_strided(size, stride, dtype=dtype, device="cuda")


def _place(stream, index, used):
    """The stream of a call on device `index`, the current one, and what makes its dense buffers, as _on's."""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(index), _new_cuda
    dev = torch.device("cuda", index)
    on, empty = _on(stream, dev, *used)
    if empty is torch.empty:
        return on, _new_cuda
    return on, lambda size, stride, dtype: empty(size, dtype=dtype, device=dev)


@functools.lru_cache(maxsize=4096)
def _dense(shape):
    """Size and strides of a dense tensor, as plain tuples."""
    stride, n = [], 1
    for d in reversed(shape):
        stride.append(n)
        n *= max(d, 1)
    return tuple(shape), tuple(reversed(stride))


def _matrix_sizes(x, what):
    """rows, last dimension and row stride of x seen as a matrix [rows, last dimension]."""
    shape = x.shape
    if not shape or shape[-1] < 1:
        raise ValueError(f"{what} must be [..., columns] with at least one column")
    cols = shape[-1]
    rows = shape[0] if len(shape) == 2 else x.numel() // cols
    if rows > 0x7FFFFF00 or cols > 0x7FFFFF00:
        raise ValueError(f"{what}: rows and columns must each fit 32 bits")
    return rows, cols, cols if x.is_contiguous() else _row_stride_of(x, what)


@functools.lru_cache(maxsize=4096)
def _rms_workspace(rows, cols):
    return lib().ff_rms_norm_workspace(rows, cols)


@functools.lru_cache(maxsize=4096)
def _fp8_shapes(rows, k):
    """Sizes and strides of an Fp8Matrix in row blocks."""
    return (rows, (k + 15) & ~15), ((k + 15) & ~15, 1), ((k + 127) // 128, rows), (max(rows, 1), 1)


def _rms_norm(x, gamma, residual, eps, out, h, fp8, stream):
    prec, dev, dt = _prec(x, "x"), x.device, x.dtype
    rows, cols, ldx = _matrix_sizes(x, "x")
    on, new = _place(stream, dev.index, (x, gamma, residual, out, h))
    ldr = ldh = ldy = 0
    pr = ph = py = pq = ps = None
    kept, given = x, None if out is None and h is None else [t for t in (out, h) if t is not None]
    if residual is not None:
        ldr, pr = _like(residual, x, "residual"), residual.data_ptr()
        if h is None:
            kept, ldh = new(*_dense(x.shape), dt), cols
        else:
            kept, ldh = h, _like(h, x, "h")
        ph = kept.data_ptr()
    elif h is not None:
        raise ValueError("h goes with a residual (without one it is x)")
    if fp8:
        out = object.__new__(Fp8Matrix)
        q, qs, s, ss = _fp8_shapes(rows, cols)
        out.q, out.scale = new(q, qs, torch.float8_e4m3fn), new(s, ss, torch.float32)
        out.rows, out.k, out.tile = rows, cols, False
        pq, ps = out.q.data_ptr(), out.scale.data_ptr()
    else:
        if out is None:
            out, ldy = new(*_dense(x.shape), dt), cols
        else:
            ldy = _like(out, x, "out")
            if residual is None and rows and out.data_ptr() == x.data_ptr():
                kept = None  # x's values are gone
        py = out.data_ptr()
    rstd = new((rows,), (1,), torch.float32)
    _check(lib().ff_rms_norm(x.data_ptr(), ldx, pr, ldr, rows, cols, _vector(gamma, cols, "gamma", dev), eps, prec, ph, ldh, py,
                             ldy, pq, ps, rstd.data_ptr(), on), "ff_rms_norm")
    if given:
        _written(given)
    if (x.requires_grad or (gamma is not None and gamma.requires_grad)
            or (residual is not None and residual.requires_grad)):
        _unrecorded("rms_norm_fp8" if fp8 else "rms_norm", depth=5)
    return out, kept, rstd


@_on_device_of_first
def rms_norm(x, gamma, residual=None, eps: float = 1e-5, out=None, h=None, stream=None):
    """ff_rms_norm: h = x + residual, y = gamma * h * rstd with rstd = 1 /
    sqrt(mean h^2 + eps) over the last dimension.  x, residual [..., cols] (bf16
    or fp32, evenly spaced rows), gamma fp32 [cols] or None.  Returns (y, h,
    rstd): h is x itself without a residual (None if out is x: the gradient
    needs the values that are then gone), rstd fp32 [rows].  out and h are
    optional buffers; either may be x or the residual, not both the same.  Not
    recorded by autograd: its gradient is rms_norm_backward."""
    return _rms_norm(x, gamma, residual, eps, out, h, False, stream)


@_on_device_of_first
def rms_norm_fp8(x, gamma, residual=None, eps: float = 1e-5, h=None, stream=None):
    """ff_rms_norm with its output as an Fp8Matrix in row blocks, for
    fp8_matmul.  Returns (a, h, rstd) as rms_norm does.  Not recorded by autograd."""
    return _rms_norm(x, gamma, residual, eps, None, h, True, stream)


@_on_device_of_first
def rms_norm_backward(dy, h, rstd, gamma, dh=None, out=None, stream=None):
    """ff_rms_norm_backward: the gradient of rms_norm, from the h and rstd that
    it returned; dh is what the residual stream hands back and is added.
    Returns (dx, dgamma): dx is the gradient of x and of the residual; out may
    be dy, h or dh."""
    prec, dev = _prec(dy, "dy"), dy.device
    rows, cols, lddy = _matrix_sizes(dy, "dy")
    on, new = _place(stream, dev.index, (dy, h, rstd, gamma, dh, out))
    ldh = _like(h, dy, "h")
    lddh = 0 if dh is None else _like(dh, dy, "dh")
    if rstd is None:
        raise ValueError("rstd of the forward pass is needed")
    given = out
    if out is None:
        out, lddx = new(*_dense(dy.shape), dy.dtype), cols
    else:
        lddx = _like(out, dy, "out")
    dgamma = new((cols,), (1,), torch.float32)
    need = _rms_workspace(rows, cols)
    ws = new((need,), (1,), torch.uint8) if need > 0 else None
    _check(lib().ff_rms_norm_backward(dy.data_ptr(), lddy, h.data_ptr(), ldh, rows, cols, _vector(rstd, rows, "rstd", dev),
                                      _vector(gamma, cols, "gamma", dev), None if dh is None else dh.data_ptr(), lddh, prec,
                                      out.data_ptr(), lddx, dgamma.data_ptr(), None if ws is None else ws.data_ptr(), need,
                                      on), "ff_rms_norm_backward")
    if given is not None:
        _written(given)
    return out, dgamma


class LabelLogprobs:
    """What label_logprobs returns: logp and entropy [rows] fp32, top_logp [rows,
    top] fp32 and top_index [rows, top] int32, stats [rows, 2] fp32 (the row's
    maximum and log sum, for the gradient).  logp is None without labels."""

    __slots__ = ("logp", "entropy", "top_logp", "top_index", "stats")


def _labels(labels, rows, dev):
    if not (isinstance(labels, torch.Tensor) and labels.dtype is torch.int32 and labels.device == dev
            and labels.numel() == rows and labels.is_contiguous()):
        _ptr(labels, torch.int32, "labels")  # says what is wrong with the tensor itself
        if labels.numel() != rows:
            raise ValueError("labels must have one entry per row")
        _same_device(labels, dev, "labels")
    return labels.data_ptr()


@_on_device_of_first
def label_logprobs(logits, labels, top: int = 0, stream=None):
    """ff_label_logprobs: under the softmax of each row of logits [..., classes]
    (bf16 or fp32, evenly spaced rows), the log-probability of its label (int32
    [rows]; 0 for a label outside the classes; labels None: not wanted), the
    entropy, and the `top` (up to 32) likeliest classes with theirs.  Returns a
    LabelLogprobs.  Not recorded by autograd: its gradient is
    label_logprobs_backward."""
    prec, dev = _prec(logits, "logits"), logits.device
    rows, classes, ld = _matrix_sizes(logits, "logits")
    top = int(top)
    if not 0 <= top <= min(32, classes):
        raise ValueError("top must be 0 .. min(32, classes)")
    on, new = _place(stream, dev.index, (logits, labels))
    f32 = torch.float32
    r = object.__new__(LabelLogprobs)
    pl = pp = r.logp = None
    if labels is not None:
        pl = _labels(labels, rows, dev)
        r.logp = new((rows,), (1,), f32)
        pp = r.logp.data_ptr()
    r.entropy = new((rows,), (1,), f32)
    r.top_logp = new((rows, top), (top or 1, 1), f32)
    r.top_index = new((rows, top), (top or 1, 1), torch.int32)
    r.stats = new((rows, 2), (2, 1), f32)
    _check(lib().ff_label_logprobs(logits.data_ptr(), ld, rows, classes, prec, pl, pp, r.entropy.data_ptr(), top,
                                   r.top_logp.data_ptr(), r.top_index.data_ptr(), r.stats.data_ptr(), on),
           "ff_label_logprobs")
    if logits.requires_grad:
        _unrecorded("label_logprobs")
    return r


@_on_device_of_first
def label_logprobs_backward(logits, labels, stats, dlogp, entropy=None, dentropy=None, out=None, stream=None):
    """ff_label_logprobs_backward: the gradient of label_logprobs at the logits,
    dlogp (1[label] - p) - dentropy p (ln p + entropy), from its stats (and, for
    dentropy, its entropy).  dlogp or dentropy fp32 [rows] may be None.  Returns
    a tensor like logits; out may be the logits."""
    prec, dev = _prec(logits, "logits"), logits.device
    rows, classes, ld = _matrix_sizes(logits, "logits")
    if stats is None:
        raise ValueError("stats of the forward pass are needed")
    if dlogp is not None and labels is None:
        raise ValueError("dlogp needs the labels")
    if dentropy is not None and entropy is None:
        raise ValueError("dentropy needs the forward pass's entropy")
    on, new = _place(stream, dev.index, (logits, labels, stats, dlogp, entropy, dentropy, out))
    given = out
    if out is None:
        out, ldo = new(*_dense(logits.shape), logits.dtype), classes
    else:
        ldo = _like(out, logits, "out")
    _check(lib().ff_label_logprobs_backward(
        logits.data_ptr(), ld, rows, classes, prec, None if labels is None else _labels(labels, rows, dev),
        _vector(stats, 2 * rows, "stats", dev), _vector(dlogp, rows, "dlogp", dev), _vector(entropy, rows, "entropy", dev),
        _vector(dentropy, rows, "dentropy", dev), out.data_ptr(), ldo, on), "ff_label_logprobs_backward")
    if given is not None:
        _written(given)
    return out


@functools.lru_cache(maxsize=256)
def _clip_workspace(n):
    return lib().ff_clip_grad_norm_workspace(n)


def clip_grad_norm(grads, max_norm: float, out=None, stream=None):
    """ff_clip_grad_norm: the 2-norm over all tensors of grads (bf16 or fp32,
    contiguous, one device) together, and the tensors scaled so that it is at
    most max_norm, in place or into `out` (a list of tensors like them).
    Returns the norm before clipping, fp32 [1], without a wait.  max_norm
    math.inf leaves the values as they are, whatever the norm.  Outputs that
    overlap each other, or gradients other than their own, are refused (so a
    tensor comes twice only with an output for each)."""
    grads = list(grads)
    n = len(grads)
    if n == 0 or not isinstance(grads[0], torch.Tensor):
        raise ValueError("grads must be a non-empty list of tensors")
    index = grads[0].get_device()
    if index < 0:
        raise ValueError("grads must be CUDA tensors")
    if index != torch._C._cuda_getDevice():
        with torch.cuda.device(index):
            return clip_grad_norm(grads, max_norm, out, stream)
    try:
        kinds = [_PREC[g.dtype] for g in grads]
        if set(map(torch.Tensor.get_device, grads)) != {index} or not all(map(torch.Tensor.is_contiguous, grads)):
            raise AttributeError
        ptrs, counts = list(map(torch.Tensor.data_ptr, grads)), list(map(torch.Tensor.numel, grads))
    except KeyError:
        raise TypeError("grads must be torch.bfloat16 or torch.float32") from None
    except (AttributeError, TypeError):
        raise ValueError(f"grads must be contiguous tensors on cuda:{index}") from None
    to = ptrs
    if out is not None:
        out = list(out)
        if len(out) != n:
            raise ValueError("out must have a tensor for each of grads")
        try:
            like = (set(map(torch.Tensor.get_device, out)) == {index} and all(map(torch.Tensor.is_contiguous, out))
                    and [o.shape for o in out] == [g.shape for g in grads] and [o.dtype for o in out] == [g.dtype for g in grads])
        except TypeError:  # not a tensor
            like = False
        if not like:
            raise ValueError("out must match grads in shape, type and device, and be contiguous")
        to = list(map(torch.Tensor.data_ptr, out))
    on, new = _place(stream, index, () if stream is None else (*grads, *(out or ())))
    need = _clip_workspace(n)
    # (the array module's: ctypes' own arrays take four times as long to fill, 15 us for 60 tensors)
    host, types = array.array("q", ptrs + to + counts), array.array("i", kinds)
    at = host.buffer_info()[0]
    norm = new((1,), (1,), torch.float32)
    ws = new((need,), (1,), torch.uint8)
    _check(lib().ff_clip_grad_norm(at, at + 8 * n, at + 16 * n, types.buffer_info()[0], n, max_norm, norm.data_ptr(), ws.data_ptr(), need,
                                   on), "ff_clip_grad_norm")
    _written(grads if out is None else out)
    return norm


# ------------------------------------------------------------ 4-bit matrices
class Fp4Matrix:
    """A 4-bit matrix [rows, k]: e2m1 pairs q [rows, ff_fp4_stride(k)] and
    power-of-two scales [ceil(rows / 128), ceil(k / 128), 32, 4, 4], both bytes
    (see ff_fp4_quantize in include/ff.h)."""

    __slots__ = ("q", "scale", "rows", "k")

    def __init__(self, q, scale, rows: int, k: int):
        self.q, self.scale, self.rows, self.k = q, scale, rows, k
        if (k < 1 or q.shape != (rows, (k + 31) // 32 * 16) or q.element_size() != 1 or not q.is_contiguous()
                or not q.is_cuda):
            raise ValueError("q must be a contiguous one-byte CUDA tensor [rows, ff_fp4_stride(k)]")
        if (scale.shape != ((rows + 127) // 128, (k + 127) // 128, 32, 4, 4) or scale.element_size() != 1
                or not scale.is_contiguous() or scale.device != q.device):
            raise ValueError("scale must be contiguous bytes [ceil(rows / 128), ceil(k / 128), 32, 4, 4] beside q")

    def get_device(self):
        """The CUDA device's index, as of a tensor."""
        return self.q.get_device()


@functools.lru_cache(maxsize=4096)
def _fp4_shapes(rows, k):
    """Sizes and strides of an Fp4Matrix."""
    stride, tiles = (k + 31) // 32 * 16, ((rows + 127) // 128, (k + 127) // 128, 32, 4, 4)
    return ((rows, stride), (stride, 1)) + _dense(tiles)


def _fp4_new(new, rows, k):
    q, qs, s, ss = _fp4_shapes(rows, k)
    m = object.__new__(Fp4Matrix)
    m.q, m.scale, m.rows, m.k = new(q, qs, torch.uint8), new(s, ss, torch.uint8), rows, k
    return m


@_on_device_of_first
def _fp4_quantize(x, straight, transposed, stream):
    prec = _prec(x, "x")
    if x.dim() != 2:
        raise ValueError("x must be [rows, k] with k >= 1")
    rows, k, ldx = _matrix_sizes(x, "x")
    if transposed and rows < 1:
        raise ValueError("the transpose needs at least one row")
    on, new = _place(stream, x.get_device(), (x,))
    a = t = pa = sa = pt = st = None
    if straight:
        a = _fp4_new(new, rows, k)
        pa, sa = a.q.data_ptr(), a.scale.data_ptr()
    if transposed:
        t = _fp4_new(new, k, rows)
        pt, st = t.q.data_ptr(), t.scale.data_ptr()
    _check(lib().ff_fp4_quantize(x.data_ptr(), ldx, rows, k, prec, pa, sa, pt, st, on), "ff_fp4_quantize")
    if x.requires_grad:
        _unrecorded("fp4_quantize", depth=5)
    return a, t


def fp4_quantize(x, transpose: bool = False, stream=None):
    """ff_fp4_quantize: x [rows, k] (bf16 or fp32, evenly spaced rows) as an
    Fp4Matrix; transpose=True gives x's transpose instead.  Not recorded by
    autograd."""
    return _fp4_quantize(x, not transpose, transpose, stream)[1 if transpose else 0]


def fp4_quantize_both(x, stream=None):
    """ff_fp4_quantize, both ways round from one read of x: (x, x's transpose)."""
    return _fp4_quantize(x, True, True, stream)


@_on_device_of_first
def fp4_dequantize(m, out=None, out_dtype=torch.bfloat16, stream=None):
    """ff_fp4_dequantize: the values [rows, k] that an Fp4Matrix stands for,
    exactly, in out_dtype (torch.bfloat16 or torch.float32) or out's type."""
    if not isinstance(m, Fp4Matrix):
        raise TypeError("m must be a Fp4Matrix")
    rows, k = m.rows, m.k
    on, new = _place(stream, m.q.get_device(), (m.q, m.scale, out))
    given = out
    if out is None:
        prec = _PREC.get(out_dtype)
        if prec is None:
            raise TypeError("out_dtype must be torch.bfloat16 or torch.float32")
        out, ldy = new((rows, k), (k, 1), out_dtype), k
    else:
        if out.shape != (rows, k):
            raise ValueError("out must be [rows, k]")
        _same_device(out, m.q.device, "out")
        prec, ldy = _prec(out, "out"), _row_stride_of(out, "out")
    _check(lib().ff_fp4_dequantize(m.q.data_ptr(), m.scale.data_ptr(), rows, k, prec, out.data_ptr(), ldy, on),
           "ff_fp4_dequantize")
    if given is not None:
        _written(given)
    return out


@_on_device_of_first
def fp4_matmul(a, b, bias=None, relu: bool = False, out=None, out_dtype=torch.bfloat16, status=None, stream=None):
    """ff_fp4_matmul: act(a b^T + bias) of two Fp4Matrix, otherwise as
    fp8_matmul: returns [a.rows, b.rows] in out_dtype or out's type, bias fp32
    [b.rows], status an optional int32 word for timed-out waits (without one,
    fp8_check reports them).  Not recorded by autograd."""
    if not isinstance(a, Fp4Matrix) or not isinstance(b, Fp4Matrix):
        raise TypeError("a and b must be Fp4Matrix")
    if a.k != b.k:
        raise ValueError("a and b must have the same k")
    dev = a.q.device
    _same_device(b.q, dev, "b")
    on, new = _place(stream, dev.index, (a.q, a.scale, b.q, b.scale, bias, out, status))
    m, n = a.rows, b.rows
    given = out
    if out is None:
        prec = _PREC.get(out_dtype)
        if prec is None:
            raise TypeError("out_dtype must be torch.bfloat16 or torch.float32")
        out, ldc = new((m, n), (n or 1, 1), out_dtype), n
    else:
        if out.shape != (m, n):
            raise ValueError("out must be [a.rows, b.rows]")
        _same_device(out, dev, "out")
        prec, ldc = _prec(out, "out"), _row_stride_of(out, "out")
    if status is not None:
        _same_device(status, dev, "status")
    _check(lib().ff_fp4_matmul(a.q.data_ptr(), a.scale.data_ptr(), b.q.data_ptr(), b.scale.data_ptr(), m, n, a.k,
                               _vector(bias, n, "bias", dev), 1 if relu else 0, prec, out.data_ptr(), ldc,
                               _ptr(status, torch.int32, "status"), on), "ff_fp4_matmul")
    if given is not None:
        _written(given)
    if bias is not None and bias.requires_grad:
        _unrecorded("fp4_matmul")
    return out
