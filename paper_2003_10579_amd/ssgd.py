"""ctypes binding of libssgd.so: the same names as include/ssgd.h, argument
marshalling only.  PyTorch supplies device memory and the stream handle."""
from __future__ import annotations

import ctypes as C
import os
import warnings

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libssgd.so")

LSQ, SOFTMAX, MLP2 = 0, 1, 2
K_SYNC, K_BATCH_SYNC, K_ASYNC, K_BATCH_ASYNC = 0, 1, 2, 3
EXP, SHIFTED_EXP, PARETO, TABLE = 0, 1, 2, 3
OK, EINVAL, ENOMEM, EDEVICE, ESTATE = 0, 1, 2, 3, 4
_VARIANTS = {"k_sync": K_SYNC, "k_batch_sync": K_BATCH_SYNC, "k_async": K_ASYNC, "k_batch_async": K_BATCH_ASYNC}
F32, BF16 = 0, 1
MX_FP4, MX_FP8 = 0, 1
_FORMATS = {"fp4": MX_FP4, "fp8": MX_FP8}
ACT_NONE, ACT_RELU, ACT_GELU, ACT_SILU = 0, 1, 2, 3
_ACTIVATIONS = {None: ACT_NONE, "relu": ACT_RELU, "gelu": ACT_GELU, "silu": ACT_SILU}
_KINDS = {"lsq": LSQ, "softmax": SOFTMAX, "mlp2": MLP2}

EXPORTS = [
    "ssgd_create", "ssgd_run", "ssgd_reserve_trace", "ssgd_step", "ssgd_param_count", "ssgd_updates_done", "ssgd_current_K",
    "ssgd_trace_width", "ssgd_get_trace", "ssgd_get_params", "ssgd_set_params", "ssgd_force_K",
    "ssgd_get_workers", "ssgd_state_bytes", "ssgd_get_state", "ssgd_set_state", "ssgd_full_loss",
    "ssgd_full_gradient", "ssgd_full_gradient_static",
    "ssgd_runtime_mc", "ssgd_debug_delays", "ssgd_debug_batch", "ssgd_stream_read_rate", "ssgd_last_error",
    "ssgd_last_kernel_ms", "ssgd_adamw_state_elements", "ssgd_adamw_create", "ssgd_adamw_step", "ssgd_adamw_destroy",
    "ssgd_mx_row_bytes", "ssgd_mx_quantize", "ssgd_mx_dequantize",
    "ssgd_mx_matmul_work_bytes", "ssgd_mx_matmul", "ssgd_mx_linear_work_bytes", "ssgd_mx_linear",
    "ssgd_mx_dense_work_bytes", "ssgd_mx_dense", "ssgd_mx_activation_backward_work_floats", "ssgd_mx_activation_backward", "ssgd_mx_transpose",
    "ssgd_rmsnorm", "ssgd_rmsnorm_work_floats", "ssgd_rmsnorm_backward",
    "ssgd_block_norm", "ssgd_block_norm_work_floats", "ssgd_block_norm_backward",
    "ssgd_destroy",
]


class SsgdError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"ssgd status {status}: {msg}")
        self.status = status


class DelayDist(C.Structure):
    _fields_ = [("kind", C.c_int32), ("shift", C.c_double), ("rate", C.c_double), ("alpha", C.c_double),
                ("scale", C.c_double), ("table", C.POINTER(C.c_float)), ("table_len", C.c_int64)]


class ModelDesc(C.Structure):
    _fields_ = [("kind", C.c_int32), ("d", C.c_int32), ("classes", C.c_int32), ("hidden", C.c_int32),
                ("bf16", C.c_int32), ("X", C.c_void_p), ("y", C.c_void_p), ("N", C.c_int64)]


class AdaSync(C.Structure):
    _fields_ = [("mode", C.c_int32), ("K0", C.c_int32), ("Kmax", C.c_int32), ("window", C.c_int32),
                ("rel_tol", C.c_double), ("interval_t", C.c_double)]


class AdamWOptions(C.Structure):
    _fields_ = [("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double), ("max_norm", C.c_double),
                ("state_bits", C.c_int32), ("seed", C.c_uint64)]


class MxEpilogue(C.Structure):
    _fields_ = [("gated", C.c_int32), ("activation", C.c_int32), ("bias_dtype", C.c_int32), ("residual_dtype", C.c_int32), ("out_dtype", C.c_int32),
                ("kept_dtype", C.c_int32), ("bias", C.c_void_p), ("residual", C.c_void_p), ("residual_pitch", C.c_int64), ("out", C.c_void_p),
                ("out_pitch", C.c_int64), ("values", C.c_void_p), ("scales", C.c_void_p), ("kept", C.c_void_p), ("kept_pitch", C.c_int64),
                ("kept_values", C.c_void_p), ("kept_scales", C.c_void_p)]


_lib = None


def _preload_hip_runtime():
    """PyTorch ships its own HIP runtime; the library must bind to that copy (one runtime per
    process), so it is loaded first, by path, whether or not torch has been imported yet."""
    import importlib.util
    spec = importlib.util.find_spec("torch")
    if spec is not None and spec.origin:
        cand = os.path.join(os.path.dirname(spec.origin), "lib", "libamdhip64.so")
        if os.path.exists(cand):
            C.CDLL(cand, mode=C.RTLD_GLOBAL)


def lib():
    """Load the built library; there is no fallback when it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise ImportError(f"{_LIB_PATH} is not built: run `python -m paper_2003_10579_amd.build`")
        _preload_hip_runtime()
        L = C.CDLL(_LIB_PATH)
        L.ssgd_create.argtypes = [C.POINTER(ModelDesc), C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                  C.POINTER(DelayDist), C.c_double, C.c_uint64, C.c_int32, C.POINTER(AdaSync),
                                  C.c_void_p, C.POINTER(C.c_void_p)]
        L.ssgd_run.argtypes = [C.c_void_p, C.c_int64]
        L.ssgd_reserve_trace.argtypes = [C.c_void_p, C.c_int64]
        L.ssgd_step.argtypes = [C.c_void_p, C.c_void_p]
        L.ssgd_param_count.restype = C.c_int64
        L.ssgd_param_count.argtypes = [C.c_void_p]
        L.ssgd_updates_done.restype = C.c_int64
        L.ssgd_updates_done.argtypes = [C.c_void_p]
        L.ssgd_current_K.argtypes = [C.c_void_p, C.c_int32]
        L.ssgd_trace_width.argtypes = [C.c_void_p]
        L.ssgd_get_trace.argtypes = [C.c_void_p, C.c_int32, C.c_int64, C.c_int64] + [C.c_void_p] * 6
        L.ssgd_get_params.argtypes = [C.c_void_p, C.c_int32, C.c_void_p]
        L.ssgd_set_params.argtypes = [C.c_void_p, C.c_int32, C.c_void_p]
        L.ssgd_force_K.argtypes = [C.c_void_p, C.c_int32]
        L.ssgd_full_loss.argtypes = [C.c_void_p, C.c_int32, C.POINTER(C.c_double)]
        L.ssgd_full_gradient.argtypes = [C.c_void_p, C.c_int32, C.c_void_p]
        L.ssgd_full_gradient_static.argtypes = [C.c_void_p, C.c_int32, C.c_void_p]
        L.ssgd_get_workers.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]
        L.ssgd_state_bytes.argtypes = [C.c_void_p, C.POINTER(C.c_int64)]
        L.ssgd_get_state.argtypes = [C.c_void_p, C.c_void_p, C.c_int64]
        L.ssgd_set_state.argtypes = [C.c_void_p, C.c_void_p, C.c_int64]
        L.ssgd_runtime_mc.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.POINTER(DelayDist), C.c_int64,
                                      C.c_int64, C.c_int32, C.c_uint64, C.c_void_p] + [C.c_void_p] * 5
        L.ssgd_debug_delays.argtypes = [C.POINTER(DelayDist), C.c_void_p, C.c_int64, C.c_void_p]
        L.ssgd_debug_batch.argtypes = [C.c_uint64, C.c_uint32, C.c_uint32, C.c_uint32, C.c_uint32, C.c_int32,
                                       C.c_int64, C.c_void_p]
        L.ssgd_stream_read_rate.argtypes = [C.c_void_p, C.c_int64, C.c_int32, C.c_void_p, C.POINTER(C.c_double)]
        L.ssgd_last_error.restype = C.c_char_p
        L.ssgd_last_error.argtypes = [C.c_void_p]
        L.ssgd_last_kernel_ms.argtypes = [C.c_void_p, C.POINTER(C.c_double), C.POINTER(C.c_int64)]
        L.ssgd_destroy.argtypes = [C.c_void_p]
        L.ssgd_adamw_state_elements.restype = C.c_int64
        L.ssgd_adamw_state_elements.argtypes = [C.c_int32, C.c_void_p]
        L.ssgd_adamw_create.argtypes = [C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.POINTER(AdamWOptions)] + [C.c_void_p] * 5
        L.ssgd_adamw_step.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_double, C.c_int64, C.c_void_p, C.c_void_p]
        L.ssgd_adamw_destroy.argtypes = [C.c_void_p]
        i32, i64, ptr = C.c_int32, C.c_int64, C.c_void_p
        L.ssgd_mx_row_bytes.restype = i64
        L.ssgd_mx_row_bytes.argtypes = [i32, i64]
        L.ssgd_mx_quantize.argtypes = [ptr, i32, i64, i64, i64, i32, ptr, ptr, i32, ptr, ptr, ptr]
        L.ssgd_mx_dequantize.argtypes = [ptr, ptr, i32, i64, i64, ptr, i32, i64, ptr]
        L.ssgd_mx_matmul_work_bytes.restype = i64
        L.ssgd_mx_matmul_work_bytes.argtypes = [i32, i64, i64, i64]
        L.ssgd_mx_matmul.argtypes = [ptr, ptr, i32, i64, ptr, ptr, i64, i64, ptr, i32, i64, ptr, ptr]
        L.ssgd_mx_linear_work_bytes.restype = i64
        L.ssgd_mx_linear_work_bytes.argtypes = [i32, i64, i64, i64]
        L.ssgd_mx_linear.argtypes = [ptr, i32, i64, i64, i32, ptr, ptr, i64, i64, ptr, i32, i64, ptr, ptr]
        L.ssgd_mx_dense_work_bytes.restype = i64
        L.ssgd_mx_dense_work_bytes.argtypes = [i32, i32, i32, i64, i64, i64]
        L.ssgd_mx_dense.argtypes = [ptr, i32, i64, ptr, ptr, i32, i64, ptr, ptr, i64, i64, C.POINTER(MxEpilogue), ptr, ptr]
        L.ssgd_mx_activation_backward_work_floats.restype = i64
        L.ssgd_mx_activation_backward_work_floats.argtypes = [i64, i64]
        L.ssgd_mx_activation_backward.argtypes = [ptr, i32, i64, i64, i64, i32, i32, ptr, i32, i64, ptr, ptr] + [i32, ptr, ptr] * 3 + [ptr, ptr, ptr]
        L.ssgd_mx_transpose.argtypes = [ptr, ptr, i32, i64, i64, i32, ptr, ptr, ptr]
        L.ssgd_block_norm.argtypes = ([ptr, i64, ptr, i64, ptr, i32, ptr, i32, ptr, i32, i64, i64, C.c_double, C.c_double, i32, i64, i64, ptr, i64, ptr, i64] +
                                      [ptr] * 5)
        L.ssgd_block_norm_work_floats.restype = i64
        L.ssgd_block_norm_work_floats.argtypes = [i64, i64, i64]
        L.ssgd_block_norm_backward.argtypes = ([ptr, i64, ptr, i64, ptr, i64, ptr, i32, ptr, i32, ptr, i32, i64, i64, C.c_double, ptr, ptr, ptr, i64, i32, i64, i64,
                                                ptr, i64, ptr, i64] + [ptr] * 5)
        L.ssgd_rmsnorm.argtypes = [ptr, i64, ptr, i64, ptr, i32, i32, i64, i64, C.c_double, ptr, i64, ptr, i64, ptr, ptr, ptr, ptr]
        L.ssgd_rmsnorm_work_floats.restype = i64
        L.ssgd_rmsnorm_work_floats.argtypes = [i64, i64]
        L.ssgd_rmsnorm_backward.argtypes = [ptr, i64, ptr, i64, ptr, i32, i32, ptr, ptr, i64, i64, i64, ptr, i64, ptr, ptr, ptr]
        _lib = L
    return _lib


def _check(status, ctx=None):
    if status != OK:
        raise SsgdError(status, (lib().ssgd_last_error(ctx) or b"").decode())


def delay_dist(kind, *args):
    """('exp', rate) | ('shifted_exp', shift, rate) | ('pareto', alpha, scale) | ('table', host array)."""
    d = DelayDist()
    d.shift, d.rate, d.alpha, d.scale, d.table, d.table_len = 0.0, 1.0, 1.0, 1.0, None, 0
    keep = None
    if kind == "exp":
        d.kind, d.rate = EXP, float(args[0])
    elif kind == "shifted_exp":
        d.kind, d.shift, d.rate = SHIFTED_EXP, float(args[0]), float(args[1])
    elif kind == "pareto":
        d.kind, d.alpha, d.scale = PARETO, float(args[0]), float(args[1])
    elif kind == "table":
        keep = np.ascontiguousarray(args[0], dtype=np.float32)
        d.kind, d.table, d.table_len = TABLE, keep.ctypes.data_as(C.POINTER(C.c_float)), keep.size
    else:
        raise ValueError(kind)
    d._keep = keep
    return d


class Context:
    """ssgd_ctx with the device tensors it borrows kept alive."""

    def __init__(self, kind, X, y, P, K, m, variant, dist, lr, seed=0, replicas=1, classes=1, hidden=0, bf16=0,
                 adasync=None, stream=None):
        import torch
        assert X.is_cuda and X.dtype == torch.float32 and X.is_contiguous()
        assert y.is_cuda and y.is_contiguous()
        self._X, self._y, self._dist = X, y, dist
        md = ModelDesc()
        md.kind = _KINDS[kind]
        md.N, md.d = X.shape
        md.classes, md.hidden, md.bf16 = classes, hidden, bf16
        md.X, md.y = X.data_ptr(), y.data_ptr()
        ada = None
        if adasync is not None:
            a = AdaSync()
            a.mode = adasync.get("mode", 0)
            a.K0 = adasync.get("K0", K)
            a.Kmax = adasync.get("Kmax", K)
            a.window = adasync.get("window", 200)
            a.rel_tol = adasync.get("rel_tol", 0.01)
            a.interval_t = adasync.get("interval_t", 1.0)
            ada = C.byref(a)
        if stream is None:
            stream = torch.cuda.current_stream(X.device).cuda_stream
        self.stream = stream
        h = C.c_void_p()
        with torch.cuda.device(X.device):
            _check(lib().ssgd_create(C.byref(md), P, K, m, _VARIANTS[variant], C.byref(dist), float(lr), seed,
                                     replicas, ada, C.c_void_p(stream), C.byref(h)))
        self.h = h
        self.P, self.replicas = P, replicas
        self.nw = int(lib().ssgd_param_count(h))
        self.width = int(lib().ssgd_trace_width(h))

    def close(self):
        if getattr(self, "h", None):
            lib().ssgd_destroy(self.h)
            self.h = None

    def __del__(self):
        self.close()

    def run(self, J):
        _check(lib().ssgd_run(self.h, J), self.h)

    def reserve_trace(self, updates):
        _check(lib().ssgd_reserve_trace(self.h, updates), self.h)

    def step(self, agg_out=None):
        _check(lib().ssgd_step(self.h, agg_out.data_ptr() if agg_out is not None else None), self.h)

    @property
    def updates(self):
        return int(lib().ssgd_updates_done(self.h))

    def current_K(self, replica=0):
        return int(lib().ssgd_current_K(self.h, replica))

    def force_K(self, K):
        _check(lib().ssgd_force_K(self.h, K), self.h)

    def full_loss(self, replica=0):
        v = C.c_double()
        _check(lib().ssgd_full_loss(self.h, replica, C.byref(v)), self.h)
        return v.value

    def full_gradient(self, replica=0):
        g = np.zeros(self.nw, dtype=np.float32)
        _check(lib().ssgd_full_gradient(self.h, replica, g.ctypes.data), self.h)
        return g

    def full_gradient_static(self, out, replica=0):
        """Same gradient into `out` (a device tensor of |w| floats), through the library's static scratch array:
        nothing is allocated, nothing is awaited (the work is enqueued on the context's stream)."""
        assert out.is_cuda and out.is_contiguous() and out.numel() >= self.nw and out.element_size() == 4
        _check(lib().ssgd_full_gradient_static(self.h, replica, out.data_ptr()), self.h)

    def workers(self, replica=0):
        tau = np.zeros(self.P, dtype=np.int32)
        ordn = np.zeros(self.P, dtype=np.int32)
        finish = np.zeros(self.P, dtype=np.float64)
        _check(lib().ssgd_get_workers(self.h, replica, tau.ctypes.data, ordn.ctypes.data, finish.ctypes.data), self.h)
        return dict(tau=tau, ordinal=ordn, finish=finish)

    def get_state(self):
        n = C.c_int64()
        _check(lib().ssgd_state_bytes(self.h, C.byref(n)), self.h)
        buf = np.zeros(n.value, dtype=np.uint8)
        _check(lib().ssgd_get_state(self.h, buf.ctypes.data, n.value), self.h)
        return buf

    def set_state(self, buf):
        buf = np.ascontiguousarray(buf, dtype=np.uint8)
        _check(lib().ssgd_set_state(self.h, buf.ctypes.data, buf.size), self.h)

    def params(self, replica=0):
        w = np.zeros(self.nw, dtype=np.float32)
        _check(lib().ssgd_get_params(self.h, replica, w.ctypes.data), self.h)
        return w

    def set_params(self, w, replica=0):
        w = np.ascontiguousarray(w, dtype=np.float32)
        assert w.size == self.nw
        _check(lib().ssgd_set_params(self.h, replica, w.ctypes.data), self.h)

    def trace(self, replica=0, start=0, n=None):
        n = self.updates - start if n is None else n
        W = self.width
        t = np.zeros(n, dtype=np.float64)
        loss = np.zeros(n, dtype=np.float32)
        K = np.zeros(n, dtype=np.int32)
        sel = np.zeros((n, W), dtype=np.int32)
        stale = np.zeros((n, W), dtype=np.int32)
        ordn = np.zeros((n, W), dtype=np.int32)
        _check(lib().ssgd_get_trace(self.h, replica, start, n, t.ctypes.data, loss.ctypes.data, K.ctypes.data,
                                    sel.ctypes.data, stale.ctypes.data, ordn.ctypes.data), self.h)
        return dict(t=t, loss=loss, K=K, sel=sel, staleness=stale, ordinal=ordn)

    def last_kernel_ms(self):
        ms, n = C.c_double(), C.c_int64()
        lib().ssgd_last_kernel_ms(self.h, C.byref(ms), C.byref(n))
        return ms.value, n.value


def runtime_mc(variant, P, Kmin, Kmax, dist, trials, chain_len, seed=0, trial0=0, per_trial=False, stream=None):
    nK = Kmax - Kmin + 1
    mean = np.zeros((nK, chain_len)); var = np.zeros((nK, chain_len))
    s = np.zeros((nK, chain_len)); s2 = np.zeros((nK, chain_len))
    pt = np.zeros((trials, nK, chain_len)) if per_trial else None
    _check(lib().ssgd_runtime_mc(_VARIANTS[variant], P, Kmin, Kmax, C.byref(dist), trial0, trials, chain_len, seed,
                                 C.c_void_p(stream) if stream else None, mean.ctypes.data, var.ctypes.data,
                                 s.ctypes.data, s2.ctypes.data, pt.ctypes.data if per_trial else None))
    return dict(mean=mean, var=var, sum=s, sumsq=s2, per_trial=pt)


def debug_delays(dist, bits):
    bits = np.ascontiguousarray(bits, dtype=np.uint32)
    out = np.zeros(bits.size, dtype=np.float32)
    _check(lib().ssgd_debug_delays(C.byref(dist), bits.ctypes.data, bits.size, out.ctypes.data))
    return out


def stream_read_rate(tensor, passes=10, stream=None):
    """Bytes per second of a plain streaming read of a device tensor (the achievable HBM ceiling)."""
    import torch
    handle = (stream or torch.cuda.current_stream()).cuda_stream
    out = C.c_double(0.0)
    _check(lib().ssgd_stream_read_rate(C.c_void_p(tensor.data_ptr()), tensor.numel() * tensor.element_size(), passes,
                                       C.c_void_p(handle), C.byref(out)))
    return out.value


def debug_batch(seed, replica, worker, ordinal, version, m, N):
    out = np.zeros(m, dtype=np.uint32)
    _check(lib().ssgd_debug_batch(seed, replica, worker, ordinal, version, m, N, out.ctypes.data))
    return out


# ---- operators of a low-precision training step: on the device and the current stream of their tensors ----------------
# They record no graph for autograd: backward passes are calls of their own (rmsnorm_backward, products with transposed quantisations), and a tensor
# that requires a gradient is taken with a warning where torch would record one.
# (A call's host time is what its caller waits for where the kernels are short, so checks build no text unless they fail and
# outputs share an allocation.)

_torch = _raw_stream = _device_now = _changed = None
_DTYPES = {}


def _load():
    """torch and what every call needs of it, looked up once."""
    global _torch, _raw_stream, _device_now, _changed
    import torch
    from torch.autograd.graph import increment_version as _changed
    lib()
    _DTYPES.update({torch.float32: F32, torch.bfloat16: BF16})
    _raw_stream, _device_now = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
    torch.cuda.init()
    _torch = torch


def _refuse(msg):
    raise SsgdError(EINVAL, msg)


def _dtype(t):
    kind = _DTYPES.get(t)
    return _refuse(f"float32 or bfloat16 is wanted, not {t}") if kind is None else kind


def _call(entry, device, *args):
    """One library call on the device and its current stream, which is the last argument of every operator."""
    index = device.index
    if _device_now() == index:
        status = entry(*args, _raw_stream(index))
    else:
        with _torch.cuda.device(device):
            status = entry(*args, _raw_stream(index))
    if status != OK:
        _check(status)


def _moment(name):
    """An array of the optimizer's state: its handle keeps the address, so what is assigned is copied into it."""
    def get(self):
        return self._moments[name]

    def put(self, value):
        own = self._moments[name]
        if own is None and value is None:
            return
        if not (own is not None and isinstance(value, _torch.Tensor) and value.shape == own.shape and value.dtype == own.dtype):
            _refuse(f"adamw: {name} takes a tensor of its own shape and type, where there is one")
        own.copy_(value.detach())
    return property(get, put)


class AdamW:
    """AdamW over many tensors at once (ssgd_adamw_*): fp32 parameters, updated in place; `copies` (a list of bfloat16
    tensors, entries may be None) receive them rounded.  The moments are `m` and `v`, flat arrays of 32-bit numbers or, with
    `state_bits=8`, of E4M3 values (of m and of the root of v) with a scale per 128 elements in `m_scale`, `v_scale`; `t`
    counts the updates.  These five are all that a checkpoint needs (a tensor that is assigned to one of the arrays is copied
    into it).  With `max_norm` gradients are clipped to that norm over all tensors, and `grad_norm` (one element on the
    device) holds the norm of the last step's."""

    m, v, m_scale, v_scale = (_moment(name) for name in ("m", "v", "m_scale", "v_scale"))

    def __init__(self, params, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, max_norm=0.0, state_bits=32, seed=0, copies=None):
        _torch or _load()
        torch = _torch
        self.h = None
        params = list(params)
        if not params:
            _refuse("adamw: at least one tensor")
        dev = params[0].device
        copies = [None] * len(params) if copies is None else list(copies)
        decay = [float(weight_decay)] * len(params) if isinstance(weight_decay, (int, float)) else [float(w) for w in weight_decay]
        if len(copies) != len(params) or len(decay) != len(params):
            _refuse("adamw: one copy and one weight decay per tensor")
        for p, c in zip(params, copies):
            if not (p.is_cuda and p.device == dev and p.dtype == torch.float32 and p.is_contiguous()):
                _refuse("adamw: parameters are contiguous float32 tensors of one GPU")
            if not (c is None or (c.device == dev and c.dtype == torch.bfloat16 and c.is_contiguous() and c.numel() == p.numel())):
                _refuse("adamw: copies are contiguous bfloat16 tensors of their parameter's size")
        n = len(params)
        self._sizes = [p.numel() for p in params]
        sizes = (C.c_int64 * n)(*self._sizes)
        total = lib().ssgd_adamw_state_elements(n, sizes)
        if state_bits not in (8, 32):
            _refuse("adamw: state_bits is 8 or 32")
        moment = lambda: torch.zeros(total, device=dev, dtype=torch.float32 if state_bits == 32 else torch.float8_e4m3fn)  # noqa: E731
        scale = lambda: torch.zeros(total // 128, device=dev) if state_bits == 8 else None  # noqa: E731
        self._moments = {"m": moment(), "v": moment(), "m_scale": scale(), "v_scale": scale()}
        self.grad_norm = torch.zeros(1, device=dev) if max_norm else None
        self.t = 0
        self._written = params + [c for c in copies if c is not None]
        self._places = [p.data_ptr() for p in self._written]
        self._device, self._grads = dev, (C.c_void_p * n)()
        pointers = C.c_void_p * n
        o = AdamWOptions(float(betas[0]), float(betas[1]), float(eps), float(max_norm), state_bits, seed)
        h = C.c_void_p()
        with torch.cuda.device(dev):
            _check(lib().ssgd_adamw_create(
                n, sizes, pointers(*[p.data_ptr() for p in params]), pointers(*[None if c is None else c.data_ptr() for c in copies]),
                (C.c_double * n)(*decay), C.byref(o), self.m.data_ptr(), self.v.data_ptr(),
                None if self.m_scale is None else self.m_scale.data_ptr(), None if self.v_scale is None else self.v_scale.data_ptr(), C.byref(h)))
        self.h = h

    def step(self, grads, lr):
        """One update with a list of gradients, contiguous tensors of one type (float32 or bfloat16) and their parameters' sizes.
        Parameters and copies have to be where they were when the optimizer was made."""
        if self.h is None:
            _refuse("adamw: closed")
        if len(grads) != len(self._sizes):
            _refuse("adamw step: one gradient per tensor")
        place_of = _torch.Tensor.data_ptr
        if list(map(place_of, self._written)) != self._places:
            _refuse("adamw step: a parameter or its copy has moved since the optimizer was made")
        kind, dev, at = grads[0].dtype, self._device, self._grads
        for g, n in zip(grads, self._sizes):
            if not (g.dtype is kind and g.numel() == n and g.device == dev and g.is_contiguous()):
                _refuse("adamw step: gradients are contiguous tensors of one type, of their parameters' sizes and device")
        at[:] = list(map(place_of, grads))
        _call(_lib.ssgd_adamw_step, dev, self.h, at, _dtype(kind), lr, self.t + 1, None if self.grad_norm is None else self.grad_norm.data_ptr())
        _changed(self._written)        # (autograd's check of what it has kept for a backward pass)
        self.t += 1

    def close(self):
        if getattr(self, "h", None):
            _lib.ssgd_adamw_destroy(self.h)
            self.h = None

    def __reduce__(self):          # (both would free the handle)
        _refuse("adamw: an optimizer cannot be copied or pickled; its state is m, v, m_scale, v_scale and t")

    def __del__(self):
        if _lib is not None:        # the interpreter may be past it
            self.close()


def _unrecorded(what):
    warnings.warn(f"{what}: no graph is recorded, so this tensor gets no gradient through it (the gradients have calls of their own; "
                  "detached tensors or torch.no_grad() say that this is meant)", stacklevel=4)


def _matrix(x, what):
    """(device, dtype, rows, cols, pitch) of a matrix with contiguous rows."""
    _torch or _load()
    if not x.is_cuda or x.dim() != 2:
        _refuse(f"{what}: a matrix on the GPU is wanted")
    if x.requires_grad and _torch.is_grad_enabled():
        _unrecorded(what)
    rows, cols = x.shape
    pitch, step = x.stride()
    if rows <= 1:
        pitch = cols
    if (step != 1 and cols > 1) or pitch < cols:
        _refuse(f"{what}: rows have to be contiguous")
    kind = _DTYPES.get(x.dtype)
    return x.device, _dtype(x.dtype) if kind is None else kind, rows, cols, pitch


class MxTensor:
    """A microscaled matrix: `values` (uint8, rows x bytes; two E2M1 or one E4M3 number to a byte) and `scales` (uint8, 2^(byte - 127) per
    32 columns), both padded with zeros to a multiple of 128 columns.  `format` is "fp4" or "fp8", `shape` (rows, cols)."""

    __slots__ = ("format", "shape", "device", "_values", "_scales", "_room", "_at")

    def __init__(self, values, scales, format, shape):
        if format not in _FORMATS:
            _refuse("mx: the format is 'fp4' or 'fp8'")
        rows, cols = shape
        wide = -(-cols // 128) * 128
        if not (values.is_cuda and values.is_contiguous() and scales.is_contiguous() and scales.device == values.device and
                values.element_size() == scales.element_size() == 1 and
                tuple(values.shape) == (rows, wide // 2 if format == "fp4" else wide) and tuple(scales.shape) == (rows, wide // 32)):
            _refuse(f"mx: values and scales do not have the layout of {rows} x {cols}")
        _torch or _load()          # (with stored arrays this may be a program's first call)
        self.format, self.shape, self.device, self._room = format, (rows, cols), values.device, None
        self._values, self._scales, self._at = values, scales, (values.data_ptr(), scales.data_ptr())

    def __reduce__(self):          # (a copy or a stored one has addresses of its own)
        return MxTensor, (self.values, self.scales, self.format, self.shape)

    @classmethod
    def empty(cls, rows, cols, format, device):
        _torch or _load()
        if format not in _FORMATS:
            _refuse("mx: the format is 'fp4' or 'fp8'")
        q = cls.__new__(cls)
        wide = (cols + 127) // 128 * 128
        bytes = rows * (wide // 2 if format == "fp4" else wide)
        q._room = room = _torch.empty(bytes + rows * (wide // 32), dtype=_torch.uint8, device=device)
        at = room.data_ptr()
        q.format, q.shape, q.device, q._values, q._scales, q._at = format, (rows, cols), room.device, None, None, (at, at + bytes)
        return q

    # (views of one allocation, made when they are asked for)
    def _view(self, first, width):
        return self._room.as_strided((self.shape[0], width), (width, 1), first)

    @property
    def values(self):
        if self._values is None:
            wide = (self.shape[1] + 127) // 128 * 128
            self._values = self._view(0, wide // 2 if self.format == "fp4" else wide)
        return self._values

    @property
    def scales(self):
        if self._scales is None:
            self._scales = self._view(self._at[1] - self._at[0], (self.shape[1] + 127) // 128 * 4)
        return self._scales


def mx_quantize(x, format="fp4"):
    """The rows of a matrix (float32 or bfloat16) as an MxTensor."""
    dev, kind, rows, cols, pitch = _matrix(x, "mx_quantize")
    q = MxTensor.empty(rows, cols, format, dev)
    _call(_lib.ssgd_mx_quantize, dev, x.data_ptr(), kind, rows, cols, pitch, _FORMATS[format], *q._at, 0, None, None)
    return q


def mx_quantize_transposed(x, format="fp4"):
    """The columns of a matrix as the rows of an MxTensor."""
    dev, kind, rows, cols, pitch = _matrix(x, "mx_quantize_transposed")
    q = MxTensor.empty(cols, rows, format, dev)
    _call(_lib.ssgd_mx_quantize, dev, x.data_ptr(), kind, rows, cols, pitch, 0, None, None, _FORMATS[format], *q._at)
    return q


def mx_quantize_both(x, format="fp4", format_transposed="fp4"):
    """(mx_quantize(x), mx_quantize_transposed(x)) from one read of x."""
    dev, kind, rows, cols, pitch = _matrix(x, "mx_quantize_both")
    q, t = MxTensor.empty(rows, cols, format, dev), MxTensor.empty(cols, rows, format_transposed, dev)
    _call(_lib.ssgd_mx_quantize, dev, x.data_ptr(), kind, rows, cols, pitch, _FORMATS[format], *q._at, _FORMATS[format_transposed], *t._at)
    return q, t


def mx_dequantize(q, dtype=None):
    """The values of an MxTensor as a matrix of `dtype` (float32 unless it is given, or bfloat16)."""
    if not isinstance(q, MxTensor):
        _refuse("mx_dequantize: an MxTensor is wanted")
    rows, cols = q.shape
    kind = F32 if dtype is None else _dtype(dtype)
    out = _torch.empty(rows, cols, dtype=dtype or _torch.float32, device=q.device)
    _call(_lib.ssgd_mx_dequantize, q.device, *q._at, _FORMATS[q.format], rows, cols, out.data_ptr(), kind, cols)
    return out


def _work(bytes, device):
    return _torch.empty(bytes, dtype=_torch.uint8, device=device) if bytes > 0 else None


def mx_matmul(a, b, dtype=None):
    """a b^T of two MxTensors with equal numbers of columns, a in either format, b in "fp4", as a matrix of `dtype` (bfloat16 unless
    it is given, or float32).  With a in "fp4" float32 results are rounded as fp32 sums are; with a in "fp8" the matrix unit drops
    what is below about 2^-14 of the largest of 128 products, 4e-6 of a typical result, so float32 does not add what bfloat16 lacks."""
    if not (isinstance(a, MxTensor) and isinstance(b, MxTensor) and b.format == "fp4" and a.shape[1] == b.shape[1] and a.device == b.device):
        _refuse("mx_matmul: an MxTensor and an 'fp4' MxTensor of as many columns on its device are wanted")
    (M, K), N, dev = a.shape, b.shape[0], a.device
    kind = BF16 if dtype is None else _dtype(dtype)
    out = _torch.empty(M, N, dtype=dtype or _torch.bfloat16, device=dev)
    f = _FORMATS[a.format]
    work = _work(_lib.ssgd_mx_matmul_work_bytes(f, M, N, K), dev)
    _call(_lib.ssgd_mx_matmul, dev, *a._at, f, M, *b._at, N, K, out.data_ptr(), kind, N, None if work is None else work.data_ptr())
    return out


def mx_linear(x, w, format="fp8", dtype=None):
    """x w^T for rows x (float32 or bfloat16), quantised to `format` on the way, and an "fp4" MxTensor w (outputs x inputs), as a
    matrix of `dtype` (x's unless it is given).  Autograd records nothing."""
    dev, kind, M, K, pitch = _matrix(x, "mx_linear")
    if format not in _FORMATS:
        _refuse("mx_linear: the format is 'fp4' or 'fp8'")
    if not (isinstance(w, MxTensor) and w.format == "fp4" and w.shape[1] == K and w.device == dev):
        _refuse("mx_linear: w is an 'fp4' MxTensor with x's columns, on its device")
    N, f = w.shape[0], _FORMATS[format]
    out_kind = kind if dtype is None else _dtype(dtype)
    out = _torch.empty(M, N, dtype=dtype or x.dtype, device=dev)
    work = _work(_lib.ssgd_mx_linear_work_bytes(f, M, N, K), dev)
    _call(_lib.ssgd_mx_linear, dev, x.data_ptr(), kind, pitch, M, f, *w._at, N, K, out.data_ptr(), out_kind, N, None if work is None else work.data_ptr())
    return out


def _beside(t, x, what):
    """(pointer, pitch) of a matrix of the shape, type and device of x, or of none."""
    if t is None:
        return None, 0
    if t.shape != x.shape or t.dtype != x.dtype or t.device != x.device:
        _refuse(f"{what}: the shape, type and device of the first matrix are wanted")
    return t.data_ptr(), _matrix(t, what)[4]


def _weight(w, x, what):
    if not (w.dim() == 1 and w.numel() == x.shape[1] and w.is_contiguous() and w.device == x.device):
        _refuse(f"{what}: a contiguous weight per column is wanted")
    if w.requires_grad and _torch.is_grad_enabled():
        _unrecorded(what)
    return w.data_ptr(), _dtype(w.dtype)


def rmsnorm(x, weight, residual=None, eps=1e-6, output=None):
    """(y, s, rstd) of the root-mean-square norm of the rows of s = x + residual (s = x without one).  y has x's type or, with
    output="fp8", is an MxTensor for the product behind it; s and rstd are what rmsnorm_backward takes (autograd records nothing)."""
    dev, kind, rows, d, pitch = _matrix(x, "rmsnorm")
    if output is not None and output != "fp8":
        _refuse("rmsnorm: the output is None (x's type) or 'fp8'")
    w, w_kind = _weight(weight, x, "rmsnorm")
    r, r_pitch = _beside(residual, x, "rmsnorm")
    if residual is None:
        total, total_at = x, None
    else:
        total = _torch.empty(rows, d, dtype=x.dtype, device=dev)
        total_at = total.data_ptr()
    rstd = _torch.empty(rows, dtype=_torch.float32, device=dev)
    if output is None:
        y = _torch.empty(rows, d, dtype=x.dtype, device=dev)
        to = (y.data_ptr(), d, None, None)
    else:
        y = MxTensor.empty(rows, d, "fp8", dev)
        to = (None, 0, *y._at)
    _call(_lib.ssgd_rmsnorm, dev, x.data_ptr(), pitch, r, r_pitch, w, kind, w_kind, rows, d, eps, total_at, d, *to, rstd.data_ptr())
    return y, total, rstd


def rmsnorm_backward(dy, s, weight, rstd, dsum=None):
    """(dx, dweight) from the gradient dy of the norm's output and, where there is one, dsum that reaches s past it.  dx is the
    gradient of x and of the residual; dweight is float32."""
    dev, kind, rows, d, pitch = _matrix(dy, "rmsnorm_backward")
    w, w_kind = _weight(weight, dy, "rmsnorm_backward")
    s_at, s_pitch = _beside(s, dy, "rmsnorm_backward")
    if not (rstd.dtype == _torch.float32 and rstd.shape == (rows,) and rstd.is_contiguous() and rstd.device == dev):
        _refuse("rmsnorm_backward: one float32 rstd per row is wanted")
    more, more_pitch = _beside(dsum, dy, "rmsnorm_backward")
    dx = _torch.empty(rows, d, dtype=dy.dtype, device=dev)
    dw = _torch.empty(d, dtype=_torch.float32, device=dev)
    floats = _lib.ssgd_rmsnorm_work_floats(rows, d)
    if floats < 0:
        _refuse("rmsnorm_backward: 1 <= columns < 2^25")
    work = _torch.empty(floats, dtype=_torch.float32, device=dev)
    _call(_lib.ssgd_rmsnorm_backward, dev, dy.data_ptr(), pitch, s_at, s_pitch, w, kind, w_kind, rstd.data_ptr(), more, more_pitch, rows, d, dx.data_ptr(), d,
          dw.data_ptr(), work.data_ptr())
    return dx, dw


# ---- a gated feed-forward block in few bits: what lies between its products ---------------------------------------------------------------------------

def _activation(name, what):
    kind = _ACTIVATIONS.get(name)
    return _refuse(f"{what}: the activation is None, 'relu', 'gelu' or 'silu'") if kind is None else kind


def _epilogue(what, x, w, gated, activation, bias, residual, format, dtype, output, keep):
    if isinstance(x, MxTensor):
        (M, K), dev, f = x.shape, x.device, _FORMATS[x.format]
        rows, kind, like = (None, 0, 0, *x._at), BF16, _torch.bfloat16
    else:
        dev, kind, M, K, pitch = _matrix(x, what)
        if format not in _FORMATS:
            _refuse(f"{what}: the format is 'fp4' or 'fp8'")
        f, rows, like = _FORMATS[format], (x.data_ptr(), kind, pitch, None, None), x.dtype
    if not (isinstance(w, MxTensor) and w.format == "fp4" and w.shape[1] == K and w.device == dev):
        _refuse(f"{what}: w is an 'fp4' MxTensor with x's columns, on its device")
    N = w.shape[0]
    if gated and N % 2:
        _refuse(f"{what}: w has gate and up rows in turn")
    if dtype is not None:
        kind, like = _dtype(dtype), dtype
    if output is not None and output != "fp8":
        _refuse(f"{what}: the output is None (a matrix) or 'fp8'")
    if keep is not None and keep != "same" and keep != "fp8":
        _refuse(f"{what}: what is kept is None, 'same' (a matrix of the output's type) or 'fp8'")
    e = MxEpilogue(gated, _activation(activation, what))
    if bias is not None:
        if not (bias.dim() == 1 and bias.numel() == N and bias.is_contiguous() and bias.device == dev):
            _refuse(f"{what}: a contiguous bias per output is wanted")
        if bias.requires_grad and _torch.is_grad_enabled():
            _unrecorded(what)
        e.bias, e.bias_dtype = bias.data_ptr(), _dtype(bias.dtype)
    if residual is not None:
        if residual.shape != (M, N) or residual.device != dev:
            _refuse(f"{what}: a residual of the output's shape, on its device, is wanted")
        _, e.residual_dtype, _, _, e.residual_pitch = _matrix(residual, what)
        e.residual = residual.data_ptr()
    results = N // 2 if gated else N
    if output is None:
        out = _torch.empty(M, results, dtype=like, device=dev)
        e.out, e.out_pitch, e.out_dtype = out.data_ptr(), results, kind
    else:
        out = MxTensor.empty(M, results, "fp8", dev)
        e.values, e.scales = out._at
    if keep is not None:
        if keep == "fp8":
            kept = MxTensor.empty(M, N, "fp8", dev)
            e.kept_values, e.kept_scales = kept._at
        else:
            kept = _torch.empty(M, N, dtype=like, device=dev)
            e.kept, e.kept_pitch, e.kept_dtype = kept.data_ptr(), N, kind
    work = _work(_lib.ssgd_mx_dense_work_bytes(f, rows[0] is not None, output is not None or keep == "fp8", M, N, K), dev)
    _call(_lib.ssgd_mx_dense, dev, *rows, f, M, *w._at, N, K, e, None if work is None else work.data_ptr())
    return out if keep is None else (out, kept)


def mx_dense(x, w, bias=None, activation=None, residual=None, format="fp8", dtype=None, output=None, keep=None):
    """residual + act(x w^T + bias) in one pass, for an MxTensor x or rows (float32 or bfloat16) that are quantised to `format` on the way, and an "fp4"
    MxTensor w (outputs x inputs).  activation: None, "relu", "gelu" or "silu".  The result is a matrix of `dtype` (x's unless it is given, bfloat16 for an
    MxTensor) or, with output="fp8", an MxTensor for the product behind it.  keep="same" (a matrix of dtype) or "fp8" (an MxTensor, a checkpoint in 8 bits)
    gives (result, x w^T + bias): what mx_dense_backward takes.  The product is as exact as mx_matmul's.  Autograd records nothing."""
    return _epilogue("mx_dense", x, w, 0, activation, bias, residual, format, dtype, output, keep)


def gate_up(gate, up):
    """The weight of mx_gated from those of both projections (hidden x inputs each): their rows in turn."""
    if gate.dim() != 2 or gate.shape != up.shape or gate.dtype != up.dtype or gate.device != up.device:
        _refuse("gate_up: two matrices of one shape, type and device are wanted")
    import torch
    return torch.stack((gate, up), 1).flatten(0, 1)


def mx_gated(x, w, activation="silu", format="fp8", dtype=None, output=None, keep=None):
    """Both projections of a gated feed-forward block, its activation and their product in one pass: h[:, c] = act(p[:, 2 c]) p[:, 2 c + 1] with
    p = x w^T, w an "fp4" MxTensor whose rows are gate and up in turn (gate_up).  The other arguments, and (h, p), as for mx_dense; p is what
    mx_gated_backward takes."""
    return _epilogue("mx_gated", x, w, 1, activation, None, None, format, dtype, output, keep)


def _activation_backward(what, dy, p, gated, activation, hidden, format, format_transposed, bias):
    dev, kind, rows, cols, pitch = _matrix(dy, what)
    act = _activation(activation, what)
    wide = 2 * cols if gated else cols
    if p is None and not gated and act == ACT_NONE and hidden is None:
        kept = (None, 0, 0, None, None)
    elif isinstance(p, MxTensor):
        if p.format != "fp8" or p.shape != (rows, wide) or p.device != dev:
            _refuse(f"{what}: what the forward pass has kept is wanted")
        kept = (None, 0, 0, *p._at)
    else:
        if p is None or p.shape != (rows, wide) or p.device != dev:
            _refuse(f"{what}: what the forward pass has kept is wanted")
        _, p_kind, _, _, p_pitch = _matrix(p, what)
        kept = (p.data_ptr(), p_kind, p_pitch, None, None)
    q, t = MxTensor.empty(rows, wide, format, dev), MxTensor.empty(wide, rows, format_transposed, dev)
    h = None if hidden is None else MxTensor.empty(cols, rows, hidden, dev)
    db = work = None
    if bias:
        floats = _lib.ssgd_mx_activation_backward_work_floats(rows, cols)
        if floats < 0:
            _refuse(f"{what}: rows < 2^31, columns up to 2^24 - 128")
        db = _torch.empty(cols, dtype=_torch.float32, device=dev)
        work = _torch.empty(floats, dtype=_torch.float32, device=dev) if floats else None
    _call(_lib.ssgd_mx_activation_backward, dev, dy.data_ptr(), kind, pitch, rows, cols, gated, act, *kept, _FORMATS[format], *q._at, _FORMATS[format_transposed], *t._at,
          *((0, None, None) if h is None else (_FORMATS[hidden], *h._at)), None if db is None else db.data_ptr(), None if work is None else work.data_ptr())
    return q, t, h, db


def mx_dense_backward(dy, p, activation=None, hidden=None, format="fp8", format_transposed="fp8", bias=True):
    """(d, dt, ht, dbias) from the gradient dy of act(p), p = x w^T + bias as mx_dense has kept it (a matrix or an "fp8" MxTensor; None will do without an
    activation).  d = dy act'(p) along its rows is for the gradient of x (a product with w's transposed quantisation), dt along its columns for that of w (one with
    x's, which mx_transpose gives); ht is act(p) along its columns in the format `hidden`, for the next weight's gradient, or None; dbias is float32, or None."""
    return _activation_backward("mx_dense_backward", dy, p, 0, activation, hidden, format, format_transposed, bias)


def mx_gated_backward(dh, p, activation="silu", hidden="fp4", format="fp8", format_transposed="fp8"):
    """(d, dt, ht) from the gradient dh of a gated block's h and its p as mx_gated has kept it: d and dt are the gradient of p, gate and up in turn, along its
    rows and columns, and ht is h along its columns in the format `hidden`, or None."""
    return _activation_backward("mx_gated_backward", dh, p, 1, activation, hidden, format, format_transposed, False)[:3]


def mx_transpose(q, format="fp4"):
    """The columns of an MxTensor, from the values that it stands for, as the rows of one in `format`: a checkpoint as the right operand of a weight's
    gradient."""
    if not isinstance(q, MxTensor):
        _refuse("mx_transpose: an MxTensor is wanted")
    rows, cols = q.shape
    t = MxTensor.empty(cols, rows, format, q.device)
    _call(_lib.ssgd_mx_transpose, q.device, *q._at, _FORMATS[q.format], rows, cols, _FORMATS[format], *t._at)
    return t


def _gate(gate, rows, d, dev, what):
    """(pointer, type, number, pitch) of a gate per column (d), or of one for each of several runs of rows (gates x d)."""
    if gate is None:
        return None, 0, 1, 0
    if gate.dim() == 1 and gate.numel() == d and gate.is_contiguous() and gate.device == dev:
        if gate.requires_grad and _torch.is_grad_enabled():
            _unrecorded(what)
        return gate.data_ptr(), _dtype(gate.dtype), 1, d
    if not (gate.shape == (d,) or (gate.dim() == 2 and gate.shape[1] == d and gate.shape[0] > 0 and rows % gate.shape[0] == 0)) or gate.device != dev:
        _refuse(f"{what}: a gate per column, or one for each of several equal runs of rows, is wanted")
    _, kind, gates, _, pitch = _matrix(gate if gate.dim() == 2 else gate.unsqueeze(0), what)
    return gate.data_ptr(), kind, gates, pitch


def block_norm(o, s, post_weight, weight, gate=None, scale=1.0, eps=1e-6, output=None):
    """(y, sum, rstd_o, rstd) between two blocks of a residual stream: sum = scale s + gate norm(o) post_weight and y = norm(sum) weight, with the root-mean-square
    norm of rows.  gate: None, one value per column, or a row of them for each of several equal runs of rows; scale: a number.  y has the rows' type or, with
    output="fp8", is an MxTensor for the product behind it; the rest is what block_norm_backward takes (autograd records nothing)."""
    dev, kind, rows, d, pitch = _matrix(o, "block_norm")
    if output is not None and output != "fp8":
        _refuse("block_norm: the output is None (the rows' type) or 'fp8'")
    s_at, s_pitch = _beside(s, o, "block_norm")
    post, post_kind = _weight(post_weight, o, "block_norm")
    w, w_kind = _weight(weight, o, "block_norm")
    gate_at, gate_kind, gates, gate_pitch = _gate(gate, rows, d, dev, "block_norm")
    total, rstd_o, rstd = _torch.empty(rows, d, dtype=o.dtype, device=dev), _torch.empty(rows, dtype=_torch.float32, device=dev), _torch.empty(rows, dtype=_torch.float32, device=dev)
    if output is None:
        y = _torch.empty(rows, d, dtype=o.dtype, device=dev)
        to = (y.data_ptr(), d, None, None)
    else:
        y = MxTensor.empty(rows, d, "fp8", dev)
        to = (None, 0, *y._at)
    _call(_lib.ssgd_block_norm, dev, o.data_ptr(), pitch, s_at, s_pitch, post, post_kind, w, w_kind, gate_at, gate_kind, gates, gate_pitch, scale, eps, kind, rows, d,
          total.data_ptr(), d, *to, rstd_o.data_ptr(), rstd.data_ptr())
    return y, total, rstd_o, rstd


def block_norm_backward(dy, o, sum, post_weight, weight, rstd_o, rstd, gate=None, scale=1.0, dsum=None):
    """(do, ds, dpost_weight, dweight, dgate) from the gradient dy of block_norm's y and, where there is one, dsum that reaches the sum past the second norm.
    The gradients of the weights and of the gate (None without one) are float32."""
    dev, kind, rows, d, pitch = _matrix(dy, "block_norm_backward")
    o_at, o_pitch = _beside(o, dy, "block_norm_backward")
    sum_at, sum_pitch = _beside(sum, dy, "block_norm_backward")
    more, more_pitch = _beside(dsum, dy, "block_norm_backward")
    post, post_kind = _weight(post_weight, dy, "block_norm_backward")
    w, w_kind = _weight(weight, dy, "block_norm_backward")
    for r in (rstd_o, rstd):
        if not (r.dtype == _torch.float32 and r.shape == (rows,) and r.is_contiguous() and r.device == dev):
            _refuse("block_norm_backward: one float32 rstd per row of both norms is wanted")
    gate_at, gate_kind, gates, gate_pitch = _gate(gate, rows, d, dev, "block_norm_backward")
    grad_o, grad_s = _torch.empty(rows, d, dtype=dy.dtype, device=dev), _torch.empty(rows, d, dtype=dy.dtype, device=dev)
    dpost, dw = _torch.empty(d, dtype=_torch.float32, device=dev), _torch.empty(d, dtype=_torch.float32, device=dev)
    dgate = None if gate is None else _torch.empty(gate.shape, dtype=_torch.float32, device=dev)
    floats = _lib.ssgd_block_norm_work_floats(rows, d, gates)
    if floats < 0:
        _refuse("block_norm_backward: rows < 2^31, 1 <= columns < 2^24")
    work = _torch.empty(floats, dtype=_torch.float32, device=dev)
    _call(_lib.ssgd_block_norm_backward, dev, dy.data_ptr(), pitch, o_at, o_pitch, sum_at, sum_pitch, post, post_kind, w, w_kind, gate_at, gate_kind, gates, gate_pitch, scale,
          rstd_o.data_ptr(), rstd.data_ptr(), more, more_pitch, kind, rows, d, grad_o.data_ptr(), d, grad_s.data_ptr(), d, dpost.data_ptr(), dw.data_ptr(), None if dgate is None else dgate.data_ptr(),
          work.data_ptr())
    return grad_o, grad_s, dpost, dw, dgate
