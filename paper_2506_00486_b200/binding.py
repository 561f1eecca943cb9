"""ctypes binding of libgg_b200.so: argument marshalling only.

Every step of the pass runs in the CUDA library; this module turns torch tensors into the
pointers and sizes of the C interface (include/gg.h) and allocates output tensors.  There is
no CPU fallback: if the library is missing or the device is not a B200-class GPU the calls raise.
"""
import ctypes
import os

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# GG_B200_LIB selects another build of the same library (the bounds-checking one of build.py --bounds)
_LIB_PATH = os.environ.get("GG_B200_LIB") or os.path.join(_HERE, "libgg_b200.so")

GG_F32, GG_BF16 = 0, 1
GG_SUM, GG_MEAN = 0, 1
GG_PARAMS_FITTED, GG_PARAMS_GIVEN, GG_RATE_EG = 0, 1, 2
GG_STEP_GIVEN, GG_STEP_FROM_ALPHA = 0, 1
FLAG_DEGENERATE, FLAG_BETA_CLAMPED_LO, FLAG_BETA_CLAMPED_HI, FLAG_NONFINITE, FLAG_CLAMPED_SYMBOLS = 1, 2, 4, 8, 16
FLAG_TIMEOUT = 32
HOOK_RESIDENT_MODE, HOOK_EXTRA_ARRIVALS, HOOK_WAIT_CAP, HOOK_CLUSTER_MODE = 0, 1, 2, 3
BETA_LO, BETA_HI = 0.05, 20.0
ACTIVATIONS = {"silu": 0, "gelu": 1, "gelu_tanh": 2, "relu": 3}
ADAMW_BLOCK = 256          # elements that share one scale of an 8-bit AdamW state
DROPOUT_SEED = 1 << 32     # make_dropout's default: not make_adamw_step's, which would round by the bits that drop

_SEG_DTYPE = np.dtype([("ptr", np.uint64), ("len", np.int64)])
_P = ctypes.c_void_p


class FusedArgs(ctypes.Structure):
    """Mirror of gg_fused_args."""
    _fields_ = [
        ("segs", _P), ("n_seg", ctypes.c_int32), ("in_dtype", ctypes.c_int32),
        ("beta", _P), ("alpha", _P), ("sum_abs", _P), ("sum_sq", _P), ("count", _P), ("flags", _P),
        ("param_mode", ctypes.c_int32), ("beta_in", _P), ("alpha_in", _P),
        ("lam", ctypes.c_double), ("reduction", ctypes.c_int32),
        ("grad", _P), ("grad_dtype", ctypes.c_int32), ("accumulate_grad", ctypes.c_int32),
        ("penalty", _P),
        ("step_mode", ctypes.c_int32), ("step", _P), ("step_scale", ctypes.c_double), ("step_out", _P),
        ("hist_id", _P), ("n_hist", ctypes.c_int32), ("qmin", ctypes.c_int32), ("qmax", ctypes.c_int32),
        ("hist", _P), ("accumulate_hist", ctypes.c_int32), ("entropy_bits", _P), ("clamped_lo_hi", _P),
        ("eg_k", ctypes.c_int32), ("eg_bits", _P),
    ]


class ChannelArgs(ctypes.Structure):
    """Mirror of gg_channel_args."""
    _fields_ = [
        ("x", _P), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("ld", ctypes.c_int64),
        ("in_dtype", ctypes.c_int32),
        ("beta", _P), ("alpha", _P), ("sum_abs", _P), ("sum_sq", _P), ("count", _P), ("flags", _P),
        ("lam", ctypes.c_double), ("reduction", ctypes.c_int32),
        ("grad", _P), ("grad_ld", ctypes.c_int64), ("grad_dtype", ctypes.c_int32),
        ("accumulate_grad", ctypes.c_int32), ("penalty", _P),
        ("step", ctypes.c_float), ("qmin", ctypes.c_int32), ("qmax", ctypes.c_int32),
        ("hist", _P), ("accumulate_hist", ctypes.c_int32), ("entropy_bits", _P), ("clamped_lo_hi", _P),
    ]


class LayerNormArgs(ctypes.Structure):
    """Mirror of gg_layer_norm_args."""
    _fields_ = [
        ("x", _P), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("x_ld", ctypes.c_int64), ("dtype", ctypes.c_int32),
        ("weight", _P), ("bias", _P), ("w_dtype", ctypes.c_int32), ("eps", ctypes.c_double),
        ("y", _P), ("y_ld", ctypes.c_int64), ("mean", _P), ("rstd", _P),
    ]


class LayerNormGradArgs(ctypes.Structure):
    """Mirror of gg_layer_norm_grad_args."""
    _fields_ = [
        ("dy", _P), ("x", _P), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("dy_ld", ctypes.c_int64),
        ("x_ld", ctypes.c_int64), ("dtype", ctypes.c_int32), ("mean", _P), ("rstd", _P),
        ("weight", _P), ("w_dtype", ctypes.c_int32), ("dx", _P), ("dx_ld", ctypes.c_int64),
        ("dweight", _P), ("dbias", _P), ("accumulate", ctypes.c_int32),
    ]


class AdamwArgs(ctypes.Structure):
    """Mirror of gg_adamw_args."""
    _fields_ = [
        ("n_seg", ctypes.c_int32), ("w", _P), ("w_dtype", ctypes.c_int32), ("g", _P), ("g_dtype", ctypes.c_int32),
        ("w_copy", _P), ("state_bits", ctypes.c_int32), ("m", _P), ("v", _P), ("m_scale", _P), ("v_scale", _P),
        ("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double),
        ("weight_decay", ctypes.c_double), ("decay", _P), ("grad_scale", _P), ("t", ctypes.c_int64), ("seed", ctypes.c_uint64),
    ]


class CrossEntropyArgs(ctypes.Structure):
    """Mirror of gg_cross_entropy_args."""
    _fields_ = [
        ("h", _P), ("rows", ctypes.c_int64), ("width", ctypes.c_int64), ("h_ld", ctypes.c_int64), ("w", _P),
        ("vocab", ctypes.c_int64), ("w_ld", ctypes.c_int64), ("dtype", ctypes.c_int32), ("target", _P), ("loss", _P), ("lse", _P),
    ]


class CrossEntropyGradArgs(ctypes.Structure):
    """Mirror of gg_cross_entropy_grad_args."""
    _fields_ = [
        ("dloss", _P), ("h", _P), ("rows", ctypes.c_int64), ("width", ctypes.c_int64), ("h_ld", ctypes.c_int64), ("w", _P),
        ("vocab", ctypes.c_int64), ("w_ld", ctypes.c_int64), ("dtype", ctypes.c_int32), ("target", _P), ("lse", _P),
        ("dh", _P), ("dh_ld", ctypes.c_int64), ("dw", _P), ("dw_ld", ctypes.c_int64), ("accumulate", ctypes.c_int32),
    ]


class GatedLinearArgs(ctypes.Structure):
    """Mirror of gg_gated_linear_args."""
    _fields_ = [
        ("x", _P), ("rows", ctypes.c_int64), ("width", ctypes.c_int64), ("x_ld", ctypes.c_int64), ("w_gate", _P), ("w_up", _P),
        ("hidden", ctypes.c_int64), ("w_gate_ld", ctypes.c_int64), ("w_up_ld", ctypes.c_int64), ("dtype", ctypes.c_int32),
        ("act", ctypes.c_int32), ("h", _P), ("h_ld", ctypes.c_int64), ("gate", _P), ("up", _P), ("gate_ld", ctypes.c_int64),
        ("up_ld", ctypes.c_int64),
    ]


class GatedLinearGradArgs(ctypes.Structure):
    """Mirror of gg_gated_linear_grad_args."""
    _fields_ = [
        ("dh", _P), ("gate", _P), ("up", _P), ("dh_ld", ctypes.c_int64), ("gate_ld", ctypes.c_int64), ("up_ld", ctypes.c_int64),
        ("x", _P), ("rows", ctypes.c_int64), ("width", ctypes.c_int64), ("x_ld", ctypes.c_int64), ("w_gate", _P), ("w_up", _P),
        ("hidden", ctypes.c_int64), ("w_gate_ld", ctypes.c_int64), ("w_up_ld", ctypes.c_int64), ("dtype", ctypes.c_int32),
        ("act", ctypes.c_int32), ("dx", _P), ("dx_ld", ctypes.c_int64), ("dw_gate", _P), ("dw_up", _P),
        ("dw_gate_ld", ctypes.c_int64), ("dw_up_ld", ctypes.c_int64), ("accumulate", ctypes.c_int32),
    ]


class DropoutArgs(ctypes.Structure):
    """Mirror of gg_dropout_args."""
    _fields_ = [
        ("x", _P), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("x_ld", ctypes.c_int64), ("dtype", ctypes.c_int32),
        ("residual", _P), ("residual_ld", ctypes.c_int64), ("y", _P), ("y_ld", ctypes.c_int64), ("p", ctypes.c_double),
        ("seed", ctypes.c_uint64), ("t", ctypes.c_int64), ("t_dev", _P), ("tensor_id", ctypes.c_uint32),
    ]


class GGError(RuntimeError):
    def __init__(self, status, text):
        super().__init__(f"gg status {status}: {text}")
        self.status = status


_lib = None


def lib():
    """Loads the CUDA library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(f"{_LIB_PATH} is missing: run paper_2506_00486_b200/build.py "
                               "(there is no CPU fallback)")
        L = ctypes.CDLL(_LIB_PATH)
        i32, i64, u32, u64, d = (ctypes.c_int32, ctypes.c_int64, ctypes.c_uint32, ctypes.c_uint64,
                                 ctypes.c_double)
        L.gg_create.argtypes = [ctypes.POINTER(_P), ctypes.c_int]
        L.gg_destroy.argtypes = [_P]
        L.gg_status_str.argtypes = [ctypes.c_int]
        L.gg_status_str.restype = ctypes.c_char_p
        L.gg_version.restype = ctypes.c_int
        L.gg_last_cuda_error.argtypes = [_P]
        L.gg_last_cuda_error.restype = ctypes.c_char_p
        L.gg_launch_count.argtypes = [_P]
        L.gg_launch_count.restype = i64
        L.gg_plan_stats.argtypes = [_P, i32]
        L.gg_plan_stats.restype = i64
        for name, args in (("gg_alpha_from_std", [d, d]), ("gg_init_alpha", [i64, d, d]),
                           ("gg_diff_entropy_bits", [d, d])):
            getattr(L, name).argtypes = args
            getattr(L, name).restype = d
        L.gg_fit.argtypes = [_P, _P, i32, ctypes.c_int, _P, _P, _P, _P, _P, _P, _P]
        L.gg_penalty_grad.argtypes = [_P, _P, i32, ctypes.c_int, _P, _P, d, ctypes.c_int, _P,
                                      ctypes.c_int, ctypes.c_int, _P, _P]
        L.gg_rate_hist.argtypes = [_P, _P, i32, ctypes.c_int, _P, _P, i32, i32, i32, _P, ctypes.c_int,
                                   _P, _P, _P]
        L.gg_sample.argtypes = [_P, _P, i32, ctypes.c_int, _P, _P, u64, u32, _P, _P]
        L.gg_fused.argtypes = [_P, ctypes.POINTER(FusedArgs), _P]
        L.gg_fused_host.argtypes = [_P, ctypes.POINTER(FusedArgs), i64]
        L.gg_fused_channels.argtypes = [_P, ctypes.POINTER(ChannelArgs), _P]
        L.gg_fused_channels.restype = ctypes.c_int
        L.gg_timing_enable.argtypes = [_P, ctypes.c_int]
        L.gg_timing_read.argtypes = [_P, ctypes.POINTER(d), ctypes.POINTER(i64), ctypes.POINTER(d),
                                     ctypes.POINTER(i64)]
        L.gg_debug_bounds_violations.restype = i64
        L.gg_test_hook.argtypes = [_P, i32, i64]
        L.gg_test_hook.restype = ctypes.c_int
        L.gg_fit_noalloc.argtypes = [ctypes.c_int, _P, i64, ctypes.c_int, _P, _P, _P, _P, _P, _P, _P]
        L.gg_fit_noalloc.restype = ctypes.c_int
        L.gg_fit_noalloc_max_len.restype = i64
        L.gg_eg_rate.argtypes = [_P, _P, i32, i32, i32, i32, _P, _P]
        L.gg_eg_rate_grad.argtypes = [_P, _P, i32, ctypes.c_int, _P, i32, d, i32, i32, _P, ctypes.c_int, ctypes.c_int, _P]
        L.gg_code_stats.argtypes = [_P, _P, i32, i32, i32, i32, _P, _P, _P, _P]
        L.gg_gct_step.argtypes = [_P, _P, i32, ctypes.c_int, _P, _P, _P, i32, i32, i32, d, d, d, i64, _P]
        L.gg_layer_norm.argtypes = [_P, ctypes.POINTER(LayerNormArgs), _P]
        L.gg_layer_norm_grad.argtypes = [_P, ctypes.POINTER(LayerNormGradArgs), _P]
        L.gg_grad_norm.argtypes = [_P, _P, i32, ctypes.c_int, d, _P, _P, _P]
        L.gg_adamw_step.argtypes = [_P, ctypes.POINTER(AdamwArgs), _P]
        L.gg_product_status.argtypes = [_P]
        L.gg_cross_entropy.argtypes = [_P, ctypes.POINTER(CrossEntropyArgs), _P]
        L.gg_cross_entropy_grad.argtypes = [_P, ctypes.POINTER(CrossEntropyGradArgs), _P]
        L.gg_gated_linear.argtypes = [_P, ctypes.POINTER(GatedLinearArgs), _P]
        L.gg_gated_linear_grad.argtypes = [_P, ctypes.POINTER(GatedLinearGradArgs), _P]
        L.gg_dropout.argtypes = [_P, ctypes.POINTER(DropoutArgs), _P]
        for name in ("gg_layer_norm", "gg_layer_norm_grad", "gg_grad_norm", "gg_adamw_step", "gg_product_status", "gg_cross_entropy",
                     "gg_cross_entropy_grad",
                     "gg_gated_linear", "gg_gated_linear_grad", "gg_dropout"):
            getattr(L, name).restype = ctypes.c_int
        L.gg_compression_ratio.argtypes = [d, d]
        L.gg_compression_ratio.restype = d
        for name in ("gg_eg_rate", "gg_eg_rate_grad", "gg_code_stats", "gg_gct_step"):
            getattr(L, name).restype = ctypes.c_int
        for name in ("gg_create", "gg_destroy", "gg_fit", "gg_penalty_grad", "gg_rate_hist", "gg_sample",
                     "gg_fused", "gg_fused_host", "gg_timing_enable", "gg_timing_read"):
            getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


def gg_alpha_from_std(std, beta):
    return lib().gg_alpha_from_std(float(std), float(beta))


def gg_init_alpha(d_in, xi, beta):
    return lib().gg_init_alpha(int(d_in), float(xi), float(beta))


def gg_diff_entropy_bits(alpha, beta):
    return lib().gg_diff_entropy_bits(float(alpha), float(beta))


def gg_fit_noalloc(x, out=None):
    """Moments and fit of one contiguous CUDA tensor through the entry point that allocates nothing.

    For callers that cannot allocate device memory at the time of the call, `out` carries the six
    one-element device tensors (beta, alpha, sum_abs, sum_sq: float64; count: int64; flags: int32)
    prepared beforehand; without it they are created here with torch (which does allocate)."""
    if not x.is_cuda or not x.is_contiguous():
        raise ValueError("need a contiguous CUDA tensor")
    dev = x.device
    if out is None:
        out = dict(beta=torch.empty(1, dtype=torch.float64, device=dev), alpha=torch.empty(1, dtype=torch.float64, device=dev),
                   sum_abs=torch.empty(1, dtype=torch.float64, device=dev), sum_sq=torch.empty(1, dtype=torch.float64, device=dev),
                   count=torch.empty(1, dtype=torch.int64, device=dev), flags=torch.empty(1, dtype=torch.int32, device=dev))
    status = lib().gg_fit_noalloc(dev.index or 0, x.data_ptr() if x.numel() else None, x.numel(), _dtype_code(x.dtype),
                                  _ptr(out["beta"]), _ptr(out["alpha"]), _ptr(out["sum_abs"]), _ptr(out["sum_sq"]),
                                  _ptr(out["count"]), _ptr(out["flags"]), _stream_ptr(dev))
    if status != 0:
        raise GGError(status, lib().gg_status_str(status).decode())
    return out


def gg_compression_ratio(bits, fixed_length_bits):
    return lib().gg_compression_ratio(float(bits), float(fixed_length_bits))


def _dtype_code(dt):
    if dt == torch.float32:
        return GG_F32
    if dt == torch.bfloat16:
        return GG_BF16
    raise TypeError(f"unsupported dtype {dt}: the library takes float32 and bfloat16")


class Segments:
    """A host array of gg_seg built once from tensors (kept alive here).

    `Segments(list_of_tensors)`: one segment per tensor (flattened, must be contiguous).
    `Segments.rows(t)`: one segment per row of a contiguous 2-D tensor."""

    def __init__(self, tensors):
        tensors = list(tensors)
        self.tensors = tensors
        self.dtype = tensors[0].dtype if tensors else torch.float32
        arr = np.zeros(len(tensors), dtype=_SEG_DTYPE)
        for i, t in enumerate(tensors):
            if t.dtype != self.dtype:
                raise TypeError("all segments of one call share a dtype")
            if not t.is_contiguous():
                raise ValueError("segments must be contiguous")
            arr["ptr"][i] = t.data_ptr() if t.numel() else 0
            arr["len"][i] = t.numel()
        self.array = arr

    @classmethod
    def rows(cls, t):
        if t.dim() != 2 or not t.is_contiguous():
            raise ValueError("need a contiguous 2-D tensor")
        self = cls.__new__(cls)
        self.tensors = [t]
        self.dtype = t.dtype
        arr = np.zeros(t.shape[0], dtype=_SEG_DTYPE)
        row_bytes = t.shape[1] * t.element_size()
        arr["ptr"] = t.data_ptr() + np.arange(t.shape[0], dtype=np.uint64) * np.uint64(row_bytes)
        arr["len"] = t.shape[1]
        self.array = arr
        return self

    @classmethod
    def slices(cls, flat, offsets, lens):
        """Segments flat[offsets[i] : offsets[i] + lens[i]] of one flat tensor."""
        self = cls.__new__(cls)
        self.tensors = [flat]
        self.dtype = flat.dtype
        arr = np.zeros(len(lens), dtype=_SEG_DTYPE)
        arr["ptr"] = flat.data_ptr() + np.asarray(offsets, dtype=np.uint64) * np.uint64(flat.element_size())
        arr["len"] = np.asarray(lens, dtype=np.int64)
        self.array = arr
        return self

    def __len__(self):
        return len(self.array)

    @property
    def lens(self):
        return self.array["len"]

    @property
    def ptr(self):
        return self.array.ctypes.data

    @property
    def code(self):
        return _dtype_code(self.dtype)

    def device(self):
        return self.tensors[0].device


def _as_segments(x):
    return x if isinstance(x, Segments) else Segments(x)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _ld(t):
    """Row stride of a 2-D tensor, in elements."""
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


# the current stream's handle without a Stream object around it (0.1 instead of 2.2 us of a call's 6)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_ptr(device):
    if _raw_stream is None or device.index is None:
        return torch.cuda.current_stream(device).cuda_stream
    return _raw_stream(device.index)


class Context:
    """One gg_ctx on one CUDA device.  Use from one stream at a time."""

    GUARD_BYTES, GUARD_FILL = 256, 0xA5

    def __init__(self, device=0, guard=False):
        """guard=True puts 256 bytes of a fill pattern before and after every output tensor this object allocates
        (fit results, penalties, histograms, entropies, counters); check_guards() then tells whether a kernel
        wrote outside an output."""
        self._guard = bool(guard)
        self._guarded = []
        self.device = torch.device("cuda", device) if isinstance(device, int) else torch.device(device)
        if self.device.type != "cuda":
            raise RuntimeError("the GG library runs on CUDA devices only")
        if not torch.cuda.is_available():
            raise RuntimeError("no CUDA device: the GG library has no CPU fallback")
        torch.cuda.init()
        with torch.cuda.device(self.device):
            torch.empty(1, device=self.device)          # make sure the primary context exists
        h = _P()
        self._check(lib().gg_create(ctypes.byref(h), self.device.index or 0), None)
        self._h = h

    def close(self):
        if getattr(self, "_h", None):
            lib().gg_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, status, h=True):
        if status != 0:
            text = lib().gg_status_str(status).decode()
            if status == 6 and h and getattr(self, "_h", None):
                text += ": " + lib().gg_last_cuda_error(self._h).decode()
            raise GGError(status, text)

    @property
    def launch_count(self):
        return lib().gg_launch_count(self._h)

    @property
    def plan_stats(self):
        """(plans built, plans pointed at other addresses) since the context was created."""
        return lib().gg_plan_stats(self._h, 0), lib().gg_plan_stats(self._h, 1)

    def gg_test_hook(self, what, value):
        """Knobs of the one-launch fitted pass (HOOK_*), for tests and measurements."""
        self._check(lib().gg_test_hook(self._h, int(what), int(value)))

    def _new(self, n, dtype, zero=False):
        shape = (n,) if isinstance(n, int) else tuple(n)
        if not self._guard:
            return (torch.zeros if zero else torch.empty)(shape, dtype=dtype, device=self.device)
        import weakref
        nbytes = int(np.prod(shape)) * torch.empty(0, dtype=dtype).element_size()
        pad = self.GUARD_BYTES
        raw = torch.full((nbytes + 2 * pad,), self.GUARD_FILL, dtype=torch.uint8, device=self.device)
        body = raw[pad:pad + nbytes]
        if zero:
            body.zero_()
        out = body.view(dtype).view(shape)
        self._guarded.append((weakref.ref(out), raw, nbytes))
        return out

    def check_guards(self):
        """Raises if any byte around a live guarded output has changed (after waiting for the device)."""
        torch.cuda.synchronize(self.device)
        pad, keep = self.GUARD_BYTES, []
        for ref, raw, nbytes in self._guarded:
            if ref() is None:
                continue
            keep.append((ref, raw, nbytes))
            ok = bool((raw[:pad] == self.GUARD_FILL).all()) and bool((raw[pad + nbytes:] == self.GUARD_FILL).all())
            if not ok:
                raise AssertionError(f"a kernel wrote outside an output of {nbytes} bytes")
        self._guarded = keep

    # ------------------------------------------------------------------ gg_fit
    def gg_fit(self, segs):
        """Moments and fit per segment.  Returns a dict of device tensors."""
        segs = _as_segments(segs)
        n = len(segs)
        out = dict(beta=self._new(n, torch.float64), alpha=self._new(n, torch.float64),
                   sum_abs=self._new(n, torch.float64), sum_sq=self._new(n, torch.float64),
                   count=self._new(n, torch.int64), flags=self._new(n, torch.int32))
        self._check(lib().gg_fit(self._h, segs.ptr, n, segs.code, _ptr(out["beta"]), _ptr(out["alpha"]),
                                 _ptr(out["sum_abs"]), _ptr(out["sum_sq"]), _ptr(out["count"]),
                                 _ptr(out["flags"]), _stream_ptr(self.device)))
        return out

    # -------------------------------------------------------- gg_penalty_grad
    def gg_penalty_grad(self, segs, beta, alpha, lam, grad=None, reduction=GG_SUM, accumulate=False,
                        want_penalty=True):
        """Penalty per segment (device float64) and the gradient written into `grad` segments."""
        segs = _as_segments(segs)
        n = len(segs)
        gsegs = None if grad is None else _as_segments(grad)
        pen = self._new(n, torch.float64) if want_penalty else None
        self._check(lib().gg_penalty_grad(
            self._h, segs.ptr, n, segs.code, _ptr(beta), _ptr(alpha), float(lam), int(reduction),
            None if gsegs is None else gsegs.ptr, GG_F32 if gsegs is None else gsegs.code,
            int(bool(accumulate)), _ptr(pen), _stream_ptr(self.device)))
        return pen

    # ------------------------------------------------------------ gg_rate_hist
    def gg_rate_hist(self, segs, step, hist_id=None, n_hist=None, qmin=-32768, qmax=32767, hist=None,
                     accumulate=False):
        """Histogram(s) of the quantised symbols, entropy in bits/symbol, clamp counters."""
        segs = _as_segments(segs)
        n = len(segs)
        n_hist = n if n_hist is None else int(n_hist)
        nb = qmax - qmin + 1
        if hist is None:
            hist = self._new((n_hist, nb), torch.int64)
            if accumulate:
                hist.zero_()
        ent = self._new(n_hist, torch.float64)
        clamped = self._new((n_hist, 2), torch.int64, zero=True)
        hid = None if hist_id is None else np.ascontiguousarray(hist_id, dtype=np.int32)
        self._check(lib().gg_rate_hist(
            self._h, segs.ptr, n, segs.code, _ptr(step), None if hid is None else hid.ctypes.data,
            n_hist, int(qmin), int(qmax), _ptr(hist), int(bool(accumulate)), _ptr(ent), _ptr(clamped),
            _stream_ptr(self.device)))
        return dict(hist=hist, entropy_bits=ent, clamped=clamped)

    # --------------------------------------------------------------- gg_sample
    def gg_sample(self, out, beta, alpha, seed, tensor_id0=0, want_attempts=True):
        """Fills the `out` segments with GG variates; beta, alpha are host sequences."""
        segs = _as_segments(out)
        n = len(segs)
        b = np.ascontiguousarray(beta, dtype=np.float64)
        a = np.ascontiguousarray(alpha, dtype=np.float64)
        if b.size != n or a.size != n:
            raise ValueError("beta and alpha need one entry per segment")
        att = self._new(n, torch.int32) if want_attempts else None
        self._check(lib().gg_sample(self._h, segs.ptr, n, segs.code, b.ctypes.data, a.ctypes.data,
                                    int(seed) & (2 ** 64 - 1), int(tensor_id0) & 0xFFFFFFFF, _ptr(att),
                                    _stream_ptr(self.device)))
        return att

    # ---------------------------------------------------------------- gg_fused
    def make_fused(self, segs, grad=None, lam=1e-4, reduction=GG_SUM, accumulate_grad=False,
                   param_mode=GG_PARAMS_FITTED, beta_in=None, alpha_in=None, want_penalty=True,
                   step=None, step_scale=None, hist_id=None, n_hist=None, qmin=-32768, qmax=32767,
                   want_hist=True, accumulate_hist=False, hist=None, eg_k=0):
        """Allocates the outputs of the fused pass once and returns a callable that enqueues it.

        step: device float32 tensor [n_seg] (GG_STEP_GIVEN); or step_scale: float, step = alpha * scale.
        param_mode=GG_RATE_EG: the gradient and penalty of the Exponential-Golomb rate of order eg_k (Eq. 6-7)
        instead of the GG penalty; out["eg_bits"] holds the mean code length per histogram."""
        segs = _as_segments(segs)
        n = len(segs)
        gsegs = None if grad is None else _as_segments(grad)
        out = dict(beta=self._new(n, torch.float64), alpha=self._new(n, torch.float64),
                   sum_abs=self._new(n, torch.float64), sum_sq=self._new(n, torch.float64),
                   count=self._new(n, torch.int64), flags=self._new(n, torch.int32))
        out["penalty"] = self._new(n, torch.float64) if want_penalty else None
        a = FusedArgs()
        keep = [segs, gsegs, beta_in, alpha_in, step]
        a.segs, a.n_seg, a.in_dtype = segs.ptr, n, segs.code
        for k in ("beta", "alpha", "sum_abs", "sum_sq", "count", "flags", "penalty"):
            setattr(a, k, _ptr(out[k]))
        a.param_mode = int(param_mode)
        a.beta_in, a.alpha_in = _ptr(beta_in), _ptr(alpha_in)
        a.lam, a.reduction = float(lam), int(reduction)
        a.grad = None if gsegs is None else gsegs.ptr
        a.grad_dtype = GG_F32 if gsegs is None else gsegs.code
        a.accumulate_grad = int(bool(accumulate_grad))
        if want_hist:
            n_hist = n if n_hist is None else int(n_hist)
            nb = qmax - qmin + 1
            if hist is None:
                hist = self._new((n_hist, nb), torch.int64, zero=True)
            out["hist"] = hist
            out["entropy_bits"] = self._new(n_hist, torch.float64)
            out["clamped"] = self._new((n_hist, 2), torch.int64, zero=True)
            if step is not None:
                a.step_mode, a.step = GG_STEP_GIVEN, _ptr(step)
                out["step"] = step
            else:
                out["step"] = self._new(n, torch.float32)
                a.step_mode, a.step_scale, a.step_out = GG_STEP_FROM_ALPHA, float(step_scale), _ptr(out["step"])
            hid = None if hist_id is None else np.ascontiguousarray(hist_id, dtype=np.int32)
            keep.append(hid)
            a.hist_id = None if hid is None else hid.ctypes.data
            a.n_hist, a.qmin, a.qmax = n_hist, int(qmin), int(qmax)
            a.hist, a.accumulate_hist = _ptr(hist), int(bool(accumulate_hist))
            a.entropy_bits, a.clamped_lo_hi = _ptr(out["entropy_bits"]), _ptr(out["clamped"])
            if int(param_mode) == GG_RATE_EG:
                out["eg_bits"] = self._new(n_hist, torch.float64)
                a.eg_k, a.eg_bits = int(eg_k), _ptr(out["eg_bits"])

        def run():
            self._check(lib().gg_fused(self._h, ctypes.byref(a), _stream_ptr(self.device)))
            return out

        run.outputs = out
        run.args = a
        run._keep = keep
        return run

    def gg_fused(self, segs, **kw):
        """One-shot form of make_fused(...)()."""
        return self.make_fused(segs, **kw)()

    # ------------------------------------------------------- gg_fused_channels
    def make_fused_channels(self, x, grad=None, lam=1e-4, reduction=GG_SUM, accumulate_grad=False,
                            want_penalty=True, step=None, qmin=-32768, qmax=32767, accumulate_hist=False,
                            hist=None):
        """The fused pass over the COLUMNS of the 2-D tensor x (rows may be strided: x.stride(1) == 1).

        Allocates the per-column outputs once and returns a callable that enqueues the pass.
        step: float, one quantiser step for the matrix; None skips the histogram."""
        if x.dim() != 2 or (x.shape[1] > 1 and x.stride(1) != 1):
            raise ValueError("x must be 2-D with contiguous rows")
        rows, cols = x.shape
        out = dict(beta=self._new(cols, torch.float64), alpha=self._new(cols, torch.float64),
                   sum_abs=self._new(cols, torch.float64), sum_sq=self._new(cols, torch.float64),
                   count=self._new(cols, torch.int64), flags=self._new(cols, torch.int32))
        out["penalty"] = self._new(cols, torch.float64) if want_penalty else None
        a = ChannelArgs()
        a.x, a.rows, a.cols, a.ld, a.in_dtype = _ptr(x), rows, cols, (x.stride(0) if rows > 1 else cols), _dtype_code(x.dtype)
        for k in ("beta", "alpha", "sum_abs", "sum_sq", "count", "flags", "penalty"):
            setattr(a, k, _ptr(out[k]))
        a.lam, a.reduction = float(lam), int(reduction)
        if grad is not None:
            if grad.shape != x.shape or (cols > 1 and grad.stride(1) != 1):
                raise ValueError("grad must have the shape of x and contiguous rows")
            a.grad, a.grad_ld, a.grad_dtype = _ptr(grad), (grad.stride(0) if rows > 1 else cols), _dtype_code(grad.dtype)
        a.accumulate_grad = int(bool(accumulate_grad))
        if step is not None:
            nb = qmax - qmin + 1
            if hist is None:
                hist = self._new(nb, torch.int64, zero=True)
            out["hist"] = hist
            out["entropy_bits"] = self._new(1, torch.float64)
            out["clamped"] = self._new(2, torch.int64, zero=True)
            a.step, a.qmin, a.qmax = float(step), int(qmin), int(qmax)
            a.hist, a.accumulate_hist = _ptr(hist), int(bool(accumulate_hist))
            a.entropy_bits, a.clamped_lo_hi = _ptr(out["entropy_bits"]), _ptr(out["clamped"])

        def run():
            self._check(lib().gg_fused_channels(self._h, ctypes.byref(a), _stream_ptr(self.device)))
            return out

        run.outputs = out
        run.args = a
        run._keep = [x, grad, hist]
        return run

    def gg_fused_channels(self, x, **kw):
        """One-shot form of make_fused_channels(...)()."""
        return self.make_fused_channels(x, **kw)()

    # ----------------------------------------------------------- gg_fused_host
    def make_fused_host(self, segs, grad=None, lam=1e-4, reduction=GG_SUM, step=None, step_scale=None,
                        hist_id=None, n_hist=None, qmin=-32768, qmax=32767, want_hist=True,
                        chunk_bytes=0, pin=True):
        """The fused pass on HOST tensors (CPU torch tensors; pinned ones copy asynchronously).

        Allocates the host outputs once (pinned if `pin`) and returns a callable; each call copies
        the inputs to the device in chunks, runs the pass and returns with all results on the host."""
        segs = _as_segments(segs)
        n = len(segs)
        gsegs = None if grad is None else _as_segments(grad)

        def host(n_, dtype):
            return torch.empty(n_, dtype=dtype, pin_memory=pin)

        out = dict(beta=host(n, torch.float64), alpha=host(n, torch.float64), sum_abs=host(n, torch.float64),
                   sum_sq=host(n, torch.float64), count=host(n, torch.int64), flags=host(n, torch.int32),
                   penalty=host(n, torch.float64))
        a = FusedArgs()
        keep = [segs, gsegs, step]
        a.segs, a.n_seg, a.in_dtype = segs.ptr, n, segs.code
        for k in ("beta", "alpha", "sum_abs", "sum_sq", "count", "flags", "penalty"):
            setattr(a, k, _ptr(out[k]))
        a.param_mode, a.lam, a.reduction = GG_PARAMS_FITTED, float(lam), int(reduction)
        a.grad = None if gsegs is None else gsegs.ptr
        a.grad_dtype = GG_F32 if gsegs is None else gsegs.code
        if want_hist:
            n_hist = n if n_hist is None else int(n_hist)
            nb = qmax - qmin + 1
            out["hist"] = torch.empty((n_hist, nb), dtype=torch.int64, pin_memory=pin)
            out["entropy_bits"] = host(n_hist, torch.float64)
            out["clamped"] = torch.empty((n_hist, 2), dtype=torch.int64, pin_memory=pin)
            if step is not None:
                a.step_mode, a.step = GG_STEP_GIVEN, _ptr(step)
                out["step"] = step
            else:
                out["step"] = host(n, torch.float32)
                a.step_mode, a.step_scale, a.step_out = GG_STEP_FROM_ALPHA, float(step_scale), _ptr(out["step"])
            hid = None if hist_id is None else np.ascontiguousarray(hist_id, dtype=np.int32)
            keep.append(hid)
            a.hist_id = None if hid is None else hid.ctypes.data
            a.n_hist, a.qmin, a.qmax = n_hist, int(qmin), int(qmax)
            a.hist, a.entropy_bits, a.clamped_lo_hi = _ptr(out["hist"]), _ptr(out["entropy_bits"]), _ptr(out["clamped"])

        def run():
            self._check(lib().gg_fused_host(self._h, ctypes.byref(a), int(chunk_bytes)))
            return out

        run.outputs = out
        run._keep = keep
        return run

    def gg_fused_host(self, segs, **kw):
        return self.make_fused_host(segs, **kw)()

    # ------------------------------------------------------------ code lengths
    def gg_eg_rate(self, hist, k=0, qmin=-32768, qmax=32767):
        """Average Exponential-Golomb code length per histogram (device float64)."""
        n_hist = hist.shape[0]
        out = self._new(n_hist, torch.float64)
        self._check(lib().gg_eg_rate(self._h, _ptr(hist), n_hist, int(qmin), int(qmax), int(k), _ptr(out),
                                     _stream_ptr(self.device)))
        return out

    def gg_eg_rate_grad(self, segs, step, lam, grad, k=0, qmin=-32768, qmax=32767, accumulate=False):
        """Writes the gradient of lam * (Exponential-Golomb rate) into the `grad` segments."""
        segs, gsegs = _as_segments(segs), _as_segments(grad)
        self._check(lib().gg_eg_rate_grad(self._h, segs.ptr, len(segs), segs.code, _ptr(step), int(k), float(lam),
                                          int(qmin), int(qmax), gsegs.ptr, gsegs.code, int(bool(accumulate)),
                                          _stream_ptr(self.device)))

    def gg_code_stats(self, hist, k=0, qmin=-32768, qmax=32767):
        """EG, Huffman and fixed-length bits per histogram as numpy arrays (synchronises the stream)."""
        n_hist = hist.shape[0]
        eg, hm, fl = (np.empty(n_hist, dtype=np.float64) for _ in range(3))
        self._check(lib().gg_code_stats(self._h, _ptr(hist), n_hist, int(qmin), int(qmax), int(k), eg.ctypes.data,
                                        hm.ctypes.data, fl.ctypes.data, _stream_ptr(self.device)))
        return dict(eg_bits=eg, hm_bits=hm, fl_bits=fl)

    def gg_gct_step(self, g, ghat, w, step, eta, lam, eps, t, k=0, qmin=-32768, qmax=32767):
        """One GCT step in place: `ghat` (float32 segments) and `w` (float32 segments) are updated."""
        gs, hs, ws = _as_segments(g), _as_segments(ghat), _as_segments(w)
        if hs.dtype != torch.float32 or ws.dtype != torch.float32:
            raise TypeError("ghat and w are float32")
        self._check(lib().gg_gct_step(self._h, gs.ptr, len(gs), gs.code, hs.ptr, ws.ptr, _ptr(step), int(k), int(qmin),
                                      int(qmax), float(eta), float(lam), float(eps), int(t), _stream_ptr(self.device)))

    # -------------------------------------------------------------- layer norm
    def make_layer_norm(self, x, weight=None, bias=None, eps=1e-5, out=None, want_stats=True):
        """Layer norm over the rows of the 2-D tensor x (rows may be strided: x.stride(1) == 1).

        Allocates the outputs once (y unless `out` is given; it may be x) and returns a callable that enqueues the
        pass and returns dict(y, mean, rstd); mean and rstd (float32 per row) are what the gradient needs."""
        rows, cols = self._rows(x, "x")
        y = self._new(x.shape, x.dtype) if out is None else out
        self._rows(y, "out", x)
        res = dict(y=y, mean=self._new(rows, torch.float32) if want_stats else None,
                   rstd=self._new(rows, torch.float32) if want_stats else None)
        a = LayerNormArgs()
        a.x, a.rows, a.cols, a.x_ld, a.dtype = _ptr(x), rows, cols, _ld(x), _dtype_code(x.dtype)
        a.weight, a.bias, a.w_dtype = self._affine(cols, weight, bias)
        a.eps, a.y, a.y_ld, a.mean, a.rstd = float(eps), _ptr(y), _ld(y), _ptr(res["mean"]), _ptr(res["rstd"])
        return self._callable("gg_layer_norm", a, res, [x, weight, bias, y])

    def gg_layer_norm(self, x, weight=None, bias=None, **kw):
        """One-shot form of make_layer_norm(...)()."""
        return self.make_layer_norm(x, weight, bias, **kw)()

    def make_layer_norm_grad(self, dy, x, mean, rstd, weight=None, dx=None, dweight=None, dbias=None, want_dx=True,
                             want_dweight=None, accumulate=False):
        """Gradient of layer norm for dy, the x of the forward pass and the mean and rstd that it returned.

        Allocates dx (like x, unless given; it may be dy or x) and dweight, dbias (float32 [cols], unless given) once
        and returns a callable that enqueues the pass and returns dict(dx, dweight, dbias).  want_dweight: None = if
        there is a weight or a tensor for the sums; accumulate adds to dweight and dbias instead of overwriting."""
        rows, cols = self._rows(x, "x")
        self._rows(dy, "dy", x)
        for name, t in (("mean", mean), ("rstd", rstd)):
            self._vector(name, t, rows)
        if dx is None and want_dx:
            dx = self._new(x.shape, x.dtype)
        if dx is not None:
            self._rows(dx, "dx", x)
        if want_dweight is None:
            want_dweight = weight is not None
        if accumulate and want_dweight and (dweight is None or dbias is None):
            raise ValueError("accumulate adds to dweight and dbias: give both")
        if want_dweight:
            dweight = self._new(cols, torch.float32) if dweight is None else dweight
            dbias = self._new(cols, torch.float32) if dbias is None else dbias
        for name, t in (("dweight", dweight), ("dbias", dbias)):
            if t is not None:
                self._vector(name, t, cols)
        a = LayerNormGradArgs()
        a.dy, a.x, a.rows, a.cols, a.dy_ld, a.x_ld, a.dtype = _ptr(dy), _ptr(x), rows, cols, _ld(dy), _ld(x), _dtype_code(x.dtype)
        a.mean, a.rstd = _ptr(mean), _ptr(rstd)
        a.weight, _, a.w_dtype = self._affine(cols, weight, None)
        a.dx, a.dx_ld = _ptr(dx), cols if dx is None else _ld(dx)
        a.dweight, a.dbias, a.accumulate = _ptr(dweight), _ptr(dbias), int(bool(accumulate))
        return self._callable("gg_layer_norm_grad", a, dict(dx=dx, dweight=dweight, dbias=dbias), [dy, x, mean, rstd, weight])

    def gg_layer_norm_grad(self, dy, x, mean, rstd, weight=None, **kw):
        """One-shot form of make_layer_norm_grad(...)()."""
        return self.make_layer_norm_grad(dy, x, mean, rstd, weight, **kw)()

    def _rows(self, t, name, like=None):
        if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1) or (t.shape[0] > 1 and t.stride(0) < t.shape[1]):
            raise ValueError(f"{name} must be 2-D with contiguous rows")
        if t.device.type != "cuda":
            raise ValueError(f"{name} must be a CUDA tensor")
        if like is not None and (t.shape != like.shape or t.dtype != like.dtype):
            raise ValueError(f"{name} must have the shape and dtype of x")
        return t.shape

    def _vector(self, name, t, n, dtype=torch.float32):
        if t.device.type != "cuda" or t.dtype != dtype or t.numel() != n or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous CUDA tensor of {n} {dtype} values")

    def _affine(self, cols, weight, bias):
        given = [t for t in (weight, bias) if t is not None]
        for t in given:
            self._vector("weight and bias", t, cols, given[0].dtype)
        return _ptr(weight), _ptr(bias), _dtype_code(given[0].dtype) if given else GG_F32

    def _callable(self, entry, a, res, keep):
        call, arg = getattr(lib(), entry), ctypes.byref(a)

        def run():
            self._check(call(self._h, arg, _stream_ptr(self.device)))
            return res

        run.outputs = res
        run.args = a
        run._keep = keep
        return run

    # ------------------------------------------------- gradient norm and AdamW
    def gg_grad_norm(self, g, max_norm=float("inf"), out=None):
        """dict(norm, scale), on the device: the norm of all segments together (float64) and min(1, max_norm / norm)
        (float32), both nan if an entry is not finite."""
        segs = _as_segments(g)
        if out is None:
            out = dict(norm=self._new(1, torch.float64), scale=self._new(1, torch.float32))
        self._check(lib().gg_grad_norm(self._h, segs.ptr, len(segs), segs.code, float(max_norm), _ptr(out["norm"]),
                                       _ptr(out["scale"]), _stream_ptr(self.device)))
        return out

    def adamw_state(self, w, bits=32):
        """The state before the first step for the segments w: dict(m, v) of lists of tensors, with 8 bits also
        scales = (m_scale, v_scale).  The keys are arguments of make_adamw_step."""
        segs = _as_segments(w)
        if bits not in (32, 8):
            raise ValueError("states have 32 or 8 bits")
        dtype = torch.float32 if bits == 32 else torch.float8_e4m3fn
        lens = [int(n) for n in segs.lens]
        out = {k: [torch.zeros(n, dtype=dtype, device=self.device) for n in lens] for k in ("m", "v")}
        if bits == 8:
            blocks = sum(-(-n // ADAMW_BLOCK) for n in lens)
            out["scales"] = tuple(torch.zeros(blocks, dtype=torch.float32, device=self.device) for _ in range(2))
        return out

    def make_adamw_step(self, w, g, m, v, scales=None, w_copy=None, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01,
                        max_norm=None, grad_scale=None, seed=0):
        """Returns step(t, lr), which enqueues one AdamW step over all segments, in place.

        w (float32 or bfloat16), g (float32 or bfloat16) and the states m, v (float32; float8_e4m3fn with `scales`)
        are lists of tensors or Segments of the same lengths; w_copy: bfloat16 segments that get the new weights.
        weight_decay: a number, or a float32 device tensor with one entry per segment.  max_norm clips the gradient
        by its global norm first; grad_scale (float32 [1], on the device) scales it instead.  seed: of the rounding of
        bfloat16 weights and 8-bit states.  step returns dict(norm, scale) (of the clipping, else empty)."""
        ws, gs, ms, vs = (_as_segments(t) for t in (w, g, m, v))
        cs = None if w_copy is None else _as_segments(w_copy)
        states = (torch.float32,) if scales is None else (torch.float8_e4m3fn, torch.uint8)
        if ms.dtype not in states or vs.dtype not in states:
            raise TypeError("m and v are float32, or float8_e4m3fn with scales")
        if cs is not None and cs.dtype != torch.bfloat16:
            raise TypeError("w_copy is bfloat16")
        if max_norm is not None and grad_scale is not None:
            raise ValueError("max_norm or grad_scale, not both")
        for name, t in (("g", gs), ("m", ms), ("v", vs), ("w_copy", cs)):
            if t is not None and not np.array_equal(t.lens, ws.lens):
                raise ValueError(f"{name} must have the lengths of w")
        a = AdamwArgs()
        a.n_seg, a.w, a.w_dtype, a.g, a.g_dtype = len(ws), ws.ptr, ws.code, gs.ptr, gs.code
        a.w_copy = None if cs is None else cs.ptr
        a.state_bits, a.m, a.v = 32 if scales is None else 8, ms.ptr, vs.ptr
        if scales is not None:
            blocks = int((-(-ws.lens // ADAMW_BLOCK)).sum())
            for name, t in zip(("m_scale", "v_scale"), scales, strict=True):
                self._vector(name, t, blocks)
            a.m_scale, a.v_scale = _ptr(scales[0]), _ptr(scales[1])
        a.beta1, a.beta2, a.eps, a.seed = float(beta1), float(beta2), float(eps), int(seed) & (2 ** 64 - 1)
        if isinstance(weight_decay, torch.Tensor):
            self._vector("weight_decay", weight_decay, len(ws))
            a.decay = _ptr(weight_decay)
        else:
            a.weight_decay = float(weight_decay)
        out = {}
        if max_norm is not None:
            out = dict(norm=self._new(1, torch.float64), scale=self._new(1, torch.float32))
            grad_scale = out["scale"]
        if grad_scale is not None:
            self._vector("grad_scale", grad_scale, 1)
            a.grad_scale = _ptr(grad_scale)
        call, arg = lib().gg_adamw_step, ctypes.byref(a)

        def step(t, lr):
            if max_norm is not None:
                self.gg_grad_norm(gs, max_norm, out)
            a.t, a.lr = int(t), float(lr)
            self._check(call(self._h, arg, _stream_ptr(self.device)))
            return out

        step.outputs = out
        step.args = a
        step._keep = [ws, gs, ms, vs, cs, scales, weight_decay, grad_scale]
        return step

    def gg_adamw_step(self, w, g, m, v, t, lr, **kw):
        """One-shot form of make_adamw_step(...)(t, lr)."""
        return self.make_adamw_step(w, g, m, v, **kw)(t, lr)

    # --------------------------------------------------------- vocabulary loss
    def gg_product_status(self):
        """Raises GGError if a wait ran out in a kernel of the vocabulary loss, the gated block or their gradients and nothing has
        reported it: what they wrote is not to be used.  It tells of the kernels that have ended, so synchronise first."""
        self._check(lib().gg_product_status(self._h))

    def make_cross_entropy(self, h, w, target):
        """Softmax cross entropy of the logits h @ w.t(), which are never stored.

        h: bfloat16 [rows, width], w: bfloat16 [vocab, width] (rows may be strided), target: int64 [rows], negative where a
        position has none.  Allocates the outputs once and returns a callable that enqueues the pass and returns
        dict(loss, lse) (float32 [rows]); lse is what the gradient needs."""
        a = CrossEntropyArgs()
        self._features(a, h, w, target)
        res = dict(loss=self._new(h.shape[0], torch.float32), lse=self._new(h.shape[0], torch.float32))
        a.loss, a.lse = _ptr(res["loss"]), _ptr(res["lse"])
        return self._callable("gg_cross_entropy", a, res, [h, w, target])

    def gg_cross_entropy(self, h, w, target):
        """One-shot form of make_cross_entropy(...)()."""
        return self.make_cross_entropy(h, w, target)()

    def make_cross_entropy_grad(self, dloss, h, w, target, lse, dh=None, dw=None, want_dh=True, want_dw=True, accumulate=False):
        """Gradient of cross_entropy for dloss (float32 [rows]) and the lse that it returned.

        Allocates dh and dw (bfloat16, like h and w, unless given) once and returns a callable that enqueues the pass and returns
        dict(dh, dw).  accumulate adds to dw instead of overwriting it."""
        a = CrossEntropyGradArgs()
        rows, width = self._features(a, h, w, target)
        self._vector("dloss", dloss, rows)
        self._vector("lse", lse, rows)
        self._here(dloss=dloss, lse=lse)
        if accumulate and want_dw and dw is None:
            raise ValueError("accumulate adds to dw: give it")
        dh, dw = self._result("dh", dh, h, want_dh), self._result("dw", dw, w, want_dw)
        a.dloss, a.lse = _ptr(dloss), _ptr(lse)
        a.dh, a.dh_ld = _ptr(dh), width if dh is None else _ld(dh)
        a.dw, a.dw_ld = _ptr(dw), width if dw is None else _ld(dw)
        a.accumulate = int(bool(accumulate))
        return self._callable("gg_cross_entropy_grad", a, dict(dh=dh, dw=dw), [dloss, h, w, target, lse])

    def gg_cross_entropy_grad(self, dloss, h, w, target, lse, **kw):
        """One-shot form of make_cross_entropy_grad(...)()."""
        return self.make_cross_entropy_grad(dloss, h, w, target, lse, **kw)()

    def _features(self, a, h, w, target):
        rows, width = self._operand(h, "h")
        vocab, _ = self._operand(w, "w", cols=width)
        self._vector("target", target, rows, torch.int64)
        self._here(target=target)
        a.h, a.rows, a.width, a.h_ld, a.dtype = _ptr(h), rows, width, _ld(h), GG_BF16
        a.w, a.vocab, a.w_ld, a.target = _ptr(w), vocab, _ld(w), _ptr(target)
        return rows, width

    def _here(self, **tensors):
        for name, t in tensors.items():
            if t is not None and t.is_cuda and t.device.index != (self.device.index or 0):
                raise ValueError(f"{name} is on {t.device}, the context on cuda:{self.device.index or 0}")

    def _operand(self, t, name, rows=None, cols=None):
        """A matrix of a product: bfloat16, what the tensor cores take."""
        shape = self._rows(t, name)
        self._here(**{name: t})
        if t.dtype != torch.bfloat16:
            raise TypeError(f"{name} must be bfloat16 (AdamW keeps a bfloat16 copy of float32 weights: w_copy)")
        if (rows is not None and shape[0] != rows) or (cols is not None and shape[1] != cols):
            raise ValueError(f"{name} must be [{'rows' if rows is None else rows}, {'cols' if cols is None else cols}], not {list(shape)}")
        return shape

    def _result(self, name, t, like, want=True):
        if not want:
            return None
        if t is None:
            return self._new(like.shape, like.dtype)
        self._rows(t, name, like)
        self._here(**{name: t})
        return t

    # ------------------------------------------------------------- gated block
    def make_gated_linear(self, x, w_gate, w_up, act="silu", out=None, keep=False):
        """h = act(x @ w_gate.t()) * (x @ w_up.t()), both products and the activation in one kernel.

        x: bfloat16 [rows, width], w_gate, w_up: bfloat16 [hidden, width] (rows may be strided; halves of one matrix will do),
        act: "silu", "gelu", "gelu_tanh" or "relu".  Allocates h (unless `out` is given) once and returns a callable that
        enqueues the pass and returns dict(h, gate, up); gate and up, the products that the gradient needs, only with `keep`."""
        rows, width = self._operand(x, "x")
        hidden, _ = self._operand(w_gate, "w_gate", cols=width)
        self._operand(w_up, "w_up", hidden, width)
        if out is None:
            out = self._new((rows, hidden), torch.bfloat16)
        self._operand(out, "out", rows, hidden)
        res = dict(h=out, gate=self._new((rows, hidden), torch.bfloat16) if keep else None,
                   up=self._new((rows, hidden), torch.bfloat16) if keep else None)
        a = GatedLinearArgs()
        a.x, a.rows, a.width, a.x_ld, a.dtype, a.act = _ptr(x), rows, width, _ld(x), GG_BF16, self._act(act)
        a.w_gate, a.w_up, a.hidden, a.w_gate_ld, a.w_up_ld = _ptr(w_gate), _ptr(w_up), hidden, _ld(w_gate), _ld(w_up)
        a.h, a.h_ld, a.gate, a.up, a.gate_ld, a.up_ld = _ptr(out), _ld(out), _ptr(res["gate"]), _ptr(res["up"]), hidden, hidden
        return self._callable("gg_gated_linear", a, res, [x, w_gate, w_up])

    def gg_gated_linear(self, x, w_gate, w_up, **kw):
        """One-shot form of make_gated_linear(...)()."""
        return self.make_gated_linear(x, w_gate, w_up, **kw)()

    def make_gated_linear_grad(self, dh, x, w_gate, w_up, gate, up, act="silu", dx=None, dw_gate=None, dw_up=None, want_dx=True,
                               want_dweight=True, accumulate=False):
        """Gradient of gated_linear for dh, its operands and the gate and up that it kept.

        Allocates dx, dw_gate and dw_up (bfloat16, like x and the weights, unless given) once and returns a callable that enqueues
        the pass and returns dict(dx, dw_gate, dw_up).  accumulate adds to dw_gate and dw_up instead of overwriting them."""
        rows, width = self._operand(x, "x")
        hidden, _ = self._operand(w_gate, "w_gate", cols=width)
        self._operand(w_up, "w_up", hidden, width)
        for name, t in (("dh", dh), ("gate", gate), ("up", up)):
            self._operand(t, name, rows, hidden)
        if accumulate and want_dweight and (dw_gate is None or dw_up is None):
            raise ValueError("accumulate adds to dw_gate and dw_up: give both")
        res = dict(dx=self._result("dx", dx, x, want_dx), dw_gate=self._result("dw_gate", dw_gate, w_gate, want_dweight),
                   dw_up=self._result("dw_up", dw_up, w_up, want_dweight))
        a = GatedLinearGradArgs()
        a.dh, a.gate, a.up, a.dh_ld, a.gate_ld, a.up_ld = _ptr(dh), _ptr(gate), _ptr(up), _ld(dh), _ld(gate), _ld(up)
        a.x, a.rows, a.width, a.x_ld, a.dtype, a.act = _ptr(x), rows, width, _ld(x), GG_BF16, self._act(act)
        a.w_gate, a.w_up, a.hidden, a.w_gate_ld, a.w_up_ld = _ptr(w_gate), _ptr(w_up), hidden, _ld(w_gate), _ld(w_up)
        for name, t in res.items():
            setattr(a, name, _ptr(t))
            setattr(a, name + "_ld", width if t is None else _ld(t))
        a.accumulate = int(bool(accumulate))
        return self._callable("gg_gated_linear_grad", a, res, [dh, x, w_gate, w_up, gate, up])

    def gg_gated_linear_grad(self, dh, x, w_gate, w_up, gate, up, **kw):
        """One-shot form of make_gated_linear_grad(...)()."""
        return self.make_gated_linear_grad(dh, x, w_gate, w_up, gate, up, **kw)()

    @staticmethod
    def _act(act):
        if act not in ACTIVATIONS:
            raise ValueError(f"act must be one of {', '.join(ACTIVATIONS)}, not {act!r}")
        return ACTIVATIONS[act]

    # ----------------------------------------------------------------- dropout
    def make_dropout(self, x, p, residual=None, out=None, seed=DROPOUT_SEED, tensor_id=0, t_dev=None):
        """Dropout of the 2-D tensor x (rows may be strided) with a mask that is drawn, not stored.

        Returns drop(t), which enqueues y = [residual +] x * mask / (1 - p) and returns dict(y); y is allocated once unless
        `out` is given (it may be x or residual).  The mask depends on seed, tensor_id, t and the shape alone: the gradient is drop(t) of
        another make_dropout on dy.  seed: another one than AdamW's and the sampler's, which draw from the same generator.  t_dev: an int64
        device tensor of one value that is added to t, for captured graphs."""
        rows, cols = self._rows(x, "x")
        if residual is not None:
            self._rows(residual, "residual", x)
        y = self._result("out", out, x)
        if t_dev is not None:
            self._vector("t_dev", t_dev, 1, torch.int64)
        self._here(x=x, residual=residual, t_dev=t_dev)
        a = DropoutArgs()
        a.x, a.rows, a.cols, a.x_ld, a.dtype = _ptr(x), rows, cols, _ld(x), _dtype_code(x.dtype)
        a.residual, a.residual_ld = _ptr(residual), cols if residual is None else _ld(residual)
        a.y, a.y_ld, a.p, a.seed, a.t_dev = _ptr(y), _ld(y), float(p), int(seed) & (2 ** 64 - 1), _ptr(t_dev)
        a.tensor_id = int(tensor_id) & 0xFFFFFFFF
        enqueue = self._callable("gg_dropout", a, dict(y=y), [x, residual, t_dev])

        def drop(t=0):
            a.t = int(t)
            return enqueue()

        drop.outputs, drop.args = enqueue.outputs, a
        return drop

    def gg_dropout(self, x, p, t=0, **kw):
        """One-shot form of make_dropout(...)(t)."""
        return self.make_dropout(x, p, **kw)(t)

    # ------------------------------------------------------------------ timing
    def timing_enable(self, on=True):
        self._check(lib().gg_timing_enable(self._h, int(bool(on))))

    def timing_read(self):
        """(ms of first sweeps, their count, ms of second sweeps, their count) since the last read."""
        m0, m1 = ctypes.c_double(), ctypes.c_double()
        n0, n1 = ctypes.c_int64(), ctypes.c_int64()
        self._check(lib().gg_timing_read(self._h, ctypes.byref(m0), ctypes.byref(n0), ctypes.byref(m1),
                                         ctypes.byref(n1)))
        return m0.value, n0.value, m1.value, n1.value
