"""ctypes binding of include/gsq.h, gsq_products.h, gsq_routing.h and gsq_adapters.h: argument marshalling only.

Every computation runs in ``libgsq.so``; this module passes device pointers
(``tensor.data_ptr()``) and the current HIP stream to it and turns status codes
into exceptions.  Loading fails loudly when the library has not been built.
"""
import ctypes
import os
from dataclasses import dataclass, field

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libgsq.so")

GSQ_OK, GSQ_EINVAL, GSQ_ENOMEM, GSQ_EHIP, GSQ_ENONFINITE, GSQ_EUNSUPPORTED = 0, -1, -2, -3, -4, -5
LAYOUT_GROUP, LAYOUT_SUPERBLOCK, LAYOUT_BASE3 = 0, 1, 2
RELAX_GRID, RELAX_SHIFT, RELAX_TERNARY = 0, 1, 2
MAX_LEVELS = 16             # GSQ_MAX_LEVELS
SHIFT_WINDOW = 5            # GSQ_SHIFT_WINDOW
PREC_FP32, PREC_BF16 = 0, 1
DT_FP32, DT_BF16, DT_FP16 = 0, 1, 2
OPT_ADAM, OPT_LION = 0, 1
MAX_SAMPLES = 16            # GSQ_MAX_SAMPLES
SCORE_SOFTMAX, SCORE_SIGMOID = 0, 1
GROUP_MAX, GROUP_TOP2 = 0, 1
STATUS_NAMES = {0: "GSQ_OK", -1: "GSQ_EINVAL", -2: "GSQ_ENOMEM", -3: "GSQ_EHIP",
                -4: "GSQ_ENONFINITE", -5: "GSQ_EUNSUPPORTED"}

EXPORTS = ("gsq_layer_init", "gsq_step", "gsq_step_static", "gsq_harden", "gsq_packed_size",
           "gsq_pack", "gsq_get_state", "gsq_set_state", "gsq_get_intermediates", "gsq_gumbel", "gsq_check",
           "gsq_layer_destroy", "gsq_release_cached", "gsq_last_error", "gsq_timing", "gsq_timing_read")
PRODUCT_EXPORTS = ("gsq_grouped_forward", "gsq_grouped_input_grad", "gsq_grouped_weight_grad", "gsq_gram",
                   "gsq_quantize_rows", "gsq_grouped_forward_i8", "gsq_linear_init", "gsq_linear_forward",
                   "gsq_linear_destroy")
ROUTING_EXPORTS = ("gsq_route", "gsq_route_grad", "gsq_group_rows", "gsq_dispatch_rows", "gsq_combine_rows",
                   "gsq_combine_rows_grad")
ADAPTER_EXPORTS = ("gsq_adapter_forward", "gsq_adapter_input_grad", "gsq_adapter_weight_grad")
KERNEL_NAMES = ("init", "forward", "contract", "reduce", "backward", "harden", "pack")


class GsqError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


def _int32(name, value):
    """`value`, which has to fit the library's 32-bit argument: ctypes would keep its low bits in silence."""
    if not -(1 << 31) <= value < 1 << 31:
        raise ValueError(f"{name} does not fit 32 bits: {value}")
    return value


class CConfig(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("out_features", ctypes.c_int32),
                ("in_features", ctypes.c_int32), ("n_levels", ctypes.c_int32),
                ("levels", ctypes.c_float * MAX_LEVELS), ("group_size", ctypes.c_int32),
                ("layout", ctypes.c_int32), ("precision", ctypes.c_int32),
                ("seed", ctypes.c_uint64), ("alpha", ctypes.c_float), ("sigma_init", ctypes.c_float),
                ("init_noise", ctypes.c_int32), ("relaxation", ctypes.c_int32)]


class CStepParams(ctypes.Structure):
    _fields_ = [("tau", ctypes.c_float), ("kappa", ctypes.c_float), ("lr_logits", ctypes.c_float),
                ("lr_scales", ctypes.c_float), ("beta1", ctypes.c_float), ("beta2", ctypes.c_float),
                ("eps", ctypes.c_float), ("gumbel_noise", ctypes.c_int32),
                ("tau_next", ctypes.c_float), ("kappa_next", ctypes.c_float),
                ("optimizer", ctypes.c_int32), ("weight_decay", ctypes.c_float),
                ("samples", ctypes.c_int32)]


class CGrouped(ctypes.Structure):
    _fields_ = [("groups", ctypes.c_int32), ("out_features", ctypes.c_int32),
                ("in_features", ctypes.c_int32), ("dtype", ctypes.c_int32), ("rows", ctypes.c_int64)]


class CRouting(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64), ("experts", ctypes.c_int32), ("top_k", ctypes.c_int32),
                ("groups", ctypes.c_int32), ("top_groups", ctypes.c_int32), ("score", ctypes.c_int32),
                ("group_score", ctypes.c_int32), ("renormalise", ctypes.c_int32), ("scale", ctypes.c_float),
                ("dtype", ctypes.c_int32)]


class CExchange(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64), ("rows", ctypes.c_int64), ("copies", ctypes.c_int32),
                ("cols", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class CAdapters(ctypes.Structure):
    _fields_ = [("segments", ctypes.c_int32), ("adapters", ctypes.c_int32), ("rank", ctypes.c_int32),
                ("out_features", ctypes.c_int32), ("in_features", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("rows", ctypes.c_int64)]


@dataclass
class LayerConfig:
    out_features: int
    in_features: int
    levels: tuple
    group_size: int = 128
    batch: int = 1
    layout: int = LAYOUT_GROUP
    precision: int = PREC_BF16
    seed: int = 0
    alpha: float = 6.0
    sigma_init: float = 1.0
    init_noise: bool = True
    relaxation: int = RELAX_GRID

    def to_c(self):
        c = CConfig()
        c.batch = _int32("batch", self.batch)
        c.out_features = _int32("out_features", self.out_features)
        c.in_features = _int32("in_features", self.in_features)
        c.n_levels = len(self.levels)
        for k, x in enumerate(self.levels):
            c.levels[k] = float(x)
        c.group_size, c.layout, c.precision = _int32("group_size", self.group_size), self.layout, self.precision
        c.seed, c.alpha, c.sigma_init = self.seed, self.alpha, self.sigma_init
        c.init_noise = 1 if self.init_noise else 0
        c.relaxation = self.relaxation
        return c

    @property
    def gs(self):
        return 16 if self.layout == LAYOUT_SUPERBLOCK else self.group_size

    @property
    def K(self):
        """Logits per coordinate."""
        return {RELAX_SHIFT: SHIFT_WINDOW, RELAX_TERNARY: 2}.get(self.relaxation, len(self.levels))


@dataclass
class StepParams:
    tau: float
    kappa: float = 1.0
    lr_logits: float = 1e-2
    lr_scales: float = 5e-5
    beta1: float = 0.9
    beta2: float = 0.95
    eps: float = 1e-8
    gumbel_noise: bool = True
    tau_next: float = 0.0
    kappa_next: float = 1.0
    optimizer: int = OPT_ADAM
    weight_decay: float = 0.0
    samples: int = 1

    def to_c(self):
        return CStepParams(self.tau, self.kappa, self.lr_logits, self.lr_scales, self.beta1,
                           self.beta2, self.eps, 1 if self.gumbel_noise else 0, self.tau_next,
                           self.kappa_next, self.optimizer, self.weight_decay, self.samples)


@dataclass
class Routing:
    """How tokens choose their experts (gsq_routing)."""
    experts: int
    top_k: int
    groups: int = 1
    top_groups: int = 1
    score: int = SCORE_SOFTMAX
    group_score: int = GROUP_TOP2
    renormalise: bool = True
    scale: float = 1.0

    def to_c(self, tokens, dtype):
        return CRouting(tokens, _int32("experts", self.experts), _int32("top_k", self.top_k),
                        _int32("groups", self.groups), _int32("top_groups", self.top_groups),
                        _int32("score", self.score), _int32("group_score", self.group_score),
                        1 if self.renormalise else 0, self.scale, dtype)


_lib = None


def load(path=None):
    """Load libgsq.so (raises if it is missing: there is no fallback path)."""
    global _lib
    if _lib is not None:
        return _lib
    path = path or _LIB_PATH
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with __graft_entry__.build() "
                           "(hipcc, gfx950); the GSQ step has no other implementation")
    lib = ctypes.CDLL(path)
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    lib.gsq_layer_init.argtypes = [ctypes.POINTER(CConfig), vp, i32, vp, vp, vp, ctypes.POINTER(vp)]
    lib.gsq_step.argtypes = [vp, ctypes.POINTER(CStepParams), vp, vp]
    lib.gsq_step_static.argtypes = [vp, ctypes.POINTER(CStepParams), vp, vp]
    lib.gsq_harden.argtypes = [vp, vp, vp, vp, vp]
    lib.gsq_packed_size.argtypes = [ctypes.POINTER(CConfig)]
    lib.gsq_packed_size.restype = sz
    lib.gsq_pack.argtypes = [vp, vp, sz, vp]
    lib.gsq_get_state.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, ctypes.POINTER(i64), vp]
    lib.gsq_set_state.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, i64, vp]
    lib.gsq_get_intermediates.argtypes = [vp, vp, vp, vp]
    lib.gsq_gumbel.argtypes = [ctypes.POINTER(CConfig), i64, i64, i64, vp, vp]
    lib.gsq_check.argtypes = [vp, vp]
    lib.gsq_layer_destroy.argtypes = [vp]
    lib.gsq_release_cached.argtypes = []
    lib.gsq_last_error.restype = ctypes.c_char_p
    lib.gsq_timing.argtypes = [vp, i32]
    lib.gsq_timing_read.argtypes = [vp, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(i64), i32, vp]
    gp = ctypes.POINTER(CGrouped)
    lib.gsq_grouped_forward.argtypes = [gp, vp, vp, vp, vp, vp]
    lib.gsq_grouped_input_grad.argtypes = [gp, vp, vp, vp, vp, vp]
    lib.gsq_grouped_weight_grad.argtypes = [gp, vp, vp, vp, vp, i32, i32, vp]
    lib.gsq_gram.argtypes = [gp, vp, vp, vp, i32, vp]
    lib.gsq_quantize_rows.argtypes = [vp, i32, i64, i32, vp, vp, vp]
    lib.gsq_grouped_forward_i8.argtypes = [gp, vp, vp, vp, vp, vp, vp, vp]
    lib.gsq_linear_init.argtypes = [ctypes.POINTER(CConfig), vp, sz, vp, ctypes.POINTER(vp)]
    lib.gsq_linear_forward.argtypes = [vp, vp, i32, i64, vp, vp, vp]
    lib.gsq_linear_destroy.argtypes = [vp]
    rp, xp = ctypes.POINTER(CRouting), ctypes.POINTER(CExchange)
    lib.gsq_route.argtypes = [rp, vp, vp, vp, vp, vp]
    lib.gsq_route_grad.argtypes = [rp, vp, vp, vp, vp, vp]
    lib.gsq_group_rows.argtypes = [vp, i64, i32, vp, vp, vp, vp]
    lib.gsq_dispatch_rows.argtypes = [xp, vp, vp, vp, vp]
    lib.gsq_combine_rows.argtypes = [xp, vp, vp, vp, vp, vp]
    lib.gsq_combine_rows_grad.argtypes = [xp, vp, vp, vp, vp, vp, vp, vp]
    ap = ctypes.POINTER(CAdapters)
    lib.gsq_adapter_forward.argtypes = [ap, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.gsq_adapter_input_grad.argtypes = [ap, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.gsq_adapter_weight_grad.argtypes = [ap, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, vp]
    for name in PRODUCT_EXPORTS + ROUTING_EXPORTS + ADAPTER_EXPORTS:
        getattr(lib, name).restype = ctypes.c_int
    for name in ("gsq_layer_init", "gsq_step", "gsq_step_static", "gsq_harden", "gsq_pack",
                 "gsq_get_state", "gsq_set_state", "gsq_get_intermediates", "gsq_gumbel", "gsq_check",
                 "gsq_layer_destroy", "gsq_release_cached", "gsq_timing", "gsq_timing_read"):
        getattr(lib, name).restype = ctypes.c_int
    _lib = lib
    return lib


def _check(status):
    if status != GSQ_OK:
        raise GsqError(status, load().gsq_last_error().decode())


def release_cached():
    """Free the device memory the library keeps from destroyed layers for the next ones."""
    _check(load().gsq_release_cached())


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _arg(t, name, numel, dtypes):
    """Check a tensor argument before its pointer reaches the library, which reads or writes
    exactly ``numel`` elements through it: a dense device tensor of one of ``dtypes``."""
    if t is None:
        return
    if not (t.is_cuda and t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous device tensor")
    if t.dtype not in dtypes:
        raise TypeError(f"{name} must be {' or '.join(str(d) for d in dtypes)}, got {t.dtype}")
    if t.numel() != numel:
        raise ValueError(f"{name} must hold {numel} elements, got {t.numel()}")


def _stream(stream):
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def packed_size(cfg):
    return int(load().gsq_packed_size(ctypes.byref(cfg.to_c())))


def gumbel(cfg, e0, count, t, out, stream=None):
    """Noise of coordinates [e0, e0 + count) at step t into ``out`` (cuda fp32, count x Z):
    Z = K Gumbel values, or for TERNARY the two pairs' logistic values."""
    import torch
    if count > 0:
        _arg(out, "out", count * cfg.K, (torch.float32,))
    _check(load().gsq_gumbel(ctypes.byref(cfg.to_c()), e0, count, t, _ptr(out), _stream(stream)))


class Layer:
    """One handle of the library (gsq_layer*)."""

    def __init__(self, cfg, W, H, scales_init=None, stream=None):
        import torch
        lib = load()
        self.cfg = cfg
        self._c = cfg.to_c()
        if W.dtype == torch.bfloat16:
            wdt = DT_BF16
        elif W.dtype == torch.float32:
            wdt = DT_FP32
        else:
            raise TypeError("W must be float32 or bfloat16")
        for name, t in (("W", W), ("H", H), ("scales_init", scales_init)):
            if t is not None and not (t.is_cuda and t.is_contiguous()):
                raise ValueError(f"{name} must be a contiguous device tensor")
        if H.dtype != torch.float32:
            raise TypeError("H must be float32")
        B, O, I = cfg.batch, cfg.out_features, cfg.in_features
        _arg(W, "W", B * O * I, (torch.float32, torch.bfloat16))
        _arg(H, "H", B * I * I, (torch.float32,))
        _arg(scales_init, "scales_init", B * O * (I // cfg.gs), (torch.float32,))
        h = ctypes.c_void_p()
        _check(lib.gsq_layer_init(ctypes.byref(self._c), _ptr(W), wdt, _ptr(H), _ptr(scales_init),
                                  _stream(stream), ctypes.byref(h)))
        self._h = h

    @property
    def handle(self):
        if self._h is None:
            raise RuntimeError("layer destroyed")
        return self._h

    # element counts of the caller-side tensors
    @property
    def _n(self):
        c = self.cfg
        return c.batch * c.out_features * c.in_features

    @property
    def _ng(self):
        c = self.cfg
        return c.batch * c.out_features * (c.in_features // c.gs)

    def step(self, params, loss_out=None, stream=None):
        import torch
        _arg(loss_out, "loss_out", self.cfg.batch, (torch.float32,))
        _check(load().gsq_step(self.handle, ctypes.byref(params.to_c()), _ptr(loss_out),
                               _stream(stream)))

    def step_static(self, params, loss_out=None, stream=None):
        """gsq_step_static: the same step with no allocation (static scratch of the library)."""
        import torch
        _arg(loss_out, "loss_out", self.cfg.batch, (torch.float32,))
        _check(load().gsq_step_static(self.handle, ctypes.byref(params.to_c()), _ptr(loss_out),
                                      _stream(stream)))

    def harden(self, codes=None, scales=None, hard_loss=None, stream=None):
        import torch
        _arg(codes, "codes", self._n, (torch.uint8,))
        _arg(scales, "scales", self._ng, (torch.float32,))
        _arg(hard_loss, "hard_loss", self.cfg.batch, (torch.float32,))
        _check(load().gsq_harden(self.handle, _ptr(codes), _ptr(scales), _ptr(hard_loss),
                                 _stream(stream)))

    def pack(self, out, stream=None):
        if not (out.is_cuda and out.is_contiguous()):
            raise ValueError("out must be a contiguous device tensor")
        _check(load().gsq_pack(self.handle, _ptr(out), out.numel() * out.element_size(),
                               _stream(stream)))

    def get_state(self, logits=None, m=None, v=None, scales=None, m_s=None, v_s=None, base=None,
                  stream=None):
        self._state_args(logits, m, v, scales, m_s, v_s, base)
        t = ctypes.c_int64()
        _check(load().gsq_get_state(self.handle, _ptr(logits), _ptr(m), _ptr(v), _ptr(scales),
                                    _ptr(m_s), _ptr(v_s), _ptr(base), ctypes.byref(t),
                                    _stream(stream)))
        return t.value

    def set_state(self, t, logits=None, m=None, v=None, scales=None, m_s=None, v_s=None, base=None,
                  stream=None):
        self._state_args(logits, m, v, scales, m_s, v_s, base)
        _check(load().gsq_set_state(self.handle, _ptr(logits), _ptr(m), _ptr(v), _ptr(scales),
                                    _ptr(m_s), _ptr(v_s), _ptr(base), int(t), _stream(stream)))

    def _state_args(self, logits, m, v, scales, m_s, v_s, base):
        import torch
        for name, x in (("logits", logits), ("m", m), ("v", v)):
            _arg(x, name, self._n * self.cfg.K, (torch.float32,))
        for name, x in (("scales", scales), ("m_s", m_s), ("v_s", v_s)):
            _arg(x, name, self._ng, (torch.float32,))
        _arg(base, "base", self._n, (torch.uint8,))

    def intermediates(self, residual=None, grad=None, stream=None):
        import torch
        _arg(residual, "residual", self._n,
             (torch.bfloat16,) if self.cfg.precision == PREC_BF16 else (torch.float32,))
        _arg(grad, "grad", self._n, (torch.float32,))
        _check(load().gsq_get_intermediates(self.handle, _ptr(residual), _ptr(grad), _stream(stream)))

    def timing(self, enable):
        _check(load().gsq_timing(self.handle, 1 if enable else 0))

    def timing_read(self, reset=True, stream=None):
        """{kernel: (total ms, launches)} since the last reset (synchronises the stream)."""
        n = len(KERNEL_NAMES)
        ms = (ctypes.c_double * n)()
        cnt = (ctypes.c_int64 * n)()
        _check(load().gsq_timing_read(self.handle, ms, cnt, 1 if reset else 0, _stream(stream)))
        return {KERNEL_NAMES[k]: (ms[k], cnt[k]) for k in range(n)}

    def check(self, stream=None):
        _check(load().gsq_check(self.handle, _stream(stream)))

    def destroy(self):
        if self._h is not None:
            load().gsq_layer_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


# ---- products of grouped rows: x is rows x I with the rows of all groups sorted by group, w is groups x
# O x I (or O x I for one group), and ``offsets`` a device int64 tensor of groups + 1 row offsets (None
# for one group that has every row).

def _checked(args, offsets, groups):
    """Check tensor arguments, (name, tensor, shape, dtypes) each, and the offsets: dense, of that shape and
    one of those types, and on the current device, which is returned.  These calls take microseconds, so
    the checks are made without building anything unless one fails."""
    import torch
    device = torch.cuda.current_device() if torch.cuda.is_initialized() else -1
    if offsets is not None:
        args += (("offsets", offsets, (groups + 1,), (torch.int64,)),)
    elif groups != 1:
        raise ValueError(f"{groups} groups need offsets")
    for name, t, shape, dtypes in args:
        if not (t.shape == shape and t.dtype in dtypes and t.is_contiguous() and t.get_device() == device >= 0):
            _refuse(args, device)
    return device


def _refuse(args, device):
    for name, t, shape, _ in args:
        if tuple(t.shape) != tuple(shape):
            raise ValueError(f"{name} must have the shape {tuple(shape)}, got {tuple(t.shape)}")
    for name, t, _, dtypes in args:
        _arg(t, name, t.numel(), dtypes)
        if t.get_device() != device:
            raise ValueError(f"{name} is on {t.device}, but device {device} is current")
    raise ValueError("arguments do not fit together")


def _raw_stream(stream, device):
    import torch
    if stream is not None:
        if getattr(stream, "device_index", device) != device:
            raise ValueError(f"the stream is on device {stream.device_index}, but device {device} is current")
        return stream.cuda_stream
    return torch._C._cuda_getCurrentRawStream(device)   # current_stream() without building an object


def _rows_dtype(t):
    import torch
    if t.dtype is torch.bfloat16:
        return DT_BF16
    if t.dtype is torch.float16:
        return DT_FP16
    raise TypeError(f"rows must be bfloat16 or float16, got {t.dtype}")


def _weight_sizes(w, name="w"):
    shape = w.shape
    if len(shape) == 2:
        shape = (1, *shape)
    elif len(shape) != 3:
        raise ValueError(f"{name} must be groups x O x I or O x I, got {tuple(shape)}")
    if max(shape) >= 1 << 31:
        _int32(f"the largest size of {name}", max(shape))
    return shape


def _row_count(x, name):
    if len(x.shape) != 2:
        raise ValueError(f"{name} must be rows x features, got {tuple(x.shape)}")
    return x.shape[0]


def _address(t):
    return None if t is None else t.data_ptr()


def grouped_forward(x, w, out, offsets=None, stream=None):
    """out = x W_e^T for the rows of each group (x, w, out: bfloat16 or float16)."""
    (n, o, i), r, dt, types = _weight_sizes(w), _row_count(x, "x"), _rows_dtype(x), (x.dtype,)
    dev = _checked((("x", x, (r, i), types), ("w", w, w.shape, types), ("out", out, (r, o), types)), offsets, n)
    _check(load().gsq_grouped_forward(ctypes.byref(CGrouped(n, o, i, dt, r)), x.data_ptr(), w.data_ptr(),
                                      _address(offsets), out.data_ptr(), _raw_stream(stream, dev)))


def grouped_input_grad(dy, w, out, offsets=None, stream=None):
    """out = dy W_e, the gradient of grouped_forward's x."""
    (n, o, i), r, dt, types = _weight_sizes(w), _row_count(dy, "dy"), _rows_dtype(dy), (dy.dtype,)
    dev = _checked((("dy", dy, (r, o), types), ("w", w, w.shape, types), ("out", out, (r, i), types)), offsets, n)
    _check(load().gsq_grouped_input_grad(ctypes.byref(CGrouped(n, o, i, dt, r)), dy.data_ptr(), w.data_ptr(),
                                         _address(offsets), out.data_ptr(), _raw_stream(stream, dev)))


def grouped_weight_grad(dy, x, out, offsets=None, accumulate=False, stream=None):
    """out_e = sum of dy[r]^T x[r] over the rows of group e, the gradient of grouped_forward's w, in the
    type of x or in float32; ``accumulate`` adds to a float32 out."""
    import torch
    (n, o, i), r, dt, types = _weight_sizes(out, "out"), _row_count(dy, "dy"), _rows_dtype(dy), (dy.dtype,)
    dev = _checked((("dy", dy, (r, o), types), ("x", x, (r, i), types),
                    ("out", out, out.shape, types + (torch.float32,))), offsets, n)
    _check(load().gsq_grouped_weight_grad(ctypes.byref(CGrouped(n, o, i, dt, r)), dy.data_ptr(), x.data_ptr(),
                                          _address(offsets), out.data_ptr(),
                                          DT_FP32 if out.dtype is torch.float32 else dt,
                                          1 if accumulate else 0, _raw_stream(stream, dev)))


def gram(x, out, offsets=None, accumulate=False, stream=None):
    """out_e = X_e^T X_e in float32 (groups x I x I or I x I), the H of ``Layer``; ``accumulate`` adds to it."""
    import torch
    (n, i, i2), r, dt = _weight_sizes(out, "out"), _row_count(x, "x"), _rows_dtype(x)
    if i != i2:
        raise ValueError(f"out must be square, got {tuple(out.shape)}")
    dev = _checked((("x", x, (r, i), (x.dtype,)), ("out", out, out.shape, (torch.float32,))), offsets, n)
    _check(load().gsq_gram(ctypes.byref(CGrouped(n, 0, i, dt, r)), x.data_ptr(), _address(offsets),
                           out.data_ptr(), 1 if accumulate else 0, _raw_stream(stream, dev)))


def quantize_rows(x, q, scales, stream=None):
    """Rows of x (rows x cols; float32, bfloat16 or float16) as int8 ``q`` and a float32 scale each: tokens
    of activations, or output channels of weights (a groups x O x I tensor has groups * O rows)."""
    import torch
    if len(x.shape) < 2:
        raise ValueError(f"x must be rows x columns, got {tuple(x.shape)}")
    dt, cols = DT_FP32 if x.dtype is torch.float32 else _rows_dtype(x), _int32("the columns of x", x.shape[-1])
    dev = _checked((("x", x, x.shape, (x.dtype,)), ("q", q, x.shape, (torch.int8,)),
                    ("scales", scales, x.shape[:-1], (torch.float32,))), None, 1)
    _check(load().gsq_quantize_rows(x.data_ptr(), dt, scales.numel(), cols, q.data_ptr(),
                                    scales.data_ptr(), _raw_stream(stream, dev)))


def grouped_forward_i8(x, x_scales, w, w_scales, out, offsets=None, stream=None):
    """out[r, n] = x_scales[r] w_scales[e, n] sum_k x[r, k] w[e, n, k] for int8 x and w."""
    import torch
    (n, o, i), r, dt = _weight_sizes(w), _row_count(x, "x"), _rows_dtype(out)
    ints, floats = (torch.int8,), (torch.float32,)
    dev = _checked((("x", x, (r, i), ints), ("x_scales", x_scales, (r,), floats), ("w", w, w.shape, ints),
                    ("w_scales", w_scales, w.shape[:-1], floats), ("out", out, (r, o), (out.dtype,))), offsets, n)
    _check(load().gsq_grouped_forward_i8(ctypes.byref(CGrouped(n, o, i, dt, r)), x.data_ptr(),
                                         x_scales.data_ptr(), w.data_ptr(), w_scales.data_ptr(),
                                         _address(offsets), out.data_ptr(), _raw_stream(stream, dev)))


class Linear:
    """A packed layer in use (gsq_linear*): ``packed`` holds what Layer.pack wrote for ``cfg``."""

    def __init__(self, cfg, packed, stream=None):
        self._h = None
        self.cfg = cfg
        dev = _checked((("packed", packed, packed.shape, (packed.dtype,)),), None, 1)
        h = ctypes.c_void_p()
        _check(load().gsq_linear_init(ctypes.byref(cfg.to_c()), packed.data_ptr(),
                                      packed.numel() * packed.element_size(), _raw_stream(stream, dev),
                                      ctypes.byref(h)))
        self._h = h

    def forward(self, x, out, offsets=None, stream=None):
        """out = x W_e^T with the packed weights (x, out: bfloat16 or float16)."""
        if self._h is None:
            raise RuntimeError("layer destroyed")
        c, r, dt, types = self.cfg, _row_count(x, "x"), _rows_dtype(x), (x.dtype,)
        dev = _checked((("x", x, (r, c.in_features), types), ("out", out, (r, c.out_features), types)),
                       offsets, c.batch)
        _check(load().gsq_linear_forward(self._h, x.data_ptr(), dt, r, _address(offsets), out.data_ptr(),
                                         _raw_stream(stream, dev)))

    def destroy(self):
        if self._h is not None:
            load().gsq_linear_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


# ---- rows to the routed experts and back: logits are tokens x experts, and slots (tokens x top_k, int32) say where
# each copy of a token stands among the rows of all experts (-1: nowhere).

def _float_dtype(t):
    import torch
    return DT_FP32 if t.dtype is torch.float32 else _rows_dtype(t)


def _cut(name, t):
    if len(t.shape) != 2:
        raise ValueError(f"{name} must have two dimensions, got {tuple(t.shape)}")
    return t.shape


def route(routing, logits, experts, weights, bias=None, stream=None):
    """The ``top_k`` experts (int32) and weights (float32) of each token from its logits (tokens x experts;
    float32, bfloat16 or float16); the float32 ``bias`` of each expert enters the choice only."""
    import torch
    (t, e), dt, k = _cut("logits", logits), _float_dtype(logits), routing.top_k
    args = (("logits", logits, (t, routing.experts), (logits.dtype,)),
            ("experts", experts, (t, k), (torch.int32,)), ("weights", weights, (t, k), (torch.float32,)))
    if bias is not None:
        args += (("bias", bias, (routing.experts,), (torch.float32,)),)
    dev = _checked(args, None, 1)
    _check(load().gsq_route(ctypes.byref(routing.to_c(t, dt)), logits.data_ptr(), _address(bias), experts.data_ptr(),
                            weights.data_ptr(), _raw_stream(stream, dev)))


def route_grad(routing, logits, experts, dweights, out, stream=None):
    """out = the gradient of route's logits (their shape and type) from that of its weights, for the experts that
    it chose."""
    import torch
    (t, e), dt, k = _cut("logits", logits), _float_dtype(logits), routing.top_k
    dev = _checked((("logits", logits, (t, routing.experts), (logits.dtype,)),
                    ("experts", experts, (t, k), (torch.int32,)), ("dweights", dweights, (t, k), (torch.float32,)),
                    ("out", out, (t, routing.experts), (logits.dtype,))), None, 1)
    _check(load().gsq_route_grad(ctypes.byref(routing.to_c(t, dt)), logits.data_ptr(), experts.data_ptr(),
                                 dweights.data_ptr(), out.data_ptr(), _raw_stream(stream, dev)))


def group_rows(ids, offsets, slots, sources, stream=None):
    """The stable order that brings equal ids together (int32 of any shape; one group for each of ``offsets`` but the
    last, other ids belong to none): the groups' int64 row ``offsets``, as the products take them, the int32 ``slots``
    (shape of ids) where each id goes, and the int32 ``sources`` (one for each id) that stand at each place."""
    import torch
    n, groups, ints = ids.numel(), offsets.numel() - 1, (torch.int32,)
    dev = _checked((("ids", ids, ids.shape, ints), ("slots", slots, ids.shape, ints),
                    ("sources", sources, (n,), ints), ("offsets", offsets, (groups + 1,), (torch.int64,))), None, 1)
    _check(load().gsq_group_rows(ids.data_ptr(), n, _int32("groups", groups), offsets.data_ptr(), slots.data_ptr(),
                                 sources.data_ptr(), _raw_stream(stream, dev)))


def _exchange(tokens, rows, slots, dtype):
    """The sizes of an exchange between ``tokens`` and ``rows``, and the shape of its slots."""
    (t, c), r, (_, k) = _cut("tokens", tokens), _row_count(rows, "rows"), _cut("slots", slots)
    return CExchange(t, r, _int32("the slots of a token", k), _int32("the columns", c), dtype), (t, k), (t, c), (r, c)


def dispatch_rows(x, slots, out, stream=None):
    """out[slots[t, k]] = x[t] (float32, bfloat16 or float16); rows of out that no slot names stay as they were."""
    import torch
    types = (x.dtype,)
    g, s, of_tokens, of_rows = _exchange(x, out, slots, _float_dtype(x))
    dev = _checked((("x", x, of_tokens, types), ("slots", slots, s, (torch.int32,)), ("out", out, of_rows, types)),
                   None, 1)
    _check(load().gsq_dispatch_rows(ctypes.byref(g), x.data_ptr(), slots.data_ptr(), out.data_ptr(),
                                    _raw_stream(stream, dev)))


def combine_rows(rows, slots, out, weights=None, stream=None):
    """out[t] = sum of weights[t, k] rows[slots[t, k]] over k (no weights: ones, which is dispatch_rows' gradient)."""
    import torch
    types = (rows.dtype,)
    g, s, of_tokens, of_rows = _exchange(out, rows, slots, _float_dtype(rows))
    args = (("rows", rows, of_rows, types), ("slots", slots, s, (torch.int32,)), ("out", out, of_tokens, types))
    if weights is not None:
        args += (("weights", weights, s, (torch.float32,)),)
    dev = _checked(args, None, 1)
    _check(load().gsq_combine_rows(ctypes.byref(g), rows.data_ptr(), slots.data_ptr(), _address(weights),
                                   out.data_ptr(), _raw_stream(stream, dev)))


def combine_rows_grad(dout, rows, slots, weights, drows, dweights, stream=None):
    """combine_rows' gradients: drows[slots[t, k]] = weights[t, k] dout[t], and dweights[t, k] = the product of dout[t]
    and rows[slots[t, k]]; rows of drows that no slot names stay as they were."""
    import torch
    types, floats = (dout.dtype,), (torch.float32,)
    g, s, of_tokens, of_rows = _exchange(dout, rows, slots, _float_dtype(dout))
    dev = _checked((("dout", dout, of_tokens, types), ("rows", rows, of_rows, types),
                    ("slots", slots, s, (torch.int32,)), ("weights", weights, s, floats),
                    ("drows", drows, of_rows, types), ("dweights", dweights, s, floats)), None, 1)
    _check(load().gsq_combine_rows_grad(ctypes.byref(g), dout.data_ptr(), rows.data_ptr(), slots.data_ptr(),
                                        weights.data_ptr(), drows.data_ptr(), dweights.data_ptr(),
                                        _raw_stream(stream, dev)))


# ---- low-rank adapters of many requests beside a shared projection: rows request by request, with device int64
# ``offsets`` of the requests (None: one), the int32 adapter ``index`` of each (-1: none; None: request i has adapter
# i), a: adapters x rank x I, b: adapters x O x rank, and float32 ``scales`` of the adapters (None: ones).

def _adapter_sizes(a, b, rows, dtype, offsets, index):
    """The sizes of a call from the shapes of a and b (or of their gradients), which have to fit each other."""
    if len(a) != 3 or len(b) != 3:
        raise ValueError(f"a must be adapters x rank x I and b adapters x O x rank, got {tuple(a)} and {tuple(b)}")
    (n, q, i), o = a, b[1]
    segments = 1 if offsets is None else offsets.numel() - 1
    if max(n, q, i, o, segments) >= 1 << 31:
        _int32("the largest size of the adapters", max(n, q, i, o, segments))
    if index is None and n != segments:
        raise ValueError(f"{n} adapters for {segments} requests need an index")
    if tuple(b) != (n, o, q):
        raise ValueError(f"b must have the shape {(n, o, q)}, got {tuple(b)}")
    return CAdapters(segments, n, q, o, i, dtype, rows)


def _adapter_args(g, index, scales):
    import torch
    args = ()
    if index is not None:
        args += (("index", index, (g.segments,), (torch.int32,)),)
    if scales is not None:
        args += (("scales", scales, (g.adapters,), (torch.float32,)),)
    return args


def adapter_forward(x, a, b, hidden, out, offsets=None, index=None, scales=None, base=None, stream=None):
    """out[r] = base[r] + scale B (A x[r]) with the adapter of the row's request, hidden[r] = A x[r] (float32, rows x
    rank); x, a, b, base, out: bfloat16 or float16.  ``base`` is the shared projection's output: None for zeros, or
    out itself."""
    import torch
    r, dt, types = _row_count(x, "x"), _rows_dtype(x), (x.dtype,)
    g = _adapter_sizes(a.shape, b.shape, r, dt, offsets, index)
    q, o, i = g.rank, g.out_features, g.in_features
    args = (("x", x, (r, i), types), ("a", a, a.shape, types), ("b", b, b.shape, types),
            ("hidden", hidden, (r, q), (torch.float32,)), ("out", out, (r, o), types))
    if base is not None:
        args += (("base", base, (r, o), types),)
    dev = _checked(args + _adapter_args(g, index, scales), offsets, g.segments)
    _check(load().gsq_adapter_forward(ctypes.byref(g), x.data_ptr(), a.data_ptr(), b.data_ptr(), _address(offsets),
                                      _address(index), _address(scales), _address(base), hidden.data_ptr(),
                                      out.data_ptr(), _raw_stream(stream, dev)))


def adapter_input_grad(dy, a, b, dhidden, out, offsets=None, index=None, scales=None, base=None, stream=None):
    """out[r] = base[r] + A^T dhidden[r], dhidden[r] = scale B^T dy[r] (float32, rows x rank): the gradients of
    adapter_forward's x and hidden.  ``base`` is the shared projection's gradient of x: None for zeros, or out
    itself."""
    import torch
    r, dt, types = _row_count(dy, "dy"), _rows_dtype(dy), (dy.dtype,)
    g = _adapter_sizes(a.shape, b.shape, r, dt, offsets, index)
    q, o, i = g.rank, g.out_features, g.in_features
    args = (("dy", dy, (r, o), types), ("a", a, a.shape, types), ("b", b, b.shape, types),
            ("dhidden", dhidden, (r, q), (torch.float32,)), ("out", out, (r, i), types))
    if base is not None:
        args += (("base", base, (r, i), types),)
    dev = _checked(args + _adapter_args(g, index, scales), offsets, g.segments)
    _check(load().gsq_adapter_input_grad(ctypes.byref(g), dy.data_ptr(), a.data_ptr(), b.data_ptr(),
                                         _address(offsets), _address(index), _address(scales), _address(base),
                                         dhidden.data_ptr(), out.data_ptr(), _raw_stream(stream, dev)))


def adapter_weight_grad(dy, x, hidden, dhidden, da, db, offsets=None, index=None, scales=None, accumulate=False,
                        stream=None):
    """da = sum of dhidden[r]^T x[r] and db = scale times the sum of dy[r]^T hidden[r] over each adapter's rows, in the
    type of x or in float32; ``accumulate`` adds to float32 ones."""
    import torch
    r, dt, types, floats = _row_count(x, "x"), _rows_dtype(x), (x.dtype,), (torch.float32,)
    g = _adapter_sizes(da.shape, db.shape, r, dt, offsets, index)
    q, o, i = g.rank, g.out_features, g.in_features
    args = (("dy", dy, (r, o), types), ("x", x, (r, i), types), ("hidden", hidden, (r, q), floats),
            ("dhidden", dhidden, (r, q), floats), ("da", da, da.shape, types + floats),
            ("db", db, db.shape, (da.dtype,)))
    dev = _checked(args + _adapter_args(g, index, scales), offsets, g.segments)
    _check(load().gsq_adapter_weight_grad(ctypes.byref(g), dy.data_ptr(), x.data_ptr(), hidden.data_ptr(),
                                          dhidden.data_ptr(), _address(offsets), _address(index), _address(scales),
                                          da.data_ptr(), db.data_ptr(),
                                          DT_FP32 if da.dtype is torch.float32 else dt, 1 if accumulate else 0,
                                          _raw_stream(stream, dev)))
