"""The layer around dispatch and combine (include/eep.h): the residual norm with its 8-bit codes, the router's choice,
the experts' products.  Each class is a shape that was checked once, like `binding.Context`; its `run` queues the
call.  Device buffers are torch tensors (or raw integer addresses, such as those of `Context.view_pointers`), bf16 as
bfloat16 or 16-bit integers, e4m3 codes as float8_e4m3fn or bytes; streams are raw handles or torch streams.

    norm = layer.Norm(hidden=H, in_dtype="bf16", scale_group=128)
    router = layer.Router(num_logical=E, topk=k)
    up = layer.ExpertProduct(num_slots=P, in_features=H, out_features=I, x_dtype="fp8", y_dtype="fp8",
                             gate=True, max_rows=T * k)
    down = layer.ExpertProduct(num_slots=P, in_features=I, out_features=H, x_dtype="fp8", max_rows=T * k)
    logits = layer.ExpertProduct(num_slots=1, in_features=H, out_features=E, y_dtype="f32", max_rows=T)
"""
import ctypes

from . import binding

DTYPES = binding.DTYPES
_BYTES = {binding.F32: 4, binding.BF16: 2, binding.FP8_E4M3: 1}
SCALE_BLOCK = 128


class _NormShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("hidden", "in_dtype", "gain_dtype", "out_dtype", "scale_group")] + \
               [("epsilon", ctypes.c_float)]


class _RouterShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("num_logical", "topk", "in_dtype", "over_all")]


class _ProductConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("num_slots", "in_features", "out_features", "x_dtype", "y_dtype", "gate",
                                              "max_rows")] + \
               [(n, ctypes.c_int64) for n in ("slot_stride", "scale_stride")]


_lib = None
_address = {}


def load():
    """The library with the signatures of this module's entry points."""
    global _lib
    if _lib is None:
        lib = binding.load()
        vp, i32 = ctypes.c_void_p, ctypes.c_int32
        sig = {
            "eep_residual_norm": [ctypes.POINTER(_NormShape), vp, vp, vp, vp, vp, vp, vp, i32, vp],
            "eep_route": [ctypes.POINTER(_RouterShape), vp, vp, vp, i32, vp],
            "eep_product_create": [ctypes.POINTER(_ProductConfig), ctypes.POINTER(vp)],
            "eep_product_destroy": [vp],
            "eep_expert_product": [vp, vp, vp, vp, vp, vp, vp, vp, i32, vp],
        }
        for name, argtypes in sig.items():
            fn = getattr(lib, name)
            fn.argtypes, fn.restype = argtypes, ctypes.c_int
            _address[name] = ctypes.cast(fn, vp).value
        _lib = lib
    return _lib


def _call(*args):
    """native/marshal.cpp's call_ten, which binding's first call loads (and builds if it is not there)."""
    global _call
    try:
        binding._call(None)  # loads the module; no entry point's call
    except TypeError:
        pass
    from . import _marshal
    _call = _marshal.call_ten
    return _call(*args)


def _dtype(name):
    return DTYPES[name] if isinstance(name, str) else name


def _holds(name, t, nbytes):
    """Refuses a tensor that is too small for what the call reads or writes."""
    if t is not None and not isinstance(t, int) and t.nbytes < nbytes:
        raise ValueError(f"{name} has {t.nbytes} bytes, the call needs {nbytes}")


class Norm:
    """eep_residual_norm.  in_dtype is that of x, residual and sum; scale_group 0: no codes."""

    def __init__(self, *, hidden, in_dtype="bf16", gain_dtype="bf16", out_dtype="bf16", scale_group=0, epsilon=1e-6):
        load()
        self._shape = _NormShape(hidden, _dtype(in_dtype), _dtype(gain_dtype), _dtype(out_dtype), scale_group, epsilon)
        self._at = ctypes.addressof(self._shape)
        s = self._shape
        self._in, self._out = hidden * _BYTES.get(s.in_dtype, 1), hidden * _BYTES.get(s.out_dtype, 1)
        self._gain, self._hidden = hidden * _BYTES.get(s.gain_dtype, 1), hidden
        self._scales = 4 * (hidden // scale_group) if scale_group else 0

    def run(self, x, gain, T, *, residual=None, sum=None, y=None, code=None, code_scale=None, stream=None):
        _holds("x", x, T * self._in)
        _holds("gain", gain, self._gain)
        _holds("residual", residual, T * self._in)
        _holds("sum", sum, T * self._in)
        _holds("y", y, T * self._out)
        _holds("code", code, T * self._hidden)
        _holds("code_scale", code_scale, T * self._scales)
        rc = _call(_address["eep_residual_norm"], "hpppppppis", self._at, x, residual, gain, sum, y, code, code_scale, T,
                   stream)
        if rc != binding.OK:
            raise binding.EepError(rc, "eep_residual_norm")


class Router:
    """eep_route.  over_all: weights relative to all logits, not to the chosen ones."""

    def __init__(self, *, num_logical, topk, in_dtype="f32", over_all=False):
        load()
        self._shape = _RouterShape(num_logical, topk, _dtype(in_dtype), 1 if over_all else 0)
        self._at = ctypes.addressof(self._shape)
        self._in, self._k = num_logical * _BYTES.get(self._shape.in_dtype, 1), topk

    def run(self, logits, topk_idx, topk_w, T, stream=None):
        _holds("logits", logits, T * self._in)
        _holds("topk_idx", topk_idx, 4 * T * self._k)
        _holds("topk_w", topk_w, 4 * T * self._k)
        rc = _call(_address["eep_route"], "hpppis", self._at, logits, topk_idx, topk_w, T, stream)
        if rc != binding.OK:
            raise binding.EepError(rc, "eep_route")


class ExpertProduct:
    """eep_expert_product.  gate: w has the gate's out_features rows, then the other factor's.  slot_stride and
    scale_stride: bytes from one slot's weights / scales to the next one's (None: packed)."""

    def __init__(self, *, num_slots, in_features, out_features, max_rows, x_dtype="bf16", y_dtype="bf16", gate=False,
                 slot_stride=None, scale_stride=None):
        lib = load()
        c = self.cfg = _ProductConfig(num_slots, in_features, out_features, _dtype(x_dtype), _dtype(y_dtype),
                                      1 if gate else 0, max_rows, slot_stride or 0, scale_stride or 0)
        self._h = ctypes.c_void_p()
        rc = lib.eep_product_create(ctypes.byref(c), ctypes.byref(self._h))
        if rc != binding.OK:
            raise binding.EepError(rc, "eep_product_create")
        n = out_features * (2 if gate else 1)
        self._x, self._y = in_features * _BYTES[c.x_dtype], out_features * _BYTES[c.y_dtype]
        weights = n * self._x
        self._w = (num_slots - 1) * (slot_stride or weights) + weights
        blocks = 4 * -(-n // SCALE_BLOCK) * (in_features // SCALE_BLOCK)
        self._w_scale = (num_slots - 1) * (scale_stride or blocks) + blocks
        self._x_scale, self._y_scale = 4 * (in_features // SCALE_BLOCK), 4 * (out_features // SCALE_BLOCK)
        self._offset = 4 * (num_slots + 1)

    def run(self, x, w, y, rows, *, offset=None, x_scale=None, w_scale=None, y_scale=None, stream=None):
        _holds("x", x, rows * self._x)
        _holds("w", w, self._w)
        _holds("y", y, rows * self._y)
        _holds("offset", offset, self._offset)
        _holds("x_scale", x_scale, rows * self._x_scale)
        _holds("w_scale", w_scale, self._w_scale)
        _holds("y_scale", y_scale, rows * self._y_scale)
        rc = _call(_address["eep_expert_product"], "hpppppppis", self._h.value or 0, x, x_scale, w, w_scale, offset, y,
                   y_scale, rows, stream)
        if rc != binding.OK:
            raise binding.EepError(rc, "eep_expert_product")

    def destroy(self):
        if self._h:
            rc = load().eep_product_destroy(self._h)
            self._h = ctypes.c_void_p()
            if rc != binding.OK:
                raise binding.EepError(rc, "eep_product_destroy")

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass
