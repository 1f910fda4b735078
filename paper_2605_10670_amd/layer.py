"""The layer around dispatch and combine (include/eep.h): the residual norm with its 8-bit codes, the layer norm, the
router's choice, the experts' products, and their gradients.  Each class is a shape that was checked once, like `binding.Context`; its `run` queues the
call.  Device buffers are torch tensors (or raw integer addresses, such as those of `Context.view_pointers`), bf16 as
bfloat16 or 16-bit integers, e4m3 codes as float8_e4m3fn or bytes; streams are raw handles or torch streams.

    norm = layer.Norm(hidden=H, in_dtype="bf16", scale_group=128)
    router = layer.Router(num_logical=E, topk=k)
    up = layer.ExpertProduct(num_slots=P, in_features=H, out_features=I, x_dtype="fp8", y_dtype="fp8",
                             gate=True, max_rows=T * k)
    down = layer.ExpertProduct(num_slots=P, in_features=I, out_features=H, x_dtype="fp8", max_rows=T * k)
    logits = layer.ExpertProduct(num_slots=1, in_features=H, out_features=E, y_dtype="f32", max_rows=T)

and for fine-tuning, in bf16 or fp32:

    norm_grad = layer.NormGrad(hidden=H)
    up_grad = layer.ExpertProductGrad(num_slots=P, in_features=H, out_features=I, gate=True, max_rows=T * k)
    down_grad = layer.ExpertProductGrad(num_slots=P, in_features=I, out_features=H, max_rows=T * k)
    router.grad(...)    # and Context.combine_grad, Context.dispatch_grad
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
            "eep_layer_norm": [ctypes.POINTER(_NormShape), vp, vp, vp, vp, vp, vp, i32, vp],
            "eep_route_grad": [ctypes.POINTER(_RouterShape), vp, vp, vp, vp, vp, i32, vp],
            "eep_norm_grad_create": [vp, ctypes.POINTER(vp)],
            "eep_norm_grad_destroy": [vp],
            "eep_norm_grad_run": [vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, vp],
            "eep_product_grad_create": [vp, ctypes.POINTER(vp)],
            "eep_product_grad_destroy": [vp],
            "eep_product_grad_run": [vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, vp],
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
    """native/marshal.cpp's call_sized, which binding's first call loads (and builds if it is not there)."""
    global _call
    try:
        binding._call(None)  # loads the module; no entry point's call
    except TypeError:
        pass
    from . import _marshal
    _call = _marshal.call_sized
    return _call(*args)


def _refuse(rc, name, arguments):
    """What a return code other than OK means; arguments: the entry point's, by name."""
    if rc <= -1000:
        raise ValueError(f"{name}: {arguments[-1000 - rc]} is smaller than what the call reads or writes")
    raise binding.EepError(rc, name)


def _dtype(name):
    return DTYPES[name] if isinstance(name, str) else name


class Norm:
    """eep_residual_norm.  in_dtype is that of x, residual and sum; scale_group 0: no codes."""

    def __init__(self, *, hidden, in_dtype="bf16", gain_dtype="bf16", out_dtype="bf16", scale_group=0, epsilon=1e-6):
        load()
        self._shape = _NormShape(hidden, _dtype(in_dtype), _dtype(gain_dtype), _dtype(out_dtype), scale_group, epsilon)
        self._at = ctypes.addressof(self._shape)
        s = self._shape
        size = lambda dtype: hidden * _BYTES.get(dtype, 1)
        # bytes a row, of gain in all
        self._needs = (size(s.in_dtype), size(s.in_dtype), -size(s.gain_dtype), size(s.in_dtype), size(s.out_dtype), hidden,
                       4 * (hidden // scale_group) if scale_group else 0)

    def run(self, x, gain, T, *, residual=None, sum=None, y=None, code=None, code_scale=None, stream=None):
        rc = _call(_address["eep_residual_norm"], "hpppppppis", self._needs, T, self._at, x, residual, gain, sum, y, code,
                   code_scale, T, stream)
        if rc:
            _refuse(rc, "eep_residual_norm", ("shape", "x", "residual", "gain", "sum", "y", "code", "code_scale"))


class Router:
    """eep_route.  over_all: weights relative to all logits, not to the chosen ones."""

    def __init__(self, *, num_logical, topk, in_dtype="f32", over_all=False):
        load()
        self._shape = _RouterShape(num_logical, topk, _dtype(in_dtype), 1 if over_all else 0)
        self._at = ctypes.addressof(self._shape)
        self._needs = (num_logical * _BYTES.get(self._shape.in_dtype, 1), 4 * topk, 4 * topk)

    def run(self, logits, topk_idx, topk_w, T, stream=None):
        rc = _call(_address["eep_route"], "hpppis", self._needs, T, self._at, logits, topk_idx, topk_w, T, stream)
        if rc:
            _refuse(rc, "eep_route", ("shape", "logits", "topk_idx", "topk_w"))

    def grad(self, topk_idx, topk_w, grad_w, grad_logits, T, *, logits=None, stream=None):
        """eep_route_grad: of what run returned; logits, as run had them, only with over_all."""
        _backward.route_grad(self, topk_idx, topk_w, grad_w, grad_logits, T, logits, stream)


class ExpertProduct:
    """eep_expert_product.  gate: w has the gate's out_features rows, then the other factor's.  slot_stride and
    scale_stride: bytes from one slot's weights / scales to the next one's (None: packed).  It belongs to the device that is
    current here.  With y_dtype "fp8" its calls share a workspace: they may not overlap (one stream, or events
    between); micro-batches that run side by side take a product each, as they take a staging set each."""

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
        weights = n * in_features * _BYTES[c.x_dtype]
        scales = 4 * -(-n // SCALE_BLOCK) * (in_features // SCALE_BLOCK)
        whole = lambda stride, last: -((num_slots - 1) * (stride or last) + last)
        # bytes a row, of the slots' arrays in all
        self._needs = (in_features * _BYTES[c.x_dtype], 4 * (in_features // SCALE_BLOCK), whole(slot_stride, weights),
                       whole(scale_stride, scales), -4 * (num_slots + 1), out_features * _BYTES[c.y_dtype],
                       4 * (out_features // SCALE_BLOCK))

    def run(self, x, w, y, rows, *, offset=None, x_scale=None, w_scale=None, y_scale=None, stream=None):
        rc = _call(_address["eep_expert_product"], "hpppppppis", self._needs, rows, self._h.value or 0, x, x_scale, w,
                   w_scale, offset, y, y_scale, rows, stream)
        if rc:
            _refuse(rc, "eep_expert_product", ("product", "x", "x_scale", "w", "w_scale", "offset", "y", "y_scale"))

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


from . import _backward  # noqa: E402  (which needs what is above)
from ._backward import ExpertProductGrad, LayerNorm, NormGrad  # noqa: E402, F401
