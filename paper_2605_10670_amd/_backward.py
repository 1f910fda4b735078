"""The layer norm and the backward pass of the layer: what `layer` offers as LayerNorm, NormGrad, ExpertProductGrad and
Router.grad."""
import ctypes

from . import binding, layer


class _NormGradConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("hidden", "in_dtype", "gain_dtype", "out_dtype", "centred")] + \
               [("epsilon", ctypes.c_float)]


class _ProductGradConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("num_slots", "in_features", "out_features", "dtype", "grad_w_dtype", "gate",
                                              "max_rows")] + \
               [(n, ctypes.c_int64) for n in ("slot_stride", "grad_stride")]


def route_grad(router, topk_idx, topk_w, grad_w, grad_logits, T, logits, stream):
    row, choices, weights = router._needs
    rc = layer._call(layer._address["eep_route_grad"], "hpppppis", (row, choices, weights, weights, row), T, router._at, logits, topk_idx,
                     topk_w, grad_w, grad_logits, T, stream)
    if rc:
        layer._refuse(rc, "eep_route_grad", ("shape", "logits", "topk_idx", "topk_w", "grad_w", "grad_logits"))


class LayerNorm:
    """eep_layer_norm.  in_dtype is that of x, residual and sum, gain_dtype that of gain and bias."""

    def __init__(self, *, hidden, in_dtype="bf16", gain_dtype="bf16", out_dtype="bf16", epsilon=1e-5):
        layer.load()
        self._shape = layer._NormShape(hidden, layer._dtype(in_dtype), layer._dtype(gain_dtype), layer._dtype(out_dtype), 0, epsilon)
        self._at = ctypes.addressof(self._shape)
        s = self._shape
        row, gain, out = (hidden * layer._BYTES.get(d, 1) for d in (s.in_dtype, s.gain_dtype, s.out_dtype))
        self._needs = (row, row, -gain, -gain, row, out)

    def run(self, x, gain, T, *, y, residual=None, bias=None, sum=None, stream=None):
        rc = layer._call(layer._address["eep_layer_norm"], "hppppppis", self._needs, T, self._at, x, residual, gain, bias, sum, y, T, stream)
        if rc:
            layer._refuse(rc, "eep_layer_norm", ("shape", "x", "residual", "gain", "bias", "sum", "y"))


class _Handle:
    """What the C library made for a shape, until destroy."""

    _destroy = None

    def _make(self, create, config):
        self._h = ctypes.c_void_p()
        rc = getattr(layer.load(), create)(ctypes.byref(config), ctypes.byref(self._h))
        if rc != binding.OK:
            raise binding.EepError(rc, create)

    def destroy(self):
        if self._h:
            rc = getattr(layer.load(), self._destroy)(self._h)
            self._h = ctypes.c_void_p()
            if rc != binding.OK:
                raise binding.EepError(rc, self._destroy)

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


class NormGrad(_Handle):
    """eep_norm_grad: the gradients of Norm (centred=False) and LayerNorm (centred=True).  in_dtype is that of h, grad_sum and
    grad_h, out_dtype that of grad_y; grad_gain and grad_bias are fp32.  It belongs to the device that is current here.  Its calls
    share a workspace: they may not overlap (one stream, or events between)."""

    _destroy = "eep_norm_grad_destroy"

    def __init__(self, *, hidden, in_dtype="bf16", gain_dtype="bf16", out_dtype="bf16", centred=False, epsilon=None):
        epsilon = (1e-5 if centred else 1e-6) if epsilon is None else epsilon
        c = self.cfg = _NormGradConfig(hidden, layer._dtype(in_dtype), layer._dtype(gain_dtype), layer._dtype(out_dtype), 1 if centred else 0, epsilon)
        self._make("eep_norm_grad_create", c)
        row, gain, out = (hidden * layer._BYTES[d] for d in (c.in_dtype, c.gain_dtype, c.out_dtype))
        self._needs = (row, -gain, out, row, row, -4 * hidden, -4 * hidden)

    def run(self, h, gain, grad_y, T, *, grad_sum=None, grad_h=None, grad_gain=None, grad_bias=None, accumulate=False, stream=None):
        rc = layer._call(layer._address["eep_norm_grad_run"], "hpppppppiis", self._needs, T, self._h.value or 0, h, gain, grad_y, grad_sum, grad_h,
                   grad_gain, grad_bias, 1 if accumulate else 0, T, stream)
        if rc:
            layer._refuse(rc, "eep_norm_grad_run", ("grad", "h", "gain", "grad_y", "grad_sum", "grad_h", "grad_gain", "grad_bias"))


class ExpertProductGrad(_Handle):
    """eep_product_grad: the gradients of an ExpertProduct of fp32 or bf16 operands (dtype: of grad_y, sums, grad_sums, x, w and
    grad_x).  gate: of one with a gate; `sums` then is what an ExpertProduct without one and 2 * out_features gives for the same x
    and w.  slot_stride and grad_stride: bytes from one slot's weights / gradients to the next one's (None: packed).  It belongs to
    the device that is current here.  Its calls share a workspace: they may not overlap (one stream, or events between)."""

    _destroy = "eep_product_grad_destroy"

    def __init__(self, *, num_slots, in_features, out_features, max_rows, dtype="bf16", grad_w_dtype="bf16", gate=False,
                 slot_stride=None, grad_stride=None):
        c = self.cfg = _ProductGradConfig(num_slots, in_features, out_features, layer._dtype(dtype), layer._dtype(grad_w_dtype), 1 if gate else 0,
                                          max_rows, slot_stride or 0, grad_stride or 0)
        self._make("eep_product_grad_create", c)
        size, n = layer._BYTES[c.dtype], out_features * (2 if gate else 1)
        whole = lambda stride, last: -((num_slots - 1) * (stride or last) + last)
        # bytes a row, of the slots' arrays in all
        self._needs = (out_features * size, n * size, in_features * size, whole(slot_stride, n * in_features * size),
                       -4 * (num_slots + 1), n * size, in_features * size,
                       whole(grad_stride, n * in_features * layer._BYTES[c.grad_w_dtype]))

    def run(self, grad_y, rows, *, offset=None, x=None, w=None, sums=None, grad_sums=None, grad_x=None, grad_w=None,
            accumulate=False, stream=None):
        rc = layer._call(layer._address["eep_product_grad_run"], "hppppppppiis", self._needs, rows, self._h.value or 0, grad_y, sums, x, w, offset,
                   grad_sums, grad_x, grad_w, 1 if accumulate else 0, rows, stream)
        if rc:
            layer._refuse(rc, "eep_product_grad_run", ("grad", "grad_y", "sums", "x", "w", "offset", "grad_sums", "grad_x", "grad_w"))
