"""What the entry points of the backward pass and the layer norm refuse, before anything touches a GPU."""
import ctypes

import pytest
import torch

from paper_2605_10670_amd import binding, layer

_backward = layer._backward
A = 1 << 20     # an aligned address that is never read
INVALID, ALIGN = binding.ERR_INVALID_ARG, binding.ERR_ALIGN


def refused(want, call, /, **kw):
    with pytest.raises(binding.EepError) as e:
        call(**kw)
    assert e.value.code == want, (e.value.code, kw)


def test_layer_norm():
    run = lambda T=1, x=A, gain=A, y=A, shape=None, **kw: layer.LayerNorm(**{**dict(hidden=256), **(shape or {})}).run(x, gain, T, y=y, **kw)
    refused(INVALID, run, T=-1)
    for name in ("x", "gain", "y"):
        refused(INVALID, run, **{name: None})
    for name in ("x", "gain", "y", "residual", "bias", "sum"):
        refused(ALIGN, run, **{name: A + 8})
    for bad in (dict(hidden=0), dict(hidden=65544), dict(in_dtype="fp8"), dict(out_dtype="fp8"), dict(gain_dtype=9), dict(epsilon=-1.0),
                dict(epsilon=float("nan"))):
        refused(INVALID, run, shape=bad)
    refused(ALIGN, run, shape=dict(hidden=252))
    shape = layer._NormShape(256, 1, 1, 1, 128, 1e-5)                   # codes are the other norm's
    assert layer.load().eep_layer_norm(ctypes.byref(shape), A, None, A, None, None, A, 1, None) == INVALID
    assert layer.load().eep_layer_norm(None, A, None, A, None, None, A, 1, None) == INVALID
    layer.LayerNorm(hidden=256).run(None, None, 0, y=None)              # of nothing: nothing


def test_norm_grad_shapes():
    make = lambda **kw: layer.NormGrad(**{**dict(hidden=256), **kw})
    for bad in (dict(hidden=0), dict(hidden=65544), dict(in_dtype="fp8"), dict(out_dtype="fp8"), dict(gain_dtype="fp8"), dict(epsilon=-1.0),
                dict(epsilon=float("nan"))):
        refused(INVALID, make, **bad)
    refused(ALIGN, make, hidden=252)
    lib, h = layer.load(), ctypes.c_void_p()
    assert lib.eep_norm_grad_create(None, ctypes.byref(h)) == INVALID
    assert lib.eep_norm_grad_create(ctypes.byref(_backward._NormGradConfig(256, 1, 1, 1, 0, 1e-6)), None) == INVALID
    assert lib.eep_norm_grad_create(ctypes.byref(_backward._NormGradConfig(256, 1, 1, 1, 2, 1e-6)), ctypes.byref(h)) == INVALID and not h.value
    assert lib.eep_norm_grad_destroy(None) == binding.OK
    assert lib.eep_norm_grad_run(None, A, A, A, None, A, None, None, 0, 1, None) == INVALID


def test_product_grad_shapes():
    good = dict(num_slots=4, in_features=256, out_features=128, max_rows=16)
    make = lambda **kw: layer.ExpertProductGrad(**{**good, **kw})
    for bad in (dict(num_slots=0), dict(num_slots=65537), dict(in_features=0), dict(out_features=0), dict(max_rows=-1),
                dict(max_rows=(1 << 30) + 1), dict(in_features=(1 << 21) + 8), dict(out_features=(1 << 21) + 8), dict(dtype="fp8"),
                dict(grad_w_dtype="fp8"), dict(slot_stride=256 * 128 * 2 - 16), dict(grad_stride=256 * 128 * 2 - 16), dict(slot_stride=-16),
                dict(gate=True, slot_stride=256 * 128 * 2)):
        refused(INVALID, make, **bad)
    for bad in (dict(in_features=252), dict(out_features=124), dict(dtype="f32", in_features=254), dict(dtype="f32", in_features=252),
                dict(dtype="f32", grad_w_dtype="f32", out_features=126), dict(slot_stride=256 * 128 * 2 + 8),
                dict(grad_stride=256 * 128 * 2 + 8)):
        refused(ALIGN, make, **bad)
    lib, h = layer.load(), ctypes.c_void_p()
    assert lib.eep_product_grad_create(None, ctypes.byref(h)) == INVALID
    assert lib.eep_product_grad_create(ctypes.byref(_backward._ProductGradConfig()), None) == INVALID
    bad = _backward._ProductGradConfig(4, 256, 128, 1, 1, 2, 16, 0, 0)      # no such gate
    assert lib.eep_product_grad_create(ctypes.byref(bad), ctypes.byref(h)) == INVALID and not h.value
    assert lib.eep_product_grad_destroy(None) == binding.OK
    assert lib.eep_product_grad_run(None, A, None, A, None, None, None, None, A, 0, 1, None) == INVALID


def test_route_grad():
    def run(T=1, idx=A, w=A, gw=A, out=A, logits=None, **kw):
        layer.Router(**{**dict(num_logical=64, topk=8), **kw}).grad(idx, w, gw, out, T, logits=logits)
    refused(INVALID, run, T=-1)
    for name in ("idx", "w", "gw", "out"):
        refused(INVALID, run, **{name: None})
        refused(ALIGN, run, **{name: A + 2})
    refused(INVALID, run, logits=A)                                     # only for over_all
    refused(INVALID, run, over_all=True)
    refused(ALIGN, run, over_all=True, logits=A + 2)
    refused(ALIGN, run, over_all=True, logits=A + 1, in_dtype="bf16")
    for bad in (dict(topk=0), dict(topk=33), dict(topk=65), dict(num_logical=4, topk=5), dict(num_logical=4097), dict(in_dtype="fp8")):
        refused(INVALID, run, **bad)
    run(T=0, idx=None)


def test_context_calls_without_a_context():
    lib = binding.load()
    assert lib.eep_combine_grad(None, A, A, A, A, A, 1, None) == INVALID
    assert lib.eep_dispatch_grad(None, A, A, 1, None) == INVALID


def test_tensors_too_small_are_refused_before_the_call():
    norm = layer.LayerNorm(hidden=64)
    x, short = torch.zeros((2, 64), dtype=torch.bfloat16), torch.zeros((1, 64), dtype=torch.bfloat16)
    for kw in (dict(y=short), dict(y=x, sum=short), dict(y=x, residual=short), dict(y=x, bias=short[0, :32])):
        with pytest.raises(ValueError, match=next(k for k in reversed(kw))):
            norm.run(x, x[0], 2, **kw)
    router = layer.Router(num_logical=64, topk=2)
    idx, w, out = torch.zeros((2, 2), dtype=torch.int32), torch.zeros((2, 2)), torch.zeros((2, 64))
    with pytest.raises(ValueError, match="grad_logits"):
        router.grad(idx, w, w, out[:1], 2)
    with pytest.raises(ValueError, match="grad_w"):
        router.grad(idx, w, w[:1], out, 2)
    with pytest.raises(ValueError, match="contiguous"):
        router.grad(idx, w, torch.zeros((2, 4))[:, ::2], out, 2)


def test_calls_state_their_entry_points_arguments():
    """The kinds of a call are as many as the entry point takes, pointers where it takes pointers."""
    import inspect
    import re
    lib = layer.load()
    calls = re.findall(r'\["(eep_[a-z_]+)"\],\s*"([hpis]+)"', inspect.getsource(_backward))
    assert sorted(n for n, _ in calls) == ["eep_layer_norm", "eep_norm_grad_run", "eep_product_grad_run", "eep_route_grad"]
    calls += list(binding.GRAD_KINDS.items())
    for name, kinds in calls:
        types = getattr(lib, name).argtypes
        assert len(types) == len(kinds), name
        for t, kind in zip(types, kinds):
            assert (t is ctypes.c_int32) == (kind == "i"), name
