"""What the layer's entry points refuse, before anything touches a GPU."""
import ctypes

import pytest
import torch

from paper_2605_10670_amd import binding, layer

A = 1 << 20     # an aligned address that is never read
INVALID, ALIGN = binding.ERR_INVALID_ARG, binding.ERR_ALIGN


def refused(want, call, /, **kw):
    with pytest.raises(binding.EepError) as e:
        call(**kw)
    assert e.value.code == want, (e.value.code, kw)


def test_norm():
    run = lambda T=1, x=A, gain=A, shape=None, **kw: layer.Norm(**{**dict(hidden=256, scale_group=128), **(shape or {})}).run(
        x, gain, T, **{**dict(y=A), **kw})
    refused(INVALID, run, T=-1)
    refused(INVALID, run, x=None)
    refused(INVALID, run, gain=None)
    refused(INVALID, run, y=None)                                       # nothing to write
    refused(INVALID, run, code=A)                                       # codes without scales
    refused(INVALID, run, code_scale=A)
    refused(INVALID, run, code=A, code_scale=A, shape=dict(scale_group=0))
    for group in (8, 24, 96, 1024, -128):
        refused(INVALID, run, shape=dict(hidden=24 * 256, scale_group=group))
    refused(INVALID, run, shape=dict(hidden=192))                       # groups that are not whole
    refused(INVALID, run, shape=dict(hidden=0, scale_group=0))
    refused(INVALID, run, shape=dict(hidden=65544, scale_group=0))
    refused(ALIGN, run, shape=dict(hidden=252, scale_group=0))
    refused(INVALID, run, shape=dict(in_dtype="fp8"))
    refused(INVALID, run, shape=dict(out_dtype="fp8"))
    refused(INVALID, run, shape=dict(gain_dtype=7))
    refused(INVALID, run, shape=dict(epsilon=-1.0))
    refused(INVALID, run, shape=dict(epsilon=float("nan")))
    for name in ("x", "gain", "residual", "sum", "y"):
        refused(ALIGN, run, **{name: A + 8})
    refused(ALIGN, run, code=A + 8, code_scale=A)
    refused(ALIGN, run, code=A, code_scale=A + 2)


def test_route():
    run = lambda T=1, logits=A, idx=A, w=A, **kw: layer.Router(**{**dict(num_logical=64, topk=8), **kw}).run(logits, idx, w, T)
    refused(INVALID, run, T=-1)
    for name in ("logits", "idx", "w"):
        refused(INVALID, run, **{name: None})
        refused(ALIGN, run, **{name: A + 2})
    refused(ALIGN, run, logits=A + 1, in_dtype="bf16")
    for bad in (dict(topk=0), dict(topk=33), dict(topk=65, num_logical=64), dict(num_logical=4, topk=5), dict(num_logical=0, topk=1),
                dict(num_logical=4097), dict(in_dtype="fp8"), dict(in_dtype=-1)):
        refused(INVALID, run, **bad)


GOOD = dict(num_slots=4, in_features=256, out_features=128, max_rows=16)


def test_product_shapes():
    make = lambda **kw: layer.ExpertProduct(**{**GOOD, **kw})
    for bad in (dict(num_slots=0), dict(num_slots=65537), dict(in_features=0), dict(out_features=0), dict(max_rows=-1),
                dict(max_rows=(1 << 30) + 1), dict(in_features=(1 << 24) + 8), dict(y_dtype="fp8"),
                dict(x_dtype="fp8", in_features=192), dict(x_dtype="fp8", gate=True, out_features=192),
                dict(gate=True, y_dtype="fp8", out_features=144),
                dict(slot_stride=256 * 128 * 2 - 16), dict(slot_stride=-16), dict(x_dtype="fp8", scale_stride=4)):
        refused(INVALID, make, **bad)
    for bad in (dict(in_features=252), dict(out_features=124), dict(in_features=254, x_dtype="f32"), dict(out_features=126, y_dtype="f32"),
                dict(slot_stride=256 * 128 * 2 + 8), dict(x_dtype="fp8", scale_stride=4 * 1024 + 2)):
        refused(ALIGN, make, **bad)
    lib, h = layer.load(), ctypes.c_void_p()
    assert lib.eep_product_create(None, ctypes.byref(h)) == INVALID
    assert lib.eep_product_create(ctypes.byref(layer._ProductConfig()), None) == INVALID
    assert lib.eep_product_destroy(None) == binding.OK
    bad = layer._ProductConfig(4, 256, 128, 1, 1, 2, 16, 0, 0)          # no such gate
    assert lib.eep_product_create(ctypes.byref(bad), ctypes.byref(h)) == INVALID and not h.value


def test_sizes_of_tensors():
    n = layer.Norm(hidden=256)
    t = torch.zeros((2, 256), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="residual"):
        n.run(A, A, 3, residual=t, y=A)
    with pytest.raises(ValueError, match="gain"):
        n.run(A, t[0, :128], 1, y=A)
    with pytest.raises(ValueError, match="contiguous"):
        n.run(torch.zeros((256, 256), dtype=torch.bfloat16).t(), A, 1, y=A)
    with pytest.raises(ValueError, match="topk_w"):
        layer.Router(num_logical=8, topk=4).run(A, A, torch.zeros(4), 2)


def test_every_entry_point_is_declared_with_its_arguments():
    """The kinds that the calls state are as many as the entry points take, integers where they take integers."""
    import inspect
    import re
    lib = layer.load()
    calls = re.findall(r'\["(eep_[a-z_]+)"\],\s*"([hpis]+)"', inspect.getsource(layer))
    assert sorted(name for name, _ in calls) == ["eep_expert_product", "eep_residual_norm", "eep_route"]
    for name, kinds in calls:
        want = ["i" if a is ctypes.c_int32 else "p" for a in getattr(lib, name).argtypes]
        assert [{"h": "p", "s": "p"}.get(c, c) for c in kinds] == want, name
