"""Refusals of calls whose handle or context only exists on a GPU; nothing is launched."""
import pytest
import torch

from paper_2605_10670_amd import binding, layer

pytestmark = pytest.mark.gpu
INVALID, ALIGN, STATE = binding.ERR_INVALID_ARG, binding.ERR_ALIGN, binding.ERR_STATE
A = [(i + 1) << 28 for i in range(12)]   # aligned addresses far apart that are never read


def refused(want, call, /, *args, **kw):
    with pytest.raises(binding.EepError) as e:
        call(*args, **kw)
    assert e.value.code == want, (e.value.code, args, kw)


def test_norm_grad():
    plain, centred = layer.NormGrad(hidden=64), layer.NormGrad(hidden=64, centred=True)
    run = lambda grad=plain, h=A[0], gain=A[1], gy=A[2], T=2, **kw: grad.run(h, gain, gy, T, **kw)
    refused(INVALID, run)                                               # nothing wanted
    refused(INVALID, run, grad_bias=A[3])                               # a norm without one
    refused(INVALID, run, grad_gain=A[3], grad_sum=A[4])                # a gradient that goes nowhere
    refused(INVALID, run, T=-1, grad_h=A[3])
    for name in ("h", "gain", "gy"):
        refused(INVALID, run, grad_h=A[3], **{name: None})
        refused(ALIGN, run, grad_h=A[3], **{name: A[5] + 8})
    refused(ALIGN, run, grad_h=A[3] + 8)
    refused(ALIGN, run, grad_h=A[3], grad_sum=A[4] + 8)
    refused(ALIGN, run, grad_gain=A[3] + 2)
    refused(ALIGN, run, grad=centred, grad_bias=A[3] + 2)
    small = torch.empty(63, device="cuda")
    with pytest.raises(ValueError, match="grad_gain"):
        run(grad_gain=small)
    h = plain._h
    assert layer.load().eep_norm_grad_run(h, A[0], A[1], A[2], None, A[3], None, None, 2, 2, None) == INVALID   # accumulate is 0 or 1
    plain.destroy()
    plain.destroy()
    refused(INVALID, run, grad_h=A[3])                                  # a handle that is gone


def test_product_grad():
    make = lambda **kw: layer.ExpertProductGrad(**{**dict(num_slots=2, in_features=64, out_features=64, max_rows=16), **kw})
    one, gated = make(), make(gate=True)
    names = ("offset", "x", "w", "sums", "grad_sums", "grad_x", "grad_w")
    good = dict(zip(names, A[1:]))
    def run(grad=one, gy=A[0], rows=16, **kw):
        args = {**{n: good[n] for n in names if "sums" not in n or grad is gated}, **kw}
        grad.run(gy, rows, **args)
    refused(INVALID, run, rows=-1)
    refused(INVALID, run, rows=17)
    for name in ("gy", "x", "w", "offset"):
        refused(INVALID, run, **{name: None})
    refused(INVALID, run, grad_x=None, grad_w=None)
    refused(INVALID, run, sums=A[4])
    refused(INVALID, run, grad_sums=A[4])
    refused(INVALID, run, grad=gated, sums=None)
    refused(INVALID, run, grad=gated, grad_sums=None)
    for name in names:
        refused(ALIGN, run, grad=gated, **{name: A[9] + (2 if name == "offset" else 8)})
    # results over operands and over one another
    for result in ("grad_sums", "grad_x", "grad_w"):
        for other in ("x", "w", "sums"):
            refused(INVALID, run, grad=gated, **{result: good[other] + 16})
        refused(INVALID, run, grad=gated, **{result: A[0]})
    refused(INVALID, run, grad=gated, grad_x=good["grad_w"])
    refused(INVALID, run, grad=gated, grad_sums=good["grad_w"] + 64)
    with pytest.raises(ValueError, match="grad_w"):
        run(grad_w=torch.empty(16, device="cuda"))


def test_context_calls():
    ctx = binding.Context(num_ranks=2, slots_per_rank=2, primary_slots=2, num_logical=4, max_tokens=8, topk=2, hidden=64)
    combine = lambda y=A[0], w=A[1], go=A[2], gy=A[3], gw=A[4], T=4: ctx.combine_grad(y, w, go, gy, gw, T)
    refused(STATE, combine)                                             # before a layout
    refused(STATE, ctx.dispatch_grad, A[0], A[1], 4)
    ctx.update_placement([0, 1, 2, 3])
    ctx.dispatch_layout(torch.zeros((4, 2), dtype=torch.int32, device="cuda"), 4)
    refused(STATE, combine, T=2)
    refused(INVALID, combine, T=-1)
    refused(INVALID, combine, T=10)
    refused(INVALID, combine, go=None)
    refused(INVALID, combine, gy=None, gw=None)
    refused(INVALID, combine, y=None)
    refused(INVALID, combine, w=None)
    for name in ("y", "go", "gy"):
        refused(ALIGN, combine, **{name: A[5] + 8})
    for name in ("w", "gw"):
        refused(ALIGN, combine, **{name: A[5] + 2})
    refused(INVALID, ctx.dispatch_grad, None, A[1], 4)
    refused(INVALID, ctx.dispatch_grad, A[0], None, 4)
    refused(ALIGN, ctx.dispatch_grad, A[0] + 8, A[1], 4)
    refused(ALIGN, ctx.dispatch_grad, A[0], A[1] + 4, 4)
    torch.cuda.synchronize()
