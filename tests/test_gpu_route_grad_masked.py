"""Logits that are -infinity or NaN get 0 from the router's gradient, whatever comes in from behind."""
import math

import pytest
import torch

from paper_2605_10670_amd import layer

import grad_util as gr
import layer_util as lu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [5, 4100])
@pytest.mark.parametrize("E,k", [(64, 6), (256, 8), (510, 8)])
@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("over_all", [False, True])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_masked_logits_get_nothing_of_a_gradient_that_is_not_finite(T, E, k, x, over_all, bad):
    g = lu.gen(T + E + k)
    logits = lu.randn(g, T, E)
    logits[:, 1::5] = -math.inf
    logits[:, 3::25] = math.nan
    logits = logits.to(gr.TORCH_OF[x])
    router = layer.Router(num_logical=E, topk=k, in_dtype=x, over_all=over_all)
    idx, w = torch.empty((T, k), dtype=torch.int32, device="cuda"), torch.empty((T, k), device="cuda")
    router.run(logits.cuda(), idx, w, T)
    gw = lu.randn(g, T, k)
    gw[2, 1] = bad
    out = torch.full((T, E), gr.SENTINEL, device="cuda").to(logits.dtype)
    router.grad(idx, w, gw.cuda(), out, T, logits=logits.cuda() if over_all else None)
    got = out.cpu()
    masked = ~(logits > -math.inf)
    assert (got[masked] == 0).all()
    assert not got[2].isfinite().all()
    # the other tokens know nothing of it
    rest = torch.arange(T) != 2
    want, err = gr.route_grad(idx.cpu()[rest], w.cpu()[rest], gw[rest], E, logits[rest] if over_all else None)
    gr.check("grad_logits", got[rest], want, err)
