"""The router's gradient against its definition in 64 bits, on what the router itself returned."""
import math

import pytest
import torch

from paper_2605_10670_amd import layer

import grad_util as gr
import layer_util as lu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (3, 8, 8), (5, 60, 6), (33, 256, 8), (7, 257, 1), (4, 510, 32), (2, 4096, 32), (9000, 64, 6),
                                   (4096, 256, 8), (4100, 252, 16), (4099, 512, 1), (4100, 100, 17), (4097, 4, 4), (2, 4093, 7)])
@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("over_all", [False, True])
def test_route_grad(T, E, k, x, over_all):
    g = lu.gen(T + E + k)
    logits = lu.randn(g, T, E)
    if E >= 8:
        logits[:, 1::5] = -math.inf
        logits[0, 2] = math.nan
    logits[-1, : E // 2 + 1] = -math.inf if T > 1 else 0.5   # fewer than k left, maybe
    logits = logits.to(gr.TORCH_OF[x]).cuda()
    router = layer.Router(num_logical=E, topk=k, in_dtype=x, over_all=over_all)
    idx, w = torch.empty((T, k), dtype=torch.int32, device="cuda"), torch.empty((T, k), device="cuda")
    router.run(logits, idx, w, T)
    gw = lu.randn(g, T, k)
    out = torch.full((T, E), gr.SENTINEL, device="cuda").to(logits.dtype)
    router.grad(idx, w, gw.cuda(), out, T, logits=logits if over_all else None)
    want, err = gr.route_grad(idx.cpu(), w.cpu(), gw, E, logits.cpu() if over_all else None)
    gr.check("grad_logits", out, want, err)
    if over_all:
        router.grad(idx, w, gw.cuda(), logits, T, logits=logits)   # in their place
        assert torch.equal(logits, out)


def test_rows_with_nothing_to_choose_and_odd_addresses():
    T, E, k = 3, 12, 4
    base = torch.full((T * E + 1,), -math.inf, device="cuda")
    logits = base[1:].view(T, E)                       # 4 bytes past an address of 16
    logits[1] = torch.arange(E, device="cuda").float()
    for over_all in (False, True):
        router = layer.Router(num_logical=E, topk=k, over_all=over_all)
        idx, w = torch.empty((T, k), dtype=torch.int32, device="cuda"), torch.empty((T, k), device="cuda")
        router.run(logits, idx, w, T)
        gw = lu.randn(lu.gen(1), T, k)
        out = torch.full((T * E + 1,), gr.SENTINEL, device="cuda")
        router.grad(idx, w, gw.cuda(), out[1:].view(T, E), T, logits=logits if over_all else None)
        assert out[0] == gr.SENTINEL
        got = out[1:].view(T, E)
        assert (got[0] == 0).all() and (got[2] == 0).all()
        want, err = gr.route_grad(idx.cpu(), w.cpu(), gw, E, logits.cpu() if over_all else None)
        gr.check("grad_logits", got, want, err)


@pytest.mark.parametrize("T", [1, 5000])
def test_an_index_twice_gets_both_and_one_out_of_range_nothing(T):
    idx = torch.tensor([[2, 2, 4]], dtype=torch.int32, device="cuda").repeat(T, 1)
    w, gw = torch.tensor([[0.25, 0.75, 0.0]], device="cuda").repeat(T, 1), torch.tensor([[1.0, -2.0, 3.0]], device="cuda").repeat(T, 1)
    out = torch.empty((T, 4), device="cuda")
    layer.Router(num_logical=4, topk=3).grad(idx, w, gw, out, T)
    inner = 0.25 - 1.5
    assert out.unique(dim=0).cpu().tolist() == [[0, 0, 0.25 * (1 - inner) + 0.75 * (-2 - inner), 0]]


def test_against_differences():
    E, k = 16, 4
    logits = lu.randn(lu.gen(4), 1, E).double()
    gw = lu.randn(lu.gen(6), 1, k)
    for over_all in (False, True):
        router = layer.Router(num_logical=E, topk=k, over_all=over_all)
        step = 2.0 ** -8
        probe = torch.cat([logits, logits + step * torch.eye(E), logits - step * torch.eye(E)]).float().cuda()
        n = probe.shape[0]
        idx, w = torch.empty((n, k), dtype=torch.int32, device="cuda"), torch.empty((n, k), device="cuda")
        router.run(probe, idx, w, n)
        # the weight of each expert that was chosen at the middle, whatever its rank now
        share = torch.zeros((n, E), dtype=torch.float64)
        share.scatter_(1, idx.cpu().long(), w.cpu().double())
        same = (share[:, idx[0].cpu().long()] > 0).all(dim=1)
        loss = (share[:, idx[0].cpu().long()] * gw.double()).sum(dim=1)
        slope = (loss[1:E + 1] - loss[E + 1:]) / (2 * step)
        out = torch.empty((1, E), device="cuda")
        router.grad(idx[:1], w[:1], gw.cuda(), out, 1, logits=probe[:1] if over_all else None)
        both = same[1:E + 1] & same[E + 1:]
        assert both.sum() >= E - 2
        # third derivatives of a softmax are below 1/4 of sum|gw|; weights are rounded to 2^-24
        bound = gw.abs().sum().double() * (step ** 2 / 24 + 2.0 ** -22 / step)
        assert ((slope - out[0].cpu().double()).abs()[both] < bound).all()
