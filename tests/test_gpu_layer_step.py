"""The layer's operators together, as the example uses them: one captured step, replayed before and after a failed rank's
repair, every stage against its definition on what the stage before left."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import layer_util as lu

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def load_example():
    spec = importlib.util.spec_from_file_location("moe_layer", os.path.join(ROOT, "examples", "moe_layer.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def check_stages(m, lay):
    T, k = m.T, m.k
    # norm
    h = m.x.cpu().float() + m.residual.cpu().float()
    assert torch.equal(m.sum.cpu(), h.bfloat16())
    v = h.double() * m.gain.cpu().double() / (h.double().pow(2).mean(dim=1, keepdim=True) + 1e-6).sqrt()
    err = v.abs() * 64 * 2.0 ** -24 + 2.0 ** -149
    lu.check_rounded(m.y.cpu(), v, err)
    lu.check_codes(m.code.cpu(), m.code_scale.cpu(), v, err)
    # logits and choice
    y, w = m.y.cpu().double(), m.router_w.cpu().double()
    lu.check_rounded(m.logits.cpu(), y @ w.t(), (y.abs() @ w.abs().t()) * (m.H + 8) * 2.0 ** -23)
    order = np.argsort(-m.logits.cpu().double().numpy(), axis=1, kind="stable")[:, :k]
    assert np.array_equal(m.topk_idx.cpu().numpy(), order)
    # dispatch moves codes and scales
    row = torch.from_numpy(lay["row_of"]).long()
    assert (row >= 0).all()
    token = torch.arange(T).repeat_interleave(k)
    flat = row.flatten()
    assert torch.equal(m.recv.cpu().view(torch.uint8)[flat], m.code.cpu().view(torch.uint8)[token])
    assert torch.equal(m.recv_scale.cpu()[flat], m.code_scale.cpu()[token])
    # the experts, by slot: the weights of whatever expert the placement says
    off = torch.from_numpy(lay["offset"])
    held = [m.experts[e] for e in m.p2l]
    for x, scale, first, out, out_scale, yt, N in ((m.recv, m.recv_scale, 0, m.act, m.act_scale, "fp8", m.I),
                                                   (m.act, m.act_scale, 2, m.expert_y, None, "bf16", m.H)):
        c = dict(P=m.P, rows=T * k, K=x.shape[1], N=N, xt="fp8", gate=first == 0, offset=off)
        wd = torch.stack([lu.dequantise(s[first], s[first + 1], 128) for s in held])
        lu.exact(c, lu.dequantise(x.cpu(), scale.cpu(), 1), wd)
        n = c["routed"]
        want, e = (t[:n] for t in lu.result(c, yt))
        if yt == "fp8":
            lu.check_codes(out.cpu()[:n], out_scale.cpu()[:n], want, e)
        else:
            lu.check_rounded(out.cpu()[:n], want, e + 2.0 ** -126)
    # combine
    rows = m.expert_y.cpu().double()[row]
    want = (rows * m.topk_w.cpu().double()[:, :, None]).sum(dim=1)
    lu.check_rounded(m.out.cpu(), want, (rows.abs() * m.topk_w.cpu().double()[:, :, None]).sum(dim=1) * (k + 1) * 2.0 ** -23)


def test_captured_layer_before_and_after_a_repair():
    example = load_example()
    m = example.MoeLayer(T=128, H=1024, inner=512, E=16, topk=2, R=4, primary=4, redundant=2, seed=3)
    stream = torch.cuda.Stream()
    m.step(stream)
    stream.synchronize()
    m.ctx.graph_begin(stream)
    m.step(stream)
    graph = m.ctx.graph_end(stream)
    g = torch.Generator(device="cuda").manual_seed(4)
    for replay in range(4):
        if replay == 2:
            m.fail(1, stream)
        m.x.copy_(torch.randn((m.T, m.H), generator=g, device="cuda"))
        m.residual.copy_(2 * torch.randn((m.T, m.H), generator=g, device="cuda"))
        torch.cuda.synchronize()
        graph.launch(stream)
        stream.synchronize()
        lay = m.ctx.read_layout(m.T)
        assert lay["N"] == m.T * m.k and (replay < 2 or lay["rank_count"][1] == 0)
        check_stages(m, lay)
    assert graph.counters()["instantiations"] == 1
    graph.destroy()
    m.destroy()
