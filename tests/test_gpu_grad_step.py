"""The layer's forward and backward pass together, as the example uses them: captured, replayed before and after a failed rank's repair;
every stage against its definition on what the stages around it left, and in fp32 the whole against 64-bit differentiation."""
import importlib.util
import os

import pytest
import torch

import grad_util as gr

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def load_example():
    spec = importlib.util.spec_from_file_location("moe_finetune", os.path.join(ROOT, "examples", "moe_finetune.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def check_stages(m, lay):
    c = lambda t: t.cpu()
    T, k, I, off = m.T, m.k, m.I, lay["offset"].tolist()
    row = torch.from_numpy(lay["row_of"]).long()
    assert (row >= 0).all()
    flat, token = row.flatten(), torch.arange(T).repeat_interleave(k)
    # combine
    w, go, y = c(m.topk_w), c(m.grad_out), c(m.expert_y)
    want = torch.empty((T * k, m.H), dtype=torch.float64)
    want[flat] = w.flatten().double()[:, None] * go.double()[token]
    gr.check("grad_expert_y", m.grad_expert_y, want, want.abs() * gr.U + 2.0 ** -149)
    terms = y.double()[row] * go.double()[:, None]
    gr.check("grad_topk_w", m.grad_topk_w, terms.sum(dim=2), terms.abs().sum(dim=2) * (m.H + 8) * gr.U + 2.0 ** -149)
    # experts
    up, down = c(m.weights)[:, :m.up_size].view(m.P, 2 * I, m.H), c(m.weights)[:, m.up_size:].view(m.P, m.H, I)
    grads = c(m.grad_weights)
    want = gr.product_grads(c(m.grad_expert_y), c(m.act), down, off)
    gr.check("grad_act", m.grad_act, *want["grad_x"])
    gr.check("grad_down", grads[:, m.up_size:].view(m.P, m.H, I), *want["grad_w"])
    gr.check("grad_sums", m.grad_sums, *gr.gate_grad(c(m.grad_act), c(m.sums)))
    want = gr.product_grads(c(m.grad_sums), c(m.recv), up, off)
    gr.check("grad_recv", m.grad_recv, *want["grad_x"])
    gr.check("grad_up", grads[:, :m.up_size].view(m.P, 2 * I, m.H), *want["grad_w"])
    # dispatch and the router
    each = c(m.grad_recv).double()[row]
    gr.check("grad_y_routed", m.grad_y_routed, each.sum(dim=1), each.abs().sum(dim=1) * k * gr.U)
    gr.check("grad_logits", m.grad_logits, *gr.route_grad(c(m.topk_idx), w, c(m.grad_topk_w), m.E))
    want = gr.product_grads(c(m.grad_logits), c(m.y), c(m.router_w)[None], [0, T])
    gr.check("grad_router", m.grad_router[None], *want["grad_w"])
    # the norm
    want = gr.norm_grad(c(m.sum), c(m.gain), c(m.grad_y), c(m.grad_sum), False, 1e-6)
    gr.check("grad_x", m.grad_x, *want["grad_h"])
    gr.check("grad_gain", m.grad_gain, *want["grad_gain"])


def inputs(m, g):
    for t in (m.x, m.residual, m.grad_sum):
        t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
    m.grad_out.copy_(torch.randn(m.grad_out.shape, generator=g, device="cuda") * 1e-2)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_captured_step_before_and_after_a_repair(dtype):
    m = load_example().TrainedLayer(T=96, H=264, inner=136, E=8, topk=2, R=4, primary=2, redundant=1, dtype=dtype, seed=3)
    stream = torch.cuda.Stream()
    for step in (m.forward, m.backward):
        step(stream)
    stream.synchronize()
    m.ctx.graph_begin(stream)
    m.forward(stream)
    m.backward(stream)
    graph = m.ctx.graph_end(stream)
    g = torch.Generator(device="cuda").manual_seed(4)
    for replay in range(4):
        if replay == 2:
            m.fail(1, stream)
        inputs(m, g)
        graph.launch(stream)
        stream.synchronize()
        check_stages(m, m.ctx.read_layout(m.T, stream))
        m.descend(1e-3)
        torch.cuda.synchronize()
    graph.destroy()
    m.destroy()


def test_the_whole_layer_against_64_bit_differentiation():
    """In fp32.  A dozen stages, each off by at most its terms (264 at most) times 2^-24 in the 2-norm: 2e-4 in all, of gradients that
    no stage makes much smaller; 1e-3 is asked for.  The choice of experts is the layer's own."""
    m = load_example().TrainedLayer(T=64, H=264, inner=136, E=8, topk=2, R=4, primary=2, redundant=1, dtype="f32", seed=5)
    g = torch.Generator(device="cuda").manual_seed(6)
    inputs(m, g)
    m.forward()
    m.backward()
    torch.cuda.synchronize()
    leaf = lambda t: t.cpu().double().requires_grad_()
    held = {int(e): p for p, e in enumerate(m.p2l) if e >= 0}
    x, gain, router_w = leaf(m.x), leaf(m.gain), leaf(m.router_w)
    experts = leaf(m.weights[torch.tensor([held[e] for e in range(m.E)])])
    h = x + m.residual.cpu().double()
    y = h / (h.pow(2).mean(dim=1, keepdim=True) + 1e-6).sqrt() * gain
    idx = m.topk_idx.cpu().long()
    w = torch.softmax((y @ router_w.t()).gather(1, idx), dim=1)
    out = torch.zeros((m.T, m.H), dtype=torch.float64)
    for e in range(m.E):
        t, j = (idx == e).nonzero(as_tuple=True)
        both = y[t] @ experts[e, :m.up_size].view(2 * m.I, m.H).t()
        act = torch.nn.functional.silu(both[:, :m.I]) * both[:, m.I:]
        out = out.index_add(0, t, (act @ experts[e, m.up_size:].view(m.H, m.I).t()) * w[t, j, None])
    ((out * m.grad_out.cpu().double()).sum() + (h * m.grad_sum.cpu().double()).sum()).backward()
    off = lambda a, b: float((a.cpu().double() - b).norm() / b.norm())
    assert off(m.out, out.detach()) < 1e-3
    for name, got, want in (("x", m.grad_x, x), ("gain", m.grad_gain, gain), ("router", m.grad_router, router_w),
                            ("experts", m.expert_grads(), experts)):
        assert off(got, want.grad) < 1e-3, name
    m.destroy()


def test_example_runs(capsys):
    load_example().main()
    assert capsys.readouterr().out.count("step") == 8
