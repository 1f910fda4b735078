"""Forward and backward pass of one MoE layer as a captured graph: residual norm -> router -> layout and dispatch -> experts ->
combine and back, with plain gradient steps between replays, and a rank that fails and is repaired without capturing again.

    python examples/moe_finetune.py

The layer learns to reproduce another one of the same shape.  An expert's replicas get the sum of their slots' gradients, so
that they stay alike and a repair may copy any of them.
"""
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2605_10670_amd import binding, layer, synth  # noqa: E402


class TrainedLayer:
    """Shapes, buffers and calls of one layer; dtype "bf16" or "f32": of everything but the gain's and the weights' gradients."""

    def __init__(self, T, H, inner, E, topk, R, primary, redundant, dtype="bf16", seed=0):
        self.T, self.H, self.I, self.E, self.k, self.R, self.S = T, H, inner, E, topk, R, primary + redundant
        self.P, self.primary, self.dtype = R * self.S, primary, {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
        g = torch.Generator().manual_seed(seed)
        randn = lambda *shape: torch.randn(shape, generator=g)
        cast = lambda t: t.to(self.dtype).cuda()
        types = dict(x_dtype=dtype, y_dtype=dtype)
        self.ctx = binding.Context(num_ranks=R, slots_per_rank=self.S, primary_slots=primary, num_logical=E, max_tokens=T, topk=topk,
                                   hidden=H, out_dtype=dtype, **types)
        self.p2l = synth.preferred_placement(R, primary, redundant)
        self.ctx.update_placement(self.p2l)
        # a slot's weights one behind the other, as a repair moves them: the gate's and the other factor's rows, then the second product's
        self.gain, self.router_w = cast(1 + 0.1 * randn(H)), cast(randn(E, H) * H ** -0.5)
        self.up_size, self.down_size = 2 * inner * H, H * inner
        self.expert_size = self.up_size + self.down_size
        self.weights = cast(torch.cat([randn(E, self.up_size) * H ** -0.5, randn(E, self.down_size) * inner ** -0.5], dim=1)[np.maximum(self.p2l, 0)])
        self.backup = torch.empty((E, self.expert_size), dtype=self.dtype, pin_memory=True)

        size = self.weights.element_size()
        stride = dict(slot_stride=self.expert_size * size)
        rows = self.rows = T * topk
        product = lambda n_in, n_out, **kw: layer.ExpertProduct(num_slots=self.P, in_features=n_in, out_features=n_out, max_rows=rows,
                                                                **types, **stride, **kw)
        grad = lambda n_in, n_out, **kw: layer.ExpertProductGrad(num_slots=self.P, in_features=n_in, out_features=n_out, max_rows=rows,
                                                                 dtype=dtype, grad_w_dtype="f32", grad_stride=self.expert_size * 4,
                                                                 **stride, **kw)
        self.norm = layer.Norm(hidden=H, in_dtype=dtype, gain_dtype=dtype, out_dtype=dtype)
        self.norm_grad = layer.NormGrad(hidden=H, in_dtype=dtype, gain_dtype=dtype, out_dtype=dtype)
        self.router = layer.Router(num_logical=E, topk=topk, in_dtype=dtype)
        self.logits_of = layer.ExpertProduct(num_slots=1, in_features=H, out_features=E, max_rows=T, **types)
        self.logits_grad = layer.ExpertProductGrad(num_slots=1, in_features=H, out_features=E, max_rows=T, dtype=dtype, grad_w_dtype="f32")
        self.sums_of, self.up, self.down = product(H, 2 * inner), product(H, inner, gate=True), product(inner, H)
        self.up_grad, self.down_grad = grad(H, inner, gate=True), grad(inner, H)

        new = lambda *shape, dtype=self.dtype: torch.zeros(shape, dtype=dtype, device="cuda")
        f32 = torch.float32
        self.x, self.residual, self.sum, self.y, self.out = (new(T, H) for _ in range(5))
        self.logits, self.topk_idx, self.topk_w = new(T, E), new(T, topk, dtype=torch.int32), new(T, topk, dtype=f32)
        self.recv, self.sums, self.act, self.expert_y = new(rows, H), new(rows, 2 * inner), new(rows, inner), new(rows, H)
        # what comes in from behind the layer, and the gradients
        self.grad_out, self.grad_sum = new(T, H), new(T, H)
        self.grad_expert_y, self.grad_topk_w = new(rows, H), new(T, topk, dtype=f32)
        self.grad_act, self.grad_sums, self.grad_recv = new(rows, inner), new(rows, 2 * inner), new(rows, H)
        self.grad_logits, self.grad_y, self.grad_y_routed, self.grad_x = new(T, E), new(T, H), new(T, H), new(T, H)
        self.grad_gain, self.grad_router, self.grad_weights = new(H, dtype=f32), new(E, H, dtype=f32), new(self.P, self.expert_size, dtype=f32)

    def forward(self, stream=None):
        T, rows, weights = self.T, self.rows, self.weights.data_ptr()
        down = weights + self.up_size * self.weights.element_size()
        self.norm.run(self.x, self.gain, T, residual=self.residual, sum=self.sum, y=self.y, stream=stream)
        self.logits_of.run(self.y, self.router_w, self.logits, T, stream=stream)
        self.router.run(self.logits, self.topk_idx, self.topk_w, T, stream=stream)
        self.ctx.dispatch_layout(self.topk_idx, T, stream)
        self.ctx.dispatch(self.y, self.recv, T, stream=stream)
        offset = self.ctx.view_pointers()["offset"]
        self.up.run(self.recv, weights, self.act, rows, offset=offset, stream=stream)
        self.down.run(self.act, down, self.expert_y, rows, offset=offset, stream=stream)
        self.ctx.combine(self.expert_y, self.topk_w, self.out, T, stream)

    def backward(self, stream=None):
        """From grad_out, of `out`, and grad_sum, of `sum`: grad_x (of x and of residual alike) and the weights' gradients.
        The sums before the gate are made again."""
        T, rows, weights, grads = self.T, self.rows, self.weights.data_ptr(), self.grad_weights.data_ptr()
        down, grad_down = weights + self.up_size * self.weights.element_size(), grads + self.up_size * 4
        offset = self.ctx.view_pointers()["offset"]
        self.ctx.combine_grad(self.expert_y, self.topk_w, self.grad_out, self.grad_expert_y, self.grad_topk_w, T, stream)
        self.down_grad.run(self.grad_expert_y, rows, offset=offset, x=self.act, w=down, grad_x=self.grad_act, grad_w=grad_down, stream=stream)
        self.sums_of.run(self.recv, weights, self.sums, rows, offset=offset, stream=stream)
        self.up_grad.run(self.grad_act, rows, offset=offset, x=self.recv, w=weights, sums=self.sums, grad_sums=self.grad_sums,
                         grad_x=self.grad_recv, grad_w=grads, stream=stream)
        self.ctx.dispatch_grad(self.grad_recv, self.grad_y_routed, T, stream)
        self.router.grad(self.topk_idx, self.topk_w, self.grad_topk_w, self.grad_logits, T, stream=stream)
        self.logits_grad.run(self.grad_logits, T, x=self.y, w=self.router_w, grad_x=self.grad_y, grad_w=self.grad_router, stream=stream)
        with torch.cuda.stream(stream):   # (None: the current one)
            self.grad_y.add_(self.grad_y_routed)
        self.norm_grad.run(self.sum, self.gain, self.grad_y, T, grad_sum=self.grad_sum, grad_h=self.grad_x, grad_gain=self.grad_gain,
                           stream=stream)

    def expert_grads(self):
        """[E, expert_size]: every expert's gradient, of all its replicas."""
        held = torch.from_numpy(np.flatnonzero(self.p2l >= 0)).cuda()
        expert = torch.from_numpy(self.p2l[self.p2l >= 0]).long().cuda()
        total = torch.zeros((self.E, self.expert_size), device="cuda")
        return total.index_add_(0, expert, self.grad_weights[held])

    def descend(self, rate):
        grads = self.expert_grads()
        self.weights -= (rate * grads[torch.from_numpy(np.maximum(self.p2l, 0)).long().cuda()]).to(self.dtype)
        self.router_w -= (rate * self.grad_router).to(self.dtype)
        self.gain -= (rate * self.grad_gain).to(self.dtype)

    def fail(self, rank, stream=None):
        """The rank is gone: its experts move to redundant slots, from live copies or from a backup made just now."""
        first = torch.tensor([int(np.flatnonzero(self.p2l == e)[0]) for e in range(self.E)], device="cuda")
        self.backup.copy_(self.weights[first])
        torch.cuda.synchronize()
        dead = synth.active_mask(self.R, (rank,))
        plan = binding.plan_repair(self.p2l, dead, self.R, self.S, self.primary, self.E)
        self.ctx.apply_repair(self.weights, self.backup, self.expert_size * self.weights.element_size(), plan, stream)
        self.ctx.set_membership(dead, stream)
        self.p2l = plan["p2l"]

    def destroy(self):
        for p in (self.norm_grad, self.logits_of, self.logits_grad, self.sums_of, self.up, self.down, self.up_grad, self.down_grad):
            p.destroy()
        self.ctx.destroy()


def main():
    shape = dict(T=128, H=512, inner=256, E=16, topk=2, R=4, primary=4, redundant=2)
    m, teacher = TrainedLayer(**shape), TrainedLayer(**shape, seed=1)
    stream = torch.cuda.Stream()
    for step in (m.forward, m.backward):         # once before the capture
        step(stream)
    stream.synchronize()
    graphs = []
    for step in (m.forward, m.backward):
        m.ctx.graph_begin(stream)
        step(stream)
        graphs.append(m.ctx.graph_end(stream))
    g = torch.Generator(device="cuda").manual_seed(1)
    for number in range(40):
        if number == 20:
            m.fail(2, stream)
        for t in (m.x, m.residual):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
        teacher.x.copy_(m.x)
        teacher.residual.copy_(m.residual)
        teacher.forward()
        torch.cuda.synchronize()
        graphs[0].launch(stream)
        stream.synchronize()
        off = m.out.float() - teacher.out.float()
        m.grad_out.copy_(off * (2 / off.numel()))
        torch.cuda.synchronize()
        graphs[1].launch(stream)
        stream.synchronize()
        m.descend(rate=10.0)
        if number % 10 in (0, 9):
            rows = m.ctx.read("rank_count", m.R)
            print(f"step {number}: mean square off the teacher {float((off ** 2).mean()):.5f}, rows per rank {rows.tolist()}")
            assert rows.sum() == m.rows and (number < 20 or rows[2] == 0)
    for graph in graphs:
        graph.destroy()
    m.destroy()
    teacher.destroy()


if __name__ == "__main__":
    main()
