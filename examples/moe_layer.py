"""One MoE layer as a captured graph: residual norm -> router -> layout and dispatch -> experts -> combine, with a rank that
fails between replays and is repaired, weights included, without capturing again.

    python examples/moe_layer.py

Every slot's weights lie in one slot-major store, as a repair moves them: the first product's codes and scales, then the
second's.  Random weights, fp8 codes with a scale for 128 x 128.
"""
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2605_10670_amd import binding, layer, synth  # noqa: E402

BLOCK = 128


def quantise_blocks(w):
    """fp32 [N, K] -> e4m3 codes and a scale for each 128 x 128 of them (1 where all are zero)."""
    n, k = w.shape
    b = w.view(n // BLOCK, BLOCK, k // BLOCK, BLOCK)
    scale = b.abs().amax(dim=(1, 3)) / 448
    scale = torch.where(scale == 0, 1.0, scale)
    code = (b / scale[:, None, :, None]).clamp(-448, 448).to(torch.float8_e4m3fn)
    return code.view(n, k), scale


class MoeLayer:
    """Shapes, buffers and calls of one layer.  `experts` maps an expert to (up, up_scale, down, down_scale)."""

    def __init__(self, T, H, inner, E, topk, R, primary, redundant, seed=0):
        self.T, self.H, self.I, self.E, self.k, self.R, self.S = T, H, inner, E, topk, R, primary + redundant
        self.P, self.primary = R * self.S, primary
        g = torch.Generator().manual_seed(seed)
        self.ctx = binding.Context(num_ranks=R, slots_per_rank=self.S, primary_slots=primary, num_logical=E, max_tokens=T,
                                   topk=topk, hidden=H, x_dtype="fp8")
        self.gain = (1 + 0.1 * torch.randn(H, generator=g)).bfloat16().cuda()
        self.router_w = (torch.randn((E, H), generator=g) * H ** -0.5).bfloat16().cuda()
        # the backup: every expert's weights as one slot holds them, every part at a multiple of 16 bytes
        self.parts, at = {}, 0
        for name, size in (("up", 2 * inner * H), ("up_scale", 2 * inner // BLOCK * (H // BLOCK) * 4), ("down", H * inner),
                           ("down_scale", H // BLOCK * (inner // BLOCK) * 4)):
            self.parts[name] = (at, size)
            at += (size + 15) // 16 * 16
        self.slot_bytes = at
        backup = torch.zeros((E, at), dtype=torch.uint8)
        self.experts = []
        for e in range(E):
            up, up_scale = quantise_blocks(torch.randn((2 * inner, H), generator=g) * H ** -0.5)
            down, down_scale = quantise_blocks(torch.randn((H, inner), generator=g) * inner ** -0.5)
            self.experts.append((up, up_scale, down, down_scale))
            for part, t in zip(self.parts, self.experts[-1]):
                start, size = self.parts[part]
                backup[e, start:start + size] = t.contiguous().view(-1).view(torch.uint8)
        self.backup = backup.pin_memory()
        self.p2l = synth.preferred_placement(R, primary, redundant)
        self.weights = backup[torch.from_numpy(np.maximum(self.p2l, 0)).long()].cuda()
        self.ctx.update_placement(self.p2l)

        self.norm = layer.Norm(hidden=H, scale_group=BLOCK)
        self.logits_of = layer.ExpertProduct(num_slots=1, in_features=H, out_features=E, y_dtype="f32", max_rows=T)
        self.router = layer.Router(num_logical=E, topk=topk)
        stride = self.slot_bytes
        self.up = layer.ExpertProduct(num_slots=self.P, in_features=H, out_features=inner, x_dtype="fp8", y_dtype="fp8", gate=True,
                                      max_rows=T * topk, slot_stride=stride, scale_stride=stride)
        self.down = layer.ExpertProduct(num_slots=self.P, in_features=inner, out_features=H, x_dtype="fp8",
                                        max_rows=T * topk, slot_stride=stride, scale_stride=stride)
        rows = T * topk
        new = lambda *shape, dtype=torch.bfloat16: torch.zeros(shape, dtype=dtype, device="cuda")
        fp8, f32 = torch.float8_e4m3fn, torch.float32
        self.x, self.residual, self.sum, self.y = new(T, H), new(T, H), new(T, H), new(T, H)
        self.code, self.code_scale = new(T, H, dtype=fp8), new(T, H // BLOCK, dtype=f32)
        self.logits, self.topk_idx, self.topk_w = new(T, E, dtype=f32), new(T, topk, dtype=torch.int32), new(T, topk, dtype=f32)
        self.recv, self.recv_scale = new(rows, H, dtype=fp8), new(rows, H // BLOCK, dtype=f32)
        self.act, self.act_scale = new(rows, inner, dtype=fp8), new(rows, inner // BLOCK, dtype=f32)
        self.expert_y, self.out = new(rows, H), new(T, H)

    def part(self, name):
        return self.weights.data_ptr() + self.parts[name][0]

    def step(self, stream=None):
        T, rows = self.T, self.T * self.k
        self.norm.run(self.x, self.gain, T, residual=self.residual, sum=self.sum, y=self.y, code=self.code,
                      code_scale=self.code_scale, stream=stream)
        self.logits_of.run(self.y, self.router_w, self.logits, T, stream=stream)
        self.router.run(self.logits, self.topk_idx, self.topk_w, T, stream=stream)
        self.ctx.dispatch_layout(self.topk_idx, T, stream)
        self.ctx.dispatch(self.code, self.recv, T, self.code_scale, self.recv_scale, stream)
        offset = self.ctx.view_pointers()["offset"]
        self.up.run(self.recv, self.part("up"), self.act, rows, offset=offset, x_scale=self.recv_scale,
                    w_scale=self.part("up_scale"), y_scale=self.act_scale, stream=stream)
        self.down.run(self.act, self.part("down"), self.expert_y, rows, offset=offset, x_scale=self.act_scale,
                      w_scale=self.part("down_scale"), stream=stream)
        self.ctx.combine(self.expert_y, self.topk_w, self.out, T, stream)

    def fail(self, rank, stream=None):
        """The rank is gone: its experts move to redundant slots, from live copies or the backup."""
        dead = synth.active_mask(self.R, (rank,))
        plan = binding.plan_repair(self.p2l, dead, self.R, self.S, self.primary, self.E)
        self.ctx.apply_repair(self.weights, self.backup, self.slot_bytes, plan, stream)
        self.ctx.set_membership(dead, stream)
        self.p2l = plan["p2l"]

    def plain(self):
        """The layer in fp32 from the same codes, with nothing quantised in between."""
        idx, w = self.topk_idx.cpu().long(), self.topk_w.cpu()
        x = self.code.cpu().float() * self.code_scale.cpu().repeat_interleave(BLOCK, dim=1)
        out = torch.zeros((self.T, self.H))
        wide = lambda c, s: c.float() * s.repeat_interleave(BLOCK, 0).repeat_interleave(BLOCK, 1)
        for e, (up, up_scale, down, down_scale) in enumerate(self.experts):
            t, j = (idx == e).nonzero(as_tuple=True)
            both = x[t] @ wide(up, up_scale).t()
            act = torch.nn.functional.silu(both[:, :self.I]) * both[:, self.I:]
            out.index_add_(0, t, (act @ wide(down, down_scale).t()) * w[t, j, None])
        return out

    def destroy(self):
        for p in (self.logits_of, self.up, self.down):
            p.destroy()
        self.ctx.destroy()


def main():
    m = MoeLayer(T=128, H=1024, inner=512, E=16, topk=2, R=4, primary=4, redundant=2)
    stream = torch.cuda.Stream()
    m.step(stream)                              # once before the capture
    stream.synchronize()
    m.ctx.graph_begin(stream)
    m.step(stream)
    graph = m.ctx.graph_end(stream)
    g = torch.Generator(device="cuda").manual_seed(1)
    for number, event in enumerate(("all ranks live", "rank 2 fails", "the step after")):
        if event == "rank 2 fails":
            m.fail(2, stream)
        m.x.copy_(torch.randn((m.T, m.H), generator=g, device="cuda"))
        m.residual.copy_(torch.randn((m.T, m.H), generator=g, device="cuda"))
        torch.cuda.synchronize()
        graph.launch(stream)
        stream.synchronize()
        want, got = m.plain(), m.out.float().cpu()
        off = float((got - want).norm() / want.norm())
        rows = m.ctx.read("rank_count", m.R)
        print(f"step {number} ({event}): rows per rank {rows.tolist()}, {off:.4f} off the plain layer (8-bit steps between)")
        assert off < 0.05 and (event == "all ranks live" or rows[2] == 0)
    print("captured graph:", graph.counters())
    graph.destroy()
    m.destroy()


if __name__ == "__main__":
    main()
