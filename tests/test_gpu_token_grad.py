"""The gradients of combine and dispatch against their definitions, by the layout that the forward pass left."""
import numpy as np
import pytest
import torch

from paper_2605_10670_amd import binding, synth

import grad_util as gr
import layer_util as lu

pytestmark = pytest.mark.gpu
TORCH_OF = gr.TORCH_OF


def context(T, R, primary, redundant, k, H, y="bf16", out="bf16", failed=(), **kw):
    E = R * primary
    ctx = binding.Context(num_ranks=R, slots_per_rank=primary + redundant, primary_slots=primary, num_logical=E, max_tokens=T, topk=k,
                          hidden=H, x_dtype=y, y_dtype=y, out_dtype=out, strict_coverage=False, **kw)
    ctx.update_placement(synth.preferred_placement(R, primary, redundant))
    ctx.set_membership(synth.active_mask(R, failed))
    return ctx, E


def indices(g, T, E, k, odd=True):
    idx = torch.rand((T, E), generator=g).argsort(dim=1)[:, :k].to(torch.int32)
    if odd and T > 2 and k > 1:
        idx[1, 1] = idx[1, 0]     # twice the same: the second has no row
        idx[2, 0] = -1            # masked
        idx[T - 1] = -1           # a token without any row
    return idx


def data(g, T, k, H, y, out):
    return (lu.randn(g, T * k, H).to(TORCH_OF[y]), torch.rand((T, k), generator=g), lu.randn(g, T, H).to(TORCH_OF[out]))


def want_combine(row, y, w, grad_out):
    """((grad_y, error), (grad_w, error)), rows without a pair left SENTINEL."""
    T, k = row.shape
    go = grad_out.double()
    grad_y = torch.full(y.shape, gr.SENTINEL, dtype=torch.float64)
    grad_w, e_w = torch.zeros((T, k), dtype=torch.float64), torch.zeros((T, k), dtype=torch.float64)
    for j in range(k):
        t = (row[:, j] >= 0).nonzero().flatten()
        r = row[t, j]
        grad_y[r] = w[t, j].double()[:, None] * go[t]
        terms = y[r].double() * go[t]
        grad_w[t, j] = terms.sum(dim=1)
        e_w[t, j] = terms.abs().sum(dim=1) * (y.shape[1] + 8) * gr.U
    return (grad_y, grad_y.abs() * gr.U + 2.0 ** -149), (grad_w, e_w + 2.0 ** -149)


SHAPES = [  # T, R, primary, redundant, k, H
    (4, 4, 2, 1, 2, 8), (32, 32, 8, 1, 8, 7168), (24, 24, 4, 1, 6, 2880), (1, 1, 4, 0, 1, 64), (600, 4, 4, 2, 3, 520), (512, 4, 4, 0, 1, 512),
    (528, 4, 8, 1, 32, 72), (640, 16, 8, 1, 10, 1032), (6, 2, 8, 1, 5, 16384), (1024, 4, 2, 2, 2, 256)]


@pytest.mark.parametrize("T,R,primary,redundant,k,H", SHAPES)
@pytest.mark.parametrize("y,out", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16"), ("f32", "f32")])
def test_gradients(T, R, primary, redundant, k, H, y, out):
    g = lu.gen(T + H)
    ctx, E = context(T, R, primary, redundant, k, H, y, out, failed=(1,) if R > 2 else ())
    idx = indices(g, T, E, k)
    rows, w, grad_out = data(g, T, k, H, y, out)
    idx_d, rows_d, w_d, go_d = idx.cuda(), rows.cuda(), w.cuda(), grad_out.cuda()
    ctx.dispatch_layout(idx_d, T)
    # (the layout is what counts, not what has become of the mask since)
    if R > 2:
        ctx.set_membership(synth.active_mask(R, (0,)))
    row = torch.from_numpy(ctx.read_layout(T)["row_of"]).long()
    grad_y = torch.full((T * k, H), gr.SENTINEL, device="cuda").to(TORCH_OF[y])
    grad_w = torch.full((T, k), gr.SENTINEL, device="cuda")
    ctx.combine_grad(rows_d, w_d, go_d, grad_y, grad_w, T)
    want_y, want_w = want_combine(row, rows, w, grad_out)
    gr.check("grad_y", grad_y, *want_y)
    gr.check("grad_w", grad_w, *want_w)
    # each alone, and grad_y in y's place
    alone_y, alone_w = torch.full_like(grad_y, gr.SENTINEL), torch.empty_like(grad_w)
    ctx.combine_grad(None, w_d, go_d, alone_y, None, T)
    ctx.combine_grad(rows_d, None, go_d, None, alone_w, T)
    assert torch.equal(alone_y, grad_y) and torch.equal(alone_w, grad_w)
    there = rows_d.clone()
    ctx.combine_grad(there, w_d, go_d, there, alone_w, T)
    n = int((row >= 0).sum())
    assert torch.equal(there[:n], grad_y[:n]) and torch.equal(there[n:], rows_d[n:]) and torch.equal(alone_w, grad_w)
    # dispatch: rows behind the last are anything
    grad_recv = rows.clone()
    grad_recv[n:] = float("nan")
    grad_x = torch.full((T, H), gr.SENTINEL, device="cuda").to(TORCH_OF[out])
    ctx.dispatch_grad(grad_recv.cuda(), grad_x, T)
    each = torch.where((row >= 0)[:, :, None], rows.double()[row.clamp(min=0)], 0.0)
    gr.check("grad_x", grad_x, each.sum(dim=1), each.abs().sum(dim=1) * k * gr.U)
    ctx.destroy()


def test_values_that_are_not_finite_stay_with_their_token():
    T, R, k, H = 8, 4, 2, 64
    g = lu.gen(1)
    ctx, E = context(T, R, 2, 0, k, H)
    idx = indices(g, T, E, k, odd=False).cuda()
    rows, w, grad_out = data(g, T, k, H, "bf16", "bf16")
    grad_out[3, 5] = float("inf")
    grad_out[4, 6] = float("nan")
    ctx.dispatch_layout(idx, T)
    row = torch.from_numpy(ctx.read_layout(T)["row_of"]).long()
    grad_y, grad_w = torch.empty((T * k, H), dtype=torch.bfloat16, device="cuda"), torch.empty((T, k), device="cuda")
    ctx.combine_grad(rows.cuda(), w.cuda(), grad_out.cuda(), grad_y, grad_w, T)
    finite_w = grad_w.cpu().isfinite().all(dim=1)
    assert finite_w.tolist() == [t not in (3, 4) for t in range(T)]
    bad = (~grad_y.cpu().float().isfinite()).any(dim=1).nonzero().flatten().tolist()
    assert sorted(bad) == sorted(row[3].tolist() + row[4].tolist())


@pytest.mark.parametrize("T", [64, 1024])
def test_rows_of_a_rank_that_was_dropped_within_the_step(T):
    """Failure detection strikes pairs from row_of after the experts have run: their rows took no part, and get zeros."""
    R, k, H, silent = 4, 2, 512, 2
    g = lu.gen(T)
    ctx, E = context(T, R, 4, 0, k, H)
    stream = torch.cuda.Stream()
    idx = indices(g, T, E, k).cuda()
    rows, w, grad_out = data(g, T, k, H, "bf16", "bf16")
    rows_d, w_d, go_d, out = rows.cuda(), w.cuda(), grad_out.cuda(), torch.empty((T, H), dtype=torch.bfloat16, device="cuda")
    grad_y = torch.full((T * k, H), gr.SENTINEL, device="cuda").bfloat16()
    grad_w, grad_x = torch.empty((T, k), device="cuda"), torch.empty((T, H), dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    ctx.set_detection(200_000)
    ctx.debug_withhold_signal([int(r == silent) for r in range(R)], stream)
    ctx.dispatch_layout(idx, T, stream)
    before = torch.from_numpy(ctx.read_layout(T, stream)["row_of"]).long()
    ctx.signal_experts_done(stream)
    ctx.combine(rows_d, w_d, out, T, stream)
    ctx.combine_grad(rows_d, w_d, go_d, grad_y, grad_w, T, stream)
    ctx.dispatch_grad(rows_d, grad_x, T, stream)
    stream.synchronize()
    assert ctx.read_failures(stream)[silent] == 1
    lay = ctx.read_layout(T, stream)
    row = torch.from_numpy(lay["row_of"]).long()
    struck = (before >= 0) & (row < 0)
    assert struck.any() and torch.equal(struck, (torch.from_numpy(lay["slot_of"]).long() // 4 == silent) & (before >= 0))
    want_y, want_w = want_combine(row, rows, w, grad_out)
    want_y[0][before[struck]] = 0.0
    gr.check("grad_y", grad_y, want_y[0], want_y[0].abs() * gr.U)
    gr.check("grad_w", grad_w, *want_w)
    each = torch.where((row >= 0)[:, :, None], rows.double()[row.clamp(min=0)], 0.0)
    gr.check("grad_x", grad_x, each.sum(dim=1), each.abs().sum(dim=1) * k * gr.U)


def test_fp8_payloads_have_gradients_of_the_rows_types():
    T, R, k, H = 16, 4, 2, 512
    g = lu.gen(2)
    ctx = binding.Context(num_ranks=R, slots_per_rank=2, primary_slots=2, num_logical=8, max_tokens=T, topk=k, hidden=H, x_dtype="fp8",
                          y_dtype="bf16", out_dtype="f32")
    ctx.update_placement(synth.preferred_placement(R, 2, 0))
    ctx.dispatch_layout(indices(g, T, 8, k).cuda(), T)
    row = torch.from_numpy(ctx.read_layout(T)["row_of"]).long()
    grad_recv = lu.randn(g, T * k, H).bfloat16()
    grad_x = torch.empty((T, H), device="cuda")
    ctx.dispatch_grad(grad_recv.cuda(), grad_x, T)
    each = torch.where((row >= 0)[:, :, None], grad_recv.double()[row.clamp(min=0)], 0.0)
    gr.check("grad_x", grad_x, each.sum(dim=1), each.abs().sum(dim=1) * k * gr.U)


def test_captured_step_replayed_with_other_routes():
    """Layout, combine and both gradients as one graph: replays see the routes, mask and values of their time."""
    T, R, k, H = 128, 4, 2, 256
    ctx, E = context(T, R, 4, 2, k, H)
    other, _ = context(T, R, 4, 2, k, H)
    g = lu.gen(9)
    idx = indices(g, T, E, k).cuda()
    rows, w, go = (t.cuda() for t in data(g, T, k, H, "bf16", "bf16"))
    out, grad_x = (torch.empty((T, H), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    grad_y, grad_w = torch.zeros((T * k, H), dtype=torch.bfloat16, device="cuda"), torch.empty((T, k), device="cuda")
    stream = torch.cuda.Stream()

    def step(c, st, out, grad_y, grad_w, grad_x):
        c.dispatch_layout(idx, T, st)
        c.combine(rows, w, out, T, st)
        c.combine_grad(rows, w, go, grad_y, grad_w, T, st)
        c.dispatch_grad(rows, grad_x, T, st)
    torch.cuda.synchronize()
    step(ctx, stream, out, grad_y, grad_w, grad_x)
    stream.synchronize()
    ctx.graph_begin(stream)
    step(ctx, stream, out, grad_y, grad_w, grad_x)
    graph = ctx.graph_end(stream)
    for replay in range(4):
        idx.copy_(indices(g, T, E, k))
        go.copy_(lu.randn(g, T, H))
        if replay == 2:
            for c in (ctx, other):
                c.set_membership(synth.active_mask(R, (1,)))
        grad_y.zero_()
        want = [torch.zeros_like(t) for t in (out, grad_y, grad_w, grad_x)]
        step(other, None, *want)
        torch.cuda.synchronize()
        graph.launch(stream)
        stream.synchronize()
        for a, b in zip((out, grad_y, grad_w, grad_x), want):
            assert torch.equal(a, b)
