"""The layer norm and the gradients of both norms against their definitions in 64 bits."""
import pytest
import torch

from paper_2605_10670_amd import layer

import grad_util as gr
import layer_util as lu

pytestmark = pytest.mark.gpu
TORCH_OF = gr.TORCH_OF


def rows_of(g, T, H, dtype, offset=0.1):
    large = 1 + 8 * (torch.rand(H, generator=g) < 0.05)
    return (lu.randn(g, T, H) * large + offset).to(TORCH_OF[dtype])


@pytest.mark.parametrize("T,H,x,y,gain", [(1, 8, "bf16", "bf16", "bf16"), (3, 520, "f32", "bf16", "f32"), (5, 2880, "bf16", "f32", "bf16"),
                                          (2, 7168, "bf16", "bf16", "f32"), (1100, 4104, "f32", "f32", "bf16"), (2, 16392, "bf16", "bf16", "bf16"),
                                          (2, 65536, "f32", "bf16", "bf16")])
@pytest.mark.parametrize("residual,bias", [(True, True), (False, False)])
def test_layer_norm(T, H, x, y, gain, residual, bias):
    g = lu.gen(T * H)
    xs, r = rows_of(g, T, H, x), rows_of(g, T, H, x, 3.0) if residual else None
    gn, b = (1 + 0.2 * lu.randn(g, H)).to(TORCH_OF[gain]), lu.randn(g, H).to(TORCH_OF[gain]) if bias else None
    dev = lambda t: None if t is None else t.cuda()
    s = torch.empty((T, H), dtype=TORCH_OF[x], device="cuda") if residual else None
    out = torch.empty((T, H), dtype=TORCH_OF[y], device="cuda")
    layer.LayerNorm(hidden=H, in_dtype=x, gain_dtype=gain, out_dtype=y).run(dev(xs), dev(gn), T, residual=dev(r), bias=dev(b), sum=s, y=out)
    h, want, err = gr.layer_norm(xs, r, gn, b, 1e-5)
    gr.check("y", out, want, err)
    if residual:
        assert torch.equal(s.cpu(), (xs.float() + r.float()).to(TORCH_OF[x]))


@pytest.mark.parametrize("T,H,x,y,gain,stream", [
    (1, 8, "bf16", "bf16", "bf16", True), (7, 520, "f32", "bf16", "f32", False), (64, 2880, "bf16", "f32", "bf16", True),
    (3, 4096, "bf16", "bf16", "f32", True), (700, 4104, "f32", "f32", "bf16", True), (1200, 1024, "bf16", "bf16", "bf16", True),
    (530, 7168, "bf16", "bf16", "bf16", False), (3, 16384, "f32", "f32", "bf16", True), (2, 16392, "bf16", "bf16", "bf16", True),
    (3, 65536, "bf16", "f32", "f32", True)])
@pytest.mark.parametrize("centred", [False, True])
def test_norm_grad(T, H, x, y, gain, stream, centred):
    g = lu.gen(T + H)
    h, gn = rows_of(g, T, H, x), (1 + 0.2 * lu.randn(g, H)).to(TORCH_OF[gain])
    gy = (lu.randn(g, T, H) * 1e-3).to(TORCH_OF[y])
    gs = (lu.randn(g, T, H) * 1e-3).to(TORCH_OF[x]) if stream else None
    want = gr.norm_grad(h, gn, gy, gs, centred, 1e-5)
    grad = layer.NormGrad(hidden=H, in_dtype=x, gain_dtype=gain, out_dtype=y, centred=centred, epsilon=1e-5)
    out = torch.empty((T, H), dtype=TORCH_OF[x], device="cuda")
    gg = torch.full((H,), gr.SENTINEL, device="cuda")
    gb = torch.full((H,), gr.SENTINEL, device="cuda") if centred else None
    dev = lambda t: None if t is None else t.cuda()
    hd, gnd, gyd, gsd = dev(h), dev(gn), dev(gy), dev(gs)
    grad.run(hd, gnd, gyd, T, grad_sum=gsd, grad_h=out, grad_gain=gg, grad_bias=gb)
    gr.check("grad_h", out, *want["grad_h"])
    gr.check("grad_gain", gg, *want["grad_gain"])
    if centred:
        gr.check("grad_bias", gb, *want["grad_bias"])
    # the same bits again; each result alone; added to what is there; in place
    again, first = torch.empty_like(out), gg.clone()
    grad.run(hd, gnd, gyd, T, grad_sum=gsd, grad_h=again)
    assert torch.equal(again, out)
    grad.run(hd, gnd, gyd, T, grad_gain=gg)
    assert torch.equal(gg, first)
    grad.run(hd, gnd, gyd, T, grad_gain=gg, accumulate=True)
    assert torch.equal(gg, first + first)
    if centred:
        alone = torch.empty_like(gb)
        grad.run(hd, gnd, gyd, T, grad_bias=alone)
        assert torch.equal(alone, gb)
    place = hd.clone()
    grad.run(place, gnd, gyd, T, grad_sum=gsd, grad_h=place)
    assert torch.equal(place, out)
    if stream:
        grad.run(hd, gnd, gyd, T, grad_sum=gsd, grad_h=gsd)
        assert torch.equal(gsd, out)
    if x == y and not stream:
        grad.run(hd, gnd, gyd, T, grad_h=gyd)
        assert torch.equal(gyd, out)
    grad.destroy()


def test_no_rows_give_zeros_or_leave_what_is_there():
    grad = layer.NormGrad(hidden=64, centred=True)
    gg, gb = torch.full((64,), 5.0, device="cuda"), torch.full((64,), 6.0, device="cuda")
    none = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    gain = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    grad.run(none, gain, none, 0, grad_gain=gg, grad_bias=gb, accumulate=True)
    assert (gg == 5).all() and (gb == 6).all()
    grad.run(none, gain, none, 0, grad_gain=gg, grad_bias=gb)
    assert (gg == 0).all() and (gb == 0).all()


def test_values_of_both_signs_at_the_end_of_fp32():
    """Sums of neighbours vanish, of others overflow; the squares do everywhere."""
    T, H = 2, 1024
    g = lu.gen(12)
    h = 3e38 * (1 - 2 * (torch.arange(H) % 2).float()).expand(T, H) * (0.5 + 0.5 * torch.rand((T, H), generator=g))
    h[1] = h[1].sort().values
    gain, gy = torch.ones(H), lu.randn(g, T, H)
    y = torch.empty((T, H), device="cuda")
    layer.LayerNorm(hidden=H, in_dtype="f32", gain_dtype="f32", out_dtype="f32").run(h.cuda(), gain.cuda(), T, y=y)
    _, want, err = gr.layer_norm(h, None, gain, None, 1e-5)
    gr.check("y", y, want, err)
    for centred in (False, True):
        gg = torch.empty(H, device="cuda")
        layer.NormGrad(hidden=H, in_dtype="f32", gain_dtype="f32", out_dtype="f32", centred=centred, epsilon=1e-5).run(
            h.cuda(), gain.cuda(), gy.cuda(), T, grad_gain=gg)
        gr.check("grad_gain", gg, *gr.norm_grad(h, gain, gy, None, centred, 1e-5)["grad_gain"])


def test_infinities_and_nans_stay_in_their_rows():
    T, H = 6, 2048
    g = lu.gen(13)
    h, gy = lu.randn(g, T, H), lu.randn(g, T, H)
    h[1, 3], h[2, 4], h[3, 5] = float("inf"), float("nan"), -float("inf")
    gy[4, 7] = float("nan")
    gain = torch.ones(H, device="cuda")
    y, out = torch.empty((T, H), device="cuda"), torch.empty((T, H), device="cuda")
    layer.LayerNorm(hidden=H, in_dtype="f32", gain_dtype="f32", out_dtype="f32").run(h.cuda(), gain, T, y=y)
    assert (~y.isfinite()).any(dim=1).tolist() == [False, True, True, True, False, False]
    for centred in (False, True):
        layer.NormGrad(hidden=H, in_dtype="f32", gain_dtype="f32", out_dtype="f32", centred=centred).run(h.cuda(), gain, gy.cuda(), T, grad_h=out)
        assert (~out.isfinite()).any(dim=1).tolist() == [False, True, True, True, True, False]


@pytest.mark.parametrize("scale", [1e-30, 1e25, 1e37])
@pytest.mark.parametrize("centred", [False, True])
def test_rows_whose_squares_leave_fp32(scale, centred):
    """The forward and backward of rows times a power of about `scale` are those of the rows, epsilon being nothing beside them."""
    T, H = 3, 1024
    g = lu.gen(11)
    h = (lu.randn(g, T, H) + 0.5) * scale
    gn, gy = 1 + 0.2 * lu.randn(g, H), lu.randn(g, T, H) * (1e-3 if scale < 1 else 1.0)
    eps = 0.0 if scale < 1 else 1e-5
    if scale < 1:
        gy = gy * 1e-20   # (so that the rows' gradients, which grow as the rows shrink, stay within fp32)
    grad = layer.NormGrad(hidden=H, in_dtype="f32", gain_dtype="f32", out_dtype="f32", centred=centred, epsilon=eps)
    out, gg = torch.empty((T, H), device="cuda"), torch.empty(H, device="cuda")
    grad.run(h.cuda(), gn.cuda(), gy.cuda(), T, grad_h=out, grad_gain=gg)
    want = gr.norm_grad(h, gn, gy, None, centred, eps)
    gr.check("grad_gain", gg, *want["grad_gain"])
    gr.check("grad_h", out, want["grad_h"][0], want["grad_h"][1] + 2.0 ** -140)
    if centred:
        y = torch.empty((T, H), device="cuda")
        layer.LayerNorm(hidden=H, in_dtype="f32", gain_dtype="f32", out_dtype="f32", epsilon=eps).run(h.cuda(), gn.cuda(), T, y=y)
        _, want, err = gr.layer_norm(h, None, gn, None, eps)
        gr.check("y", y, want, err)


@pytest.mark.parametrize("value", [3.0, 0.0, 2.0 ** 126])
def test_rows_of_one_value(value):
    """d is nothing: the layer norm is its bias, and the gradient that of a row of zeros."""
    T, H = 2, 512
    h = torch.full((T, H), value, device="cuda")
    gain, bias = torch.full((H,), 2.0, device="cuda"), torch.arange(H, device="cuda").float()
    y = torch.empty((T, H), device="cuda")
    layer.LayerNorm(hidden=H, in_dtype="f32", gain_dtype="f32", out_dtype="f32").run(h, gain, T, bias=bias, y=y)
    assert torch.equal(y, bias.expand(T, H))
    gy = lu.randn(lu.gen(3), T, H)
    grad = layer.NormGrad(hidden=H, in_dtype="f32", gain_dtype="f32", out_dtype="f32", centred=True)
    out = torch.empty((T, H), device="cuda")
    grad.run(h, gain, gy.cuda(), T, grad_h=out)
    want = gr.norm_grad(h.cpu(), gain.cpu(), gy, None, True, 1e-5)["grad_h"]
    gr.check("grad_h", out, *want)


@pytest.mark.parametrize("H", [2880, 7168, 8, 24])
@pytest.mark.parametrize("value", [1e6 + 0.1, 1.1e20, 1.1 * 2.0 ** 90, 1.1 * 2.0 ** 100, 1.3 * 2.0 ** 110, 1.7 * 2.0 ** 126])
def test_large_rows_of_one_value_whose_mean_is_rounded(value, H):
    """What roundings leave of the mean is taken out too, however large its squares are.  (What is left of it then is at most 2^-19 of the root:
    the sums of equal values are off by up to 24 roundings, and by no more than sqrt(mean square + epsilon) before the last of them.)"""
    T = 3
    h = torch.full((T, H), value)
    h[1] = -h[1]
    g = lu.gen(H)
    gain, bias, gy = 1 + 0.2 * lu.randn(g, H), lu.randn(g, H), lu.randn(g, T, H)
    y, out = torch.empty((T, H), device="cuda"), torch.empty((T, H), device="cuda")
    gg = torch.empty(H, device="cuda")
    layer.LayerNorm(hidden=H, in_dtype="f32", gain_dtype="f32", out_dtype="f32").run(h.cuda(), gain.cuda(), T, bias=bias.cuda(), y=y)
    u = 2.0 ** -19
    assert ((y.cpu().double() - bias.double()).abs() <= u * gain.abs() + 2.0 ** -24 * bias.abs()).all()
    grad = layer.NormGrad(hidden=H, in_dtype="f32", gain_dtype="f32", out_dtype="f32", centred=True)
    grad.run(h.cuda(), gain.cuda(), gy.cuda(), T, grad_h=out, grad_gain=gg)
    v = gy.double() * gain.double()
    root = 1e-5 ** 0.5
    # u times mean(v * u) on top of that, the mean's own 24 roundings and the root's, half of u's
    err = (v.abs() + 2 * v.abs().mean(dim=1, keepdim=True)) * u / root
    assert ((out.cpu().double() - (v - v.mean(dim=1, keepdim=True)) / root).abs() <= err).all()
    assert (gg.cpu().double().abs() <= u * gy.double().abs().sum(dim=0)).all()


@pytest.mark.parametrize("value", [1e8, 1.1 * 2.0 ** 90, 1.7 * 2.0 ** 126])
def test_rows_that_differ_in_their_last_bit(value):
    """Every third value is the next one: the layer norm of 0, 0, 1 (times their distance, beside which epsilon is nothing)."""
    T, H = 2, 2880
    h = torch.full((T, H), value)
    h[:, ::3] = torch.nextafter(h[:, ::3], torch.tensor(float("inf")))
    ones, y, out = torch.ones(H), torch.empty((T, H), device="cuda"), torch.empty((T, H), device="cuda")
    layer.LayerNorm(hidden=H, in_dtype="f32", gain_dtype="f32", out_dtype="f32").run(h.cuda(), ones.cuda(), T, y=y)
    step = h[0, 0].double() - h[0, 1].double()
    small = (torch.arange(H) % 3 == 0).double().expand(T, H) * step
    d = small - small.mean(dim=1, keepdim=True)
    root = ((d * d).mean(dim=1, keepdim=True) + 1e-5).sqrt()
    # d and the mean square are of whole steps, but for the mean that is left: 24 roundings each
    assert ((y.cpu().double() - d / root).abs() <= 2.0 ** -19 * 1.5).all()
    gy = lu.randn(lu.gen(4), T, H)
    layer.NormGrad(hidden=H, in_dtype="f32", gain_dtype="f32", out_dtype="f32", centred=True).run(h.cuda(), ones.cuda(), gy.cuda(), T, grad_h=out)
    v, u = gy.double(), d / root
    want = (v - u * (v * u).mean(dim=1, keepdim=True) - v.mean(dim=1, keepdim=True)) / root
    err = 2.0 ** -19 * 8 * (v.abs() + v.abs().mean(dim=1, keepdim=True)) / root + 2.0 ** -149
    assert ((out.cpu().double() - want).abs() <= err).all()


def test_against_differences():
    """The gradient of a weighted sum of the layer norm's outputs, by central differences of the kernel itself in fp32."""
    T, H = 2, 64
    g = lu.gen(5)
    h, gain, bias, weight = lu.randn(g, T, H), 1 + 0.2 * lu.randn(g, H), lu.randn(g, H), lu.randn(g, T, H)
    norm = layer.LayerNorm(hidden=H, in_dtype="f32", gain_dtype="f32", out_dtype="f32")
    grad = layer.NormGrad(hidden=H, in_dtype="f32", gain_dtype="f32", out_dtype="f32", centred=True)
    out, gg, gb = torch.empty((T, H), device="cuda"), torch.empty(H, device="cuda"), torch.empty(H, device="cuda")
    grad.run(h.cuda(), gain.cuda(), weight.cuda(), T, grad_h=out, grad_gain=gg, grad_bias=gb)
    step = 2.0 ** -6
    # all 2 H differences of a row at once: a row each
    probe = torch.cat([h[:1] + step * torch.eye(H), h[:1] - step * torch.eye(H)])
    y = torch.empty((2 * H, H), device="cuda")
    norm.run(probe.cuda(), gain.cuda(), 2 * H, bias=bias.cuda(), y=y)
    loss = (y.cpu().double() * weight[:1].double()).sum(dim=1)
    slope = (loss[:H] - loss[H:]) / (2 * step)
    # third derivatives of order |weight| sqrt(H) times step^2 / 6, and roundings of 2^-20 over the step
    assert (slope - out[0].cpu().double()).abs().max() < 8 * step ** 2 / 6 * 8 + 2.0 ** -20 * 64 / step


def test_captured_and_replayed_beside_eager_work():
    T, H = 300, 2048
    grad, other = layer.NormGrad(hidden=H), layer.NormGrad(hidden=H)
    g = torch.Generator(device="cuda").manual_seed(2)
    new = lambda: torch.randn((T, H), generator=g, device="cuda").bfloat16()
    h, gy, gs, gain = new(), new(), new(), torch.ones(H, dtype=torch.bfloat16, device="cuda")
    out, gg = torch.empty_like(h), torch.zeros(H, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        grad.run(h, gain, gy, T, grad_sum=gs, grad_h=out, grad_gain=gg, stream=stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        grad.run(h, gain, gy, T, grad_sum=gs, grad_h=out, grad_gain=gg, stream=stream)
    for _ in range(4):
        for t in (h, gy, gs):
            t.copy_(new())
        out.zero_()
        want, want_gain = torch.empty_like(h), torch.empty(H, device="cuda")
        other.run(h, gain, gy, T, grad_sum=gs, grad_h=want, grad_gain=want_gain)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(gg, want_gain)
