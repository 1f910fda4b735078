"""The norms' gradients where rows and gradients are within fp32, as their results are, but their products or sums are not."""
import pytest
import torch

from paper_2605_10670_amd import layer

import grad_util as gr
import layer_util as lu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,H", [(3, 520), (530, 8192), (3, 12288), (2, 16392)])
@pytest.mark.parametrize("centred", [False, True])
@pytest.mark.parametrize("size,grad_size,epsilon,along", [
    (1e15, 1e23, 1e-5, True),     # terms of one sign: their sum is beyond fp32
    (1e15, 1e30, 1e-5, False),    # so is every one of them
    (1.0, 3e37, 1e-5, True),
    (1e-15, 1e-25, 0.0, False),   # terms below fp32's normal numbers
    (1e-12, 1e-27, 0.0, True)])
def test_products_of_rows_and_gradients_that_leave_fp32(T, H, centred, size, grad_size, epsilon, along):
    g = lu.gen(T + H)
    h = lu.randn(g, T, H) * size
    gain = 1 + 0.2 * lu.randn(g, H).abs()
    gy = (h / size * (0.1 + torch.rand((T, H), generator=g)) if along else 0.1 + torch.rand((T, H), generator=g)) * grad_size
    gy[1] = lu.randn(g, H)    # (a row among them that is like others)
    want = gr.norm_grad(h, gain, gy, None, centred, epsilon)["grad_h"]
    assert want[0].abs().max() < 3e38
    grad = layer.NormGrad(hidden=H, in_dtype="f32", gain_dtype="f32", out_dtype="f32", centred=centred, epsilon=epsilon)
    out, gg = torch.empty((T, H), device="cuda"), torch.empty(H, device="cuda")
    grad.run(h.cuda(), gain.cuda(), gy.cuda(), T, grad_h=out, grad_gain=gg)
    gr.check("grad_h", out, want[0], want[1] + 2.0 ** -140)
    again, place = torch.empty_like(gg), h.cuda()
    grad.run(place, gain.cuda(), gy.cuda(), T, grad_h=place, grad_gain=again)
    assert torch.equal(place, out) and torch.equal(again, gg)
    grad.destroy()


def test_large_terms_that_cancel_beside_a_small_one():
    """A sum that is small says nothing of the size of its terms."""
    T, H = 2, 64
    h, gy = torch.ones((T, H)), torch.zeros((T, H))
    h[:, 1] = -1.0
    gy[:, 0] = gy[:, 1] = 2.0 ** 100
    gy[:, 2] = 2.0 ** -110
    want = gr.norm_grad(h, torch.ones(H), gy, None, False, 1e-5)["grad_h"]
    out = torch.empty((T, H), device="cuda")
    layer.NormGrad(hidden=H, in_dtype="f32", gain_dtype="f32", out_dtype="f32", epsilon=1e-5).run(h.cuda(), torch.ones(H).cuda(), gy.cuda(), T, grad_h=out)
    gr.check("grad_h", out, *want)
