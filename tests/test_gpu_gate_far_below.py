"""Gates so far below zero that exp(-gate) leaves fp32, beside factors that bring the product back among ordinary numbers."""
import pytest
import torch

import layer_util as lu
import product_util as pu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("y", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("form,P,rows", [("few 1 1", 1, 4), ("thin", 300, 300), ("tiled 1", 1, 200)])
def test_large_negative_gates(form, P, rows, y):
    K, N = 128, 128
    gate = -torch.arange(N, dtype=torch.float64)                     # 0 to -127; -64 in the middle of every row's codes
    up = 2.0 ** 90 * (1 + torch.arange(N, dtype=torch.float64) % 5)
    w = torch.zeros((P, 2 * N, K))
    w[:, :N, 0], w[:, N:, 1] = gate.float(), (up * 2.0 ** -60).float()
    x = torch.zeros((rows, K))
    x[:, 0], x[:, 1] = 1, 2.0 ** 60
    offset = torch.tensor([rows * p // P for p in range(P + 1)], dtype=torch.int32)
    out, y_scale, got = pu.run(x.cuda(), w.cuda(), offset.cuda(), y, True, xt="f32")
    assert got == form
    want = (gate * torch.sigmoid(gate) * up).expand(rows, N)
    # exponential, sum, quotient and products round a few times; the exponential of a gate below -87 is a multiple of 2^-149
    err = want.abs() * 16 * 2.0 ** -23 + (gate * up).abs() * 2.0 ** -149
    if y == "fp8":
        lu.check_codes(out.cpu(), y_scale.cpu(), want, err)
    else:
        lu.check_rounded(out.cpu(), want, err)
