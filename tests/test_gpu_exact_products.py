"""The experts' product of 8-bit codes: every kernel sums exact products in fp32, whatever type the result has."""
import pytest
import torch

import product_util as pu

pytestmark = pytest.mark.gpu

# (kernel that the sizes choose, slots, rows, out_features); rows lie in the slots in turn
SIZES = [("few 1 1", 1, 5, 256), ("few 1 4", 1, 64, 256), ("thin", 300, 300, 384), ("tiled 1", 1, 200, 256), ("tiled 2", 1, 8192, 1024)]


def offsets(P, rows):
    return torch.tensor([rows * p // P for p in range(P + 1)], dtype=torch.int32)


@pytest.mark.parametrize("form,P,rows,N", SIZES)
@pytest.mark.parametrize("y,gate", [("bf16", False), ("f32", False), ("bf16", True), ("f32", True), ("fp8", True)])
def test_small_products_beside_large_ones(form, P, rows, N, y, gate):
    """Of 8 neighbouring products two are +-448 * 448 and cancel, one is 1: the sum is 1, as that of any order in fp32 is."""
    if gate and form == "tiled 2":
        N = 512                                                  # (tiles have 128 features there)
    K = 384
    weight_rows = N * (2 if gate else 1)
    x, w = torch.zeros((rows, K)), torch.zeros((P, weight_rows, K))
    for at in range(128, 256, 8):
        row = torch.arange(rows) % 16 * 8 + 128 == at            # (every eight of a block has its turn)
        x[row, at + 1], x[row, at + 3], x[row, at + 6] = 448, 1, 448
        w[:, :, at + 1], w[:, :, at + 3], w[:, :, at + 6] = 448, 1, -448
    scale = dict(x_scale=torch.ones((rows, K // 128), device="cuda"),
                 w_scale=torch.ones((P, -(-weight_rows // 128), K // 128), device="cuda"))
    out, out_scale, got = pu.run(x.to(torch.float8_e4m3fn).cuda(), w.to(torch.float8_e4m3fn).cuda(), offsets(P, rows).cuda(), y, gate,
                                 xt="fp8", **scale)
    assert got == form
    v = out.cpu().float()
    if y == "fp8":
        assert (v == 448).all()
        v = out_scale.cpu().double() * 448
    want = 1 / (1 + torch.exp(torch.tensor(-1.0, dtype=torch.float64))) if gate else torch.tensor(1.0, dtype=torch.float64)
    # (exponential, quotient and product in fp32, then the result's own rounding)
    assert ((v.double() - want).abs() <= want * (8 * 2.0 ** -24 + (2.0 ** -8 if y == "bf16" else 0))).all()


@pytest.mark.parametrize("form,P,rows,N", SIZES)
@pytest.mark.parametrize("gate", [False, True])
def test_error_of_ordinary_sums(form, P, rows, N, gate):
    """fp32 results of normally distributed values: K additions, each off by 2^-24 of a partial sum at most, in no
    common direction, are off by sqrt(K) * 2^-24 of the result together (2-norm)."""
    if gate and form == "tiled 2":
        N = 512
    K = 1024
    weight_rows = N * (2 if gate else 1)
    g = torch.Generator(device="cuda").manual_seed(5)
    randn = lambda *shape: torch.randn(shape, generator=g, device="cuda")
    x, w = (100 * randn(rows, K)).clamp(-448, 448).to(torch.float8_e4m3fn), (100 * randn(P, weight_rows, K)).clamp(-448, 448).to(torch.float8_e4m3fn)
    x_scale = 0.5 + torch.rand((rows, K // 128), generator=g, device="cuda")
    # (sums near 1, where SiLU is curved)
    w_scale = (0.5 + torch.rand((P, weight_rows // 128, K // 128), generator=g, device="cuda")) * 3e-6
    offset = offsets(P, rows)
    out, _, got = pu.run(x, w, offset.cuda(), "f32", gate, xt="fp8", x_scale=x_scale, w_scale=w_scale)
    assert got == form
    wide = lambda c, s, n: c.cpu().double() * s.cpu().double().repeat_interleave(n, dim=-2).repeat_interleave(128, dim=-1)
    xd, wd = wide(x, x_scale, 1), wide(w, w_scale, 128)
    want = torch.cat([xd[offset[p]:offset[p + 1]] @ wd[p].t() for p in range(P)])
    if gate:
        want = torch.nn.functional.silu(want[:, :N]) * want[:, N:]
    off = float((out.cpu().double() - want).norm() / want.norm())
    # (through the gate both factors' errors come in, 1.1 of the first one's at most, and a few roundings)
    assert off <= (2.2 * K ** 0.5 + 8 if gate else K ** 0.5) * 2.0 ** -24, off
