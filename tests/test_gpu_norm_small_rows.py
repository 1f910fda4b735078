"""The residual norm where the squares of a row are lost in fp32: below its smallest numbers, and above its largest.  The rows are
scaled copies of one row by powers of two, so that with epsilon 0 every row's norm is that of the first."""
import pytest
import torch

import layer_util as lu
from test_gpu_norm_route import check_norm, run_norm

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,H", [(1, 8), (5, 1000), (3, 7168), (2, 16384), (1024, 1032)])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_epsilon_zero(T, H, out):
    """Down to numbers of a few units (where the row itself has fewer bits, but its norm is as exact) and up to the largest."""
    g = lu.gen(H)
    x = lu.randn(g, T, H)
    for power in (-60, -68, -75, -85, -100, -126, -140, -146, 60, 64, 100, 124):
        row = torch.ldexp(x, torch.tensor(float(power)))
        assert (row != 0).any(dim=1).all()
        check_norm(row, None, torch.ones(H), 0.0, "f32", "f32", out, 128 if H % 128 == 0 else 0, total=False)


@pytest.mark.parametrize("power", [-75, -100, -140])
def test_epsilon_beside_small_squares(power):
    """Epsilons around the mean of the squares, from negligible to ruling; those below fp32's normal numbers as they are in fp32."""
    g = lu.gen(1)
    x = torch.ldexp(lu.randn(g, 3, 2048), torch.tensor(float(power)))
    for shift in (-40, -3, 0, 3, 40, 100):
        eps = float(torch.tensor(2.0 ** (2 * power + shift)))      # (0 where fp32 has no such number)
        check_norm(x, None, 1 + 0.1 * lu.randn(g, 2048), eps, "f32", "f32", "f32", 128, total=False)


def test_small_rows_beside_a_residual():
    """The sum is the unscaled row; bf16 rows, which reach as far down as fp32 ones."""
    g = lu.gen(2)
    x, r = (torch.ldexp(lu.randn(g, 4, 1024), torch.tensor(-90.0)).bfloat16() for _ in range(2))
    check_norm(x, r, torch.ones(1024), 0.0, "bf16", "f32", "bf16", 128)


def test_rows_of_zeros():
    """0 / sqrt(0 + epsilon): zeros with any epsilon above 0, and 0 / 0 without."""
    x = torch.zeros((2, 512))
    for eps in (1e-6, 1e-38, 1e-44):
        _, y, code, scale = run_norm(x, None, torch.ones(512), eps, "f32", "f32", "f32", 128, total=False)
        assert (y == 0).all() and (code.float() == 0).all() and (scale == 1).all()
    _, y, _, _ = run_norm(x, None, torch.ones(512), 0.0, "f32", "f32", "f32", 128, total=False)
    assert y.isnan().all()


def test_large_and_small_rows_with_an_epsilon_that_rules():
    """Squares past fp32's largest number beside an epsilon of their size."""
    g = lu.gen(3)
    x = lu.randn(g, 3, 1024) * 2.0 ** 62
    check_norm(x, None, torch.ones(1024), 2.0 ** 124, "f32", "f32", "f32", 128, total=False)
    check_norm(x * 2.0 ** 4, None, torch.ones(1024), 2.0 ** 126, "f32", "f32", "f32", 128, total=False)


@pytest.mark.parametrize("power", [62, 100, 126, -75, -110])
def test_values_far_below_the_rest_of_their_row(power):
    """One value rules the row; the others, down to what fp32 holds, keep their bits."""
    g = lu.gen(4)
    x = lu.randn(g, 3, 512) * torch.ldexp(torch.tensor(1.0), torch.randint(-90, 1, (3, 512), generator=g).float())
    x = torch.ldexp(x, torch.tensor(float(min(power, 0))))
    x[:, 5] = 2.0 ** power
    check_norm(x, None, torch.ones(512), 0.0, "f32", "f32", "f32", 128, total=False)
