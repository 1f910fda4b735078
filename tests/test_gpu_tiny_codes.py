"""Groups whose scale is a subnormal of few units: its rounding leaves quotients up to 671, which saturate at 448 as those of the
quantising dispatch do.  All values here are whole units of 2^-149, so the codes are known exactly."""
import numpy as np
import pytest
import torch

import product_util as pu
from paper_2605_10670_amd import layer

pytestmark = pytest.mark.gpu

UNIT = 2.0 ** -149


def exact_codes(units):
    """units [rows, n] whole numbers -> (codes as the values that they stand for, fp32 scales) of groups of 128."""
    v = (units * UNIT).astype(np.float32)
    assert np.array_equal(v.astype(np.float64), units * UNIT)
    b = v.reshape(v.shape[0], -1, 128)
    scale = np.abs(b).max(axis=2) / np.float32(448)
    scale = np.where(scale == 0, np.float32(1), scale).astype(np.float32)
    q = (b / scale[:, :, None]).astype(np.float32).reshape(v.shape)
    return torch.from_numpy(np.clip(q, -448, 448)).to(torch.float8_e4m3fn).float(), torch.from_numpy(scale)


def check(code, scale, units):
    want_code, want_scale = exact_codes(units)
    assert torch.equal(scale.cpu(), want_scale)
    got = code.cpu().float()
    assert not got.isnan().any(), f"{int(got.isnan().sum())} codes are NaN"
    assert torch.equal(got, want_code)


def test_norm():
    """Rows of ones (the norm's inverse root is 1 exactly: 128 * 1 over 128, epsilon 0) times gains of whole units."""
    groups = 256
    rng = np.random.default_rng(1)
    top = np.concatenate([np.arange(200, 200 + groups * 26, 26)])
    units = np.stack([np.concatenate([[t], rng.integers(-t, t + 1, 127)]) for t in top]).reshape(1, -1)
    gain = torch.from_numpy((units[0] * UNIT).astype(np.float32))
    x = torch.ones((2, gain.numel()), device="cuda")
    x[1] = -1
    code = torch.empty(x.shape, dtype=torch.float8_e4m3fn, device="cuda")
    scale = torch.empty((2, groups), device="cuda")
    layer.Norm(hidden=gain.numel(), in_dtype="f32", gain_dtype="f32", scale_group=128, epsilon=0.0).run(
        x, gain.cuda(), 2, code=code, code_scale=scale)
    torch.cuda.synchronize()
    check(code, scale, np.concatenate([units, -units]))


@pytest.mark.parametrize("xt", ["fp8", "bf16", "f32"])
@pytest.mark.parametrize("form,P,rows,N", [("few 1 1", 1, 16, 256), ("few 1 4", 1, 64, 256), ("thin", 300, 300, 128),
                                           ("tiled 1", 1, 200, 256)])
def test_products(xt, form, P, rows, N):
    """Gate 2^-70, whose SiLU is 2^-71, times the other factor's whole numbers by 2^-78."""
    K = 384
    rng = np.random.default_rng(2)
    # channel 0 is the gate's; of the others the fp8 case's second block makes numbers up to some 7000
    x = np.zeros((rows, K))
    x[:, 0] = 1
    x[:, 128:128 + 8] = rng.integers(0, 9, (rows, 8))
    x[0, 128:128 + 8] = 0                                        # a row of zeros: scale 1
    w = np.zeros((P, 2 * N, K))
    w[:, :N, 0] = 1
    w[:, N:, 128:128 + 8] = rng.integers(-14, 15, (P, N, 8)) * 8
    slot = np.minimum(np.arange(rows), P - 1) if P > 1 else np.zeros(rows, dtype=int)
    units = np.einsum("rk,rnk->rn", x, w[slot][:, N:]) if P > 1 else x @ w[0, N:].T
    scales = {}
    if xt == "fp8":
        w_scale = np.full((P, 2 * N // 128, K // 128), 2.0 ** -40)
        w_scale[:, N // 128:] = 2.0 ** -48
        scales = dict(x_scale=torch.full((rows, K // 128), 2.0 ** -30, device="cuda"),
                      w_scale=torch.from_numpy(w_scale.astype(np.float32)).cuda())
    else:
        x, w = x * 2.0 ** -30, w * np.where(np.arange(2 * N) < N, 2.0 ** -40, 2.0 ** -48)[None, :, None]
    xd, wd = (torch.from_numpy(a.astype(np.float32)).to(pu.TORCH_OF[xt]) for a in (x, w))
    offset = torch.from_numpy(np.concatenate([[0], np.cumsum(np.bincount(slot, minlength=P))]).astype(np.int32)).cuda()
    y, y_scale, got = pu.run(xd.cuda(), wd.cuda(), offset, "fp8", True, xt=xt, **scales)
    assert got == form
    top = np.abs(units.reshape(rows, -1, 128)).max(axis=2)
    assert (top > 200).any() and (top < 6000).any()
    check(y, y_scale, units)
