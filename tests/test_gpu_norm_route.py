"""The residual norm and the router's choice against their definitions in 64 bits."""
import math

import numpy as np
import pytest
import torch

import layer_util as lu
from paper_2605_10670_amd import layer, synth

pytestmark = pytest.mark.gpu


def exact_norm(x, r, g, eps):
    h = x.double() if r is None else x.double() + r.double()
    inv = 1 / (h.pow(2).mean(dim=1, keepdim=True) + eps).sqrt()
    v = h * inv * g.double()
    # fp32: the addition (of the larger of the two where they cancel), the mean of H squares summed by threads of at most
    # 64 and then by halves, root, quotient and two products; below the normal numbers a rounding is 2^-150 at most
    mag = x.double().abs() + (0 if r is None else r.double().abs())
    return h, v, v.abs() * 64 * 2.0 ** -24 + mag * inv * g.double().abs() * 2.0 ** -23 + 2.0 ** -149


def run_norm(x, r, g, eps, in_dtype, gain_dtype, out, group, total=True, in_place=False):
    T, H = x.shape
    n = layer.Norm(hidden=H, in_dtype=in_dtype, gain_dtype=gain_dtype, out_dtype=out, scale_group=group, epsilon=eps)
    xd, gd = x.cuda(), g.cuda()
    rd = None if r is None else r.cuda()
    s = (rd if in_place else torch.empty_like(xd)) if total else None
    y = torch.empty((T, H), dtype=lu.TORCH_OF[out], device="cuda")
    code = torch.empty((T, H), dtype=torch.float8_e4m3fn, device="cuda") if group else None
    scale = torch.empty((T, H // group), device="cuda") if group else None
    n.run(xd, gd, T, residual=rd, sum=s, y=y, code=code, code_scale=scale)
    torch.cuda.synchronize()
    return [None if t is None else t.cpu() for t in (s, y, code, scale)]


def check_norm(x, r, g, eps, in_dtype, gain_dtype, out, group, **kw):
    h, v, err = exact_norm(x, r, g, eps)
    s, y, code, scale = run_norm(x, r, g, eps, in_dtype, gain_dtype, out, group, **kw)
    if s is not None:
        assert torch.equal(s, (x.float() if r is None else x.float() + r.float()).to(s.dtype))
    lu.check_rounded(y, v, err)
    if group:
        lu.check_codes(code, scale, v, err)


@pytest.mark.parametrize("T,H", [(1, 8), (1, 64), (3, 520), (2, 1024), (5, 2880), (1, 7168), (33, 7168), (2, 8192), (1, 8200), (2, 16384),
                                 (1, 65536), (1025, 2880), (1030, 7168), (1024, 1032), (1024, 24), (1100, 8200)])
@pytest.mark.parametrize("in_dtype,gain_dtype,out", [("bf16", "bf16", "bf16"), ("f32", "bf16", "bf16"), ("f32", "f32", "f32"), ("bf16", "f32", "f32")])
@pytest.mark.parametrize("residual", [True, False])
def test_norm(T, H, in_dtype, gain_dtype, out, residual):
    g = lu.gen(T * 7 + H)
    x = lu.randn(g, T, H).to(lu.TORCH_OF[in_dtype])
    r = (3 * lu.randn(g, T, H)).to(lu.TORCH_OF[in_dtype]) if residual else None
    gain = (1 + 0.3 * lu.randn(g, H)).to(lu.TORCH_OF[gain_dtype])
    group = next((n for n in (128, 64, 32, 16) if H % n == 0), 0)
    check_norm(x, r, gain, 1e-6, in_dtype, gain_dtype, out, group, total=residual)


@pytest.mark.parametrize("group", [16, 32, 64, 128, 256, 512])
@pytest.mark.parametrize("T", [2, 1050])
def test_scale_groups(group, T):
    g = lu.gen(group)
    x, r = lu.randn(g, T, 1536).bfloat16(), lu.randn(g, T, 1536).bfloat16()
    x[:, :512] *= 100
    x[1], r[1] = 0, 0                                   # a row of zeros: scale 1, codes 0
    check_norm(x, r, torch.ones(1536).bfloat16(), 1e-5, "bf16", "bf16", "bf16", group)
    _, _, code, scale = run_norm(x, r, torch.ones(1536).bfloat16(), 1e-5, "bf16", "bf16", "bf16", group)
    assert (scale[1] == 1).all() and (code[1].float() == 0).all()


@pytest.mark.parametrize("size", [1e-30, 1e-12, 1e12, 1e18])
def test_small_and_large_values(size):
    """Down to where epsilon rules, up to where the squares still fit."""
    g = lu.gen(3)
    x = lu.randn(g, 4, 1024) * size
    check_norm(x, None, torch.ones(1024), 1e-6, "f32", "f32", "f32", 128, total=False)
    check_norm(x, None, torch.ones(1024), 0.0 if size > 1e-15 else 1e-6, "f32", "f32", "f32", 0, total=False)


def test_codes_of_groups_of_far_apart_sizes():
    """Gains that put a group's values near the ends of the range: the codes still come from a true quotient."""
    g = lu.gen(4)
    x = lu.randn(g, 3, 1024)
    gain = torch.ones(1024)
    gain[128:256], gain[256:384], gain[384:512] = 1e-33, 1e33, 1e-38
    check_norm(x, None, gain, 1e-6, "f32", "f32", "f32", 128, total=False)


def test_sum_in_place():
    g = lu.gen(5)
    for T in (1, 2000):
        x, r = lu.randn(g, T, 2048).bfloat16(), lu.randn(g, T, 2048).bfloat16()
        check_norm(x, r, torch.ones(2048).bfloat16(), 1e-6, "bf16", "bf16", "bf16", 128, in_place=True)


def test_infinity_and_nan_stay_in_their_row():
    g = lu.gen(6)
    x = lu.randn(g, 5, 1024).bfloat16()
    x[1, 7], x[3, 1000] = float("nan"), float("inf")
    gain = torch.ones(1024).bfloat16()
    _, y, code, scale = run_norm(x, None, gain, 1e-6, "bf16", "bf16", "f32", 128, total=False)
    h = x.float()
    want = h * (1 / (h.pow(2).mean(dim=1, keepdim=True) + 1e-6).sqrt())
    assert y[1].isnan().all() and scale[1].isnan().all() and code[1].float().isnan().all()
    assert torch.equal(y[3].isnan(), want[3].isnan()) and (y[3][~y[3].isnan()] == 0).all()
    clean = run_norm(x[[0, 2, 4]], None, gain, 1e-6, "bf16", "bf16", "f32", 128, total=False)
    for got, ref in zip((y, code.view(torch.uint8), scale), (clean[1], clean[2].view(torch.uint8), clean[3])):
        assert torch.equal(got[[0, 2, 4]], ref)


def test_outputs_that_are_not_asked_for():
    g = lu.gen(7)
    x, r, gain = lu.randn(g, 3, 256).bfloat16().cuda(), lu.randn(g, 3, 256).bfloat16().cuda(), torch.ones(256).bfloat16().cuda()
    n = layer.Norm(hidden=256, scale_group=128)
    whole = [torch.empty_like(x), torch.empty_like(x), torch.empty((3, 256), dtype=torch.uint8, device="cuda"),
             torch.empty((3, 2), device="cuda")]
    n.run(x, gain, 3, residual=r, sum=whole[0], y=whole[1], code=whole[2], code_scale=whole[3])
    for only in ((0,), (1,), (2, 3)):
        part = [torch.empty_like(t) if i in only else None for i, t in enumerate(whole)]
        n.run(x, gain, 3, residual=r, sum=part[0], y=part[1], code=part[2], code_scale=part[3])
        torch.cuda.synchronize()
        for i in only:
            assert torch.equal(part[i], whole[i])
    n.run(None, None, 0)


# ---- router ------------------------------------------------------------------------------------
def exact_route(logits, k, over_all):
    v = logits.double().numpy()
    v = np.where(np.isnan(v), -np.inf, v)
    order = np.argsort(-v, axis=1, kind="stable")[:, :k]          # equal ones stay in ascending order of their index
    value = np.take_along_axis(v, order, axis=1)
    top = value[:, :1]

    def ex(a):
        with np.errstate(invalid="ignore"):
            return np.where(a == -np.inf, 0.0, np.where(a == top, 1.0, np.exp(a - top)))
    total = ex(v if over_all else value).sum(axis=1, keepdims=True)
    chosen = value > -np.inf
    w = np.divide(ex(value), total, out=np.zeros_like(value), where=chosen)
    return torch.from_numpy(np.where(chosen, order, -1).astype(np.int32)), torch.from_numpy(w)


def run_route(logits, k, over_all=False, dtype="f32"):
    T, E = logits.shape
    idx = torch.full((T, k), 99, dtype=torch.int32, device="cuda")
    w = torch.full((T, k), 99.0, device="cuda")
    layer.Router(num_logical=E, topk=k, in_dtype=dtype, over_all=over_all).run(logits.cuda(), idx, w, T)
    torch.cuda.synchronize()
    return idx.cpu(), w.cpu()


def check_route(logits, k, over_all=False, dtype="f32"):
    logits = logits.to(lu.TORCH_OF[dtype])
    idx, w = run_route(logits, k, over_all, dtype)
    want_idx, want_w = exact_route(logits, k, over_all)
    assert torch.equal(idx, want_idx)
    # the difference rounds to 2^-24 of its size, which the exponential magnifies by that size; the exponential itself,
    # the sum of up to 64 partial sums of 64 and the quotient
    size = (logits.double().abs().nan_to_num(0, 0, 0).amax(dim=1, keepdim=True) * 2)
    assert ((w.double() - want_w).abs() <= want_w * (size + 140) * 2.0 ** -24 + 1e-37).all()


@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 2, 2), (3, 8, 3), (5, 16, 2), (7, 60, 6), (4, 64, 8), (9, 65, 8), (13, 96, 6), (33, 128, 8),
                                   (66, 256, 8), (5, 257, 10), (6, 512, 32), (3, 1000, 5), (2, 1025, 4), (2, 4096, 8), (2, 4095, 32)])
@pytest.mark.parametrize("over_all", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_route(T, E, k, over_all, dtype):
    check_route(lu.randn(lu.gen(E + k), T, E) * 2, k, over_all, dtype)


@pytest.mark.parametrize("E,k", [(16, 4), (60, 6), (96, 16), (97, 8), (128, 32), (256, 8)])
@pytest.mark.parametrize("dtype,over_all", [("f32", False), ("bf16", True)])
def test_many_tokens(E, k, dtype, over_all):
    """Enough of them that several share a wavefront, the last one not full; ties among them, blocked logits and empty rows."""
    T = 8195
    logits = lu.randn(lu.gen(E), T, E)
    logits[::7] = torch.randint(-1, 2, (len(logits[::7]), E), generator=lu.gen(1)).float()
    logits[::11, E // 2:] = -math.inf
    logits[::13] = math.nan
    check_route(logits, k, over_all, dtype)


def test_ties_go_to_the_lower_index():
    g = lu.gen(8)
    for E in (16, 64, 200, 256, 1024):
        logits = torch.randint(-2, 3, (40, E), generator=g).float()
        logits[0] = 0
        logits[1] = -0.0
        logits[1, ::2] = 0.0                            # the two zeros are one value
        check_route(logits, min(8, E))


def test_blocked_rows():
    """Masks of -infinity and of the type's lowest value, rows with too few logits left, rows with none."""
    logits = lu.randn(lu.gen(9), 8, 96)
    logits[0] = -math.inf
    logits[1, 3:] = -math.inf
    logits[2, :95] = -math.inf
    logits[3] = torch.finfo(torch.float32).min
    logits[4, 1:] = torch.finfo(torch.float32).min
    logits[5, ::2] = math.nan
    logits[6] = math.nan
    logits[7, 5] = logits[7, 50] = math.inf
    for over_all in (False, True):
        check_route(logits, 6, over_all)
    idx, w = run_route(logits, 6)
    assert (idx[0] == -1).all() and (w[0] == 0).all() and idx[2, 0] == 95 and w[2, 0] == 1
    assert idx[7, :2].tolist() == [5, 50] and w[7].tolist() == [0.5, 0.5, 0, 0, 0, 0]


def test_same_choice_as_the_generator():
    logits = np.random.default_rng(10).standard_normal((64, 256), dtype=np.float32)
    idx, w = synth.router_topk(logits, 8)
    got_idx, got_w = run_route(torch.from_numpy(logits), 8)
    assert np.array_equal(got_idx.numpy(), idx)
    assert np.allclose(got_w.numpy(), w, rtol=2e-6, atol=0)


def test_logits_at_odd_addresses():
    """A row of an odd number of logits begins anywhere."""
    logits = lu.randn(lu.gen(11), 9, 61)
    store = torch.zeros(9 * 61 + 1, device="cuda")
    store[1:] = logits.flatten().cuda()
    idx = torch.empty((9, 4), dtype=torch.int32, device="cuda")
    w = torch.empty((9, 4), device="cuda")
    layer.Router(num_logical=61, topk=4).run(store.data_ptr() + 4, idx, w, 9)
    torch.cuda.synchronize()
    want, _ = exact_route(logits, 4, False)
    assert torch.equal(idx.cpu(), want)
