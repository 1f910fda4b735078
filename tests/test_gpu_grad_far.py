"""Gradients of arrays of more than 4 GiB.  Their values are -1, 0 and 1, whose sums fp32 holds exactly: results are compared
to the bit, at both ends and at rows between."""
import gc

import pytest
import torch

from paper_2605_10670_amd import binding, layer, synth

pytestmark = pytest.mark.gpu
PAST = 2 ** 32


@pytest.fixture(autouse=True)
def nothing_large_stays():
    """What lasts and is made by the way, the library's workspace for products, is made before anything large is: cut from a freed large
    block it would hold the whole of that, and later tests' allocations would come from there."""
    gc.collect()
    torch.cuda.empty_cache()
    one = torch.ones((64, 64), device="cuda")
    (one @ one).sum().item()
    yield
    gc.collect()
    torch.cuda.empty_cache()


def small_integers(seed, *shape, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-1, 2, shape, generator=g, device="cuda", dtype=torch.int8).to(dtype)


def some_of(n):
    return torch.cat([torch.arange(40), torch.randint(0, n, (400,), generator=torch.Generator().manual_seed(n)), torch.arange(n - 40, n)]).cuda()


def test_tokens():
    T, k, H, R, primary = 40000, 8, 7168, 4, 8
    assert T * k * H * 2 > PAST
    ctx = binding.Context(num_ranks=R, slots_per_rank=primary, primary_slots=primary, num_logical=R * primary, max_tokens=T, topk=k, hidden=H)
    ctx.update_placement(synth.preferred_placement(R, primary, 0))
    idx = torch.rand((T, R * primary), generator=torch.Generator().manual_seed(1)).argsort(dim=1)[:, :k].to(torch.int32).cuda()
    ctx.dispatch_layout(idx, T)
    row = torch.from_numpy(ctx.read_layout(T)["row_of"]).long().cuda()
    assert (row >= 0).all()
    y, grad_out, w = small_integers(2, T * k, H), small_integers(3, T, H), torch.rand((T, k), device="cuda")
    grad_y, grad_w = torch.full_like(y, 7.0), torch.full_like(w, 7.0)
    ctx.combine_grad(y, w, grad_out, grad_y, grad_w, T)
    t = some_of(T)
    for j in range(k):
        assert torch.equal(grad_y[row[t, j]], (w[t, j, None] * grad_out[t].float()).bfloat16())
        assert torch.equal(grad_w[t, j], (grad_out[t].float() * y[row[t, j]].float()).sum(dim=1))
    grad_x = torch.full_like(grad_out, 7.0)
    ctx.dispatch_grad(y, grad_x, T)
    assert torch.equal(grad_x[t], y[row[t].flatten()].view(len(t), k, H).float().sum(dim=1).bfloat16())
    ctx.destroy()


@pytest.mark.parametrize("K,I", [(8192, 64), (64, 8192)])
def test_rows_of_the_products(K, I):
    counts = [150000, 0, 170000]
    P, rows = len(counts), sum(counts)
    assert rows * max(K, I) * 2 > PAST
    offset = torch.tensor([0] + counts).cumsum(0).int().cuda()
    grad_y, x, w = small_integers(1, rows, I), small_integers(2, rows, K), small_integers(3, P, I, K)
    grad_x, grad_w = torch.full_like(x, 7.0), torch.full((P, I, K), 7.0, device="cuda")
    handle = layer.ExpertProductGrad(num_slots=P, in_features=K, out_features=I, max_rows=rows, grad_w_dtype="f32")
    handle.run(grad_y, rows, offset=offset, x=x, w=w, grad_x=grad_x, grad_w=grad_w)
    at, lo = some_of(rows), 0
    for p, n in enumerate(counts):
        mine = at[(at >= lo) & (at < lo + n)]
        assert torch.equal(grad_x[mine], (grad_y[mine].float() @ w[p].float()).bfloat16())
        want = torch.zeros((I, K), device="cuda")
        for first in range(lo, lo + n, 10000):
            want += grad_y[first:first + 10000].float().T.contiguous() @ x[first:first + 10000].float()
        assert torch.equal(grad_w[p], want)
        lo += n
    handle.destroy()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_slots_of_the_products(dtype):
    """A slot's weights and their gradients begin past 4 GiB."""
    K, I, counts = 264, 72, [5, 300]
    size, name = torch.finfo(dtype).bits // 8, {torch.bfloat16: "bf16", torch.float32: "f32"}[dtype]
    stride = PAST + 4096
    offset = torch.tensor([0, 5, 305]).int().cuda()
    store, grads = (torch.empty((stride + I * K * size) // size, dtype=dtype, device="cuda") for _ in range(2))
    slot = lambda t, p: t[p * stride // size:p * stride // size + I * K].view(I, K)
    for p in range(2):
        slot(store, p).copy_(small_integers(p, I, K))
    grads[I * K:I * K + 1000] = 7.0
    grad_y, x = small_integers(4, 305, I, dtype=dtype), small_integers(5, 305, K, dtype=dtype)
    grad_x = torch.empty_like(x)
    handle = layer.ExpertProductGrad(num_slots=2, in_features=K, out_features=I, max_rows=305, dtype=name, grad_w_dtype=name, slot_stride=stride,
                                     grad_stride=stride)
    handle.run(grad_y, 305, offset=offset, x=x, w=store, grad_x=grad_x, grad_w=grads)
    for p, (lo, hi) in enumerate([(0, 5), (5, 305)]):
        assert torch.equal(grad_x[lo:hi], (grad_y[lo:hi].float() @ slot(store, p).float()).to(dtype))
        assert torch.equal(slot(grads, p), (grad_y[lo:hi].float().T.contiguous() @ x[lo:hi].float()).to(dtype))
    assert (grads[I * K:I * K + 1000] == 7.0).all()
    handle.destroy()


@pytest.mark.parametrize("centred", [False, True])
def test_rows_of_the_norms(centred):
    """Every row has as many values 1 as -1 and no others, so that mean and mean square are 0 and 1; epsilon is 0."""
    T, H = 300000, 8192
    assert T * H * 2 > PAST
    h = small_integers(1, T, H // 2).abs_().mul_(2).sub_(1)
    h = torch.cat([h, -h], dim=1)
    grad_y, gain = small_integers(2, T, H), torch.ones(H, device="cuda", dtype=torch.bfloat16)
    grad_h, grad_gain = torch.full_like(h, 7.0), torch.empty(H, device="cuda")
    handle = layer.NormGrad(hidden=H, centred=centred, epsilon=0.0)
    handle.run(h, gain, grad_y, T, grad_h=grad_h, grad_gain=grad_gain)
    t = some_of(T)
    v, u = grad_y[t].float(), h[t].float()
    want = v - u * (v * u).mean(dim=1, keepdim=True) - (v.mean(dim=1, keepdim=True) if centred else 0)
    assert torch.equal(grad_h[t], want.bfloat16())   # (multiples of 2^-13: exact up to the rounding)
    total = torch.zeros(H, device="cuda")
    for first in range(0, T, 10000):
        total += (grad_y[first:first + 10000].float() * h[first:first + 10000].float()).sum(dim=0)
    assert torch.equal(grad_gain, total)
    if centred:
        y = torch.full_like(h, 7.0)
        layer.LayerNorm(hidden=H, epsilon=0.0).run(h, gain, T, y=y)
        assert torch.equal(y[t], h[t]) and torch.equal(y[-1], h[-1])
    handle.destroy()
