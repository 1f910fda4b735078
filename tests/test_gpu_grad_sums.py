"""Long sums of the experts' products' gradients: how far they are off in the 2-norm, whichever tiles the sizes get and whether
their terms are divided between workgroups or not."""
import pytest
import torch

from paper_2605_10670_amd import layer

import sums_util as su

pytestmark = pytest.mark.gpu
TORCH_OF = {"bf16": torch.bfloat16, "f32": torch.float32}
MOST_PARTS = 512   # (of at most as many workgroups as 256 CUs have at a time)


def check(dtype, w_dtype, counts, K, I, wanted, folded):
    g = torch.Generator(device="cuda").manual_seed(sum(counts) + K + I)
    randn = lambda *shape: torch.randn(shape, generator=g, device="cuda").to(TORCH_OF[dtype])
    P, rows, ends = len(counts), sum(counts), torch.tensor([0] + counts).cumsum(0).tolist()
    offset = torch.tensor(ends, dtype=torch.int32, device="cuda")
    grad_y = randn(rows, I)
    handle = layer.ExpertProductGrad(num_slots=P, in_features=K, out_features=I, max_rows=rows, dtype=dtype, grad_w_dtype=w_dtype)
    if "x" in wanted:
        w, grad_x = randn(P, I, K), torch.empty((rows, K), device="cuda", dtype=TORCH_OF[dtype])
        handle.run(grad_y, rows, offset=offset, w=w, grad_x=grad_x)
        exact = torch.cat([grad_y[ends[p]:ends[p + 1]].double() @ w[p].double() for p in range(P)])
        assert su.off(grad_x, exact) < su.bound(I, grad_x.dtype, folded, MOST_PARTS)
    if "w" in wanted:
        x, grad_w = randn(rows, K), torch.empty((P, I, K), device="cuda", dtype=TORCH_OF[w_dtype])
        handle.run(grad_y, rows, offset=offset, x=x, grad_w=grad_w)
        for p in range(P):
            at = slice(ends[p], ends[p + 1])
            exact = grad_y[at].double().t().contiguous() @ x[at].double()
            assert su.off(grad_w[p], exact) < su.bound(counts[p], grad_w.dtype, folded, MOST_PARTS), p
    handle.destroy()


@pytest.mark.parametrize("counts,K,I", [([2] * 40, 520, 5632), ([54], 2432, 5632), ([2048], 2432, 5632), ([704] * 8, 520, 5632)],
                         ids=lambda v: f"{len(v)} of {v[0]}" if isinstance(v, list) else str(v))
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows(dtype, counts, K, I):
    check(dtype, dtype, counts, K, I, "x", 512 if dtype == "f32" else 0)


@pytest.mark.parametrize("counts,K,I", [([10700], 1288, 72), ([10700], 2056, 2056), ([2990, 3003, 1, 2816], 2056, 72), ([5632], 2432, 1024),
                                        ([3000] * 8, 1032, 1032)],
                         ids=lambda v: f"{len(v)} of {v[0]}" if isinstance(v, list) else str(v))
@pytest.mark.parametrize("dtype,w_dtype", [("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"), ("bf16", "bf16")])
def test_weights(dtype, w_dtype, counts, K, I):
    check(dtype, w_dtype, counts, K, I, "w", 512 if dtype == "f32" else 0)


def test_more_parts_than_workgroups_at_a_time():
    """Tiles that fill the CUs unevenly, divided: of 520 tiles two parts each, and of 200 five."""
    check("f32", "f32", [12000] * 8, 1032, 832, "w", 512)
    check("f32", "f32", [449], 6400, 5760, "x", 512)
