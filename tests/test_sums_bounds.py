"""The bounds of long sums: they hold for sums in fp32, and not where a part of the sum was kept in fewer bits, or added in one chain
where several are asked for.  On the CPU, with mistakes that are planted in the sums here."""
import pytest
import torch

import sums_util as su


def operands(terms, dtype, rows=48, columns=48):
    g = torch.Generator().manual_seed(terms)
    a, b = (torch.randn(shape, generator=g).to(dtype).float() for shape in ((terms, rows), (terms, columns)))
    return a, b, a.double().t() @ b.double()


def summed(a, b, chain=0, keep=lambda t: t, rounded=lambda t: t):
    """One term after the other; after every `chain` of them the sum so far goes through `keep`, or, where that is None, is put aside
    through `rounded` to be added to the others' sums."""
    acc, total = torch.zeros(a.shape[1], b.shape[1]), torch.zeros(a.shape[1], b.shape[1])
    for i in range(a.shape[0]):
        acc = acc + a[i][:, None] * b[i]
        if chain and (i + 1) % chain == 0:
            if keep is None:
                total, acc = total + rounded(acc), torch.zeros_like(acc)
            else:
                acc = keep(acc)
    return total + acc if keep is not None else total + rounded(acc)


def through_bf16(t):
    return t.bfloat16().float()


@pytest.mark.parametrize("terms", [3000, 10700])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_sums_kept_in_bf16_are_seen(terms, out):
    a, b, exact = operands(terms, torch.bfloat16)
    limit = su.bound(terms, out, parts=64)
    assert su.off(summed(a, b).to(out), exact) < limit
    for wrong in (summed(a, b, 512, keep=through_bf16), summed(a, b, 128, keep=through_bf16)):
        assert su.off(wrong.to(out), exact) > limit
    if out is torch.float32:
        assert su.off(summed(a, b, 512, keep=None, rounded=through_bf16), exact) > 100 * limit


def test_one_long_chain_is_seen_where_several_are_asked_for():
    a, b, exact = operands(5632, torch.float32)
    limit = su.bound(5632, torch.float32, folded=512, parts=64)
    assert su.off(summed(a, b, 512, keep=None), exact) < limit < su.off(summed(a, b), exact)
