"""Weight gradients added to a 16-bit result: the sum is formed in float32 and rounded once, whatever the size.

The float32 sum is off by at most e = (50 + rows / 768) 2^-23 of its terms' sizes: 48 truncated steps of the tensor cores per 768
terms, two for the hand-over, and the additions.  Rounding keeps order, so a result rounded once lies between the roundings of
the exact sum less e and more e."""
import pytest
import torch

from paper_1902_01064_b200 import nn

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def randn(seed, *shape, dtype=torch.float32, mul=1.0):
    return (torch.randn(*shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV) * mul).to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n,k", [(2048, 2304), (1300, 1290), (1111, 1333), (64, 72)])      # whole lines, words, single elements; many parts
@pytest.mark.parametrize("counts", [[300, 0, 901], [5000]], ids=str)
def test_the_sum_is_rounded_once(counts, n, k, dtype):
    T, E = sum(counts), len(counts)
    off = nn.group_offsets(counts, DEV)
    a, b = randn(1, T, n, dtype=dtype), randn(2, T, k, dtype=dtype)
    base = randn(3, E, n, k, dtype=dtype, mul=30.0)
    out = base.clone()
    nn.grouped_linear_dw(a, b, off, out=out, accumulate=True)
    ends = off.tolist()
    for g in range(E):
        p, q = a[ends[g]:ends[g + 1]].double().T, b[ends[g]:ends[g + 1]].double()
        want, size = p @ q + base[g].double(), p.abs() @ q.abs() + base[g].double().abs()
        e = (50 + counts[g] / 768) * 2.0 ** -23 * size
        low, high = (want - e).to(dtype), (want + e).to(dtype)
        assert bool(((low <= out[g]) & (out[g] <= high)).all()), (g, int((~((low <= out[g]) & (out[g] <= high))).sum()))
        assert counts[g] or torch.equal(out[g], base[g])
    assert nn.linear_status(DEV) == 0


@pytest.mark.parametrize("n,k", [(2048, 2304), (1111, 1333)])
def test_a_product_beyond_half_precision_that_the_sum_brings_back(n, k):
    """Products of 80000 onto -40000: the sum, 40000, is a half-precision number, the product is not."""
    a, b = torch.full((1250, n), 8.0, dtype=torch.float16, device=DEV), torch.full((1250, k), 8.0, dtype=torch.float16, device=DEV)
    out = torch.full((1, n, k), -40000.0, dtype=torch.float16, device=DEV)
    nn.grouped_linear_dw(a, b, out=out, accumulate=True)
    assert bool((out == 40000.0).all())


def test_rows_between_strided_results_stay(n=1111, k=1333):
    a, b = randn(1, 200, n, dtype=torch.bfloat16), randn(2, 200, k, dtype=torch.bfloat16)
    for pad in (3, 8):
        big = torch.full((n, k + pad), 5.0, dtype=torch.bfloat16, device=DEV)
        out = big[None, :, :k]
        nn.grouped_linear_dw(a, b, out=out, accumulate=True)
        fresh = torch.full((1, n, k), 5.0, dtype=torch.bfloat16, device=DEV)
        nn.grouped_linear_dw(a, b, out=fresh, accumulate=True)
        assert torch.equal(out, fresh) and bool((big[:, k:] == 5).all())
