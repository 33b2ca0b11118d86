"""16-bit results of the grouped products: the sum is formed in float32 and rounded once, whatever its length and what it is added
to.  The float32 sum is off by at most e = (50 + rows / 768) 2^-23 of its terms' sizes: 48 truncated steps of the tensor cores per 768
terms, two for the hand-over, and the additions.  Rounding keeps order, so a result rounded once lies between the roundings of
the exact sum less e and more e."""
import pytest
import torch

from paper_1902_01064_b200 import hop, nn

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


# ------------------------------------------------------------------------------------------------ sums of very many terms
# All terms are positive, so truncation in the tensor cores all goes one way.  Bound of the mean error: 48 truncated steps and two of
# the hand-over before each float32 addition, 50 * 2^-23 of the value, and per addition half a unit, 2^-24: together below
# (50 + 0.5 T / 768) 2^-23; the last roundings average out over the N results: 5 * 2^-11 / sqrt(12 N) are allowed.
def positive(seed, *shape, mul=1.0):
    return (torch.rand(*shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV) * mul).to(torch.float16)


@pytest.mark.parametrize("n,k", [(1536, 2048), (1500, 2001)])
def test_weight_gradients_of_many_rows(n, k):
    T = 200_000
    dy, x = positive(1, T, n, mul=0.5), positive(2, T, k, mul=0.5)
    got = nn.grouped_linear_dw(dy, x, out_dtype=torch.float16)[0].double()
    want = sum(dy[i:i + 20000].double().T @ x[i:i + 20000].double() for i in range(0, T, 20000))
    off = (got - want) / want
    bound = (50 + 0.5 * T / 768) * 2.0 ** -23 + 5 * 2.0 ** -11 / (12 * off.numel()) ** 0.5
    assert abs(float(off.mean())) <= bound, (float(off.mean()), bound)
    assert float(off.abs().max()) <= 2.0 ** -11 + (50 + 0.5 * T / 768) * 2.0 ** -23


@pytest.mark.parametrize("way", ["fwd", "dx"])
def test_very_wide_layers(way):
    K, N, T = 100_000, 1280, 2000
    a, w = positive(1, T, K, mul=0.5), positive(2, 1, N, K, mul=0.5)
    if way == "dx":
        w = w.transpose(1, 2).contiguous()
    got = (nn.grouped_linear(a, w) if way == "fwd" else nn.grouped_linear_dx(a, w)).double()
    m = w[0].T if way == "fwd" else w[0]
    want = sum(a[:, i:i + 10000].double() @ m[i:i + 10000].double() for i in range(0, K, 10000))
    off = (got - want) / want
    bound = (50 + 0.5 * K / 768) * 2.0 ** -23 + 5 * 2.0 ** -11 / (12 * off.numel()) ** 0.5
    assert abs(float(off.mean())) <= bound, (float(off.mean()), bound)


@pytest.mark.parametrize("way,counts,n,k", [("dw", [4000, 0, 700, 333], 1111, 1333), ("dw", [4000, 0, 700, 333], 1096, 1328), ("dw", [130, 7, 0, 200] * 15, 100, 200),
                                            ("fwd", [300, 0, 200, 150], 5000, 4100), ("fwd", [30, 1, 0, 50], 5001, 4100), ("dx", [300, 0, 200, 150], 4104, 5000),
                                            ("dx", [30, 1, 0, 50], 4101, 4999)])
def test_long_sums_in_ragged_groups(way, counts, n, k):
    """Above 4096 terms half-precision results leave the tensor cores as float32 results do; e as above, one rounding."""
    T, off = sum(counts), nn.group_offsets(counts, DEV)
    ends = off.tolist()
    a = randn(1, T + 3, k if way == "fwd" else n, dtype=torch.float16)
    b = randn(2, T + 3, k, dtype=torch.float16) if way == "dw" else randn(2, len(counts), n, k, dtype=torch.float16, mul=max(n, k) ** -0.5)
    got = {"fwd": nn.grouped_linear, "dx": nn.grouped_linear_dx}[way](a, b, off) if way != "dw" else nn.grouped_linear_dw(a, b, off, out_dtype=torch.float16)
    for g, (lo, hi) in enumerate(zip(ends[:-1], ends[1:])):
        p = a[lo:hi].double()
        p, q = (p.T, b[lo:hi].double()) if way == "dw" else (p, b[g].double().T if way == "fwd" else b[g].double())
        want = p @ q
        e = (50 + p.shape[1] / 768) * 2.0 ** -23 * (p.abs() @ q.abs())
        low, high = (want - e).half(), (want + e).half()
        mine = got[g] if way == "dw" else got[lo:hi]
        assert bool(((low <= mine) & (mine <= high)).all()), g
    assert way == "dw" or bool((got[T:] == 0).all())
    assert nn.linear_status(DEV) == 0


# ------------------------------------------------------------------------------------------------ float32 results
@pytest.mark.parametrize("sign", ["random", "one"])
@pytest.mark.parametrize("T,n,k", [(300, 1536, 2048), (768, 1536, 2048), (5000, 1536, 2048), (70_000, 1536, 2048), (70_000, 64, 72), (5000, 1111, 1333)])
def test_float32_results_of_any_length(T, n, k, sign):
    """The accumulator is handed over every 768 terms.  A truncated step is off by less than a unit, 2^-23, of what has been summed,
    at most S = sum |a||b|: 48 steps, two units for the products' own sums and the hand-over, and half a unit per float32
    addition, T / 768 of them (parts: 16 more).  Element by element (50 + 0.5 (T / 768 + 16)) 2^-23 S; for terms of one sign, S is the
    result and the 50 units bound the mean error at any length (the additions round both ways: a hundredth of them allowed)."""
    make = (lambda s, *d: randn(s, *d, dtype=torch.float16)) if sign == "random" else (lambda s, *d: positive(s, *d, mul=0.5))
    dy, x = make(1, T, n), make(2, T, k)
    got = nn.grouped_linear_dw(dy, x)[0].double()
    want, size = torch.zeros_like(got), torch.zeros_like(got)
    for i in range(0, T, 20000):
        p, q = dy[i:i + 20000].double().T, x[i:i + 20000].double()
        want += p @ q
        size += p.abs() @ q.abs()
    assert bool(((got - want).abs() <= (50 + 0.5 * (T / 768 + 16)) * 2.0 ** -23 * size).all())
    if sign == "one":
        assert abs(float(((got - want) / want).mean())) <= (50 + 0.005 * (T / 768 + 16)) * 2.0 ** -23


def test_products_repeat_bit_for_bit():
    """The same inputs, other work in between: no sum depends on the order in which blocks finish."""
    off = nn.group_offsets([700, 0, 1300, 48], DEV)
    x, w, dy = randn(1, 2048, 1024, dtype=torch.bfloat16), randn(2, 4, 1536, 1024, dtype=torch.bfloat16), randn(3, 2048, 1536, dtype=torch.bfloat16)
    calls = [lambda s: nn.grouped_linear(x * s, w, off), lambda s: nn.grouped_linear_dx(dy * s, w, off), lambda s: nn.grouped_linear_dw(dy * s, x, off),
             lambda s: nn.grouped_linear_dw(dy * s, x, off, out_dtype=torch.bfloat16), lambda s: nn.grouped_linear(x[:5] * s, w[0])]
    for call in calls:
        first = call(1).clone()
        for _ in range(5):
            call(3)
            assert torch.equal(call(1), first)


def test_a_products_wait_that_runs_out_is_reported_once_and_leaves_the_context_usable():
    x, w = randn(1, 300, 256, dtype=torch.bfloat16), randn(2, 1, 256, 256, dtype=torch.bfloat16)
    want = nn.grouped_linear(x, w)
    assert nn.linear_status(DEV) == 0
    stream = torch.cuda.current_stream().cuda_stream
    assert hop.lib.hop_linear_selftest_bounded_wait(1_000_000, stream, None, 0) == hop.OK       # a millisecond
    with pytest.raises(hop.HopError) as e:
        nn.linear_status(DEV)
    assert e.value.code == hop.E_DEVICE and "wait" in str(e.value)
    assert nn.linear_status(DEV) == 0
    assert torch.equal(nn.grouped_linear(x, w), want)
    for ns in (0, -1, 10 ** 9 + 1):
        assert hop.lib.hop_linear_selftest_bounded_wait(ns, stream, None, 0) == hop.E_ARG
