"""Adapters whose numbers are near the ends of fp32's range, on the GPU against 64-bit arithmetic: what the formula holds is what comes out.

The bounds are test_adapters_gpu's, which are relative to the magnitudes.  Every number of these cases is a power of two times a number near one, every sum of one
t has one sign and stays below 2^128 whatever its order."""
import pytest
import torch

import test_adapters_gpu as lora
from paper_2506_17615_amd import binding as eq

pytestmark = pytest.mark.gpu

# t, the factor and B of each adapter: t just below 2^128, which is no bf16; a product with the factor past 2^128; sums past 2^128 without
# the factor; ordinary ones; a factor of zero
ADAPTERS = [(128, 1.0, -120), (128, 0.5, -110), (128, -1.5, -120), (100, 2.0 ** 60, -120), (120, -2.0 ** 120, -126), (127, 2.0 ** -60, 20), (3, 0.75, -2),
            (0, -3.0, 0), (128, 0.0, -1)]


def _case(M, widths, rank, K=70):
    g = torch.Generator().manual_seed(M + rank)
    n, N, R = len(ADAPTERS), sum(widths), rank * len(widths)
    sign = lambda *shape: 1.0 - 2.0 * torch.randint(0, 2, shape, generator=g)
    x, a, b = torch.zeros(M, K, dtype=torch.float64), torch.zeros(n, R, K, dtype=torch.float64), torch.randn(n, N, rank, generator=g).double()
    # ten powers of two one below the other: their sum is 2^top - 2^(top - 10)
    x[:, 9:69:6] = sign(M, 1).double() * 2.0 ** 60
    for i, (top, _, b_at) in enumerate(ADAPTERS):
        a[i, :, 9:69:6] = sign(R, 1).double() * 2.0 ** (top - 61 - torch.arange(10).double())
        b[i] *= 2.0 ** b_at
    ids = torch.arange(M) % (n + 1)
    bf16 = lambda t: t.to(torch.bfloat16)
    return dict(x=bf16(x), a=bf16(a), b=bf16(b), factors=torch.tensor([f for _, f, _ in ADAPTERS]), ids=ids.to(torch.int32), out=bf16(torch.randn(M, N, generator=g)),
                widths=widths)


@pytest.mark.parametrize("rank", (8, 40, 128))
@pytest.mark.parametrize("M,widths", ((10, (40,)), (64, (130, 7)), (400, (300,)), (4096, (64, 9)), (9000, (40,)), (30, (5,))))
def test_numbers_near_the_ends_of_the_range(M, widths, rank):
    case = lora._on(_case(M, widths, rank))
    start = case["out"].clone()
    got = lora._call(case).clone()
    case["out"] = start
    assert got.isfinite().all()
    lora._check(case, got, "cuda")


@pytest.mark.parametrize("M", (10, 400, 4096))
@pytest.mark.parametrize("factor", (0.5, 2.0))
def test_a_t_past_the_range_is_an_infinity(M, factor):
    """And meets B as one: B's sign says which, and a NaN stays one."""
    K, N, rank = 40, 72, 8
    x, a, b = torch.full((M, K), 2.0 ** 64), torch.zeros(2, rank, K), torch.zeros(2, N, rank)
    a[:, :, 3:7] = 2.0 ** 63
    sign = 1.0 - 2.0 * (torch.arange(N) % 3 == 0)
    b[:] = sign[:, None] * 2.0 ** -30
    x[M // 2, 5] = float("nan")
    dev = lora._on(dict(x=x.bfloat16(), a=a.bfloat16(), b=b.bfloat16(), factors=torch.full((2,), factor), ids=(torch.arange(M) % 3).to(torch.int32),
                        out=torch.ones(M, N).bfloat16(), widths=(N,)))
    got = lora._call(dev).float().cpu()
    want = (sign * float("inf")).expand(M, N).clone()
    want[M // 2] = float("nan")
    want[torch.arange(M) % 3 == 2] = 1.0
    assert torch.equal(got.nan_to_num(7.0, 8.0, 9.0), want.nan_to_num(7.0, 8.0, 9.0))
