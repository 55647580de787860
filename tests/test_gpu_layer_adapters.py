"""Adapters on the GPU whose B holds infinities."""
import pytest
import torch

import layer_plain as plain
from paper_2503_13565_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("m", [1, 20, 200, 600])
@pytest.mark.parametrize("rank", [8, 40, 128])
def test_adapters_with_infinities(m, rank):
    """What B's infinities give is what the formula gives: infinity where the row's number for that rank is not zero (whether or not it needs more than
    the bits of a BF16 number), NaN where it is zero or where two infinities cancel."""
    n, k, many = 136, 64, 3
    gen = torch.Generator().manual_seed(m + rank)
    x = torch.randint(-3, 4, (m, k), generator=gen).to(torch.bfloat16)
    x[m // 2] = 1.0
    a = torch.randint(-2, 3, (many, rank, k), generator=gen).to(torch.bfloat16)
    a[1] = torch.randn((rank, k), generator=gen).to(torch.bfloat16)
    b = torch.randint(-2, 3, (many, n, rank), generator=gen).to(torch.bfloat16)
    b[:, 5, 3], b[:, 70, 7], b[:, 71, 0], b[:, 71, 1], b[:, n - 1, rank - 1] = float("inf"), -float("inf"), float("inf"), float("inf"), float("inf")
    ids = (torch.arange(m, dtype=torch.int32) % (many + 1) - 1 + (m == 1)).to(DEV)
    scales = torch.tensor([1.0, 0.7, -0.5], device=DEV)
    base = torch.randn((m, n), generator=gen).to(torch.bfloat16).to(DEV)
    for given in (scales, None):
        y = binding.mxfp4_lora(x.to(DEV), a.to(DEV), b.to(DEV), ids, base=base, scales=given)
        want, off = plain.adapters(x, a, b, ids, base, given)
        plain.near(y, want, off.nan_to_num(nan=0.0, posinf=0.0))
