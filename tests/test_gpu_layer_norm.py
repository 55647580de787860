"""The norm on the GPU where a residual cancels and where the mean and eps together leave FP32, against the definition in 64 bits (layer_plain.py)."""
import pytest
import torch

import layer_plain as plain
from paper_2503_13565_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _check(x, r, eps, weight=None):
    x, r = x.to(DEV), None if r is None else r.to(DEV)
    got = binding.mxfp4_rms_norm(x, weight, residual=r, eps=eps)
    y, y_off, h, h_off = plain.norm(x, r, weight, eps)
    plain.near(got.y, y, y_off, "y")
    if r is not None:
        plain.near(got.total, h, h_off, "sum")
        own = x.clone(), r.clone()                              # in the places of the inputs, which such rows read again
        binding.mxfp4_rms_norm(own[0], weight, residual=own[1], eps=eps, y=own[0], total=own[1])
        assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(own, (got.y, got.total)))


@pytest.mark.parametrize("m", [8, 264])
@pytest.mark.parametrize("k", [8, 64, 512, 4096, 20480])
def test_norm_of_a_residual_that_cancels(m, k):
    """Rows whose sum with the residual is far below both, or nothing."""
    gen = torch.Generator().manual_seed(k)
    noise = torch.randn((m, k), generator=gen).to(torch.bfloat16)
    x, r = torch.zeros((m, k), dtype=torch.bfloat16), torch.zeros((m, k), dtype=torch.bfloat16)
    x[0], x[0, 0], r[0, 0] = 2.0 ** -60, 2.0 ** 40, -2.0 ** 40
    x[1], r[1] = noise[1], -noise[1]                            # nothing is left
    x[2], r[2] = noise[2] * 2.0 ** 110, -noise[2] * 2.0 ** 110
    x[2, k - 1], r[2, k - 1] = 2.0 ** -130, -2.0 ** -132
    x[3], r[3] = noise[3] * 2.0 ** -70, noise[3].roll(1) * -2.0 ** -70
    x[4], x[4, 0], r[4, 0] = 1.5 * 2.0 ** 63, 3.0e38, -3.0e38
    x[5], r[5] = 2.0 ** -126, -1.5 * 2.0 ** -127
    x[6], x[6, 0], r[6, 0] = noise[6] * 2.0 ** -100, 1.0, -1.0
    x[7], r[7] = noise[7], noise[7]
    x[8:], r[8:] = noise[8:], -noise[8:]
    x[8::3, 5] *= 2
    for eps in (1e-30, 0.0, 1e-38, 1e-5):
        _check(x, r, eps)


@pytest.mark.parametrize("m", [1, 300])
@pytest.mark.parametrize("k", [8, 64, 4096, 8192])
def test_norm_of_an_eps_near_the_largest_number(m, k):
    """The mean and eps are FP32 numbers, their sum is not."""
    gen = torch.Generator().manual_seed(k)
    x = (0.5 + torch.rand((m, k), generator=gen)).to(torch.bfloat16)
    for size in (2.0 ** 127 / k, 2.0 ** 126, 2.0 ** 100):
        _check((x * (size ** 0.5)).to(torch.bfloat16), None, 3.3e38)
        _check((x * (size ** 0.5)).to(torch.bfloat16), (x * (size ** 0.5) / 4).to(torch.bfloat16), 3.4e38)
