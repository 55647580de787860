"""The product of 8-bit rows in its larger blocks (gemm_a8_mid.hip, gemm_a8_block.hip) on the GPU, against the definition in 64 bits (layer_plain.py).  Which
block a call takes follows from its sizes and the device's units; the sizes here are for 256 of them."""
import pytest
import torch

import layer_plain as plain
from paper_2503_13565_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _bf16(shape, seed, scale=1.0, large=20.0):
    x = torch.randn(shape, generator=_gen(seed)) * scale
    x[..., 3] *= large
    return x.to(torch.bfloat16).to(DEV)


@pytest.mark.parametrize("m,n,k", [
    (33, 8193, 96), (35, 8195, 32), (193, 8194, 64), (33, 4097, 1376),              # blocks of 32 x 64
    (129, 8193, 160), (65, 12289, 416), (257, 4097, 96),                             # of 64 x 128
    (257, 8193, 96), (258, 8194, 32), (257, 8193, 1376)])                            # of 128 x 128
def test_product_of_a_last_block_of_a_row_and_a_column(m, n, k):
    """Blocks with a row or two, a weight row or two, and a K that is no multiple of an instruction's: less memory than a phase of whole steps."""
    x8, xs = binding.mxfp4_e4m3_direct_cast(_bf16((m, k), 1))
    q, s = binding.mxfp4_direct_cast(_bf16((n, k), 2, 0.05, 4.0))
    y = binding.mxfp4_w4a8_gemm(x8, xs, q, s)
    plain.near(y, *plain.product(x8, xs, q, s, device=DEV))
