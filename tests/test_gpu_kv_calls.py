"""What a caller of the paged cache may hand in beside the usual: the same answer whichever way a call takes through the binding."""
import numpy as np
import pytest
import torch

from paper_2503_13565_amd import binding

pytestmark = pytest.mark.gpu

from helpers import DEV  # noqa: E402
from kv_plain import Paged, tokens  # noqa: E402


@pytest.mark.parametrize("yes,no", [(True, False), (1, 0), (np.bool_(True), np.bool_(False))])
def test_truth_values_of_attention(yes, no):
    p = Paged([300, 70], 1, 16, 64, seed=1)
    table, lens = p.batch(DEV)
    cache = p.cache(DEV)
    q = tokens(torch.Generator().manual_seed(1), 4, 4, 64).to(DEV)
    want = {c: binding.mxfp4_kv_attention(q, cache, table, lens, causal=c, return_lse=True) for c in (True, False)}
    for _ in range(3):                                                # the first call on a stream takes another way than later ones
        for c, given in ((True, yes), (False, no)):
            got = binding.mxfp4_kv_attention(q, cache, table, lens, causal=given, return_lse=yes)
            assert isinstance(got, tuple) and torch.equal(got[0], want[c][0]) and torch.equal(got[1], want[c][1])
            alone = binding.mxfp4_kv_attention(q, cache, table, lens, causal=given, return_lse=no)
            assert isinstance(alone, torch.Tensor) and torch.equal(alone, want[c][0])


@pytest.mark.parametrize("window", [1 << 20, (1 << 30) - 1, 1 << 30, (1 << 30) + 1, (1 << 31) - 7, (1 << 31) - 1])
@pytest.mark.parametrize("causal", [True, False])
def test_windows_wider_than_any_row(window, causal):
    # more new tokens than cached ones: the first stand at positions below 0, and differences of positions and windows are largest
    p = Paged([3, 0, 40, 1], 1, 16, 64, seed=2)
    table, lens = p.batch(DEV)
    cache = p.cache(DEV)
    starts = torch.tensor([0, 6, 8, 53, 93], dtype=torch.int32, device=DEV)
    q = tokens(torch.Generator().manual_seed(1), 93, 2, 64).to(DEV)
    want = binding.mxfp4_kv_attention(q, cache, table, lens, starts=starts, causal=causal, return_lse=True)
    got = binding.mxfp4_kv_attention(q, cache, table, lens, starts=starts, causal=causal, window=window, return_lse=True)
    assert torch.isfinite(want[1]).any()
    for x, y in zip(got, want):
        assert torch.equal(x, y)
