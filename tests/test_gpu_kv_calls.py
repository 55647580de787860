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


def test_growing_by_more_pages_than_32_bits_count():
    # 66 rows of up to 2^26 pages each (the table's memory is asked for and never written)
    width, rows, pages = 1 << 26, 66, 100
    pool, cache = binding.mxfp4_kv_pool(pages, DEV), binding.mxfp4_kv_cache(pages, 1, 16, 32, device=DEV)
    table, lens = torch.empty((rows, width), dtype=torch.int32, device=DEV), torch.zeros(rows, dtype=torch.int32, device=DEV)
    free = pool.free.clone()
    full = 16 * width
    for adds, want in (([full] * 31, 31 * width), ([full] * 32, 32 * width), ([full] * 33, 33 * width), ([full] * 64, 64 * width),
                       ([full] * 64 + [40], 64 * width + 3), ([40] + [full] * 64, 64 * width + 3), ([full] * 66, 66 * width),
                       ([full] * 1500, 1500 * width)):                # (rows that are listed again: nothing is changed all the same)
        some = torch.arange(len(adds), dtype=torch.int32, device=DEV) % rows
        missing = binding.mxfp4_kv_extend(pool, cache, table, lens, some, torch.tensor(adds, dtype=torch.int32, device=DEV))
        assert int(missing) == min(want, 2 ** 31 - 1) - pages, (len(adds), int(missing))
        assert not lens.any() and not pool.refs.any() and torch.equal(pool.free, free), len(adds)
    some, add = torch.tensor([3, 65], dtype=torch.int32, device=DEV), torch.tensor([16 * 60, 16 * 40], dtype=torch.int32, device=DEV)
    assert int(binding.mxfp4_kv_extend(pool, cache, table, lens, some, add)) == 0
    assert table[3, :60].tolist() == list(range(60)) and table[65, :40].tolist() == list(range(60, 100))


@pytest.mark.parametrize("group", [8, 24])                            # (one tile of queries, and two)
def test_descending_starts_leave_the_counters_at_zero(group):
    # every other row's starts go back to 0: their tokens together are 256 times those of the batch, and the one long row, which would
    # be cut, stands where the launch's workgroups end
    rows, page, heads, long = 512, 64, 4, 20000
    width = long // page + 1
    cache = binding.mxfp4_kv_cache(width, heads, page, 64, device=DEV)
    for x, byte in zip(cache, (0x21, 127, 0x32, 127)):
        x.fill_(byte)
    table = torch.arange(width, dtype=torch.int32, device=DEV).repeat(rows, 1)
    q = tokens(torch.Generator().manual_seed(1), 8, group * heads, 64).to(DEV)
    need = max(binding.mxfp4_kv_attention_workspace_bytes(cache, r, 8, group * heads) for r in (rows, 1))
    ws = torch.zeros(need, dtype=torch.uint8, device=DEV)
    flat = [0, 8] * (rows // 2) + [8]
    for at in range(2, rows, 37):
        lens = torch.full((rows,), 100, dtype=torch.int32, device=DEV)
        lens[at & ~1] = long
        binding.mxfp4_kv_attention(q, cache, table, lens, starts=torch.tensor(flat, dtype=torch.int32, device=DEV), workspace=ws)
        assert not ws[: 4 * binding.KV_COUNTERS].any(), at
    one = torch.tensor([long], dtype=torch.int32, device=DEV)
    want = binding.mxfp4_kv_attention(q, cache, table[:1], one)
    assert torch.equal(binding.mxfp4_kv_attention(q, cache, table[:1], one, workspace=ws), want)
