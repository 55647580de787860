"""The copy that growing makes of a begun page that others hold too: codes and scales of keys and values, of every head and layer,
as far as tokens lie in it; nothing else changes."""
import numpy as np
import pytest
import torch

from paper_2503_13565_amd import binding

pytestmark = pytest.mark.gpu

from helpers import DEV  # noqa: E402


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("layers", [None, 3])
@pytest.mark.parametrize("heads,page,dim", [(3, 32, 96), (2, 64, 128), (2, 128, 32), (3, 128, 96), (1, 1024, 64), (2, 16, 256), (5, 64, 192)])
def test_begun_pages_are_copied_whole(layers, heads, page, dim):
    rng = np.random.RandomState(page + dim)
    # a row for each number of tokens in the begun page, and what it grows by
    begun = sorted({1, 15, 16, 17, 31, page // 2, page // 2 + 1, page - 1} - {page})
    begun = [n for n in begun if n < page]
    rows, width = 3 * len(begun), 4
    pages = rows * width
    cache = binding.mxfp4_kv_cache(pages, heads, page, dim, layers=layers, device=DEV)
    for x in cache:
        x.copy_(torch.from_numpy(rng.randint(0, 256, tuple(x.shape)).astype(np.uint8)))
    whole = cache if layers is None else binding.mxfp4_kv_all_layers(cache)
    pool = binding.mxfp4_kv_pool(pages, DEV)
    table, lens = torch.full((rows, width), -1, dtype=torch.int32, device=DEV), torch.zeros(rows, dtype=torch.int32, device=DEV)
    state = (pool, whole, table, lens)
    first = list(range(len(begun)))
    assert int(binding.mxfp4_kv_extend(*state, ints(first), ints([page + n for n in begun]))) == 0
    forks = list(range(len(begun), rows))
    binding.mxfp4_kv_fork(*state, ints(first * 2), ints(forks))
    before = [x.clone() for x in whole]
    held = table.clone()
    grown = [1 + i % (page + 3) for i in range(len(forks))]
    assert int(binding.mxfp4_kv_extend(*state, ints(forks), ints(grown))) == 0
    want = [x.clone() for x in before]
    copied = 0
    for r in forks:
        n = begun[(r - len(begun)) % len(begun)]
        old, new = int(held[r, 1]), int(table[r, 1])
        assert int(table[r, 0]) == int(held[r, 0]) and new != old     # (the row that it was forked from keeps the page)
        copied += 1
        for x, got, was in zip(want, whole, before):
            assert torch.equal(got[new, :, :n], was[old, :, :n]), (r, n)
            upto = min(page, -(-n // 16) * 16)                        # whole sixteens of tokens are copied
            x[new, :, n:upto] = got[new, :, n:upto]
            x[new, :, :n] = was[old, :, :n]
    for x, got in zip(want, whole):
        assert torch.equal(x, got)
    assert copied == 2 * len(begun)
    for x, y in zip(whole, cache):                                    # (the layers' arrays are what was written)
        assert x.data_ptr() == y.data_ptr()


def test_the_last_holder_keeps_its_page():
    pages, page = 12, 32
    cache, pool = binding.mxfp4_kv_cache(pages, 2, page, 64, device=DEV), binding.mxfp4_kv_pool(pages, DEV)
    for x in cache:
        x.copy_(torch.randint(0, 256, tuple(x.shape), generator=torch.Generator().manual_seed(0)).to(torch.uint8))
    table, lens = torch.full((3, 3), -1, dtype=torch.int32, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV)
    state = (pool, cache, table, lens)
    assert int(binding.mxfp4_kv_extend(*state, ints([0]), ints([20]))) == 0
    binding.mxfp4_kv_fork(*state, ints([0, 0]), ints([1, 2]))
    before = [x.clone() for x in cache]
    assert int(binding.mxfp4_kv_extend(*state, ints([2, 0, 1]), ints([1, 1, 1]))) == 0
    assert table[:, 0].tolist() == [2, 0, 1] and pool.refs.tolist() == [1, 1, 1] + [0] * 9
    for x, y in zip(cache, before):
        assert torch.equal(x[1, :, :20], y[0, :, :20]) and torch.equal(x[2, :, :20], y[0, :, :20]) and torch.equal(x[0], y[0])
        assert torch.equal(x[3:], y[3:]) and torch.equal(x[1:3, :, 32:], y[1:3, :, 32:])
