"""A cache with layers as one cache: the same memory, or an error; on the CPU."""
import pytest
import torch

from paper_2503_13565_amd import binding


def make(layers=3, heads=4):
    return binding.mxfp4_kv_cache(5, heads, 16, 64, layers=layers, device="cpu")


def test_all_layers_are_the_same_memory():
    cache = make()
    for part in (cache, binding.KvCache(*(x[:, 1:] for x in cache)), binding.KvCache(*(x[2:] for x in cache)), make(1), make(3, 1)):
        whole = binding.mxfp4_kv_all_layers(part)
        for x, y in zip(whole, part):
            assert x.shape == (y.shape[0], y.shape[1] * y.shape[2], *y.shape[3:]) and x.data_ptr() == y.data_ptr()
            x[-1, -1] = 7
            assert (y[-1, -1, -1] == 7).all()


@pytest.mark.parametrize("part", [lambda x: x[:, :, :2], lambda x: x[:, :, 1:], lambda x: x.transpose(1, 2), lambda x: x[:, 0]])
def test_what_would_be_a_copy_is_refused(part):
    with pytest.raises(ValueError):
        binding.mxfp4_kv_all_layers(binding.KvCache(*(part(x) for x in make())))


def test_a_cache_on_another_device_than_its_pool_is_refused():
    pool, cache = binding.mxfp4_kv_pool(4, "cpu"), binding.mxfp4_kv_cache(4, 1, 16, 32, device="meta")
    t, n = torch.zeros((1, 2), dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="the cache must be on the pool's device cpu"):
        binding.mxfp4_kv_extend(pool, cache, t, n, n, n)
