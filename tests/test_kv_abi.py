"""Refusals of the paged cache's entry points, before any GPU work: error codes and texts, never an abort."""
import ctypes

import pytest
import torch

from paper_2503_13565_amd import binding
from paper_2503_13565_amd.binding import KvAttentionArgs, KvCacheDesc, KvPoolDesc, KvRopeDesc, KvRowsDesc, KvTensorDesc

P = 4096                                          # an address that is aligned and never read
NULL, SHAPE, ALIGN, WORKSPACE, ARG = 1, 2, 3, 4, 6


def cache(**more):
    d = dict(kq=P, ks=P, vq=P, vs=P, pages=10, page_stride_q=2 * 16 * 64, page_stride_s=2 * 16 * 4, heads=2, page=16, dim=128, reserved=0)
    return KvCacheDesc(**{**d, **more})


def batch(**more):
    return KvRowsDesc(**{**dict(table=P, ldt=4, width=4, lens=P, starts=None, rows=3, tokens=6), **more})


def tensor(**more):
    return KvTensorDesc(**{**dict(data=P, token=256, head=128), **more})


def pool(**more):
    return KvPoolDesc(**{**dict(refs=P, free_bits=P, pages=10, page=16, table=P, ldt=4, width=4, rows=3, lens=P), **more})


CACHES = [
    (dict(kq=None), NULL), (dict(vs=None), NULL), (dict(page=8), SHAPE), (dict(page=48), SHAPE), (dict(page=2048), SHAPE), (dict(dim=160), SHAPE),
    (dict(dim=0), SHAPE), (dict(heads=0), SHAPE), (dict(heads=70000), SHAPE), (dict(pages=0), SHAPE), (dict(pages=1 << 31), SHAPE),
    (dict(page_stride_q=2 * 16 * 64 - 16), SHAPE), (dict(page_stride_s=112), SHAPE), (dict(page_stride_q=2 * 16 * 64 + 8), ALIGN),
    (dict(ks=P + 4), ALIGN),
]
BATCHES = [
    (dict(table=None), NULL), (dict(lens=None), NULL), (dict(tokens=7), SHAPE), (dict(rows=0), SHAPE), (dict(rows=-1), SHAPE),
    (dict(tokens=-1), SHAPE), (dict(width=0), SHAPE), (dict(ldt=3), SHAPE), (dict(width=1 << 27, ldt=1 << 27), SHAPE), (dict(lens=P + 2), ALIGN),
    (dict(table=P + 1), ALIGN), (dict(starts=P + 1), ALIGN),
]
TENSORS = [(dict(data=None), NULL), (dict(data=P + 8), ALIGN), (dict(token=260), ALIGN), (dict(head=4), ALIGN), (dict(token=-256), SHAPE)]


def append(c, b, k, v, q=None, qo=None, heads=0, rope=None):
    return binding.load().mxfp4_kv_append(c, b, k, v, q, qo, heads, rope, None)


def attend(c, b, ws=P, size=1 << 40, **more):
    args = KvAttentionArgs(**{**dict(q=tensor(), out=tensor(), lse_f32=None, tree=None, q_heads=4, window=0, scale=0.1, causal=1), **more})
    return binding.load().mxfp4_kv_attention(c, b, args, ws, size, None)


@pytest.mark.parametrize("bad,code", CACHES)
def test_caches(bad, code):
    lib, c = binding.load(), cache(**bad)
    assert append(c, batch(), tensor(), tensor()) == code and lib.mxfp4_last_error()
    assert lib.mxfp4_kv_read(c, batch(), tensor(), tensor(), None) == code
    assert attend(c, batch()) == code
    assert lib.mxfp4_kv_copy_pages(c, P, P, 1, None) == code
    assert lib.mxfp4_kv_compact(c, P, 4, 4, P, P, 4, P, 3, None) == code
    assert lib.mxfp4_kv_extend(pool(), c, P, P, 1, P, P, None) == code
    assert lib.mxfp4_kv_attention_workspace_bytes(c, batch(), 4) == 0


@pytest.mark.parametrize("bad,code", BATCHES)
def test_batches(bad, code):
    lib, b = binding.load(), batch(**bad)
    assert append(cache(), b, tensor(), tensor()) == code and lib.mxfp4_last_error()
    assert lib.mxfp4_kv_read(cache(), b, tensor(), tensor(), None) == code
    assert attend(cache(), b) == code


@pytest.mark.parametrize("bad,code", TENSORS)
def test_tensors(bad, code):
    lib, t = binding.load(), tensor(**bad)
    for args in ((t, tensor()), (tensor(), t), (tensor(), tensor(), t, tensor(data=2 * P), 4), (tensor(), tensor(), tensor(data=2 * P), t, 4)):
        assert append(cache(), batch(), *args) == code
    assert lib.mxfp4_kv_read(cache(), batch(), t, tensor(), None) == code
    assert lib.mxfp4_kv_read(cache(), batch(), None, t, None) == code
    assert attend(cache(), batch(), q=t) == code and attend(cache(), batch(), out=t) == code


@pytest.mark.parametrize("bad,code", [
    (dict(cos_f32=None), NULL), (dict(sin_f32=P + 4), ALIGN), (dict(positions=P + 1), ALIGN), (dict(dim=24), SHAPE), (dict(dim=144), SHAPE),
    (dict(dim=-16), SHAPE), (dict(length=0), SHAPE), (dict(length=1 << 31), SHAPE)])
def test_ropes(bad, code):
    rope = KvRopeDesc(**{**dict(cos_f32=P, sin_f32=P, positions=None, length=5, dim=64), **bad})
    assert append(cache(), batch(), tensor(), tensor(), rope=rope) == code


def test_queries_of_an_append():
    assert append(cache(), batch(), tensor(), tensor(), tensor(), tensor(), 4) == ARG              # in place
    assert append(cache(), batch(), tensor(), tensor(), tensor(), tensor(data=2 * P), 0) == SHAPE
    assert append(cache(), batch(), tensor(), tensor(), tensor(), None, 4) == NULL


@pytest.mark.parametrize("bad,code", [
    (dict(q_heads=3), SHAPE), (dict(q_heads=0), SHAPE), (dict(q_heads=1 << 20), SHAPE), (dict(window=-1), SHAPE), (dict(scale=0.0), ARG),
    (dict(scale=float("nan")), ARG), (dict(scale=float("inf")), ARG), (dict(tree=P + 4), ALIGN), (dict(lse_f32=P + 2), ALIGN)])
def test_attention_arguments(bad, code):
    assert attend(cache(), batch(), **bad) == code and binding.load().mxfp4_last_error()


def test_pools_and_lists():
    lib = binding.load()
    for bad, code in ((dict(refs=None), NULL), (dict(free_bits=None), NULL), (dict(lens=None), NULL), (dict(table=None), NULL), (dict(page=12), SHAPE),
                      (dict(pages=0), SHAPE), (dict(rows=0), SHAPE), (dict(ldt=1), SHAPE), (dict(refs=P + 2), ALIGN)):
        p = pool(**bad)
        assert lib.mxfp4_kv_fork(p, P, P, 1, None) == code and lib.mxfp4_kv_release(p, P, P, 1, None) == code
        assert lib.mxfp4_kv_extend(p, None, P, P, 1, P, P, None) == code
    assert lib.mxfp4_kv_fork(pool(), None, P, 1, None) == NULL and lib.mxfp4_kv_fork(pool(), P, P + 1, 1, None) == ALIGN
    assert lib.mxfp4_kv_fork(pool(), P, P, -1, None) == SHAPE and lib.mxfp4_kv_fork(pool(), None, None, 0, None) == 0
    assert lib.mxfp4_kv_release(pool(), P, None, 1, None) == NULL and lib.mxfp4_kv_release(pool(), None, None, 0, None) == 0
    assert lib.mxfp4_kv_extend(pool(), None, P, P, 5000, P, P, None) == SHAPE
    assert lib.mxfp4_kv_extend(pool(), None, P, P, 1, None, P, None) == NULL
    assert lib.mxfp4_kv_extend(pool(pages=11), cache(), P, P, 1, P, P, None) == SHAPE
    assert lib.mxfp4_kv_copy_pages(cache(), None, P, 1, None) == NULL and lib.mxfp4_kv_copy_pages(cache(), None, None, 0, None) == 0
    assert lib.mxfp4_kv_copy_pages(cache(), P, P, -1, None) == SHAPE
    assert lib.mxfp4_kv_compact(cache(), P, 4, 4, None, P, 4, P, 3, None) == NULL
    assert lib.mxfp4_kv_compact(cache(), P, 4, 4, P, P, 4, P, 0, None) == 0


def test_nothing_to_do_is_no_error():
    lib = binding.load()
    none = batch(tokens=0, rows=0, table=None, lens=None)
    assert append(cache(), none, None, None) == 0 and attend(cache(), none) == 0
    assert lib.mxfp4_kv_read(cache(), none, None, None, None) == 0
    assert lib.mxfp4_kv_read(cache(), batch(), None, None, None) == NULL


def test_descriptors_are_those_of_the_header():
    # sizes as a C compiler lays the header's structs out: pointers and 64-bit numbers first, pairs of 32-bit ones last
    sizes = {KvCacheDesc: 72, KvRowsDesc: 56, KvRopeDesc: 40, KvTensorDesc: 24, KvAttentionArgs: 88, KvPoolDesc: 72}
    for d, n in sizes.items():
        assert ctypes.sizeof(d) == n, d


def test_the_binding_refuses_tensors_that_are_not_on_the_gpu():
    c = binding.mxfp4_kv_cache(4, 1, 16, 32, device="cpu")
    t, n = torch.zeros((1, 2), dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    x = torch.zeros((1, 1, 32), dtype=torch.bfloat16)
    for call in (lambda: binding.mxfp4_kv_append(c, x, x, t, n), lambda: binding.mxfp4_kv_read(c, t, n, 1),
                 lambda: binding.mxfp4_kv_attention(x, c, t, n), lambda: binding.mxfp4_kv_copy_pages(c, n, n),
                 lambda: binding.mxfp4_kv_fork(binding.mxfp4_kv_pool(4, "cpu"), c, t, n, n, n)):
        with pytest.raises(ValueError):
            call()
