"""Calls of the paged cache that are wider than one launch: 2^24 workgroups of 256 threads are all that a launch's x holds."""
import pytest
import torch

from paper_2503_13565_amd import binding

pytestmark = pytest.mark.gpu

from helpers import DEV  # noqa: E402

MANY = (1 << 24) + 1000


def test_append_and_read_of_more_tokens_than_workgroups():
    page, heads, dim = 1024, 1, 32
    pages = MANY // page + 1
    cache = binding.mxfp4_kv_cache(pages, heads, page, dim, device=DEV)
    table = torch.arange(pages, dtype=torch.int32, device=DEV).flip(0).view(1, pages).contiguous()
    lens = torch.tensor([MANY], dtype=torch.int32, device=DEV)
    gen = torch.Generator(device=DEV).manual_seed(0)
    # values of the format's grid: what is read back is what was stored, up to the sign of zero
    grid = torch.tensor([0.5, 1, 1.5, 2, 3, 4, 6, -0.5, -1, -1.5, -2, -3, -4, -6], device=DEV).to(torch.bfloat16)
    k = grid[torch.randint(14, (MANY, heads, dim), generator=gen, device=DEV)]
    v = grid[torch.randint(14, (MANY, heads, dim), generator=gen, device=DEV)]
    k[..., 0] = v[..., 0] = 6.0                                       # (every block's scale is 1)
    q = binding.mxfp4_kv_append(cache, k, v, table, lens, q=k)
    assert torch.equal(q, k)
    rk, rv = binding.mxfp4_kv_read(cache, table, lens, MANY)
    assert torch.equal(rk, k) and torch.equal(rv, v)


def test_copies_of_more_pages_than_workgroups():
    pages = 2 * MANY
    cache = binding.mxfp4_kv_cache(pages, 1, 16, 32, device=DEV)
    gen = torch.Generator(device=DEV).manual_seed(0)
    for x in cache:
        x[:MANY].random_(0, 256, generator=gen)
    src = torch.arange(MANY, dtype=torch.int32, device=DEV)
    binding.mxfp4_kv_copy_pages(cache, src, src.flip(0) + MANY)
    for x in cache:
        assert torch.equal(x[MANY:], x[:MANY].flip(0))


def test_attention_of_more_shares_than_workgroups():
    # 300 sequences that share one page of 65535 heads, one token each: every one has the result of the first
    rows, heads, dim, page = 300, 65535, 32, 16
    cache = binding.mxfp4_kv_cache(1, heads, page, dim, device=DEV)
    gen = torch.Generator(device=DEV).manual_seed(0)
    for x, low, high in zip(cache, (0, 126, 0, 126), (256, 129, 256, 129)):
        x.random_(low, high, generator=gen)
    table = torch.zeros((rows, 1), dtype=torch.int32, device=DEV)
    lens = torch.full((rows,), page, dtype=torch.int32, device=DEV)
    q = torch.randn((1, heads, dim), generator=gen, device=DEV).to(torch.bfloat16).expand(rows, heads, dim)
    out = binding.mxfp4_kv_attention(q, cache, table, lens)
    k, v = binding.mxfp4_kv_read(cache, table[:1], lens[:1], page)
    scores = torch.einsum("hd,jhd->hj", q[0].double(), k.double()) * dim ** -0.5
    want = torch.einsum("hj,jhd->hd", scores.softmax(-1), v.double())
    room = torch.einsum("hj,jhd->hd", scores.softmax(-1), v.double().abs())
    # a weight's rounding to BF16 (half a step, 2^-8), scores and sums in FP32 (2^-16 is more than they take), the result's rounding
    assert ((out[0].double() - want).abs() <= room * (2.0 ** -8 + 2.0 ** -16) + (want.abs() + room * 2.0 ** -8) * 2.0 ** -8).all()
    for r in range(rows):
        assert torch.equal(out[r], out[0]), r
