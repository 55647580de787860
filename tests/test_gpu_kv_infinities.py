"""Attention over cached values that are no numbers: NaN blocks and infinities, which codes of 2 and more under scale byte 254 and of
4 and more under 253 are in BF16 (no cast gives such bytes; a cache may be filled otherwise).  Who sees one gets it, in that element
alone; who does not gets the bits of a cache with zeros in its place."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import test_gpu_kv_attention as plain  # noqa: E402
from helpers import DEV  # noqa: E402
from kv_plain import Paged, attention, tolerance  # noqa: E402

ROOM = 1 << 21                                                        # tokens of a table that asks for two tiles of queries


@pytest.fixture(params=[False, True], ids=["narrow", "wide"])
def wide(request, monkeypatch):
    batch = Paged.batch

    def padded(self, device):
        table, lens = batch(self, device)
        return torch.nn.functional.pad(table, (0, ROOM // self.page - table.shape[1]), value=-1), lens

    if request.param:
        monkeypatch.setattr(Paged, "batch", padded)


def spoil(p, b, at, head, block, byte, rng):
    """A value block of infinities of both signs and zeros (byte 255: of NaN) in the place of a token's."""
    page, slot = p.table[b, at // p.page], at % p.page
    odd = np.array({255: range(16), 254: [4, 5, 6, 7, 12, 13, 14, 15], 253: [6, 7, 14, 15]}[byte])
    codes = np.where(rng.rand(32) < 0.4, odd[rng.randint(len(odd), size=32)], 0).astype(np.uint8)
    p.vs[page, head, slot, block] = byte
    p.vq[page, head, slot, 16 * block: 16 * block + 16] = codes[0::2] | codes[1::2] << 4
    v = np.where(codes == 0, 0.0, np.where(codes >= 8, -np.inf, np.inf)) if byte < 255 else np.full(32, np.nan)
    p.v[b][at, head, 32 * block: 32 * block + 32] = v


def zero(p, b, at, head, block):
    page, slot = p.table[b, at // p.page], at % p.page
    p.vs[page, head, slot, block] = 127
    p.vq[page, head, slot, 16 * block: 16 * block + 16] = 0


@pytest.mark.parametrize("causal,window,tree", [(True, 0, False), (True, 20, False), (False, 37, False), (False, 0, True), (False, 0, False)])
@pytest.mark.parametrize("dim,group", [(32, 3), (64, 2), (96, 4), (128, 2), (192, 2), (256, 1)])
def test_who_sees_them_and_who_does_not(wide, dim, group, causal, window, tree):
    news, lens = [29, 1, 20], [200, 64, 20]
    rng = np.random.RandomState(dim + window)
    made = [Paged(lens, 2, 32, dim, seed=dim) for _ in range(2)]
    p, clean = made
    for b, at, head, block, byte in ((0, 180, 0, 0, 254), (0, 181, 0, 0, 253), (0, 195, 1, dim // 32 - 1, 253), (0, 199, 1, 0, 255),
                                     (0, 190, 1, 0, 254), (0, 100, 0, dim // 32 - 1, 254), (0, 5, 1, 0, 253), (2, 0, 0, 0, 254),
                                     (2, 19, 1, dim // 32 - 1, 254), (1, 63, 0, 0, 253)):
        spoil(p, b, at, head, block, byte, rng)
        zero(clean, b, at, head, block)
    trees = [[int(rng.randint(1 << 20)) | 1 << i for i in range(n)] for n in news] if tree else None
    out, lse, q = plain.run(p, news, 2 * group, causal=causal, window=window, trees=trees)
    like, like_lse, _ = plain.run(clean, news, 2 * group, causal=causal, window=window, trees=trees)
    assert torch.equal(lse, like_lse)                                 # (the keys are numbers)
    got, same, first = out.double().cpu().numpy(), (out.view(torch.int16) == like.view(torch.int16)).cpu().numpy(), 0
    kinds = set()
    for b, n in enumerate(news):
        sees = p.sees(b, n, causal, window, trees and trees[b])
        with np.errstate(invalid="ignore"):
            # (an infinity times a weight is one, whatever the weight; zeros of the unseen times them do not come into it)
            ref, _, room, off = attention(q[first: first + n].double().numpy(), p.k[b], p.v[b], sees, dim ** -0.5)
            tol = tolerance(ref, room, off, p.lens[b])
        mine, finite = got[first: first + n], np.isfinite(ref)
        assert np.array_equal(np.isnan(mine), np.isnan(ref)) and np.array_equal(np.isinf(mine), np.isinf(ref)), b
        assert np.array_equal(mine[np.isinf(ref)], ref[np.isinf(ref)])
        assert (np.abs(mine[finite] - ref[finite]) <= tol[finite]).all()
        assert same[first: first + n][finite].all()
        kinds |= {k for k, some in (("nan", np.isnan(ref)), ("inf", np.isinf(ref)), ("finite", finite)) if some.any()}
        first += n
    assert kinds == {"nan", "inf", "finite"}
