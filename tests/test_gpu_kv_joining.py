"""Rows of the paged cache that attention cuts into many parts: more than eight, whose sums are joined in groups, and more than
sixty-four, whose groups are joined in several rounds.  The keys grow along the row, so that every group and every round has
a maximum of its own and a factor that is taken from another part's shows in the result."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import test_gpu_kv_attention as plain  # noqa: E402
from kv_plain import Paged  # noqa: E402

ROOM = 1 << 21                                                        # tokens of a table that asks for two tiles of queries


def growing(lens, heads, page, dim, seed):
    """Keys twice as large from the middle of each row on, and again in its last ninth."""
    p = Paged(lens, heads, page, dim, seed=seed)
    for b, n in enumerate(lens):
        at = np.arange(n)
        step = (at >= n // 2).astype(np.uint8) + (at >= n - n // 9)
        p.ks[p.table[b, at // page], :, at % page] += step[:, None, None].astype(np.uint8)
        p.k[b] = p.k[b] * 2.0 ** step[:, None, None]
    return p


@pytest.fixture(params=[False, True], ids=["narrow", "wide"])
def wide(request, monkeypatch):
    batch = Paged.batch

    def padded(self, device):
        table, lens = batch(self, device)
        return torch.nn.functional.pad(table, (0, ROOM // self.page - table.shape[1]), value=-1), lens

    if request.param:
        monkeypatch.setattr(Paged, "batch", padded)


# tokens / 128 units in parts of at least four: 12000 gives 24 parts (three groups), 45000 88 (eleven groups, two rounds), 100000 196
# (twenty-five, four rounds); with other rows beside it a row has shorter or longer parts
@pytest.mark.parametrize("lens,heads,page,dim,group,news", [
    ([12000], 1, 64, 128, 8, [1]),
    ([12000, 700, 9000], 1, 32, 64, 8, [3, 3, 2]),
    ([45000], 1, 64, 128, 4, [1]),
    ([45000], 1, 64, 128, 8, [4]),
    ([41000], 1, 1024, 32, 3, [9]),
    ([41000], 1, 128, 256, 2, [1]),
    ([41000], 1, 128, 192, 2, [5]),
    ([100000], 1, 128, 64, 4, [6]),
    ([100000, 50], 1, 64, 64, 8, [1, 1]),
])
def test_joining(wide, lens, heads, page, dim, group, news):
    p = growing(lens, heads, page, dim, seed=dim + len(lens))
    scale = 0.2 * dim ** -0.5
    plain.check(p, news, heads * group, scale=scale, what="%r dim %d" % (lens, dim))
    first = plain.run(p, news, heads * group, scale=scale)
    for _ in range(3):
        again = plain.run(p, news, heads * group, scale=scale)
        assert torch.equal(again[0].view(torch.int16), first[0].view(torch.int16)) and torch.equal(again[1], first[1])
