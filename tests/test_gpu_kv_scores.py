"""Attention with scores as far from zero as FP32 holds: weights of finite scores are numbers, and where one token's score stands out by more than
the scores' own rounding its value is the result."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import test_gpu_kv_attention as plain  # noqa: E402
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


@pytest.mark.parametrize("scale", [1e3, 1e5, 1e9, 1e15, 1e25, 1e32])
@pytest.mark.parametrize("dim,group", [(32, 3), (64, 2), (96, 4), (128, 2), (192, 2), (256, 1)])
def test_large_scores(wide, dim, group, scale):
    # 2500 tokens of one row are cut into parts, whose maxima differ
    news = [29, 1, 40, 3]
    p = Paged([200, 64, 40, 2500], 1, 32, dim, seed=dim)
    out, lse, q = plain.run(p, news, group, scale=scale)
    got, got_lse, at, clear = out.double().cpu().numpy(), lse.double().cpu().numpy(), 0, 0
    assert np.isfinite(got).all() and np.isfinite(got_lse).all()
    for b, n in enumerate(news):
        qb, sees = q[at: at + n].double().numpy(), p.sees(b, n)
        ref, ref_lse, room, off = attention(qb, p.k[b], p.v[b], sees, scale)
        # a weight's share of error is exp(2 off) - 1, which `tolerance` takes as 2 off: right where off is small
        few = off < 0.05
        tol = tolerance(ref, room, 1.1 * off, p.lens[b])
        assert (np.abs(got[at: at + n] - ref) <= tol)[few].all(), (b, scale)
        assert (np.abs(got_lse[at: at + n] - ref_lse) <= off + (p.lens[b] + 64) * 2.0 ** -24 + (np.abs(ref_lse) + 32) * 2.0 ** -20).all(), (b, scale)
        for i in range(n):
            for h in range(group):
                z = scale * (p.k[b][sees[i], 0] @ qb[i, h])
                order = np.argsort(z)
                if len(z) == 1 or z[order[-1]] - z[order[-2]] > 2 * off[i, h] + 30:    # (e^-30 of the others is below every rounding)
                    v = p.v[b][sees[i], 0][order[-1]]
                    assert (np.abs(got[at + i, h] - v) <= np.abs(v) * 2.0 ** -7 + np.abs(p.v[b]).max() * len(z) * 2.0 ** -40).all(), (b, i, h, scale)
                    clear += 1
        at += n
    assert clear >= 10
