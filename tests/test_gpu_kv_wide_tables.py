"""Attention where the table leaves room for long sequences, so that a workgroup takes two tiles of queries: the cases of
test_gpu_kv_attention.py with more queries than one tile holds, once more with wide tables."""
import pytest
import torch

pytestmark = pytest.mark.gpu

import test_gpu_kv_attention as narrow  # noqa: E402
from kv_plain import Paged  # noqa: E402

ROOM = 1 << 21                                                        # tokens that a table row has room for


@pytest.fixture(autouse=True)
def wide(monkeypatch):
    batch = Paged.batch

    def padded(self, device):
        table, lens = batch(self, device)
        return torch.nn.functional.pad(table, (0, ROOM // self.page - table.shape[1]), value=-1), lens

    monkeypatch.setattr(Paged, "batch", padded)


@pytest.mark.parametrize("news", [[130, 1, 77, 257], [64, 100, 129, 3]])
@pytest.mark.parametrize("dim,group", [(32, 3), (64, 2), (96, 3), (128, 1), (128, 4)])
def test_pieces_of_prompts(dim, group, news):
    narrow.test_pieces_of_prompts(dim, group, news)


@pytest.mark.parametrize("window", [0, 1, 33, 200])
@pytest.mark.parametrize("dim", [32, 64, 96, 128])
def test_many_queries(dim, window):
    narrow.test_many_queries(dim, window)


@pytest.mark.parametrize("dim,group,nodes", [(128, 8, 8), (128, 1, 64), (64, 4, 17), (96, 2, 33)])
def test_draft_trees(dim, group, nodes):
    narrow.test_draft_trees(dim, group, nodes)


@pytest.mark.parametrize("page", [16, 1024])
def test_many_queries_over_long_rows_are_joined(page):
    narrow.test_many_queries_over_long_rows_are_joined(page)


@pytest.mark.parametrize("dim", [64, 128])
def test_nan_blocks(dim):
    narrow.test_many_queries_and_nan_blocks(dim)


def test_trees_windows_missing_pages_and_other_lengths():
    narrow.test_many_queries_in_trees()
    narrow.test_many_queries_more_than_tokens_and_missing_pages()
    narrow.test_all_tokens_see_all()
    narrow.test_nodes_past_the_words_are_not_seen()


@pytest.mark.parametrize("window", [1, 17, 100])
@pytest.mark.parametrize("dim", [64, 128])
def test_windows_of_many_heads(dim, window):
    p = Paged([200, 90, 40, 33], 70, 16, dim, seed=window)
    narrow.check(p, [40, 3, 40, 1], 140, window=window, what="dim %d window %d" % (dim, window))
