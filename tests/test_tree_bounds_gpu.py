"""Acceptance of drafted trees whose sequences have more rows than the batch's bound says: the lengths."""

import pytest
import torch

import paper_2609_31568_gb300 as pkg
from paper_2609_31568_gb300 import scale as S

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    pkg.build()
    S.load()


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def test_lengths_where_no_row_is_looked_at():
    """A bound of 0, and rows behind the tensors' end: nothing is accepted, and the drafted tokens do not count."""
    for starts, lens, n_rows, most in (([0, 5, 5, 9, 12], [20, 7, 3, 12], 12, 0), ([0, 4, 9], [30, 40], 4, 8), ([4, 6, 9], [30, 2], 4, 8)):
        seqs = len(lens)
        cache = S.allocate_kv_cache(8, 16, 1)
        batch = S.kv_batch(ints(starts), ints(lens), ints([[0] * 4] * seqs), n_rows, most)
        lists = [ints([-5] * n_rows) for _ in range(3)]
        out = [ints([-77] * seqs) for _ in range(3)]
        zeros = ints([0] * n_rows)
        tree = S.draft_tree(ints([-1] * n_rows), zeros, ints([[0]] * n_rows))
        moves = S.cache_moves(lists[0], lists[1], batch.tensors[0])
        S.scale_tree_accept(tree, S.cache_layers([cache]), batch, zeros + 6, zeros, ints([7] * seqs), out[0], lists[2], out[1], out[2], moves)
        rows = [y - x for x, y in zip(starts, starts[1:])]
        assert out[0].tolist() == [0] * seqs and out[1].tolist() == [7] * seqs
        assert out[2].tolist() == [n - a if n >= a else n for a, n in zip(rows, lens)], (starts, lens)
